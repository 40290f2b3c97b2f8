// Log probabilities of classes and distillation from a teacher's largest logits (include/maxk.h), over rows of logits of any width.
//
//   m = max x,  d = (x - m) scale log2 e,  S = sum 2^d,  T = sum 2^d d:   log p = ln 2 d - ln S,   H = ln S - ln 2 T / S
//   log probabilities:  dx = p (-g - u (log p + H)), + g at the given class
//   distillation:       q = softmax(scale t) of the teacher's entries;  loss = sum q (log q - log p);  dx = g scale (p - sum of q at the column)
//
// Rows of up to 2048 columns lie in the registers of a part of a wavefront or of all of it, of up to 16384 in a workgroup's, and are read once.  One pass over a longer row
// has its maximum and sums: a lane rescales its own when its maximum moves, lanes and wavefronts are joined in the end; the gradient reads the row again, from the caches, and
// writes.  Few long rows are cut into segments, a workgroup each, whose sums a second launch joins.  Many short rows go through LDS, where a lane has one of them.
//
// Bound by memory: gradients from 64 columns on (169343 x 1000 fp32, distillation 251 us, 5.5 TB/s; 4096 x 131072 bf16 456, two reads and one write, 7.0) and, without
// alternatives, forward calls on fp32 and on rows of some 5000 columns and more.  By the vector units: rows that leave lanes idle (40000 x 2500 bf16 forward 64, 39 at one
// read), and alternatives, whose keys are sorted (16000 x 2500 bf16, 5 of them 53 and 50 of them 70, where the read takes 16).  By dependent loads and launches: few
// rows (1 x 131072 with 20 alternatives 12).
#include "heads.hpp"
#include "mx_parts.hpp"
#include "rows.hpp"

namespace maxk {
namespace {

constexpr int kThreads = 256;  // of a workgroup; T below: 256 or 1024
constexpr float kLn2 = 0.69314718055994531f;
constexpr auto kNothing = [] {};
constexpr float kFar = 256.f;  // 2^-256 is 0 in fp32: a difference past it need not be told, and is cut so that 0 times it stays 0

// Of a part of a row: its largest value (the lowest fp32 value where it has none above), S and T.  -Inf adds 0, NaN and +Inf make S a NaN.
struct Sums { float m, S, T; };
constexpr float kLowest = -3.402823466e38f;
__device__ __forceinline__ Sums no_sums() { return {kLowest, 0.f, 0.f}; }

__device__ __forceinline__ float exp2_of(float d) { return __builtin_amdgcn_exp2f(d); }

__device__ __forceinline__ void move_to(Sums& a, float m, float c)  // m at least a.m
{
#pragma clang fp contract(off)
    const float shift = fminf((m - a.m) * c, kFar), f = exp2_of(-shift);
    a.T = f * fmaf(-shift, a.S, a.T);
    a.S *= f;
    a.m = m;
}

__device__ __forceinline__ float largest(const float (&x)[kRowUnit])
{
    float m = fmaxf(x[0], x[1]);
#pragma unroll
    for (int j = 2; j < kRowUnit; ++j) m = fmaxf(m, x[j]);
    return m;
}

// A lane's sums on its way along a long row.  d = x c - q is one operation with q = m c rounded; what the rounding leaves, delta = q - m c, is made good in the
// end: (x - m) c = d + delta.  delta is up to half a step of q, of which 2^d and 2^delta bear no large ones: rows whose |m c| is 2^23 and more, where that half is more than
// 1/4, are gone through again with d = (x - m) c (CAREFUL).  T is kept for ENTROPY.
// A lane whose own columns are all far below 0 (a mask of a large finite value) has q = -2^24 for theirs, of which 2^d is 0 or little: where the row's maximum is not far
// off, they add nothing to it.
constexpr float kFarOff = 0x1p23f, kFarDown = -0x1p24f;
template <bool CAREFUL, bool ENTROPY>
struct Way {
    Sums a;
    float q;
    __device__ __forceinline__ void begin() { a = no_sums(), q = kFarDown; }
    __device__ __forceinline__ void absorb(const float (&x)[kRowUnit], float top, float c)
    {
        const float m = fmaxf(a.m, top);
        if constexpr (CAREFUL) {
            move_to(a, m, c);
        } else {
            const float to = fmaxf(m * c, kFarDown), shift = fminf(to - q, kFar), f = exp2_of(-shift);
            if constexpr (ENTROPY) a.T = f * fmaf(-shift, a.S, a.T);
            a.S *= f;
            a.m = m;
            q = to;
        }
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) {
            const float d = CAREFUL ? (x[j] - a.m) * c : fmaf(x[j], c, -q), e = exp2_of(d);
            a.S += e;
            if constexpr (ENTROPY) a.T = fmaf(e, fmaxf(d, -kFar), a.T);
        }
    }
    __device__ __forceinline__ Sums end(float c)
    {
        if constexpr (!CAREFUL) {
            // (far up delta is anything: the row comes again.  Far down a NaN stays one)
            const float delta = q > kFarDown ? fmaf(-a.m, c, q) : 0.f, f = q > kFarDown ? exp2_of(delta) : 0.f;
            if constexpr (ENTROPY) a.T = f * fmaf(delta, a.S, a.T);
            a.S *= f;
        }
        return a;
    }
};

// (the same bits whichever comes first, so that all lanes that join each other's have the same: no product may be taken into the addition of one side)
__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
#pragma clang fp contract(off)
    const float m = fmaxf(a.m, b.m);
    move_to(a, m, c);
    move_to(b, m, c);
    return {m, a.S + b.S, a.T + b.T};
}

template <int L>
__device__ __forceinline__ Sums join_lanes(Sums a, float c)
{
    const auto with = [&](auto step) {
        constexpr int K = decltype(step)::value;
        a = join(a, Sums{other_lane<K>(a.m), other_lane<K>(a.S), other_lane<K>(a.T)}, c);
    };
    if constexpr (L > 1) with(std::integral_constant<int, 1>{});
    if constexpr (L > 2) with(std::integral_constant<int, 2>{});
    if constexpr (L > 4) with(std::integral_constant<int, 4>{});
    if constexpr (L > 8) with(std::integral_constant<int, 8>{});
    if constexpr (L > 16) with(std::integral_constant<int, 16>{});
    if constexpr (L > 32) with(std::integral_constant<int, 32>{});
    return a;
}

template <int T>
__device__ __forceinline__ Sums join_workgroup(Sums a, float c, Sums* room)  // (passes a barrier, room is free behind the next one)
{
    a = join_lanes<kWave>(a, c);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x / kWave] = a;
    __syncthreads();
    a = join_lanes<T / kWave>(room[threadIdx.x % (T / kWave)], c);
    return a;
}

// ---- the likeliest classes: keys are in the order of (value, lower column first) ----

__device__ __forceinline__ uint32_t value_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);  // -0 is +0
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t col) { return (uint64_t)value_key(x) << 32 | (0xFFFFFFFFu - col); }

__device__ __forceinline__ uint64_t lane_key(uint64_t k, int lane)
{
    return (uint64_t)(uint32_t)__shfl((int)(k >> 32), lane) << 32 | (uint32_t)__shfl((int)(uint32_t)k, lane);
}
__device__ __forceinline__ uint64_t key_of_lane(uint64_t k, int lane)  // (the same lane for all)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}
__device__ __forceinline__ uint64_t greater_key(uint64_t a, uint64_t b) { return a > b ? a : b; }

// of lane ^ STEP
template <int STEP>
__device__ __forceinline__ uint32_t across(uint32_t x)
{
    if constexpr (STEP == 4) x = dpp<0x1B>(dpp<0x141>(x));  // row_half_mirror, quad_perm [3,2,1,0]
    else if constexpr (STEP == 8) x = dpp<0x128>(x);        // row_ror:8
    else x = xor_lane(x, std::integral_constant<int, STEP>{});
    return x;
}
template <int STEP>
__device__ __forceinline__ uint64_t exchange(uint64_t k, int lane)
{
    const uint64_t o = (uint64_t)across<STEP>((uint32_t)(k >> 32)) << 32 | across<STEP>((uint32_t)k);
    return ((lane & STEP) == 0) == (k > o) ? k : o;
}
// runs of 2 STEP lanes whose halves are in opposite orders into falling order
template <int STEP>
__device__ __forceinline__ uint64_t settle(uint64_t k, int lane)
{
    k = exchange<STEP>(k, lane);
    if constexpr (STEP > 1) k = settle<STEP / 2>(k, lane);
    return k;
}
// the 64 greatest of two sets in falling order, in falling order
__device__ __forceinline__ uint64_t merge_keys(uint64_t a, uint64_t b, int lane)
{
    return settle<32>(greater_key(a, lane_key(b, 63 - lane)), lane);
}
constexpr int kWaiting = kWave * (kRowUnit + 1);  // keys of a wavefront that wait to be sorted in: a unit of every lane on top of less than a wavefront's
// of the wavefronts of a workgroup, for the first of them (keys: 64 of each, written)
template <int T, int ROOM>
__device__ __forceinline__ uint64_t merge_waves(uint64_t mine, uint64_t (&keys)[T / kWave][ROOM], int lane, int wave)
{
    for (int step = 1; step < T / kWave; step *= 2) {
        keys[wave][lane] = mine;
        __syncthreads();
        if (wave % (2 * step) == 0) mine = merge_keys(mine, keys[wave + step][lane], lane);
    }
    return mine;
}

// A wavefront's greatest keys: in falling order over the lanes, and those that wait in LDS to be sorted in.  A unit whose largest value is below the k-th
// greatest key costs a comparison.  Classes that are masked out (-Inf) are left out, and come in when a row has fewer than k others (fill): a masked
// stretch of a vocabulary would be all equal keys.
struct Likeliest {
    uint64_t mine, least;   // least: of a key that is still wanted (it is greater)
    float least_value;
    uint64_t* wait;         // kWaiting keys
    int waiting, k, lane;
    bool some;              // mine has any

    __device__ __forceinline__ void begin(int k_, uint64_t* wait_, int lane_)
    {
        mine = least = 0;
        least_value = -__builtin_inff();
        wait = wait_;
        waiting = 0;
        k = k_;
        lane = lane_;
        some = false;
    }
    __device__ __forceinline__ void raise(uint64_t key)
    {
        least = key > least ? key : least;
        const uint32_t high = (uint32_t)(least >> 32);  // (a bound cut short may lie below -Inf's key)
        least_value = high > 0x007FFFFFu ? key_value(high) : -__builtin_inff();
    }
    // Up to 64 of the waiting keys into the order: a key's place is the number of greater ones, which it counts
    __device__ void sort_in()
    {
        wave_fence();
        const int n = min(waiting, kWave), from = waiting - n;
        const uint64_t key = lane < n ? wait[from + lane] : 0;
        int place = 0;
#pragma unroll 4
        for (int i = 0; i < n; ++i) place += key_of_lane(key, i) > key;
        wave_fence();
        if (lane < n) wait[from + place] = key;
        wave_fence();
        const uint64_t sorted = lane < n ? wait[from + lane] : 0;
        waiting = from;
        mine = some ? merge_keys(mine, sorted, lane) : sorted;
        some = true;
        raise(key_of_lane(mine, k - 1));
    }
    // The k-th greatest of the lanes' largest values is no less than the k-th greatest value of all: a first bound, its leading 20 bits, before anything is
    // offered.  (any: the lane has one)
    static __device__ __forceinline__ uint32_t head(float top, bool any) { return any && top > -__builtin_inff() ? value_key(top) : 0u; }
    template <int R>
    __device__ __forceinline__ void expect(const uint32_t (&heads)[R])  // of R wavefronts
    {
        uint32_t bound = 0;
#pragma unroll
        for (uint32_t bit = 1u << 31; bit >= 1u << 12; bit >>= 1) {
            int n = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) n += __popcll(__ballot(heads[r] >= (bound | bit)));
            if (n >= k) bound |= bit;
        }
        raise((uint64_t)bound << 32);
    }
    __device__ __forceinline__ void expect(float top, bool any)
    {
        const uint32_t heads[1] = {head(top, any)};
        expect(heads);
    }
    // a unit at column `col`: all lanes come here, those without columns with valid < 1
    __device__ __forceinline__ void offer(const float (&x)[kRowUnit], float top, int col, int valid)
    {
        if (!__any(valid > 0 && top >= least_value && top > -__builtin_inff())) return;
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) {
            const bool perhaps = j < valid && x[j] >= least_value && x[j] > -__builtin_inff();
            if (!__any(perhaps)) continue;
            const uint64_t key = key_of(x[j], (uint32_t)(col + j));
            const bool wanted = perhaps && key > least;
            const uint64_t who = __ballot(wanted);
            if (wanted) wait[waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key;
            waiting += __popcll(who);
        }
        while (waiting >= kWave) sort_in();
    }
    __device__ __forceinline__ void end() { while (waiting > 0) sort_in(); }
};

// The keys of a row in falling order, filled up to k with its first masked columns where there are fewer.  (room: k keys in LDS of the wavefront.  A row with a NaN,
// whose S is one, has no order, and might be gone through to its end.)
template <int VT>
__device__ __forceinline__ uint64_t fill(uint64_t key, const Sums& s, const value_store_t<VT>* x, int V, int k, int lane, uint64_t* room)
{
    int have = __popcll(__ballot(lane < k && key));
    if (have >= k || s.S != s.S) return key;
    const int found = have;
    for (int base = 0; base < V && have < k; base += kWave) {
        const int col = base + lane;
        const bool masked = col < V && widen_value<VT>(x[col]) == -__builtin_inff();
        const uint64_t who = __ballot(masked);
        const int at = have + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
        if (masked && at < k) room[at] = key_of(-__builtin_inff(), (uint32_t)col);
        have += __popcll(who);
    }
    wave_fence();
    return lane >= found && lane < min(have, k) ? room[lane] : key;
}

// ---- a row ----

// Workgroups in two dimensions: in one the threads of a launch have to be fewer than 2^32
constexpr int64_t kMostGroupsAcross = 1 << 20;
dim3 groups_of(int64_t n) { return dim3((unsigned)std::min(n, kMostGroupsAcross), (unsigned)((n + kMostGroupsAcross - 1) / kMostGroupsAcross)); }
__device__ __forceinline__ int64_t group_number() { return (int64_t)blockIdx.y * kMostGroupsAcross + blockIdx.x; }

// What a row is asked for beside its logits.  (Loads without a branch on what they bring, and before anything waits: a short row's time is these.)
struct Given {
    int64_t y;         // the class, -1: none
    float g, u;        // of the log probability, of the entropy; of the loss
};
__device__ __forceinline__ Given row_given(const ClassCall& C, int64_t row)
{
    Given w = {-1, 0.f, 0.f};
    int32_t low = -1, high = -1;
    if (C.labels) {
        const int32_t* p = (const int32_t*)C.labels + row * (C.label_bytes / 4);
        low = p[0], high = p[C.label_bytes / 4 - 1];
    }
    if (C.dlogprob) w.g = C.dlogprob[row];
    if (C.dloss) w.g = C.dloss[row];
    if (C.dentropy) w.u = C.dentropy[row];
    w.y = C.label_bytes == 8 ? (int64_t)((uint64_t)(uint32_t)high << 32 | (uint32_t)low) : (int64_t)low;
    return w;
}
__device__ __forceinline__ int64_t column_of(const ClassCall& C, int64_t at)
{
    return C.index_bytes == 1 ? ((const uint8_t*)C.index)[at] : C.index_bytes == 2 ? ((const uint16_t*)C.index)[at] : ((const int32_t*)C.index)[at];
}
__device__ __forceinline__ float teacher_value(const ClassCall& C, int64_t at)
{
    if (C.data_type == MAXK_VALUE_F32) return ((const float*)C.data)[at];
    const uint16_t v = ((const uint16_t*)C.data)[at];
    return C.data_type == MAXK_VALUE_BF16 ? widen_value<MAXK_VALUE_BF16>(v) : widen_value<MAXK_VALUE_F16>(v);
}

// What a row asks of its columns beside S: log probabilities: x at the given class (x), whether there is one; distillation: the teacher's part.
// loss = C + Q (ln S + (m - ref) scale) with C = sum q (log q - (x - ref) scale) over the teacher's entries, ref the largest x among them
struct Asked { float x, C, ref, Q; };

constexpr int kMostEntries = MAXK_DISTILL_MAX_K;
struct Entries {  // of the teacher, in LDS
    int32_t col[kMostEntries];
    float q[kMostEntries], x[kMostEntries];
};

constexpr auto kMax = [](float a, float b) { return fmaxf(a, b); };

// The teacher's entries of a row by one wavefront, while the others go through the row: their q and the student's x there.  An entry whose column lies outside the
// row is none.  Of several entries of a column the first one has their sum, in the entries' order; where there are more entries than lanes all threads see to that
// in the end.
constexpr int kFewEntries = kWave;

template <int VT>
struct FewEntries {  // up to one a lane; asked for before the row is gone through, and seen to behind it
    int col;
    float t, v;
    __device__ __forceinline__ void ask(const ClassCall& C, int64_t row, int lane)
    {
        const int64_t at = lane < C.k ? column_of(C, row * C.k + lane) : -1;
        const bool there = at >= 0 && at < C.V;
        col = there ? (int)at : -1;
        t = there ? teacher_value(C, row * C.k + lane) : -__builtin_inff();
        v = there ? widen_value<VT>(((const value_store_t<VT>*)C.logits)[row * C.V + col]) : -__builtin_inff();
    }
    __device__ __forceinline__ Asked take(const ClassCall& C, int lane, bool gradient, Entries& E)
    {
        const float c = C.scale * kLog2e, top = over_lanes<kWave>(fmaxf(t, kLowest), kMax), ref = over_lanes<kWave>(fmaxf(v, kLowest), kMax);
        const float d = (t - top) * c, e = exp2_of(d), sum = over_lanes<kWave>(e, kAdd), inverse = 1.f / sum;
        float q = sum == 0.f ? 0.f : e * inverse;
        const float loss = over_lanes<kWave>(q != 0.f ? q * (fmaf(kLn2, d, -logf(sum)) - (v - ref) * C.scale) : 0.f, kAdd);
        if (gradient) {
            float all = 0.f;
            bool mine = true;
#pragma unroll 4
            for (int j = 0; j < C.k; ++j) {
                const bool same = __builtin_amdgcn_readlane(col, j) == col;
                all += same ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(q), j)) : 0.f;
                mine &= !same || j >= lane;
            }
            q = all;
            if (lane < C.k) E.col[lane] = mine ? col : -1, E.q[lane] = q, E.x[lane] = v;
        }
        return {0.f, loss, ref, sum == 0.f ? 0.f : sum * inverse};
    }
};

template <int VT>
__device__ Asked take_more_entries(const ClassCall& C, int64_t row, int lane, Entries& E)
{
    const value_store_t<VT>* x = (const value_store_t<VT>*)C.logits + row * C.V;
    float top = kLowest, ref = kLowest;
    for (int i = lane; i < C.k; i += kWave) {
        const int64_t col = column_of(C, row * C.k + i);
        const bool there = col >= 0 && col < C.V;
        E.col[i] = there ? (int32_t)col : -1;
        E.q[i] = there ? teacher_value(C, row * C.k + i) : -__builtin_inff();
        E.x[i] = there ? widen_value<VT>(x[col]) : -__builtin_inff();
        top = fmaxf(top, E.q[i]);
        ref = fmaxf(ref, E.x[i]);
    }
    top = over_lanes<kWave>(top, kMax);
    ref = over_lanes<kWave>(ref, kMax);
    const float c = C.scale * kLog2e;
    float sum = 0.f;
    for (int i = lane; i < C.k; i += kWave) sum += exp2_of((E.q[i] - top) * c);
    sum = over_lanes<kWave>(sum, kAdd);
    const float ln = logf(sum), inverse = 1.f / sum;
    float loss = 0.f;
    for (int i = lane; i < C.k; i += kWave) {
        const float d = (E.q[i] - top) * c, q = sum == 0.f ? 0.f : exp2_of(d) * inverse;
        if (q != 0.f) loss += q * (fmaf(kLn2, d, -ln) - (E.x[i] - ref) * C.scale);
        E.q[i] = q;
    }
    return {0.f, over_lanes<kWave>(loss, kAdd), ref, sum == 0.f ? 0.f : sum * inverse};
}

__device__ __forceinline__ void sum_of_column(const ClassCall& C, const Entries& E, int i, float& sum, bool& mine)
{
    sum = 0.f;
    const int col = E.col[i];
    for (int j = 0; j < C.k; ++j)
        if (E.col[j] == col) {
            mine &= j >= i;
            sum += E.q[j];
        }
}

template <int VT>
__device__ __forceinline__ Asked given_class(const ClassCall& C, int64_t row, const Given& w)
{
    return {w.y >= 0 && w.y < C.V ? widen_value<VT>(((const value_store_t<VT>*)C.logits)[row * C.V + w.y]) : 0.f, 0.f, 0.f, 0.f};
}

struct Found { float ln, logprob, entropy, loss; };  // of a whole row; ln = ln S

__device__ __forceinline__ Found row_results(const ClassCall& C, const Given& w, const Sums& s, const Asked& a)
{
    Found f = {logf(s.S), 0.f, 0.f, 0.f};
    if (C.index) {
        f.loss = a.Q == 0.f ? 0.f : s.S == 0.f ? __builtin_inff() : a.C + a.Q * (f.ln + (s.m - a.ref) * C.scale);
        return f;
    }
    f.entropy = s.S == 0.f ? 0.f : f.ln - kLn2 * (s.T / s.S);
    f.logprob = w.y < 0 ? 0.f : w.y >= C.V ? __builtin_nanf("") : s.S == 0.f ? -__builtin_inff() : (a.x - s.m) - f.ln;
    return f;
}

__device__ __forceinline__ void store_results(const ClassCall& C, int64_t row, const Found& f)
{
    if (C.logprob) C.logprob[row] = f.logprob;
    if (C.entropy) C.entropy[row] = f.entropy;
    if (C.loss) C.loss[row] = f.loss;
}

struct Alternative { float logprob; uint32_t col; };
__device__ __forceinline__ Alternative alternative(const Sums& s, float ln, uint64_t key, int i)
{
    const float x = key_value((uint32_t)(key >> 32));
    return {key == 0 || s.S != s.S ? __builtin_nanf("") : s.S == 0.f ? -__builtin_inff() : (x - s.m) - ln,
            key ? 0xFFFFFFFFu - (uint32_t)key : (uint32_t)i};  // (a row of NaN leaves none)
}
__device__ __forceinline__ void store_likeliest(const ClassCall& C, int64_t row, const Sums& s, float ln, uint64_t key, int i)
{
    if (i >= C.top_k) return;
    const int64_t at = row * C.top_k + i;
    const Alternative a = alternative(s, ln, key, i);
    C.top_data[at] = a.logprob;
    if (C.top_index_bytes == 1) ((uint8_t*)C.top_index)[at] = (uint8_t)a.col;
    else if (C.top_index_bytes == 2) ((uint16_t*)C.top_index)[at] = (uint16_t)a.col;
    else ((uint32_t*)C.top_index)[at] = a.col;
}

// dx = e (A + B d) + g at the given class
struct Slope { float A, B, g; int64_t y; };
__device__ __forceinline__ Slope row_slope(const ClassCall& C, const Given& w, const Sums& s, const Asked& a, const Found& f)
{
    const float inverse = 1.f / s.S;
    if (C.index) {
        const float g = w.g * C.scale;
        return {s.S == 0.f ? 0.f : g * a.Q * inverse, 0.f, s.S == 0.f ? 0.f : g, -1};
    }
    const float g = !C.dlogprob || w.y < 0 ? 0.f : w.y >= C.V ? __builtin_nanf("") : w.g, u = w.u;
    if (s.S == 0.f) return {g != g ? g : 0.f, 0.f, 0.f, -1};
    return {(-g + u * (f.ln - f.entropy)) * inverse, -u * kLn2 * inverse, g, w.y};
}

// Columns from `first` on up to the next line of 128 bytes in memory (fewer: up to `last`)
template <int VT>
__device__ __forceinline__ int line_start(const value_store_t<VT>* row, int first, int last)
{
    constexpr int kSize = sizeof(value_store_t<VT>);
    const int past = (int)(reinterpret_cast<uintptr_t>(row + first) & 127);
    return min(first + (past ? (128 - past) / kSize : 0), last);
}

// Columns [first, last) of a row by a workgroup, `whole` being where its lines start (line_start): those before it and those behind the last whole step (32 bytes a
// thread, kStep units) go to part(unit, column, valid columns), then the steps to step(units, first one's column), each while the next one is under way.
template <int VT> constexpr int kStep = VT == MAXK_VALUE_F32 ? 1 : 2;
// (EDGES_LAST: in the other order, at the price of their registers)
template <int VT, int T, bool EDGES_LAST, typename F, typename G>
__device__ __forceinline__ void walk(const value_store_t<VT>* x, int first, int whole, int last, const value_store_t<VT>* end, F&& step, G&& part)
{
    constexpr int K = kStep<VT>, kRun = T * kRowUnit, kWhole = K * kRun;
    const int at = threadIdx.x * kRowUnit, rest = whole + (last - whole) / kWhole * kWhole;
    const RawUnit<VT> head = fetch_row_unit<VT>(x + first + at, whole - first - at, end);
    RawUnit<VT> tail[K], raw[K] = {};
#pragma unroll
    for (int i = 0; i < K; ++i) tail[i] = fetch_row_unit<VT>(x + rest + i * kRun + at, last - rest - i * kRun - at, end);
    if (whole < rest) {
#pragma unroll
        for (int i = 0; i < K; ++i) raw[i] = whole_unit<VT>(x + whole + i * kRun + at);
    }
    const auto edges = [&] {
        if (first < whole) part(head, first + at, whole - first - at);
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (rest + i * kRun < last) part(tail[i], rest + i * kRun + at, last - rest - i * kRun - at);
    };
    if (!EDGES_LAST) edges();
    int base = whole;
    for (; base + kWhole < rest; base += kWhole) {
        RawUnit<VT> next[K];
#pragma unroll
        for (int i = 0; i < K; ++i) next[i] = whole_unit<VT>(x + base + kWhole + i * kRun + at);
        step(raw, base + at);
#pragma unroll
        for (int i = 0; i < K; ++i) raw[i] = next[i];
    }
    if (whole < rest) step(raw, base + at);
    if (EDGES_LAST) edges();
}

// Columns [first, last) of a row by a workgroup: their sums, and the likeliest of them in every wavefront
template <int VT, int T, bool CAREFUL, bool ENTROPY, bool TOP>
__device__ __forceinline__ Sums sum_columns(const ClassCall& C, int64_t row, int first, int last, Likeliest& best)
{
    using S = value_store_t<VT>;
    const S *x = (const S*)C.logits + row * C.V, *end = (const S*)C.logits + C.N * C.V;
    const float c = C.scale * kLog2e;
    Way<CAREFUL, ENTROPY> sums;
    sums.begin();
    bool begun = false;
    const auto part = [&](const RawUnit<VT>& raw, int col, int valid) {
        float v[kRowUnit];
        unit_values<VT>(raw, valid, -__builtin_inff(), v);
        const float top = largest(v);
        sums.absorb(v, top, c);
        if constexpr (TOP) {
            if (!begun) best.expect(top, valid > 0);
            begun = true;
            best.offer(v, top, col, valid);
        }
    };
    walk<VT, T, TOP>(
        x, first, first, last, end,  // (wherever it lies: the sums' bits do not depend on it)
        [&](const RawUnit<VT>(&raw)[kStep<VT>], int col) {
            float v[kStep<VT>][kRowUnit], top[kStep<VT>], most;
#pragma unroll
            for (int i = 0; i < kStep<VT>; ++i) {
                unit_values<VT>(raw[i], kRowUnit, 0.f, v[i]);
                top[i] = largest(v[i]);
                most = i ? fmaxf(most, top[i]) : top[i];
            }
#pragma unroll
            for (int i = 0; i < kStep<VT>; ++i) sums.absorb(v[i], top[i], c);
            if constexpr (TOP) {
                if (!begun) best.expect(most, true);
                begun = true;
#pragma unroll
                for (int i = 0; i < kStep<VT>; ++i) best.offer(v[i], top[i], col + i * T * kRowUnit, kRowUnit);
            }
        },
        part);
    return sums.end(c);
}

__device__ __forceinline__ bool far_off(const Sums& s, float c) { return !(fabsf(s.m * c) < kFarOff); }

// The workgroup's sums of these columns (`room` is free behind the next barrier); what other wavefronts left in LDS before is there
template <int VT, int T, bool ENTROPY, bool TOP, typename F>
__device__ __forceinline__ Sums sum_row(const ClassCall& C, int64_t row, int first, int last, Likeliest& best, Sums* room, F&& before_joining)
{
    const float c = C.scale * kLog2e;
    Sums s = sum_columns<VT, T, false, ENTROPY, TOP>(C, row, first, last, best);
    before_joining();
    s = join_workgroup<T>(s, c, room);
    if (far_off(s, c)) {
        s = sum_columns<VT, T, true, ENTROPY, false>(C, row, first, last, best);
        __syncthreads();
        s = join_workgroup<T>(s, c, room);
    }
    return s;
}

// Their gradient; distillation's entries in these columns follow
template <int VT, int T, bool CAREFUL, bool DISTILL, typename F>
__device__ __forceinline__ void store_columns(const ClassCall& C, int64_t row, int first, int last, const Sums& s, const Slope& k, const Entries* E, F&& before_entries)
{
    using S = value_store_t<VT>;
    const S *x = (const S*)C.logits + row * C.V, *end = (const S*)C.logits + C.N * C.V;
    S* dx = (S*)C.dlogits + row * C.V;
    // (the quick form of d as in Way: its rest goes into A and B)
    const float c = C.scale * kLog2e, q = s.m * c, delta = CAREFUL ? 0.f : fmaf(-s.m, c, q), f = exp2_of(delta), A = f * fmaf(k.B, delta, k.A), B = f * k.B;
    const auto slope = [&](float v, float g) {  // (one rounding, whichever way a column comes here: bits do not depend on where the row starts)
        const float d = CAREFUL ? (v - s.m) * c : fmaf(v, c, -q);
        return fmaf(exp2_of(d), DISTILL ? A : fmaf(B, fmaxf(d, -kFar), A), g);
    };
    const auto unit = [&](float (&v)[kRowUnit], int col) {
        if (!DISTILL && (uint64_t)(k.y - col) < kRowUnit) {
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) v[j] = slope(v[j], j == (int)(k.y - col) ? k.g : 0.f);
        } else {
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) v[j] = slope(v[j], 0.f);
        }
    };
    const bool once = past_l2(C.N * C.V * (int64_t)sizeof(S));
    walk<VT, T, false>(
        x, first, line_start<VT>(dx, first, last), last, end,
        [&](const RawUnit<VT>(&raw)[kStep<VT>], int col) {
#pragma unroll
            for (int i = 0; i < kStep<VT>; ++i, col += T * kRowUnit) {
                float v[kRowUnit];
                unit_values<VT>(raw[i], kRowUnit, 0.f, v);
                unit(v, col);
                if (once) store_unit_once<VT>(dx + col, v);
                else store_whole_unit<VT>(dx + col, v);
            }
        },
        [&](const RawUnit<VT>& raw, int col, int valid) {
            if (valid < 1) return;
            float v[kRowUnit];
            unit_values<VT>(raw, valid, 0.f, v);
            unit(v, col);
            store_row_unit<VT>(dx + col, valid, v);
        });
    before_entries();
    if constexpr (DISTILL) {
        __syncthreads();  // what is stored above at their columns is stored again
        for (int i = threadIdx.x; i < C.k; i += T) {
            const int col = E->col[i];
            if (col < first || col >= last) continue;
            float sum = E->q[i];
            bool mine = true;
            if (C.k > kFewEntries) sum_of_column(C, *E, i, sum, mine);
            if (mine) dx[col] = round_value<VT>(slope(E->x[i], -k.g * sum));
        }
    }
}

template <int VT, int T, bool DISTILL, typename F>
__device__ __forceinline__ void store_gradient(const ClassCall& C, int64_t row, int first, int last, const Sums& s, const Slope& k, const Entries* E, F&& before_entries)
{
    if (far_off(s, C.scale * kLog2e)) store_columns<VT, T, true, DISTILL>(C, row, first, last, s, k, E, before_entries);
    else store_columns<VT, T, false, DISTILL>(C, row, first, last, s, k, E, before_entries);
}

// ---- a row in the registers of L lanes, U units of 8 columns each ----

// Of keys as doubles, which are none of them NaN: what fmax and fmin would do to NaN first costs as much again
__device__ __forceinline__ double greater_of(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double lesser_of(double a, double b)
{
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// The k greatest of the L lanes' keys, in turn: a key is a double in [1, 2) whose last 20 bits hold the column, so that the greatest is one operation
// a step; rows are of at most 2048 columns.  A key that was taken is below 1.
__device__ __forceinline__ double pair_key(float x, int col)
{
    const uint32_t v = value_key(x);
    return __hiloint2double((int)(0x3FF00000u | v >> 12), (int)(v << 20 | (0xFFFFFu - (uint32_t)col)));
}
__device__ __forceinline__ uint64_t unpaired(double key)
{
    const uint32_t high = (uint32_t)__double2hiint(key), low = (uint32_t)__double2loint(key);
    return high < 0x3FF00000u ? 0 : (uint64_t)(high << 12 | low >> 20) << 32 | (0xFFFFFFFFu - (0xFFFFFu - (low & 0xFFFFFu)));
}

// Entries of the teacher by the lanes of a row: the loss's part, and (GRAD) the sums of q at every column to `spread`, LDS for the columns of the row.
template <int VT, int L, int U, bool GRAD>
struct TeamEntries {
    const ClassCall& C;
    const value_store_t<VT>* x;
    int64_t at;
    int lane, first;   // column of the lane's own entry, which it has where there are no more than lanes
    float own;
    float* spread;

    __device__ __forceinline__ int column(int i) const
    {
        const int64_t col = column_of(C, at + i);
        return col >= 0 && col < C.V ? (int)col : -1;
    }
    __device__ __forceinline__ float value(int i, int col) const { return col >= 0 ? teacher_value(C, at + i) : -__builtin_inff(); }
    __device__ __forceinline__ float logit(int col) const { return col >= 0 ? widen_value<VT>(x[col]) : -__builtin_inff(); }

    __device__ __forceinline__ TeamEntries(const ClassCall& C_, int64_t row, int lane_, float* spread_)
        : C(C_), x((const value_store_t<VT>*)C_.logits + row * C_.V), at(row * C_.k), lane(lane_), spread(spread_)
    {
        if (C.k > L) return;
        first = lane < C.k ? column(lane) : -1;
        own = value(lane, first);
    }

    // columns without an entry have 0; those of one have the entry's number + 1 (of several: of one of them).  Whether there are several
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < kRowUnit; j += 4) *reinterpret_cast<float4*>(spread + (lane + u * L) * kRowUnit + j) = make_float4(0.f, 0.f, 0.f, 0.f);
        wave_fence();
    }
    __device__ __forceinline__ bool others(int i, int col) const { return col >= 0 && __float_as_int(spread[col]) != i + 1; }
    __device__ __forceinline__ bool any(bool b) const { return over_lanes<L>((uint32_t)b, [](uint32_t p, uint32_t q) { return p | q; }) != 0; }

    __device__ __forceinline__ Asked take()
    {
        const float c = C.scale * kLog2e;
        if (C.k <= L) return take_some<1>(c);
        if (C.k <= 4 * L) return take_some<4>(c);
        if (U == 1 || C.k <= 8 * L) return take_some<8>(c);  // (no row has more columns)
        return take_more(c);
    }

    template <int R>
    __device__ __forceinline__ Asked take_some(float c)  // up to R entries a lane
    {
        int col[R];
        float t[R], v[R], q[R], top = kLowest, ref = kLowest;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = lane + r * L;
            col[r] = R == 1 ? first : i < C.k ? column(i) : -1;
            t[r] = R == 1 ? own : value(i, col[r]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            v[r] = logit(col[r]);
            top = fmaxf(top, t[r]);
        }
        top = over_lanes<L>(top, kMax);
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            t[r] = (t[r] - top) * c;
            q[r] = exp2_of(t[r]);
            sum += q[r];
            ref = fmaxf(ref, v[r]);
        }
        sum = over_lanes<L>(sum, kAdd);
        ref = over_lanes<L>(ref, kMax);
        const float ln = logf(sum), inverse = 1.f / sum;
        float loss = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            q[r] = sum == 0.f ? 0.f : q[r] * inverse;
            loss += q[r] != 0.f ? q[r] * (fmaf(kLn2, t[r], -ln) - (v[r] - ref) * C.scale) : 0.f;
        }
        loss = over_lanes<L>(loss, kAdd);
        if constexpr (GRAD) {
            clear();
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (col[r] >= 0) spread[col[r]] = __int_as_float(lane + r * L + 1);
            wave_fence();
            uint32_t other = 0;  // entries that are not the one that writes their column
#pragma unroll
            for (int r = 0; r < R; ++r) other |= (uint32_t)others(lane + r * L, col[r]) << r;
            if (any(other != 0)) {  // sums in the entries' order
                float all[R] = {};
#pragma unroll
                for (int from = 0; from < R; ++from)
                    for (int l = 0; l < L; ++l) {
                        const int there = __shfl(col[from], l, L);
                        const float p = __shfl(q[from], l, L);
#pragma unroll
                        for (int r = 0; r < R; ++r) all[r] += there == col[r] ? p : 0.f;
                    }
#pragma unroll
                for (int r = 0; r < R; ++r) q[r] = all[r];
            }
            wave_fence();
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (col[r] >= 0 && !(other >> r & 1)) spread[col[r]] = q[r];
            wave_fence();
        }
        return {0.f, loss, ref, sum == 0.f ? 0.f : sum * inverse};
    }

    __device__ Asked take_more(float c)
    {
        float top = kLowest, ref = kLowest;
        for (int i = lane; i < C.k; i += L) {
            const int col = column(i);
            top = fmaxf(top, value(i, col));
            ref = fmaxf(ref, logit(col));
        }
        top = over_lanes<L>(top, kMax);
        ref = over_lanes<L>(ref, kMax);
        float sum = 0.f;
        for (int i = lane; i < C.k; i += L) sum += exp2_of((value(i, column(i)) - top) * c);
        sum = over_lanes<L>(sum, kAdd);
        const float ln = logf(sum), inverse = 1.f / sum;
        const auto weight = [&](float d) { return sum == 0.f ? 0.f : exp2_of(d) * inverse; };
        if constexpr (GRAD) {
            clear();
            for (int i = lane; i < C.k; i += L)
                if (const int col = column(i); col >= 0) spread[col] = __int_as_float(i + 1);
            wave_fence();
        }
        float loss = 0.f;
        bool several = false;
        for (int i = lane; i < C.k; i += L) {
            const int col = column(i);
            const float d = (value(i, col) - top) * c, q = weight(d);
            if (q != 0.f) loss += q * (fmaf(kLn2, d, -ln) - (logit(col) - ref) * C.scale);
            if constexpr (GRAD) several |= others(i, col);
        }
        if constexpr (GRAD) {
            several = any(several);  // (all marks are read before the first sum is written)
            wave_fence();
            for (int i = lane; i < C.k; i += L) {
                const int col = column(i);
                if (col < 0) continue;
                float q = 0.f;
                if (several) {  // sums in the entries' order.  (an entry that finds a sum where its mark was writes the same sum)
                    if (others(i, col)) continue;
                    for (int j = 0; j < C.k; ++j)
                        if (column(j) == col) q += weight((value(j, col) - top) * c);
                } else {
                    q = weight((value(i, col) - top) * c);
                }
                spread[col] = q;
            }
            wave_fence();
        }
        return {0.f, over_lanes<L>(loss, kAdd), ref, sum == 0.f ? 0.f : sum * inverse};
    }
};

template <int L>
__device__ __forceinline__ void likeliest_in_turn(const ClassCall& C, int64_t row, const Sums& s, float ln, const float (&v)[kRowUnit], int lane)
{
    double key[kRowUnit];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) key[j] = lane * kRowUnit + j < C.V ? pair_key(v[j], lane * kRowUnit + j) : 0.0;
    double taken = 0.0;
    for (int i = 0; i < C.top_k; ++i) {
        double best = key[0];
#pragma unroll
        for (int j = 1; j < kRowUnit; ++j) best = greater_of(best, key[j]);
        best = over_lanes<L>(best, [](double a, double b) { return greater_of(a, b); });
        const int col = (int)(0xFFFFFu - ((uint32_t)__double2loint(best) & 0xFFFFFu));
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j)
            if (col == lane * kRowUnit + j) key[j] = __hiloint2double(0, __double2loint(key[j]));
        if (i % L == lane) taken = best;
        if (i % L == L - 1 || i == C.top_k - 1) {
            const int at = i - i % L + lane;
            if (at <= i) store_likeliest(C, row, s, ln, unpaired(taken), at);
        }
    }
}

// Keys of a row in order: of fp32 as above, of 16-bit values, which leave the last 12 bits of theirs alone, in 32 bits with the column (rows are of up to 256) in the last 8.
template <int VT>
__device__ __forceinline__ auto short_key(float x, int col)
{
    if constexpr (VT == MAXK_VALUE_F32) return pair_key(x, col);
    else return (value_key(x) & ~0xFFu) | (uint32_t)(255 - col);
}
__device__ __forceinline__ uint64_t long_key(double key) { return unpaired(key); }
__device__ __forceinline__ uint64_t long_key(uint32_t key)  // (the value's last bits: as those of a negative one, or none)
{
    const uint32_t v = key & ~0xFFu;
    return (uint64_t)(v & 0x80000000u ? v : v | 0xFFu) << 32 | (0xFFFFFFFFu - (255 - (key & 0xFFu)));
}
__device__ __forceinline__ uint32_t greater_of(uint32_t a, uint32_t b) { return max(a, b); }
__device__ __forceinline__ uint32_t lesser_of(uint32_t a, uint32_t b) { return min(a, b); }
template <typename K>
__device__ __forceinline__ void in_order(K& a, K& b)
{
    const K less = lesser_of(a, b);
    a = greater_of(a, b);
    b = less;
}
// of lane ^ X, X all ones (a group's lanes from its other end) or one bit
template <int X>
__device__ __forceinline__ uint32_t partner(uint32_t x)
{
    if constexpr (X == 3) return dpp<0x1B>(x);                // quad_perm [3,2,1,0]
    else if constexpr (X == 7) return dpp<0x141>(x);          // row_half_mirror
    else if constexpr (X == 15) return dpp<0x140>(x);         // row_mirror
    else if constexpr (X == 31) return across<16>(dpp<0x140>(x));
    else return across<X>(x);
}
template <int X>
__device__ __forceinline__ double partner(double x)
{
    return __hiloint2double((int)partner<X>((uint32_t)__double2hiint(x)), (int)partner<X>((uint32_t)__double2loint(x)));
}
template <typename K>
__device__ __forceinline__ K end_of(K mine, K other, bool greater) { return greater ? greater_of(mine, other) : lesser_of(mine, other); }
// runs of eight in a lane whose halves are neither before nor behind each other in order, once their greater and lesser ones are apart
template <int STEP, typename K>
__device__ __forceinline__ void settle_unit(K (&key)[kRowUnit])
{
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j)
        if ((j & STEP) == 0) in_order(key[j], key[j + STEP]);
    if constexpr (STEP > 1) settle_unit<STEP / 2>(key);
}
template <int STEP, typename K>
__device__ __forceinline__ void settle_lanes(K (&key)[kRowUnit], int lane)
{
    if constexpr (STEP > 0) {
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) key[j] = end_of(key[j], partner<STEP>(key[j]), (lane & STEP) == 0);
        settle_lanes<STEP / 2>(key, lane);
    }
}
// Two groups of M lanes, each in order, into one: the first against the last of the other, the second against the last but one ...
template <int M, int L, typename K>
__device__ __forceinline__ void merge_groups(K (&key)[kRowUnit], int lane)
{
    if constexpr (M < L) {
        K other[kRowUnit];
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) other[j] = partner<2 * M - 1>(key[kRowUnit - 1 - j]);
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) key[j] = end_of(key[j], other[j], (lane & M) == 0);
        settle_lanes<M / 2>(key, lane);
        settle_unit<4>(key);
        merge_groups<2 * M, L>(key, lane);
    }
}
template <int VT, int L>
__device__ __forceinline__ void likeliest_in_order(const ClassCall& C, int64_t row, const Sums& s, float ln, const float (&v)[kRowUnit], int lane)
{
    using K = decltype(short_key<VT>(0.f, 0));
    K key[kRowUnit];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) key[j] = lane * kRowUnit + j < C.V ? short_key<VT>(v[j], lane * kRowUnit + j) : K(0);
#pragma unroll
    for (int size = 2; size <= kRowUnit; size *= 2) {
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j)
            if ((j & (size / 2)) == 0) in_order(key[j], key[j ^ (size - 1)]);
#pragma unroll
        for (int step = size / 4; step > 0; step /= 2)
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j)
                if ((j & step) == 0) in_order(key[j], key[j + step]);
    }
    merge_groups<1, L>(key, lane);
    float data[kRowUnit];
    uint32_t index[kRowUnit];
    uint16_t short_index[kRowUnit];
    uint8_t byte_index[kRowUnit];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) {
        const Alternative a = alternative(s, ln, long_key(key[j]), lane * kRowUnit + j);
        data[j] = a.logprob, index[j] = a.col, short_index[j] = (uint16_t)a.col, byte_index[j] = (uint8_t)a.col;
    }
    const int64_t at = row * C.top_k + lane * kRowUnit;
    const int valid = C.top_k - lane * kRowUnit;
    store_values(C.top_data + at, valid, data);
    if (C.top_index_bytes == 1) store_values((uint8_t*)C.top_index + at, valid, byte_index);
    else if (C.top_index_bytes == 2) store_values((uint16_t*)C.top_index + at, valid, short_index);
    else store_values((uint32_t*)C.top_index + at, valid, index);
}

// Rounds cost some sixty instructions for each alternative, an order of the whole row 150 to 400.  us, in turn / in order: 150000 x 200 bf16 1 alternative 41 / 98, 12 105 / 107,
// 16 130 / 107, 64 426 / 108; 300000 x 100 fp32 12 93 / 94, 16 112 / 94, 64 279 / 95; 500000 x 47 bf16 10 69 / 59, fp32 12 79 / 70; 130000 x 20 bf16 8 16 / 10.
template <int L> constexpr int kFewInTurn = L == 4 ? 7 : L == 8 ? 10 : 13;


struct Nothing {
    __device__ __forceinline__ Nothing(const ClassCall&, int64_t, int, float*) {}
};

template <int VT, int L, int U, bool DISTILL, bool GRAD, bool TOP>
__global__ void __launch_bounds__(kThreads) class_team_kernel(ClassCall C)
{
    using S = value_store_t<VT>;
    constexpr int kTeams = kThreads / L;
    __shared__ __attribute__((aligned(16))) float spread[DISTILL && GRAD ? kTeams * L * U * kRowUnit : 1];
    __shared__ uint64_t keys[TOP && L == kWave ? kThreads / kWave : 1][TOP && L == kWave ? kWaiting : 1];
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int64_t row = group_number() * kTeams + team;
    if (row >= C.N) return;
    const S *x = (const S*)C.logits + row * C.V, *end = (const S*)C.logits + C.N * C.V;
    const float c = C.scale * kLog2e;
    RawUnit<VT> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int col = (lane + u * L) * kRowUnit;
        raw[u] = fetch_row_unit<VT>(x + col, C.V - col, end);
    }
    float* mine = spread + (DISTILL && GRAD ? team * L * U * kRowUnit : 0);
    Asked asked;
    std::conditional_t<DISTILL, TeamEntries<VT, L, U, GRAD>, Nothing> entries(C, row, lane, mine);
    const Given given = row_given(C, row);
    float v[U][kRowUnit];
#pragma unroll
    for (int u = 0; u < U; ++u) unit_values<VT>(raw[u], C.V - (lane + u * L) * kRowUnit, -__builtin_inff(), v[u]);
    Sums s = no_sums();
    float lane_top = largest(v[0]);
#pragma unroll
    for (int u = 1; u < U; ++u) lane_top = fmaxf(lane_top, largest(v[u]));
    s.m = over_lanes<L>(fmaxf(lane_top, kLowest), kMax);
    float e[U][kRowUnit];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) {
            const float d = (v[u][j] - s.m) * c;
            e[u][j] = exp2_of(d);
            s.S += e[u][j];
            if constexpr (!DISTILL) s.T = fmaf(e[u][j], fmaxf(d, -kFar), s.T);
        }
    s.S = over_lanes<L>(s.S, kAdd);
    if constexpr (!DISTILL) s.T = over_lanes<L>(s.T, kAdd);
    if constexpr (DISTILL) {
        asked = entries.take();
    } else {
        float x_given = 0.f;  // of the lane that has the class
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) x_given = given.y == (lane + u * L) * kRowUnit + j ? v[u][j] : x_given;
        asked = {over_lanes<L>(x_given, kAdd), 0.f, 0.f, 0.f};
    }
    const Found f = row_results(C, given, s, asked);
    if (lane == 0) store_results(C, row, f);
    if constexpr (TOP && L == kWave) {
        Likeliest best;
        best.begin(C.top_k, keys[team], lane);
        best.expect(lane_top, lane * kRowUnit < C.V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (lane + u * L) * kRowUnit;
            best.offer(v[u], largest(v[u]), col, C.V - col);
        }
        best.end();
        store_likeliest(C, row, s, f.ln, fill<VT>(best.mine, s, x, C.V, C.top_k, lane, keys[team]), lane);
    } else if constexpr (TOP) {
        static_assert(U == 1);
        if (C.top_k < kFewInTurn<L>) likeliest_in_turn<L>(C, row, s, f.ln, v[0], lane);
        else likeliest_in_order<VT, L>(C, row, s, f.ln, v[0], lane);
    }
    if constexpr (GRAD) {
        const Slope k = row_slope(C, given, s, asked, f);
        S* dx = (S*)C.dlogits + row * C.V;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (lane + u * L) * kRowUnit;
            float g[kRowUnit];
            if constexpr (DISTILL) {
                const float4 a = *reinterpret_cast<const float4*>(mine + col), b = *reinterpret_cast<const float4*>(mine + col + 4);
                const float q[kRowUnit] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int j = 0; j < kRowUnit; ++j) g[j] = fmaf(-k.g, q[j], e[u][j] * k.A);
            } else {
#pragma unroll
                for (int j = 0; j < kRowUnit; ++j) {
                    g[j] = e[u][j] * fmaf(k.B, fmaxf((v[u][j] - s.m) * c, -kFar), k.A);
                    if (k.y == col + j) g[j] += k.g;
                }
            }
            store_row_unit<VT>(dx + col, C.V - col, g);
        }
    }
}

// ---- few classes, few alternatives: a lane a row ----

// Rows of up to 64 columns of which few alternatives are wanted: eight lanes bring a row into LDS, then every lane has one for itself and keeps its K greatest
// keys in order, two operations a column and key.  (Between lanes a round costs some sixty instructions for each alternative: 2.4 M rows of 47 fp32, 5 of
// them, 230 us.)  A key of 32 bits has the column in its last 6 and the leading 26 of the value, all that a 16-bit value has.  Of fp32 one more key than alternatives
// is kept: where two neighbours share their 26 bits, the row is gone through again with keys of 64 bits, twice the time (all of them so: 185 us).
constexpr int kLaneRowMost = 64, kLaneRowKeys = 8;
__host__ __device__ constexpr int lane_row_pitch(int V) { return (V + 7) / 8 * 8 + 1; }  // whole units, and lanes on different banks
template <int VT, int K>
__global__ void __launch_bounds__(kThreads) class_lane_kernel(ClassCall C)
{
    using S = value_store_t<VT>;
    constexpr int kBring = kThreads / 8;  // rows an access
    extern __shared__ float rows_of_lanes[];
    const int pitch = lane_row_pitch(C.V), part = threadIdx.x % 8 * kRowUnit;
    const int64_t row0 = group_number() * kThreads, row = row0 + threadIdx.x;
    if (row0 >= C.N) return;
    const S *x = (const S*)C.logits, *end = x + C.N * C.V;
    RawUnit<VT> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = row0 + i * kBring + threadIdx.x / 8;
        raw[i] = fetch_row_unit<VT>(x + r * C.V + part, r < C.N ? C.V - part : 0, end);
    }
    const Given given = row_given(C, min(row, C.N - 1));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float* to = rows_of_lanes + (i * kBring + threadIdx.x / 8) * pitch + part;
        if (part < pitch - 1) {
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) to[j] = raw_value<VT>(raw[i], j);
        }
    }
    __syncthreads();
    if (row >= C.N) return;
    const float *mine = rows_of_lanes + threadIdx.x * pitch, c = C.scale * kLog2e;
    uint32_t few[K];
#pragma unroll
    for (int i = 0; i < K; ++i) few[i] = 0;
#pragma unroll 4
    for (int j = 0; j < C.V; ++j) {
        uint32_t key = (value_key(mine[j]) & ~63u) | (uint32_t)(63 - j);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const uint32_t less = min(few[i], key);
            few[i] = max(few[i], key);
            key = less;
        }
    }
    uint64_t best[K];
#pragma unroll
    for (int i = 0; i < K; ++i) best[i] = few[i] ? key_of(mine[63 - (few[i] & 63u)], 63 - (few[i] & 63u)) : 0;
    if constexpr (VT == MAXK_VALUE_F32) {
        bool near = false;
#pragma unroll
        for (int i = 0; i + 1 < K; ++i) near |= i < C.top_k && (few[i] ^ few[i + 1]) < 64u;
        if (near) {
            double whole[K];
#pragma unroll
            for (int i = 0; i < K; ++i) whole[i] = 0.0;
            for (int j = 0; j < C.V; ++j) {
                double key = pair_key(mine[j], j);
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    const double less = lesser_of(whole[i], key);
                    whole[i] = greater_of(whole[i], key);
                    key = less;
                }
            }
#pragma unroll
            for (int i = 0; i < K; ++i) best[i] = unpaired(whole[i]);
        }
    }
    const Asked asked = {given.y >= 0 && given.y < C.V ? mine[given.y] : 0.f, 0.f, 0.f, 0.f};
    Sums s = no_sums();
    s.m = fmaxf(key_value((uint32_t)(best[0] >> 32)), s.m);  // (a NaN, which is greater than all others, makes S one)
#pragma unroll 4
    for (int j = 0; j < C.V; ++j) {
        const float d = (mine[j] - s.m) * c, e = exp2_of(d);
        s.S += e;
        s.T = fmaf(e, fmaxf(d, -kFar), s.T);
    }
    const Found f = row_results(C, given, s, asked);
    store_results(C, row, f);
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i < C.top_k) store_likeliest(C, row, s, f.ln, best[i], i);
}

// ---- few classes of many rows, without alternatives: a lane a row ----

// The rows of a workgroup are one stretch of memory, which goes to LDS and back 16 bytes an access whatever a row's length, and every lane has one of them
// there, as it is stored, for itself: sums over a row pass no lane.  Where a row is an even number of words one more lies behind it, so that lanes are on different banks.
struct Stretch {
    int row;           // bytes of a row, of up to 64 elements and 8 at least
    int words;         // of a row with one more behind it, 0: rows lie side by side
    uint32_t inverse;  // of words

    __host__ __device__ static Stretch of(int n, int size)
    {
        Stretch s = {n * size, 0, 0};
        if (s.row % 8 == 0 && s.row >= 16) s.words = s.row / 4, s.inverse = (uint32_t)(((1ull << 32) + s.words - 1) / s.words);  // (exact: words there are fewer than 2^15)
        return s;
    }
    __host__ __device__ int pitch() const { return words ? row + 4 : row; }
    __host__ __device__ int room() const { return (kThreads * pitch() + 15) / 16 * 16; }
    __device__ __forceinline__ int place(int byte) const { return words ? byte + 4 * (int)__umulhi((uint32_t)byte / 4, inverse) : byte; }
    // a piece of 16 bytes: of at most two rows where a row is four words and more
    template <typename F>
    __device__ __forceinline__ void in_words(int piece, F&& word) const
    {
        const int first = piece * 4, number = (int)__umulhi((uint32_t)first, inverse), next = (number + 1) * words;
#pragma unroll
        for (int i = 0; i < 4; ++i) word(i, first + i + number + (first + i >= next));
    }
    __device__ __forceinline__ void put(char* room, int piece, uint4 v) const
    {
        if (!words) {
            *reinterpret_cast<uint4*>(room + piece * 16) = v;
            return;
        }
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        in_words(piece, [&](int i, int at) { reinterpret_cast<uint32_t*>(room)[at] = w[i]; });
    }
    __device__ __forceinline__ uint4 get(const char* room, int piece) const
    {
        if (!words) return *reinterpret_cast<const uint4*>(room + piece * 16);
        uint32_t w[4];
        in_words(piece, [&](int i, int at) { w[i] = reinterpret_cast<const uint32_t*>(room)[at]; });
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // `bytes` of memory to LDS, PIECES of 16 a lane under way at a time
    template <int PIECES>
    __device__ __forceinline__ void bring(const char* from, int bytes, char* room) const
    {
        const int pieces = bytes / 16;
        for (int base = threadIdx.x; base < pieces; base += PIECES * kThreads) {
            uint4 v[PIECES];
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (base + i * kThreads < pieces) v[i] = read16(from + (int64_t)(base + i * kThreads) * 16);
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (base + i * kThreads < pieces) put(room, base + i * kThreads, v[i]);
        }
        if (const int at = pieces * 16 + threadIdx.x; at < bytes) room[place(at)] = from[at];
    }
    __device__ __forceinline__ void take(const char* room, int bytes, char* to) const
    {
        const int pieces = bytes / 16;
        for (int piece = threadIdx.x; piece < pieces; piece += kThreads) write16(to + (int64_t)piece * 16, get(room, piece));
        if (const int at = pieces * 16 + threadIdx.x; at < bytes) to[at] = room[place(at)];
    }
};
constexpr int kLaneRowLeast = 8;   // (four words a row and more: in_words)
constexpr int kOwnEntries = 8;   // of a teacher, in the lane's registers
template <int VT, bool DISTILL, bool GRAD, bool ENTROPY>
__global__ void __launch_bounds__(kThreads) class_own_kernel(ClassCall C, Stretch R)
{
    using S = value_store_t<VT>;
    constexpr int K = DISTILL ? kOwnEntries : 1;
    extern __shared__ uint4 rooms_of_rows[];
    char* const rows = reinterpret_cast<char*>(rooms_of_rows);
    const int64_t row0 = group_number() * kThreads, row = row0 + threadIdx.x;
    if (row0 >= C.N) return;
    const int bytes = (int)min(C.N - row0, (int64_t)kThreads) * R.row;
    R.bring<sizeof(S) * kLaneRowMost / 16>((const char*)C.logits + row0 * R.row, bytes, rows);
    const int64_t known = min(row, C.N - 1);
    const Given given = row_given(C, known);
    int col[K];
    float t[K], v[K];
    if constexpr (DISTILL) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int64_t at = known * C.k + min(i, C.k - 1), there = column_of(C, at);
            col[i] = i < C.k && there >= 0 && there < C.V ? (int)there : -1;
            t[i] = teacher_value(C, at);
        }
    }
    __syncthreads();
    if (row < C.N) {
        S* const mine = reinterpret_cast<S*>(rows + threadIdx.x * R.pitch());
        const float c = C.scale * kLog2e;
        Sums s = no_sums();
#pragma unroll 8
        for (int j = 0; j < C.V; ++j) s.m = fmaxf(s.m, widen_value<VT>(mine[j]));
#pragma unroll 8
        for (int j = 0; j < C.V; ++j) {
            const float d = (widen_value<VT>(mine[j]) - s.m) * c, e = exp2_of(d);
            s.S += e;
            if constexpr (ENTROPY) s.T = fmaf(e, fmaxf(d, -kFar), s.T);
        }
        Asked asked = {0.f, 0.f, 0.f, 0.f};
        if constexpr (!DISTILL) asked.x = given.y >= 0 && given.y < C.V ? widen_value<VT>(mine[given.y]) : 0.f;
        if constexpr (DISTILL) {
            float top = kLowest, sum = 0.f;
            asked.ref = kLowest;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                v[i] = col[i] >= 0 ? widen_value<VT>(mine[col[i]]) : -__builtin_inff();
                t[i] = col[i] >= 0 ? t[i] : -__builtin_inff();
                top = fmaxf(top, t[i]);
                asked.ref = fmaxf(asked.ref, v[i]);
            }
#pragma unroll
            for (int i = 0; i < K; ++i) {
                t[i] = (t[i] - top) * c;
                sum += exp2_of(t[i]);
            }
            const float ln = logf(sum), inverse = 1.f / sum;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const float q = sum == 0.f ? 0.f : exp2_of(t[i]) * inverse;
                asked.C += q != 0.f ? q * (fmaf(kLn2, t[i], -ln) - (v[i] - asked.ref) * C.scale) : 0.f;
                t[i] = q;
            }
            asked.Q = sum == 0.f ? 0.f : sum * inverse;
        }
        const Found f = row_results(C, given, s, asked);
        store_results(C, row, f);
        if constexpr (GRAD) {
            const Slope k = row_slope(C, given, s, asked, f);
            const int y = k.y < C.V ? (int)k.y : -1;
#pragma unroll 8
            for (int j = 0; j < C.V; ++j) {
                const float d = (widen_value<VT>(mine[j]) - s.m) * c;
                mine[j] = round_value<VT>(fmaf(exp2_of(d), ENTROPY ? fmaf(k.B, fmaxf(d, -kFar), k.A) : k.A, !DISTILL && y == j ? k.g : 0.f));
            }
            if constexpr (DISTILL) {  // what is stored above at their columns is stored again
                uint64_t columns = 0;
                bool several = false;  // entries of one column
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    const uint64_t bit = col[i] >= 0 ? 1ull << col[i] : 0;
                    several |= (columns & bit) != 0;
                    columns |= bit;
                }
                float q[K];
#pragma unroll
                for (int i = 0; i < K; ++i) q[i] = t[i];
                if (several) {
#pragma unroll
                    for (int i = 0; i < K; ++i) {
                        q[i] = 0.f;
#pragma unroll
                        for (int j = 0; j < K; ++j) q[i] += col[j] == col[i] ? t[j] : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < K; ++i)
                    if (col[i] >= 0) mine[col[i]] = round_value<VT>(fmaf(-k.g, q[i], exp2_of((v[i] - s.m) * c) * k.A));
            }
        }
    }
    if constexpr (GRAD) {
        __syncthreads();
        R.take(rows, bytes, (char*)C.dlogits + row0 * R.row);
    }
}

// ---- a row in the registers of a workgroup ----

// U units of 8 columns a thread: the maximum is known before the first exponential, so that wavefronts add up sums instead of joining them (six steps of two
// exponentials each, which cost a wavefront as much as its columns in rows of 4000).
template <int T, typename F>
__device__ __forceinline__ float over_workgroup(float x, F&& f, float* room)  // (passes a barrier, room is free behind the next one)
{
    x = over_lanes<kWave>(x, f);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x / kWave] = x;
    __syncthreads();
    return over_lanes<T / kWave>(room[threadIdx.x % (T / kWave)], f);
}

template <int VT, int T, int U, bool DISTILL, bool GRAD, bool TOP>
__global__ void __launch_bounds__(T) class_held_kernel(ClassCall C)
{
    using S = value_store_t<VT>;
    __shared__ float tops[T / kWave], sums_S[T / kWave], sums_T[T / kWave];
    __shared__ Asked asked_room;
    __shared__ std::conditional_t<DISTILL, Entries, int> entries;
    __shared__ uint64_t keys[TOP ? T / kWave : 1][kWaiting];
    __shared__ uint32_t heads[TOP ? T : 1];
    const int64_t row = group_number();
    if (row >= C.N) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave;
    const S *x = (const S*)C.logits + row * C.V, *end = (const S*)C.logits + C.N * C.V;
    const float c = C.scale * kLog2e;
    RawUnit<VT> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int col = (threadIdx.x + u * T) * kRowUnit;
        raw[u] = fetch_row_unit<VT>(x + col, C.V - col, end);
    }
    const Given given = row_given(C, row);
    FewEntries<VT> few;
    if constexpr (DISTILL) {
        if (wave == 0 && C.k <= kFewEntries) few.ask(C, row, lane);
    }
    Asked asked = {0.f, 0.f, 0.f, 0.f};
    if constexpr (!DISTILL) asked = given_class<VT>(C, row, given);
    float v[U][kRowUnit];
#pragma unroll
    for (int u = 0; u < U; ++u) unit_values<VT>(raw[u], C.V - (int)(threadIdx.x + u * T) * kRowUnit, -__builtin_inff(), v[u]);
    Sums s = no_sums();
    float lane_top = largest(v[0]);
#pragma unroll
    for (int u = 1; u < U; ++u) lane_top = fmaxf(lane_top, largest(v[u]));
    if constexpr (DISTILL) {
        if (wave == 0) {
            asked = C.k <= kFewEntries ? few.take(C, lane, GRAD, entries) : take_more_entries<VT>(C, row, lane, entries);
            if (lane == 0) asked_room = asked;
        }
    }
    if constexpr (TOP) heads[threadIdx.x] = Likeliest::head(lane_top, (int)threadIdx.x * kRowUnit < C.V);
    s.m = over_workgroup<T>(fmaxf(lane_top, kLowest), kMax, tops);
    const auto distance = [&](float value) { return (value - s.m) * c; };
    float e[U][kRowUnit];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) {
            const float d = distance(v[u][j]);
            e[u][j] = exp2_of(d);
            s.S += e[u][j];
            if constexpr (!DISTILL) s.T = fmaf(e[u][j], fmaxf(d, -kFar), s.T);
        }
    if constexpr (!DISTILL) s.T = over_lanes<kWave>(s.T, kAdd);
    if (!DISTILL && lane == 0) sums_T[wave] = s.T;
    s.S = over_workgroup<T>(s.S, kAdd, sums_S);
    if constexpr (!DISTILL) s.T = over_lanes<T / kWave>(sums_T[threadIdx.x % (T / kWave)], kAdd);
    if constexpr (DISTILL) asked = asked_room;
    const Found f = row_results(C, given, s, asked);
    if (threadIdx.x == 0) store_results(C, row, f);
    if constexpr (TOP) {
        Likeliest best;
        best.begin(C.top_k, keys[wave], lane);
        uint32_t all[T / kWave];  // (the whole row's lanes: of 2500 columns' 50 greatest keys a wavefront then has 15 instead of 70.  16000 rows
        // of them, bf16: 76 us, 123 with a bound of its own)
#pragma unroll
        for (int r = 0; r < T / kWave; ++r) all[r] = heads[lane + r * kWave];
        best.expect(all);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (threadIdx.x + u * T) * kRowUnit;
            best.offer(v[u], largest(v[u]), col, C.V - col);
        }
        best.end();
        const uint64_t key = merge_waves<T>(best.mine, keys, lane, wave);
        if (wave == 0) store_likeliest(C, row, s, f.ln, fill<VT>(key, s, x, C.V, C.top_k, lane, keys[0]), lane);
    }
    if constexpr (GRAD) {
        const Slope k = row_slope(C, given, s, asked, f);
        S* dx = (S*)C.dlogits + row * C.V;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (threadIdx.x + u * T) * kRowUnit;
            float g[kRowUnit];
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) {
                g[j] = e[u][j] * (DISTILL ? k.A : fmaf(k.B, fmaxf(distance(v[u][j]), -kFar), k.A));
                if (!DISTILL && k.y == col + j) g[j] += k.g;
            }
            store_row_unit<VT>(dx + col, C.V - col, g);
        }
        if constexpr (DISTILL) {
            __syncthreads();  // what is stored above at their columns is stored again
            for (int i = threadIdx.x; i < C.k; i += T) {
                const int col = entries.col[i];
                if (col < 0) continue;
                float q = entries.q[i];
                bool mine = true;
                if (C.k > kFewEntries) sum_of_column(C, entries, i, q, mine);
                if (mine) dx[col] = round_value<VT>(fmaf(-k.g, q, exp2_of(distance(entries.x[i])) * k.A));
            }
        }
    }
}

// ---- a workgroup a row ----

template <int VT, int T, bool DISTILL, bool GRAD, bool TOP>
__global__ void __launch_bounds__(T, TOP ? 4 : 8) class_rows_kernel(ClassCall C)
{
    __shared__ Sums room[T / kWave];
    __shared__ Asked asked_room;
    __shared__ std::conditional_t<DISTILL, Entries, int> entries;
    __shared__ uint64_t keys[TOP ? T / kWave : 1][kWaiting];
    const int64_t row = group_number();
    if (row >= C.N) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave;
    Likeliest best;
    if constexpr (TOP) best.begin(C.top_k, keys[wave], lane);
    Asked asked;
    if constexpr (DISTILL) {
        if (wave == 0) {  // (before its share of the row: the other wavefronts are on their way)
            FewEntries<VT> few;
            if (C.k <= kFewEntries) few.ask(C, row, lane), asked = few.take(C, lane, GRAD, entries);
            else asked = take_more_entries<VT>(C, row, lane, entries);
            if (lane == 0) asked_room = asked;
        }
    }
    const Given given = row_given(C, row);
    const Sums s = sum_row<VT, T, !DISTILL, TOP>(C, row, 0, C.V, best, room, [&] {
        if constexpr (!DISTILL) asked = given_class<VT>(C, row, given);
    });
    if constexpr (DISTILL) asked = asked_room;
    const Found f = row_results(C, given, s, asked);
    if constexpr (TOP) {
        best.end();
        const uint64_t key = merge_waves<T>(best.mine, keys, lane, wave);
        if (wave == 0)
            store_likeliest(C, row, s, f.ln, fill<VT>(key, s, (const value_store_t<VT>*)C.logits + row * C.V, C.V, C.top_k, lane, keys[0]), lane);
    }
    if (threadIdx.x == 0) store_results(C, row, f);
    if constexpr (GRAD) {
        const Slope k = row_slope(C, given, s, asked, f);
        if constexpr (DISTILL) store_gradient<VT, T, true>(C, row, 0, C.V, s, k, &entries, kNothing);
        else store_gradient<VT, T, false>(C, row, 0, C.V, s, k, nullptr, kNothing);
    }
}

// ---- rows in segments ----

struct Parts {
    int segments, width;  // columns of a segment
    Sums* sums;           // [N x segments]
    Asked* asked;         // [N]
    uint64_t* keys;       // [N x segments x top_k]
};

template <int VT, bool DISTILL, bool TOP>
__global__ void __launch_bounds__(kThreads) class_parts_kernel(ClassCall C, Parts P)
{
    constexpr int T = kThreads;
    __shared__ Sums room[T / kWave];
    __shared__ std::conditional_t<DISTILL, Entries, int> entries;
    __shared__ uint64_t keys[TOP ? T / kWave : 1][kWaiting];
    const int64_t row = blockIdx.x / P.segments;
    const int segment = blockIdx.x % P.segments, first = segment * P.width, last = min(first + P.width, C.V);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave;
    Likeliest best;
    if constexpr (TOP) best.begin(C.top_k, keys[wave], lane);
    const bool asks = segment == 0 && wave == 0;
    Asked asked;
    FewEntries<VT> few;
    Given given;
    if (asks) {
        if constexpr (!DISTILL) given = row_given(C, row);
        else if (C.k <= kFewEntries) few.ask(C, row, lane);
    }
    const Sums s = sum_row<VT, T, !DISTILL, TOP>(C, row, first, last, best, room, [&] {
        if (!asks) return;
        if constexpr (DISTILL) asked = C.k <= kFewEntries ? few.take(C, lane, false, entries) : take_more_entries<VT>(C, row, lane, entries);
        else asked = given_class<VT>(C, row, given);
        if (lane == 0) P.asked[row] = asked;
    });
    if (threadIdx.x == 0) P.sums[blockIdx.x] = s;
    if constexpr (TOP) {
        best.end();
        const uint64_t key = merge_waves<T>(best.mine, keys, lane, wave);
        if (wave == 0 && lane < C.top_k) P.keys[(int64_t)blockIdx.x * C.top_k + lane] = key;
    }
}

template <int T>
__device__ __forceinline__ Sums join_segments(const ClassCall& C, const Parts& P, int64_t row, Sums* room)
{
    Sums s = no_sums();
    for (int i = threadIdx.x; i < P.segments; i += T) s = join(s, P.sums[row * P.segments + i], C.scale * kLog2e);
    return join_workgroup<T>(s, C.scale * kLog2e, room);
}

// The likeliest of the segments' lists: keys no less than the k-th greatest of the lists' first ones (of 64 sets of lists) are few, and each counts those that are greater.
// Where they are many (equal values), wavefronts merge the lists.
constexpr int kCandidates = 1024;
template <int VT, int T, bool TOP>
__global__ void __launch_bounds__(T) class_join_kernel(ClassCall C, Parts P)
{
    __shared__ Sums sums_room[T / kWave];
    __shared__ uint64_t keys[TOP ? T / kWave : 1][kWave];  // (16 x 64: room for the candidates)
    __shared__ int candidates;
    static_assert(!TOP || T == kCandidates);
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave;
    if constexpr (TOP) {
        if (threadIdx.x == 0) candidates = 0;
    }
    const Sums s = join_segments<T>(C, P, row, sums_room);
    const Found f = row_results(C, row_given(C, row), s, P.asked[row]);
    if (threadIdx.x == 0) store_results(C, row, f);
    if constexpr (TOP) {
        const uint64_t* all = P.keys + row * P.segments * C.top_k;
        const int n = P.segments * C.top_k;
        uint32_t head = 0;
        for (int i = lane; i < P.segments; i += kWave) head = max(head, (uint32_t)(all[(int64_t)i * C.top_k] >> 32));
        uint32_t bound = 1;  // (0 is no key)
#pragma unroll
        for (uint32_t bit = 1u << 31; bit >= 1u << 12; bit >>= 1)
            if (const uint32_t to = (bound & ~1u) | bit; __popcll(__ballot(head >= to)) >= C.top_k) bound = to;
        for (int i = threadIdx.x; i < n; i += T) {
            const uint64_t key = all[i];
            if ((uint32_t)(key >> 32) < bound) continue;
            const int at = atomicAdd(&candidates, 1);  // (in any order: their places are their own)
            if (at < kCandidates) keys[at / kWave][at % kWave] = key;
        }
        __syncthreads();
        const int found = candidates;
        const uint64_t* list = &keys[0][0];
        if (found >= C.top_k && found <= kCandidates) {
            if ((int)threadIdx.x >= found) return;
            const uint64_t mine = list[threadIdx.x];
            int place = 0;
#pragma unroll 4
            for (int i = 0; i < found; ++i) place += list[i] > mine;
            store_likeliest(C, row, s, f.ln, mine, place);
            return;
        }
        __syncthreads();
        uint64_t mine = 0;
        for (int i = wave; i < P.segments; i += T / kWave) mine = merge_keys(mine, lane < C.top_k ? all[(int64_t)i * C.top_k + lane] : 0, lane);
        mine = merge_waves<T>(mine, keys, lane, wave);
        if (wave == 0)
            store_likeliest(C, row, s, f.ln, fill<VT>(mine, s, (const value_store_t<VT>*)C.logits + row * C.V, C.V, C.top_k, lane, keys[0]), lane);
    }
}

template <int VT, bool DISTILL>
__global__ void __launch_bounds__(kThreads) class_gradient_kernel(ClassCall C, Parts P)
{
    constexpr int T = kThreads;
    __shared__ Sums room[T / kWave];
    __shared__ std::conditional_t<DISTILL, Entries, int> entries;
    const int64_t row = blockIdx.x / P.segments;
    const int segment = blockIdx.x % P.segments, first = segment * P.width, last = min(first + P.width, C.V);
    // (x of other segments may have been overwritten: of the entries only those of this one are used)
    FewEntries<VT> few;
    if constexpr (DISTILL) {
        if (threadIdx.x < kWave) {
            if (C.k <= kFewEntries) few.ask(C, row, threadIdx.x);
            else take_more_entries<VT>(C, row, threadIdx.x, entries);
        }
    }
    const Sums s = join_segments<T>(C, P, row, room);
    const Asked asked = P.asked[row];
    const Given given = row_given(C, row);
    const Found f = row_results(C, given, s, asked);
    if (segment == 0 && threadIdx.x == 0) store_results(C, row, f);
    const Slope k = row_slope(C, given, s, asked, f);
    if constexpr (DISTILL)
        store_gradient<VT, T, true>(C, row, first, last, s, k, &entries, [&] {
            if (threadIdx.x < kWave && C.k <= kFewEntries) few.take(C, threadIdx.x, true, entries);
        });
    else store_gradient<VT, T, false>(C, row, first, last, s, k, nullptr, kNothing);
}

// Threads of a workgroup that has a row.  The gradient reads its rows again: those that all CUs work on at a time have to stay in the Infinity Cache.
template <int VT>
int threads_of(int V)
{
    const double of_256 = 256.0 * 8 * V * sizeof(value_store_t<VT>), most = 128.0 * (1 << 20);
    return of_256 <= most ? 256 : of_256 <= 2 * most ? 512 : 1024;
}

// Segments of a row
struct Cut { int segments, width; };
constexpr int kLeastSegment = kThreads * kRowUnit;
constexpr int kFewRows = 128;        // fewer are cut
constexpr int kRowsOf1024 = 512;     // of rows that are not held, up to so many have 1024 threads each,
constexpr int kRowsOf512 = 1024;     // up to so many 512
Cut cut_of(int64_t N, int V)
{
    constexpr int kGroups = 512;
    if (N >= kFewRows || V < 8 * kLeastSegment) return {1, V};
    const int most = (V + kLeastSegment - 1) / kLeastSegment, wanted = (int)((kGroups + N - 1) / std::max<int64_t>(N, 1));
    const int per = (most + std::min(most, wanted) - 1) / std::min(most, wanted);
    return {(most + per - 1) / per, per * kLeastSegment};
}

int64_t up16(int64_t n) { return (n + 15) & ~15ll; }

template <int VT, int L, int U, bool DISTILL, bool GRAD, bool TOP>
maxk_status run_teams(const ClassCall& C, hipStream_t s)
{
    constexpr int kTeams = kThreads / L;
    hipLaunchKernelGGL((class_team_kernel<VT, L, U, DISTILL, GRAD, TOP>), groups_of((C.N + kTeams - 1) / kTeams), dim3(kThreads), 0, s, C);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <int VT, int T, int U, bool DISTILL, bool GRAD, bool TOP>
maxk_status run_held(const ClassCall& C, hipStream_t s)
{
    hipLaunchKernelGGL((class_held_kernel<VT, T, U, DISTILL, GRAD, TOP>), groups_of(C.N), dim3(T), 0, s, C);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <int VT, int T, bool DISTILL, bool GRAD, bool TOP>
maxk_status run_rows(const ClassCall& C, hipStream_t s)
{
    hipLaunchKernelGGL((class_rows_kernel<VT, T, DISTILL, GRAD, TOP>), groups_of(C.N), dim3(T), 0, s, C);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

// Rows for two such workgroups on a CU; fewer are better off with lanes that share a row.  us, a lane a row / eight lanes, 47 fp32 with 5 alternatives: 1024 rows 8.2 /
// 4.6, 20 k 10.7 / 5.6, 100 k 15.1 / 13.6, 300 k 26.6 / 31.8, 2.4 M 171 / 259
constexpr int kManyRows = 2 * 256 * kThreads;
template <int VT, int K>
maxk_status run_lane_rows(const ClassCall& C, hipStream_t s)
{
    hipLaunchKernelGGL((class_lane_kernel<VT, K>), groups_of((C.N + kThreads - 1) / kThreads), dim3(kThreads), kThreads * lane_row_pitch(C.V) * sizeof(float), s, C);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

// Where rows leave a quarter and more of a team's columns idle (distillation: an eighth) and there are many of them.  us, a lane a row / a team, 2.45 M rows, log
// probabilities and gradient: 9 bf16 32 / 60, 17 48 / 60, 33 87 / 118, 47 123 / 139 (alone, without a gradient, 59 / 83), 47 fp32 184 / 240; 32 bf16 87 / 64, 56 143 / 127,
// 64 162 / 130; 600 k rows: 9 11 / 18, 33 27 / 32, 41 33 / 33; 170 k: 47 16 / 13.  Distillation, 5 entries: 9 bf16 56 / 127, 33 130 / 207, 47 171 / 223, fp32 219 / 269, 24 137 /
// 180, 48 217 / 248; 56 256 / 258, 64 290 / 265; 524 k rows: 33 34 / 48, 47 49 / 55.  (More entries, which a lane cannot hold, from LDS: 16 of 47 bf16 376 / 313.)
constexpr int kManyOwnRows = 1 << 19;
bool own_rows(int64_t N, int V, int eighths) { return N >= kManyOwnRows && V >= kLaneRowLeast && 8 * V < eighths * (V <= 4 * kRowUnit ? 4 : 8) * kRowUnit; }
template <int VT, bool DISTILL, bool GRAD, bool ENTROPY>
maxk_status run_own_rows(const ClassCall& C, hipStream_t s)
{
    const Stretch R = Stretch::of(C.V, sizeof(value_store_t<VT>));
    hipLaunchKernelGGL((class_own_kernel<VT, DISTILL, GRAD, ENTROPY>), groups_of((C.N + kThreads - 1) / kThreads), dim3(kThreads), R.room(), s, C, R);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <int VT, bool DISTILL, bool GRAD, bool TOP>
maxk_status run_classes(const ClassCall& C, void* workspace, hipStream_t s)
{
    if constexpr (TOP)
        if (const int keys = C.top_k + (VT == MAXK_VALUE_F32); C.V <= kLaneRowMost && keys <= kLaneRowKeys && C.N >= kManyRows) {
            if (keys <= 2) return run_lane_rows<VT, 2>(C, s);
            if (keys <= 4) return run_lane_rows<VT, 4>(C, s);
            if (keys <= 6) return run_lane_rows<VT, 6>(C, s);
            return run_lane_rows<VT, kLaneRowKeys>(C, s);
        }
    if constexpr (!TOP)
        if (own_rows(C.N, C.V, DISTILL ? 7 : 6) && (!DISTILL || C.k <= kOwnEntries)) {
            if constexpr (!DISTILL)
                if (C.entropy || C.dentropy) return run_own_rows<VT, DISTILL, GRAD, true>(C, s);
            return run_own_rows<VT, DISTILL, GRAD, false>(C, s);
        }
    const int units = (C.V + kRowUnit - 1) / kRowUnit;
    if (units <= 4) return run_teams<VT, 4, 1, DISTILL, GRAD, TOP>(C, s);
    if (units <= 8) return run_teams<VT, 8, 1, DISTILL, GRAD, TOP>(C, s);
    if (units <= 16) return run_teams<VT, 16, 1, DISTILL, GRAD, TOP>(C, s);
    if (units <= 32) return run_teams<VT, 32, 1, DISTILL, GRAD, TOP>(C, s);
    if (units <= 64) return run_teams<VT, 64, 1, DISTILL, GRAD, TOP>(C, s);
    if (units <= 128) return run_teams<VT, 64, 2, DISTILL, GRAD, TOP>(C, s);
    if (units <= 256) return run_teams<VT, 64, 4, DISTILL, GRAD, TOP>(C, s);
    // Held and read once, or gone through twice?  us, held / gone through:
    //   gradient (forward alone)                                       alternatives        5        20        24        50
    //   40000 x 2500   bf16 104 (64) / 153 (99)  fp32 149 (66) / 172 (100)   16000 x 2500   bf16  53 / 67   60 / 87   61 / 93   70 / 146
    //   24396 x 4099   bf16  88 (54) / 124 (75)                               9800 x 4099   bf16  40 / 44   46 / 56   47 / 59   52 / 89
    //   12207 x 8192   bf16  75 (43) /  87 (44)  fp32 143      / 178          5000 x 8192   bf16  28 / 31   32 / 45   33 / 50   37 / 73
    //     243 x 4099          4      /   6                                    (fp32 the same or more in favour of held)
    // with 512 threads:
    //    7142 x 14000  bf16  83 (42) /  95 (39)  fp32 145 (68) / 190 (69)     4444 x 9000   bf16  51 / 32   55 / 47   56 / 51   60 / 73   fp32  54 / 44   58 / 57   59 / 60   62 / 88
    //     365 x 8200          7  (5) /  12  (8)                               2857 x 14000  bf16  39 / 30   43 / 43   43 / 44   46 / 64   fp32  43 / 44   47 / 52   47 / 55   50 / 76
    // with 1024 threads: 3571 x 28000 bf16, gradient, 125 / 101.
    if (units <= 512) return run_held<VT, 256, 2, DISTILL, GRAD, TOP>(C, s);
    if (units <= 768) return run_held<VT, 256, 3, DISTILL, GRAD, TOP>(C, s);
    if (units <= 1024) return run_held<VT, 256, 4, DISTILL, GRAD, TOP>(C, s);
    const Cut cut = cut_of(C.N, C.V);
    if (cut.segments == 1 && (GRAD || C.N <= kRowsOf1024 || C.top_k >= 24)) {
        if (units <= 1536) return run_held<VT, 512, 3, DISTILL, GRAD, TOP>(C, s);
        if (units <= 2048) return run_held<VT, 512, 4, DISTILL, GRAD, TOP>(C, s);
    }
    if (cut.segments == 1) {
        const int T = C.N <= kRowsOf1024 ? 1024 : C.N <= kRowsOf512 ? 512 : GRAD ? threads_of<VT>(C.V) : kThreads;
        if (T == 1024) return run_rows<VT, 1024, DISTILL, GRAD, TOP>(C, s);
        if (T == 512) return run_rows<VT, 512, DISTILL, GRAD, TOP>(C, s);
        return run_rows<VT, kThreads, DISTILL, GRAD, TOP>(C, s);
    }
    char* at = (char*)workspace;
    Parts P = {cut.segments, cut.width, (Sums*)at, nullptr, nullptr};
    at += up16(C.N * cut.segments * (int64_t)sizeof(Sums));
    P.asked = (Asked*)at;
    at += up16(C.N * (int64_t)sizeof(Asked));
    P.keys = (uint64_t*)at;
    const unsigned groups = (unsigned)(C.N * cut.segments);
    hipLaunchKernelGGL((class_parts_kernel<VT, DISTILL, TOP>), dim3(groups), dim3(kThreads), 0, s, C, P);
    MAXK_LAUNCH_CHECK();
    if constexpr (GRAD) hipLaunchKernelGGL((class_gradient_kernel<VT, DISTILL>), dim3(groups), dim3(kThreads), 0, s, C, P);
    else hipLaunchKernelGGL((class_join_kernel<VT, TOP ? 1024 : kThreads, TOP>), dim3((unsigned)C.N), dim3(TOP ? 1024 : kThreads), 0, s, C, P);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <int VT>
maxk_status run_type(const ClassCall& C, void* workspace, hipStream_t s)
{
    if (C.index) return C.dlogits ? run_classes<VT, true, true, false>(C, workspace, s) : run_classes<VT, true, false, false>(C, workspace, s);
    if (C.dlogits) return run_classes<VT, false, true, false>(C, workspace, s);
    return C.top_data ? run_classes<VT, false, false, true>(C, workspace, s) : run_classes<VT, false, false, false>(C, workspace, s);
}

}  // namespace

int64_t classes_workspace(int64_t N, int32_t V, int32_t top_k)
{
    const Cut cut = cut_of(N, V);
    if (cut.segments == 1) return 0;
    return up16(N * cut.segments * (int64_t)sizeof(Sums)) + up16(N * (int64_t)sizeof(Asked)) + N * cut.segments * (int64_t)top_k * 8;
}

maxk_status launch_classes(const ClassCall& C, int value_type, void* workspace, hipStream_t s)
{
    if (value_type == MAXK_VALUE_F32) return run_type<MAXK_VALUE_F32>(C, workspace, s);
    if (value_type == MAXK_VALUE_BF16) return run_type<MAXK_VALUE_BF16>(C, workspace, s);
    return run_type<MAXK_VALUE_F16>(C, workspace, s);
}

}  // namespace maxk
