// Input gradient of the linear map with 4-bit weights (include/maxk.h): dX = dH W.
//
// On bf16 matrix instructions with fp32 accumulators.  W is exact in bf16, and a gradient is cut into bf16 parts that add up to it
// exactly (fp32 three, fp16 two), so every product is exact and only the sums round.  A wavefront keeps the columns of dX that are its own,
// 32 * IT of them, as rows of W in its registers and walks over tiles of 32 rows of dH, which the four wavefronts of a group bring to LDS
// together: a CBSR gradient as its k values a row, spread over zeros.  A workgroup has two groups; one fills its tile while the other multiplies.
#include <algorithm>
#include <type_traits>

#include "mx_parts.hpp"

namespace maxk {
namespace {

constexpr int kRows = 32;  // of a tile

// KC steps of 16 columns of dH in registers and LDS, IT x 32 columns of dX a wavefront, WI wavefronts a group, GR groups
template <int KC_, int IT_, int WI_, int GR_>
struct Shape {
    static constexpr int KC = KC_, IT = IT_, WI = WI_, GR = GR_, THREADS = 64 * WI * GR, SPAN = 32 * IT * WI;
    static constexpr int ROWS = kRows / WI;                 // rows of a tile that a wavefront brings
    static constexpr int UNITS = ROWS * 2 * KC / 64;        // units of 8 columns of them a lane brings
};

// Dense gradients in 16-byte pieces (V) or element by element.
enum Kind { kCbsr1, kCbsr2, kCbsr4, kF32, kF32V, kBf16, kBf16V, kF16, kF16V };  // CBSR: by the bytes of a column
__host__ __device__ constexpr int type_of(int kind) { return kind <= kF32V ? MAXK_VALUE_F32 : kind <= kBf16V ? MAXK_VALUE_BF16 : MAXK_VALUE_F16; }
__host__ __device__ constexpr int parts_of(int kind) { return kind <= kF32V ? 3 : kind <= kBf16V ? 1 : 2; }

template <int KIND> using column_t = std::conditional_t<KIND == kCbsr1, uint8_t, std::conditional_t<KIND == kCbsr2, uint16_t, uint32_t>>;


struct Args {
    MxGrad G;
    int64_t N;
    MxMatrix W;
    int din, dout, nb, spans, chunks;
    int64_t slots;  // workgroups that walk
    void* dX;
    int dx_type;
    bool pairs;  // two neighbouring columns of dX in one store
};

// CHUNKED: dH is wider than a tile, which takes it in chunks (W comes anew with each)
// E: CBSR entries of its rows that a lane has under way; those of wider rows come in turns
template <class S, int KIND, int E, bool CHUNKED>
__global__ void __launch_bounds__(S::THREADS) input_grad_kernel(const Args A)
{
    constexpr int P = parts_of(KIND), VT = type_of(KIND), PART = kRows * S::KC * 32, TILE = P * PART;
    __shared__ __align__(16) uint8_t lds[S::GR * TILE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave / S::WI, w = wave % S::WI;
    // the spans of a slot run on one XCD, whose L2 holds the rows that they share
    const int at = blockIdx.x / 8, span = at % A.spans;
    const int64_t slot = (int64_t)(at / A.spans) * 8 + blockIdx.x % 8;
    if (slot >= A.slots) return;
    const int64_t tiles = (A.N + kRows - 1) / kRows, stride = A.slots * S::GR;
    const int64_t rounds = (tiles - slot * S::GR + stride - 1) / stride;  // of the first group; the others may have one tile less
    const int i0 = span * S::SPAN + w * 32 * S::IT, l = lane & 31, h = lane >> 5;
    uint8_t* const tile = lds + group * TILE;
    // a unit is 8 columns (a run) of a row; rows lie within a run, in an order in which the runs of a row fall on different banks
    const auto unit_at = [](int run, int row) { return (run * kRows + (row ^ (run & 7))) * 16; };

    bf16x8 weight[S::KC][S::IT];
    const auto load_weights = [&](int chunk) {
        const int i = min(i0 + l * S::IT, A.din - 1);  // IT == 2: a byte has both columns
#pragma unroll
        for (int s = 0; s < S::KC; ++s) {
            float x[8][2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // columns o of dH (rows of W): a for the lower lanes, b for the upper ones; the same for all of them, so addresses are scalar
                const int o = (chunk * S::KC + s) * 16 + j, a = min(o, A.dout - 1), b = min(o + 8, A.dout - 1);
                const uint8_t* codes = A.W.codes + (int64_t)a * A.nb * 16;
                const uint8_t* scales = A.W.scales + (int64_t)a * A.nb;
                const uint32_t code = codes[(uint32_t)((h ? (b - a) * A.nb * 16 : 0) + i / 2)];
                const auto two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, mx_scale(scales[(uint32_t)((h ? (b - a) * A.nb : 0) + i / kMxBlock)]), 0);
                const bool there = o + (h ? 8 : 0) < A.dout;
                x[j][0] = there ? (S::IT == 2 || !(i & 1) ? two[0] : two[1]) : 0.f;
                x[j][1] = there ? two[1] : 0.f;
            }
#pragma unroll
            for (int t = 0; t < S::IT; ++t) {
                uint4 u = make_uint4(uppers(x[0][t], x[1][t]), uppers(x[2][t], x[3][t]), uppers(x[4][t], x[5][t]), uppers(x[6][t], x[7][t]));
                asm("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));  // made here: put off to their use, all bytes and scales would be kept instead
                weight[s][t] = __builtin_bit_cast(bf16x8, u);
            }
            __builtin_amdgcn_sched_barrier(0);  // 16 loads under way, not all of them: they would not fit
        }
    };

    const int k = A.G.k;
    int erow[E];
    if constexpr (KIND <= kCbsr4) {
#pragma unroll
        for (int e = 0; e < E; ++e) erow[e] = (lane + 64 * e) / k;
    }
    constexpr int VALS = KIND <= kCbsr4 ? E : VT == MAXK_VALUE_F32 || KIND == kBf16 || KIND == kF16 ? S::UNITS * 8 : S::UNITS * 4;
    float val[VALS];  // 16-byte pieces of 16-bit values: two to a register
    uint32_t idx[KIND <= kCbsr4 ? E : 1];
    const auto load = [&](int64_t t, int chunk) {
        const int64_t row0 = min(t, tiles - 1) * kRows;
        const int lim = (int)min(A.N - 1 - row0, (int64_t)kRows - 1);  // rows past the last one are read from it; what they give is not stored
        if constexpr (KIND <= kCbsr4) {
            const int end = (lim + 1) * k - 1;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t p = (uint32_t)min(w * S::ROWS * k + lane + 64 * e, end);
                val[e] = ((const float*)A.G.values + row0 * k)[p];
                idx[e] = ((const column_t<KIND>*)A.G.sp_index + row0 * k)[p];
            }
        } else {
#pragma unroll
            for (int u = 0; u < S::UNITS; ++u) {
                const int unit = lane + 64 * u, run = unit % (2 * S::KC), row = min(w * S::ROWS + unit / (2 * S::KC), lim), o = (chunk * S::KC * 2 + run) * 8;
                const value_store_t<VT>* values = (const value_store_t<VT>*)A.G.values + row0 * A.dout;
                const int p = row * A.dout;
                if constexpr (KIND == kF32V) {
                    *reinterpret_cast<f32x4*>(val + u * 8) = *reinterpret_cast<const f32x4*>(values + (uint32_t)(p + min(o, A.dout - 4)));
                    *reinterpret_cast<f32x4*>(val + u * 8 + 4) = *reinterpret_cast<const f32x4*>(values + (uint32_t)(p + min(o + 4, A.dout - 4)));
                } else if constexpr (KIND == kBf16V || KIND == kF16V) {
                    *reinterpret_cast<f32x4*>(val + u * 4) = *reinterpret_cast<const f32x4*>(values + (uint32_t)(p + min(o, A.dout - 8)));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const value_store_t<VT> x = values[(uint32_t)(p + min(o + j, A.dout - 1))];
                        if constexpr (KIND == kF32) val[u * 8 + j] = x;
                        else val[u * 8 + j] = __uint_as_float(x);  // widened when it is used
                    }
                }
            }
        }
    };
    const auto fill = [&](int64_t t, int chunk) {
        if constexpr (KIND <= kCbsr4) {
            // a wavefront's rows are its own, zeros and entries: its LDS operations stay in order
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int u = 0; u < S::UNITS; ++u) {
                    const int unit = lane + 64 * u;
                    *reinterpret_cast<uint4*>(tile + p * PART + unit_at(unit / S::ROWS, w * S::ROWS + unit % S::ROWS)) = make_uint4(0, 0, 0, 0);
                }
            wave_fence();
            const auto put = [&](int row, uint32_t column, float x) {
                const uint32_t o = column - (uint32_t)(chunk * S::KC * 16);
                if (o < (uint32_t)(S::KC * 16)) {
                    float part[3];
                    split<P>(x, part);
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        *reinterpret_cast<uint16_t*>(tile + p * PART + unit_at((int)o / 8, row) + (o & 7) * 2) = (uint16_t)(__float_as_uint(part[p]) >> 16);
                }
            };
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (erow[e] < S::ROWS) put(w * S::ROWS + erow[e], idx[e], val[e]);
            const int64_t row0 = min(t, tiles - 1) * kRows;
            const int end = min(((int)min(A.N - row0, (int64_t)kRows) - w * S::ROWS) * k, S::ROWS * k) - 1;
            for (int e0 = 64 * E; e0 <= end; e0 += 64 * E) {
                const int64_t mine = (row0 + w * S::ROWS) * k;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t p = (uint32_t)min(e0 + lane + 64 * e, end);
                    val[e] = ((const float*)A.G.values + mine)[p];
                    idx[e] = ((const column_t<KIND>*)A.G.sp_index + mine)[p];
                }
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e0 + lane + 64 * e <= end) put(w * S::ROWS + (e0 + lane + 64 * e) / k, idx[e], val[e]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < S::UNITS; ++u) {
                const int unit = lane + 64 * u, run = unit % (2 * S::KC), row = w * S::ROWS + unit / (2 * S::KC), o = (chunk * S::KC * 2 + run) * 8;
                float part[8][3];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float x;
                    if constexpr (KIND == kBf16V || KIND == kF16V) x = widen_value<VT>((uint16_t)(__float_as_uint(val[u * 4 + j / 2]) >> (16 * (j & 1))));
                    else if constexpr (KIND == kF32 || KIND == kF32V) x = val[u * 8 + j];
                    else x = widen_value<VT>((uint16_t)__float_as_uint(val[u * 8 + j]));
                    split<P>(o + j < A.dout ? x : 0.f, part[j]);
                }
#pragma unroll
                for (int p = 0; p < P; ++p)
                    *reinterpret_cast<uint4*>(tile + p * PART + unit_at(run, row)) =
                        make_uint4(uppers(part[0][p], part[1][p]), uppers(part[2][p], part[3][p]), uppers(part[4][p], part[5][p]), uppers(part[6][p], part[7][p]));
            }
        }
    };

    f32x16 sum[S::IT];
    const auto clear = [&]() {
#pragma unroll
        for (int t = 0; t < S::IT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[t][r] = 0.f;
    };
    const auto multiply = [&]() {
        // operands from LDS a few steps ahead of the products that need them, and no further: registers are full of weights
        constexpr int AHEAD = P * S::IT >= 6 ? 1 : P * S::IT >= 3 ? 2 : 4;
        bf16x8 d[AHEAD + 1][P];
        const auto fetch = [&](int s) {
#pragma unroll
            for (int p = 0; p < P; ++p) d[s % (AHEAD + 1)][p] = *reinterpret_cast<const bf16x8*>(tile + p * PART + unit_at(2 * s + h, l));
        };
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) fetch(s);
#pragma unroll
        for (int s = 0; s < S::KC; ++s) {
            if (s + AHEAD < S::KC) fetch(s + AHEAD);
#pragma unroll
            for (int p = P - 1; p >= 0; --p)
#pragma unroll
                for (int t = 0; t < S::IT; ++t) sum[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d[s % (AHEAD + 1)][p], weight[s][t], sum[t], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto store = [&](int64_t t) {
        const int i = i0 + l * S::IT;
        if (t >= tiles || i >= A.din) return;
        const int64_t row0 = t * kRows;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t row = row0 + 8 * (r / 4) + 4 * h + r % 4;
            if (row >= A.N) continue;
            const int64_t at = row * A.din + i;
            if (A.dx_type == MAXK_VALUE_F32) {
                float* p = (float*)A.dX + at;
                if (S::IT == 2 && A.pairs) *reinterpret_cast<float2*>(p) = make_float2(sum[0][r], sum[S::IT - 1][r]);
                else {
                    p[0] = sum[0][r];
                    if (S::IT == 2 && i + 1 < A.din) p[1] = sum[S::IT - 1][r];
                }
            } else {
                const bool bf = A.dx_type == MAXK_VALUE_BF16;
                const uint16_t a = bf ? narrow_value<MAXK_VALUE_BF16>(sum[0][r]) : narrow_value<MAXK_VALUE_F16>(sum[0][r]);
                const uint16_t b = bf ? narrow_value<MAXK_VALUE_BF16>(sum[S::IT - 1][r]) : narrow_value<MAXK_VALUE_F16>(sum[S::IT - 1][r]);
                uint16_t* p = (uint16_t*)A.dX + at;
                if (S::IT == 2 && A.pairs) *reinterpret_cast<uint32_t*>(p) = (uint32_t)a | (uint32_t)b << 16;
                else {
                    p[0] = a;
                    if (S::IT == 2 && i + 1 < A.din) p[1] = b;
                }
            }
        }
    };

    int64_t t = slot * S::GR + group;
    load(t, 0);
    load_weights(0);
    if (S::GR > 1 && (group & 1)) local_fence();  // half a round behind the other group
    for (int64_t round = 0; round < rounds; ++round, t += stride) {
        clear();
        for (int chunk = 0; chunk < (CHUNKED ? A.chunks : 1); ++chunk) {
            fill(t, chunk);
            local_fence();
            if (CHUNKED && chunk + 1 < A.chunks) load(t, chunk + 1);
            else load(t + stride, 0);
            multiply();
            if constexpr (CHUNKED) load_weights(chunk + 1 < A.chunks ? chunk + 1 : 0);
            if (!CHUNKED || chunk + 1 == A.chunks) store(t);
            local_fence();
        }
    }
    if (S::GR > 1 && !(group & 1)) local_fence();
}

template <class S, int KIND, int E, bool CHUNKED = false>
maxk_status run(Args A, hipStream_t s)
{
    A.spans = (A.din + S::SPAN - 1) / S::SPAN;
    A.chunks = (A.dout + 16 * S::KC - 1) / (16 * S::KC);
    const int64_t tiles = (A.N + kRows - 1) / kRows;
    A.slots = std::max<int64_t>(1, std::min((tiles + S::GR - 1) / S::GR, (int64_t)512 / A.spans));
    const int64_t grid = (A.slots + 7) / 8 * A.spans * 8;
    hipLaunchKernelGGL((input_grad_kernel<S, KIND, E, CHUNKED>), dim3((unsigned)grid), dim3(S::THREADS), 0, s, A);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <int KIND, int E = 1>
maxk_status run_kind(const Args& A, hipStream_t s)
{
    const bool two = A.din > 128;  // columns of dX that four wavefronts hold, 32 each
    if (A.dout <= 64) return two ? run<Shape<4, 2, 4, 2>, KIND, E>(A, s) : run<Shape<4, 1, 4, 2>, KIND, E>(A, s);
    if (A.dout <= 128) return two ? run<Shape<8, 2, 4, 2>, KIND, E>(A, s) : run<Shape<8, 1, 4, 2>, KIND, E>(A, s);
    if (A.dout <= 256) return two ? run<Shape<16, 2, 4, 2>, KIND, E>(A, s) : run<Shape<16, 1, 4, 2>, KIND, E>(A, s);
    if (A.dout <= 512) return run<Shape<32, 1, 8, 1>, KIND, E>(A, s);
    return run<Shape<16, 2, 4, 2>, KIND, E, true>(A, s);
}

}  // namespace

maxk_status launch_mx_input_grad(const MxGrad& G, int64_t N, const MxMatrix& W, int din, int dout, void* dX, int value_type, hipStream_t s)
{
    const size_t xb = value_type == MAXK_VALUE_F32 ? 4 : 2, gb = G.value_type == MAXK_VALUE_F32 ? 4 : 2;
    const Args A = {G, N, W, din, dout, mx_blocks(din), 0, 0, 0, dX, value_type, din % 2 == 0 && aligned(dX, 2 * xb)};
#define MAXK_ENTRIES(KIND) (G.k <= 32 ? run_kind<KIND, 4>(A, s) : run_kind<KIND, 8>(A, s))
    if (G.k) return G.index_bytes == 1 ? MAXK_ENTRIES(kCbsr1) : G.index_bytes == 2 ? MAXK_ENTRIES(kCbsr2) : MAXK_ENTRIES(kCbsr4);
#undef MAXK_ENTRIES
    const bool pieces = dout * gb % 16 == 0 && aligned(G.values, 16);
    if (G.value_type == MAXK_VALUE_F32) return pieces ? run_kind<kF32V>(A, s) : run_kind<kF32>(A, s);
    if (G.value_type == MAXK_VALUE_BF16) return pieces ? run_kind<kBf16V>(A, s) : run_kind<kBf16>(A, s);
    return pieces ? run_kind<kF16V>(A, s) : run_kind<kF16>(A, s);
}

}  // namespace maxk
