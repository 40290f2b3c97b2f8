// Input gradient of the linear map with 4-bit weights (include/maxk.h): dX = dH W.
//
// On bf16 matrix instructions with fp32 accumulators.  W is exact in bf16, and a gradient is cut into bf16 parts that add up to it
// exactly (fp32 three, fp16 two; mx_parts.hpp), so every product is exact and only the sums round.  A wavefront has 32 * IT columns of dX: it keeps those columns of W in
// its registers and walks over tiles of 32 rows of dH, which the four wavefronts of a group bring to LDS together: a CBSR gradient as its k values a
// row, spread over zeros.  A workgroup has two groups; one fills its tile while the other multiplies.
//
// Bound by the way to memory where dH is dense (169 thousand rows, 256 x 256, fp32: 75 us, 4.6 TB/s, 59 to 65 with dH in the Infinity Cache; bf16 38, 4.5 TB/s; fp16 46), by the
// three parts' products beside the stores of dX where it is CBSR (233 thousand, k = 32: 63 to 72 us by the card's clock; the products alone 37, the stores 43).  Dense rows that
// are not whole 16-byte pieces come element by element: bf16 dH of 255 columns 150 us.
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

struct Args {
    MxGrad G;
    int64_t N;
    MxMatrix W;
    int din, dout, nb, spans, chunks;
    int64_t slots;  // workgroups that walk
    void* dX;
    int dx_type;
    bool pairs;  // two neighbouring columns of dX in one store
    bool once;   // dX passes by L2
};

// CHUNKED: dH is wider than a tile, which takes it in chunks (W comes anew with each)
// E: CBSR entries of its rows that a lane has under way; those of wider rows come in turns
template <class S, int KIND, int E, bool CHUNKED>
__global__ void __launch_bounds__(S::THREADS) input_grad_kernel(const Args A)
{
    static_assert(!CHUNKED || S::GR == 1);  // W comes by way of the tiles
    constexpr bool CBSR = KIND <= kCbsr4;
    constexpr int P = parts_of(KIND), VT = type_of(KIND), VB = VT == MAXK_VALUE_F32 ? 4 : 2, PART = kRows * S::KC * 32, TILE = P * PART;
    constexpr int LDS = S::GR * TILE > S::THREADS * 32 ? S::GR * TILE : S::THREADS * 32;  // 16 values of W a thread at least
    __shared__ __align__(16) uint8_t lds[LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave / S::WI, w = wave % S::WI;
    // the spans of a slot run on one XCD, whose L2 holds the rows that they share
    const int at = blockIdx.x / 8, span = at % A.spans;
    const int64_t slot = (int64_t)(at / A.spans) * 8 + blockIdx.x % 8;
    if (slot >= A.slots) return;
    const int64_t tiles = (A.N + kRows - 1) / kRows, stride = A.slots * S::GR;
    const int64_t rounds = (tiles - slot * S::GR + stride - 1) / stride;  // of the first group; the others may have one tile less
    const int s0 = span * S::SPAN, l = lane & 31, h = lane >> 5;
    uint8_t* const tile = lds + group * TILE;
    // a unit is 8 columns (a run) of a row; rows lie within a run, in an order in which the runs of a row fall on different banks
    const auto unit_at = [](int run, int row) { return (run * kRows + (row ^ (run & 7))) * 16; };

    // Rows of W (columns of dH) come to LDS in bf16, as many at a time as it holds, and are read transposed: a lane's operand is 8 of them in one
    // column of dX.  With IT == 2 a wavefront's even columns come before its odd ones, so that a lane has two neighbours.
    bf16x8 weight[S::KC][S::IT];
    const auto load_weights = [&](int chunk) {
        constexpr int PITCH = S::SPAN * 2, PIECES = S::SPAN / 16, STEP = S::THREADS / PIECES, ITEMS = S::KC * 16 / STEP;  // pieces of 16 columns
        constexpr int PASS = LDS / PITCH / STEP * STEP < S::KC * 16 ? LDS / PITCH / STEP * STEP : S::KC * 16;             // rows at a time
        static_assert(S::THREADS % PIECES == 0 && S::KC * 16 % STEP == 0 && STEP % 16 == 0 && PASS >= STEP);
        const int piece = threadIdx.x % PIECES, row0 = threadIdx.x / PIECES, col = min(s0 + piece * 16, A.nb * kMxBlock - 16);
        uint2 code[ITEMS];
        uint32_t scale[ITEMS];
#pragma unroll
        for (int n = 0; n < ITEMS; ++n) {
            const int64_t row = min(chunk * S::KC * 16 + row0 + n * STEP, A.dout - 1);
            code[n] = *reinterpret_cast<const uint2*>(A.W.codes + (row * A.nb * 16 + col / 2));
            scale[n] = A.W.scales[row * A.nb + col / kMxBlock];
        }
#pragma unroll
        for (int pass = 0; pass < (S::KC * 16 + PASS - 1) / PASS; ++pass) {
            if (pass) local_fence();
#pragma unroll
            for (int n = pass * PASS / STEP; n < (pass + 1) * PASS / STEP && n < ITEMS; ++n) {
                const int row = row0 + n * STEP, r = row - pass * PASS;
                const bool there = chunk * S::KC * 16 + row < A.dout;
                const float unit = mx_scale(scale[n]);
                uint32_t x[8];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t c = there ? (j ? code[n].y : code[n].x) : 0u;
                    const float u = there ? unit : 1.f;
                    x[4 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, u, 0));
                    x[4 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, u, 1));
                    x[4 * j + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, u, 2));
                    x[4 * j + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, u, 3));
                }
                if constexpr (S::IT == 2) {
                    uint32_t even[4], odd[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        even[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
                        odd[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
                    }
                    const int byte = piece / 4 * 128 + piece % 4 * 16;  // a wavefront has four pieces
                    *reinterpret_cast<uint4*>(lds + at_byte(r, byte, PITCH)) = make_uint4(even[0], even[1], even[2], even[3]);
                    *reinterpret_cast<uint4*>(lds + at_byte(r, byte + 64, PITCH)) = make_uint4(odd[0], odd[1], odd[2], odd[3]);
                } else {
                    uint4* to = reinterpret_cast<uint4*>(lds + at_byte(r, piece * 32, PITCH));
                    to[0] = make_uint4(x[0], x[1], x[2], x[3]);
                    to[1] = make_uint4(x[4], x[5], x[6], x[7]);
                }
            }
            local_fence();
#pragma unroll
            for (int s = pass * PASS / 16; s < (pass + 1) * PASS / 16 && s < S::KC; ++s)
#pragma unroll
                for (int t = 0; t < S::IT; ++t) weight[s][t] = transposed_operand(lds, PITCH, w * S::IT + t, (s - pass * PASS / 16) * 16, lane);
        }
        local_fence();
    };

    const int k = A.G.k;
    int erow[E];
    if constexpr (CBSR) {
#pragma unroll
        for (int e = 0; e < E; ++e) erow[e] = (lane + 64 * e) / k;
    }
    constexpr int VALS = CBSR ? E : VT == MAXK_VALUE_F32 || KIND == kBf16 || KIND == kF16 ? S::UNITS * 8 : S::UNITS * 4;
    uint32_t val[VALS];  // 16-byte pieces of 16-bit values: two to a register
    uint32_t idx[CBSR ? E : 1];
    // rows of the tile that are there; what is read past them is 0
    const auto rows_of = [&](int64_t t) { return (int)max((int64_t)0, min(A.N - t * kRows, (int64_t)kRows)); };
    const auto load = [&](int64_t t, int chunk) {
        const int64_t row0 = min(t, tiles - 1) * kRows;
        if constexpr (CBSR) {
            constexpr int IB = sizeof(column_t<KIND>);
            const int entries = rows_of(t) * k, first = w * S::ROWS * k + lane;
            const auto values = buffer_of((const float*)A.G.values + row0 * k, entries * 4), columns = buffer_of((const column_t<KIND>*)A.G.sp_index + row0 * k, entries * IB);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                val[e] = __builtin_amdgcn_raw_buffer_load_b32(values, (first + 64 * e) * 4, 0, 0);
                if constexpr (IB == 1) idx[e] = __builtin_amdgcn_raw_buffer_load_b8(columns, first + 64 * e, 0, 0);
                else if constexpr (IB == 2) idx[e] = __builtin_amdgcn_raw_buffer_load_b16(columns, (first + 64 * e) * 2, 0, 0);
                else idx[e] = __builtin_amdgcn_raw_buffer_load_b32(columns, (first + 64 * e) * 4, 0, 0);
            }
        } else {
            const auto values = buffer_of((const value_store_t<VT>*)A.G.values + row0 * A.dout, rows_of(t) * A.dout * VB);
#pragma unroll
            for (int u = 0; u < S::UNITS; ++u) {
                const int unit = lane + 64 * u, run = unit % (2 * S::KC), row = w * S::ROWS + unit / (2 * S::KC), o = (chunk * S::KC * 2 + run) * 8;
                const auto offset = [&](int o) { return o < A.dout ? (row * A.dout + o) * VB : kNowhere; };
                if constexpr (KIND == kF32V) {
                    *reinterpret_cast<u32x4*>(val + u * 8) = __builtin_amdgcn_raw_buffer_load_b128(values, offset(o), 0, 0);
                    *reinterpret_cast<u32x4*>(val + u * 8 + 4) = __builtin_amdgcn_raw_buffer_load_b128(values, offset(o + 4), 0, 0);
                } else if constexpr (KIND == kBf16V || KIND == kF16V) {
                    *reinterpret_cast<u32x4*>(val + u * 4) = __builtin_amdgcn_raw_buffer_load_b128(values, offset(o), 0, 0);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if constexpr (VB == 4) val[u * 8 + j] = __builtin_amdgcn_raw_buffer_load_b32(values, offset(o + j), 0, 0);
                        else val[u * 8 + j] = __builtin_amdgcn_raw_buffer_load_b16(values, offset(o + j), 0, 0);
                    }
                }
            }
        }
    };
    const auto fill = [&](int64_t t, int chunk) {
        if constexpr (CBSR) {
            // a wavefront's rows are its own, zeros and entries: its LDS operations stay in order
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int u = 0; u < S::UNITS; ++u) {
                    const int unit = lane + 64 * u;
                    *reinterpret_cast<uint4*>(tile + p * PART + unit_at(unit / S::ROWS, w * S::ROWS + unit % S::ROWS)) = make_uint4(0, 0, 0, 0);
                }
            wave_fence();
            const auto put = [&](int row, uint32_t column, uint32_t value) {
                const uint32_t o = column - (uint32_t)(chunk * S::KC * 16);
                if (o < (uint32_t)(S::KC * 16)) {
                    float part[3];
                    split<P>(__uint_as_float(value), part);
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        *reinterpret_cast<uint16_t*>(tile + p * PART + unit_at((int)o / 8, row) + (o & 7) * 2) = (uint16_t)(__float_as_uint(part[p]) >> 16);
                }
            };
            const int there = rows_of(t) - w * S::ROWS;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (erow[e] < min(S::ROWS, there)) put(w * S::ROWS + erow[e], idx[e], val[e]);
            const int end = min(there, S::ROWS) * k - 1;
            for (int e0 = 64 * E; e0 <= end; e0 += 64 * E) {
                const int64_t mine = (t * kRows + w * S::ROWS) * k;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t p = (uint32_t)min(e0 + lane + 64 * e, end);
                    val[e] = ((const uint32_t*)A.G.values + mine)[p];
                    idx[e] = ((const column_t<KIND>*)A.G.sp_index + mine)[p];
                }
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e0 + lane + 64 * e <= end) put(w * S::ROWS + (e0 + lane + 64 * e) / k, idx[e], val[e]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < S::UNITS; ++u) {
                const int unit = lane + 64 * u, run = unit % (2 * S::KC), row = w * S::ROWS + unit / (2 * S::KC);
                if constexpr (KIND == kBf16V) {  // as it is
                    *reinterpret_cast<u32x4*>(tile + unit_at(run, row)) = *reinterpret_cast<const u32x4*>(val + u * 4);
                    continue;
                }
                float part[8][3];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float x;
                    if constexpr (KIND == kF16V) x = widen_value<VT>((uint16_t)(val[u * 4 + j / 2] >> (16 * (j & 1))));
                    else if constexpr (VB == 4) x = __uint_as_float(val[u * 8 + j]);
                    else x = widen_value<VT>((uint16_t)val[u * 8 + j]);
                    split<P>(x, part[j]);
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
    // Rows and columns that are not there are left out by the buffer's bounds.
    const auto store = [&](int64_t t) {
        const int i = s0 + (w * 32 + l) * S::IT;
        const auto put = [&](auto vb, auto pairs, auto aux) {
            constexpr int B = decltype(vb)::value;
            const auto to = buffer_of((uint8_t*)A.dX + min(t, tiles - 1) * kRows * A.din * B, rows_of(t) * A.din * B);
            const int din = A.din;
            int a = i < din ? (4 * h * din + i) * B : kNowhere, b = i + 1 < din ? (4 * h * din + i + 1) * B : kNowhere;
            asm volatile("" : "+v"(a), "+v"(b));  // added up here: kept from round to round, the offsets of every row would take the weights' registers
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = (8 * (r / 4) + r % 4) * din * B;
                const float x = sum[0][r], y = sum[S::IT - 1][r];
                if constexpr (B == 4) {
                    if constexpr (decltype(pairs)::value) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(x), __float_as_uint(y)}, to, row + a, 0, decltype(aux)::value);
                    else {
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), to, row + a, 0, 0);
                        if constexpr (S::IT == 2) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(y), to, row + b, 0, 0);
                    }
                } else {
                    const bool bf = A.dx_type == MAXK_VALUE_BF16;
                    const uint16_t u = bf ? narrow_value<MAXK_VALUE_BF16>(x) : narrow_value<MAXK_VALUE_F16>(x), v = bf ? narrow_value<MAXK_VALUE_BF16>(y) : narrow_value<MAXK_VALUE_F16>(y);
                    if constexpr (decltype(pairs)::value) __builtin_amdgcn_raw_buffer_store_b32((uint32_t)u | (uint32_t)v << 16, to, row + a, 0, decltype(aux)::value);
                    else {
                        __builtin_amdgcn_raw_buffer_store_b16(u, to, row + a, 0, 0);
                        if constexpr (S::IT == 2) __builtin_amdgcn_raw_buffer_store_b16(v, to, row + b, 0, 0);
                    }
                }
            }
        };
        constexpr std::integral_constant<int, 4> four;
        constexpr std::integral_constant<int, 2> two;  // bytes of an element; also: past L2
        constexpr std::integral_constant<int, 0> plain;
        constexpr std::integral_constant<bool, S::IT == 2> paired;
        constexpr std::false_type single;
        if (A.dx_type == MAXK_VALUE_F32) {
            if (!paired.value || !A.pairs) put(four, single, plain);
            else if (A.once) put(four, paired, two);
            else put(four, paired, plain);
        } else {
            if (!paired.value || !A.pairs) put(two, single, plain);
            else if (A.once) put(two, paired, two);
            else put(two, paired, plain);
        }
    };

    int64_t t = slot * S::GR + group;
    load(t, 0);
    load_weights(0);
    if (S::GR > 1 && (group & 1)) local_fence();  // half a round behind the other group
    if constexpr (CHUNKED) {
        for (int64_t n = 0; n < rounds; ++n, t += stride) {
            clear();
            for (int chunk = 0; chunk < A.chunks; ++chunk) {
                fill(t, chunk);
                local_fence();
                if (chunk + 1 < A.chunks) load(t, chunk + 1);
                else load(t + stride, 0);
                multiply();
                if (chunk + 1 == A.chunks) store(t);
                local_fence();
                load_weights(chunk + 1 < A.chunks ? chunk + 1 : 0);
            }
        }
    } else {
        // A round's results leave while the next one's tile is filled: at the end of the products their way out would hold up the barrier, and the other
        // group with it (932 thousand rows, 256 x 256, CBSR k = 32: 251 to 265 us, 282 there).
        const auto multiply_next = [&]() {
            load(t + stride, 0);
            local_fence();
            __builtin_amdgcn_s_setprio(3);  // products first: the other group's stores to LDS can wait, the operands cannot
            clear();
            multiply();
            __builtin_amdgcn_s_setprio(0);
            local_fence();
        };
        fill(t, 0);
        multiply_next();
        for (int64_t n = 1; n < rounds; ++n) {
            t += stride;
            fill(t, 0);
            store(t - stride);
            multiply_next();
        }
        store(t);
    }
    if (S::GR > 1 && !(group & 1)) local_fence();
}

template <class S, int KIND, int E, bool CHUNKED = false>
maxk_status run(Args A, hipStream_t s)
{
    A.spans = (A.din + S::SPAN - 1) / S::SPAN;
    A.chunks = (A.dout + 16 * S::KC - 1) / (16 * S::KC);
    const int64_t tiles = (A.N + kRows - 1) / kRows;
    // two workgroups a CU where W takes up to 8 operands a lane (most of those use up to 128 registers; CBSR of up to 64 columns at din above 128, and at k above 32, uses 130 to 160, and
    // its 512 take two turns), else one
    A.slots = std::max<int64_t>(1, std::min((tiles + S::GR - 1) / S::GR, (int64_t)(S::KC * S::IT <= 8 ? 512 : 256) / A.spans));
    const int64_t grid = (A.slots + 7) / 8 * A.spans * 8;
    hipLaunchKernelGGL((input_grad_kernel<S, KIND, E, CHUNKED>), dim3((unsigned)grid), dim3(S::THREADS), 0, s, A);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <int KIND, int E = 1>
maxk_status run_kind(const Args& A, hipStream_t s)
{
    // Four wavefronts hold 128 columns of dX, 32 each, or 256.  dH up to 256 columns leaves them the registers for two blocks of W each; up to 384 LDS holds two
    // groups' tiles (200 thousand rows, CBSR k = 32, 384 -> 256 columns: 89 to 92 us, 162 as below); up to 512 one group of eight wavefronts fills and multiplies in turn
    // (512 -> 384: 376 us); wider dH comes in chunks of 256 columns, and W anew with each (600 -> 256: 375 us).  Registers that are spilled to memory: with dH of 385 to 512 columns 14 to 49
    // in CBSR forms, 1 to 36 in dense ones; with two blocks of W of 129 to 256 columns 1 to 4 at k above 32, and 12 to 29 in dense rows that come element by element, which spill 6 to 22 up
    // to 384 columns; elsewhere none.
    const bool two = A.din > 128;
    if (A.dout <= 64) return two ? run<Shape<4, 2, 4, 2>, KIND, E>(A, s) : run<Shape<4, 1, 4, 2>, KIND, E>(A, s);
    if (A.dout <= 128) return two ? run<Shape<8, 2, 4, 2>, KIND, E>(A, s) : run<Shape<8, 1, 4, 2>, KIND, E>(A, s);
    if constexpr (KIND != kCbsr1) {  // (columns of a byte are below 256)
        if (A.dout > 512) return run<Shape<16, 2, 4, 1>, KIND, E, true>(A, s);
        if (A.dout > 384) return run<Shape<32, 1, 8, 1>, KIND, E>(A, s);
        if (A.dout > 256) return run<Shape<24, 1, 4, 2>, KIND, E>(A, s);
    }
    return two ? run<Shape<16, 2, 4, 2>, KIND, E>(A, s) : run<Shape<16, 1, 4, 2>, KIND, E>(A, s);
}

}  // namespace

maxk_status launch_mx_input_grad(const MxGrad& G, int64_t N, const MxMatrix& W, int din, int dout, void* dX, int value_type, hipStream_t s)
{
    const size_t xb = value_type == MAXK_VALUE_F32 ? 4 : 2, gb = G.value_type == MAXK_VALUE_F32 ? 4 : 2;
    const Args A = {G, N, W, din, dout, mx_blocks(din), 0, 0, 0, dX, value_type, din % 2 == 0 && aligned(dX, 2 * xb), past_l2(N * din * (int64_t)xb)};
#define MAXK_ENTRIES(KIND) (G.k <= 32 ? run_kind<KIND, 4>(A, s) : run_kind<KIND, 8>(A, s))
    if (G.k) return G.index_bytes == 1 ? MAXK_ENTRIES(kCbsr1) : G.index_bytes == 2 ? MAXK_ENTRIES(kCbsr2) : MAXK_ENTRIES(kCbsr4);
#undef MAXK_ENTRIES
    const bool pieces = dout * gb % 16 == 0 && aligned(G.values, 16);
    if (G.value_type == MAXK_VALUE_F32) return pieces ? run_kind<kF32V>(A, s) : run_kind<kF32>(A, s);
    if (G.value_type == MAXK_VALUE_BF16) return pieces ? run_kind<kBf16V>(A, s) : run_kind<kBf16>(A, s);
    return pieces ? run_kind<kF16V>(A, s) : run_kind<kF16>(A, s);
}

}  // namespace maxk
