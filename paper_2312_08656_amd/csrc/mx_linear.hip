// Y = X W^T + b of 4-bit operands (include/maxk.h).
//
// The matrix instruction takes 4-bit codes with a scale byte for 32 products: 16 x 16 outputs over 128 columns, a lane holding one block of
// either operand.  Rows are many and widths small, so a wavefront keeps 64 rows of W (all their columns) in its registers and walks
// over the rows of X, 16 at a time; the next 16 are on their way meanwhile.  Wavefronts that share rows of X lie in one workgroup, so X is read through L1.
//
// Bound by the way to memory, mostly Y's way out: 2.4 M rows, 256 to 256, fp32 Y 570 us (2.84 GB, 5.0 TB/s, what a large copy reaches); 1 M rows
// 181 us with X in the Infinity Cache (6.4 TB/s), 259 without (4.5); 1.1 M rows, 384 to 256, bf16 Y 149 to 153 and 200 us.  One row, 256 to 256: 3.9 us a call, two round
// trips to memory and the launch.  Farther from it: 16-bit Y (2.4 M rows, 256 to 256, bf16 420 us, the bytes 310; 256 to 100, whose rows leave a column a lane, 242 and 157) and
// more than 512 columns in (1 M rows, 768 to 256, fp32 597 us and 341; 1433 to 256, whose Y leaves in pieces of 64 bytes, 1180 and 637).
#include <algorithm>

#include "mx_parts.hpp"

namespace maxk {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kTileRows = 16;     // rows of X in a step
constexpr int kGroup = 64;        // columns of Y (rows of W) of a wavefront
constexpr int kTiles = kGroup / 16;
constexpr int kChunkBlocks = 4;   // blocks of 32 columns that an instruction takes: one for each 16 lanes

template <int BYTE>  // of the scale registers
__device__ __forceinline__ f32x4 mfma(const uint4& a, uint32_t sa, const uint4& b, uint32_t sb, f32x4 c)
{
    const i32x8 A = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, B = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4, 4, BYTE, (int)sa, BYTE, (int)sb);  // 4: E2M1
}

template <int C>
struct Blocks {  // one lane's blocks of a row
    uint4 code[C];
    uint32_t scale[(C + 3) / 4];  // a byte each
};
template <int C>
struct Loaded {
    uint4 code[C];
    uint32_t scale[C];
};
template <int C>
__device__ __forceinline__ Blocks<C> packed(const Loaded<C>& x)
{
    Blocks<C> y;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        y.code[c] = x.code[c];
        y.scale[c / 4] = c % 4 ? y.scale[c / 4] | x.scale[c] << (8 * (c % 4)) : x.scale[c];
    }
    return y;
}

// sum + the products of all blocks
template <int C, int c = 0>
__device__ __forceinline__ f32x4 products(const Blocks<C>& a, const Blocks<C>& b, f32x4 sum)
{
    if constexpr (c < C) return products<C, c + 1>(a, b, mfma<c % 4>(a.code[c], a.scale[c / 4], b.code[c], b.scale[c / 4], sum));
    else return sum;
}

// Blocks g, 4 + g, ... of row `row` of those from `first` on.  Past its end: the last block again for X, zeros for W, whose products are
// then 0 (or NaN where that block of X stands for NaN, and the row's sums with it).
template <int C, bool ZERO>
__device__ __forceinline__ void load_blocks(Loaded<C>& x, const MxMatrix& A, int64_t first, int row, int g, int nb)
{
    const uint8_t *codes = A.codes + first * nb * 16, *scales = A.scales + first * nb;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int b = c * kChunkBlocks + g, at = row * nb + min(b, nb - 1);
        x.code[c] = *reinterpret_cast<const uint4*>(codes + (uint32_t)at * 16u);
        x.scale[c] = scales[(uint32_t)at];
        if (ZERO && b >= nb) x.code[c] = make_uint4(0, 0, 0, 0), x.scale[c] = 127;
    }
}

constexpr int kMaxGroups = 6;     // of a workgroup: up to 384 columns of Y
constexpr int kPad = 4;           // floats at the end of a row in LDS, so that rows begin in different banks

// A workgroup makes 16 m rows of Y, up to 384 columns of each, in a step: `gcols` wavefronts side by side, m below each other.  The matrix
// instruction leaves four columns a lane over 16 rows; the outputs are turned round in LDS and leave as whole rows.  (As they are, 64 bytes of 16 rows a
// store: 989 us for 2.4 M rows, 256 to 256 columns; through LDS, 256 bytes of 4 rows: 666.)
// WIDE: rows of Y are whole 16-byte pieces from a 16-byte boundary; else a column a lane.
// ONCE: Y passes by L2.
template <int C, int VT, bool WIDE, bool ONCE>
__global__ void __launch_bounds__(64 * kMaxGroups) linear_kernel(MxMatrix X, int64_t N, MxMatrix W, int nb, int dout, int gcols, int m, bool pace,
                                                                 const float* __restrict__ bias, value_store_t<VT>* __restrict__ Y)
{
    extern __shared__ __align__(16) float turned[];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int threads = 64 * gcols * m, left = blockIdx.y * gcols * kGroup, cols = min(gcols * kGroup, dout - left);
    const int first = left + wave % gcols * kGroup, pitch = gcols * kGroup + kPad, rows_step = kTileRows * m;
    const int64_t steps = (N + rows_step - 1) / rows_step;

    Blocks<C> w[kTiles];
    f32x4 start[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        Loaded<C> row;
        load_blocks<C, true>(row, W, 0, min(first + t * 16 + r, dout - 1), g, nb);  // (the last wavefronts may lie past dout)
        w[t] = packed(row);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int o = first + t * 16 + g * 4 + j;
            start[t][j] = bias && o < dout ? bias[o] : 0.f;
        }
    }
    // The pieces of a whole step that this thread stores.  Every thread makes as many stores, the spare ones of the last piece again, so that
    // the number of stores behind a load is known and a load can be waited for without them.
    constexpr int V = WIDE ? 16 / (int)sizeof(value_store_t<VT>) : 1, S = WIDE ? 16 / V : 1;
    const int pieces = (cols + V - 1) / V;
    int from[S], to[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int q = min((int)threadIdx.x + i * threads, rows_step * pieces - 1), row = q / pieces, col = (q - row * pieces) * V;
        from[i] = row * pitch + col;
        to[i] = row * dout + col;
    }
    const int below = wave / gcols * kTileRows;
    const auto load = [&](Loaded<C>& x, int64_t step) {
        const int64_t row = min(min(step, steps - 1) * rows_step + below, N - 1);
        load_blocks<C, false>(x, X, row, min(r, (int)min(N - 1 - row, (int64_t)kTileRows - 1)), g, nb);
    };
    Loaded<C> next;
    load(next, blockIdx.x);
    float* room = turned;
    float* other = turned + rows_step * pitch;
    int64_t step = blockIdx.x;
    const auto make = [&]() {  // the outputs of a step, in `room`
        const Blocks<C> x = packed(next);
        load(next, step + gridDim.x);
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
            *reinterpret_cast<f32x4*>(room + (below + r) * pitch + wave % gcols * kGroup + t * 16 + g * 4) = products(w[t], x, start[t]);
        local_fence();  // the room of the step before was read before the one barrier, and is written after the next
    };
    const auto whole_step = [&]() {
        if (pace) __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
        make();
        value_store_t<VT>* out = Y + step * rows_step * dout + left;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            f32x4 y = *reinterpret_cast<const f32x4*>(room + from[i]);
            if constexpr (VT != MAXK_VALUE_F32) {
                const f32x4 z = *reinterpret_cast<const f32x4*>(room + from[i] + 4);
                const auto two = [](float a, float b) { return __uint_as_float((uint32_t)narrow_value<VT>(a) | (uint32_t)narrow_value<VT>(b) << 16); };
                y = f32x4{two(y[0], y[1]), two(y[2], y[3]), two(z[0], z[1]), two(z[2], z[3])};
            }
            f32x4* p = reinterpret_cast<f32x4*>(out + to[i]);
            if constexpr (ONCE) __builtin_nontemporal_store(y, p);
            else *p = y;
        }
        float* const swap = room;
        room = other, other = swap;
        step += gridDim.x;
    };
    if constexpr (WIDE) {
        const int64_t whole = N / rows_step;
        if (step < whole) {
            whole_step();  // by itself: its loads have no stores behind them, and the loop's wait would be the same for both
            while (step < whole) whole_step();
        }
    }
    for (; step < steps; step += gridDim.x) {
        make();
        const int64_t row0 = step * rows_step;
        const int rows = (int)min(N - row0, (int64_t)rows_step);
        for (int row = wave; row < rows; row += gcols * m)
            for (int col = lane; col < cols; col += 64) Y[(row0 + row) * dout + left + col] = narrow_value<VT>(room[row * pitch + col]);
        float* const swap = room;
        room = other, other = swap;
    }
}

// Rows wider than the registers hold: 64 rows of X by 64 of W a wavefront, blocks of either straight from memory.
template <int VT>
__global__ void __launch_bounds__(256) linear_long_kernel(MxMatrix X, int64_t N, MxMatrix W, int nb, int dout, int groups, const float* __restrict__ bias,
                                                          value_store_t<VT>* __restrict__ Y)
{
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = (int)(wave % groups) * kGroup;
    const int64_t row0 = wave / groups * 64;
    if (row0 >= N) return;
    f32x4 sum[4][kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int o = first + t * 16 + r;
#pragma unroll
        for (int m = 0; m < 4; ++m) sum[m][t] = bias && o < dout ? f32x4{bias[o], bias[o], bias[o], bias[o]} : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int c = 0; c < nb; c += kChunkBlocks) {
        Blocks<1> x[4], w[kTiles];
        const int b = min(c + g, nb - 1);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int64_t at = min(row0 + m * 16 + r, N - 1) * nb + b;
            x[m].code[0] = *reinterpret_cast<const uint4*>(X.codes + at * 16);
            x[m].scale[0] = X.scales[at];
            const int64_t wt = (int64_t)min(first + m * 16 + r, dout - 1) * nb + b;
            w[m].code[0] = *reinterpret_cast<const uint4*>(W.codes + wt * 16);
            w[m].scale[0] = W.scales[wt];
            if (c + g >= nb) w[m].code[0] = make_uint4(0, 0, 0, 0), w[m].scale[0] = 127;
        }
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) sum[m][t] = products(x[m], w[t], sum[m][t]);
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t row = row0 + m * 16 + g * 4 + j;
                const int o = first + t * 16 + r;
                if (row < N && o < dout) Y[row * dout + o] = narrow_value<VT>(sum[m][t][j]);
            }
}

// 3 for each of the 1024 SIMDs.  us at 2048 / 2600 / 3 x 1024 / 3400 / 4096 wavefronts, 2.4 M rows, 256 to 256, fp32 Y: 677 / 662 / 570 / 671 / 612, 1 M rows 185 / 212 / 180 / 210 /
// 197 (whole workgroups a CU are faster than odd ones).  One number for all instances, and not the best of each: bf16 Y, 2.4 M rows 504 / 490 / 420 / 408 / 317; 768 to 256
// columns, where 256 registers a lane (18 more are spilled for fp32 Y) leave room for 2 a SIMD, 1 M rows 457 / 675 / 598 / 556 / 501; 256 to 320, five column
// groups, 1.2 M rows 314 / 367 / 322 / 305 / 353.
constexpr int64_t kWaves = 3 * 1024;

template <int C, int VT>
void launch_chunks(const MxMatrix& X, int64_t N, const MxMatrix& W, int nb, int dout, const float* bias, value_store_t<VT>* Y, hipStream_t s)
{
    const int groups = (dout + kGroup - 1) / kGroup, sides = (groups + kMaxGroups - 1) / kMaxGroups, gcols = (groups + sides - 1) / sides, m = std::max(1, 4 / gcols);
    const int64_t steps = (N + kTileRows * m - 1) / (kTileRows * m), blocks = std::min(steps, std::max<int64_t>(1, kWaves / (gcols * m * sides)));
    const size_t lds = 2 * sizeof(float) * (size_t)(kTileRows * m) * (gcols * kGroup + kPad);
    // Where X does not stay in the Infinity Cache its reads share the way to memory with Y's writes, and do better if a step waits for the writes of the
    // one before.  us, with / without: 2.4 M rows, 256 to 256 569 / 626, bf16 Y 421 / 407; 1.2 M, 512 to 384 615 / 594; below that size 1.6 M, 256 to 256 303 / 293,
    // 0.1 M 21.9 / 20.9.
    const bool pace = (double)N * nb * 17 > kInfinityCache;
    const dim3 grid((unsigned)blocks, (unsigned)sides), block(64 * gcols * m);
#define MAXK_LINEAR(WIDE, ONCE) hipLaunchKernelGGL((linear_kernel<C, VT, WIDE, ONCE>), grid, block, lds, s, X, N, W, nb, dout, gcols, m, pace, bias, Y)
    if (dout * sizeof(*Y) % 16 != 0 || !aligned(Y, 16)) MAXK_LINEAR(false, false);
    else if (past_l2(N * dout * (int64_t)sizeof(*Y))) MAXK_LINEAR(true, true);
    else MAXK_LINEAR(true, false);
#undef MAXK_LINEAR
}

template <int VT>
maxk_status launch(const MxMatrix& X, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, value_store_t<VT>* Y, hipStream_t s)
{
    const int nb = mx_blocks(din), chunks = (nb + kChunkBlocks - 1) / kChunkBlocks;
    if (chunks <= 1) launch_chunks<1, VT>(X, N, W, nb, dout, bias, Y, s);
    else if (chunks <= 2) launch_chunks<2, VT>(X, N, W, nb, dout, bias, Y, s);
    else if (chunks <= 4) launch_chunks<4, VT>(X, N, W, nb, dout, bias, Y, s);
    else if (chunks <= 8) launch_chunks<8, VT>(X, N, W, nb, dout, bias, Y, s);
    else {
        const int groups = (dout + kGroup - 1) / kGroup;
        const int64_t grid = ((N + 63) / 64 * groups + 3) / 4;
        if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
        hipLaunchKernelGGL((linear_long_kernel<VT>), dim3((unsigned)grid), dim3(256), 0, s, X, N, W, nb, dout, groups, bias, Y);
    }
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace

maxk_status launch_mx_linear(const MxMatrix& X, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int value_type,
                             hipStream_t s)
{
    if (value_type == MAXK_VALUE_F32) return launch<MAXK_VALUE_F32>(X, N, W, din, dout, bias, (float*)Y, s);
    if (value_type == MAXK_VALUE_BF16) return launch<MAXK_VALUE_BF16>(X, N, W, din, dout, bias, (uint16_t*)Y, s);
    return launch<MAXK_VALUE_F16>(X, N, W, din, dout, bias, (uint16_t*)Y, s);
}

}  // namespace maxk
