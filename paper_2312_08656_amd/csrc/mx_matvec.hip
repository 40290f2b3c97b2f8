// Y = X W^T + b for few rows of X in 32 or 16 bits and W in 4 (include/maxk.h): one node's or token's features through a layer.
//
// Bound by the reading of W, 17 bytes for 32 columns of a row.
//
// One row of X (two of 4 or 2 bytes in more than one bf16 part): a lane has a block of 32 columns of X in registers and takes that block of one row of W after the other,
// 16 bytes a load, 16 conversions and 32 multiply-adds; the lanes of a row are added up.  100003 rows of 4096 columns, bf16: 37.7 us (5.8 TB/s, what
// stays in the Infinity Cache included; matrix instructions: 50); fp32 45.7 (83).
//
// More rows: matrix instructions take W as it decodes, exact in bf16, and X in bf16 parts that add up to it (three of fp32, two of fp16), so that products are
// exact, and 16 rows cost little more than three (4096 to 100003, us of 1, 2, 3 and 16 rows: fp32 48, 70, 81, 89, bf16 37, 48, 49, 59).  A wavefront has 16 TILES rows of W and
// 512 columns at a time; the wavefronts of a workgroup share out the columns and are joined in LDS.  The cutting of X takes the vector units 10 us of 16 rows of fp32 by 8192 x 8192, 19 in all, bf16 12.6 (W alone: 7); 16 rows of bf16, 4096 to 100003, 59.
#include "mx_parts.hpp"
#include "rows.hpp"

namespace maxk {
namespace {

typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;      // of X a pass
constexpr int kBlocks = 16;    // blocks of a row of W that a wavefront has at a time: four a lane, four lanes a row
constexpr int kMostWaves = 8;  // of a workgroup, each with a share of the columns

template <int VT> constexpr int kParts = VT == MAXK_VALUE_F32 ? 3 : VT == MAXK_VALUE_BF16 ? 1 : 2;

// 8 columns of X in bf16 parts
template <int VT>
__device__ __forceinline__ void x_parts(const float (&x)[kRowUnit], bf16x8 (&part)[kParts<VT>])
{
    float cut[kRowUnit][kParts<VT>];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) split<kParts<VT>>(x[j], cut[j]);
#pragma unroll
    for (int p = 0; p < kParts<VT>; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = uppers(cut[2 * j][p], cut[2 * j + 1][p]);
        part[p] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

// Rows of W and of X as a lane has them
template <int VT, int TILES>
struct Operands {
    const uint8_t *code[TILES], *scale[TILES];  // its row of each tile as a matrix operand
    const uint8_t* line[TILES];                 // its row and block as it reads memory
    const value_store_t<VT>*x, *x_end;
    int din, nb, quarter;
};

// A row's four lanes have a block each; after it each has a quarter of every one of the four: 8 columns, those of its place in the row's four lanes, so that
// what a matrix instruction takes of X is 32 columns of a row side by side.
__device__ __forceinline__ void share_blocks(uint4& c)
{
    const auto xz = __builtin_amdgcn_permlane32_swap(c.x, c.z, false, false), yw = __builtin_amdgcn_permlane32_swap(c.y, c.w, false, false);
    const auto low = __builtin_amdgcn_permlane16_swap(xz[0], yw[0], false, false), high = __builtin_amdgcn_permlane16_swap(xz[1], yw[1], false, false);
    c = make_uint4(low[0], low[1], high[0], high[1]);
}

// Scale bytes of four blocks from b on, as many as there are
__device__ __forceinline__ uint32_t four_scales(const uint8_t* s, int b, int nb)
{
    uint32_t w = 0;
    if (b + 4 <= nb) {
        __builtin_memcpy(&w, s + b, 4);
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (b + j < nb) w |= (uint32_t)s[b + j] << (8 * j);
    }
    return w;
}

// 4 blocks (128 columns) of X and of W for a wavefront: four lanes have 64 bytes of a row side by side, as the caches want them, and write them to LDS, where the lanes read what
// the matrix instruction takes of 16 rows.  (Read from memory in that order, neighbouring lanes have different rows, and an access is 64 of the
// cache's instead of 16: 16 rows, 4096 to 100003, fp32 108 us, bf16 77.)
// Pieces of 16 bytes lie in each fourth row at another place, so that rows fall on different banks.
__device__ __forceinline__ int own_piece(int lane) { return (lane & 3) ^ (lane >> 4 & 3); }  // as memory is read: of row lane / 4
__device__ __forceinline__ int piece_at(int row, int piece) { return row * 64 + (piece ^ (row >> 2 & 3)) * 16; }
template <int VT>
struct Staged {
    static constexpr int kLoads = VT == MAXK_VALUE_F32 ? 8 : 4;      // of 1 KiB
    static constexpr int kElements = VT == MAXK_VALUE_F32 ? 4 : 8;   // of 16 bytes
    const value_store_t<VT>* x;  // this lane's row and piece as it reads memory
    uint8_t* room;               // kLoads KiB, and one for each tile of W
    int lane;
    uint4 way[kLoads];

    __device__ __forceinline__ void begin(const value_store_t<VT>* X, int64_t n0, int64_t N, int din, uint8_t* room_, int lane_)
    {
        lane = lane_, room = room_;
        const int row = lane >> 2;
        x = X + min(n0 + row, N - 1) * din + own_piece(lane) * kElements;  // (rows behind the last one of X: it again)
    }
    __device__ __forceinline__ void ask(int block)
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) way[j] = read16(x + block * kMxBlock + j * 4 * kElements);
    }
    template <int TILES>
    __device__ __forceinline__ void put(uint4 (&code)[TILES][4], int i)  // and block i of each lane's codes, which come back for the other order
    {
        uint8_t* w = room + kLoads * 1024;
        wave_fence();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) *reinterpret_cast<uint4*>(room + j * 1024 + lane * 16) = way[j];
#pragma unroll
        for (int t = 0; t < TILES; ++t) *reinterpret_cast<uint4*>(w + t * 1024 + lane * 16) = code[t][i];
        wave_fence();
#pragma unroll
        for (int t = 0; t < TILES; ++t) code[t][i] = *reinterpret_cast<const uint4*>(w + t * 1024 + piece_at(lane & 15, lane >> 4));
    }
    __device__ __forceinline__ uint4 piece(int i) const  // of 16 bytes of the lane's row as a matrix operand
    {
        return *reinterpret_cast<const uint4*>(room + (i >> 2) * 1024 + piece_at(lane & 15, i & 3));
    }
    __device__ __forceinline__ RawUnit<VT> get(int q) const  // the lane's 8 columns of block q
    {
        const int quarter = lane >> 4;
        RawUnit<VT> u;
        if constexpr (VT == MAXK_VALUE_F32) u.w[0] = piece(8 * q + 2 * quarter), u.w[1] = piece(8 * q + 2 * quarter + 1);
        else u.w[0] = piece(4 * q + quarter);
        return u;
    }
};

// 16 blocks of columns from block b0 on (WHOLE: all of them lie in the rows)
template <int VT, int TILES, bool WHOLE>
__device__ __forceinline__ void multiply(const Operands<VT, TILES>& O, Staged<VT>& staged, int b0, f32x4v (&sum)[TILES])
{
    if constexpr (WHOLE) staged.ask(b0);
    uint4 code[TILES][4];
    uint32_t scale[TILES][4];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        if constexpr (WHOLE) {
            const uint4 s = read16(O.scale[t] + b0);
            scale[t][0] = s.x, scale[t][1] = s.y, scale[t][2] = s.z, scale[t][3] = s.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = b0 + i * 4 + O.quarter;
            if constexpr (!WHOLE) scale[t][i] = four_scales(O.scale[t], b0 + i * 4, O.nb);
            code[t][i] = make_uint4(0, 0, 0, 0);
            if constexpr (WHOLE) code[t][i] = *reinterpret_cast<const uint4*>(O.line[t] + (b0 + i * 4) * 16);
            else if (b < O.nb) code[t][i] = *reinterpret_cast<const uint4*>(O.code[t] + b * 16);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (!WHOLE && b0 + i * 4 >= O.nb) break;
        const int first = (b0 + i * 4) * kMxBlock + O.quarter * kRowUnit;
        RawUnit<VT> raw[4];
        if constexpr (WHOLE) {
            staged.put(code, i);
            if (i < 3) staged.ask(b0 + (i + 1) * 4);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = first + q * kMxBlock;
            if constexpr (WHOLE) raw[q] = staged.get(q);
            else raw[q] = fetch_row_unit<VT>(O.x + col, O.din - col, O.x_end);
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) share_blocks(code[t][i]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            bf16x8 part[kParts<VT>];
            if constexpr (WHOLE && VT == MAXK_VALUE_BF16) {
                part[0] = __builtin_bit_cast(bf16x8, raw[q].w[0]);
            } else {
                float v[kRowUnit];
                unit_values<VT>(raw[q], WHOLE ? kRowUnit : O.din - first - q * kMxBlock, 0.f, v);
                x_parts<VT>(v, part);
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const uint32_t w[4] = {code[t][i].x, code[t][i].y, code[t][i].z, code[t][i].w};
                const float unit = mx_scale(scale[t][i] >> (8 * q) & 0xFFu);
                uint4 a;
                a.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit, 0));
                a.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit, 1));
                a.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit, 2));
                a.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit, 3));
#pragma unroll
                for (int p = 0; p < kParts<VT>; ++p)
                    sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), part[p], sum[t], 0, 0, 0);
            }
        }
    }
}

template <int VT, int TILES> constexpr int matvec_room = (Staged<VT>::kLoads + TILES) * 1024;  // of a wavefront: what is staged, its sums in the end

template <int VT, int TILES>
__global__ void __launch_bounds__(kMostWaves* kWave) matvec_kernel(const value_store_t<VT>* X, int64_t N, const uint8_t* codes, const uint8_t* scales, int din,
                                                                   int dout, const float* bias, void* Y, int y_type)
{
    extern __shared__ uint4 rooms[];  // of every wavefront
    constexpr int kRoom = matvec_room<VT, TILES>;
    uint8_t* room = reinterpret_cast<uint8_t*>(rooms);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    const int nb = mx_blocks(din), row16 = lane & 15, quarter = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.y * kRows, n = n0 + row16;
    const int64_t o0 = (int64_t)blockIdx.x * (16 * TILES);
    Operands<VT, TILES> O;
    O.x = X + min(n, N - 1) * din;  // (lanes behind the last row of X repeat it: what they add up is not stored)
    O.x_end = X + N * din;
    O.din = din, O.nb = nb, O.quarter = quarter;
    f32x4v sum[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        sum[t] = f32x4v{0.f, 0.f, 0.f, 0.f};
        const int64_t o = min(o0 + t * 16 + row16, (int64_t)dout - 1);
        O.code[t] = codes + o * nb * 16;
        O.scale[t] = scales + o * nb;
        O.line[t] = codes + (min(o0 + t * 16 + (lane >> 2), (int64_t)dout - 1) * nb + own_piece(lane)) * 16;
    }
    Staged<VT> staged;
    staged.begin(X, n0, N, din, room + wave * kRoom, lane);
    for (int b0 = wave * kBlocks; b0 < nb; b0 += waves * kBlocks) {
        if ((b0 + kBlocks) * kMxBlock <= din) multiply<VT, TILES, true>(O, staged, b0, sum);
        else multiply<VT, TILES, false>(O, staged, b0, sum);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) *reinterpret_cast<f32x4v*>(room + wave * kRoom + t * 1024 + lane * 16) = sum[t];
    __syncthreads();
    if (n >= N) return;
    for (int t = wave; t < TILES; t += waves) {
        f32x4v y = *reinterpret_cast<const f32x4v*>(room + t * 1024 + lane * 16);
        for (int w = 1; w < waves; ++w) y += *reinterpret_cast<const f32x4v*>(room + w * kRoom + t * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t o = o0 + t * 16 + quarter * 4 + j, at = n * dout + o;
            if (o >= dout) continue;
            const float v = y[j] + (bias ? bias[o] : 0.f);
            if (y_type == MAXK_VALUE_F32) ((float*)Y)[at] = v;
            else if (y_type == MAXK_VALUE_BF16) ((uint16_t*)Y)[at] = round_value<MAXK_VALUE_BF16>(v);
            else ((uint16_t*)Y)[at] = round_value<MAXK_VALUE_F16>(v);
        }
    }
}

template <int VT, int TILES>
maxk_status run_matvec(const void* X, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type, int waves, hipStream_t s)
{
    const unsigned room = (unsigned)waves * matvec_room<VT, TILES>;
    hipLaunchKernelGGL((matvec_kernel<VT, TILES>), dim3((unsigned)((dout + 16 * TILES - 1) / (16 * TILES)), (unsigned)((N + kRows - 1) / kRows)), dim3(waves * kWave), room, s,
                       (const value_store_t<VT>*)X, N, W.codes, W.scales, din, dout, bias, Y, y_type);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

// ---- one row of X, or two: no matrix instructions ----

constexpr int kMostGroupsAcross = 1 << 20;  // (in one dimension the threads of a launch have to be fewer than 2^32)

// LANES lanes (a block of columns each) and COLS wavefronts share a row of W; a wavefront has BATCH of its rows, or 64 / LANES times as many, under way.
template <int LANES, int COLS>
struct LaneForm {
    static constexpr int kBatch = LANES == kWave && COLS < 16 ? 8 : 4;
    static constexpr int kWaves = COLS <= 2 ? 4 : COLS <= 4 ? 8 : COLS, kThreads = kWaves * kWave;
    static constexpr int kSide = kWave / LANES, kStep = kSide * kBatch;  // rows of W that an access has; that a wavefront has
    static constexpr int kRows = kStep * (kWaves / COLS);               // of a workgroup
};

template <int VT, int N, int LANES, int COLS>
__global__ void __launch_bounds__((LaneForm<LANES, COLS>::kThreads))
    matvec_lanes_kernel(const value_store_t<VT>* X, const uint8_t* codes, const uint8_t* scales, int din, int dout, const float* bias, void* Y, int y_type)
{
    using F = LaneForm<LANES, COLS>;
    __shared__ float sums[COLS > 1 ? F::kWaves : 1][N][F::kStep];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave, part = wave % COLS, group = wave / COLS;
    const int nb = mx_blocks(din), b = part * LANES + lane % LANES;
    const int64_t o0 = ((int64_t)blockIdx.y * kMostGroupsAcross + blockIdx.x) * F::kRows + group * F::kStep;
    uint4 code[F::kBatch];
    uint32_t scale[F::kBatch];
#pragma unroll
    for (int i = 0; i < F::kBatch; ++i) {
        const int64_t o = min(o0 + i * F::kSide + lane / LANES, (int64_t)dout - 1);
        code[i] = make_uint4(0, 0, 0, 0);
        scale[i] = 0;
        if (b < nb) {
            code[i] = *reinterpret_cast<const uint4*>(codes + (o * nb + b) * 16);
            scale[i] = scales[o * nb + b];
        }
    }
    RawUnit<VT> raw[N][4];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = b * kMxBlock + q * kRowUnit;
            raw[n][q] = fetch_row_unit<VT>(X + n * (int64_t)din + col, din - col, X + N * (int64_t)din);
        }
    float x[N][4][kRowUnit];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) unit_values<VT>(raw[n][q], din - b * kMxBlock - q * kRowUnit, 0.f, x[n][q]);
    float sum[N][F::kBatch];
#pragma unroll
    for (int i = 0; i < F::kBatch; ++i) {
        const float unit = mx_scale(scale[i]);
        const uint32_t w[4] = {code[i].x, code[i].y, code[i].z, code[i].w};
#pragma unroll
        for (int n = 0; n < N; ++n) sum[n][i] = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const decltype(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(0u, 1.f, 0)) v[4] = {
                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[q], unit, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[q], unit, 1),
                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[q], unit, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[q], unit, 3)};
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sum[n][i] = fmaf(v[j][0], x[n][q][2 * j], sum[n][i]);
                    sum[n][i] = fmaf(v[j][1], x[n][q][2 * j + 1], sum[n][i]);
                }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) sum[n][i] = over_lanes<LANES>(sum[n][i], kAdd);
    }
    const auto store = [&](int n, int64_t o, float y) {
        if (o >= dout) return;
        y += bias ? bias[o] : 0.f;
        const int64_t at = n * (int64_t)dout + o;
        if (y_type == MAXK_VALUE_F32) ((float*)Y)[at] = y;
        else if (y_type == MAXK_VALUE_BF16) ((uint16_t*)Y)[at] = round_value<MAXK_VALUE_BF16>(y);
        else ((uint16_t*)Y)[at] = round_value<MAXK_VALUE_F16>(y);
    };
    if constexpr (COLS == 1) {
        if (lane % LANES != 0) return;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < F::kBatch; ++i) store(n, o0 + i * F::kSide + lane / LANES, sum[n][i]);
    } else {
        if (lane == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < F::kBatch; ++i) sums[wave][n][i] = sum[n][i];
        }
        __syncthreads();
        if (part > 0 || lane >= F::kStep) return;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float y = sums[wave][n][lane];
#pragma unroll
            for (int c = 1; c < COLS; ++c) y += sums[wave + c][n][lane];
            store(n, o0 + lane, y);
        }
    }
}

template <int VT, int N, int LANES, int COLS>
maxk_status run_lanes(const void* X, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type, hipStream_t s)
{
    using F = LaneForm<LANES, COLS>;
    const int groups = (dout + F::kRows - 1) / F::kRows;
    const dim3 grid((unsigned)std::min(groups, kMostGroupsAcross), (unsigned)((groups + kMostGroupsAcross - 1) / kMostGroupsAcross));
    hipLaunchKernelGGL((matvec_lanes_kernel<VT, N, LANES, COLS>), grid, dim3(F::kThreads), 0, s,
                       (const value_store_t<VT>*)X, W.codes, W.scales, din, dout, bias, Y, y_type);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

constexpr int kMostLaneBlocks = 16 * kWave;  // blocks of a row that the lanes of a workgroup have at once
template <int VT, int N>
maxk_status matvec_lanes(const void* X, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type, hipStream_t s)
{
    const int nb = mx_blocks(din);
    if (nb <= 4) return run_lanes<VT, N, 4, 1>(X, W, din, dout, bias, Y, y_type, s);
    if (nb <= 8) return run_lanes<VT, N, 8, 1>(X, W, din, dout, bias, Y, y_type, s);
    if (nb <= 16) return run_lanes<VT, N, 16, 1>(X, W, din, dout, bias, Y, y_type, s);
    if (nb <= 32) return run_lanes<VT, N, 32, 1>(X, W, din, dout, bias, Y, y_type, s);
    if (nb <= 64) return run_lanes<VT, N, 64, 1>(X, W, din, dout, bias, Y, y_type, s);
    if (nb <= 128) return run_lanes<VT, N, 64, 2>(X, W, din, dout, bias, Y, y_type, s);
    if (nb <= 256) return run_lanes<VT, N, 64, 4>(X, W, din, dout, bias, Y, y_type, s);
    if (nb <= 512) return run_lanes<VT, N, 64, 8>(X, W, din, dout, bias, Y, y_type, s);
    return run_lanes<VT, N, 64, 16>(X, W, din, dout, bias, Y, y_type, s);
}

template <int VT>
maxk_status matvec(const void* X, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type, hipStream_t s)
{
    if (mx_blocks(din) <= kMostLaneBlocks) {
        if (N == 1) return matvec_lanes<VT, 1>(X, W, din, dout, bias, Y, y_type, s);
        // a second row costs the matrix instructions nothing but fp32's and fp16's parts: 100003 x 4096, two rows, lanes / matrix instructions 63 / 83 us fp32, 56 / 50 bf16
        if constexpr (kParts<VT> > 1)
            if (N == 2) return matvec_lanes<VT, 2>(X, W, din, dout, bias, Y, y_type, s);
    }
    // Two tiles a wavefront, for which X is read and cut up once, where that leaves workgroups for three quarters of the CUs; four wavefronts with larger shares of
    // the columns where there are four workgroups a CU and more.  us, 1 tile and 8 wavefronts / 2 and 8 / 2 and 4 / 4 and 4, 16 rows: fp32 4096 x 4096 9.3 / 10.1 / 11.4 /
    // 16.5, 8192 x 8192 22.3 / 19.0 / 22.2 / 30.7, 4096 to 100003 137 / 124 / 92 / 90; bf16 8192 x 8192 13.9 / 12.6 / 14.8 / 19.6, 4096 to 100003 89 / 61 / 59 / 62
    const int shares = (mx_blocks(din) + kBlocks - 1) / kBlocks, pairs = (dout + 31) / 32;
    if (pairs < 192) return run_matvec<VT, 1>(X, N, W, din, dout, bias, Y, y_type, std::min(shares, kMostWaves), s);
    return run_matvec<VT, 2>(X, N, W, din, dout, bias, Y, y_type, std::min(shares, pairs < 4 * 256 ? kMostWaves : kMostWaves / 2), s);
}

}  // namespace

maxk_status launch_mx_matvec(const void* X, int value_type, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type,
                             hipStream_t s)
{
    if (value_type == MAXK_VALUE_F32) return matvec<MAXK_VALUE_F32>(X, N, W, din, dout, bias, Y, y_type, s);
    if (value_type == MAXK_VALUE_BF16) return matvec<MAXK_VALUE_BF16>(X, N, W, din, dout, bias, Y, y_type, s);
    return matvec<MAXK_VALUE_F16>(X, N, W, din, dout, bias, Y, y_type, s);
}

}  // namespace maxk
