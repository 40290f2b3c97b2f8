// Microscaled storage written and read (include/maxk.h): X into codes and scales, and back.
//
// Both directions are streams: what they read and write once is all they cost.  A lane takes a unit of 8 columns, four lanes a
// block: 16-byte loads or stores on the side of X, 8 or 4 bytes of codes, and the largest magnitude of a block is two DPP steps away.
// A thread has kUnits units under way, a workgroup's width apart.  717 thousand rows of 384 bf16 to 8 bits 125 to 131 us (6.5 TB/s), back 143 to 150 (5.7); a large copy
// reaches 5.1 TB/s.  Rows that are not whole 16-byte pieces go element by element, bound by the number of accesses: 2.4 M rows of 100 bf16, to 8 bits and back, 722 us
// where the bytes would take 311.
#include "mx.hpp"

namespace maxk {
namespace {

constexpr int kUnit = 8;    // columns a lane takes at a time
constexpr int kUnits = 4;   // units under way
constexpr int kThreads = 256;

// How the rows of X lie: rows of whole blocks from a 16-byte boundary (units of X are then one long run), rows of whole 16-byte pieces, any
enum Rows { kRun, kPieces, kAny };

struct UnitAt {
    int64_t x;   // first element
    int valid;   // elements before the end of the row (0 or less: none)
};

// Position of unit u of [rows x nb blocks]
template <Rows R>
__device__ __forceinline__ UnitAt unit_at(int64_t u, int nb, int din)
{
    if constexpr (R == kRun) return {u * kUnit, kUnit};
    const uint64_t block = (uint64_t)u >> 2;
    const uint64_t row = block >> 32 ? block / (uint32_t)nb : (uint64_t)((uint32_t)block / (uint32_t)nb);  // (32-bit division: a third of the time)
    const int col = (int)(block - row * nb) * kMxBlock + (int)(u & 3) * kUnit;
    return {(int64_t)row * din + col, din - col};
}

template <int VT, Rows R>
__device__ __forceinline__ void load_unit(const value_store_t<VT>* X, const UnitAt& at, float* x)
{
    if constexpr (R == kAny) {
#pragma unroll
        for (int j = 0; j < kUnit; ++j) x[j] = j < at.valid ? widen_value<VT>(X[at.x + j]) : 0.f;
    } else if constexpr (VT == MAXK_VALUE_F32) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (R == kRun || at.valid > 0) a = load_once(reinterpret_cast<const float4*>(X + at.x));
        if (R == kRun || at.valid > 4) b = load_once(reinterpret_cast<const float4*>(X + at.x + 4));
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        if (R == kRun || at.valid > 0) a = load_once(reinterpret_cast<const float4*>(X + at.x));
        const uint32_t w[4] = {__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(a.z), __float_as_uint(a.w)};
#pragma unroll
        for (int j = 0; j < kUnit; ++j) x[j] = widen_value<VT>((uint16_t)(w[j / 2] >> (16 * (j & 1))));
    }
}

// the largest of four neighbouring lanes
__device__ __forceinline__ uint32_t max_of_four(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));   // quad_perm [1,0,3,2]
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
}

template <int VT, Rows R, int FMT>
__global__ void __launch_bounds__(kThreads) quantize_kernel(const value_store_t<VT>* __restrict__ X, int64_t units, int din, int nb,
                                                            uint8_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    const int64_t base = (int64_t)blockIdx.x * (kThreads * kUnits) + threadIdx.x;
    float x[kUnits][kUnit];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int64_t u = base + i * kThreads;
        if (u < units) load_unit<VT, R>(X, unit_at<R>(u, nb, din), x[i]);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int64_t u = base + i * kThreads;
        if (u >= units) break;  // whole blocks of four lanes: units are a multiple of 4
        uint32_t top = 0;       // patterns of magnitudes are in the magnitudes' order, Inf and NaN above all others
#pragma unroll
        for (int j = 0; j < kUnit; ++j) top = max(top, __float_as_uint(x[i][j]) & 0x7FFFFFFFu);
        uint32_t s = max_of_four(top) >> 23;
        const bool finite = s != 255u;
        if constexpr (FMT == MAXK_MX_8) {
            uint32_t w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t q[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // adding 1.5 * 2^23 rounds to a whole number, halfway cases to even, and leaves it in the low byte
                    const float y = __builtin_amdgcn_ldexpf(x[i][4 * h + j], 133 - (int)s);
                    q[j] = __float_as_uint(__builtin_amdgcn_fmed3f(y, -127.f, 127.f) + 0x1.8p23f);
                }
                const uint32_t low = __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), high = __builtin_amdgcn_perm(q[3], q[2], 0x04000C0Cu);
                w[h] = finite ? low | high : 0u;
            }
            *reinterpret_cast<uint2*>(codes + u * kUnit) = make_uint2(w[0], w[1]);
        } else {
            if (finite) s = s > 2u ? s - 2u : 0u;
            const float scale = mx_scale(s);
            uint32_t w = 0;  // the conversion divides by the scale, rounds to nearest even and saturates
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][0], x[i][1], scale, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][2], x[i][3], scale, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][4], x[i][5], scale, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][6], x[i][7], scale, 3);
            *reinterpret_cast<uint32_t*>(codes + u * (kUnit / 2)) = finite ? w : 0u;
        }
        if ((threadIdx.x & 3) == 0) scales[u >> 2] = (uint8_t)s;
    }
}

template <int VT, Rows R>
__device__ __forceinline__ void store_unit(value_store_t<VT>* X, const UnitAt& at, const float* x)
{
    if constexpr (R == kAny) {
#pragma unroll
        for (int j = 0; j < kUnit; ++j)
            if (j < at.valid) X[at.x + j] = narrow_value<VT>(x[j]);
    } else if constexpr (VT == MAXK_VALUE_F32) {
        if (R == kRun || at.valid > 0) *reinterpret_cast<float4*>(X + at.x) = make_float4(x[0], x[1], x[2], x[3]);
        if (R == kRun || at.valid > 4) *reinterpret_cast<float4*>(X + at.x + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (VT == MAXK_VALUE_BF16) w[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]), 0x07060302u);  // exact
            else w[j] = (uint32_t)narrow_value<VT>(x[2 * j]) | (uint32_t)narrow_value<VT>(x[2 * j + 1]) << 16;
        }
        if (R == kRun || at.valid > 0) *reinterpret_cast<uint4*>(X + at.x) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int VT, Rows R, int FMT>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t units,
                                                              int din, int nb, value_store_t<VT>* __restrict__ X)
{
    const int64_t base = (int64_t)blockIdx.x * (kThreads * kUnits) + threadIdx.x;
    uint2 w[kUnits];
    uint32_t s[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int64_t u = base + i * kThreads;
        w[i] = make_uint2(0, 0);
        s[i] = 0;
        if (u >= units) continue;
        if constexpr (FMT == MAXK_MX_8) w[i] = *reinterpret_cast<const uint2*>(codes + u * kUnit);
        else w[i].x = *reinterpret_cast<const uint32_t*>(codes + u * (kUnit / 2));
        s[i] = scales[u >> 2];
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int64_t u = base + i * kThreads;
        if (u >= units) break;
        float x[kUnit];
        if constexpr (FMT == MAXK_MX_8) {
            const float unit = mx8_unit(s[i]);
#pragma unroll
            for (int j = 0; j < kUnit; ++j) x[j] = (float)(int8_t)((j < 4 ? w[i].x : w[i].y) >> (8 * (j & 3))) * unit;
        } else {
            const float scale = mx_scale(s[i]);
            const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, scale, 1);
            const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i].x, scale, 3);
            x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
        }
        store_unit<VT, R>(X, unit_at<R>(u, nb, din), x);
    }
}

template <int VT>
Rows rows_of(const void* X, int din)
{
    if (!aligned(X, 16) || din * (int)sizeof(value_store_t<VT>) % 16 != 0) return kAny;
    return din % kMxBlock == 0 ? kRun : kPieces;
}

template <int VT, int FMT>
maxk_status quantize(const void* X, int64_t N, int din, uint8_t* codes, uint8_t* scales, hipStream_t s)
{
    const int nb = mx_blocks(din);
    const int64_t units = N * nb * 4, grid = (units + kThreads * kUnits - 1) / (kThreads * kUnits);
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
#define MAXK_QUANTIZE(R) \
    hipLaunchKernelGGL((quantize_kernel<VT, R, FMT>), dim3((unsigned)grid), dim3(kThreads), 0, s, (const value_store_t<VT>*)X, units, din, nb, codes, scales)
    switch (rows_of<VT>(X, din)) {
        case kRun: MAXK_QUANTIZE(kRun); break;
        case kPieces: MAXK_QUANTIZE(kPieces); break;
        default: MAXK_QUANTIZE(kAny);
    }
#undef MAXK_QUANTIZE
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <int VT, int FMT>
maxk_status dequantize(const MxMatrix& A, int64_t N, int din, void* X, hipStream_t s)
{
    const int nb = mx_blocks(din);
    const int64_t units = N * nb * 4, grid = (units + kThreads * kUnits - 1) / (kThreads * kUnits);
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
#define MAXK_DEQUANTIZE(R)                                                                                                                  \
    hipLaunchKernelGGL((dequantize_kernel<VT, R, FMT>), dim3((unsigned)grid), dim3(kThreads), 0, s, A.codes, A.scales, units, din, nb, \
                       (value_store_t<VT>*)X)
    switch (rows_of<VT>(X, din)) {
        case kRun: MAXK_DEQUANTIZE(kRun); break;
        case kPieces: MAXK_DEQUANTIZE(kPieces); break;
        default: MAXK_DEQUANTIZE(kAny);
    }
#undef MAXK_DEQUANTIZE
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace

maxk_status launch_mx_quantize(const void* X, int value_type, int64_t N, int din, int format, uint8_t* codes, uint8_t* scales, hipStream_t s)
{
#define MAXK_BY_FORMAT(VT) (format == MAXK_MX_8 ? quantize<VT, MAXK_MX_8>(X, N, din, codes, scales, s) : quantize<VT, MAXK_MX_4>(X, N, din, codes, scales, s))
    if (value_type == MAXK_VALUE_F32) return MAXK_BY_FORMAT(MAXK_VALUE_F32);
    if (value_type == MAXK_VALUE_BF16) return MAXK_BY_FORMAT(MAXK_VALUE_BF16);
    return MAXK_BY_FORMAT(MAXK_VALUE_F16);
#undef MAXK_BY_FORMAT
}

maxk_status launch_mx_dequantize(const MxMatrix& A, int64_t N, int din, void* X, int value_type, hipStream_t s)
{
#define MAXK_BY_FORMAT(VT) (A.format == MAXK_MX_8 ? dequantize<VT, MAXK_MX_8>(A, N, din, X, s) : dequantize<VT, MAXK_MX_4>(A, N, din, X, s))
    if (value_type == MAXK_VALUE_F32) return MAXK_BY_FORMAT(MAXK_VALUE_F32);
    if (value_type == MAXK_VALUE_BF16) return MAXK_BY_FORMAT(MAXK_VALUE_BF16);
    return MAXK_BY_FORMAT(MAXK_VALUE_F16);
#undef MAXK_BY_FORMAT
}

}  // namespace maxk
