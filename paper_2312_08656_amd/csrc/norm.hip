// Root-mean-square norm of rows with the residual's addition, stored in its type, in 8 or in 4 bits, and its gradients (include/maxk.h).
//
//   h = round(x + residual),  r = 1 / sqrt(mean h^2 + eps),  y = h r gamma
//   dx = r (dy gamma - x^ mean(dy gamma x^)) + dh,  x^ = h r;   dgamma = sum over rows of dy x^
//
// Streams: what they read and write once is what they cost.  L lanes have a row in their registers, U units of 8 columns each, so that it is read
// once; for rows of up to 2048 columns that is part of a wavefront or all of it and no barrier is passed.  716847 x 384 bf16 with residual and 8-bit codes 378 us, 5.1 TB/s;
// 232965 x 256 fp32 182 and the gradient 202 (5.2 and 4.7; a copy: 5.0 to 5.1); 50000 x 4096 bf16 149 and 245.  Rows that are short and no whole 16-byte pieces leave lanes
// idle and end in three stores: 2449029 x 47 bf16 148, where the memory would take 90.
#include "heads.hpp"
#include "rows.hpp"

namespace maxk {
namespace {

constexpr int kThreads = 256;
__host__ __device__ constexpr int norm_threads(int L) { return L > kThreads ? L : kThreads; }

// Squares are added up in 64 bits: the sum does not depend on how a row is dealt to lanes beyond a rounding that is lost in r's, and codes that
// lie next to a border between two come out the same on either side.  The vector units are busy for 47 % of 716847 x 384's time, for 17 % of fp32's.
template <int VT, int L, int U>
__global__ void __launch_bounds__(norm_threads(L)) norm_kernel(NormCall C, int64_t N, int dim)
{
    using S = value_store_t<VT>;
    constexpr int kTeams = norm_threads(L) / L;
    __shared__ double room[2][L > kWave ? L / kWave : 1];
    const S *X = (const S*)C.X, *R = (const S*)C.residual;
    const S *X_end = X + N * dim, *R_end = R + N * dim;
    const int lane = threadIdx.x % L, nb = mx_blocks(dim);
    float gamma[U][kRowUnit];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int col = (lane + u * L) * kRowUnit;
        load_row_unit<MAXK_VALUE_F32>(C.gamma + col, dim - col, C.gamma + dim, 0.f, gamma[u]);
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / L; row < N; row += (int64_t)gridDim.x * kTeams, turn ^= 1) {
        float h[U][kRowUnit];
        RawUnit<VT> raw[U], added[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (lane + u * L) * kRowUnit;
            raw[u] = fetch_row_unit<VT>(X + row * dim + col, dim - col, X_end);
            if (R) added[u] = fetch_row_unit<VT>(R + row * dim + col, dim - col, R_end);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) unit_values<VT>(raw[u], dim - (lane + u * L) * kRowUnit, 0.f, h[u]);
        if (R) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float r[kRowUnit];
                unit_values<VT>(added[u], dim - (lane + u * L) * kRowUnit, 0.f, r);
#pragma unroll
                for (int j = 0; j < kRowUnit; ++j) h[u][j] = rounded<VT>(h[u][j] + r[j]);
            }
        }
        double sum = 0.0;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) sum = fma((double)h[u][j], (double)h[u][j], sum);
        sum = row_sum<L>(sum, room[turn]);
        const float rstd = (float)rsqrt(sum / (double)dim + C.eps);
        if (C.rstd && lane == 0) C.rstd[row] = rstd;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * L, col = unit * kRowUnit;
            if (R) store_row_unit<VT>((S*)C.H + row * dim + col, dim - col, h[u]);
            float y[kRowUnit];
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) y[j] = h[u][j] * rstd * gamma[u][j];
            if (C.Y) store_row_unit<VT>((S*)C.Y + row * dim + col, dim - col, y);
            if (C.codes && unit < nb * 4) {  // whole blocks of four lanes
                const int64_t at = row * nb * 4 + unit;
                const uint32_t s = C.format == MAXK_MX_8 ? encode_unit<MAXK_MX_8>(y, C.codes + at * 8) : encode_unit<MAXK_MX_4>(y, C.codes + at * 4);
                if ((lane & 3) == 0) C.scales[at >> 2] = (uint8_t)s;
            }
        }
    }
}

// dgamma: a lane adds up its columns over the rows that it works on, a workgroup its teams' sums through LDS, and a second kernel the workgroups' sums, in a
// fixed order.
template <int VT, int L, int U>
__global__ void __launch_bounds__(norm_threads(L)) norm_grad_kernel(NormGradCall C, float* parts, int64_t N, int dim)
{
    using S = value_store_t<VT>;
    constexpr int kTeams = norm_threads(L) / L, kCols = L * U * kRowUnit;
    __shared__ float room[2][L > kWave ? L / kWave : 1];
    __shared__ float sums[kTeams > 1 ? kTeams * kCols : 1];
    const S *dY = (const S*)C.dY, *H = (const S*)C.H, *dH = (const S*)C.dH;
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    float gamma[U][kRowUnit], total[U][kRowUnit];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int col = (lane + u * L) * kRowUnit;
        load_row_unit<MAXK_VALUE_F32>(C.gamma + col, dim - col, C.gamma + dim, 0.f, gamma[u]);
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) total[u][j] = 0.f;
    }
    const float inverse = 1.f / (float)dim;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kTeams + team; row < N; row += (int64_t)gridDim.x * kTeams, turn ^= 1) {
        float x[U][kRowUnit], dy[U][kRowUnit];
        const float rstd = C.rstd[row];
        RawUnit<VT> raw_h[U], raw_dy[U], raw_dh[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (lane + u * L) * kRowUnit;
            raw_h[u] = fetch_row_unit<VT>(H + row * dim + col, dim - col, H + N * dim);
            raw_dy[u] = fetch_row_unit<VT>(dY + row * dim + col, dim - col, dY + N * dim);
            if (dH) raw_dh[u] = fetch_row_unit<VT>(dH + row * dim + col, dim - col, dH + N * dim);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int valid = dim - (lane + u * L) * kRowUnit;
            unit_values<VT>(raw_h[u], valid, 0.f, x[u]);
            unit_values<VT>(raw_dy[u], valid, 0.f, dy[u]);
        }
        float dot = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) {
                x[u][j] *= rstd;
                total[u][j] = fmaf(dy[u][j], x[u][j], total[u][j]);
                dy[u][j] *= gamma[u][j];
                dot = fmaf(dy[u][j], x[u][j], dot);
            }
        dot = row_sum<L>(dot, room[turn]) * inverse;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (lane + u * L) * kRowUnit;
            float dh[kRowUnit] = {};
            if (dH) unit_values<VT>(raw_dh[u], dim - col, 0.f, dh);
            float dx[kRowUnit];
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) dx[j] = fmaf(rstd, fmaf(-dot, x[u][j], dy[u][j]), dh[j]);
            store_row_unit<VT>((S*)C.dX + row * dim + col, dim - col, dx);
        }
    }
    if (!parts) return;
    float* out = parts + (int64_t)blockIdx.x * dim;
    if constexpr (kTeams == 1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = (lane + u * L) * kRowUnit;
            store_row_unit<MAXK_VALUE_F32>(out + col, dim - col, total[u]);
        }
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < kRowUnit; ++j) sums[(team * U + u) * L * kRowUnit + lane * kRowUnit + j] = total[u][j];
        __syncthreads();
        for (int col = threadIdx.x; col < dim; col += norm_threads(L)) {
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < kTeams; ++t) sum += sums[t * kCols + col];
            out[col] = sum;
        }
    }
}

// dgamma of the workgroups' sums: 16 columns and 64 ranges of them a workgroup
constexpr int kRanges = 64;
__global__ void __launch_bounds__(16 * kRanges) add_parts_kernel(const float* parts, int n, int dim, float* dgamma)
{
    __shared__ double room[kRanges][17];
    const int c = threadIdx.x & 15, at = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    double sum = 0.0;
    if (col < dim) {
#pragma unroll 8
        for (int i = at; i < n; i += kRanges) sum += (double)parts[(int64_t)i * dim + col];
    }
    room[at][c] = sum;
    for (int half = kRanges / 2; half > 0; half /= 2) {
        __syncthreads();
        if (at < half) room[at][c] += room[at + half][c];
    }
    if (at == 0 && col < dim) dgamma[col] = (float)room[0][c];
}

// Lanes of a row and units of a lane: of the forms below the one with the fewest lanes and units that a row fills
struct RowForm { int lanes, units; };
RowForm row_form(int dim)
{
    const int units = (dim + kRowUnit - 1) / kRowUnit;
    constexpr RowForm forms[] = {{4, 1}, {8, 1}, {16, 1}, {32, 1}, {16, 3}, {64, 1}, {32, 3}, {64, 2}, {64, 3}, {64, 4}, {256, 2}, {256, 4}, {1024, 2}};
    for (const RowForm& f : forms)
        if (units <= f.lanes * f.units) return f;
    return {0, 0};
}

int teams_of(const RowForm& f) { return norm_threads(f.lanes) / f.lanes; }

template <typename F>
maxk_status with_form(const RowForm& f, F&& call)
{
#define MAXK_FORM(L, U) \
    if (f.lanes == L && f.units == U) return call(std::integral_constant<int, L>{}, std::integral_constant<int, U>{})
    MAXK_FORM(4, 1);
    MAXK_FORM(8, 1);
    MAXK_FORM(16, 1);
    MAXK_FORM(32, 1);
    MAXK_FORM(16, 3);
    MAXK_FORM(64, 1);
    MAXK_FORM(32, 3);
    MAXK_FORM(64, 2);
    MAXK_FORM(64, 3);
    MAXK_FORM(64, 4);
    MAXK_FORM(256, 2);
    MAXK_FORM(256, 4);
    MAXK_FORM(1024, 2);
#undef MAXK_FORM
    return MAXK_UNSUPPORTED;
}

constexpr int kMostGroups = 8192;

int64_t norm_groups(int64_t N, int dim)
{
    const int teams = teams_of(row_form(dim));
    return std::min<int64_t>((N + teams - 1) / teams, kMostGroups);
}

// The gradient's leave a row of dim sums each: 8 rows for each, so that these are few beside them, and four of 256 threads on a CU at most.
int64_t grad_groups(int64_t N, int dim)
{
    const int teams = teams_of(row_form(dim));
    const int64_t all = (N + teams - 1) / teams, resident = 4 * 256 * kThreads / norm_threads(row_form(dim).lanes);
    return all <= 4 ? 1 : std::min({all, resident, std::max<int64_t>(256, N / 8)});  // (a few rounds of one workgroup cost less than a second launch)
}

template <int VT>
maxk_status norm(const NormCall& C, int64_t N, int dim, hipStream_t s)
{
    return with_form(row_form(dim), [&](auto L, auto U) -> maxk_status {
        hipLaunchKernelGGL((norm_kernel<VT, L.value, U.value>), dim3((unsigned)norm_groups(N, dim)), dim3(norm_threads(L.value)), 0, s, C, N, dim);
        MAXK_LAUNCH_CHECK();
        return MAXK_OK;
    });
}

template <int VT>
maxk_status norm_grad(const NormGradCall& C, int64_t N, int dim, hipStream_t s)
{
    const int64_t groups = grad_groups(N, dim);
    float* parts = !C.dgamma ? nullptr : groups == 1 ? C.dgamma : C.workspace;
    const maxk_status st = with_form(row_form(dim), [&](auto L, auto U) -> maxk_status {
        hipLaunchKernelGGL((norm_grad_kernel<VT, L.value, U.value>), dim3((unsigned)groups), dim3(norm_threads(L.value)), 0, s, C, parts, N, dim);
        MAXK_LAUNCH_CHECK();
        return MAXK_OK;
    });
    if (st != MAXK_OK || !C.dgamma || groups == 1) return st;
    hipLaunchKernelGGL(add_parts_kernel, dim3((dim + 15) / 16), dim3(16 * kRanges), 0, s, parts, (int)groups, dim, C.dgamma);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace

maxk_status launch_rms_norm(const NormCall& C, int value_type, int64_t N, int dim, hipStream_t s)
{
    if (value_type == MAXK_VALUE_F32) return norm<MAXK_VALUE_F32>(C, N, dim, s);
    if (value_type == MAXK_VALUE_BF16) return norm<MAXK_VALUE_BF16>(C, N, dim, s);
    return norm<MAXK_VALUE_F16>(C, N, dim, s);
}

int64_t rms_norm_grad_workspace(int64_t N, int dim)
{
    return std::max<int64_t>(16, N == 0 ? 0 : grad_groups(N, dim) * dim * (int64_t)sizeof(float));
}

maxk_status launch_rms_norm_grad(const NormGradCall& C, int value_type, int64_t N, int dim, hipStream_t s)
{
    if (N == 0) return C.dgamma ? launch_fill_zero(C.dgamma, dim, s) : MAXK_OK;
    if (value_type == MAXK_VALUE_F32) return norm_grad<MAXK_VALUE_F32>(C, N, dim, s);
    if (value_type == MAXK_VALUE_BF16) return norm_grad<MAXK_VALUE_BF16>(C, N, dim, s);
    return norm_grad<MAXK_VALUE_F16>(C, N, dim, s);
}

}  // namespace maxk
