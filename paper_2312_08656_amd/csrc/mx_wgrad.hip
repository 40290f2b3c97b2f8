// Weight gradient from a microscaled checkpoint (include/maxk.h): dW = dH^T X over N rows, and db.
//
// A product with few outputs and a long sum, on bf16 matrix instructions with fp32 accumulators.  X is exact in bf16 in either format.  An fp32
// gradient is cut into three bf16 parts of 8 bits that add up to it exactly, fp16 into two: every product is exact, and only the
// sums round, as in fp32.  A CBSR gradient is spread over a row of zeros in LDS, so it is read as k values and columns.
//
// Rows are cut into ranges.  A workgroup owns a tile of dW for a range; it has GR groups of wavefronts that take its steps of 32 rows in
// turn, each with its own tiles of X and dH in LDS, and adds the groups' sums up in LDS at the end.  With two groups one fills its tiles while the other
// multiplies.  The ranges' sums go to the workspace and a second kernel adds them up, always in the same order.
#include <algorithm>

#include "mx_parts.hpp"

namespace maxk {
namespace {

constexpr int kStep = 32;  // rows

// GR groups of WO x WI wavefronts; a wavefront has 64 rows of dW (columns of dH) and 32 * WIT of its columns
template <int GR_, int WO_, int WI_, int WIT_>
struct Shape {
    static constexpr int GR = GR_, WO = WO_, WI = WI_, WIT = WIT_;
    static constexpr int TO = 64 * WO, TI = 32 * WIT * WI, WAVES = WO * WI, THREADS = 64 * GR * WAVES;
    static constexpr int ACC = 2 * WIT * 16;               // accumulators a lane
    static constexpr int TILE = WAVES * 64 * ACC;          // outputs
    static constexpr int KGW = 4 / WAVES;                  // of the four runs of 8 rows of a step: those whose dH a wavefront brings
    static constexpr int XITEMS = TI / 4 * 8 / (64 * WAVES);  // pieces of 4 columns x 4 rows of X a thread brings
};
using Small = Shape<8, 1, 1, 2>;   // 64 x 64: a wavefront a group
using Middle = Shape<2, 2, 2, 2>;  // 128 x 128
using Wide = Shape<2, 4, 1, 4>;    // 256 x 128

enum Kind { kCbsr, kF32, kBf16, kF16 };
__host__ __device__ constexpr int parts_of(int kind) { return kind == kBf16 ? 1 : kind == kF16 ? 2 : 3; }

struct Args {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t N;
    int din, dout, nb;
    MxGrad G;
    int64_t ranges;
    int otiles, itiles;
    float* sums;   // [ranges][tiles][TILE]
    float* dbsums; // [ranges][otiles * TO], or null
    float* dW;     // written at once where there is one range
    float* db;
};

constexpr int kEntries = 4;  // entries of a run of 8 CBSR rows that a lane has under way (k <= 32: all of them)

template <class S, int FMT, int KIND>
__global__ void __launch_bounds__(S::THREADS) weight_grad_kernel(const Args A)
{
    constexpr int P = parts_of(KIND), XBYTES = S::TI * 64, DPART = S::TO * 64, GROUP = XBYTES + P * DPART;
    constexpr int LOOP = S::GR * GROUP, JOIN = S::GR / 2 * S::TILE * 4, DBS = S::GR * S::TO * 4;
    __shared__ __align__(16) uint8_t lds[(LOOP > JOIN ? LOOP : JOIN) > DBS ? (LOOP > JOIN ? LOOP : JOIN) : DBS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave / S::WAVES, w = wave % S::WAVES;
    const int wo = w % S::WO, wi = w / S::WO;
    // a range's tiles run on one XCD, whose L2 holds the rows that they share
    const int tiles = A.otiles * A.itiles, at = blockIdx.x / 8, xcd = blockIdx.x % 8;
    const int tile = at % tiles;
    const int64_t range = (int64_t)(at / tiles) * 8 + xcd;
    if (range >= A.ranges) return;
    const int o0 = tile / A.itiles * S::TO, i0 = tile % A.itiles * S::TI;
    const int64_t all_steps = (A.N + kStep - 1) / kStep, first = all_steps * range / A.ranges, last = all_steps * (range + 1) / A.ranges;
    const int rounds = (int)((last - first + S::GR - 1) / S::GR);
    uint8_t* const xtile = lds + group * GROUP;
    uint8_t* const dtile = xtile + XBYTES;

    // what this thread brings of X: 4 columns of 4 rows; their places in LDS are [8 rows][column][row], columns 4c + j at j * TI / 4 + c
    const int xrow_bytes = A.nb * (FMT == MAXK_MX_8 ? 32 : 16);
    int xrow[S::XITEMS], xcol[S::XITEMS], xput[S::XITEMS], xblock[S::XITEMS];
#pragma unroll
    for (int n = 0; n < S::XITEMS; ++n) {
        const int item = w * 64 + lane + n * 64 * S::WAVES, half = item & 1, c = (item >> 1) % (S::TI / 4), run = (item >> 1) / (S::TI / 4);
        const int col = min(i0 + 4 * c, A.nb * kMxBlock - 4);
        xrow[n] = run * 8 + half * 4;
        xcol[n] = FMT == MAXK_MX_8 ? col : col / 2;
        xblock[n] = col / kMxBlock;
        xput[n] = (run * S::TI + c) * 16 + half * 8;
    }
    // and of dH: runs of 8 rows, whole
    int erow[kEntries];  // CBSR: row of the lane's entries in a run
    if constexpr (KIND == kCbsr) {
#pragma unroll
        for (int e = 0; e < kEntries; ++e) erow[e] = (lane + 64 * e) / A.G.k;
    }

    uint32_t xcode[S::XITEMS][4], xscale[S::XITEMS][4];
    constexpr int VALS = KIND == kCbsr ? kEntries : S::TO / 64 * 8;
    float val[S::KGW][VALS];
    uint32_t idx[S::KGW][KIND == kCbsr ? kEntries : 1];

    const auto index_at = [&](int64_t p) -> uint32_t {
        return A.G.index_bytes == 1 ? ((const uint8_t*)A.G.sp_index)[p] : A.G.index_bytes == 2 ? ((const uint16_t*)A.G.sp_index)[p] : ((const uint32_t*)A.G.sp_index)[p];
    };
    const auto load = [&](int round) {
        const int64_t row0 = min((first + (int64_t)round * S::GR + group) * kStep, A.N - 1);
        const int lim = (int)min(A.N - 1 - row0, (int64_t)kStep - 1);  // the last row that is there; rows past it are read from it, and are multiplied by 0
        const uint8_t* codes = A.codes + row0 * xrow_bytes;
        const uint8_t* scales = A.scales + row0 * A.nb;
#pragma unroll
        for (int n = 0; n < S::XITEMS; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = min(xrow[n] + j, lim);
                const uint8_t* p = codes + (uint32_t)(row * xrow_bytes + xcol[n]);
                xcode[n][j] = FMT == MAXK_MX_8 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
                xscale[n][j] = scales[(uint32_t)(row * A.nb + xblock[n])];
            }
#pragma unroll
        for (int q = 0; q < S::KGW; ++q) {
            const int run = w * S::KGW + q;
            if constexpr (KIND == kCbsr) {
                const float* v = (const float*)A.G.values + row0 * A.G.k;
                const int end = (lim + 1) * A.G.k - 1;
#pragma unroll
                for (int e = 0; e < kEntries; ++e) {
                    const int p = min(run * 8 * A.G.k + lane + 64 * e, end);
                    val[q][e] = v[(uint32_t)p];
                    idx[q][e] = index_at(row0 * A.G.k + p);
                }
            } else {
#pragma unroll
                for (int c = 0; c < S::TO / 64; ++c) {
                    const int o = min(o0 + c * 64 + lane, A.dout - 1);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int64_t p = row0 * A.dout + (uint32_t)(min(run * 8 + j, lim) * A.dout + o);
                        if constexpr (KIND == kF32) val[q][c * 8 + j] = ((const float*)A.G.values)[p];
                        else val[q][c * 8 + j] = __uint_as_float(((const uint16_t*)A.G.values)[p]);  // widened when it is used
                    }
                }
            }
        }
    };

    const auto put_entry = [&](int run, int row, uint32_t column, float x, int rows) {
        const uint32_t o = column - (uint32_t)o0;
        if (row < 8 && run * 8 + row < rows && o < (uint32_t)S::TO) {
            float part[3];
            split<P>(x, part);
#pragma unroll
            for (int p = 0; p < P; ++p)
                *reinterpret_cast<uint16_t*>(dtile + p * DPART + (run * S::TO + o) * 16 + row * 2) = (uint16_t)(__float_as_uint(part[p]) >> 16);
        }
    };
    const auto fill = [&](int round) {
        const int64_t row0 = (first + (int64_t)round * S::GR + group) * kStep;
        const int rows = (int)max((int64_t)0, min(min(last * kStep, A.N) - row0, (int64_t)kStep));
#pragma unroll
        for (int n = 0; n < S::XITEMS; ++n) {
            float x[4][4];  // [row][column]
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (FMT == MAXK_MX_8) {
                    const float unit = mx8_unit(xscale[n][j]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[j][c] = (float)(int8_t)(xcode[n][j] >> (8 * c)) * unit;
                } else {
                    const float scale = mx_scale(xscale[n][j]);
                    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(xcode[n][j], scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(xcode[n][j], scale, 1);
                    x[j][0] = a[0], x[j][1] = a[1], x[j][2] = b[0], x[j][3] = b[1];
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *reinterpret_cast<uint2*>(xtile + xput[n] + c * (S::TI / 4) * 16) = make_uint2(uppers(x[0][c], x[1][c]), uppers(x[2][c], x[3][c]));
        }
#pragma unroll
        for (int q = 0; q < S::KGW; ++q) {
            const int run = w * S::KGW + q;
            if constexpr (KIND == kCbsr) {
                // a run's zeros and its entries come from one wavefront, whose LDS operations stay in order
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int c = 0; c < S::TO / 64; ++c)
                        *reinterpret_cast<uint4*>(dtile + p * DPART + (run * S::TO + c * 64 + lane) * 16) = make_uint4(0, 0, 0, 0);
                wave_fence();
#pragma unroll
                for (int e = 0; e < kEntries; ++e) put_entry(run, erow[e], idx[q][e], val[q][e], rows);
                const int here = min(8, rows - run * 8) * A.G.k;
                for (int e = lane + 64 * kEntries; e < here; e += 64) {  // k above 32
                    const int64_t p = (row0 + run * 8) * A.G.k + e;
                    put_entry(run, e / A.G.k, index_at(p), ((const float*)A.G.values)[p], rows);
                }
            } else {
#pragma unroll
                for (int c = 0; c < S::TO / 64; ++c) {
                    float part[8][3];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float x = val[q][c * 8 + j];
                        if constexpr (KIND == kBf16) x = widen_value<MAXK_VALUE_BF16>((uint16_t)__float_as_uint(x));
                        if constexpr (KIND == kF16) x = widen_value<MAXK_VALUE_F16>((uint16_t)__float_as_uint(x));
                        split<P>(run * 8 + j < rows ? x : 0.f, part[j]);
                    }
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        *reinterpret_cast<uint4*>(dtile + p * DPART + (run * S::TO + c * 64 + lane) * 16) =
                            make_uint4(uppers(part[0][p], part[1][p]), uppers(part[2][p], part[3][p]), uppers(part[4][p], part[5][p]), uppers(part[6][p], part[7][p]));
                }
            }
        }
    };

    f32x16 sum[2][S::WIT];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < S::WIT; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[a][b][r] = 0.f;
    const bool sums_db = A.dbsums && i0 == 0 && wi == 0;
    float dbsum[2] = {0.f, 0.f};
    const auto multiply = [&]() {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int run = 2 * h + (lane >> 5), l = lane & 31;
            bf16x8 x[S::WIT];
#pragma unroll
            for (int b = 0; b < S::WIT; ++b) x[b] = *reinterpret_cast<const bf16x8*>(xtile + (run * S::TI + (wi * S::WIT + b) * 32 + l) * 16);
#pragma unroll
            for (int p = P - 1; p >= 0; --p)  // the smallest first
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const bf16x8 d = *reinterpret_cast<const bf16x8*>(dtile + p * DPART + (run * S::TO + wo * 64 + a * 32 + l) * 16);
#pragma unroll
                    for (int b = 0; b < S::WIT; ++b) sum[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d, x[b], sum[a][b], 0, 0, 0);
                    if (sums_db) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) dbsum[a] += (float)d[j];
                    }
                }
        }
    };
    const auto sync = [&]() {
        if constexpr (S::WAVES == 1) wave_fence();
        else local_fence();
    };

    load(0);
    if constexpr (S::WAVES > 1) {
        if (group & 1) local_fence();  // half a round behind the other group
    }
    for (int round = 0; round < rounds; ++round) {
        fill(round);
        sync();
        load(round + 1);
        multiply();
        sync();
    }
    if constexpr (S::WAVES > 1) {
        if (!(group & 1)) local_fence();
    }
    local_fence();

    // the groups' sums: the upper half of the groups hands its own over, until one is left
    float* const room = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int half = S::GR / 2; half >= 1; half /= 2) {
        float* mine = room + ((group % half) * S::WAVES + w) * 64 * S::ACC + lane;
        if (group >= half && group < 2 * half) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int b = 0; b < S::WIT; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) mine[((a * S::WIT + b) * 16 + r) * 64] = sum[a][b][r];
        }
        local_fence();
        if (group < half) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int b = 0; b < S::WIT; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum[a][b][r] += mine[((a * S::WIT + b) * 16 + r) * 64];
        }
        local_fence();
    }
    if (sums_db) {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const float s = dbsum[a] + __shfl_xor(dbsum[a], 32);
            if (lane < 32) room[group * S::TO + wo * 64 + a * 32 + lane] = s;
        }
    }
    local_fence();
    if (A.dbsums && i0 == 0) {
        for (int o = threadIdx.x; o < S::TO; o += S::THREADS) {
            float s = 0.f;
#pragma unroll
            for (int g = 0; g < S::GR; ++g) s += room[g * S::TO + o];
            if (A.ranges > 1) A.dbsums[range * A.otiles * S::TO + o0 + o] = s;
            else if (o0 + o < A.dout) A.db[o0 + o] = s;
        }
    }
    if (group != 0) return;
    if (A.ranges > 1) {
        float* out = A.sums + ((range * tiles + tile) * S::WAVES + w) * 64 * S::ACC + lane;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < S::WIT; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) out[((a * S::WIT + b) * 16 + r) * 64] = sum[a][b][r];
    } else {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < S::WIT; ++b) {
                const int p = (wi * S::WIT + b) * 32 + (lane & 31), i = i0 + p % (S::TI / 4) * 4 + p / (S::TI / 4);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int o = o0 + wo * 64 + a * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
                    if (o < A.dout && i < A.din) A.dW[(int64_t)o * A.din + i] = sum[a][b][r];
                }
            }
    }
}

// dW and db from the ranges' sums: 64 outputs a workgroup, its four wavefronts a quarter of the ranges each
template <class S>
__global__ void __launch_bounds__(256) add_ranges_kernel(const Args A)
{
    __shared__ float quarter[4][64];
    const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, tiles = A.otiles * A.itiles;
    const int64_t outputs = (int64_t)tiles * S::TILE;
    const int64_t at = (int64_t)blockIdx.x * 64 + lane;
    const bool is_db = at >= outputs;
    const int64_t stride = is_db ? (int64_t)A.otiles * S::TO : outputs;
    const float* p = is_db ? A.dbsums + (at - outputs) : A.sums + at;
    float s = 0.f;
#pragma unroll 8
    for (int64_t r = A.ranges * q / 4; r < A.ranges * (q + 1) / 4; ++r) s += p[r * stride];
    quarter[q][lane] = s;
    __syncthreads();
    if (q) return;
    s = (quarter[0][lane] + quarter[1][lane]) + (quarter[2][lane] + quarter[3][lane]);
    if (is_db) {
        if (at - outputs < A.dout) A.db[at - outputs] = s;
        return;
    }
    const int tile = (int)(at / S::TILE), in = (int)(at % S::TILE), w = in / (64 * S::ACC), reg = in / 64 % S::ACC;
    const int wo = w % S::WO, wi = w / S::WO, a = reg / (16 * S::WIT), b = reg / 16 % S::WIT, r = reg % 16;
    const int pos = (wi * S::WIT + b) * 32 + (lane & 31), i = tile % A.itiles * S::TI + pos % (S::TI / 4) * 4 + pos / (S::TI / 4);
    const int o = tile / A.itiles * S::TO + wo * 64 + a * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
    if (o < A.dout && i < A.din) A.dW[(int64_t)o * A.din + i] = s;
}

struct Plan {
    int shape;  // 0 Small, 1 Middle, 2 Wide
    int otiles, itiles;
    int64_t ranges, sums, dbsums;  // floats of the workspace
};

template <class S>
Plan plan_of(int shape, int64_t N, int din, int dout)
{
    Plan p;
    p.shape = shape;
    p.otiles = (dout + S::TO - 1) / S::TO;
    p.itiles = (din + S::TI - 1) / S::TI;
    const int64_t tiles = (int64_t)p.otiles * p.itiles, steps = (N + kStep - 1) / kStep;
    const int64_t resident = S::ACC > 64 ? 256 : 512;  // workgroups that run at a time
    // each of them once, if every group has two steps
    p.ranges = std::max<int64_t>(1, std::min(resident / tiles, steps / (2 * S::GR)));
    p.sums = p.ranges * tiles * S::TILE;
    p.dbsums = p.ranges * p.otiles * S::TO;
    return p;
}

Plan plan(int64_t N, int din, int dout)
{
    if (din <= 64 && dout <= 64) return plan_of<Small>(0, N, din, dout);
    if (dout > 128 && (dout + 255) / 256 * 2 == (dout + 127) / 128) return plan_of<Wide>(2, N, din, dout);
    return plan_of<Middle>(1, N, din, dout);
}

template <class S, int FMT, int KIND>
maxk_status run(const Args& A, hipStream_t s)
{
    const int64_t tiles = (int64_t)A.otiles * A.itiles, grid = (A.ranges + 7) / 8 * tiles * 8;
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
    hipLaunchKernelGGL((weight_grad_kernel<S, FMT, KIND>), dim3((unsigned)grid), dim3(S::THREADS), 0, s, A);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <class S>
maxk_status run_shape(const Args& A, int format, hipStream_t s)
{
    maxk_status st;
#define MAXK_KIND(KIND) st = format == MAXK_MX_8 ? run<S, MAXK_MX_8, KIND>(A, s) : run<S, MAXK_MX_4, KIND>(A, s)
    if (A.G.k) MAXK_KIND(kCbsr);
    else if (A.G.value_type == MAXK_VALUE_F32) MAXK_KIND(kF32);
    else if (A.G.value_type == MAXK_VALUE_BF16) MAXK_KIND(kBf16);
    else MAXK_KIND(kF16);
#undef MAXK_KIND
    if (st != MAXK_OK || A.ranges == 1) return st;
    const int64_t outputs = (int64_t)A.otiles * A.itiles * S::TILE + (A.dbsums ? (int64_t)A.otiles * S::TO : 0);
    hipLaunchKernelGGL((add_ranges_kernel<S>), dim3((unsigned)(outputs / 64)), dim3(256), 0, s, A);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace

int64_t mx_weight_grad_workspace(int64_t N, int din, int dout)
{
    const Plan p = plan(N, din, dout);
    return (p.sums + p.dbsums) * (int64_t)sizeof(float);
}

maxk_status launch_mx_weight_grad(const MxMatrix& X, int64_t N, int din, int dout, const MxGrad& G, float* dW, float* db, float* workspace,
                                  hipStream_t s)
{
    if (N == 0) {
        if (const maxk_status st = launch_fill_zero(dW, (int64_t)dout * din, s)) return st;
        return db ? launch_fill_zero(db, dout, s) : MAXK_OK;
    }
    const Plan p = plan(N, din, dout);
    const Args A = {X.codes, X.scales, N, din, dout, mx_blocks(din), G, p.ranges, p.otiles, p.itiles, workspace, db ? workspace + p.sums : nullptr, dW, db};
    return p.shape == 0 ? run_shape<Small>(A, X.format, s) : p.shape == 1 ? run_shape<Middle>(A, X.format, s) : run_shape<Wide>(A, X.format, s);
}

}  // namespace maxk
