// Weight gradient from a microscaled checkpoint (include/maxk.h): dW = dH^T X over N rows, and db.
//
// A product with few outputs and a long sum, on bf16 matrix instructions with fp32 accumulators.  X is exact in bf16 in either format.  An fp32
// gradient is cut into three bf16 parts of 8 bits that add up to it exactly, fp16 into two (mx_parts.hpp): every product is exact, and only the
// sums round, as in fp32.  A CBSR gradient is spread over a row of zeros in LDS, so it is read as k values and columns.
//
// Rows are cut into ranges.  A workgroup owns a tile of dW for a range; it has GR groups of wavefronts that take its steps of 32 rows in
// turn, each with its own tiles of X and dH in LDS, and adds the groups' sums up in LDS at the end.  With two groups one fills its tiles while the other
// multiplies.  The ranges' sums go to the workspace and a second kernel adds them up, always in the same order.
//
// What it takes, 233 thousand rows, 256 x 256, CBSR k = 32: 84 to 90 us by the card's clock, of which 7 are the second kernel and 15 the start, the joining of groups and 32 MB
// of sums on their way out; the rounds run at 60 % of what the three parts' products alone would (bound by the barriers between two groups that take turns; matrix
// units 44 % busy, LDS a third).  Where it took 82: without db 80, without bringing dH and X 54 and those 22.  2.4 M rows, 64 x 64, dense fp32: 158 us (4.9 TB/s, memory);
// 717 thousand, 384 x 384, from 4 bits: bf16 281 to 303 us (2.4 TB/s; a phase of products is short against the way to memory, and the registers hold one round's values),
// fp16 484 to 503 (two parts).
#include <algorithm>
#include <type_traits>

#include "mx_parts.hpp"

namespace maxk {
namespace {

constexpr int kStep = 32;      // rows
constexpr int kTogether = 16;  // ranges from which a range's tiles share an XCD

// GR groups of WO x WI wavefronts; a wavefront has 64 rows of dW (columns of dH) and 32 * WIT of its columns
template <int GR_, int WO_, int WI_, int WIT_>
struct Shape {
    static constexpr int GR = GR_, WO = WO_, WI = WI_, WIT = WIT_;
    static constexpr int TO = 64 * WO, TI = 32 * WIT * WI, WAVES = WO * WI, LANES = 64 * WAVES, THREADS = GR * LANES;
    static constexpr int ACC = 2 * WIT * 16;                // accumulators a lane
    static constexpr int TILE = LANES * ACC;                // outputs
    static constexpr int KGW = 4 / WAVES;                   // of the four runs of 8 rows of a step: those whose CBSR entries a wavefront brings
    static constexpr int XITEMS = TI / 16 * kStep / LANES;  // pieces of 16 columns of a row of X that a lane brings
};
using Small = Shape<8, 1, 1, 2>;   // 64 x 64: a wavefront a group
using Middle = Shape<2, 2, 2, 2>;  // 128 x 128
using Wide = Shape<2, 4, 1, 4>;    // 256 x 128

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

// E: entries of a run of 8 CBSR rows that a lane has under way (k / 8, up to 16; those of wider rows come in turns)
template <class S, int FMT, int KIND, int E>
__global__ void __launch_bounds__(S::THREADS) weight_grad_kernel(const Args A)
{
    constexpr bool CBSR = KIND <= kCbsr4;
    constexpr int P = parts_of(KIND), VT = type_of(KIND), V = piece_of(KIND);
    constexpr int XPITCH = S::TI * 2, DPITCH = S::TO * 2, XBYTES = kStep * XPITCH, DPART = kStep * DPITCH, GROUP = XBYTES + P * DPART;
    constexpr int LOOP = S::GR * GROUP, JOIN = S::GR / 2 * S::TILE * 4;
    // db: sums of a lane's operands, or of its columns over the rows that it brings; a copy each for what no lane adds up
    constexpr int PIECES = S::TO / V, DITEMS = CBSR ? 1 : PIECES * kStep / S::LANES, COPIES = S::GR * (CBSR ? 1 : S::LANES / PIECES);
    static_assert(CBSR || S::LANES % PIECES == 0);  // a lane's columns are the same in every row
    constexpr int DBS = COPIES * S::TO * 4, ROOM = LOOP > JOIN ? LOOP : JOIN, LDS = ROOM > DBS ? ROOM : DBS;
    __shared__ __align__(16) uint8_t lds[LDS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave / S::WAVES, w = wave % S::WAVES;
    const int wo = w % S::WO, wi = w / S::WO, me = w * 64 + lane;
    // a range's tiles run on one XCD, whose L2 holds the rows that they share; few ranges spread over all of them
    const int tiles = A.otiles * A.itiles, at = blockIdx.x / 8, xcd = blockIdx.x % 8;
    const bool together = A.ranges >= kTogether;
    const int tile = (together ? at : (int)blockIdx.x) % tiles;
    const int64_t range = together ? (int64_t)(at / tiles) * 8 + xcd : blockIdx.x / tiles;
    if (range >= A.ranges) return;
    const int o0 = tile / A.itiles * S::TO, i0 = tile % A.itiles * S::TI;
    const int64_t all_steps = (A.N + kStep - 1) / kStep, first = all_steps * range / A.ranges, last = all_steps * (range + 1) / A.ranges;
    const int rounds = (int)((last - first + S::GR - 1) / S::GR);
    uint8_t* const xtile = lds + group * GROUP;
    uint8_t* const dtile = xtile + XBYTES;
    // db is summed up once: for a dense gradient by the range's first tile, for a CBSR one, where it costs more, half each by the first two
    const int itile = tile % A.itiles, second = CBSR && A.itiles > 1 ? 1 : 0;
    const bool sums_db = A.dbsums && itile <= second, sums_even = A.dbsums && itile == 0, sums_odd = A.dbsums && itile == second;
    float* const dbcopies = reinterpret_cast<float*>(lds);

    // what this lane brings of X: 16 columns of a row
    constexpr int XWORDS = FMT == MAXK_MX_8 ? 4 : 2, XROW = S::TI / 16;
    const int xrow_bytes = A.nb * (FMT == MAXK_MX_8 ? 32 : 16), xcol = min(i0 + me % XROW * 16, A.nb * kMxBlock - 16);
    uint32_t xcode[S::XITEMS][XWORDS], xscale[S::XITEMS];
    int erow[E];  // CBSR: row of the lane's entries in a run
    if constexpr (CBSR) {
#pragma unroll
        for (int e = 0; e < E; ++e) erow[e] = (lane + 64 * e) / A.G.k;
    }
    constexpr int VALS = CBSR ? E : DITEMS * (V == 1 ? 1 : 4);
    float val[S::KGW][VALS];
    uint32_t idx[S::KGW][CBSR ? E : 1];
    float dbsum[CBSR ? 2 : V];  // CBSR: of the two blocks' column that is the lane's
#pragma unroll
    for (int j = 0; j < (CBSR ? 2 : V); ++j) dbsum[j] = 0.f;

    const auto load = [&](int round) {
        const int64_t row0 = min((first + (int64_t)round * S::GR + group) * kStep, A.N - 1);
        const int lim = (int)min(A.N - 1 - row0, (int64_t)kStep - 1);  // the last row that is there; rows past it are read from it, and are multiplied by 0
        const uint8_t* codes = A.codes + row0 * xrow_bytes;
        const uint8_t* scales = A.scales + row0 * A.nb;
#pragma unroll
        for (int n = 0; n < S::XITEMS; ++n) {
            const int row = min(me / XROW + n * (S::LANES / XROW), lim);
            const uint8_t* p = codes + (uint32_t)(row * xrow_bytes + (FMT == MAXK_MX_8 ? xcol : xcol / 2));
            if constexpr (FMT == MAXK_MX_8) *reinterpret_cast<uint4*>(xcode[n]) = *reinterpret_cast<const uint4*>(p);
            else *reinterpret_cast<uint2*>(xcode[n]) = *reinterpret_cast<const uint2*>(p);
            xscale[n] = scales[(uint32_t)(row * A.nb + xcol / kMxBlock)];
        }
        if constexpr (CBSR) {
            const float* v = (const float*)A.G.values + row0 * A.G.k;
            const column_t<KIND>* columns = (const column_t<KIND>*)A.G.sp_index + row0 * A.G.k;
            const int end = (lim + 1) * A.G.k - 1;
#pragma unroll
            for (int q = 0; q < S::KGW; ++q)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t p = (uint32_t)min((w * S::KGW + q) * 8 * A.G.k + lane + 64 * e, end);
                    val[q][e] = v[p];
                    idx[q][e] = columns[p];
                }
        } else {
            const value_store_t<VT>* values = (const value_store_t<VT>*)A.G.values + row0 * A.dout;
#pragma unroll
            for (int n = 0; n < DITEMS; ++n) {
                const int item = me + n * S::LANES;
                const uint32_t p = (uint32_t)(min(item / PIECES, lim) * A.dout + min(o0 + item % PIECES * V, A.dout - V));
                if constexpr (V > 1) *reinterpret_cast<f32x4*>(&val[0][n * 4]) = *reinterpret_cast<const f32x4*>(values + p);
                else if constexpr (VT == MAXK_VALUE_F32) val[0][n] = values[p];
                else val[0][n] = __uint_as_float(values[p]);  // widened when it is used
            }
        }
    };

    const auto put_entry = [&](int row, uint32_t column, float x) {
        const uint32_t o = column - (uint32_t)o0;
        if (o < (uint32_t)S::TO) {
            float part[3];
            split<P>(x, part);
#pragma unroll
            for (int p = 0; p < P; ++p)
                *reinterpret_cast<uint16_t*>(dtile + p * DPART + at_byte(row, (int)o * 2, DPITCH)) = (uint16_t)(__float_as_uint(part[p]) >> 16);
        }
    };
    const auto fill = [&](int round) {
        const int64_t row0 = (first + (int64_t)round * S::GR + group) * kStep;
        const int rows = (int)max((int64_t)0, min(min(last * kStep, A.N) - row0, (int64_t)kStep));
#pragma unroll
        for (int n = 0; n < S::XITEMS; ++n) {
            uint32_t x[8];
            if constexpr (FMT == MAXK_MX_8) {
                const float unit = mx8_unit(xscale[n]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t c = xcode[n][j / 2] >> (16 * (j & 1));
                    x[j] = uppers((float)(int8_t)c * unit, (float)(int8_t)(c >> 8) * unit);
                }
            } else {
                const float scale = mx_scale(xscale[n]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    x[4 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(xcode[n][j], scale, 0));
                    x[4 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(xcode[n][j], scale, 1));
                    x[4 * j + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(xcode[n][j], scale, 2));
                    x[4 * j + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(xcode[n][j], scale, 3));
                }
            }
            uint4* to = reinterpret_cast<uint4*>(xtile + at_byte(me / XROW + n * (S::LANES / XROW), me % XROW * 32, XPITCH));
            to[0] = make_uint4(x[0], x[1], x[2], x[3]);
            to[1] = make_uint4(x[4], x[5], x[6], x[7]);
        }
        if constexpr (CBSR) {
#pragma unroll
            for (int q = 0; q < S::KGW; ++q) {
                const int run = w * S::KGW + q;
                if constexpr (S::WI > 1) {  // a run's zeros and its entries come from one wavefront, whose LDS operations stay in order
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int c = 0; c < S::TO / 64; ++c) *reinterpret_cast<uint4*>(dtile + p * DPART + run * 8 * DPITCH + (c * 64 + lane) * 16) = make_uint4(0, 0, 0, 0);
                    wave_fence();
                }
                const int there = min(8, rows - run * 8);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (erow[e] < there) put_entry(run * 8 + erow[e], idx[q][e], val[q][e]);
                for (int e0 = 64 * E; e0 < there * A.G.k; e0 += 64 * E) {
                    const int64_t run0 = (row0 + run * 8) * A.G.k;
                    const int end = there * A.G.k - 1;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const uint32_t p = (uint32_t)min(e0 + lane + 64 * e, end);
                        val[q][e] = ((const float*)A.G.values + run0)[p];
                        idx[q][e] = ((const column_t<KIND>*)A.G.sp_index + run0)[p];
                    }
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (e0 + lane + 64 * e <= end) put_entry(run * 8 + (e0 + lane + 64 * e) / A.G.k, idx[q][e], val[q][e]);
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < DITEMS; ++n) {
                const int item = me + n * S::LANES, row = item / PIECES, byte = item % PIECES * V * 2;
                uint8_t* to = dtile + at_byte(row, byte, DPITCH);
                const bool there = row < rows;
                if constexpr (KIND == kBf16V) {  // as it is
                    uint4 u = __builtin_bit_cast(uint4, *reinterpret_cast<const f32x4*>(&val[0][n * 4]));
                    if (!there) u = make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4*>(to) = u;
                    const uint32_t word[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                    for (int j = 0; sums_db && j < 4; ++j) {
                        dbsum[2 * j] += __uint_as_float(word[j] << 16);
                        dbsum[2 * j + 1] += __uint_as_float(word[j] & 0xFFFF0000u);
                    }
                } else {
                    float part[V][3];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float x;
                        if constexpr (KIND == kF16V) x = widen_value<VT>((uint16_t)(__float_as_uint(val[0][n * 4 + j / 2]) >> (16 * (j & 1))));
                        else if constexpr (VT == MAXK_VALUE_F32) x = val[0][n * (V == 1 ? 1 : 4) + j];
                        else x = widen_value<VT>((uint16_t)__float_as_uint(val[0][n]));
                        x = there ? x : 0.f;
                        dbsum[j] += x;
                        split<P>(x, part[j]);
                    }
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        if constexpr (V == 8)
                            *reinterpret_cast<uint4*>(to + p * DPART) = make_uint4(uppers(part[0][p], part[1][p]), uppers(part[2][p], part[3][p]),
                                                                                   uppers(part[4][p], part[5][p]), uppers(part[6][p], part[7][p]));
                        else if constexpr (V == 4) *reinterpret_cast<uint2*>(to + p * DPART) = make_uint2(uppers(part[0][p], part[1][p]), uppers(part[2][p], part[3][p]));
                        else *reinterpret_cast<uint16_t*>(to + p * DPART) = (uint16_t)(__float_as_uint(part[0][p]) >> 16);
                    }
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
    // CBSR: the tile of dH is zeros between the steps.  Where one wavefront alone reads its 64 columns, it clears them as it goes, so that
    // the clearing is spread over the products and does not hold up the other group's first reads.
    constexpr bool CLEARS = CBSR && S::WI == 1;
    const auto clear_d = [&](int p, int half) {
        uint8_t* to = dtile + p * DPART + at_byte(half * 16 + lane / 8, wo * 128 + lane % 8 * 16, DPITCH);
        *reinterpret_cast<uint4*>(to) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(to + 8 * DPITCH) = make_uint4(0, 0, 0, 0);
    };
    // meanwhile: what else the wavefront has to do, once the first products are under way
    const auto multiply = [&](auto meanwhile) {
        // 2 halves of 16 rows x P parts (the smallest first) x 2 blocks of 32 columns of dH, each with all blocks of X; operands are read
        // AHEAD products before they are needed, the second half's of X meanwhile
        constexpr int STEPS = 4 * P, AHEAD = 2, MEANWHILE = 0;
        bf16x8 x[2][S::WIT], d[AHEAD + 1];
        const auto fetch_x = [&](int half, int b) { x[half][b] = transposed_operand(xtile, XPITCH, wi * S::WIT + b, half * 16, lane); };
        const auto fetch_d = [&](int t) { d[t % (AHEAD + 1)] = transposed_operand(dtile + (P - 1 - t % (2 * P) / 2) * DPART, DPITCH, wo * 2 + t % 2, t / (2 * P) * 16, lane); };
#pragma unroll
        for (int b = 0; b < S::WIT; ++b) fetch_x(0, b);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) fetch_d(t);
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
            if (t + AHEAD < STEPS) fetch_d(t + AHEAD);
            if (CLEARS && t % 2 == 1) clear_d(P - 1 - t % (2 * P) / 2, t / (2 * P));  // both blocks have been read
#pragma unroll
            for (int b = 0; b < S::WIT; ++b)
                if (t < 2 * P && b * 2 * P / S::WIT == t) fetch_x(1, b);
#pragma unroll
            for (int b = 0; b < S::WIT; ++b)
                sum[t % 2][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d[t % (AHEAD + 1)], x[t / (2 * P)][b], sum[t % 2][b], 0, 0, 0);
            if (CBSR && (t % 2 ? sums_odd : sums_even)) {  // db while the products run
                const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
                const bf16x8& y = d[t % (AHEAD + 1)];
                float even = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(y, y, 0, 1), one, dbsum[t % 2], false);
                even = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(y, y, 2, 3), one, even, false);
                even = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(y, y, 4, 5), one, even, false);
                dbsum[t % 2] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(y, y, 6, 7), one, even, false);
            }
            if (t == MEANWHILE) meanwhile();
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto sync = [&]() {
        if constexpr (S::WAVES == 1) wave_fence();
        else local_fence();
    };

    load(0);
    if constexpr (CLEARS) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int half = 0; half < 2; ++half) clear_d(p, half);
        sync();
    }
    if constexpr (S::WAVES > 1) {
        if (group & 1) local_fence();  // half a round behind the other group
    }
    for (int round = 0; round < rounds; ++round) {
        fill(round);
        if constexpr (CBSR) load(round + 1);  // (as many loads as a dense gradient's would hold up the barrier)
        sync();
        __builtin_amdgcn_s_setprio(3);  // products first: the other group's stores to LDS can wait, the operands cannot
        multiply([&]() {
            if constexpr (!CBSR) load(round + 1);
        });
        __builtin_amdgcn_s_setprio(0);
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
        if (last - first <= half) continue;  // the upper groups had no step
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
        if constexpr (CBSR) {
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const float both = dbsum[a] + __shfl_xor(dbsum[a], 32);  // the lanes' rows
                if (wi == 0 && lane < 32) dbcopies[group * S::TO + wo * 64 + a * 32 + lane] = both;
            }
        } else {
            float* mine = dbcopies + (group * (COPIES / S::GR) + me / PIECES) * S::TO + me % PIECES * V;
#pragma unroll
            for (int j = 0; j < V; ++j) mine[j] = dbsum[j];
        }
        local_fence();
        for (int o = threadIdx.x; o < S::TO; o += S::THREADS) {
            float s = 0.f;
#pragma unroll
            for (int g = 0; g < COPIES; ++g) s += dbcopies[g * S::TO + o];
            if (!(o & 32 ? sums_odd : sums_even)) continue;
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
                const int i = i0 + (wi * S::WIT + b) * 32 + (lane & 31);
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
    const int i = tile % A.itiles * S::TI + (wi * S::WIT + b) * 32 + (lane & 31);
    const int o = tile / A.itiles * S::TO + wo * 64 + a * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
    if (o < A.dout && i < A.din) A.dW[(int64_t)o * A.din + i] = s;
}

struct Plan {
    int shape;  // 0 Small, 1 Middle, 2 Wide
    int otiles, itiles;
    int64_t ranges, sums, dbsums;  // floats of the workspace: none where one range writes dW and db itself
};

template <class S>
Plan plan_of(int shape, int64_t N, int din, int dout)
{
    Plan p;
    p.shape = shape;
    p.otiles = (dout + S::TO - 1) / S::TO;
    p.itiles = (din + S::TI - 1) / S::TI;
    const int64_t tiles = (int64_t)p.otiles * p.itiles, steps = (N + kStep - 1) / kStep;
    // Workgroups that ranges are made for: one a CU, or two where a lane has 64 accumulators.  Two run at a time for aligned bf16 gradients as Middle alone; elsewhere LDS (Small)
    // or registers (Middle) leave room for one, and 512 take two turns.  us at 512 / 256: 717 thousand rows, 384 x 384, bf16 286 / 400; 200 thousand, fp32, 384 x 384 209 / 220,
    // 256 x 384 152 / 146; 2.4 M, 64 x 64, fp32 158 / 145, bf16 97 / 90, CBSR k = 8 105 / 95; 500 thousand, 100 x 100, k = 13 73 / 65.
    const int64_t resident = S::ACC > 64 ? 256 : 512, rounds = (steps + S::GR - 1) / S::GR;  // rounds of a single range
    // A round takes about 2 us, the second kernel 3 and more with more ranges: one range up to two rounds, a range each up to 32, then two rounds a range
    // until there are as many workgroups.  (us, 256 x 256 as Wide, CBSR k = 32: 256 rows 18.2 as one range / 12.5 as four; 4000 rows 19.8 as 31 / 21.7 as 63;
    // 64 x 64, 1024 rows, k = 8: 15.9 as one / 10.6 as four.)
    // Every XCD has an eighth of the ranges, and of the workgroups: one range more would take it another turn (384 x 384: 6 tiles).
    const int64_t most = tiles <= resident / 8 ? resident / 8 / tiles * 8 : std::max<int64_t>(1, resident / tiles);
    p.ranges = rounds <= 2 ? 1 : std::min(most, std::max(std::min<int64_t>(rounds, 32), rounds / 2));
    p.sums = p.ranges > 1 ? p.ranges * tiles * S::TILE : 0;
    p.dbsums = p.ranges > 1 ? p.ranges * p.otiles * S::TO : 0;
    return p;
}

// us, 200 thousand rows, din x dout, as Middle / Wide: CBSR k = 8, 64 x 384 83 / 74, 256 x 384 154 / 127, 384 x 384 212 / 195, k = 64 108 / 80, 207 / 141, 286 / 215 (every tile
// of dH looks at all entries of its rows); dense fp32 86 / 92, 152 / 165, 209 / 242, bf16 256 x 384 65 / 77; fp32 384 x 256, whose columns of dH fill Wide, 151 / 133.
Plan plan(int64_t N, int din, int dout, bool cbsr)
{
    // Few rows: small tiles, as long as 512 workgroups give all of them one for every round, with eight groups a round (256 run at a time).  us as above / so, CBSR k = 16: 256 x 256,
    // 100 rows 13.5 / 8.8, 4000 18.2 / 13.5; 384 x 384, 1000 rows 19.9 / 12.6, 8000 30.9 / 34.5; 64 x 256, 8000 rows 19.5 / 11.6.  One tile of Middle is its equal up to 4000 rows
    // (100 x 100: 500 rows 9.8 / 12.0, 8000 15.0 / 11.6).  Dense fp32: 256 x 256, 100 rows 12.7 / 8.0, 4000 17.9 / 12.6; 384 x 384, 1000 rows 14.8 / 11.5.
    const int64_t steps = (N + kStep - 1) / kStep, tiles = (int64_t)((din + 63) / 64) * ((dout + 63) / 64);
    const bool few = (steps + Small::GR - 1) / Small::GR * tiles <= 512 && (din > 128 || dout > 128 || steps > 128);
    if (few || (din <= 64 && dout <= 64)) return plan_of<Small>(0, N, din, dout);
    if (dout > 128 && (cbsr || (dout + 255) / 256 * 2 == (dout + 127) / 128)) return plan_of<Wide>(2, N, din, dout);
    return plan_of<Middle>(1, N, din, dout);
}

template <class S, int FMT, int KIND, int E = 1>
maxk_status run(const Args& A, hipStream_t s)
{
    const int64_t tiles = (int64_t)A.otiles * A.itiles, grid = (A.ranges >= kTogether ? (A.ranges + 7) / 8 * 8 : A.ranges) * tiles;
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
    hipLaunchKernelGGL((weight_grad_kernel<S, FMT, KIND, E>), dim3((unsigned)grid), dim3(S::THREADS), 0, s, A);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

template <class S>
maxk_status run_shape(const Args& A, int format, hipStream_t s)
{
    maxk_status st;
    constexpr int WIDEST = S::TO == 128 ? 16 : 8;  // (16 would not fit Wide's registers, and Small's rows are few or have k up to 64; of 8, Small spills 2 to 4 registers at two-byte columns)
    const bool pieces = aligned(A.G.values, 16) && A.dout * (A.G.value_type == MAXK_VALUE_F32 ? 4 : 2) % 16 == 0;  // rows of whole 16-byte pieces
#define MAXK_ENTRIES(KIND)                                                                                                                            \
    st = A.G.k <= 32   ? (format == MAXK_MX_8 ? run<S, MAXK_MX_8, KIND, 4>(A, s) : run<S, MAXK_MX_4, KIND, 4>(A, s))                                  \
         : A.G.k <= 64 ? (format == MAXK_MX_8 ? run<S, MAXK_MX_8, KIND, 8>(A, s) : run<S, MAXK_MX_4, KIND, 8>(A, s))                                  \
                       : (format == MAXK_MX_8 ? run<S, MAXK_MX_8, KIND, WIDEST>(A, s) : run<S, MAXK_MX_4, KIND, WIDEST>(A, s))
#define MAXK_KIND(KIND) st = format == MAXK_MX_8 ? run<S, MAXK_MX_8, KIND>(A, s) : run<S, MAXK_MX_4, KIND>(A, s)
    if (A.G.k && A.G.index_bytes == 1) MAXK_ENTRIES(kCbsr1);
    else if (A.G.k && A.G.index_bytes == 2) MAXK_ENTRIES(kCbsr2);
    else if (A.G.k) MAXK_ENTRIES(kCbsr4);
    else if (A.G.value_type == MAXK_VALUE_F32) {
        if (pieces) MAXK_KIND(kF32V);
        else MAXK_KIND(kF32);
    } else if (A.G.value_type == MAXK_VALUE_BF16) {
        if (pieces) MAXK_KIND(kBf16V);
        else MAXK_KIND(kBf16);
    } else {
        if (pieces) MAXK_KIND(kF16V);
        else MAXK_KIND(kF16);
    }
#undef MAXK_KIND
#undef MAXK_ENTRIES
    if (st != MAXK_OK || A.ranges == 1) return st;
    const int64_t outputs = (int64_t)A.otiles * A.itiles * S::TILE + (A.dbsums ? (int64_t)A.otiles * S::TO : 0);
    hipLaunchKernelGGL((add_ranges_kernel<S>), dim3((unsigned)(outputs / 64)), dim3(256), 0, s, A);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace

int64_t mx_weight_grad_workspace(int64_t N, int din, int dout)
{
    const Plan dense = plan(N, din, dout, false), cbsr = plan(N, din, dout, true);
    return std::max<int64_t>({16, (dense.sums + dense.dbsums) * (int64_t)sizeof(float), (cbsr.sums + cbsr.dbsums) * (int64_t)sizeof(float)});
}

maxk_status launch_mx_weight_grad(const MxMatrix& X, int64_t N, int din, int dout, const MxGrad& G, float* dW, float* db, float* workspace,
                                  hipStream_t s)
{
    if (N == 0) {
        if (const maxk_status st = launch_fill_zero(dW, (int64_t)dout * din, s)) return st;
        return db ? launch_fill_zero(db, dout, s) : MAXK_OK;
    }
    const Plan p = plan(N, din, dout, G.k > 0);
    const Args A = {X.codes, X.scales, N, din, dout, mx_blocks(din), G, p.ranges, p.otiles, p.itiles, workspace, db ? workspace + p.sums : nullptr, dW, db};
    return p.shape == 0 ? run_shape<Small>(A, X.format, s) : p.shape == 1 ? run_shape<Middle>(A, X.format, s) : run_shape<Wide>(A, X.format, s);
}

}  // namespace maxk
