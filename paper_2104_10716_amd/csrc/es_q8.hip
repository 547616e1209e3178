// es_q8.hip -- the entry points on 8-bit rows (include/es_spmm.h): argument checks and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "es_spmm.h"

#include "es_common.h"
#include "es_q8_rows.h"
#include "es_q8_spmm.h"
#include "es_q8_grad.h"

namespace {

constexpr int32_t kMaxF = INT32_MAX - 15;
constexpr int32_t kMaxValsF = 1 << 30;                         // es_q8_vals_kernel counts columns in 32 bits, past the last one
constexpr int kComputeUnits = 256;

int element_bytes(int32_t type) { return type == ES_FP32 ? 4 : type == ES_FP16 || type == ES_BF16 ? 2 : 0; }

bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

// A table of 8-bit rows as every entry point takes it.
int check_table(int64_t N, int32_t F, int32_t ldq)
{
    if (N < 0 || N > INT32_MAX || F < 1 || F > kMaxF || ldq % 16 || ldq < F) return ES_ERR_INVALID_ARG;
    return ES_OK;
}

bool bad_table(const int8_t* codes, const float* scale)
{
    return !codes || !scale || misaligned(codes, 16) || misaligned(scale, 4);
}

int next_pow2(int64_t v)
{
    int p = 1;
    while (p < v) p <<= 1;
    return p;
}

int launched() { return hipGetLastError() == hipSuccess ? ES_OK : ES_ERR_LAUNCH; }

// A launch holds fewer than 2^32 threads along x.
constexpr int64_t kMostBlocks = UINT32_MAX / kBlockThreads;
// Rows of a table that one launch writes or reads, a workgroup for each of them at most; longer lists take several.
constexpr int64_t kLaunchRows = (1 << 24) - 4096;
static_assert(kLaunchRows <= kMostBlocks && kQ8Claims <= kMostBlocks, "");

uint32_t blocks_of(int64_t items, int64_t per_block) { return (uint32_t)((items + per_block - 1) / per_block); }

// Lanes to a row of so many 16-byte accesses, accesses per lane, and rows at a time: the fewest idle lanes.  233 k rows of 602
// bf16 with 64 lanes throughout: written in 127 us and read in 100, this way 95 and 93; of 602 fp32: read in 188, 154.
#define ES_TEAMS(X) X(4, 1, 4) X(8, 1, 4) X(16, 1, 4) X(32, 1, 4) X(16, 3, 2) X(64, 1, 4) X(16, 5, 1) X(32, 3, 2) X(64, 2, 2) \
    X(32, 5, 1) X(64, 3, 1) X(64, 4, 1)

// The lanes that launch_write gives a row.
template <class T>
int write_team(int32_t F)
{
    const int64_t loads = ((int64_t)F + 15) / 16 * (16 / Dense<T>::V);
#define ES_TEAM(TEAM_, K_, UR_) if (loads <= (TEAM_) * (K_)) return TEAM_;
    ES_TEAMS(ES_TEAM)
#undef ES_TEAM
    return kWaveSize;
}

template <class T, int MAP>
int launch_write(const Q8Write& a, hipStream_t st)
{
    const int64_t loads = ((int64_t)a.F + 15) / 16 * (16 / Dense<T>::V);
#define ES_WRITE(TEAM_, K_, UR_)                                                                                            \
    if (loads <= (TEAM_) * (K_)) {                                                                                          \
        const uint32_t grid = blocks_of(a.n, (int64_t)(kBlockThreads / (TEAM_)) * (UR_));                                   \
        hipLaunchKernelGGL((es_q8_write_kernel<T, TEAM_, K_, UR_, MAP>), dim3(grid), dim3(kBlockThreads), 0, st, a);        \
        return launched();                                                                                                  \
    }
    ES_TEAMS(ES_WRITE)
    if constexpr (Dense<T>::V == 4) { ES_WRITE(64, 8, 1) }
#undef ES_WRITE
    hipLaunchKernelGGL((es_q8_write_wide_kernel<T, MAP>), dim3((uint32_t)a.n), dim3(kBlockThreads), 0, st, a);
    return launched();
}

template <class T>
int launch_read(const Q8Read& a, hipStream_t st)
{
    const int64_t stores = ((int64_t)a.F + Dense<T>::V - 1) / Dense<T>::V;
#define ES_READ(TEAM_, K_, UR_)                                                                                             \
    if (stores <= (TEAM_) * (K_) || (TEAM_) * (K_) == 256) {                                                                \
        const uint32_t grid = blocks_of(a.n, (int64_t)(kBlockThreads / (TEAM_)) * (UR_));                                   \
        hipLaunchKernelGGL((es_q8_read_kernel<T, TEAM_, K_, UR_>), dim3(grid), dim3(kBlockThreads), 0, st, a);              \
        return launched();                                                                                                  \
    }
    ES_READ(2, 1, 4)
    ES_TEAMS(ES_READ)
#undef ES_READ
    return ES_ERR_UNSUPPORTED;
}

template <class T>
int run_write(Q8Write a, hipStream_t st)
{
    const size_t row_bytes = (size_t)a.ldx * sizeof(T);
    const int64_t total = a.n;
    if (!a.rows) {
        for (int64_t done = 0; done < total; done += kLaunchRows) {
            Q8Write b = a;
            b.n = total - done < kLaunchRows ? total - done : kLaunchRows;
            b.X = static_cast<const char*>(a.X) + (size_t)done * row_bytes;
            b.codes = a.codes + done * a.ldq;
            b.scale = a.scale + done;
            const int rc = launch_write<T, Q8_ALL>(b, st);
            if (rc != ES_OK) return rc;
        }
        return ES_OK;
    }
    if (a.n <= kQ8Scan * write_team<T>(a.F)) return launch_write<T, Q8_SCANNED>(a, st);
    for (int64_t done = 0; done < total; done += kQ8Claims) {  // in order: a later piece's rows replace an earlier one's
        Q8Write b = a;
        b.n = total - done < kQ8Claims ? total - done : kQ8Claims;
        b.rows = a.rows + done;
        b.X = static_cast<const char*>(a.X) + (size_t)done * row_bytes;
        const uint32_t grid = blocks_of(b.n, kBlockThreads);
        hipLaunchKernelGGL(es_q8_claim_kernel<false>, dim3(grid), dim3(kBlockThreads), 0, st, b);
        if (launched() != ES_OK) return ES_ERR_LAUNCH;
        hipLaunchKernelGGL(es_q8_claim_kernel<true>, dim3(grid), dim3(kBlockThreads), 0, st, b);
        if (launched() != ES_OK) return ES_ERR_LAUNCH;
        const int rc = launch_write<T, Q8_CLAIMED>(b, st);
        if (rc != ES_OK) return rc;
    }
    return ES_OK;
}

template <class T>
int run_read(const Q8Read& a, hipStream_t st)
{
    for (int64_t done = 0; done < a.n; done += kLaunchRows) {
        Q8Read b = a;
        b.n = a.n - done < kLaunchRows ? a.n - done : kLaunchRows;
        b.Y = static_cast<T*>(a.Y) + done * a.ldy;
        if (a.rows) {
            b.rows = a.rows + done;
        } else {
            b.codes = a.codes + done * a.ldq;
            b.scale = a.scale + done;
            b.N = a.N - done;
        }
        const int rc = launch_read<T>(b, st);
        if (rc != ES_OK) return rc;
    }
    return ES_OK;
}

// What both products on a graph check.
int check_product(int64_t N, int64_t nnz, int32_t F, int32_t ldq, int32_t ld, int32_t W, int32_t mode, int32_t norm)
{
    if (check_table(N, F, ldq) != ES_OK || nnz < 0 || nnz > INT32_MAX || ld < F) return ES_ERR_INVALID_ARG;
    if (norm < ES_NORM_NONE || norm > ES_NORM_INV_DEGREE) return ES_ERR_INVALID_ARG;
    if (mode != ES_FULL && mode != ES_BUCKET && mode != ES_FASTRAND) return ES_ERR_INVALID_ARG;
    if (mode != ES_FULL && W < 1) return ES_ERR_INVALID_ARG;
    return ES_OK;
}

// Lanes to a row.  As few as cover its columns leave little to sum across lanes and the fewest lanes idle; half a wave
// is done with a row sooner, which counts where rows are few, or long and of very different lengths (uniform ids, us with G or 4 lanes /
// 32 / 64; m: mean length of the whole rows):
//  * exact, 2700 rows, F = 16, m = 5: 15.2 / 8.2 / 8.9, F = 64, m = 30: 18.8 / 10.1 / 9.3, m = 100: 45 / 12.4 / 10.8; 8000 rows: 15.6 /
//    8.3 / 9.6, 19.2 / 13.8 / 12.6, 51 / 20 / 20; 20 k rows: 17.8 / 14.1 / 17.5, 29 / 23 / 22, 82 / 41 / 40
//  * 60 k rows, F = 16, m = 5: 22 / 25 / 37, F = 64, m = 30: 56 / 48 / 55, F = 128, FastRand of 100, m = 100: 70 / 53 / 59
//  * 233 k rows, F = 64, m = 30: 162 / 148 / 172, Bucket 24: 60 / 64 / 112, exact, m = 490: 2402 / 1843 / 1827, F = 128: 2483 / 2137 /
//    2098, FastRand of 200, m = 200: 546 / 452 / 421, Bucket 32, m = 490: 111 / 117 / 124, F = 256, exact: 4365 / 4326 / 4415
//  * 700 k rows, F = 64, m = 30: 581 / 583 / 596, F = 19, Bucket 60, m = 150: 824 / 756 / 759, F = 128, m = 60: 1172 / 1187 / 1171, FastRand
//    of 200, m = 150: 1638 / 1528 / 1414; 2.45 M, F = 128, FastRand of 64, m = 49: 2151 / 2247 / 2131
// The edge gradient: 2700 rows, F = 64, m = 30: 19.8 / 9.4 / 7.9; 20 k: 28 / 22 / 22; 233 k, F = 64, m = 100: 545 / 401 / 415, F = 128, m = 5:
// 66 / 99 / 144.
// The rule goes by the mean kept; of these it loses 8 % (233 k, F = 64, m = 30), 7 % (FastRand of 200 on 233 k rows) and 14 % (on 700 k).
int pick_team(int G, int64_t n_rows, double mean)
{
    const int least = G < 4 ? 4 : G;
    if (n_rows <= 4096) return kWaveSize;
    if (n_rows <= 24'576) return G < 32 ? 32 : G;
    if (G <= 8 && mean >= 56.0 && (G <= 4 || n_rows <= 300'000 || mean >= 150.0)) return 32;
    if (G <= 8 && mean >= 28.0 && n_rows <= 98'304) return 32;
    return least;
}

// The same for the edge gradient of FastRand, whose kept entries wait in LDS: 256 of a row with 16 lanes, 512 with 32, 1024 with 64.
// The wider the sample, the more its rows differ in length.  16 / 32 / 64 lanes, us (m: mean of the whole row):
//  * 2700 rows, m = 14, F = 100, W = 100: 13.1 / 9.0 / 8.0; 8000 rows, m = 5, F = 16, W = 50: 7.2 / 7.0 / 8.2, m = 30, F = 128, W = 200: 25 / 19 / 15
//  * 60 k rows, m = 5, F = 128, W = 50: 33 / 35 / 53, m = 14, F = 100, W = 100: 50 / 47 / 68, m = 100, F = 128, W = 250: 128 / 95 / 97; F = 300,
//    m = 30, W = 16: - / 60 / 80, F = 400, W = 500: - / 245 / 191
//  * 233 k rows, m = 5, F = 128, W = 50: 93 / 111 / 155, m = 30, W = 200: 167 / 157 / 194, m = 100, W = 250: 312 / 304 / 293; F = 300, W = 16: - / 227 / 278,
//    F = 400, W = 500: - / 588 / 537; 700 k, m = 14, F = 100, W = 100: 412 / 519 / 658, m = 30, F = 128, W = 200: 460 / 481 / 597
int pick_random_team(int G, int64_t n_rows, int32_t W)
{
    const bool many = n_rows > 98'304;
    if (G > 32 || n_rows <= 4096 || W > 384 || (!many && W > (G <= 16 ? 224 : 127))) return kWaveSize;
    return G <= 16 && W <= 256 && (many || (W <= 64 && n_rows > 12'288)) ? 16 : 32;
}

// Everything the host decides about one product on 8-bit rows.
struct Q8Plan {
    int G;                     // lanes per row of codes
    int team;                  // lanes per row of the graph
    bool random;               // edge gradient: Q8_RANDOM
    int32_t wave_rows;         // rows a wave takes
    int64_t slices;            // blocks of 16 G columns
    bool few;                  // es_q8_few_kernel
    int32_t splits;            // its pieces per row
    int32_t long_k, piece;
    int64_t pieces;            // sums of pieces the workspace holds
    int64_t nblocks, per_xcd, long_blocks, grid_x;
};

constexpr int64_t kFewRows = 512;

// Rows to waves, and which rows are long, for rows that keep `mean` entries, at most Wk.
void plan_rows(Q8Plan& p, int64_t n_rows, double mean, int64_t Wk)
{
    // Rows per wave: the more, the more alike are those that run side by side; but every SIMD wants some waves, and long rows in
    // a wave's own order stray further from their neighbours' codes.  32 / 64: 2.45 M rows, F = 128, FastRand of 64 1301 / 1360 us, 2.06 M,
    // F = 96, mean 4.6 468 / 455; the edge gradient, 544 k, F = 102, mean 41 533 / 549, 1.2 M, F = 48, mean 16 551 / 522.
    const int side = kWaveSize / p.team;                       // rows side by side
    p.wave_rows = mean >= 24.0 ? 32 : 64;
    // Where one row or two run at a time, their order counts for less than even ends, 32 waves per SIMD instead of 8: 233 k rows, Bucket 64, F = 64
    // 180 / 171 us; the edge gradient, 224 k, Bucket 27, F = 344 303 / 278, 233 k, FastRand 500, F = 400 567 / 536.  Two rows of FastRand's edge
    // gradient, whose last pass takes them in turn, 60 k, W = 100, F = 100 47.5 / 51.7; eight of 170 k, mean 14 102 / 106.  It costs one row of
    // the edge gradient's at F = 128, FastRand of 250, 60 k rows: 90 / 99.
    const int64_t waves = (side == 1 || (side == 2 && !p.random) ? 32 : 8) * 4 * kComputeUnits;
    while (p.wave_rows > side && n_rows / p.wave_rows < waves) p.wave_rows /= 2;
    // a lane retires a batch of entries in some 1.5 us; a row should not take it a tenth of the launch
    const double us = mean * (double)n_rows * (double)(p.slices * (p.G * 16 + 12)) / 5.0e6;
    const double side_by_side = (double)p.team / (double)p.G;  // entries of a row
    double k = side_by_side * kQ8Batch * 0.07 * us;
    if (k < 4.0 * mean) k = 4.0 * mean;
    const double least = 64.0 * (side_by_side < 8.0 ? side_by_side : 8.0);
    p.long_k = k < least ? (int32_t)least : k > 1.0e9 ? 1000000000 : (int32_t)k;
    if (p.random) p.long_k = INT32_MAX;                        // W bounds them
    p.long_blocks = Wk > p.long_k ? (n_rows + kQ8ScanRows - 1) / kQ8ScanRows * kQ8Share : 0;
    p.nblocks = (n_rows + kWavesPerBlock * p.wave_rows - 1) / (kWavesPerBlock * p.wave_rows);
    p.per_xcd = (p.nblocks + kNumXcd - 1) / kNumXcd;
    p.grid_x = p.per_xcd * kNumXcd + p.long_blocks;
}

Q8Plan plan_q8(int64_t N, int64_t nnz, int32_t F, int32_t W, int32_t mode, int64_t n_rows, bool may_split = true)
{
    Q8Plan p = {};
    const int64_t chunks = ((int64_t)F + 15) / 16;
    p.G = chunks >= 16 ? 16 : next_pow2(chunks);
    // Wider rows go in blocks of 256 columns, each of which gathers the entries' scales and values anew.  Blocks of 128, 128 k
    // rows of mean 50, F = 256 / 272 / 602: 310 / 513 / 870 us, of 256: 233 / 432 / 693.  The last block's columns as a launch of its
    // own with fewer lanes: 0.92 to 1.05 of the time from 60 k rows on (F = 272 to 1072), 1.0 to 1.4 below.
    p.slices = (chunks + p.G - 1) / p.G;
    const int64_t Wk = mode == ES_FULL ? INT32_MAX : W;
    double mean = N > 0 ? (double)nnz / (double)N : 0.0;
    if (mean > (double)Wk) mean = (double)Wk;
    if (mean < 1.0) mean = 1.0;

    p.few = may_split && n_rows <= kFewRows && Wk > 128;
    if (p.few) {
        p.splits = (int32_t)(2048 / n_rows);
        if (p.splits > 64) p.splits = 64;
        const int64_t most = nnz < Wk ? nnz : Wk;              // no row has more
        if (p.splits > (most + 127) / 128) p.splits = (int32_t)((most + 127) / 128);
        if (p.splits < 1) p.splits = 1;
        p.pieces = p.splits > 1 ? n_rows * p.splits : 0;
        p.grid_x = n_rows * p.splits;
        p.piece = p.long_k = INT32_MAX;
        return p;
    }
    p.team = pick_team(p.G, n_rows, mean);
    plan_rows(p, n_rows, mean, Wk);
    // The join sums every row that keeps more than `piece`, so all of those have to be long ones, which workgroups cut: a wave stores
    // a row of up to long_k by itself.
    int64_t piece = 1024;
    while (piece * 8192 < nnz || piece < p.long_k) piece *= 2;
    p.pieces = Wk > piece && nnz > piece ? 2 * (nnz / piece + 1) : 0;
    p.piece = p.pieces ? (int32_t)piece : INT32_MAX;
    return p;
}

Q8Plan plan_vals(int64_t N, int64_t nnz, int32_t F, int32_t W, int32_t mode)
{
    Q8Plan p = {};
    const int64_t chunks = ((int64_t)F + 15) / 16;
    p.G = chunks >= 64 ? 64 : next_pow2(chunks);
    p.slices = 1;
    const int64_t Wk = mode == ES_FULL ? INT32_MAX : W;
    double mean = (double)nnz / (double)N;
    if (mean > (double)Wk) mean = (double)Wk;
    p.team = pick_team(p.G, N, mean);
    p.random = mode == ES_FASTRAND && W <= kQ8MostRandom;
    if (p.random) p.team = pick_random_team(p.G, N, W);
    plan_rows(p, N, mean < 1.0 ? 1.0 : mean, p.random ? 0 : Wk);
    p.piece = 1024;                                            // each entry is for itself: pieces need no room and no join
    return p;
}

template <bool WIDE>
int launch_q8(const Q8Args& a, const Q8Plan& p, hipStream_t st)
{
    const dim3 grid((uint32_t)p.grid_x, (uint32_t)p.slices), block(kBlockThreads);
    if (p.few) {
#define ES_Q8(G_) case G_: hipLaunchKernelGGL((es_q8_few_kernel<G_, WIDE>), grid, block, 0, st, a); break;
        switch (p.G) { ES_Q8(1) ES_Q8(2) ES_Q8(4) ES_Q8(8) ES_Q8(16) }
#undef ES_Q8
        if (launched() != ES_OK) return ES_ERR_LAUNCH;
        if (p.splits > 1) {
            const uint32_t gy = (uint32_t)(((int64_t)a.F + kBlockThreads - 1) / kBlockThreads);
            hipLaunchKernelGGL(es_q8_few_join_kernel, dim3((uint32_t)a.n_rows, gy < 64 ? gy : 64), block, 0, st, a);
        }
        return launched();
    }
#define ES_SPMM(G_, TEAM_)                                                                                     \
    if (p.team == (TEAM_)) {                                                                                   \
        if (p.long_blocks) hipLaunchKernelGGL((es_q8_spmm_kernel<G_, TEAM_, true, WIDE>), grid, block, 0, st, a);  \
        else hipLaunchKernelGGL((es_q8_spmm_kernel<G_, TEAM_, false, WIDE>), grid, block, 0, st, a);           \
        break;                                                                                                 \
    }
#define ES_Q8(G_) case G_: ES_SPMM(G_, (G_) < 4 ? 4 : G_) ES_SPMM(G_, 32) ES_SPMM(G_, 64) break;
    switch (p.G) { ES_Q8(1) ES_Q8(2) ES_Q8(4) ES_Q8(8) ES_Q8(16) }
#undef ES_Q8
#undef ES_SPMM
    if (launched() != ES_OK) return ES_ERR_LAUNCH;
    if (p.pieces) {
        hipLaunchKernelGGL(es_q8_join_kernel, dim3((uint32_t)((a.n_rows + kQ8ScanRows - 1) / kQ8ScanRows)), block, 0, st, a);
        return launched();
    }
    return ES_OK;
}

template <bool WIDE>
int launch_vals(const Q8Args& a, const Q8Plan& p, hipStream_t st)
{
    const dim3 grid((uint32_t)p.grid_x), block(kBlockThreads);
    const int kind = p.random ? Q8_RANDOM : p.long_blocks ? Q8_LONG : Q8_PREFIX;
    if (a.mode == ES_FASTRAND && !p.random) {
        hipLaunchKernelGGL(es_q8_zero_kernel, dim3(8 * kComputeUnits), block, 0, st, a);
        if (launched() != ES_OK) return ES_ERR_LAUNCH;
    }
#define ES_VALS(G_, TEAM_, KIND_)                                                                                 \
    if (p.team == (TEAM_) && kind == KIND_) {                                                                     \
        hipLaunchKernelGGL((es_q8_vals_kernel<G_, TEAM_, KIND_, WIDE>), grid, block, 0, st, a);                   \
        break;                                                                                                    \
    }
#define ES_TEAM(G_, TEAM_) ES_VALS(G_, TEAM_, Q8_PREFIX) ES_VALS(G_, TEAM_, Q8_LONG)
#define ES_Q8(G_)                                                                                                 \
    case G_:                                                                                                      \
        ES_TEAM(G_, (G_) < 4 ? 4 : G_)                                                                            \
        if constexpr ((G_) < 32) { ES_TEAM(G_, 32) }                                                              \
        if constexpr ((G_) < 64) { ES_TEAM(G_, 64) }                                                              \
        if constexpr ((G_) <= 16) { ES_VALS(G_, 16, Q8_RANDOM) }                                                  \
        if constexpr ((G_) <= 32) { ES_VALS(G_, 32, Q8_RANDOM) }                                                  \
        ES_VALS(G_, 64, Q8_RANDOM)                                                                                \
        break;
    switch (p.G) { ES_Q8(1) ES_Q8(2) ES_Q8(4) ES_Q8(8) ES_Q8(16) ES_Q8(32) ES_Q8(64) }
#undef ES_Q8
#undef ES_TEAM
#undef ES_VALS
    return launched();
}

}  // namespace

extern "C" {

int32_t es_q8_row_bytes(int32_t F) { return F < 1 || F > kMaxF ? 0 : (F + 15) / 16 * 16; }

int es_q8_write(const void* X, int32_t type, int64_t n, int32_t F, int32_t ldx, const int32_t* rows, int64_t N,
                int8_t* codes, int32_t ldq, float* scale, void* stream)
{
    const int size = element_bytes(type);
    if (check_table(N, F, ldq) != ES_OK || !size || n < 0 || n > INT32_MAX || ldx < F || (!rows && n > N)) return ES_ERR_INVALID_ARG;
    if (n == 0 || N == 0) return ES_OK;
    if (!X || misaligned(X, size) || bad_table(codes, scale) || misaligned(rows, 4)) return ES_ERR_INVALID_ARG;
    const Q8Write a = {X, rows, codes, scale, n, N, F, ldx, ldq};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return type == ES_FP32 ? run_write<float>(a, st) : type == ES_FP16 ? run_write<_Float16>(a, st) : run_write<__bf16>(a, st);
}

int es_q8_read(const int8_t* codes, int32_t ldq, const float* scale, int64_t N, int32_t F, const int32_t* rows, int64_t n,
               void* Y, int32_t type, int32_t ldy, void* stream)
{
    const int size = element_bytes(type);
    if (check_table(N, F, ldq) != ES_OK || !size || n < 0 || n > INT32_MAX || ldy < F || (!rows && n > N)) return ES_ERR_INVALID_ARG;
    if (n == 0) return ES_OK;
    if (!Y || misaligned(Y, size) || misaligned(rows, 4) || (N > 0 && bad_table(codes, scale))) return ES_ERR_INVALID_ARG;
    const Q8Read a = {codes, scale, rows, Y, n, N, F, ldq, ldy};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return type == ES_FP32 ? run_read<float>(a, st) : type == ES_FP16 ? run_read<_Float16>(a, st) : run_read<__bf16>(a, st);
}

size_t es_spmm_q8_workspace_bytes(int64_t N, int64_t nnz, int32_t F, int32_t W, int32_t mode, int64_t n_rows)
{
    if (check_product(N, nnz, F, 16 * (int32_t)(((int64_t)F + 15) / 16), F, W, mode, ES_NORM_NONE) != ES_OK || n_rows < 1 ||
        n_rows > INT32_MAX)
        return 0;
    const Q8Plan p = plan_q8(N, nnz, F, W, mode, n_rows);
    return (size_t)p.pieces * (size_t)F * sizeof(float);
}

int es_spmm_q8(const int32_t* rowptr, const int32_t* colidx, const float* vals, const int8_t* codes, int32_t ldq,
               const float* scale, float* Y, int64_t N, int64_t nnz, int32_t F, int32_t ldy, int32_t W, int32_t mode,
               uint64_t seed, int32_t norm, const int32_t* rows, int64_t n_rows, void* workspace, size_t workspace_bytes,
               void* stream)
{
    const int bad = check_product(N, nnz, F, ldq, ldy, W, mode, norm);
    if (bad != ES_OK) return bad;
    if (n_rows < 0 || n_rows > INT32_MAX || (!rows && n_rows != 0 && n_rows != N)) return ES_ERR_INVALID_ARG;
    if (n_rows == 0) return ES_OK;
    if (!Y || misaligned(Y, 4) || misaligned(rows, 4) || misaligned(workspace, 16)) return ES_ERR_INVALID_ARG;
    if (N > 0 && (!rowptr || bad_table(codes, scale) || (nnz > 0 && !colidx))) return ES_ERR_INVALID_ARG;
    Q8Args a = {};
    a.rowptr = rowptr; a.colidx = colidx; a.vals = vals; a.codes = codes; a.scale = scale; a.rows = rows; a.Y = Y;
    a.N = N; a.n_rows = n_rows; a.seed = seed; a.F = F; a.ldq = ldq; a.ldy = ldy;
    a.W = mode == ES_FULL ? INT32_MAX : W; a.mode = mode; a.norm = norm;
    Q8Plan p = plan_q8(N, nnz, F, W, mode, n_rows);
    if (p.pieces && (!workspace || workspace_bytes < (size_t)p.pieces * (size_t)F * sizeof(float))) {
        if (p.few) p = plan_q8(N, nnz, F, W, mode, n_rows, false);
        p.pieces = 0;                                          // a long row is one workgroup's
        p.piece = INT32_MAX;
    }
    const bool wide = (uint64_t)N * (uint64_t)(ldq / kQ8Cols) > 0xFFFFFFFFull;
    a.row_units = wide ? 0u : (uint32_t)(ldq / kQ8Cols);
    a.partial = static_cast<float*>(workspace);
    a.pieces = p.pieces; a.piece = p.piece; a.long_k = p.long_k; a.splits = p.splits; a.wave_rows = p.wave_rows;
    if (p.grid_x > kMostBlocks || p.slices > 65535) return ES_ERR_UNSUPPORTED;
    a.nblocks = (uint32_t)p.nblocks; a.blocks_per_xcd = (uint32_t)p.per_xcd; a.long_blocks = (uint32_t)p.long_blocks;
    return wide ? launch_q8<true>(a, p, static_cast<hipStream_t>(stream)) : launch_q8<false>(a, p, static_cast<hipStream_t>(stream));
}

int es_spmm_q8_backward_vals(const int32_t* rowptr, const int32_t* colidx, const float* dY, int32_t ldy, const int8_t* codes,
                             int32_t ldq, const float* scale, float* dvals, int64_t N, int64_t nnz, int32_t F, int32_t W,
                             int32_t mode, uint64_t seed, int32_t norm, void* stream)
{
    const int bad = check_product(N, nnz, F, ldq, ldy, W, mode, norm);
    if (bad != ES_OK) return bad;
    if (N == 0 || nnz == 0) return ES_OK;
    if (!rowptr || !colidx || !dY || !dvals || misaligned(dY, 4) || misaligned(dvals, 4) || bad_table(codes, scale))
        return ES_ERR_INVALID_ARG;
    Q8Args a = {};
    a.rowptr = rowptr; a.colidx = colidx; a.codes = codes; a.scale = scale; a.Y = dvals; a.dY = dY;
    a.N = a.n_rows = N; a.seed = seed; a.F = F; a.ldq = ldq; a.ldy = ldy;
    a.W = mode == ES_FULL ? INT32_MAX : W; a.mode = mode; a.norm = norm;
    const bool wide = (uint64_t)N * (uint64_t)(ldq / kQ8Cols) > 0xFFFFFFFFull;
    a.row_units = wide ? 0u : (uint32_t)(ldq / kQ8Cols);
    const Q8Plan p = plan_vals(N, nnz, F, W, mode);
    a.piece = p.piece; a.long_k = p.long_k; a.wave_rows = p.wave_rows;
    if (p.grid_x > kMostBlocks || F > kMaxValsF) return ES_ERR_UNSUPPORTED;
    a.nblocks = (uint32_t)p.nblocks; a.blocks_per_xcd = (uint32_t)p.per_xcd; a.long_blocks = (uint32_t)p.long_blocks;
    return wide ? launch_vals<true>(a, p, static_cast<hipStream_t>(stream)) : launch_vals<false>(a, p, static_cast<hipStream_t>(stream));
}

}  // extern "C"

namespace {

// The parts that the rows of X are cut into: two workgroups per compute unit in all, and a step of each wave or more.
struct GradPlan {
    int MT, NT;                // tiles of the instruction per wave, along F and along H
    int64_t tiles_m, tiles, parts, part_rows;
};

GradPlan plan_grad(int64_t N, int32_t F, int32_t H, size_t workspace_bytes)
{
    GradPlan p;
    p.MT = F <= kGradTile ? 1 : F <= 2 * kGradTile ? 2 : 4;
    p.NT = H <= kGradTile ? 1 : 2;
    const int64_t m = p.MT * kGradTile, n = p.NT * kGradTile;
    p.tiles_m = (F + m - 1) / m;
    p.tiles = p.tiles_m * ((H + n - 1) / n);
    p.parts = 2 * kComputeUnits / p.tiles;
    if (p.parts > N / kGradRows) p.parts = N / kGradRows;
    if (p.parts > kNumXcd) p.parts -= p.parts % kNumXcd;       // each XCD as many
    if (p.parts < 1) p.parts = 1;
    p.part_rows = ((N + p.parts - 1) / p.parts + kGradRows - 1) / kGradRows * kGradRows;
    p.parts = p.part_rows ? (N + p.part_rows - 1) / p.part_rows : 1;
    if (p.parts > 1 && workspace_bytes < (size_t)F * (size_t)H * sizeof(float) * (size_t)p.parts) {
        p.parts = 1;
        p.part_rows = N;
    }
    return p;
}

}  // namespace

extern "C" {

size_t es_q8_weight_grad_workspace_bytes(int64_t N, int32_t F, int32_t H)
{
    if (N < 1 || N > INT32_MAX || F < 1 || F > kMaxF || H < 1) return 0;
    const GradPlan p = plan_grad(N, F, H, SIZE_MAX);
    return p.parts > 1 ? (size_t)F * (size_t)H * sizeof(float) * (size_t)p.parts : 0;
}

int es_q8_weight_grad(const int8_t* codes, int32_t ldq, const float* scale, const float* G, int32_t ldg, float* dW,
                      int32_t ldw, int64_t N, int32_t F, int32_t H, void* workspace, size_t workspace_bytes, void* stream)
{
    if (check_table(N, F, ldq) != ES_OK || H < 1 || ldg < H || ldw < H) return ES_ERR_INVALID_ARG;
    if (!dW || misaligned(dW, 4) || misaligned(workspace, 16)) return ES_ERR_INVALID_ARG;
    if (N > 0 && (!G || misaligned(G, 4) || bad_table(codes, scale))) return ES_ERR_INVALID_ARG;
    const GradPlan p = plan_grad(N, F, H, workspace ? workspace_bytes : 0);
    if (ldq >= 1 << 27 || ldg >= 1 << 26) return ES_ERR_UNSUPPORTED;  // a lane's byte offset inside 9 rows is held in 32 bits
    const int64_t grid = (p.parts < kNumXcd ? p.parts : (p.parts + kNumXcd - 1) / kNumXcd * kNumXcd) * p.tiles;
    if (grid > kMostBlocks) return ES_ERR_UNSUPPORTED;
    const bool join = p.parts > 1;
    const Q8Grad a = {codes, scale, G, join ? static_cast<float*>(workspace) : dW, N, F, H, ldq, ldg, join ? H : ldw,
                      (int32_t)p.tiles_m, (int32_t)p.tiles, p.part_rows, (int32_t)p.parts};
    hipStream_t st = static_cast<hipStream_t>(stream);
#define ES_GRAD(MT_, NT_)                                                                                            \
    if (p.MT == MT_ && p.NT == NT_)                                                                                  \
        hipLaunchKernelGGL((es_q8_grad_kernel<MT_, NT_>), dim3((uint32_t)grid), dim3(kBlockThreads), 0, st, a);
    ES_GRAD(1, 1) ES_GRAD(1, 2) ES_GRAD(2, 1) ES_GRAD(2, 2) ES_GRAD(4, 1) ES_GRAD(4, 2)
#undef ES_GRAD
    if (launched() != ES_OK) return ES_ERR_LAUNCH;
    if (!join) return ES_OK;
    const uint32_t gj = blocks_of((int64_t)F * H, kWaveSize);      // several parts: 256 tiles of dW or fewer
    hipLaunchKernelGGL(es_q8_grad_join_kernel, dim3(gj), dim3(kGradJoin * kWaveSize), 0, st, a.dW, (int)p.parts, F, H, dW, ldw);
    return launched();
}

}  // extern "C"
