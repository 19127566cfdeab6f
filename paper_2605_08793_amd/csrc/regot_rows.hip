// Row operators on a model's scores: log probabilities, entropy and alternatives; distillation; routing; and their gradients.
// Checks of arguments, how rows are shared out, launches.  The kernels are in regot_rows_logprob.hpp, regot_rows_grad.hpp and
// regot_rows_route.hpp.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "regot.h"
#include "regot_overlap.hpp"
#include "regot_rows_grad.hpp"
#include "regot_rows_logprob.hpp"
#include "regot_rows_route.hpp"

namespace {

using namespace regot;

constexpr int64_t kMaxDim = 2147483647LL;
constexpr size_t kAlign = 256;

bool misaligned(const void *p, size_t a) { return ((uintptr_t)p % a) != 0; }
int hip_status() { return hipGetLastError() == hipSuccess ? REGOT_OK : REGOT_ERR_HIP; }

int element_bytes(int type) { return type == REGOT_F32 ? 4 : 2; }

int check_rows(int64_t n, int64_t m, const void *S, int type, int64_t ldS, double eta)
{
    if (n < 0 || m < 0 || n > kMaxDim || m > kMaxDim) return REGOT_ERR_DIM;
    if (type != REGOT_F32 && type != REGOT_BF16 && type != REGOT_F16) return REGOT_ERR_ARG;
    // (1 / eta has to be a 32-bit number other than 0)
    if (!(eta > 0.0) || !isfinite(eta) || !isfinite((float)(1.4426950408889634 / eta)) || (float)(1.0 / eta) < 1e-37f) return REGOT_ERR_ETA;
    if (n > 0 && m > 0 && !S) return REGOT_ERR_NULL;
    if (ldS < m) return REGOT_ERR_LD;
    if (misaligned(S, element_bytes(type))) return REGOT_ERR_ALIGN;
    return REGOT_OK;
}

RowArgs row_args(int64_t n, int64_t m, const void *S, int64_t ldS, const float *bias, double eta)
{
    RowArgs A{};
    A.n = n;
    A.m = (uint32_t)m;
    A.S = S;
    A.ldS = ldS;
    A.bias = bias;
    A.inv_eta = (float)(1.0 / eta);
    A.log2_scale = (float)(1.4426950408889634 / eta);
    return A;
}

constexpr int64_t kMaxGrid = 1 << 22;  // (rows beyond are the same workgroups')

// How the rows of a call are shared out: a few long rows are several workgroups' each, whose findings a second launch joins.  (One
// workgroup takes 5.5 us and 0.45 for each slice of 4096 columns, the two launches 10.5 us and the reading.  us, one workgroup a row / parts, bf16, 20
// alternatives: 1 x 131072 19.7 / 10.6, 8 x 131072 20.3 / 11.2, 64 x 50000 11.8 / 10.8, 128 x 32768 10.5 / 11.7, 256 x 131072 25.9 / 26.8.)
constexpr int kFewRows = 192, kLongRow = 13, kPlaces = 512, kLeastParts = 8, kMostParts = 64;

struct RowPlan {
    int block = 1, blocks = 1, parts = 1, part_blocks = 1;  // slices of a block, blocks of a row, workgroups of a row, blocks of each
    size_t max = 0, total = 0;                              // workspace: where the maxima are, and all of it
};

int64_t power_of_two(int64_t least)
{
    int64_t p = 1;
    while (p < least) p *= 2;
    return p;
}

RowPlan plan_rows(int64_t n, int64_t m, int k, int few = kFewRows)
{
    RowPlan P;
    const int64_t slices = std::max<int64_t>((m + kSlice - 1) / kSlice, 1);
    int64_t parts = 1;
    // (alternatives: the second launch looks through all blocks of a row.  1 x 131072 bf16 16 blocks 9.5 us, 32 9.7, 64 9.9; 64 rows of them 12.7, 13.9, 13.9;
    // 4 x 1000000 19.1, 15.6, 14.3)
    const int64_t most_blocks = k == 0 ? kMostParts : slices <= 32 ? kPartBlocks / 2 : kPartBlocks;
    if (n > 0 && n <= few && slices >= kLongRow) parts = std::min<int64_t>({slices, most_blocks, std::max<int64_t>(kPlaces / n, kLeastParts)});
    if (parts > 1) {
        const int64_t of_part = (slices + parts - 1) / parts;  // slices of a part
        const int64_t most = std::max<int64_t>(most_blocks / parts, 1);   // blocks of a part
        P.block = (int)power_of_two((of_part + most - 1) / most);
        P.part_blocks = (int)((of_part + P.block - 1) / P.block);
        P.blocks = (int)((slices + P.block - 1) / P.block);
        P.parts = (P.blocks + P.part_blocks - 1) / P.part_blocks;
    }
    if (P.parts > 1) {
        P.max = ((size_t)n * P.parts * 3 * sizeof(float) + kAlign - 1) / kAlign * kAlign;
        P.total = P.max + (k > 0 ? (size_t)n * P.blocks * kThreads * sizeof(float) : 0);
    } else {
        P.block = (int)power_of_two((slices + kWholeBlocks - 1) / kWholeBlocks);
        P.blocks = P.part_blocks = (int)((slices + P.block - 1) / P.block);
    }
    P.total = std::max((P.total + kAlign - 1) / kAlign * kAlign, kAlign);
    return P;
}

template <int TYPE, bool BIAS, bool TOP>
void launch_logprob(const RowArgs &A, const RowPlan &P, hipStream_t s)
{
    constexpr int kVecs = 4;  // 16-byte loads in flight (8: 4096 x 131072 bf16, 20 alternatives 179 us and 181, but 10000 x 5000 77 and 59)
    constexpr uint32_t kLoad = kLanes * Score<TYPE>::kVec;  // columns of a wave's load
    const dim3 threads(kThreads);
    const auto grid = [](int64_t blocks) { return dim3((unsigned)std::min(blocks, kMaxGrid)); };
    const dim3 by_wave = grid((A.n + kWaves - 1) / kWaves);
    if (A.m <= 2 * kLanes) {
        hipLaunchKernelGGL((row_logprob_narrow_kernel<TYPE + kSingle, BIAS, TOP, 2>), by_wave, threads, 0, s, A);
    } else if (A.m <= kLoad) {
        hipLaunchKernelGGL((row_logprob_narrow_kernel<TYPE, BIAS, TOP, 1>), by_wave, threads, 0, s, A);
    } else if (A.m <= 2 * kLoad) {
        hipLaunchKernelGGL((row_logprob_narrow_kernel<TYPE, BIAS, TOP, 2>), by_wave, threads, 0, s, A);
    } else if (A.m <= 8 * kLoad && P.parts == 1) {
        hipLaunchKernelGGL((row_logprob_narrow_kernel<TYPE, BIAS, TOP, 8>), by_wave, threads, 0, s, A);
    } else if (P.parts > 1) {
        hipLaunchKernelGGL((row_logprob_kernel<TYPE, BIAS, TOP, kVecs, true>), grid(A.n * P.parts), threads, 0, s, A);
        hipLaunchKernelGGL((row_logprob_join_kernel<TYPE, BIAS, TOP>), grid(A.n), threads, 0, s, A);
    } else {
        hipLaunchKernelGGL((row_logprob_kernel<TYPE, BIAS, TOP, kVecs, false>), grid(A.n), threads, 0, s, A);
    }
}

template <int TYPE>
void launch_logprob(const RowArgs &A, const RowPlan &P, hipStream_t s)
{
    if (A.bias) A.k > 0 ? launch_logprob<TYPE, true, true>(A, P, s) : launch_logprob<TYPE, true, false>(A, P, s);
    else A.k > 0 ? launch_logprob<TYPE, false, true>(A, P, s) : launch_logprob<TYPE, false, false>(A, P, s);
}

void take_plan(RowArgs &A, const RowPlan &P, void *workspace)
{
    A.block = P.block;
    A.block_log2 = cbits(P.block);
    A.blocks = P.blocks;
    A.scan_log2 = cbits(power_of_two(P.blocks));
    A.parts = P.parts;
    A.part_blocks = P.part_blocks;
    A.part_columns = (uint32_t)P.part_blocks * P.block * kSlice;
    A.part_sums = static_cast<float *>(workspace);
    A.part_max = reinterpret_cast<float *>(static_cast<char *>(workspace) + P.max);
}

// Gradients of log probabilities: parts of rows, so that there are workgroups enough.
template <int TYPE, bool BIAS>
void launch_logprob_grad(RowArgs &A, hipStream_t s)
{
    constexpr int kVecs = 4;
    const auto grid = [](int64_t blocks) { return dim3((unsigned)std::min(blocks, kMaxGrid)); };
    if (A.m <= 2 * kLanes) {
        A.parts = 1;
        A.part_columns = A.m;
        hipLaunchKernelGGL((row_logprob_grad_kernel<TYPE + kSingle, BIAS, 1, 2>), grid((A.n + kWaves - 1) / kWaves), dim3(kThreads), 0, s, A);
    } else if (A.m <= kVecs * kLanes * Score<TYPE>::kVec) {
        A.parts = 1;
        A.part_columns = A.m;
        hipLaunchKernelGGL((row_logprob_grad_kernel<TYPE, BIAS, 1, kVecs>), grid((A.n + kWaves - 1) / kWaves), dim3(kThreads), 0, s, A);
    } else {
        constexpr uint32_t kColumns = kVecs * kThreads * Score<TYPE>::kVec;
        A.part_columns = kColumns;
        A.parts = (int)((A.m + kColumns - 1) / kColumns);
        hipLaunchKernelGGL((row_logprob_grad_kernel<TYPE, BIAS, kWaves, kVecs>), grid(A.n * A.parts), dim3(kThreads), 0, s, A);
    }
}

template <int TYPE>
void launch_logprob_grad(RowArgs &A, hipStream_t s)
{
    A.bias ? launch_logprob_grad<TYPE, true>(A, s) : launch_logprob_grad<TYPE, false>(A, s);
}

void launch_logprob_grad(RowArgs &A, int type, hipStream_t s)
{
    if (type == REGOT_F32) launch_logprob_grad<REGOT_F32>(A, s);
    else if (type == REGOT_BF16) launch_logprob_grad<REGOT_BF16>(A, s);
    else launch_logprob_grad<REGOT_F16>(A, s);
}

// Parts as for log probabilities, up to the rows at which a team of 16 waves each is as fast: 64 x 131072 bf16 19.4 us in parts and 25.8, 128 rows
// 28.5 and 27.4, 192 rows 36.3 and 30.6; 1 row 10.8 and 25.2.
constexpr int kFewDistilled = 96;
RowPlan plan_distill(int64_t n, int64_t m) { return plan_rows(n, m, 0, kFewDistilled); }

constexpr int kCUs = 256;

template <int TYPE, int WAVES, int VECS, int KEPT>
void launch_team(const RowArgs &A, hipStream_t s)
{
    const dim3 grid((unsigned)std::min(WAVES == 1 ? (A.n + kWaves - 1) / kWaves : A.n, kMaxGrid)), threads(Team<WAVES>::kBlock);
    if constexpr (WAVES == 1)
        if (A.k <= 128) {
            hipLaunchKernelGGL((row_distill_kernel<TYPE, WAVES, VECS, KEPT, false, 128>), grid, threads, 0, s, A);
            return;
        }
    hipLaunchKernelGGL((row_distill_kernel<TYPE, WAVES, VECS, KEPT, false>), grid, threads, 0, s, A);
}

template <int TYPE>
void launch_distill(const RowArgs &A, hipStream_t s)
{
    const auto grid = [](int64_t blocks) { return dim3((unsigned)std::min(blocks, kMaxGrid)); };
    // Teams of more waves hold more of a row between its two reads (the last stretch in registers, the one before in LDS) and
    // make less of the traffic; of fewer, they keep more rows under way.  us: 16384 x 1000 bf16 1 wave 25, 4 waves 63; 4096 x 10000 4 waves
    // 47, 8 waves 78; 4096 x 32768 4 waves 123, 8 waves holding 134; 999 x 33333 4 waves 43, 8 waves holding 39; 4096 x 131072 4 waves 526, 8
    // waves 513, holding 431, 16 waves holding 468; 256 x 131072 8 waves holding 40, 16 waves holding 33; 256 x 10000 fp32 4 waves 9.9, 8 waves 8.9.
    const uint32_t loads = A.m / Score<TYPE>::kVec;
    if (A.parts > 1) {
        hipLaunchKernelGGL((row_logprob_kernel<TYPE, false, false, 4, true>), grid(A.n * A.parts), dim3(kThreads), 0, s, A);
        hipLaunchKernelGGL((row_distill_kernel<TYPE, kWaves, 4, 0, true>), grid(A.n * A.parts), dim3(kThreads), 0, s, A);
    } else if (A.m <= 2 * kLanes) {
        launch_team<TYPE + kSingle, 1, 2, 0>(A, s);
    } else if (A.n > 512 && loads <= 2 * kLanes) {
        launch_team<TYPE, 1, 2, 0>(A, s);
    } else if (A.n > 512 && loads <= 4 * kLanes) {
        launch_team<TYPE, 1, 4, 0>(A, s);
    } else if (A.n > 512 && loads <= 8 * kLanes) {
        launch_team<TYPE, 1, 8, 0>(A, s);
    } else if (loads <= (A.n > 512 ? 64 : 8) * kLanes) {
        launch_team<TYPE, 4, 2, 0>(A, s);
    } else if (loads <= 64 * kLanes) {
        launch_team<TYPE, 8, 4, 0>(A, s);
    } else if (A.n > kCUs) {
        launch_team<TYPE, 8, 8, 8>(A, s);
    } else {
        launch_team<TYPE, 16, 8, 8>(A, s);
    }
}

void launch_distill(const RowArgs &A, int type, hipStream_t s)
{
    if (type == REGOT_F32) launch_distill<REGOT_F32>(A, s);
    else if (type == REGOT_BF16) launch_distill<REGOT_BF16>(A, s);
    else launch_distill<REGOT_F16>(A, s);
}

void launch_logprob(const RowArgs &A, int type, const RowPlan &P, hipStream_t s)
{
    if (type == REGOT_F32) launch_logprob<REGOT_F32>(A, P, s);
    else if (type == REGOT_BF16) launch_logprob<REGOT_BF16>(A, P, s);
    else launch_logprob<REGOT_F16>(A, P, s);
}

// Rows of a route by their length: 8 lanes with 4, 8 or 16 scores each, 16 with 8 or 16, 32 with 16, or a wave with 16.  Fewer lanes with more
// scores each merge less, and hide less of a row's latency.  us: 65536 x 32 bf16, 4 choices 8 lanes 6.5, 16 lanes 11.0; 65536 x 64 fp32, 2 choices 8 lanes
// 7.7, 16 lanes 11.4; 65536 x 128 bf16, 8 choices 8 lanes 13.4, 16 lanes 17.5, but 1 row 3.6 and 3.3, 512 rows 4.5 and 4.0; 65536 x 256 fp32,
// 8 choices 8 lanes 29, 16 lanes 27; 16384 x 512 fp32, 8 choices 16 lanes 13.7, 32 lanes 15.6, a wave 20.3, but 1 row 5.6, 4.0 and 3.7.
// Loads of 16 bytes where the columns of each lie in one group; otherwise, and for short rows, a score at a time (65536 x 64 fp32: 8.7 us).
template <int TYPE, int LANES, int VALUES>
void launch_route(const RouteArgs &A, hipStream_t s)
{
    const dim3 grid((unsigned)std::min((A.n + kThreads / LANES - 1) / (kThreads / LANES), kMaxGrid));
    if (A.k <= 4) hipLaunchKernelGGL((row_route_kernel<TYPE, LANES, VALUES, 4>), grid, dim3(kThreads), 0, s, A);
    else if (A.k <= 8) hipLaunchKernelGGL((row_route_kernel<TYPE, LANES, VALUES, 8>), grid, dim3(kThreads), 0, s, A);
    else if (A.k <= 16) hipLaunchKernelGGL((row_route_kernel<TYPE, LANES, VALUES, 16>), grid, dim3(kThreads), 0, s, A);
    else hipLaunchKernelGGL((row_route_kernel<TYPE, LANES, VALUES, REGOT_ROW_MAX_CHOICES>), grid, dim3(kThreads), 0, s, A);
}

template <int TYPE>
void launch_route(RouteArgs &A, hipStream_t s)
{
    const bool wide = A.m >= Score<TYPE>::kVec && (A.groups == 1 || A.group_size % Score<TYPE>::kVec == 0);
    const bool many = A.n > 4096;
    const int lanes = A.m <= 64 || (A.m <= 128 && wide && many) ? 8 : A.m <= 256 ? 16 : A.m <= 512 ? 32 : kLanes;
    A.group_lanes = (int)std::max<int64_t>(lanes / power_of_two(A.groups), 1);
    if (A.m <= 32) launch_route<TYPE + kSingle, 8, 4>(A, s);
    else if (A.m <= 64) wide ? launch_route<TYPE, 8, 8>(A, s) : launch_route<TYPE + kSingle, 8, 8>(A, s);
    else if (A.m <= 128 && wide && many) launch_route<TYPE, 8, 16>(A, s);
    else if (A.m <= 128) wide ? launch_route<TYPE, 16, 8>(A, s) : launch_route<TYPE + kSingle, 16, 8>(A, s);
    else if (A.m <= 256) wide ? launch_route<TYPE, 16, 16>(A, s) : launch_route<TYPE + kSingle, 16, 16>(A, s);
    else if (A.m <= 512) wide ? launch_route<TYPE, 32, 16>(A, s) : launch_route<TYPE + kSingle, 32, 16>(A, s);
    else wide ? launch_route<TYPE, kLanes, 16>(A, s) : launch_route<TYPE + kSingle, kLanes, 16>(A, s);
}

void launch_route(RouteArgs &A, int type, hipStream_t s)
{
    if (type == REGOT_F32) launch_route<REGOT_F32>(A, s);
    else if (type == REGOT_BF16) launch_route<REGOT_BF16>(A, s);
    else launch_route<REGOT_F16>(A, s);
}

template <int TYPE, int LANES, int VALUES>
void launch_route_grad(const RouteArgs &A, hipStream_t s)
{
    const dim3 grid((unsigned)std::min((A.n + kThreads / LANES - 1) / (kThreads / LANES), kMaxGrid));
    if (A.k <= 8) hipLaunchKernelGGL((row_route_grad_kernel<TYPE, LANES, VALUES, 8>), grid, dim3(kThreads), 0, s, A);
    else hipLaunchKernelGGL((row_route_grad_kernel<TYPE, LANES, VALUES, REGOT_ROW_MAX_CHOICES>), grid, dim3(kThreads), 0, s, A);
}

template <int TYPE>
void launch_route_grad(const RouteArgs &A, hipStream_t s)
{
    if (A.m <= 32) launch_route_grad<TYPE + kSingle, 8, 4>(A, s);
    else if (A.m <= 64) launch_route_grad<TYPE, 8, 8>(A, s);
    else if (A.m <= 128) launch_route_grad<TYPE, 16, 8>(A, s);
    else if (A.m <= 256) launch_route_grad<TYPE, 16, 16>(A, s);
    else if (A.m <= 512) launch_route_grad<TYPE, 32, 16>(A, s);
    else launch_route_grad<TYPE, kLanes, 16>(A, s);
}

void launch_route_grad(const RouteArgs &A, int type, hipStream_t s)
{
    if (type == REGOT_F32) launch_route_grad<REGOT_F32>(A, s);
    else if (type == REGOT_BF16) launch_route_grad<REGOT_BF16>(A, s);
    else launch_route_grad<REGOT_F16>(A, s);
}

}  // namespace

extern "C" {

int regot_row_logprob_workspace_bytes(int64_t n, int64_t m, int k, size_t *bytes)
{
    if (!bytes) return REGOT_ERR_NULL;
    if (n < 0 || m < 0 || n > kMaxDim || m > kMaxDim) return REGOT_ERR_DIM;
    if (k < 0 || k > REGOT_ROW_MAX_TOP) return REGOT_ERR_ARG;
    *bytes = plan_rows(n, m, k).total;
    return REGOT_OK;
}

int regot_row_logprob(int64_t n, int64_t m, const void *S, int type, int64_t ldS, const float *bias, double eta,
                      const int32_t *target, int targets, int k, float *logprob, float *entropy, float *stats,
                      int32_t *top_idx, float *top_logprob, void *workspace, size_t workspace_bytes, regot_stream_t stream)
{
    int st = check_rows(n, m, S, type, ldS, eta);
    if (st != REGOT_OK) return st;
    if (targets < 0 || targets > REGOT_ROW_MAX_LIST || k < 0 || k > REGOT_ROW_MAX_TOP) return REGOT_ERR_ARG;
    if (n > 0 && ((targets > 0 && (!target || !logprob)) || (k > 0 && (!top_idx || !top_logprob)))) return REGOT_ERR_NULL;
    if (misaligned(bias, 4) || misaligned(target, 4) || misaligned(logprob, 4) || misaligned(entropy, 4) || misaligned(stats, 4) ||
        misaligned(top_idx, 4) || misaligned(top_logprob, 4))
        return REGOT_ERR_ALIGN;
    const RowPlan P = plan_rows(n, m, k);
    if (!workspace) return REGOT_ERR_NULL;
    if (misaligned(workspace, kAlign)) return REGOT_ERR_ALIGN;
    if (workspace_bytes < P.total) return REGOT_ERR_WORKSPACE;
    if (n == 0) return REGOT_OK;
    RowArgs A = row_args(n, m, S, ldS, bias, eta);
    A.target = target;
    A.targets = targets;
    A.k = k;
    A.logprob = logprob;
    A.entropy = entropy;
    A.stats = stats;
    A.top_idx = top_idx;
    A.top_logprob = top_logprob;
    take_plan(A, P, workspace);
    launch_logprob(A, type, P, static_cast<hipStream_t>(stream));
    return hip_status();
}

int regot_row_logprob_grad(int64_t n, int64_t m, const void *S, int type, int64_t ldS, const float *bias, double eta,
                           const int32_t *target, int targets, const float *stats, const float *entropy,
                           const float *g_logprob, const float *g_entropy, void *dS, int64_t ldD, regot_stream_t stream)
{
    int st = check_rows(n, m, S, type, ldS, eta);
    if (st != REGOT_OK) return st;
    if (targets < 0 || targets > REGOT_ROW_MAX_LIST) return REGOT_ERR_ARG;
    if (n > 0 && (!stats || (targets > 0 && (!target || !g_logprob)) || (g_entropy && !entropy) || (m > 0 && !dS))) return REGOT_ERR_NULL;
    if (ldD < m) return REGOT_ERR_LD;
    if (misaligned(bias, 4) || misaligned(target, 4) || misaligned(stats, 4) || misaligned(entropy, 4) || misaligned(g_logprob, 4) ||
        misaligned(g_entropy, 4) || misaligned(dS, element_bytes(type)))
        return REGOT_ERR_ALIGN;
    if (n == 0 || m == 0) return REGOT_OK;
    if (overlap(n, m, S, ldS, dS, ldD, element_bytes(type))) return REGOT_ERR_ARG;
    RowArgs A = row_args(n, m, S, ldS, bias, eta);
    A.target = target;
    A.targets = targets;
    A.stats_in = stats;
    A.entropy_in = entropy;
    A.g_logprob = g_logprob;
    A.g_entropy = g_entropy;
    A.dS = dS;
    A.ldD = ldD;
    launch_logprob_grad(A, type, static_cast<hipStream_t>(stream));
    return hip_status();
}

int regot_row_distill_workspace_bytes(int64_t n, int64_t m, int k, size_t *bytes)
{
    if (!bytes) return REGOT_ERR_NULL;
    if (n < 0 || m < 0 || n > kMaxDim || m > kMaxDim) return REGOT_ERR_DIM;
    if (k < 1 || k > REGOT_ROW_MAX_LIST) return REGOT_ERR_ARG;
    *bytes = plan_distill(n, m).total;
    return REGOT_OK;
}

int regot_row_distill(int64_t n, int64_t m, const void *S, int type, int64_t ldS, double eta, const int32_t *t_idx,
                      const float *t_score, int k, const float *row_weight, float *loss, void *dS, int64_t ldD,
                      void *workspace, size_t workspace_bytes, regot_stream_t stream)
{
    int st = check_rows(n, m, S, type, ldS, eta);
    if (st != REGOT_OK) return st;
    if (k < 1 || k > REGOT_ROW_MAX_LIST) return REGOT_ERR_ARG;
    if (n > 0 && (!t_idx || !t_score || !loss)) return REGOT_ERR_NULL;
    if (dS && ldD < m) return REGOT_ERR_LD;
    if (misaligned(t_idx, 4) || misaligned(t_score, 4) || misaligned(row_weight, 4) || misaligned(loss, 4) ||
        misaligned(dS, element_bytes(type)))
        return REGOT_ERR_ALIGN;
    const RowPlan P = plan_distill(n, m);
    if (!workspace) return REGOT_ERR_NULL;
    if (misaligned(workspace, kAlign)) return REGOT_ERR_ALIGN;
    if (workspace_bytes < P.total) return REGOT_ERR_WORKSPACE;
    if (n == 0) return REGOT_OK;
    if (dS && overlap(n, m, S, ldS, dS, ldD, element_bytes(type))) return REGOT_ERR_ARG;
    RowArgs A = row_args(n, m, S, ldS, nullptr, eta);
    A.target = t_idx;
    A.t_score = t_score;
    A.k = k;
    A.row_weight = row_weight;
    A.loss = loss;
    A.dS = dS;
    A.ldD = ldD;
    take_plan(A, P, workspace);
    launch_distill(A, type, static_cast<hipStream_t>(stream));
    return hip_status();
}

int regot_row_route(int64_t n, int64_t m, const void *S, int type, int64_t ldS, const float *bias, int bias_on, int score,
                    int groups, int groups_kept, int group_by, int k, int renormalise, double scale, int32_t *idx,
                    float *weight, regot_stream_t stream)
{
    int st = check_rows(n, m, S, type, ldS, 1.0);
    if (st != REGOT_OK) return st;
    if (m > REGOT_ROW_MAX_EXPERTS) return REGOT_ERR_DIM;
    if (k < 1 || k > REGOT_ROW_MAX_CHOICES || (score != REGOT_SOFTMAX && score != REGOT_SIGMOID) ||
        (bias && bias_on != REGOT_BIAS_SCORE && bias_on != REGOT_BIAS_LOGIT) || groups < 1 || groups > kMaxGroups ||
        groups_kept < 1 || groups_kept > groups || (m % groups != 0) || (group_by != REGOT_GROUP_MAX && group_by != REGOT_GROUP_TOP2) ||
        (renormalise != 0 && renormalise != 1) || !isfinite((float)scale))
        return REGOT_ERR_ARG;
    if (n > 0 && (!idx || !weight)) return REGOT_ERR_NULL;
    if (misaligned(bias, 4) || misaligned(idx, 4) || misaligned(weight, 4)) return REGOT_ERR_ALIGN;
    if (n == 0) return REGOT_OK;
    RouteArgs A{};
    A.n = n;
    A.m = (uint32_t)m;
    A.S = S;
    A.ldS = ldS;
    A.bias = bias;
    A.bias_on = bias_on;
    A.score = score;
    A.groups = groups;
    A.groups_kept = groups_kept;
    A.group_by = group_by;
    A.k = k;
    A.renormalise = renormalise;
    A.scale = (float)scale;
    A.idx = idx;
    A.weight = weight;
    A.group_size = (uint32_t)(m / groups);
    A.group_magic = A.group_size > 1 ? (uint32_t)(((1ull << 32) + A.group_size - 1) / A.group_size) : 0;
    launch_route(A, type, static_cast<hipStream_t>(stream));
    return hip_status();
}

int regot_row_route_grad(int64_t n, int64_t m, const void *S, int type, int64_t ldS, int score, const int32_t *idx, int k,
                         int renormalise, double scale, const float *g_weight, void *dS, int64_t ldD, regot_stream_t stream)
{
    int st = check_rows(n, m, S, type, ldS, 1.0);
    if (st != REGOT_OK) return st;
    if (m > REGOT_ROW_MAX_EXPERTS) return REGOT_ERR_DIM;
    if (k < 1 || k > REGOT_ROW_MAX_CHOICES || (score != REGOT_SOFTMAX && score != REGOT_SIGMOID) ||
        (renormalise != 0 && renormalise != 1) || !isfinite((float)scale))
        return REGOT_ERR_ARG;
    if (n > 0 && (!idx || !g_weight || (m > 0 && !dS))) return REGOT_ERR_NULL;
    if (ldD < m) return REGOT_ERR_LD;
    if (misaligned(idx, 4) || misaligned(g_weight, 4) || misaligned(dS, element_bytes(type))) return REGOT_ERR_ALIGN;
    if (n == 0 || m == 0) return REGOT_OK;
    if (overlap(n, m, S, ldS, dS, ldD, element_bytes(type))) return REGOT_ERR_ARG;
    RouteArgs A{};
    A.n = n;
    A.m = (uint32_t)m;
    A.S = S;
    A.ldS = ldS;
    A.score = score;
    A.k = k;
    A.renormalise = renormalise;
    A.scale = (float)scale;
    A.idx_in = idx;
    A.g_weight = g_weight;
    A.dS = dS;
    A.ldD = ldD;
    launch_route_grad(A, type, static_cast<hipStream_t>(stream));
    return hip_status();
}

}  // extern "C"
