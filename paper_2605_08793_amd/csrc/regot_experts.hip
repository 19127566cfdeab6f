// What follows a router's choices: their order by expert, products grouped by expert and their gradients, the weighted sum of the
// experts' rows, and the norm over all gradients with clipping.  Checks of arguments, how work is shared out, launches; the products' kernels
// are built for each type of numbers in a source of their own.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>
#include <memory>
#include <new>

#include "regot.h"
#include "regot_experts_launch.hpp"
#include "regot_experts_order.hpp"
#include "regot_gradients.hpp"
#include "regot_overlap.hpp"

namespace regot {
void expert_tiles_bf16(const GroupArgs &A, const TilePlan &P, hipStream_t s);
void expert_tiles_f16(const GroupArgs &A, const TilePlan &P, hipStream_t s);
void expert_tiles_f32(const GroupArgs &A, const TilePlan &P, hipStream_t s);
}  // namespace regot

namespace {

using namespace regot;

constexpr int64_t kMaxDim = 2147483647LL;
constexpr int64_t kMaxGrid = 1 << 22;
constexpr int64_t kMaxTiles = (1 << 23) - 1;     // workgroups of 512 threads: a launch has fewer than 2^32 threads
constexpr int64_t kMaxNumbers = (int64_t)1 << 40;  // of a tensor
constexpr size_t kAlign = 256;
constexpr int kCUs = 256;

bool misaligned(const void *p, size_t a) { return ((uintptr_t)p % a) != 0; }
int hip_status() { return hipGetLastError() == hipSuccess ? REGOT_OK : REGOT_ERR_HIP; }
bool bad_type(int type) { return type != REGOT_F32 && type != REGOT_BF16 && type != REGOT_F16; }
int element_bytes(int type) { return type == REGOT_F32 ? 4 : 2; }
bool bad_dim(int64_t v) { return v < 0 || v > kMaxDim; }
size_t padded(size_t bytes) { return std::max((bytes + kAlign - 1) / kAlign * kAlign, kAlign); }
unsigned grid_of(int64_t blocks) { return (unsigned)std::min(blocks, kMaxGrid); }

// ---- the order of choices ----

constexpr int64_t kOneGroup = 8192;  // choices that one workgroup puts in order, in one launch
constexpr int kMostGroups = 128;     // (us for 524288 choices, 64 / 128 / 256 groups: 17.2 / 15.0 / 16.6)
constexpr int64_t kLeastChoices = 2048;  // of a group (us for 32768 choices, 8192 / 4096 / 2048: 12.4 / 9.8 / 8.5)

struct OrderPlan {
    int64_t each = 0;
    int groups = 1;
    size_t total = 0;
};

OrderPlan plan_order(int64_t count, int64_t experts)
{
    OrderPlan P;
    P.each = count;
    if (count > kOneGroup) {
        P.each = std::max<int64_t>((count + kMostGroups - 1) / kMostGroups, kLeastChoices);
        P.groups = (int)((count + P.each - 1) / P.each);
    }
    P.total = padded(P.groups > 1 ? (size_t)P.groups * (experts + 1) * sizeof(uint32_t) : 0);
    return P;
}

int check_order(int64_t n, int k, int64_t experts)
{
    if (n < 0 || experts < 0 || experts > REGOT_ROW_MAX_EXPERTS) return REGOT_ERR_DIM;
    if (k < 1 || k > REGOT_ROW_MAX_CHOICES) return REGOT_ERR_ARG;
    if (n > kMaxDim / k) return REGOT_ERR_DIM;
    return REGOT_OK;
}

// ---- memory that two matrices share ----

struct Memory {
    const void *p;
    int64_t n, m, ld;  // rows, numbers of each, distance of rows
    int bytes;         // of a number
};

// Whether an element of one may be one of the other's.  Rows of one may lie between those of the other where their distances are the same.
bool meet(const Memory &a, const Memory &b)
{
    typedef __int128 wide;
    if (!a.p || !b.p || a.n == 0 || a.m == 0 || b.n == 0 || b.m == 0) return false;
    const wide a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p, ra = (wide)a.m * a.bytes, rb = (wide)b.m * b.bytes;
    const wide sa = (wide)a.ld * a.bytes, sb = (wide)b.ld * b.bytes;
    if (a0 >= b0 + (b.n - 1) * sb + rb || b0 >= a0 + (a.n - 1) * sa + ra) return false;
    if (sa != sb || a.n == 1 || b.n == 1) return true;
    const wide off = ((b0 - a0) % sa + sa) % sa;  // where b's rows begin in a's
    return off < ra || off + rb > sa;
}

// (for each output, the inputs and the outputs before it)
bool meets(const Memory &a, std::initializer_list<Memory> others)
{
    return std::any_of(others.begin(), others.end(), [&](const Memory &b) { return meet(a, b); });
}

Memory list_of(const void *p, int64_t count, int bytes) { return {p, 1, count, 0, bytes}; }

// The matrix of a call's weights: experts blocks, as rows one after the other
Memory blocks_of(const void *p, int64_t experts, int64_t n, int64_t m, int64_t ld, int64_t stride, int bytes)
{
    if (experts == 0 || n == 0 || m == 0) return {nullptr, 0, 0, 0, bytes};
    return {p, 1, (experts - 1) * stride + (n - 1) * ld + m, 0, bytes};
}

// ---- products ----

int check_group(int64_t rows, int64_t m, int64_t d, int64_t experts, const int64_t *start, int type)
{
    if (bad_dim(rows) || bad_dim(m) || bad_dim(d) || experts < 0 || experts > REGOT_ROW_MAX_EXPERTS) return REGOT_ERR_DIM;
    if (bad_type(type)) return REGOT_ERR_ARG;
    if (experts > 0 && !start) return REGOT_ERR_NULL;
    if (misaligned(start, 8)) return REGOT_ERR_ALIGN;
    return REGOT_OK;
}

// Rows of X that a product or a weight gradient takes
int check_source(int64_t rows, int64_t d, const void *X, int64_t ldX, int64_t x_rows, const int32_t *order, int k, int type)
{
    if (bad_dim(x_rows)) return REGOT_ERR_DIM;
    if (k < 1 || k > REGOT_ROW_MAX_CHOICES) return REGOT_ERR_ARG;
    if (rows > 0 && d > 0 && !X) return REGOT_ERR_NULL;
    if (rows > 0 && (order ? x_rows == 0 : x_rows < rows)) return REGOT_ERR_DIM;
    if (ldX < d) return REGOT_ERR_LD;
    if (misaligned(X, element_bytes(type)) || misaligned(order, 4)) return REGOT_ERR_ALIGN;
    return REGOT_OK;
}

// Chunks of 16 bytes that begin at multiples of 16 bytes
bool whole_chunks(const void *p, int64_t numbers, int64_t ld, int bytes)
{
    return !misaligned(p, 16) && numbers % (16 / bytes) == 0 && ld % (16 / bytes) == 0;
}

GroupArgs group_args(int64_t rows, int64_t m, int64_t d, int64_t experts, const int64_t *start, const void *X, int64_t ldX, int64_t x_rows,
                     const int32_t *order, int k)
{
    GroupArgs A{};
    A.start = start;
    A.rows = rows;
    A.experts = (int)experts;
    A.order = order;
    A.by_k = divide_by((uint32_t)k);
    A.x_rows = x_rows;
    A.X = X;
    A.ldX = ldX;
    A.m = m;
    A.d = d;
    A.splits = 1;
    return A;
}

void launch(const GroupArgs &A, const TilePlan &P, int type, hipStream_t s)
{
    if (type == REGOT_F32) expert_tiles_f32(A, P, s);
    else if (type == REGOT_BF16) expert_tiles_bf16(A, P, s);
    else expert_tiles_f16(A, P, s);
}

// Tiles of 256 x 256 (one to a compute unit, 128 x 128 for each wave) do more of the products for what they read than those of 128 x 128 (two to a unit) or 64 x 128
// (three), and leave more of the chip empty in the last round.  us, 256 / 128: 131072 rows of 64 experts, 1024 x 2048: product 577 / 715 (4400 tiles of 256),
// weight gradient 648 / 778 (2048 tiles); 32768 rows of 60, 2048 by 2 x 1024 with the gate 353 / 390 (1264); 8192 rows of 8, 2048 x 1408: 87 / 83 (216), weight gradient
// 80 / 69 (384).  128 / 64 rows: gradients of 2997 rows of 12 experts, 555 x 777: fp32 285 / 161, bf16 50 / 46 (250 and 420 tiles of 128).
// So they are taken from `least` tiles on:
// weight gradients 2 rounds; products 2.5 (576 tiles: 16384 rows of 16, 1024 x 2048 90 / 80; 720: 2048 x 2560 188 / 206), but none of fewer than 192 rows an expert, which
// leave most of a tall tile empty (600 rows of 128, 1024 x 2048 133 / 109, 16384 rows 160 / 156); behind the gate, where a tile ends with as many reads as writes and nothing
// else runs on its unit, 4 rounds of long sums (65536 rows of 64, 1024 outputs, sums of 512 238 / 201, 1024 296 / 273, 2048 411 / 417, 4096 655 / 711; where each expert has 1024 rows, which
// fill tall tiles, sums of 1536 306 / 324, 2048 352 / 388, 4096 556 / 650).
constexpr int64_t kNever = INT64_MAX;

int64_t least_tall(int kind, int64_t rows, int64_t d, int64_t experts)
{
    if (kind == kWeightGrad) return 2 * kCUs;
    if (rows < 192 * experts) return kNever;
    return kind != kGateGrad ? 5 * kCUs / 2 : d >= 2048 ? 4 * kCUs : kNever;
}

template <typename Tiles>
int choose_tile(int type, bool direct, int64_t least, Tiles tiles)
{
    if (direct && type != REGOT_F32 && tiles(tile_shape(kTileBig)) >= least) return kTileBig;
    const bool small = tiles(tile_shape(kTileDirect)) < 2 * kCUs;
    return direct ? small ? kTileDirectSmall : kTileDirect : small ? kTileStagedSmall : kTileStaged;
}

// (us, tiles of 64 x 128 / few rows, bf16, 60 experts: 1400 x 2048, 480 rows 79 / 68, 960 72 / 86; 1400 x 4096 147 / 129, 148 / 167; 512 x 4096 55 / 45, 53 / 57; 16 of 2048 x 4096, 256
// rows 58 / 52; fp32, 4 / 8 / 12 / 16 rows of each: 60 of 1400 x 2048 204 / 138, 187 / 137, 187 / 149, 187 / 174, 16 of 2048 x 2048 117 / 59, 114 / 59, 114 / 59, 114 / 60, 256 of 1024 x
// 512 151 / 118, 147 / 118, 145 / 119, 145 / 178; bf16, short sums: 60 of 1400 x 1024 33 / 40, 33 / 41, 34 / 46, 34 / 58)
constexpr int64_t kFewRows = 12;  // rows of an expert, on average

// How many stretches of 32 rows of W a workgroup of the kernel for few rows has, of `all` that each of `runs` experts' weights have: four rounds of workgroups, one to a
// compute unit, so that the last one does not weigh much, or one where two stretches are enough for that.  us, 1 / 2 / 4 / 8 / 16 stretches: 256 rows of 60 experts, 1400 x
// 2048 fp16 104 / 81 / 70 / 81 / 98; 8 rows of 256 experts, 2048 x 2 x 1024 bf16 with the gate 13.7 to 18 / 14.3 / 15 / 20 / 34.
int64_t few_groups(int64_t runs, int64_t all)
{
    const auto rounds = [&](int64_t n) { return (runs * all + n * kCUs - 1) / (n * kCUs); };
    return std::min(all, std::max(rounds(4), std::min<int64_t>(rounds(1), 2)));
}

// A weight gradient of few tiles is summed in parts of so many rows at least, which a second launch adds up.  us, parts of 512 / 256 / 128 / 64 rows: fp32, 71904 rows
// of 120 experts, 64 x 111 91 / 56 / 37 / 37, 2048 of 8, 256 x 256 22 / 22 / 18 / 17; bf16, 71904 rows of 120, 64 x 128 11 / 15 / 18 / 18, 1000 of 4, 512 x 512 8 / 8 / 8 / 15.
constexpr int64_t kPart = 512, kPartF32 = 128;

struct GradPlan {
    int64_t tiles_m = 0, tiles_d = 0;
    int splits = 1;
    size_t total = 0;
    int64_t tiles(int64_t experts) const { return tiles_m * tiles_d * experts * splits; }
};

GradPlan plan_weight_grad(int64_t rows, int64_t m, int64_t d, int64_t experts, int tile, int64_t part)
{
    GradPlan P;
    const TileShape T = tile_shape(tile);
    P.tiles_m = (m + T.rows - 1) / T.rows;
    P.tiles_d = (d + T.cols - 1) / T.cols;
    const int64_t tiles = P.tiles_m * P.tiles_d * experts;
    if (tiles > 0 && tiles < kCUs) P.splits = (int)std::max<int64_t>(std::min<int64_t>(2 * kCUs / tiles, rows / experts / part), 1);
    P.total = padded(P.splits > 1 ? (size_t)P.splits * experts * m * d * sizeof(float) : 0);
    return P;
}

struct JoinArgs {
    const float *parts;
    int64_t numbers, m, d;  // of a part; of an expert's matrix
    int splits;
    void *out;
    int64_t ld, stride;
};

// The parts of a weight gradient, in their order
template <int OUT>
__global__ void __launch_bounds__(kThreads) expert_join_kernel(const JoinArgs A)
{
    using T = Score<OUT>;
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < A.numbers; i += step) {
        float v = 0.f;
        for (int s = 0; s < A.splits; ++s) v += A.parts[s * A.numbers + i];
        const int64_t row = i / A.d, c = i % A.d;
        static_cast<typename T::Raw *>(A.out)[row / A.m * A.stride + row % A.m * A.ld + c] = T::put(v);
    }
}

// ---- the norm ----

constexpr int64_t kLeastEach = 8 * kThreads;  // numbers of a workgroup
constexpr int64_t kMostParts = 16384;  // (4096: 1.2 GB in 300 tensors 759 us in the place of 692, the ends of the launches are longer)
constexpr uint32_t kFewParts = 2048;           // partial sums that each workgroup of the scaling adds up itself

int check_tensors(int64_t count, const regot_tensor *list, bool clip)
{
    if (count < 0 || count > kMaxDim) return REGOT_ERR_DIM;
    if (count > 0 && !list) return REGOT_ERR_NULL;
    for (int64_t t = 0; t < count; ++t) {
        if (list[t].count < 0 || list[t].count > kMaxNumbers) return REGOT_ERR_DIM;
        if (bad_type(list[t].type)) return REGOT_ERR_ARG;
        if (list[t].count > 0 && (!list[t].data || (clip && !list[t].out))) return REGOT_ERR_NULL;
        const size_t b = element_bytes(list[t].type);
        if (misaligned(list[t].data, b) || (clip && misaligned(list[t].out, b))) return REGOT_ERR_ALIGN;
    }
    return REGOT_OK;
}

// Numbers of a workgroup, and workgroups of all tensors: as many as a sum takes, whatever the tensors' sizes are
struct ClipPlan {
    int64_t each = kLeastEach, parts = 0;
};

ClipPlan plan_clip(int64_t count, const regot_tensor *list)
{
    ClipPlan P;
    int64_t all = 0;
    for (int64_t t = 0; t < count; ++t) all += list[t].count / kLeastEach + 1;
    while (all / (P.each / kLeastEach) > kMostParts && P.each < kMaxNumbers) P.each *= 2;
    for (int64_t t = 0; t < count; ++t) P.parts += (list[t].count + P.each - 1) / P.each;
    return P;
}

template <typename Launch>
void for_lists(int64_t count, const regot_tensor *list, ClipArgs &A, Launch launch)
{
    int64_t t = 0;
    A.part = 0;
    while (t < count) {
        A.tensors = 0;
        A.blocks = 0;
        for (; t < count && A.tensors < kListed; ++t) {
            if (list[t].count == 0) continue;
            A.list[A.tensors++] = {list[t].data, list[t].out, list[t].count, A.blocks, list[t].type};
            A.blocks += (uint32_t)((list[t].count + A.each - 1) / A.each);
        }
        if (A.blocks > 0) launch();
        A.part += A.blocks;
    }
}

int clip(int64_t count, const regot_tensor *list, double max_norm, float *norm, float *factor, void *workspace, size_t workspace_bytes,
         hipStream_t s, bool scale)
{
    const ClipPlan P = plan_clip(count, list);
    if (!workspace) return REGOT_ERR_NULL;
    if (misaligned(workspace, kAlign)) return REGOT_ERR_ALIGN;
    if (workspace_bytes < padded(P.parts * sizeof(double))) return REGOT_ERR_WORKSPACE;
    const Memory norms = list_of(norm, 1, 4), factors = list_of(factor, 1, 4);
    if (meet(norms, factors)) return REGOT_ERR_ARG;
    for (int64_t t = 0; t < count; ++t) {
        const int b = element_bytes(list[t].type);
        const Memory in = list_of(list[t].data, list[t].count, b), out = list_of(scale ? list[t].out : nullptr, list[t].count, b);
        if (meets(norms, {in, out}) || meets(factors, {in, out})) return REGOT_ERR_ARG;
    }
    ClipArgs A{};
    A.each = P.each;
    A.parts = (uint32_t)P.parts;
    A.max_norm = max_norm;
    A.sums = static_cast<double *>(workspace);
    A.norm = norm;
    A.factor = factor;
    for_lists(count, list, A, [&] { hipLaunchKernelGGL(grad_norm_kernel, dim3(A.blocks), dim3(kThreads), 0, s, A); });
    const bool few = scale && P.parts > 0 && P.parts <= kFewParts;
    if (!few) hipLaunchKernelGGL(grad_factor_kernel, dim3(1), dim3(kThreads), 0, s, A);
    if (!scale) return hip_status();
    A.backwards = 1;
    for_lists(count, list, A, [&] {
        if (few) hipLaunchKernelGGL(grad_scale_kernel<true>, dim3(A.blocks), dim3(kThreads), 0, s, A);
        else hipLaunchKernelGGL(grad_scale_kernel<false>, dim3(A.blocks), dim3(kThreads), 0, s, A);
    });
    return hip_status();
}

// Memory that two tensors of a list share would be scaled twice, or read after it was written.  (REGOT_ERR_HIP: no host memory to find out with.)
int check_apart(int64_t count, const regot_tensor *list)
{
    struct Part {
        uintptr_t from, to;
        bool out;
    };
    const std::unique_ptr<Part[]> parts(new (std::nothrow) Part[2 * (size_t)count + 1]);
    if (!parts) return REGOT_ERR_HIP;
    size_t n = 0;
    for (int64_t t = 0; t < count; ++t) {
        if (list[t].count == 0) continue;
        const size_t bytes = (size_t)list[t].count * element_bytes(list[t].type);
        const uintptr_t in = (uintptr_t)list[t].data, out = (uintptr_t)list[t].out;
        if (out != in) parts[n++] = {in, in + bytes, false};
        parts[n++] = {out, out + bytes, true};
    }
    std::sort(parts.get(), parts.get() + n, [](const Part &a, const Part &b) { return a.from < b.from; });
    uintptr_t end = 0, out_end = 0;  // of the parts so far, and of those that are written
    for (size_t i = 0; i < n; ++i) {
        const Part &p = parts[i];
        if (p.from < (p.out ? end : out_end)) return REGOT_ERR_ARG;
        end = std::max(end, p.to);
        if (p.out) out_end = std::max(out_end, p.to);
    }
    return REGOT_OK;
}

}  // namespace

extern "C" {

int regot_expert_order_workspace_bytes(int64_t n, int k, int64_t experts, size_t *bytes)
{
    if (!bytes) return REGOT_ERR_NULL;
    const int st = check_order(n, k, experts);
    if (st != REGOT_OK) return st;
    *bytes = plan_order(n * k, experts).total;
    return REGOT_OK;
}

int regot_expert_order(int64_t n, int k, int64_t experts, const int32_t *idx, int64_t *start, int32_t *order, int32_t *place, void *workspace,
                       size_t workspace_bytes, regot_stream_t stream)
{
    const int st = check_order(n, k, experts);
    if (st != REGOT_OK) return st;
    if (!start || (n > 0 && (!idx || !order || !place))) return REGOT_ERR_NULL;
    if (misaligned(start, 8) || misaligned(idx, 4) || misaligned(order, 4) || misaligned(place, 4)) return REGOT_ERR_ALIGN;
    const OrderPlan P = plan_order(n * k, experts);
    if (!workspace) return REGOT_ERR_NULL;
    if (misaligned(workspace, kAlign)) return REGOT_ERR_ALIGN;
    if (workspace_bytes < P.total) return REGOT_ERR_WORKSPACE;
    const Memory in = list_of(idx, n * k, 4), to = list_of(order, n * k, 4), back = list_of(place, n * k, 4), runs = list_of(start, experts + 1, 8);
    if (meet(to, in) || meets(back, {in, to}) || meets(runs, {in, to, back})) return REGOT_ERR_ARG;
    OrderArgs A{};
    A.idx = idx;
    A.count = n * k;
    A.experts = (int)experts;
    while ((1 << A.key_bits) <= A.experts) ++A.key_bits;
    A.each = P.each;
    A.groups = P.groups;
    A.counts = static_cast<uint32_t *>(workspace);
    A.start = start;
    A.order = order;
    A.place = place;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (P.groups > 1) hipLaunchKernelGGL(expert_count_kernel, dim3(P.groups), dim3(kOrderThreads), 0, s, A);
    hipLaunchKernelGGL(expert_order_kernel, dim3(P.groups), dim3(kOrderThreads), 0, s, A);
    return hip_status();
}

int regot_expert_product(int64_t rows, int64_t m, int64_t d, int64_t experts, const int64_t *start, const void *X, int type, int64_t ldX,
                         int64_t x_rows, const int32_t *order, int k, const void *W, int w_by, int64_t ldW, int64_t strideW, int act, void *Y,
                         int64_t ldY, void *saved, int64_t ldSaved, regot_stream_t stream)
{
    int st = check_group(rows, m, d, experts, start, type);
    if (st == REGOT_OK) st = check_source(rows, d, X, ldX, x_rows, order, k, type);
    if (st != REGOT_OK) return st;
    if ((w_by != REGOT_W_OUTPUTS && w_by != REGOT_W_INPUTS) || (act != REGOT_ACT_NONE && act != REGOT_ACT_GATE && act != REGOT_ACT_GATE_GRAD))
        return REGOT_ERR_ARG;
    const int64_t wide = act == REGOT_ACT_GATE ? 2 * m : m, out = act == REGOT_ACT_GATE_GRAD ? 2 * m : m;
    if (2 * m > kMaxDim) return REGOT_ERR_DIM;
    const int64_t w_rows = w_by == REGOT_W_OUTPUTS ? wide : d, w_cols = w_by == REGOT_W_OUTPUTS ? d : wide;
    const bool work = rows > 0 && m > 0 && experts > 0;
    if (work && (!Y || (d > 0 && !W) || (act == REGOT_ACT_GATE_GRAD && !saved))) return REGOT_ERR_NULL;
    if (ldW < w_cols || strideW < 0 || ldY < out || (saved && ldSaved < 2 * m)) return REGOT_ERR_LD;
    const int b = element_bytes(type);
    if (misaligned(W, b) || misaligned(Y, b) || misaligned(saved, b)) return REGOT_ERR_ALIGN;
    if (act == REGOT_ACT_NONE) saved = nullptr;
    if (!work) return REGOT_OK;
    const Memory y{Y, rows, out, ldY, b}, x{X, x_rows, d, ldX, b}, kept{saved, rows, 2 * m, ldSaved, b};
    const Memory w = blocks_of(W, experts, w_rows, w_cols, ldW, strideW, b);
    const Memory runs = list_of(start, experts + 1, 8), slots = list_of(order, rows, 4);
    if (meets(y, {x, w, kept, runs, slots}) || (act == REGOT_ACT_GATE && meets(kept, {x, w, runs, slots}))) return REGOT_ERR_ARG;
    GroupArgs A = group_args(rows, m, d, experts, start, X, ldX, x_rows, order, k);
    A.W = W;
    A.ldW = ldW;
    A.strideW = strideW;
    A.Y = Y;
    A.ldY = ldY;
    A.saved = saved;
    A.ldSaved = ldSaved;
    TilePlan P{};
    P.kind = act == REGOT_ACT_NONE ? kPlain : act == REGOT_ACT_GATE ? kGate : kGateGrad;
    P.across = w_by == REGOT_W_INPUTS;
    P.out_type = type;
    const bool direct = d > 0 && whole_chunks(X, d, ldX, b) && whole_chunks(W, w_cols, ldW, b) && strideW % (16 / b) == 0 && (!P.across || m % (16 / b) == 0);
    // (a half's numbers end with a chunk too)
    A.whole = whole_chunks(Y, m, ldY, b) && (!saved || whole_chunks(saved, m, ldSaved, b));
    P.units = (d * b + 128 * kFewWaves - 1) / (128 * kFewWaves);
    if (direct && !P.across && P.kind != kGateGrad && rows <= kFewRows * experts && P.units <= kFewUnits) {
        P.tile = kTileFew;
        A.groups = (int)few_groups(std::min(rows, experts), (wide + 31) / 32);
    } else {
        // (tiles of a call, where each expert's last one is half empty)
        P.tile = choose_tile(type, direct, least_tall(P.kind, rows, d, experts), [&](TileShape T) { return (rows / T.rows + experts / 2) * ((wide + T.cols - 1) / T.cols); });
    }
    const TileShape T = tile_shape(P.tile);
    const int64_t cols = P.tile == kTileFew ? T.cols * A.groups : T.cols;
    A.single = rows < rows / T.rows + experts;
    const int64_t row_tiles = A.single ? rows : rows / T.rows + experts, col_tiles = (wide + cols - 1) / cols;
    if (row_tiles * col_tiles > kMaxTiles) return REGOT_ERR_DIM;
    A.row_tiles = (uint32_t)row_tiles;
    A.col_tiles = (uint32_t)col_tiles;
    A.tiles = (uint32_t)(row_tiles * col_tiles);
    launch(A, P, type, static_cast<hipStream_t>(stream));
    return hip_status();
}

int regot_expert_weight_grad_workspace_bytes(int64_t rows, int64_t m, int64_t d, int64_t experts, size_t *bytes)
{
    if (!bytes) return REGOT_ERR_NULL;
    if (bad_dim(rows) || bad_dim(m) || bad_dim(d) || experts < 0 || experts > REGOT_ROW_MAX_EXPERTS) return REGOT_ERR_DIM;
    *bytes = plan_weight_grad(rows, m, d, experts, kTileDirectSmall, kPartF32).total;  // (larger tiles are many, and not in parts)
    return REGOT_OK;
}

int regot_expert_weight_grad(int64_t rows, int64_t m, int64_t d, int64_t experts, const int64_t *start, const void *dY, int type, int64_t ldY,
                             const void *X, int64_t ldX, int64_t x_rows, const int32_t *order, int k, void *dW, int out_type, int64_t ldW,
                             int64_t strideW, void *workspace, size_t workspace_bytes, regot_stream_t stream)
{
    int st = check_group(rows, m, d, experts, start, type);
    if (st == REGOT_OK) st = check_source(rows, d, X, ldX, x_rows, order, k, type);
    if (st != REGOT_OK) return st;
    if (out_type != type && out_type != REGOT_F32) return REGOT_ERR_ARG;
    const bool work = m > 0 && d > 0 && experts > 0;
    if (work && (!dW || (rows > 0 && !dY))) return REGOT_ERR_NULL;
    if (ldY < m || ldW < d || (experts > 1 && m > 0 && strideW < (m - 1) * ldW + d)) return REGOT_ERR_LD;
    const int b = element_bytes(type), ob = element_bytes(out_type);
    if (misaligned(dY, b) || misaligned(dW, ob)) return REGOT_ERR_ALIGN;
    const int64_t part = type == REGOT_F32 ? kPartF32 : kPart;
    GradPlan G = plan_weight_grad(rows, m, d, experts, kTileDirectSmall, part);
    if (!workspace) return REGOT_ERR_NULL;
    if (misaligned(workspace, kAlign)) return REGOT_ERR_ALIGN;
    if (workspace_bytes < G.total) return REGOT_ERR_WORKSPACE;
    if (!work) return REGOT_OK;
    const Memory w = blocks_of(dW, experts, m, d, ldW, strideW, ob);
    if (meets(w, {{dY, rows, m, ldY, b}, {X, x_rows, d, ldX, b}, list_of(start, experts + 1, 8), list_of(order, rows, 4)})) return REGOT_ERR_ARG;
    GroupArgs A = group_args(rows, m, d, experts, start, X, ldX, x_rows, order, k);
    A.W = dY;
    A.ldW = ldY;
    A.splits = G.splits;
    TilePlan P{};
    P.kind = kWeightGrad;
    P.across = 1;
    P.gather = order != nullptr;
    const bool parts = G.splits > 1;
    P.out_type = parts ? REGOT_F32 : out_type;
    A.Y = parts ? workspace : dW;
    A.ldY = parts ? d : ldW;
    A.strideY = parts ? m * d : strideW;
    const int pb = element_bytes(P.out_type);
    const bool direct = whole_chunks(X, d, ldX, b) && whole_chunks(dY, m, ldY, b);
    A.whole = whole_chunks(A.Y, d, A.ldY, pb) && A.strideY % (16 / pb) == 0;
    P.tile = kTileDirectSmall;
    if (!parts) P.tile = choose_tile(type, direct, least_tall(kWeightGrad, rows, d, experts), [&](TileShape T) { return (m + T.rows - 1) / T.rows * ((d + T.cols - 1) / T.cols) * experts; });
    else if (!direct) P.tile = kTileStagedSmall;
    if (!parts) {
        G = plan_weight_grad(rows, m, d, experts, P.tile, part);
        G.splits = 1;
    }
    const int64_t tiles = G.tiles(experts);
    if (tiles > kMaxTiles) return REGOT_ERR_DIM;
    A.row_tiles = (uint32_t)G.tiles_m;
    A.col_tiles = (uint32_t)G.tiles_d;
    A.tiles = (uint32_t)tiles;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    launch(A, P, type, s);
    if (parts) {
        const JoinArgs J{static_cast<const float *>(workspace), experts * m * d, m, d, G.splits, dW, ldW, strideW};
        const dim3 grid(grid_of((J.numbers + kThreads - 1) / kThreads));
        if (out_type == REGOT_F32) hipLaunchKernelGGL(expert_join_kernel<REGOT_F32>, grid, dim3(kThreads), 0, s, J);
        else if (out_type == REGOT_BF16) hipLaunchKernelGGL(expert_join_kernel<REGOT_BF16>, grid, dim3(kThreads), 0, s, J);
        else hipLaunchKernelGGL(expert_join_kernel<REGOT_F16>, grid, dim3(kThreads), 0, s, J);
    }
    return hip_status();
}

static int check_combine(int64_t n, int k, int64_t m, int64_t rows, int type, const void *Y, int64_t ldY, const int32_t *place, const float *weight)
{
    if (n < 0 || bad_dim(m) || bad_dim(rows)) return REGOT_ERR_DIM;
    if (k < 1 || k > REGOT_ROW_MAX_CHOICES || bad_type(type)) return REGOT_ERR_ARG;
    if (n > kMaxDim / k) return REGOT_ERR_DIM;
    if (n > 0 && (!place || (rows > 0 && m > 0 && !Y))) return REGOT_ERR_NULL;
    if (ldY < m) return REGOT_ERR_LD;
    if (misaligned(Y, element_bytes(type)) || misaligned(place, 4) || misaligned(weight, 4)) return REGOT_ERR_ALIGN;
    return REGOT_OK;
}

static CombineArgs combine_args(int64_t n, int k, int64_t m, int64_t rows, const void *Y, int64_t ldY, const int32_t *place, const float *weight)
{
    CombineArgs A{};
    A.n = n;
    A.m = m;
    A.rows = rows;
    A.k = k;
    A.Y = Y;
    A.ldY = ldY;
    A.place = place;
    A.weight = weight;
    return A;
}

int regot_expert_combine(int64_t n, int k, int64_t m, int64_t rows, const void *Y, int type, int64_t ldY, const int32_t *place, const float *weight,
                         void *out, int64_t ldO, regot_stream_t stream)
{
    const int st = check_combine(n, k, m, rows, type, Y, ldY, place, weight);
    if (st != REGOT_OK) return st;
    if (n > 0 && m > 0 && !out) return REGOT_ERR_NULL;
    if (ldO < m) return REGOT_ERR_LD;
    const int b = element_bytes(type);
    if (misaligned(out, b)) return REGOT_ERR_ALIGN;
    if (n == 0 || m == 0) return REGOT_OK;
    if (meets({out, n, m, ldO, b}, {{Y, rows, m, ldY, b}, list_of(place, n * k, 4), list_of(weight, n * k, 4)})) return REGOT_ERR_ARG;
    CombineArgs A = combine_args(n, k, m, rows, Y, ldY, place, weight);
    A.out = out;
    A.ldO = ldO;
    const int64_t columns = kLanes * 16 / b;
    A.parts = (uint32_t)((m + columns - 1) / columns);
    const dim3 grid(grid_of((n * A.parts + kWaves - 1) / kWaves));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == REGOT_F32) hipLaunchKernelGGL(expert_combine_kernel<REGOT_F32>, grid, dim3(kThreads), 0, s, A);
    else if (type == REGOT_BF16) hipLaunchKernelGGL(expert_combine_kernel<REGOT_BF16>, grid, dim3(kThreads), 0, s, A);
    else hipLaunchKernelGGL(expert_combine_kernel<REGOT_F16>, grid, dim3(kThreads), 0, s, A);
    return hip_status();
}

int regot_expert_combine_grad(int64_t n, int k, int64_t m, int64_t rows, const void *g_out, int type, int64_t ldG, const void *Y, int64_t ldY,
                              const int32_t *place, const float *weight, void *dY, int64_t ldD, float *g_weight, regot_stream_t stream)
{
    const int st = check_combine(n, k, m, rows, type, g_weight ? Y : g_out, g_weight ? ldY : m, place, weight);
    if (st != REGOT_OK) return st;
    if (n > 0 && m > 0 && (!g_out || (rows > 0 && !dY))) return REGOT_ERR_NULL;
    if (ldG < m || ldD < m) return REGOT_ERR_LD;
    const int b = element_bytes(type);
    if (misaligned(g_out, b) || misaligned(dY, b) || misaligned(g_weight, 4)) return REGOT_ERR_ALIGN;
    if (n == 0) return REGOT_OK;
    const Memory d{dY, rows, m, ldD, b}, g{g_out, n, m, ldG, b}, y{g_weight ? Y : nullptr, rows, m, ldY, b};
    const Memory places = list_of(place, n * k, 4), weights = list_of(weight, n * k, 4);
    if (meets(d, {g, y, places, weights}) || meets(list_of(g_weight, n * k, 4), {d, g, y, places, weights})) return REGOT_ERR_ARG;
    CombineArgs A = combine_args(n, k, m, rows, Y, ldY, place, weight);
    A.g = g_out;
    A.ldG = ldG;
    A.out = dY;
    A.ldO = ldD;
    A.g_weight = g_weight;
    const dim3 grid(grid_of((n * k + kWaves - 1) / kWaves));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == REGOT_F32) hipLaunchKernelGGL(expert_combine_grad_kernel<REGOT_F32>, grid, dim3(kThreads), 0, s, A);
    else if (type == REGOT_BF16) hipLaunchKernelGGL(expert_combine_grad_kernel<REGOT_BF16>, grid, dim3(kThreads), 0, s, A);
    else hipLaunchKernelGGL(expert_combine_grad_kernel<REGOT_F16>, grid, dim3(kThreads), 0, s, A);
    return hip_status();
}

int regot_grad_norm_workspace_bytes(int64_t count, const regot_tensor *list, size_t *bytes)
{
    if (!bytes) return REGOT_ERR_NULL;
    const int st = check_tensors(count, list, false);
    if (st != REGOT_OK) return st;
    *bytes = padded(plan_clip(count, list).parts * sizeof(double));
    return REGOT_OK;
}

int regot_grad_norm(int64_t count, const regot_tensor *list, float *norm, void *workspace, size_t workspace_bytes, regot_stream_t stream)
{
    const int st = check_tensors(count, list, false);
    if (st != REGOT_OK) return st;
    if (!norm) return REGOT_ERR_NULL;
    if (misaligned(norm, 4)) return REGOT_ERR_ALIGN;
    return clip(count, list, 1.0, norm, nullptr, workspace, workspace_bytes, static_cast<hipStream_t>(stream), false);
}

int regot_grad_clip(int64_t count, const regot_tensor *list, double max_norm, float *norm, float *factor, void *workspace, size_t workspace_bytes,
                    regot_stream_t stream)
{
    int st = check_tensors(count, list, true);
    if (st != REGOT_OK) return st;
    if (!(max_norm > 0.0)) return REGOT_ERR_ARG;
    if (!norm || !factor) return REGOT_ERR_NULL;
    if (misaligned(norm, 4) || misaligned(factor, 4)) return REGOT_ERR_ALIGN;
    st = check_apart(count, list);
    if (st != REGOT_OK) return st;
    return clip(count, list, max_norm, norm, factor, workspace, workspace_bytes, static_cast<hipStream_t>(stream), true);
}

}  // extern "C"
