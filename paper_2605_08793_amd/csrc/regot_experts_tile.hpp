// Products grouped by expert: tiles of a matrix product on the matrix cores (gfx950, wave64).
#pragma once

#include "regot_experts.hpp"

namespace regot {

// What a tile's product becomes: stored; put through the gate; put through the gate's gradient; a weight gradient's (part of a) sum
enum { kPlain = 0, kGate = 1, kGateGrad = 2, kWeightGrad = 3 };

__device__ const uint32_t kNoNumbers[8] = {};  // what is loaded in the place of numbers that are not there: 0

// 64 lanes' 16 bytes each from memory to LDS, one lane's behind the other's from `lds` on (the same in all lanes), without registers between.  Nothing waits
// for it but s_waitcnt vmcnt.  (As the compiler's builtin it would make every read of LDS behind it wait, whatever it reads.)
__device__ __forceinline__ void load_to_lds(const char *p, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// One side of a tile: EXT rows (or columns) of a matrix, 128 bytes of each along the sum at a time.  LDS holds them
//   TRANS = false (numbers along the sum are neighbours in memory): row after row, 8 chunks of 16 bytes each
//   TRANS = true (the matrix is read across): for each of the kSum places of the sum its EXT numbers
// with the chunks of a row in an order that depends on the row, so that the lanes that read together meet different banks.
// Row of fragment f (16 rows) that lane i (of 16) reads, from the pair p = f / 2 on:
//   TRANS = false 32 p + 8 (i / 4) + 4 (f % 2) + i % 4 (so that a lane's results are 8 neighbours), TRANS = true 16 f + i
template <int TYPE, int EXT, bool TRANS, int THREADS>
struct Side {
    using Raw = typename Score<TYPE>::Raw;
    static constexpr int kElem = sizeof(Raw), kChunk = 16 / kElem, kSum = 128 / kElem;
    static constexpr int kBytes = EXT * 128, kLoads = kBytes / (16 * THREADS);
    static constexpr int kRowChunks = TRANS ? EXT / kChunk : 8;
    static_assert(kLoads * 16 * THREADS == kBytes, "every thread loads whole chunks");

    static __device__ __forceinline__ int turn(int row)
    {
        if constexpr (TRANS) return (((row & 3) | ((row >> 3) & 1) << 2) << 1) & (kRowChunks - 1);
        return ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
    }
    // place ii of this thread: row of LDS and chunk of it
    static __device__ __forceinline__ int place(int ii)
    {
        const int wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
        return (wave * kLoads + ii) * kLanes + lane;
    }
    static __device__ __forceinline__ int lds_row(int ii) { return place(ii) / kRowChunks; }
    static __device__ __forceinline__ int chunk(int ii) { return (place(ii) % kRowChunks) ^ turn(lds_row(ii)); }

    // the 16 bytes of a fragment that lane (16 g + i) has at step `step` of 64 bytes along the sum
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int f0, int f, int step)
    {
        const int lane = threadIdx.x % kLanes, g = lane / 16, i = lane % 16;
        if constexpr (!TRANS) {
            const int row = f0 * 16 + (f / 2) * 32 + 8 * (i / 4) + 4 * (f % 2) + i % 4;
            return *reinterpret_cast<const u32x4 *>(lds + row * 128 + ((step * 4 + g) ^ turn(row)) * 16);
        } else if constexpr (kElem == 2) {
            u32x4 v;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = step * 32 + 8 * g + 4 * h + i / 4, at = (f0 + f) * 16 + 4 * (i % 4);
                const char *from = lds + k * (EXT * 2) + ((at / 8) ^ turn(k)) * 16 + (at % 8) * 2;
                const i16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(const_cast<char *>(from)));
                __builtin_memcpy(reinterpret_cast<char *>(&v) + 8 * h, &part, 8);
            }
            return v;
        } else {
            u32x4 v;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int k = step * 16 + 4 * g + s, at = (f0 + f) * 16 + i;
                v[s] = *reinterpret_cast<const uint32_t *>(lds + k * (EXT * 4) + ((at / 4) ^ turn(k)) * 16 + (at % 4) * 4);
            }
            return v;
        }
    }
};

// Loads of one side, kSum places of the sum at a time.  DIRECT: whole chunks that are 16 bytes aligned, from memory straight into LDS;
// the first `rest` places of a sum, which need not be kSum, come first, the others in whole stretches behind them.  Otherwise through registers, at any
// alignment, numbers beyond the matrix as 0, the last stretch as short as it is.
template <int TYPE, int EXT, bool TRANS, int THREADS, bool DIRECT, bool GATHER, bool HALVES>
struct Loader {
    using S = Side<TYPE, EXT, TRANS, THREADS>;
    using Raw = typename S::Raw;
    const char *at[S::kLoads];  // of the next chunks (GATHER: of their columns)
    int64_t step;               // to those after them
    u32x4 kept[DIRECT ? 1 : S::kLoads];
    int32_t next_slot[GATHER ? S::kLoads : 1];
    const GroupArgs *args;
    int64_t ld;

    // TRANS = false: row(i) is the address of the i-th row, from the sum's first place on
    template <typename Row>
    __device__ __forceinline__ void rows(Row row)
    {
        step = 128;
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) at[ii] = row(S::lds_row(ii)) + S::chunk(ii) * 16;
    }
    // TRANS = true: the matrix at p, numbers first .. extent - 1 of its rows, whose distance is ld_ numbers.  HALVES: half of the tile's are
    // those, and half the numbers of the same places behind extent.
    static __device__ __forceinline__ int column(int ii) { return S::chunk(ii) * S::kChunk % (HALVES ? EXT / 2 : EXT); }
    __device__ __forceinline__ void across(const char *p, int64_t ld_, int64_t first, int64_t extent)
    {
        ld = ld_ * S::kElem;
        step = S::kSum * ld;
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) {
            int64_t c = first + column(ii);
            if constexpr (DIRECT) c = min(c, extent - S::kChunk);  // (what is loaded there is not used)
            if (HALVES && S::chunk(ii) * S::kChunk >= EXT / 2) c += extent;
            at[ii] = p + c * S::kElem + (GATHER ? 0 : S::lds_row(ii) * ld);
        }
    }
    // which slots the next kSum places of a gathered sum are, the first of them row `row`, all before `end`: asked for while the stretch before is on its
    // way, and there (`gathered`) when the waves have met, so that nothing waits for them
    __device__ __forceinline__ void gather(const GroupArgs &A, int64_t row, int64_t end)
    {
        args = &A;
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) next_slot[ii] = A.order[min(row + S::lds_row(ii), end - 1)];
    }
    __device__ __forceinline__ void gathered()
    {
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) asm volatile("" : "+v"(next_slot[ii]));
    }
    __device__ __forceinline__ const char *chunk_at(int ii) const { return GATHER ? at[ii] + row_of_slot(*args, next_slot[ii]) * ld : at[ii]; }

    // DIRECT: the first `rest` places; then whole stretches, load ii of one, and the way to the next (none where there is no next)
    __device__ __forceinline__ void first(uint32_t lds, int rest)
    {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) {
            const int k = TRANS ? S::lds_row(ii) : S::chunk(ii) * S::kChunk;
            load_to_lds(k < rest ? chunk_at(ii) : reinterpret_cast<const char *>(kNoNumbers), lds + (wave * S::kLoads + ii) * 1024);
            if constexpr (!GATHER) at[ii] += TRANS ? rest * ld : rest * S::kElem;
        }
    }
    __device__ __forceinline__ void load(int ii, uint32_t lds, int64_t by)
    {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
        load_to_lds(chunk_at(ii), lds + (wave * S::kLoads + ii) * 1024);
        if constexpr (!GATHER) at[ii] += by;
    }

    // through registers: the chunks of places done .. of a sum of `sum` places; first, extent: as for across
    __device__ __forceinline__ void fetch(int64_t done, int64_t sum, int64_t first, int64_t extent)
    {
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) {
            const char *p = chunk_at(ii);
            if constexpr (!GATHER) at[ii] += step;
            const int64_t k = done + (TRANS ? S::lds_row(ii) : S::chunk(ii) * S::kChunk);
            const int64_t left = TRANS ? (k < sum ? extent - first - column(ii) : 0) : sum - k;
            u32x4 v = {0, 0, 0, 0};
            if (left >= S::kChunk) {
                __builtin_memcpy(&v, p, 16);
            } else {
                Raw part[S::kChunk];
#pragma unroll
                for (int c = 0; c < S::kChunk; ++c) part[c] = c < left ? reinterpret_cast<const Raw *>(p)[c] : Raw(0.f);
                __builtin_memcpy(&v, part, 16);
            }
            kept[ii] = v;
        }
    }
    __device__ __forceinline__ void put(char *lds)
    {
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) *reinterpret_cast<u32x4 *>(lds + S::place(ii) * 16) = kept[ii];
    }
};

template <int TYPE>
__device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (TYPE == REGOT_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (TYPE == REGOT_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[s]), __uint_as_float(b[s]), c, 0, 0, 0);
        return c;
    }
}

// 8 numbers of 32 bits, times 2^24, as three of 8 significant bits each.  The scaled number's last bit is not below 2^-125, so the pieces are normal numbers or 0, and add up to it exactly,
// whatever number of 32 bits it was.  (Numbers that are not finite, or from 2^104 on, give a NaN or an infinity.)
struct Pieces {
    static constexpr float kScale = 0x1p24f, kUnscale = 0x1p-48f;  // of a number; of a product of two

    u32x4 high, mid, low;
    static __device__ __forceinline__ uint32_t rounded(float x, float y)
    {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
    }
    __device__ __forceinline__ Pieces(u32x4 a, u32x4 b)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = kScale * __uint_as_float(i < 2 ? a[2 * i] : b[2 * i - 4]), y = kScale * __uint_as_float(i < 2 ? a[2 * i + 1] : b[2 * i - 3]);
            high[i] = rounded(x, y);
            x -= __uint_as_float(high[i] << 16);
            y -= __uint_as_float(high[i] & 0xffff0000u);
            mid[i] = rounded(x, y);
            x -= __uint_as_float(mid[i] << 16);
            y -= __uint_as_float(mid[i] & 0xffff0000u);
            low[i] = rounded(x, y);
        }
    }
};

// The products of pieces that are not below 2^-24 of the whole, the smallest first: 6 of 16 cycles in the place of 8 of 32 for the same numbers as they are
template <int COUNT>
__device__ __forceinline__ void multiply_pieces(const Pieces (&a)[COUNT], const Pieces &b, f32x4 (&c)[COUNT])
{
    const auto add = [&](u32x4 Pieces::*p, u32x4 Pieces::*q) {
#pragma unroll
        for (int y = 0; y < COUNT; ++y) c[y] = multiply<REGOT_BF16>(a[y].*p, b.*q, c[y]);
    };
    add(&Pieces::low, &Pieces::high);
    add(&Pieces::high, &Pieces::low);
    add(&Pieces::mid, &Pieces::mid);
    add(&Pieces::mid, &Pieces::high);
    add(&Pieces::high, &Pieces::mid);
    add(&Pieces::high, &Pieces::high);
}

// A product of 16 bits where it stands and with the sum in the accumulation registers: as a builtin the compiler keeps sums of 256 registers a lane in
// the others, moves and spills them, and gathers the reads of LDS in front of the products.  What the compiler does not know to keep apart here: a
// number that an instruction other than a load writes may be multiplied two cycles later (s_nop 1, in the shadow of the product before), and sums are read
// behind `multiplied`.
template <int TYPE>
__device__ __forceinline__ void multiply_here(u32x4 a, u32x4 b, f32x4 &c)
{
    if constexpr (TYPE == REGOT_BF16) asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    else asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// 0, as a product's result
__device__ __forceinline__ void clear_here(f32x4 &c)
{
    const u32x4 none = {0, 0, 0, 0};
    asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_f16 %0, %1, %1, 0" : "=a"(c) : "v"(none));
}

// Products' results before other instructions read them, which takes 18 cycles at most behind the last product: behind the wait for that, each goes
// through an empty instruction, or its reads could come before the wait.
template <int COUNT>
__device__ __forceinline__ void multiplied(f32x4 (&c)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) asm volatile("" : "+a"(c[i]));
}

// A wave's results, ROWS x COLS fragments, through its own part of LDS, so that they go to memory as whole rows and not as the pieces of 8 or
// 16 bytes that a lane has (131072 x 1024 by 64 x 2048 x 1024, bf16: 693 us without, see the table at the kernel).  value(x, y, e): result e of run y (of 8
// neighbours, or 4 where ACROSS) in fragment row x; take(x, i, c, v, asked): 16 bytes of numbers of type TYPE, row i of fragment row x, from column c on, with
// what ask(x, i, c) gave, which is asked for eight times before the first is taken.
// Chunks of 16 bytes lie in an order that depends on their row, as in Side.
template <int TYPE, int ROWS, int COLS, bool ACROSS, int BYTES, typename Value, typename Ask, typename Take>
__device__ __forceinline__ void through_lds(char *mine, Value value, Ask ask, Take take)
{
    using Raw = typename Score<TYPE>::Raw;
    constexpr int kElem = sizeof(Raw), kRun = ACROSS ? 4 : 8, kRow = COLS * 16 * kElem, kChunks = kRow / 16, kPiece = kRun * kElem < 16 ? kRun * kElem : 16;
    constexpr int kFit = BYTES / (16 * kRow), kPass = kFit < ROWS ? kFit : ROWS;
    static_assert(kPass >= 1, "a row of fragments fits");
    const int lane = threadIdx.x % kLanes, g = lane / 16, i = lane % 16;
#pragma unroll
    for (int x0 = 0; x0 < ROWS; x0 += kPass) {
#pragma unroll
        for (int x = x0; x < min(x0 + kPass, ROWS); ++x)
#pragma unroll
            for (int y = 0; y < COLS * 4 / kRun; ++y) {
                Raw v[kRun];
#pragma unroll
                for (int e = 0; e < kRun; ++e) v[e] = Score<TYPE>::put(value(x, y, e));
#pragma unroll
                for (int p = 0; p < kRun * kElem; p += kPiece) {
                    const int at = (y * 4 * kRun + kRun * g) * kElem + p;
                    char *to = mine + ((x - x0) * 16 + i) * kRow + ((at / 16) ^ (i & (kChunks - 1))) * 16 + at % 16;
                    __builtin_memcpy(__builtin_assume_aligned(to, kPiece), reinterpret_cast<const char *>(v) + p, kPiece);
                }
            }
        wave_lds();
        constexpr int kRowsAtOnce = kLanes / kChunks, kAsked = 8;
        const int row = lane / kChunks, chunk = lane % kChunks;
        const int all = min(kPass, ROWS - x0) * 16 / kRowsAtOnce;
#pragma unroll 1
        for (int it0 = 0; it0 < all; it0 += kAsked) {
            decltype(ask(0, 0, 0)) asked[kAsked];
#pragma unroll
            for (int j = 0; j < kAsked; ++j) {
                const int at = min(it0 + j, all - 1) * kRowsAtOnce + row;
                asked[j] = ask(x0 + at / 16, at % 16, chunk * 16 / kElem);
            }
#pragma unroll
            for (int j = 0; j < kAsked; ++j) {
                const int at = (it0 + j) * kRowsAtOnce + row, of = at % 16;
                if (it0 + j >= all) break;
                take(x0 + at / 16, of, chunk * 16 / kElem, *reinterpret_cast<const u32x4 *>(mine + at * kRow + (chunk ^ (of & (kChunks - 1))) * 16), asked[j]);
            }
        }
        wave_lds();
    }
}

// The same without LDS, where a lane's 8 neighbours are 16 bytes (of 64 that follow each other): the same product with weights by outputs 634 us, through LDS 653.
template <int TYPE, int ROWS, int COLS, bool ACROSS, int BYTES, typename Value, typename Take>
__device__ __forceinline__ void results(char *mine, Value value, Take take)
{
    using Raw = typename Score<TYPE>::Raw;
    if constexpr (ACROSS) {
        through_lds<TYPE, ROWS, COLS, ACROSS, BYTES>(mine, value, [](int, int, int) { return 0; }, [&](int x, int i, int c, u32x4 v, int) { take(x, i, c, v); });
    } else {
        constexpr int kChunk = 16 / sizeof(Raw);
        const int lane = threadIdx.x % kLanes, g = lane / 16, i = lane % 16;
#pragma unroll
        for (int x = 0; x < ROWS; ++x)
#pragma unroll
            for (int y = 0; y < COLS / 2; ++y)
#pragma unroll
                for (int p = 0; p < 8; p += kChunk) {
                    Raw v[kChunk];
#pragma unroll
                    for (int e = 0; e < kChunk; ++e) v[e] = Score<TYPE>::put(value(x, y, p + e));
                    take(x, i, y * 32 + 8 * g + p, WideChunk::pack(v));
                }
    }
}

// The numbers of a chunk of which a row has `left` more, at any multiple of their element; whole: it has all or none, at a multiple of the chunk
template <int TYPE, int COUNT>
__device__ __forceinline__ void store_run(void *p, const typename Score<TYPE>::Raw *v, int64_t left, bool whole)
{
    using Raw = typename Score<TYPE>::Raw;
    if (whole) {
        if (left > 0) __builtin_memcpy(__builtin_assume_aligned(p, COUNT * sizeof(Raw)), v, COUNT * sizeof(Raw));
    } else if (left >= COUNT) {
        typedef uint32_t Any __attribute__((ext_vector_type(COUNT * sizeof(Raw) / 4), aligned(alignof(uint16_t))));
        __builtin_memcpy(static_cast<Any *>(p), v, sizeof(Any));
    } else {
#pragma unroll
        for (int c = 0; c < COUNT - 1; ++c)
            if (c < left) static_cast<Raw *>(p)[c] = v[c];
    }
}

template <int TYPE, int COUNT>
__device__ __forceinline__ void load_run(float *v, const void *p, int64_t left, bool whole)
{
    using Raw = typename Score<TYPE>::Raw;
    Raw part[COUNT];
    if (whole) {
        __builtin_memcpy(part, __builtin_assume_aligned(p, COUNT * sizeof(Raw)), COUNT * sizeof(Raw));
    } else if (left >= COUNT) {
        __builtin_memcpy(part, p, COUNT * sizeof(Raw));
    } else {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) part[c] = c < left ? static_cast<const Raw *>(p)[c] : Raw(0.f);
    }
#pragma unroll
    for (int c = 0; c < COUNT; ++c) v[c] = Score<TYPE>::get(part[c]);
}

// A tile of BM rows and BN columns, WM x WN waves.  Columns come first in the matrix instruction, so that a lane's four results are neighbours
// in a row.  Rows: of X (product), or columns of dY (weight gradient, summed over rows).  Columns: rows of W (of its columns where ACROSS;
// with the gate half of them are g's and half u's), or columns of X.
//
// 16 bits, DIRECT: what bounds it is the way of the numbers into LDS and the writing of the results.  8192 x 8192 x 8192 bf16 in a copy that leaves parts out, 256 x 256: 1064
// TFLOP/s; every load from the same place 1230, no loads 1430, products alone 1573 (a library product on this card 1190 to 1317); 192 x 128 (two workgroups to a
// unit) 1107, 128 x 128 843.  192 x 128 was no faster on runs of some hundred rows (32768 rows of 60 experts 355 and 353 us).  Measured here: 131072 rows, 64 experts,
// 1024 x 2048: product 591 us = 930 TFLOP/s (writing the 0.54 GB of results is 100 of them), weight gradient of gathered rows
// to fp32 637 us = 863, of rows as they are to bf16 537 = 1024.
// The sums have to be where the loop has them in one block: with an exit in its middle the compiler copies all of them (256 registers) each time round.
template <int TYPE, int BM, int BN, int WM, int WN, bool ACROSS, int KIND, bool DIRECT, int OUT, bool GATHER>
__device__ __forceinline__ void expert_tile(const GroupArgs &A, const Run &run, uint32_t b, char *lds)
{
    constexpr int kThreadsHere = WM * WN * kLanes;
    constexpr bool kAcrossRows = KIND == kWeightGrad;
    using Rows = Side<TYPE, BM, kAcrossRows, kThreadsHere>;
    using Cols = Side<TYPE, BN, ACROSS, kThreadsHere>;
    using Raw = typename Score<TYPE>::Raw;
    constexpr int kElem = sizeof(Raw), kSum = Rows::kSum;
    constexpr int kFragRows = BM / WM / 16, kFragCols = BN / WN / 16;
    static_assert(kFragCols % 2 == 0 && (kAcrossRows || kFragRows % 2 == 0), "fragments come in pairs");
    // two stretches of the sum: the rows' numbers, and the columns' behind them
    constexpr int kStretch = Rows::kBytes + Cols::kBytes;
    Loader<TYPE, BM, kAcrossRows, kThreadsHere, DIRECT, false, false> rows;
    Loader<TYPE, BN, ACROSS, kThreadsHere, DIRECT, KIND == kWeightGrad && GATHER, KIND == kGate> cols;
    int64_t first_row, row_end, first_col, col_end, sum, from = 0;
    int expert, part = 0;
    if constexpr (KIND == kWeightGrad) {
        const uint32_t per = A.row_tiles * A.col_tiles, tile = b % per;
        expert = b / per % A.experts;
        part = b / per / A.experts;
        first_row = (int64_t)(tile / A.col_tiles) * BM;
        first_col = (int64_t)(tile % A.col_tiles) * BN;
        row_end = A.m;
        col_end = A.d;
        const int64_t s = run_start(A, expert), count = max(run_start(A, expert + 1) - s, (int64_t)0);
        const int64_t each = ((count + kSum - 1) / kSum + A.splits - 1) / A.splits * kSum;
        from = s + min(part * each, count);
        sum = min(each, count - min(part * each, count));
    } else {
        expert = run.expert;
        first_row = run.first;
        row_end = run.end;
        first_col = (int64_t)(b % A.col_tiles) * (KIND == kGate ? BN / 2 : BN);
        col_end = A.m;
        sum = A.d;
    }
    const auto begin = [&] {
        if constexpr (KIND == kWeightGrad) {
            rows.across(static_cast<const char *>(A.W) + from * A.ldW * kElem, A.ldW, first_row, row_end);
            cols.across(static_cast<const char *>(A.X) + (GATHER ? 0 : from * A.ldX * kElem), A.ldX, first_col, col_end);
            if constexpr (GATHER)
                if (sum > 0) cols.gather(A, from, from + sum);
        } else {
            const char *W = static_cast<const char *>(A.W) + expert * A.strideW * kElem;
            rows.rows([&](int i) { return static_cast<const char *>(A.X) + source_row(A, min(first_row + i, row_end - 1)) * A.ldX * kElem; });
            if constexpr (ACROSS) {
                cols.across(W, A.ldW, first_col, col_end);
            } else {
                cols.rows([&](int i) {
                    const int64_t c = KIND == kGate ? min(first_col + i % (BN / 2), col_end - 1) + (i >= BN / 2 ? col_end : 0) : min(first_col + i, col_end - 1);
                    return W + c * A.ldW * kElem;
                });
            }
        }
    };

    const int wave = threadIdx.x / kLanes;
    const int wm = wave / WN, wn = wave % WN;
    // with the gate a wave's columns are kFragCols / 2 fragments of g and as many of u
    const auto col_fragment = [&](const char *lds, int f, int step) {
        if constexpr (KIND == kGate) {
            constexpr int kHalf = kFragCols / 2;
            return Cols::fragment(lds, (f < kHalf ? 0 : BN / 32) + wn * kHalf, f % kHalf, step);
        } else {
            return Cols::fragment(lds, wn * kFragCols, f, step);
        }
    };
    constexpr bool kHere = DIRECT && TYPE != REGOT_F32;
    f32x4 acc[kFragRows][kFragCols];
    const auto clear = [&] {
#pragma unroll
        for (int xy = 0; xy < kFragRows * kFragCols; ++xy) {
            if constexpr (kHere) clear_here(acc[xy / kFragCols][xy % kFragCols]);
            else acc[xy / kFragCols][xy % kFragCols] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    struct Fragments {
        u32x4 rows[kFragRows], cols[kFragCols];
    };
    constexpr int kFragments = kFragRows + kFragCols, kAtOnce = kFragRows * kFragCols / kFragments;
    const auto read_one = [&](Fragments &F, const char *from, int step, int f) {
        if (f < kFragCols) F.cols[f] = col_fragment(from + Rows::kBytes, f, step);
        else F.rows[f - kFragCols] = Rows::fragment(from, wm * kFragRows, f - kFragCols, step);
    };
    const auto read = [&](Fragments &F, const char *from, int step) {
#pragma unroll
        for (int f = 0; f < kFragments; ++f) read_one(F, from, step, f);
    };
    const auto add_some = [&](const Fragments &F, int first, int last) {
#pragma unroll
        for (int xy = first; xy < last; ++xy) {
            const int x = xy / kFragCols, y = xy % kFragCols;
            if constexpr (kHere) multiply_here<TYPE>(F.cols[y], F.rows[x], acc[x][y]);
            else acc[x][y] = multiply<TYPE>(F.cols[y], F.rows[x], acc[x][y]);
        }
    };
    const auto add = [&](const Fragments &F) { add_some(F, 0, kFragRows * kFragCols); };
    if constexpr (kHere) {
        begin();
        clear();
        // Two stretches of the sum are in LDS or on their way.  While a step's fragments are multiplied, the next step's are read; when the last of a stretch have
        // been read (by all waves: the barrier), its place is filled with the stretch after the next.
        constexpr int kLoads = decltype(rows)::S::kLoads + decltype(cols)::S::kLoads, kRowLoads = decltype(rows)::S::kLoads;
        const int stretches = (int)((sum + kSum - 1) / kSum);
        const uint32_t lds_at = lds_address(lds);
        const auto load_one = [&](int ii, uint32_t to, bool more) {
            if (ii < kRowLoads) rows.load(ii, to, more ? rows.step : 0);
            else cols.load(ii - kRowLoads, to + Rows::kBytes, more ? cols.step : 0);
        };
        const auto all_there = [&] {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (this wave's loads into LDS)
            __syncthreads();
            if constexpr (KIND == kWeightGrad && GATHER) cols.gathered();
        };
        if (stretches > 0) {
            int64_t done = sum - (int64_t)(stretches - 1) * kSum;
            const auto next_rows = [&] {
                if constexpr (KIND == kWeightGrad && GATHER) cols.gather(A, from + done, from + sum);
            };
            Fragments even, odd;
            rows.first(lds_at, (int)done);
            cols.first(lds_at + Rows::kBytes, (int)done);
            next_rows();
            all_there();
            if (stretches > 1) {
#pragma unroll
                for (int ii = 0; ii < kLoads; ++ii) load_one(ii, lds_at + kStretch, stretches > 2);
                done += stretches > 2 ? kSum : 0;
                next_rows();
            }
            read(even, lds, 0);
            uint32_t here = 0;
            // kAtOnce products for each fragment that is read, so that neither waits for the other
            const auto first_half = [&] {
#pragma unroll
                for (int f = 0; f < kFragments; ++f) {
                    read_one(odd, lds + here, 1, f);
                    add_some(even, f * kAtOnce, f + 1 < kFragments ? (f + 1) * kAtOnce : kFragRows * kFragCols);
                }
            };
            for (int t = 1; t < stretches; ++t) {
                first_half();
                all_there();
                const bool more = t + 2 < stretches;  // (where there is no stretch after the next, the next one is loaded once more, for nobody)
                constexpr int kEach = (kLoads + kFragments - 1) / kFragments;
#pragma unroll
                for (int f = 0; f < kFragments; ++f) {
#pragma unroll
                    for (int ii = f * kEach; ii < min((f + 1) * kEach, kLoads); ++ii) load_one(ii, lds_at + here, more);
                    read_one(even, lds + (here ^ kStretch), 0, f);
                    add_some(odd, f * kAtOnce, f + 1 < kFragments ? (f + 1) * kAtOnce : kFragRows * kFragCols);
                }
                done += more ? kSum : 0;
                next_rows();
                here ^= kStretch;
            }
            first_half();
            add(odd);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing is on its way into LDS when the workgroup ends)
        }
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int x = 0; x < kFragRows; ++x) multiplied(acc[x]);
    } else {
        // Numbers of 32 bits are multiplied in pieces.  A tile whose sums are not all finite is summed once more as the numbers are, and gives its results in the place of
        // those that are not, so that infinities and NaNs are those of the numbers (and those from 2^80 on, which the scale takes beyond 32 bits, are right too).  us, pieces /
        // numbers as they are: 8192 rows of 60 experts, 2048 by 2 x 1024 with the gate 591 / 775, gradients of 2048 x 1024 608 / 840, of 777 x 555 with 2997 rows of 12 115 / 134.  The
        // splitting (430 vector instructions for 96 products) bounds it; 64 of them are the scale's (without it, and with what it keeps lost: 568, 584, 110).
        const auto stretch = [&](const char *at, bool pieces) {
            if constexpr (TYPE == REGOT_F32) {
                if (pieces) {
                    const auto of_col = [&](int f) { return Pieces(col_fragment(at + Rows::kBytes, f, 0), col_fragment(at + Rows::kBytes, f, 1)); };
                    const auto of_row = [&](int f) { return Pieces(Rows::fragment(at, wm * kFragRows, f, 0), Rows::fragment(at, wm * kFragRows, f, 1)); };
                    if constexpr (kFragCols == 4) {
                        const Pieces c[4] = {of_col(0), of_col(1), of_col(2), of_col(3)};
#pragma unroll
                        for (int x = 0; x < kFragRows; ++x) multiply_pieces(c, of_row(x), acc[x]);
                    }
                    return;
                }
            }
            Fragments F;
            read(F, at, 0);
            add(F);
            read(F, at, 1);
            add(F);
        };
        const auto pass = [&](bool pieces) {
            begin();
            clear();
            if constexpr (DIRECT) {
                const int stretches = (int)((sum + kSum - 1) / kSum);
                const uint32_t lds_at = lds_address(lds);
                if (stretches > 0) {
                    int64_t done = sum - (int64_t)(stretches - 1) * kSum;
                    const auto next_rows = [&] {
                        if constexpr (KIND == kWeightGrad && GATHER) cols.gather(A, from + done, from + sum);
                    };
                    rows.first(lds_at, (int)done);
                    cols.first(lds_at + Rows::kBytes, (int)done);
                    next_rows();
                    uint32_t here = 0;
                    for (int t = 1; t <= stretches; ++t) {
                        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (this wave's loads into LDS)
                        __syncthreads();
                        if (t < stretches) {
                            if constexpr (KIND == kWeightGrad && GATHER) cols.gathered();
                            const uint32_t to = lds_at + (here ^ kStretch);
#pragma unroll
                            for (int ii = 0; ii < decltype(rows)::S::kLoads; ++ii) rows.load(ii, to, rows.step);
#pragma unroll
                            for (int ii = 0; ii < decltype(cols)::S::kLoads; ++ii) cols.load(ii, to + Rows::kBytes, cols.step);
                            done += kSum;
                            next_rows();
                        }
                        stretch(lds + here, pieces);
                        here ^= kStretch;
                    }
                }
            } else if (sum > 0) {
                int64_t done = 0;  // of the sum: what has been asked for
                const auto load = [&] {
                    rows.fetch(done, sum, first_row, row_end);
                    cols.fetch(done, sum, first_col, col_end);
                    done += kSum;
                    if constexpr (KIND == kWeightGrad && GATHER)
                        if (done < sum) cols.gather(A, from + done, from + sum);
                };
                const auto put = [&](char *to) {
                    rows.put(to);
                    cols.put(to + Rows::kBytes);
                };
                load();
                put(lds);
                for (uint32_t here = 0;; here ^= kStretch) {
                    __syncthreads();
                    const bool more = done < sum;
                    if (more) load();
                    stretch(lds + here, pieces);
                    if (!more) break;
                    put(lds + (here ^ kStretch));
                }
            }
        };
        pass(TYPE == REGOT_F32);
        if constexpr (TYPE == REGOT_F32) {
            const auto finite = [](const f32x4 &v) { return fabsf(v[0]) < kInf && fabsf(v[1]) < kInf && fabsf(v[2]) < kInf && fabsf(v[3]) < kInf; };
            bool all_finite = true;
#pragma unroll
            for (int xy = 0; xy < kFragRows * kFragCols; ++xy) all_finite &= finite(acc[xy / kFragCols][xy % kFragCols]);
            const bool again = !__syncthreads_and(all_finite);
#pragma unroll
            for (int xy = 0; xy < kFragRows * kFragCols; ++xy) acc[xy / kFragCols][xy % kFragCols] *= Pieces::kUnscale;
            if (__builtin_expect(again, 0)) {
                f32x4 first[kFragRows][kFragCols];
                __builtin_memcpy(first, acc, sizeof(acc));
                pass(false);
#pragma unroll
                for (int xy = 0; xy < kFragRows * kFragCols; ++xy)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (fabsf(first[xy / kFragCols][xy % kFragCols][e]) < kInf) acc[xy / kFragCols][xy % kFragCols][e] = first[xy / kFragCols][xy % kFragCols][e];
            }
        }
    }

    // results: a run y of 8 neighbours is that of fragments 2 y and 2 y + 1, one of 4 (ACROSS) that of fragment y
    __syncthreads();
    constexpr int kOutElem = sizeof(typename Score<OUT>::Raw), kMine = 2 * kStretch / (WM * WN);
    char *const mine = lds + wave * kMine;
    const auto row_of = [&](int x, int i) {
        return first_row + (wm * kFragRows + (kAcrossRows ? x : x / 2 * 2)) * 16 + (kAcrossRows ? i : 8 * (i / 4) + 4 * (x % 2) + i % 4);
    };
    const auto result = [&](int x, int y, int e) { return acc[x][ACROSS ? y : 2 * y + e / 4][e % 4]; };
    if constexpr (KIND == kGate) {
        constexpr int kHalf = kFragCols / 2;
        static_assert(KIND != kGate || kHalf % 2 == 0, "halves are pairs of fragments");
        constexpr int kUp = ACROSS ? kHalf : kHalf / 2;  // runs of g
        const auto store = [&](char *to, int64_t ld) {
            return [=, &A](int x, int i, int c, u32x4 v) {
                const int64_t r = row_of(x, i), col = first_col + wn * kHalf * 16 + c;
                Raw part[16 / kElem];
                __builtin_memcpy(part, &v, 16);
                if (r < row_end) store_run<TYPE, 16 / kElem>(to + (r * ld + col) * kElem, part, col_end - col, A.whole);
            };
        };
        results<TYPE, kFragRows, kHalf, ACROSS, kMine>(mine, [&](int x, int y, int e) {
            const float gate = result(x, y, e);
            return gate * sigmoid<TYPE>(gate) * result(x, kUp + y, e);
        }, store(static_cast<char *>(A.Y), A.ldY));
        if (A.saved) {
            results<TYPE, kFragRows, kHalf, ACROSS, kMine>(mine, result, store(static_cast<char *>(A.saved), A.ldSaved));
            results<TYPE, kFragRows, kHalf, ACROSS, kMine>(mine, [&](int x, int y, int e) { return result(x, kUp + y, e); },
                                                               store(static_cast<char *>(A.saved) + col_end * kElem, A.ldSaved));
        }
    } else if constexpr (KIND == kGateGrad) {
        struct Gate {
            float g[4], u[4];
        };
        const auto saved_at = [&](int64_t r, int64_t col) { return static_cast<const char *>(A.saved) + (r * A.ldSaved + col) * kElem; };
        const auto column = [&](int c) { return first_col + wn * kFragCols * 16 + c; };
        const auto take = [&](int x, int i, int c, u32x4 v, const Gate &of) {
            const int64_t r = row_of(x, i), col = column(c), left = col_end - col;
            if (r >= row_end || left <= 0) return;
            Raw dg[4], du[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = sigmoid<TYPE>(of.g[e]), D = __uint_as_float(v[e]);
                dg[e] = Score<TYPE>::put(D * of.u[e] * (p * (1.0f + of.g[e] * (1.0f - p))));
                du[e] = Score<TYPE>::put(D * (of.g[e] * p));
            }
            char *to = static_cast<char *>(A.Y) + (r * A.ldY + col) * kElem;
            store_run<TYPE, 4>(to, dg, left, A.whole);
            store_run<TYPE, 4>(to + col_end * kElem, du, left, A.whole);
        };
        if (A.whole) {  // (the place of what is beyond the matrix is one inside, so that nothing stands between the loads)
            through_lds<REGOT_F32, kFragRows, kFragCols, ACROSS, kMine>(mine, result, [&](int x, int i, int c) {
                const char *s = saved_at(min(row_of(x, i), row_end - 1), min(column(c), col_end - 4));
                Gate of;
                load_run<TYPE, 4>(of.g, s, 4, true);
                load_run<TYPE, 4>(of.u, s + col_end * kElem, 4, true);
                return of;
            }, take);
        } else {
            through_lds<REGOT_F32, kFragRows, kFragCols, ACROSS, kMine>(mine, result, [](int, int, int) { return 0; }, [&](int x, int i, int c, u32x4 v, int) {
                const int64_t r = row_of(x, i), col = column(c), left = col_end - col;
                if (r >= row_end || left <= 0) return;
                Gate of;
                load_run<TYPE, 4>(of.g, saved_at(r, col), left, false);
                load_run<TYPE, 4>(of.u, saved_at(r, col + col_end), left, false);
                take(x, i, c, v, of);
            });
        }
    } else {
        char *Y = static_cast<char *>(A.Y);
        if constexpr (KIND == kWeightGrad) Y += ((int64_t)part * A.experts + expert) * A.strideY * kOutElem;
        results<OUT, kFragRows, kFragCols, ACROSS, kMine>(mine, result, [&](int x, int i, int c, u32x4 v) {
            const int64_t r = row_of(x, i), col = first_col + wn * kFragCols * 16 + c;
            typename Score<OUT>::Raw of[16 / kOutElem];
            __builtin_memcpy(of, &v, 16);
            if (KIND == kWeightGrad && A.whole) {
                // nothing reads them soon: they go past the caches, which keep what other tiles read too (256 rows of each of 60 experts, 2048 x 2048 bf16 265 us, and so 200;
                // 4 of each 142 and 123; 512 of 8, 14336 x 4096 868 and 722.  A product's results are read next: a layer's way forward is 208 us, and would be 228)
                if (r < row_end && col < col_end) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(Y + (r * A.ldY + col) * kOutElem));
                return;
            }
            if (r < row_end) store_run<OUT, 16 / kOutElem>(Y + (r * A.ldY + col) * kOutElem, of, col_end - col, A.whole);
        });
    }
}

// A workgroup: one tile.  A run's last tile that has half of its rows or less is one of half the height.
template <int TYPE, int BM, int BN, int WM, int WN, bool ACROSS, int KIND, bool DIRECT, int OUT, bool GATHER>
__global__ void __launch_bounds__(WM *WN *kLanes, BM + BN <= 320 ? 2 : 1) expert_tile_kernel(const GroupArgs A)
{
    __shared__ __attribute__((aligned(1024))) char lds[2 * 128 * (BM + BN)];
    const uint32_t b = die_order(blockIdx.x, A.tiles);
    if constexpr (KIND == kWeightGrad) {
        expert_tile<TYPE, BM, BN, WM, WN, ACROSS, KIND, DIRECT, OUT, GATHER>(A, Run{}, b, lds);
    } else {
        const Run run = find_run<BM>(A, b / A.col_tiles);
        if (run.first >= run.end) return;
        if constexpr (BM / WM % 64 == 0) {
            if (run.end - run.first <= BM / 2) {
                expert_tile<TYPE, BM / 2, BN, WM, WN, ACROSS, KIND, DIRECT, OUT, GATHER>(A, run, b, lds);
                return;
            }
        }
        expert_tile<TYPE, BM, BN, WM, WN, ACROSS, KIND, DIRECT, OUT, GATHER>(A, run, b, lds);
    }
}

}  // namespace regot
