// Attention over packed sequences and over a paged cache: arguments of the
// kernels, and the device code they share.
//
// Rows. The heads of a group share their keys, so a work item is a range of
// the rows (token, head of the group) of one sequence and one key head: row
// r is token r / group, head r % group. A tile of rows then spans few tokens,
// which keeps causal tiles narrow, reads every key once per group, and fills
// a matrix instruction from a single token of many heads.
//
// Tiles of 16-bit rows lie in LDS row by row, quads (16 bytes) permuted by
// quad ^ swizzle(row) since neither padded rows nor another order can be had
// from loads that write LDS directly. Two kinds of reads have to be spread over
// the 64 banks: 16-byte reads of one quad of 16 consecutive rows (their places
// within 256 bytes differ: 1 KB in four cycles), and the transposing reads,
// where 32 lanes read four rows x 64 contiguous bytes (the four take different
// quarters of 256 bytes; with places that differ within 128 bytes only, a read
// took four cycles instead of two).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_index.h"
#include "ep_device.h"
#include "split.h"

namespace ep {

struct Rows {                 // element (t, h, c) at p[t row + h head + c]
    char* p;                  // 16-bit elements; strides in bytes
    int64_t row, head;
};

struct AttnArgs {
    Rows q, k, v, o;          // o: out; the gradients' kernels use the rest
    Rows dout, dq, dk, dv;
    float* lse;               // [tokens_q][heads], may be NULL where written
    float* lse2;              // [tokens_q][heads], for the gradients: log-sums in units of
    float* delta;             //   log 2, and the sums of out * dout
    const int* start_q;       // batch + 1
    const int* start_k;       // batch + 1 (packed keys)
    int64_t tokens_q, tokens_k;
    int batch, heads, kv_heads, group;
    unsigned group_magic;     // (attn_index.h)
    int dim;
    float scale, scale_log2;  // scale, scale * log2(e)
    int causal;
    int window;               // 0: none
    // paged keys (k.p, v.p: the pages; e4m3 pages: one byte an element)
    const int* table;
    int64_t cols;
    const int* lengths;
    int pages, page_shift;
    const float* k_scale;
    const float* v_scale;
    int* err;                 // may be NULL
    // keys cut into `splits` ranges: normalised partial outputs
    // [splits][tokens_q][heads][dim] and their log-sums, in units of log 2
    int splits;
    float* part;
    float* part_lse;
    // gradients: the rows that a range of keys meets cut into row_splits
    // ranges; partial sums [row_splits][dv, dk][tokens_k][kv_heads][dim]
    int row_splits;
    float* part_kv;
    // and the keys that a tile of rows meets, into key_splits ranges; partial
    // sums [key_splits][tokens_q][heads][dim]
    int key_splits;
    float* part_q;
};

// How a forward pass runs: rows of a tile (32: the four waves of a workgroup
// share the rows and split the keys; 128: 32 rows each), and cuts of the keys.
struct AttnPlan {
    int tile;
    int splits;
    int64_t bytes;            // of partial results
};
int attn_key_splits(int64_t batch, int64_t tokens_q, int64_t tokens_k, int64_t heads, int64_t kv_heads);
int attn_row_splits(int64_t batch, int64_t tokens_q, int64_t tokens_k, int64_t heads, int64_t kv_heads);
AttnPlan attn_plan(int64_t batch, int64_t tokens_q, int64_t heads, int64_t kv_heads, int64_t dim,
                   int64_t most_keys);

// Workgroups of a launch over tiles of `size` rows.
inline int64_t attn_groups(int64_t kv_heads, int64_t rows, int64_t size, int64_t batch) {
    return kv_heads * (rows / size + batch);
}
constexpr int kRowTile = 128;         // rows of a workgroup: 32 per wave
constexpr int kFewRows = 32;          // rows of a workgroup whose waves split the keys
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;   // of 256 threads: below 2^32

// Where keys lie: packed rows; pages of 16-bit rows, of at least 16 tokens or
// fewer; pages of e4m3 rows, the same.
enum { kPacked = 0, kPaged = 1, kPagedSmall = 2, kE4m3 = 3, kE4m3Small = 4 };

hipError_t attn_forward_launch(const AttnArgs& a, const AttnPlan& p, bool bf, int source,
                               hipStream_t s);
hipError_t attn_backward_launch(const AttnArgs& a, bool bf, hipStream_t s);

struct CacheArgs {
    Rows k, v;                // rows written from or read into
    char* kp;                 // pages: [page][slot][head][dim]
    char* vp;
    float* ks;                // scales [page][slot][head] (e4m3)
    float* vs;
    const int* table;
    int64_t cols;
    const int* lengths;
    const int* start;
    int64_t tokens;
    int batch, kv_heads, dim, pages, page_shift;
    int* err;
};
hipError_t cache_write_launch(const CacheArgs& a, bool bf, bool e4m3, hipStream_t s);
hipError_t cache_read_launch(const CacheArgs& a, bool bf, bool e4m3, hipStream_t s);

// ---- device code ----

// Workgroups are numbered key head first: those of one head are 8 apart where
// kv_heads is a multiple of 8, and so run on one XCD (workgroups go to the 8
// XCDs round robin), whose L2 then holds few heads' keys. tiles: of the launch.
__device__ __forceinline__ void head_and_tile(int kv_heads, int& head, int& tile, int& tiles) {
    head = blockIdx.x % kv_heads;
    tile = blockIdx.x / kv_heads;
    tiles = gridDim.x / kv_heads;
}
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

template <bool BF>
__device__ __forceinline__ floatx16 mfma16(uintx4 a, uintx4 b, floatx16 c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a),
                                                      __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

// Two floats rounded to nearest, the first in the low half.
template <bool BF>
__device__ __forceinline__ unsigned pack16(float a, float b) {
    if constexpr (BF) return pack_bf16(a, b);
    const floatx2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, half2v));
}
template <bool BF>
__device__ __forceinline__ float lo16(unsigned u) {
    if constexpr (BF) return bf16_lo(u);
    return (float)__builtin_bit_cast(half2v, u)[0];
}
template <bool BF>
__device__ __forceinline__ float hi16(unsigned u) {
    if constexpr (BF) return bf16_hi(u);
    return (float)__builtin_bit_cast(half2v, u)[1];
}

// The values of the two lanes (l % 32, l % 32 + 32) that share a row. (The
// elements are copied before the cast: __builtin_bit_cast of a vector's
// element takes the first one.)
__device__ __forceinline__ void pair_of(float x, float& a, float& b) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned lo = r[0], hi = r[1];
    a = __builtin_bit_cast(float, lo);
    b = __builtin_bit_cast(float, hi);
}
__device__ __forceinline__ float pair_sum(float x) {
    float a, b;
    pair_of(x, a, b);
    return a + b;
}
__device__ __forceinline__ float pair_max(float x) {
    float a, b;
    pair_of(x, a, b);
    return fmaxf(a, b);
}

// Quads a row of a tile for products of depth dp (64, 96 or 128). Rows of 96
// take the places of 128, whose last quarter is loaded twice and not read.
constexpr int tile_quads(int dp) { return dp > 64 ? 16 : 8; }

template <int QUADS>                  // quads a row (16 or 8)
__device__ __forceinline__ int swizzle(int row) {
    if constexpr (QUADS == 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    return ((row & 2) << 1) | ((row >> 2) & 3);      // (two rows to 256 bytes)
}

__device__ __forceinline__ void load_lds16(const char* p, uintx4* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) unsigned*)p,
                                     (__attribute__((address_space(3))) unsigned*)lds, 16, 0, 0);
}
__device__ __forceinline__ void load_lds4(const float* p, float* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) unsigned*)p,
                                     (__attribute__((address_space(3))) unsigned*)lds, 4, 0, 0);
}

// A wave's part of a tile that is loaded straight into LDS: ROWS rows from
// row ROWS * wave on, one kilobyte a load. A lane's offset from the first of
// them stays the same from tile to tile, so a load costs a scalar base.
template <int QUADS, int ROWS>
struct TileLoader {
    static constexpr int kLoads = ROWS * QUADS / 64;
    static constexpr int kStep = 64 / QUADS;         // rows a load
    int row0;                         // of the first load, within the wave's rows
    int quad_[kLoads];                // bytes into a row

    __device__ __forceinline__ TileLoader(int lane, int wave, int dim) {
        row0 = lane / QUADS;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            quad_[i] = 16 * min((lane % QUADS) ^ swizzle<QUADS>(ROWS * wave + row(i)), dim / 8 - 1);
    }
    __device__ __forceinline__ int row(int i) const { return row0 + kStep * i; }
    __device__ __forceinline__ int quad(int i) const { return quad_[i]; }
    // base: the wave's first row; left: rows that exist from there on (>= 1;
    // the others read the last); stride: bytes a row, below 2^25; to: the
    // wave's part of the tile.
    __device__ __forceinline__ void load(const char* base, int left, int64_t stride, uintx4* to) const {
        const unsigned st = (unsigned)stride;
        if (left >= ROWS) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load_lds16(base + (row(i) * st + quad_[i]), to + 64 * i);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                load_lds16(base + (min(row(i), left - 1) * st + quad_[i]), to + 64 * i);
        }
    }
};

// Operands from a tile. rows(): 32 rows x 16 depth, lane l holding row l % 32
// from row0 on (a multiple of 32), depth 16 step + 8 (l / 32) .. + 7.
// columns(): 32 columns (from column 32 block on) x 16 rows (from row0 on, a
// multiple of 16), transposed: lane l holds column l % 32 and rows 4 h .. 4 h + 3,
// 8 + 4 h .. 8 + 4 h + 3 (h = l / 32) of the sixteen: the order in which a
// lane's accumulators 8 i .. 8 i + 7 hold the rows of a 32 x 32 product. A
// transposing read gives lane i of 16 column i of the four rows that lanes
// 0..3, 4..7, 8..11, 12..15 address.
//
// Both are an exclusive or of a lane's one offset and a constant, plus
// constants that fit the instruction. fresh(), once a tile, keeps the compiler
// from holding all these sums in registers over the loop (50 of them, spilled,
// in the gradients' kernels).
template <int QUADS>
struct TileReader {
    unsigned r, c;
    __device__ __forceinline__ explicit TileReader(int lane) {
        const int row = lane & 31;
        r = (row * QUADS + ((lane >> 5) ^ swizzle<QUADS>(row))) * 16;
        const int i = lane & 15, g = lane >> 4;
        const int k = 4 * (g >> 1) + (i >> 2);
        c = (k * QUADS + ((2 * (g & 1) + ((i & 3) >> 1)) ^ swizzle<QUADS>(k))) * 16 + (i & 1) * 8;
    }
    __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(r), "+v"(c)); }
    __device__ __forceinline__ uintx4 rows(const uintx4* tile, int row0, int step) const {
        const char* t = reinterpret_cast<const char*>(tile) + row0 * QUADS * 16;
        return *reinterpret_cast<const uintx4*>(t + (r ^ (32 * step)));
    }
    __device__ __forceinline__ uintx4 columns(const uintx4* tile, int row0, int block) const {
        // (eight rows on, the swizzle differs in bit 1)
        const char* t = reinterpret_cast<const char*>(tile) + row0 * QUADS * 16;
        const char* a = t + (c ^ (64 * block));
        const char* b = t + 8 * QUADS * 16 + (c ^ (64 * block) ^ 32);
        const shortx4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)a);
        const shortx4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)b);
        typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
        const uintx2 u = __builtin_bit_cast(uintx2, x), w = __builtin_bit_cast(uintx2, y);
        return uintx4{u[0], u[1], w[0], w[1]};
    }
};

// Part `split` of the range begin .. end, whole tiles of `size`, cut into
// `splits` parts.
__device__ __forceinline__ void split_range(int split, int splits, int size, int& begin, int& end) {
    const int tiles = (end - begin + size - 1) / size;
    const int per = (tiles + splits - 1) / splits;
    const int from = begin + min(split * per, tiles) * size;
    end = min(end, begin + min((split + 1) * per, tiles) * size);
    begin = from;
}

// One sequence as a workgroup sees it.
struct Seq {
    int b;
    int q0, n;                // first packed query row (token) and their number
    int k0, m;                // first packed key row (packed keys) and their number
    int tile;                 // of its tiles
    int rows;                 // n * group
    int off;                  // position of query 0: m - n
};

// The sequence and tile (of `size` of its queries' rows, or of its keys) that
// is the u-th of `tiles` to start. Longest first: of a causal sequence its
// last rows (first keys) before the others, and up to 64 sequences of
// different lengths by their length, so that what starts last ends soon
// (chunks of four sequences over the cache 415 us in the order of the batch,
// 371 like this; 64 single tokens 446 and 419; 24 ragged sequences 84 and 81).
// With a window tiles cost alike whatever their sequence's length, and the
// search costs more than the order gains (gradients of 12 sequences, window
// 512: 177 us in the order of the batch, 187 longest first). Starts and
// lengths of 64 sequences are fetched at once, those of the one that is found
// taken from its lane: a call of a single token waits for few loads one after
// another. More sequences are searched 64 at a time, and not ordered.
// Whatever the starts hold, the ranges lie within their arrays; s.tile may come
// out negative or past the sequence's tiles, which the caller leaves out.
template <int SOURCE, bool KEYS = false>
__device__ __forceinline__ Seq find_seq(const AttnArgs& a, int size, int u, int tiles) {
    const int lane = threadIdx.x & 63;
    const int per = KEYS ? 1 : a.group;
    const int* start = KEYS ? a.start_k : a.start_q;
    const int tokens = (int)(KEYS ? a.tokens_k : a.tokens_q);
    const int t = KEYS ? u : tiles - 1 - u;
    int low = 0, left = a.batch;                     // the sequence is one of these
    while (left > 64) {
        const int stride = (left + 63) / 64;
        const int b = low + lane * stride;
        const bool below = lane * stride < left &&
                           first_tile(start[min(b, a.batch - 1)], tokens, b, per, size) <= t;
        const int skip = max(__builtin_popcountll(__ballot(below)) - 1, 0) * stride;
        low += skip;
        left = min(stride, left - skip);
    }
    const int b = min(low + lane, a.batch - 1);
    int q0, n, k0, m;
    held_range(a.start_q[b], a.start_q[b + 1], (int)a.tokens_q, q0, n);
    if constexpr (SOURCE == kPacked) {
        held_range(a.start_k[b], a.start_k[b + 1], (int)a.tokens_k, k0, m);
    } else {
        const int length = a.lengths[b];
        k0 = 0;
        m = held_length(length, a.cols, a.page_shift);
        if (m != length && a.err) *a.err = 1;
    }
    Seq s;
    int at;
    const int cost = KEYS ? n : m;                   // of a tile
    if (a.batch <= 64 && !a.window && !__all(cost == __builtin_amdgcn_readfirstlane(cost))) {
        const int own = lane >= a.batch ? 0 : KEYS ? (m + size - 1) / size : (n * per + size - 1) / size;
        int before = 0;                              // tiles of longer sequences
        for (int i = 0; i < a.batch; ++i) {
            const int other = __builtin_amdgcn_readlane(cost, i);
            if (other > cost || (other == cost && i < lane)) before += __builtin_amdgcn_readlane(own, i);
        }
        const uint64_t mine = __ballot(u >= before && u < before + own);
        at = mine ? __builtin_ctzll(mine) : 0;
        const int within = u - __builtin_amdgcn_readlane(before, at);
        s.tile = !mine ? -1 : KEYS ? within : __builtin_amdgcn_readlane(own, at) - 1 - within;
    } else {
        const int begin = (int)first_tile(start[b], tokens, b, per, size);
        at = max(__builtin_popcountll(__ballot(lane < left && begin <= t)) - 1, 0);
        s.tile = t - __builtin_amdgcn_readlane(begin, at);
    }
    s.b = low + at;
    s.q0 = __builtin_amdgcn_readlane(q0, at);
    s.n = __builtin_amdgcn_readlane(n, at);
    s.k0 = __builtin_amdgcn_readlane(k0, at);
    s.m = __builtin_amdgcn_readlane(m, at);
    s.rows = s.n * a.group;
    s.off = s.m - s.n;
    return s;
}

__device__ __forceinline__ int row_token(const AttnArgs& a, int r) {
    return row_token(r, a.group, a.group_magic);
}
__device__ __forceinline__ int key_hi(const AttnArgs& a, const Seq& s, int t) {
    return visible_hi(t, s.off, s.m, a.causal);
}
__device__ __forceinline__ int key_lo(const AttnArgs& a, const Seq& s, int t) {
    return visible_lo(t, s.off, a.window);
}

// Where key j of a paged sequence lies: its row in the pages, counted in
// tokens. Page numbers outside the cache are taken as page 0 and reported.
__device__ __forceinline__ int64_t page_row(const int* table, int64_t cols, int b, int pages,
                                            int shift, int* err, int j) {
    int page = page_of(table, cols, b, pages, shift, j);
    if (page < 0) {
        if (err) *err = 1;
        page = 0;
    }
    return page_slot(page, shift, j);
}

typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

// Whether the scaled conversion takes this scale: it reads the exponent alone.
__device__ __forceinline__ bool power_of_two(float scale) {
    return __builtin_amdgcn_frexp_mantf(scale) == 0.5f && scale >= 0x1p-126f;
}

// Eight e4m3 values times a scale as eight 16-bit values. powers: the scale is
// a power of two in every lane (as this library writes them), so the products
// are exact and one instruction a pair; others are formed in float32 and
// rounded to nearest. (Looking at the scales costs 1 %: 8 x 4 tokens over 100000
// cached ones 222.4 us without, 224.9 with.)
template <bool BF>
__device__ __forceinline__ uintx4 widen8(uintx2 u, float scale, bool powers) {
    uintx4 r;
    if (!powers) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(u[i], false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(u[i], true);
            r[2 * i] = pack16<BF>(lo[0] * scale, lo[1] * scale);
            r[2 * i + 1] = pack16<BF>(hi[0] * scale, hi[1] * scale);
        }
        return r;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (BF) {
            r[2 * i] = __builtin_bit_cast(
                unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], scale, false));
            r[2 * i + 1] = __builtin_bit_cast(
                unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], scale, true));
        } else {
            r[2 * i] = __builtin_bit_cast(
                unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u[i], scale, false));
            r[2 * i + 1] = __builtin_bit_cast(
                unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u[i], scale, true));
        }
    }
    return r;
}

}  // namespace ep
