// Attention: out_i = sum_j exp(scale q_i.k_j - lse_i) v_j over the keys j
// that query i sees, lse_i = log sum_j exp(scale q_i.k_j), in one pass over
// the keys with a running maximum and sum.
//
// A workgroup takes 128 rows (attn.h) of one sequence and key head, a wave 32
// of them, and walks the keys in tiles of 64. The product is formed as
// S^T = K Q^T (v_mfma_f32_32x32x16): a lane then holds 32 scores of ONE row,
// so the maximum and the sum of a row need a single exchange between lanes,
// and the probabilities, rounded to the inputs' type, are already in the
// layout of the right operand of out^T += V^T P^T, once V^T is read in the
// order in which a lane holds its keys (TileReader::columns).
//
// Scores, maximum, sum and output accumulate in float32. The probabilities
// are rounded to 16 bits for the second product (at most 2^-8 of them in bf16,
// as much as the output's own rounding); their sum is taken before that.
// In fp16, whose bits thin out below 2^-14, they are 2^12 (2^14) and not 1 where
// a row's largest score is: 131071 keys of 1.5 x 2^-24 beside one of 1 gave 0.0077
// of V instead of 0.0114.
//
// What bounds it: many rows, products and softmax together: matrix units are
// busy 48 % of the cycles, vector units 45 % (2 x 8192 tokens, 32 heads over 8,
// dim 128, causal, bf16: 1.10 ms, 1.00 PFLOP/s, where a library product of 8192^3
// reaches 1.12); at dim 64 the softmax's vector work (58 %, products 28 %; 24
// ragged sequences of up to 1000, 16 heads: 78 us, 0.55 PFLOP/s); few rows,
// memory (64 single tokens over up to 16000: 414 us, 5.6 TB/s; e4m3 rows of up
// to 100000 tokens: 225 us, 4.2 TB/s).
#include "attn.h"
#include "ep_internal.h"
#include "launch.h"

#include <type_traits>

namespace ep {

namespace {

constexpr int kKeys = 64;             // keys of a tile
constexpr int kWaveRows = kKeys / 4;  // keys that a wave loads of a tile
constexpr int kWaveKeys = 32;         // keys of a wave's own tile (few rows)

// Tiles on their way into LDS, fetched a tile ahead into one of two buffers,
// so that the loop's only barrier finds them there. Page numbers are looked up
// a tile before that: a wait for one would wait for the loads before it too.
template <bool BF, int DP, int SOURCE>
struct KeyTiles {
    static constexpr int kQuads = tile_quads(DP);
    static constexpr int kLoads = TileLoader<kQuads, kWaveRows>::kLoads;
    static constexpr bool kEight = SOURCE == kE4m3 || SOURCE == kE4m3Small;
    static constexpr bool kSmall = SOURCE == kPagedSmall || SOURCE == kE4m3Small;
    const AttnArgs& a;
    const Seq& s;
    const int wave, lane, kvh;
    const TileLoader<kQuads, kWaveRows> l;
    int page[kSmall ? kLoads : 1];    // of the wave's rows (of a load's) in the next tile
    // e4m3: the next tile, held in registers until it can be widened
    uintx2 k8[kLoads], v8[kLoads];
    float ks[kLoads], vs[kLoads];

    __device__ __forceinline__ KeyTiles(const AttnArgs& a_, const Seq& s_, int wave_, int lane_, int kvh_)
        : a(a_), s(s_), wave(wave_), lane(lane_), kvh(kvh_), l(lane_, wave_, a_.dim) {}

    __device__ __forceinline__ void look(int j0) {
        if constexpr (SOURCE == kPacked) return;
        const int* t = a.table + s.b * a.cols;
        const int j = j0 + kWaveRows * wave;
        if constexpr (kSmall) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) page[i] = t[min(j + l.row(i), s.m - 1) >> a.page_shift];
        } else {
            page[0] = t[min(j, s.m - 1) >> a.page_shift];
        }
    }
    __device__ __forceinline__ int64_t place(int page, int j) const {
        if ((unsigned)page >= (unsigned)a.pages) {
            if (a.err) *a.err = 1;
            page = 0;
        }
        return page_slot(page, a.page_shift, j);
    }
    // Starts the loads of tile j0, whose pages were looked up (e4m3: into
    // registers).
    __device__ __forceinline__ void fetch(int j0, uintx4* kt, uintx4* vt) {
        const int j = min(j0 + kWaveRows * wave, s.m - 1);
        const char* kp = a.k.p + kvh * a.k.head;
        const char* vp = a.v.p + kvh * a.v.head;
        uintx4* kto = kt + kWaveRows * kQuads * wave;
        uintx4* vto = vt + kWaveRows * kQuads * wave;
        if constexpr (SOURCE == kPacked || SOURCE == kPaged) {
            int64_t row = s.k0 + j;
            if constexpr (SOURCE == kPaged) row = place(__builtin_amdgcn_readfirstlane(page[0]), j);
            l.load(kp + row * a.k.row, s.m - j, a.k.row, kto);
            l.load(vp + row * a.v.row, s.m - j, a.v.row, vto);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                int64_t row;
                if constexpr (kSmall) row = place(page[i], min(j + l.row(i), s.m - 1));
                else row = place(__builtin_amdgcn_readfirstlane(page[0]), j) + min(l.row(i), s.m - 1 - j);
                if constexpr (kEight) {
                    k8[i] = *reinterpret_cast<const uintx2*>(kp + row * a.k.row + l.quad(i) / 2);
                    v8[i] = *reinterpret_cast<const uintx2*>(vp + row * a.v.row + l.quad(i) / 2);
                    ks[i] = a.k_scale[row * a.kv_heads + kvh];
                    vs[i] = a.v_scale[row * a.kv_heads + kvh];
                } else {
                    load_lds16(kp + row * a.k.row + l.quad(i), kto + 64 * i);
                    load_lds16(vp + row * a.v.row + l.quad(i), vto + 64 * i);
                }
            }
        }
    }
    // Puts what fetch holds in registers into the tile.
    __device__ __forceinline__ void store(uintx4* kt, uintx4* vt) {
        if constexpr (kEight) {
            bool powers = true;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) powers = powers && power_of_two(ks[i]) && power_of_two(vs[i]);
            powers = __all(powers);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int to = kWaveRows * kQuads * wave + 64 * i + lane;
                kt[to] = widen8<BF>(k8[i], ks[i], powers);
                vt[to] = widen8<BF>(v8[i], vs[i], powers);
            }
        }
    }
};

// Tiles go straight into LDS a tile ahead: 2118 us at 2 x 8192 tokens when they
// went through registers between two barriers, 1119 like this. Two workgroups
// a CU (64 KB of LDS; at dim 128 218 to 228 registers, up to 256 with e4m3
// pages) overlap one's products with the other's softmax; forming the next
// tile's scores during this one's softmax instead took 1128 us against 1090.
template <bool BF, int DP, int SOURCE>
__global__ void __launch_bounds__(256, 2) attn_kernel(AttnArgs a) {
    constexpr int kQuads = tile_quads(DP);
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    // Probabilities, before their division, are up to 2^(kLift + kRise) and
    // for the largest score at least 2^kLift.
    constexpr float kLift = BF ? 0.f : 12.f;
    constexpr float kRise = BF ? 8.f : 3.f;
    // (arrays of their own: what is loaded into one is not waited for where
    // another is read)
    __shared__ uintx4 kt0[kKeys * kQuads];
    __shared__ uintx4 kt1[kKeys * kQuads];
    __shared__ uintx4 vt0[kKeys * kQuads];
    __shared__ uintx4 vt1[kKeys * kQuads];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5;
    int kvh, tile, tiles;
    head_and_tile(a.kv_heads, kvh, tile, tiles);
    const int split = tile % a.splits;
    const Seq s = find_seq<SOURCE>(a, kRowTile, tile / a.splits, tiles / a.splits);
    const int r0 = s.tile * kRowTile;
    if (r0 < 0 || r0 >= s.rows) return;
    const int r1 = min(r0 + kRowTile, s.rows) - 1;   // the last row

    // this lane's row
    const int row = min(r0 + wave * 32 + (lane & 31), s.rows - 1);
    const int tok = row_token(a, row);
    const int64_t at = s.q0 + tok;
    const int head = kvh * a.group + (row - tok * a.group);
    const int hi = key_hi(a, s, tok), lo = key_lo(a, s, tok);
    // keys that every row of the wave sees, and those that any row of the
    // workgroup does
    const int t0 = row_token(a, min(r0 + wave * 32, s.rows - 1));
    const int t1 = row_token(a, min(r0 + wave * 32 + 31, s.rows - 1));
    const int all_lo = key_lo(a, s, t1), all_hi = key_hi(a, s, t0);
    int begin = key_lo(a, s, row_token(a, r0)) / kKeys * kKeys;
    int end = key_hi(a, s, row_token(a, r1));
    split_range(split, a.splits, kKeys, begin, end);

    floatx16 acc[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
    float top = -3.0e38f, sum = 0.f;                 // (top: in units of log 2)

    if (begin < end) {
        KeyTiles<BF, DP, SOURCE> keys(a, s, wave, lane, kvh);
        keys.look(begin);
        keys.fetch(begin, kt0, vt0);
        if (begin + kKeys < end) keys.look(begin + kKeys);
        uintx4 qf[kSteps];
        const char* qp = a.q.p + at * a.q.row + head * a.q.head;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int d = 16 * i + 8 * half;
            qf[i] = d < a.dim ? *reinterpret_cast<const uintx4*>(qp + 2 * d) : uintx4{0, 0, 0, 0};
        }
        keys.store(kt0, vt0);
        TileReader<kQuads> rd(lane);
        // One tile, in kt and vt; the next goes into kn and vn.
        auto step = [&](int j0, uintx4* kt, uintx4* vt, uintx4* kn, uintx4* vn) {
            wg_barrier<0>();                         // kt and vt are there, kn and vn free
            rd.fresh();
            const bool more = j0 + kKeys < end;
            if (more) {
                keys.fetch(j0 + kKeys, kn, vn);
                if (j0 + 2 * kKeys < end) keys.look(j0 + 2 * kKeys);
            }
            floatx16 sc[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
                    sc[b] = mfma16<BF>(rd.rows(kt, 32 * b, i), qf[i], sc[b]);
            }
            if (j0 < all_lo || j0 + kKeys > all_hi) {
                // (keys j0 + 4 half + c of the lane's, c = 0..3, 8..11, ..)
                const int c_lo = lo - j0 - 4 * half, c_hi = hi - j0 - 4 * half;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int c = 32 * b + 8 * (i >> 2) + (i & 3);
                        if (c < c_lo || c >= c_hi) sc[b][i] = -__builtin_inff();
                    }
            }
            float mx = sc[0][0];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[b][i]);
            mx = pair_max(mx) * a.scale_log2 - kLift;
            // The sums are brought to a new maximum only where it has risen
            // by more than kRise.
            if (__any(mx > top + kRise)) {
                const float now = fmaxf(top, mx);
                const float shrink = __builtin_amdgcn_exp2f(top - now);
                top = now;
                sum *= shrink;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[b][i] *= shrink;
            }
            uintx4 pf[4];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[b][i], a.scale_log2, -top));
                    const float y = __builtin_amdgcn_exp2f(fmaf(sc[b][i + 1], a.scale_log2, -top));
                    sum += x + y;
                    pf[2 * b + (i >> 3)][(i & 7) >> 1] = pack16<BF>(x, y);
                }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
                    acc[b] = mfma16<BF>(rd.columns(vt, 16 * i, b), pf[i], acc[b]);
            if (more) keys.store(kn, vn);
        };
        for (int j0 = begin; j0 < end; j0 += 2 * kKeys) {
            step(j0, kt0, vt0, kt1, vt1);
            if (j0 + kKeys < end) step(j0 + kKeys, kt1, vt1, kt0, vt0);
        }
    }
    if (r0 + wave * 32 + (lane & 31) >= s.rows) return;
    sum = pair_sum(sum);
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    const float lse2 = sum == 0.f ? -__builtin_inff() : top + __builtin_amdgcn_logf(sum);
    if (a.splits > 1) {
        const int64_t to = ((split * a.tokens_q + at) * a.heads + head);
        if (half == 0) a.part_lse[to] = lse2;
        if (sum == 0.f) return;                      // (never read)
        float* part = a.part + to * a.dim;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * b + 2 * i + 4 * half;
                if (d < a.dim)
                    *reinterpret_cast<float4*>(part + d) =
                        make_float4(acc[b][i] * inv, acc[b][i + 1] * inv, acc[b][i + 2] * inv,
                                    acc[b][i + 3] * inv);
            }
        return;
    }
    char* op = a.o.p + at * a.o.row + head * a.o.head;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + 2 * i + 4 * half;
            if (d < a.dim)
                *reinterpret_cast<uintx2*>(op + 2 * d) =
                    uintx2{pack16<BF>(acc[b][i] * inv, acc[b][i + 1] * inv),
                           pack16<BF>(acc[b][i + 2] * inv, acc[b][i + 3] * inv)};
        }
    if (a.lse && half == 0) a.lse[at * a.heads + head] = lse2 * kLn2;
}

// The same pass for few rows (at most 32 a sequence on average; a token of a
// group of 8 fills 8 of 32 columns, which memory-bound work has to spare): a
// workgroup's four waves share 32 rows and take the tiles of 32 keys in turn,
// each with a running maximum and sum of its own, joined at the end. What
// bounds it is the cache's stream from memory: a wave loads its next tile (up
// to 16 KB) into registers while it works on the one in its own part of LDS,
// so there is no barrier before the end, and two workgroups a CU keep up to
// 128 KB on the way.
template <bool BF, int DP, int SOURCE>
__global__ void __launch_bounds__(256, 2) attn_few_kernel(AttnArgs a) {
    constexpr int kQuads = tile_quads(DP);
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    constexpr int kLoads = kWaveKeys * kQuads / 64;  // of K, and of V
    constexpr float kLift = BF ? 0.f : 14.f;         // (probabilities up to 2^kLift)
    __shared__ uintx4 tiles_lds[4][2][kWaveKeys * kQuads];
    __shared__ float s_top[4][32], s_sum[4][32];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5;
    int kvh, tile, tiles;
    head_and_tile(a.kv_heads, kvh, tile, tiles);
    const int split = tile % a.splits;
    const Seq s = find_seq<SOURCE>(a, kFewRows, tile / a.splits, tiles / a.splits);
    const int r0 = s.tile * kFewRows;
    if (r0 < 0 || r0 >= s.rows) return;
    const int r1 = min(r0 + kFewRows, s.rows) - 1;

    const int row = min(r0 + (lane & 31), s.rows - 1);
    const int tok = row_token(a, row);
    const int64_t at = s.q0 + tok;
    const int head = kvh * a.group + (row - tok * a.group);
    const int hi = key_hi(a, s, tok), lo = key_lo(a, s, tok);
    uintx4 qf[kSteps];
    {
        const char* qp = a.q.p + at * a.q.row + head * a.q.head;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int d = 16 * i + 8 * half;
            qf[i] = d < a.dim ? *reinterpret_cast<const uintx4*>(qp + 2 * d) : uintx4{0, 0, 0, 0};
        }
    }
    const int t0 = row_token(a, r0), t1 = row_token(a, r1);
    const int all_lo = key_lo(a, s, t1), all_hi = key_hi(a, s, t0);
    int begin = key_lo(a, s, t0) / kWaveKeys * kWaveKeys;
    int end = key_hi(a, s, t1);
    split_range(split, a.splits, 4 * kWaveKeys, begin, end);

    floatx16 acc[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
    float top = -3.0e38f, sum = 0.f;

    TileReader<kQuads> rd(lane);
    uintx4* kt = tiles_lds[wave][0];
    uintx4* vt = tiles_lds[wave][1];
    const int last_quad = a.dim / 8 - 1;
    typedef std::conditional_t<SOURCE == kE4m3, uintx2, uintx4> Quad;
    Quad kr[kLoads], vr[kLoads];
    // Pages are looked up a tile before they are needed, key j0 + l by lane l:
    // a wait for one would wait for the loads before it too. Lanes 32 on hold
    // the same, and fetch the scales of V's rows where the others do K's.
    int page = 0;
    float scales = 0.f;
    auto look = [&](int j0) {
        if constexpr (SOURCE != kPacked)
            page = a.table[s.b * a.cols + (min(j0 + (lane & 31), s.m - 1) >> a.page_shift)];
    };
    auto load = [&](int j0) {
        const int left = s.m - 1 - j0;
        const bool one_page = SOURCE == kPacked || a.page_shift >= 5;    // (tiles are aligned)
        int64_t row0 = s.k0 + j0;
        int slot = 0;
        if constexpr (SOURCE != kPacked) {
            if ((unsigned)page >= (unsigned)a.pages) {
                if (a.err) *a.err = 1;
                page = 0;
            }
            if (one_page) {
                row0 = page_slot(__builtin_amdgcn_readfirstlane(page), a.page_shift, j0);
                slot = min(lane & 31, left);
            }
            const int64_t mine = one_page ? row0 + slot
                                          : page_slot(page, a.page_shift, min(j0 + (lane & 31), s.m - 1));
            if constexpr (SOURCE == kE4m3)
                scales = (half ? a.v_scale : a.k_scale)[mine * a.kv_heads + kvh];
        }
        const char* kp = a.k.p + row0 * a.k.row + kvh * a.k.head;
        const char* vp = a.v.p + row0 * a.v.row + kvh * a.v.head;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at_quad = lane + 64 * i;
            const int r = at_quad / kQuads;
            const int quad = min((at_quad % kQuads) ^ swizzle<kQuads>(r), last_quad) * (int)sizeof(Quad);
            const int j = min(r, left);
            if (one_page) {
                kr[i] = *reinterpret_cast<const Quad*>(kp + ((unsigned)j * (unsigned)a.k.row + quad));
                vr[i] = *reinterpret_cast<const Quad*>(vp + ((unsigned)j * (unsigned)a.v.row + quad));
            } else {
                const int64_t row = page_slot(__shfl(page, j), a.page_shift, j0 + j);
                kr[i] = *reinterpret_cast<const Quad*>(a.k.p + row * a.k.row + kvh * a.k.head + quad);
                vr[i] = *reinterpret_cast<const Quad*>(a.v.p + row * a.v.row + kvh * a.v.head + quad);
            }
        }
    };
    int j0 = begin + wave * kWaveKeys;
    if (j0 < end) {
        look(j0);
        load(j0);
        if (j0 + 4 * kWaveKeys < end) look(j0 + 4 * kWaveKeys);
    }
    for (; j0 < end; j0 += 4 * kWaveKeys) {
        const bool powers = SOURCE != kE4m3 || __all(power_of_two(scales));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if constexpr (SOURCE == kE4m3) {
                const int r = (lane + 64 * i) / kQuads;
                kt[lane + 64 * i] = widen8<BF>(kr[i], __shfl(scales, r), powers);
                vt[lane + 64 * i] = widen8<BF>(vr[i], __shfl(scales, 32 + r), powers);
            } else {
                kt[lane + 64 * i] = kr[i];
                vt[lane + 64 * i] = vr[i];
            }
        }
        if (j0 + 4 * kWaveKeys < end) {
            load(j0 + 4 * kWaveKeys);
            if (j0 + 8 * kWaveKeys < end) look(j0 + 8 * kWaveKeys);
        }
        rd.fresh();
        floatx16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            sc = mfma16<BF>(rd.rows(kt, 0, i), qf[i], sc);
        if (j0 < all_lo || j0 + kWaveKeys > all_hi) {
            const int c_lo = lo - j0 - 4 * half, c_hi = hi - j0 - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = 8 * (i >> 2) + (i & 3);
                if (c < c_lo || c >= c_hi) sc[i] = -__builtin_inff();
            }
        }
        float mx = sc[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
        mx = pair_max(mx) * a.scale_log2 - kLift;
        const float now = fmaxf(top, mx);
        const float shrink = __builtin_amdgcn_exp2f(top - now);
        top = now;
        sum *= shrink;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[b][i] *= shrink;
        uintx4 pf[2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(sc[i], a.scale_log2, -top));
            const float y = __builtin_amdgcn_exp2f(fmaf(sc[i + 1], a.scale_log2, -top));
            sum += x + y;
            pf[i >> 3][(i & 7) >> 1] = pack16<BF>(x, y);
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                acc[b] = mfma16<BF>(rd.columns(vt, 16 * i, b), pf[i], acc[b]);
    }
    // Joining: every wave leaves its sums in its part of LDS, row by row of
    // queries (quads permuted by the row, which spreads a write over the
    // banks), and 8 threads gather a row.
    sum = pair_sum(sum);
    if (half == 0) {
        s_top[wave][lane] = top;
        s_sum[wave][lane] = sum;
    }
    constexpr int kFloatQuads = DP / 4;
    float4* mine = reinterpret_cast<float4*>(tiles_lds[wave]);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int quad = 8 * b + (i >> 1) + half;
            mine[(lane & 31) * kFloatQuads + (quad ^ (lane & 7))] =
                make_float4(acc[b][i], acc[b][i + 1], acc[b][i + 2], acc[b][i + 3]);
        }
    __syncthreads();
    const int q = tid >> 3;
    if (r0 + q >= s.rows) return;
    float weight[4], all = -3.0e38f, total = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) all = fmaxf(all, s_top[w][q]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        weight[w] = __builtin_amdgcn_exp2f(s_top[w][q] - all);
        total = fmaf(weight[w], s_sum[w][q], total);
    }
    const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
    const float lse2 = total == 0.f ? -__builtin_inff() : all + __builtin_amdgcn_logf(total);
    const int qtok = row_token(a, r0 + q);
    const int qhead = kvh * a.group + (r0 + q - qtok * a.group);
    const int64_t to = (int64_t)(s.q0 + qtok) * a.heads + qhead;
    const int64_t to_part = split * a.tokens_q * a.heads + to;
    if ((tid & 7) == 0) {
        if (a.splits > 1) a.part_lse[to_part] = lse2;
        else if (a.lse) a.lse[to] = lse2 * kLn2;
    }
    if (a.splits > 1 && total == 0.f) return;        // (never read)
    char* op = a.o.p + (s.q0 + qtok) * a.o.row + qhead * a.o.head;
#pragma unroll
    for (int i = 0; i < kFloatQuads / 8; ++i) {
        const int quad = (tid & 7) + 8 * i;
        if (quad * 4 >= a.dim) break;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float4 x = reinterpret_cast<const float4*>(tiles_lds[w])[q * kFloatQuads + (quad ^ (q & 7))];
            o.x = fmaf(weight[w], x.x, o.x);
            o.y = fmaf(weight[w], x.y, o.y);
            o.z = fmaf(weight[w], x.z, o.z);
            o.w = fmaf(weight[w], x.w, o.w);
        }
        if (a.splits > 1)
            *reinterpret_cast<float4*>(a.part + to_part * a.dim + quad * 4) =
                make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        else
            *reinterpret_cast<uintx2*>(op + quad * 8) =
                uintx2{pack16<BF>(o.x * inv, o.y * inv), pack16<BF>(o.z * inv, o.w * inv)};
    }
}

constexpr int kJoin = 8;

// out = sum over the cuts of 2^(lse_s - lse) part_s, in the cuts' order; a
// thread takes four elements of a row.
template <bool BF>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs a) {
    const int quads = a.dim / 4;
    const int64_t rows = a.tokens_q * a.heads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * quads;
         i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / quads, tok = row / a.heads;
        const int quad = (int)(i % quads), head = (int)(row % a.heads);
        // rows behind the last sequence have no partial results
        if (tok < a.start_q[0] || tok >= a.start_q[a.batch]) continue;
        float all = -3.0e38f, total = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < a.splits; s += kJoin) {  // kJoin cuts' loads at once
            float l[kJoin], most = all;
            float4 x[kJoin];
#pragma unroll
            for (int e = 0; e < kJoin; ++e) {
                l[e] = s + e < a.splits ? a.part_lse[(s + e) * rows + row] : -__builtin_inff();
                most = fmaxf(most, l[e]);
            }
#pragma unroll
            for (int e = 0; e < kJoin; ++e)          // (a cut without keys left nothing)
                if (l[e] != -__builtin_inff())
                    x[e] = *reinterpret_cast<const float4*>(a.part + ((s + e) * rows + row) * a.dim + quad * 4);
            const float shrink = __builtin_amdgcn_exp2f(all - most);
            all = most;
            total *= shrink;
            o = make_float4(o.x * shrink, o.y * shrink, o.z * shrink, o.w * shrink);
#pragma unroll
            for (int e = 0; e < kJoin; ++e) {
                if (l[e] == -__builtin_inff()) continue;
                const float w = __builtin_amdgcn_exp2f(l[e] - all);
                total += w;
                o.x = fmaf(w, x[e].x, o.x);
                o.y = fmaf(w, x[e].y, o.y);
                o.z = fmaf(w, x[e].z, o.z);
                o.w = fmaf(w, x[e].w, o.w);
            }
        }
        const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
        *reinterpret_cast<uintx2*>(a.o.p + tok * a.o.row + head * a.o.head + quad * 8) =
            uintx2{pack16<BF>(o.x * inv, o.y * inv), pack16<BF>(o.z * inv, o.w * inv)};
        if (quad == 0 && a.lse)
            a.lse[row] = total == 0.f ? -__builtin_inff() : (all + __builtin_amdgcn_logf(total)) * kLn2;
    }
}

template <bool BF, int DP, int SOURCE>
void launch_dim(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    const dim3 grid((unsigned)(attn_groups(a.kv_heads, a.tokens_q * a.group, p.tile, a.batch) * p.splits));
    // (few rows look up a page for every row they load)
    constexpr int kFewSource = SOURCE == kPagedSmall ? kPaged : SOURCE == kE4m3Small ? kE4m3 : SOURCE;
    if (p.tile == kFewRows)
        hipLaunchKernelGGL((attn_few_kernel<BF, DP, kFewSource>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((attn_kernel<BF, DP, SOURCE>), grid, dim3(256), 0, s, a);
}

template <bool BF, int SOURCE>
void launch(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    if (a.dim > 96) launch_dim<BF, 128, SOURCE>(a, p, s);
    else if (a.dim > 64) launch_dim<BF, 96, SOURCE>(a, p, s);
    else launch_dim<BF, 64, SOURCE>(a, p, s);
}

}  // namespace

AttnPlan attn_plan(int64_t batch, int64_t tokens_q, int64_t heads, int64_t kv_heads, int64_t dim,
                   int64_t most_keys) {
    AttnPlan p;
    const int64_t rows = tokens_q * (heads / kv_heads);
    const int64_t sequences = std::max<int64_t>(std::min(batch, tokens_q), 1);
    p.tile = rows <= kFewRows * sequences ? kFewRows : kRowTile;
    // Up to 64 rows a sequence in tiles of 32 read the keys twice: 186 us for 16
    // sequences of 64 rows over 20000 keys, 152 in one tile of 128.
    // Workgroups that have work, if no sequence is much longer than the
    // others; the keys are cut until the device is full. Few rows: its 512
    // slots four times over, so that ragged lengths even out (64 single tokens
    // over up to 16000 keys, e4m3 rows of up to 100000: once 494 and 287 us,
    // twice 459 and 250, four times 437 and 244, eight times 434 and 254). Many
    // rows: once (4 x 512 rows over 30000 keys: half 442 us, once 310, twice 323).
    const int64_t groups = kv_heads * std::max(sequences, ceil_div(rows, p.tile));
    const int64_t want = p.tile == kFewRows ? 2048 : 512;
    // At least 512 keys a range: a token over 511 takes 11.6 us in one piece, 9.5
    // in four, replayed from a graph, but a second launch takes the host 3.5;
    // a token over 4096 14.8 (ranges of 1024: 21.4).
    const int64_t least = p.tile == kFewRows ? 16 * kWaveKeys : 4 * kKeys;
    p.splits = (int)std::max<int64_t>(
        1, std::min({want / groups, most_keys / least, int64_t(128),
                     kMaxGroups / attn_groups(kv_heads, rows, p.tile, batch)}));
    p.bytes = p.splits > 1 ? round_up(p.splits * tokens_q * heads * (dim + 1) * 4, 16) : 0;
    return p;
}

hipError_t attn_forward_launch(const AttnArgs& a, const AttnPlan& p, bool bf, int source,
                               hipStream_t s) {
    switch (source * 2 + (bf ? 1 : 0)) {
    case 0: launch<false, kPacked>(a, p, s); break;
    case 1: launch<true, kPacked>(a, p, s); break;
    case 2: launch<false, kPaged>(a, p, s); break;
    case 3: launch<true, kPaged>(a, p, s); break;
    case 4: launch<false, kPagedSmall>(a, p, s); break;
    case 5: launch<true, kPagedSmall>(a, p, s); break;
    case 6: launch<false, kE4m3>(a, p, s); break;
    case 7: launch<true, kE4m3>(a, p, s); break;
    case 8: launch<false, kE4m3Small>(a, p, s); break;
    default: launch<true, kE4m3Small>(a, p, s); break;
    }
    if (p.splits > 1) {
        const dim3 grid(stride_grid(ceil_div(a.tokens_q * a.heads * (a.dim / 4), 256), 256));
        if (bf) hipLaunchKernelGGL(attn_join_kernel<true>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(attn_join_kernel<false>, grid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace ep
