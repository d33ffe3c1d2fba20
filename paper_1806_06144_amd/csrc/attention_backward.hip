// Gradients of attention (attention.hip): with p_ij = exp(scale q_i.k_j -
// lse_i) formed again from the stored log-sums, dp_ij = dout_i.v_j, D_i =
// sum_j p_ij dp_ij = out_i.dout_i and ds_ij = p_ij (dp_ij - D_i),
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,
//   dv_j = sum_i p_ij dout_i,
// the sums over i running over the heads of a group too.
//
// What bounds them (matrix units' busy cycles, waves' waiting ones): 2 x 4096
// tokens, 32 heads over 8, dim 128, bf16: at least 412 us for dq (49 %, 37 %) and
// 664 for dk and dv (39 %, 34 %), 1036 one after another, 0.93 PFLOP/s of the
// seven products; at dim 64 with short ranges barriers and vector work (12
// ragged sequences of up to 2047 with a window of 512, 12 heads, fp16: 81 us
// (23 %, 37 %) and 102 (23 %, 39 %)).
//
// Two kernels, each owning what it sums, so there are no atomics and the
// results do not depend on the order of the workgroups: dq walks the keys as
// the forward pass does (three products a tile), dk and dv walk the rows
// (four). Sharing the two products that both form would take five instead of
// seven, but needs dq summed over workgroups in float32 memory.
//
// Scores, probabilities and sums are float32; p and ds are rounded to the
// inputs' type for their products, as the probabilities of the forward pass.
// fp16 has all its bits from 2^-14 to 65504 only, while p is 1 / keys and ds
// that much smaller too: both enter their products times a power of two, which
// the float32 sums are divided by at the end (exactly). p is at most one and
// takes 2^14. What ds may be depends on dout, so a row's (for dk a key's) power
// starts high and comes down as its largest ds asks for, as a softmax's maximum
// rises. Without, at 131072 keys dv was 6.6 times as far off as the exact one
// rounded, and dq 45 times for dout of 2^-8; like this 1.4 and 1.03. It costs
// fp16 2 to 4 % (2 x 4096 tokens, 32 heads over 8: at dim 128 dq 410 us without,
// 417 like this, dk and dv 610 and 630; at dim 64 236 and 242, 523 and 538).
#include "attn.h"
#include "ep_internal.h"
#include "launch.h"

#include <type_traits>

namespace ep {

namespace {

constexpr int kKeyTile = 64;          // keys of a tile (dq)
constexpr int kWaveKeys = 16;         // of these, loaded by a wave
// D_i = out_i.dout_i carries the rounding of out, which beside ds counts as
// 1 / sqrt(keys): rows of at most this many keys sum p_ij dp_ij in a sweep of
// their own instead. 12 sequences of 201 (256, 512) in bf16, 12 heads of 64, dq's
// error beside that of the exact one rounded: without 1.49 (1.57, 1.48) in 32 (35,
// 57) us, up to 256 keys 1.40 (1.44, 1.41) in 37 (39, 61), up to 512 keys 1.40
// (1.44, 1.40) in 37 (39, 68), where the second sweep gains nothing any more. (Up
// to 128 keys: 1.41 (1.45, 1.41) in 33 (35, 58).)
constexpr int kSummedKeys = 256;
constexpr int kStepRows = 32;         // rows of a tile (dk, dv)
constexpr int kWaveRows = 8;          // of these, loaded by a wave
constexpr int kStages = 4;            // tiles of rows in LDS (three are in use)
constexpr int kKeyRange = 128;        // keys of a workgroup (dk, dv): 32 per wave

constexpr int kLiftP = 14;           // fp16: exponents of the powers of two of p,
constexpr int kLiftSlope = 60;       // and of ds where a row or key starts

// x: ds times 2^lift of a lane's row or key (which lanes l and l + 32 share),
// acc its sums. Where one is past 2^15, brings them down to 2^11, which leaves
// room to grow: 25 binades below hold all their bits.
template <int BLOCKS>
__device__ __forceinline__ bool keep_in_range(floatx16& x, floatx16 (&acc)[BLOCKS], int& lift) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(x[i]));
    if (!__any(most > 0x1p15f)) return false;
    most = pair_max(most);
    const int drop = most > 0x1p15f ? __builtin_amdgcn_frexp_expf(most) - 11 : 0;
    const float by = __builtin_amdgcn_ldexpf(1.f, -drop);
    lift -= drop;
    x *= by;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) acc[b] *= by;
    return true;
}

template <bool BF, int DP>
__global__ void __launch_bounds__(256, 2) attn_dq_kernel(AttnArgs a) {
    constexpr int kQuads = tile_quads(DP);
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    __shared__ uintx4 kt0[kKeyTile * kQuads];
    __shared__ uintx4 kt1[kKeyTile * kQuads];
    __shared__ uintx4 vt0[kKeyTile * kQuads];
    __shared__ uintx4 vt1[kKeyTile * kQuads];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5;
    int kvh, tile, tiles;
    head_and_tile(a.kv_heads, kvh, tile, tiles);
    const int split = tile % a.key_splits;
    const Seq s = find_seq<kPacked>(a, kRowTile, tile / a.key_splits, tiles / a.key_splits);
    const int r0 = s.tile * kRowTile;
    if (r0 < 0 || r0 >= s.rows) return;
    const int r1 = min(r0 + kRowTile, s.rows) - 1;

    const int row = min(r0 + wave * 32 + (lane & 31), s.rows - 1);
    const int tok = row_token(a, row);
    const int64_t at = s.q0 + tok;
    const int head = kvh * a.group + (row - tok * a.group);
    const int hi = key_hi(a, s, tok), lo = key_lo(a, s, tok);
    const int t0 = row_token(a, min(r0 + wave * 32, s.rows - 1));
    const int t1 = row_token(a, min(r0 + wave * 32 + 31, s.rows - 1));
    const int all_lo = key_lo(a, s, t1), all_hi = key_hi(a, s, t0);
    int begin = key_lo(a, s, row_token(a, r0)) / kKeyTile * kKeyTile;
    int end = key_hi(a, s, row_token(a, r1));
    // D from p and dp (from out where the keys are cut: there are many)
    const bool summed = end - begin <= kSummedKeys;
    const bool cut = a.key_splits > 1 && !summed;
    if (cut) split_range(split, a.key_splits, kKeyTile, begin, end);
    else if (split > 0) end = begin;                 // (the first workgroup takes them all)
    const bool single = hi - lo == 1;                // one key: p is 1, D is dp, ds nothing

    const TileLoader<kQuads, kWaveKeys> l(lane, wave, a.dim);
    TileReader<kQuads> rd(lane);
    auto fetch = [&](int j0, uintx4* kt, uintx4* vt) {
        const int j = min(j0 + kWaveKeys * wave, s.m - 1);
        const int to = kWaveKeys * kQuads * wave;
        l.load(a.k.p + kvh * a.k.head + (int64_t)(s.k0 + j) * a.k.row, s.m - j, a.k.row, kt + to);
        l.load(a.v.p + kvh * a.v.head + (int64_t)(s.k0 + j) * a.v.row, s.m - j, a.v.row, vt + to);
    };
    if (begin < end) fetch(begin, kt0, vt0);
    uintx4 qf[kSteps], gf[kSteps];
    float delta = 0.f;
    {
        const char* qp = a.q.p + at * a.q.row + head * a.q.head;
        const char* gp = a.dout.p + at * a.dout.row + head * a.dout.head;
        const char* op = a.o.p + at * a.o.row + head * a.o.head;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int d = 16 * i + 8 * half;
            const uintx4 zero = {0, 0, 0, 0};
            qf[i] = d < a.dim ? *reinterpret_cast<const uintx4*>(qp + 2 * d) : zero;
            gf[i] = d < a.dim ? *reinterpret_cast<const uintx4*>(gp + 2 * d) : zero;
        }
        if (!summed) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int d = 16 * i + 8 * half;
                const uintx4 o = d < a.dim ? *reinterpret_cast<const uintx4*>(op + 2 * d) : uintx4{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    delta = fmaf(lo16<BF>(o[e]), lo16<BF>(gf[i][e]), delta);
                    delta = fmaf(hi16<BF>(o[e]), hi16<BF>(gf[i][e]), delta);
                }
            }
            delta = pair_sum(delta);
        }
    }
    const bool mine = r0 + wave * 32 + (lane & 31) < s.rows;
    const float lse2 = a.lse[at * a.heads + head] * kLog2e;
    if (mine && half == 0 && split == 0) a.lse2[at * a.heads + head] = BF ? lse2 : lse2 - kLiftP;
    int lift = BF ? 0 : kLiftSlope;                  // (of this lane's row)

    floatx16 acc[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;

    // One tile, in kt and vt; the next goes into kn and vn. ds: adds to acc;
    // else to delta.
    auto step = [&](auto ds, int j0, const uintx4* kt, const uintx4* vt, uintx4* kn,
                    uintx4* vn) __attribute__((always_inline)) {
        wg_barrier<0>();                             // kt and vt are there, kn and vn free
        rd.fresh();
        if (j0 + kKeyTile < end) fetch(j0 + kKeyTile, kn, vn);
        const bool masked = j0 < all_lo || j0 + kKeyTile > all_hi;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            floatx16 sc, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                sc = mfma16<BF>(rd.rows(kt, 32 * b, i), qf[i], sc);
                dp = mfma16<BF>(rd.rows(vt, 32 * b, i), gf[i], dp);
            }
            float p[16];
            const float base = !BF && decltype(ds)::value ? (float)lift - lse2 : -lse2;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.scale_log2, base));
            if (masked) {                            // (a row that sees nothing has lse = -inf)
                const int c_lo = lo - j0 - 4 * half, c_hi = hi - j0 - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int c = 32 * b + 8 * (i >> 2) + (i & 3);
                    p[i] = c >= c_lo && c < c_hi ? p[i] : 0.f;
                }
            }
            if constexpr (!decltype(ds)::value) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    delta = fmaf(single && p[i] != 0.f ? 1.f : p[i], dp[i], delta);
            } else {
                uintx4 df[2];
#pragma unroll
                for (int i = 0; i < 16; ++i) dp[i] = p[i] * (dp[i] - delta);
                if constexpr (!BF) keep_in_range(dp, acc, lift);
#pragma unroll
                for (int i = 0; i < 16; i += 2) df[i >> 3][(i & 7) >> 1] = pack16<BF>(dp[i], dp[i + 1]);
#pragma unroll
                for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        acc[c] = mfma16<BF>(rd.columns(kt, 32 * b + 16 * i, c), df[i], acc[c]);
            }
        }
    };
    auto sweep = [&](auto ds) __attribute__((always_inline)) {
        for (int j0 = begin; j0 < end; j0 += 2 * kKeyTile) {
            step(ds, j0, kt0, vt0, kt1, vt1);
            if (j0 + kKeyTile < end) step(ds, j0 + kKeyTile, kt1, vt1, kt0, vt0);
        }
    };
    if (summed && begin < end) {
        sweep(std::false_type{});
        delta = pair_sum(delta);
        wg_barrier<-1>();                            // (every wave has left the tiles)
        fetch(begin, kt0, vt0);
    }
    sweep(std::true_type{});
    if (!mine) return;
    if (half == 0 && split == 0) a.delta[at * a.heads + head] = delta;
    const float scale = BF ? a.scale : __builtin_amdgcn_ldexpf(a.scale, -lift);
    if (a.key_splits > 1) {
        float* p = a.part_q + ((split * a.tokens_q + at) * a.heads + head) * a.dim;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * b + 2 * i + 4 * half;
                if (d < a.dim)
                    *reinterpret_cast<float4*>(p + d) =
                        make_float4(acc[b][i] * scale, acc[b][i + 1] * scale,
                                    acc[b][i + 2] * scale, acc[b][i + 3] * scale);
            }
        return;
    }
    char* out = a.dq.p + at * a.dq.row + head * a.dq.head;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + 2 * i + 4 * half;
            if (d < a.dim)
                *reinterpret_cast<uintx2*>(out + 2 * d) =
                    uintx2{pack16<BF>(acc[b][i] * scale, acc[b][i + 1] * scale),
                           pack16<BF>(acc[b][i + 2] * scale, acc[b][i + 3] * scale)};
        }
}

// Two waves own 32 keys: one forms S = Q K^T, P and dv^T += dout^T P, the
// other dP = dout V^T, dS from it and the first one's P (float32, through LDS),
// and dk^T += Q^T dS, a tile of rows behind. Each holds its operand of K or V
// (32 registers at dim 128) and one sum (64), which leaves room for two waves
// a SIMD, one of each kind, whose matrix products, exponentials and LDS reads
// overlap. One wave with both operands and sums (192 registers) ran alone on its
// SIMD: 880 us at 2 x 4096 tokens, 32 heads over 8, dim 128, where pairs took 690
// with all else the same. Products whose result has a key a lane (16 rows of ONE
// key) leave P and dS in the order in which the second products take them.
template <bool BF, int DP>
__global__ void __launch_bounds__(512, DP == 64 ? 4 : 2) attn_dkv_kernel(AttnArgs a) {
    constexpr int kQuads = tile_quads(DP);
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    // (arrays of their own: what is loaded into one is not waited for where
    // another is read)
    __shared__ uintx4 qt0[kStepRows * kQuads], qt1[kStepRows * kQuads];
    __shared__ uintx4 qt2[kStepRows * kQuads], qt3[kStepRows * kQuads];
    __shared__ uintx4 gt0[kStepRows * kQuads], gt1[kStepRows * kQuads];
    __shared__ uintx4 gt2[kStepRows * kQuads], gt3[kStepRows * kQuads];
    __shared__ float4 rw0[kStepRows / 2], rw1[kStepRows / 2];            // lse2, delta
    __shared__ float4 rw2[kStepRows / 2], rw3[kStepRows / 2];
    __shared__ float4 p0[4 * 4 * 64], p1[4 * 4 * 64];                    // P of four pairs

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pair = wave & 3;
    const bool second = wave >= 4;                   // the wave of dP, dS and dk
    const int half = lane >> 5;
    int kvh, tile, tiles;
    head_and_tile(a.kv_heads, kvh, tile, tiles);
    const int split = tile % a.row_splits;
    const Seq s = find_seq<kPacked, true>(a, kKeyRange, tile / a.row_splits, tiles / a.row_splits);
    const int k0 = s.tile * kKeyRange;
    if (k0 < 0 || k0 >= s.m) return;
    const int k1 = min(k0 + kKeyRange, s.m) - 1;

    auto from_row = [&](int j) { return seen_from(j, s.off, s.n, a.group, a.causal); };
    auto to_row = [&](int j) { return seen_to(j, s.off, s.n, a.group, a.window); };
    const int key = min(k0 + pair * 32 + (lane & 31), s.m - 1);
    const int lo = from_row(key), hi = to_row(key);
    const int wk0 = min(k0 + pair * 32, s.m - 1), wk1 = min(k0 + pair * 32 + 31, s.m - 1);
    // (rows past the last are rows that see nothing)
    const int all_lo = from_row(wk1), all_hi = min(to_row(wk0), s.rows);
    int begin = from_row(k0) / kStepRows * kStepRows, end = to_row(k1);
    split_range(split, a.row_splits, kStepRows, begin, end);

    const TileLoader<kQuads, kWaveRows> l(lane, pair, a.dim);
    TileReader<kQuads> rd(lane);
    const Rows in = second ? a.dout : a.q;           // the rows that this wave loads
    // Where the group divides the tile, a lane's rows are the same tokens and
    // heads of every tile, counted from its first.
    const bool even = kStepRows % a.group == 0 && in.head * a.group < (1 << 30);
    unsigned off[l.kLoads], off_row;
    {
        const unsigned st = (unsigned)in.row, sh = even ? (unsigned)in.head : 0;
#pragma unroll
        for (int i = 0; i < l.kLoads; ++i) {
            const int r = kWaveRows * pair + l.row(i);
            const unsigned t = row_token(a, r);
            off[i] = t * st + (r - t * a.group) * sh + l.quad(i);
        }
        const unsigned t = row_token(a, lane & 31);
        off_row = t * a.heads + ((lane & 31) - t * a.group);
    }
    auto fetch = [&](int i0, uintx4* qt, uintx4* gt, float4* rows) {
        // the tile's first row is (tok0, rem0)
        const int tok0 = row_token(a, i0), rem0 = i0 - tok0 * a.group;
        const char* p = in.p + (int64_t)(s.q0 + tok0) * in.row + kvh * a.group * in.head;
        const int64_t at = (int64_t)(s.q0 + tok0) * a.heads + kvh * a.group;
        uintx4* to = (second ? gt : qt) + kWaveRows * kQuads * pair;
        const int last = s.rows - 1 - i0;
        if (even && last >= kStepRows - 1) {
#pragma unroll
            for (int i = 0; i < l.kLoads; ++i) load_lds16(p + off[i], to + 64 * i);
            if (wave == 0) load_lds4((half ? a.delta : a.lse2) + at + off_row, reinterpret_cast<float*>(rows));
            return;
        }
#pragma unroll
        for (int i = 0; i < l.kLoads; ++i) {
            const int r = rem0 + min(kWaveRows * pair + l.row(i), last);
            const unsigned t = row_token(a, r), h = r - t * a.group;
            load_lds16(p + (t * (uint64_t)in.row + h * (uint64_t)in.head) + l.quad(i), to + 64 * i);
        }
        if (wave == 0) {
            const int r = rem0 + min(lane & 31, last);
            const int t = row_token(a, r);
            load_lds4((half ? a.delta : a.lse2) + at + (t * (int64_t)a.heads + (r - t * a.group)),
                      reinterpret_cast<float*>(rows));
        }
    };
    if (begin < end) fetch(begin, qt0, gt0, rw0);
    uintx4 kv[kSteps];                               // the wave's keys' rows of K or V
    {
        const Rows& x = second ? a.v : a.k;
        const char* p = x.p + (int64_t)(s.k0 + key) * x.row + kvh * x.head;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int d = 16 * i + 8 * half;
            kv[i] = d < a.dim ? *reinterpret_cast<const uintx4*>(p + 2 * d) : uintx4{0, 0, 0, 0};
        }
    }
    floatx16 acc[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;

    int lift = kLiftSlope - kLiftP;                  // (fp16; of this lane's key)
    float up = __builtin_amdgcn_ldexpf(1.f, lift);
    auto product = [&](const uintx4* x) {            // x kv^T, 32 rows x 32 keys
        floatx16 y;
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) y = mfma16<BF>(rd.rows(x, 0, i), kv[i], y);
        return y;
    };
    auto add = [&](const uintx4* x, const floatx16& y) {     // acc += x^T y
        uintx4 f[2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) f[i >> 3][(i & 7) >> 1] = pack16<BF>(y[i], y[i + 1]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) acc[c] = mfma16<BF>(rd.columns(x, 16 * i, c), f[i], acc[c]);
    };
    // The first wave's part of the tile at i0.
    auto probabilities = [&](int i0, const uintx4* qt, const uintx4* gt, const float4* rows, float4* p) {
        floatx16 x = product(qt);
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 l4 = rows[2 * (i >> 2) + half];
            x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], a.scale_log2, -l4.x));
            x[i + 1] = __builtin_amdgcn_exp2f(fmaf(x[i + 1], a.scale_log2, -l4.y));
            x[i + 2] = __builtin_amdgcn_exp2f(fmaf(x[i + 2], a.scale_log2, -l4.z));
            x[i + 3] = __builtin_amdgcn_exp2f(fmaf(x[i + 3], a.scale_log2, -l4.w));
        }
        if (i0 < all_lo || i0 + kStepRows > all_hi) {
            // (rows i0 + 4 half + c of the lane's, c = 0..3, 8..11, ..)
            const int c_lo = lo - i0 - 4 * half, c_hi = min(hi, s.rows) - i0 - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = 8 * (i >> 2) + (i & 3);
                x[i] = c >= c_lo && c < c_hi ? x[i] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            p[(4 * pair + (i >> 2)) * 64 + lane] = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        add(gt, x);
    };
    // The second wave's.
    auto slopes = [&](const uintx4* qt, const uintx4* gt, const float4* rows, const float4* p) {
        floatx16 x = product(gt);
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 d4 = rows[kStepRows / 4 + 2 * (i >> 2) + half];
            const float4 p4 = p[(4 * pair + (i >> 2)) * 64 + lane];
            x[i] = p4.x * (x[i] - d4.x);
            x[i + 1] = p4.y * (x[i + 1] - d4.y);
            x[i + 2] = p4.z * (x[i + 2] - d4.z);
            x[i + 3] = p4.w * (x[i + 3] - d4.w);
        }
        if constexpr (!BF) {
            x *= up;
            if (keep_in_range(x, acc, lift)) up = __builtin_amdgcn_ldexpf(1.f, lift);
        }
        add(qt, x);
    };
    // Iteration i0: tile i0 for the first waves (there is none past the end),
    // the one before it for the second, the next on its way.
    auto enter = [&](int i0, uintx4* qn, uintx4* gn, float4* rn) {
        wg_barrier<0>();                             // tile i0 and the P before it are there
        rd.fresh();
        if (i0 + kStepRows < end) fetch(i0 + kStepRows, qn, gn, rn);
    };
    const int stop = end + kStepRows;                // (a tile more for the second waves)
    if (begin < end) {
        if (!second) {
            for (int i0 = begin; i0 < stop; i0 += kStages * kStepRows) {
                enter(i0, qt1, gt1, rw1);
                if (i0 < end) probabilities(i0, qt0, gt0, rw0, p0);
                if (i0 + kStepRows >= stop) break;
                enter(i0 + kStepRows, qt2, gt2, rw2);
                if (i0 + kStepRows < end) probabilities(i0 + kStepRows, qt1, gt1, rw1, p1);
                if (i0 + 2 * kStepRows >= stop) break;
                enter(i0 + 2 * kStepRows, qt3, gt3, rw3);
                if (i0 + 2 * kStepRows < end) probabilities(i0 + 2 * kStepRows, qt2, gt2, rw2, p0);
                if (i0 + 3 * kStepRows >= stop) break;
                enter(i0 + 3 * kStepRows, qt0, gt0, rw0);
                if (i0 + 3 * kStepRows < end) probabilities(i0 + 3 * kStepRows, qt3, gt3, rw3, p1);
            }
        } else {
            for (int i0 = begin; i0 < stop; i0 += kStages * kStepRows) {
                enter(i0, qt1, gt1, rw1);
                if (i0 > begin) slopes(qt3, gt3, rw3, p1);
                if (i0 + kStepRows >= stop) break;
                enter(i0 + kStepRows, qt2, gt2, rw2);
                slopes(qt0, gt0, rw0, p0);
                if (i0 + 2 * kStepRows >= stop) break;
                enter(i0 + 2 * kStepRows, qt3, gt3, rw3);
                slopes(qt1, gt1, rw1, p1);
                if (i0 + 3 * kStepRows >= stop) break;
                enter(i0 + 3 * kStepRows, qt0, gt0, rw0);
                slopes(qt2, gt2, rw2, p0);
            }
        }
    }
    if (k0 + pair * 32 + (lane & 31) >= s.m) return;
    float scale = second ? a.scale : 1.f;
    if constexpr (!BF) scale = __builtin_amdgcn_ldexpf(scale, -kLiftP - (second ? lift : 0));
    if (a.row_splits > 1) {
        float* p = a.part_kv + (((split * 2 + (second ? 1 : 0)) * a.tokens_k + s.k0 + key) * a.kv_heads + kvh) * a.dim;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * b + 2 * i + 4 * half;
                if (d < a.dim)
                    *reinterpret_cast<float4*>(p + d) =
                        make_float4(acc[b][i] * scale, acc[b][i + 1] * scale, acc[b][i + 2] * scale,
                                    acc[b][i + 3] * scale);
            }
        return;
    }
    const Rows& out = second ? a.dk : a.dv;
    char* p = out.p + (int64_t)(s.k0 + key) * out.row + kvh * out.head;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + 2 * i + 4 * half;
            if (d < a.dim)
                *reinterpret_cast<uintx2*>(p + 2 * d) =
                    uintx2{pack16<BF>(acc[b][i] * scale, acc[b][i + 1] * scale),
                           pack16<BF>(acc[b][i + 2] * scale, acc[b][i + 3] * scale)};
        }
}

// Outputs (blockIdx.y) from their cuts' partial sums, in the cuts' order; a
// thread takes four elements.
struct SumArgs {
    const float* part[2];
    int splits;
    int64_t stride;               // floats from cut to cut
    Rows out[2];
    const int* start;
    int64_t tokens;
    int batch, heads, dim;
};

template <bool BF>
__global__ void __launch_bounds__(256) attn_sum_kernel(SumArgs a) {
    const int quads = a.dim / 4;
    const Rows out = a.out[blockIdx.y];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.tokens * a.heads * quads;
         i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / quads, tok = row / a.heads;
        const int quad = (int)(i % quads), head = (int)(row % a.heads);
        // rows behind the last sequence have no partial sums
        if (tok < a.start[0] || tok >= a.start[a.batch]) continue;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        const float* p = a.part[blockIdx.y] + row * a.dim + quad * 4;
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s, p += a.stride) {
            const float4 x = *reinterpret_cast<const float4*>(p);
            y = make_float4(y.x + x.x, y.y + x.y, y.z + x.z, y.w + x.w);
        }
        *reinterpret_cast<uintx2*>(out.p + tok * out.row + head * out.head + quad * 8) =
            uintx2{pack16<BF>(y.x, y.y), pack16<BF>(y.z, y.w)};
    }
}

template <bool BF>
void sum(const SumArgs& x, int outputs, hipStream_t s) {
    const dim3 grid(stride_grid(ceil_div(x.tokens * x.heads * (x.dim / 4), 256), 256), outputs);
    if (grid.x) hipLaunchKernelGGL(attn_sum_kernel<BF>, grid, dim3(256), 0, s, x);
}

template <bool BF, int DP>
void launch(const AttnArgs& a, hipStream_t s) {
    const dim3 rows((unsigned)(attn_groups(a.kv_heads, a.tokens_q * a.group, kRowTile, a.batch) * a.key_splits));
    const dim3 keys((unsigned)(attn_groups(a.kv_heads, a.tokens_k, kKeyRange, a.batch) * a.row_splits));
    hipLaunchKernelGGL((attn_dq_kernel<BF, DP>), rows, dim3(256), 0, s, a);
    if (a.key_splits > 1)
        sum<BF>({{a.part_q, nullptr}, a.key_splits, a.tokens_q * a.heads * a.dim, {a.dq, {}}, a.start_q,
                 a.tokens_q, a.batch, a.heads, a.dim}, 1, s);
    hipLaunchKernelGGL((attn_dkv_kernel<BF, DP>), keys, dim3(512), 0, s, a);
    if (a.row_splits > 1) {
        const int64_t size = a.tokens_k * a.kv_heads * a.dim;
        sum<BF>({{a.part_kv, a.part_kv + size}, a.row_splits, 2 * size, {a.dv, a.dk}, a.start_k,
                 a.tokens_k, a.batch, a.kv_heads, a.dim}, 2, s);
    }
}

}  // namespace

// Cuts of the rows, where ranges of 128 keys alone leave the device's 256
// workgroups idle: at least 4 tiles of rows each (all gradients, 8 heads of 128,
// 512 rows over 64 keys: 31 us uncut, 23.2 like this, 22.6 from 2 tiles on, 26.5
// from 8; 32 heads over 8, 256 rows and keys: 60, 44, 47, 44).
int attn_row_splits(int64_t batch, int64_t tokens_q, int64_t tokens_k, int64_t heads, int64_t kv_heads) {
    const int64_t sequences = std::max<int64_t>(std::min(batch, tokens_k), 1);
    const int64_t groups = kv_heads * std::max(sequences, ceil_div(tokens_k, kKeyRange));
    const int64_t tiles = ceil_div(tokens_q * (heads / kv_heads), sequences * kStepRows);
    return (int)std::max<int64_t>(
        1, std::min({256 / groups, tiles / 4, int64_t(32),
                     kMaxGroups / 2 / attn_groups(kv_heads, tokens_k, kKeyRange, batch)}));
}

// Cuts of the keys, where tiles of 128 rows alone leave its 512 slots idle: at
// least 512 keys each (all gradients, 8 heads of 128, 64 rows over 4096 keys: 126
// us uncut, 38 like this, 34 from 256 keys on, 51 from 1024; 512 rows over 8192
// keys: 283, 100, 98, 102).
int attn_key_splits(int64_t batch, int64_t tokens_q, int64_t tokens_k, int64_t heads, int64_t kv_heads) {
    const int64_t sequences = std::max<int64_t>(std::min(batch, tokens_q), 1);
    const int64_t rows = tokens_q * (heads / kv_heads);
    const int64_t groups = kv_heads * std::max(sequences, ceil_div(rows, kRowTile));
    return (int)std::max<int64_t>(
        1, std::min({512 / groups, ceil_div(tokens_k, sequences) / 512, int64_t(32),
                     kMaxGroups / attn_groups(kv_heads, rows, kRowTile, batch)}));
}

hipError_t attn_backward_launch(const AttnArgs& a, bool bf, hipStream_t s) {
    if (bf) {
        if (a.dim > 96) launch<true, 128>(a, s);
        else if (a.dim > 64) launch<true, 96>(a, s);
        else launch<true, 64>(a, s);
    } else {
        if (a.dim > 96) launch<false, 128>(a, s);
        else if (a.dim > 64) launch<false, 96>(a, s);
        else launch<false, 64>(a, s);
    }
    return hipGetLastError();
}

}  // namespace ep
