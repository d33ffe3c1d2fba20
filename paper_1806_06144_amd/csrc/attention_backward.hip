// Gradients of attention (attention.hip): with p_ij = exp(scale q_i.k_j -
// lse_i) formed again from the stored log-sums, D_i = out_i.dout_i and
// ds_ij = p_ij (dout_i.v_j - D_i),
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,
//   dv_j = sum_i p_ij dout_i,
// the sums over i running over the heads of a group too.
//
// Two kernels, each owning what it sums, so there are no atomics and the
// results do not depend on the order of the workgroups: dq walks the keys as
// the forward pass does (three products a tile), dk and dv walk the rows
// (four). Sharing the two products that both form would take five instead of
// seven, but needs dq summed over workgroups in float32 memory.
//
// Scores, probabilities and sums are float32; p and ds are rounded to the
// inputs' type for their products, as the probabilities of the forward pass.
#include "attn.h"
#include "ep_internal.h"

namespace ep {

namespace {

constexpr int kKeyTile = 64;          // keys of a tile (dq)
#ifndef SBM
#define SBM 1
#endif
#define SB(m) if constexpr ((SBM & (m)) != 0) __builtin_amdgcn_sched_barrier(0)
#ifndef DKVOCC
#define DKVOCC 1
#endif
constexpr int kStepRows = 64;         // rows of a tile (dk, dv)
constexpr int kKeyRange = 128;        // keys of a workgroup (dk, dv): 32 per wave

template <bool BF, int DP>
__global__ void __launch_bounds__(256, 2) attn_dq_kernel(AttnArgs a) {
    constexpr int kQuads = DP / 8;
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    __shared__ uintx4 kt0[kKeyTile * kQuads];
    __shared__ uintx4 kt1[kKeyTile * kQuads];
    __shared__ uintx4 vt0[kKeyTile * kQuads];
    __shared__ uintx4 vt1[kKeyTile * kQuads];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5;
    int kvh, tile, tiles, first;
    head_and_tile(a.kv_heads, kvh, tile, tiles);
    tile = tiles - 1 - tile;                         // long causal tiles first
    Seq s;
    seq_bounds<kPacked>(a, find_seq(a.start_q, a.tokens_q, a.batch, a.group, kRowTile, tile, first), s);
    const int r0 = (tile - first) * kRowTile;
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
    const int begin = key_lo(a, s, row_token(a, r0)) / kKeyTile * kKeyTile;
    const int end = key_hi(a, s, row_token(a, r1));

    const TileLoader<kQuads> l(lane, a.dim);
    TileReader<kQuads> rd(lane);
    auto fetch = [&](int j0, uintx4* kt, uintx4* vt) {
        const int j = min(j0 + kWaveRows * wave, s.m - 1);
        const int to = kWaveRows * kQuads * wave;
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
            const uintx4 o = d < a.dim ? *reinterpret_cast<const uintx4*>(op + 2 * d) : zero;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                delta = fmaf(lo16<BF>(o[e]), lo16<BF>(gf[i][e]), delta);
                delta = fmaf(hi16<BF>(o[e]), hi16<BF>(gf[i][e]), delta);
            }
        }
        delta = pair_sum(delta);
    }
    const bool mine = r0 + wave * 32 + (lane & 31) < s.rows;
    const float lse2 = a.lse[at * a.heads + head] * kLog2e;
    if (mine && half == 0) {
        a.lse2[at * a.heads + head] = lse2;
        a.delta[at * a.heads + head] = delta;
    }

    floatx16 acc[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;

    // One tile, in kt and vt; the next goes into kn and vn.
    auto step = [&](int j0, const uintx4* kt, const uintx4* vt, uintx4* kn, uintx4* vn) {
        wg_barrier<0>();                             // kt and vt are there, kn and vn free
        rd.fresh();
        if (j0 + kKeyTile < end) fetch(j0 + kKeyTile, kn, vn);
        const bool masked = j0 < all_lo || j0 + kKeyTile > all_hi;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            SB(1);
            floatx16 sc, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                sc = mfma16<BF>(rd.rows(kt, 32 * b, i), qf[i], sc);
                dp = mfma16<BF>(rd.rows(vt, 32 * b, i), gf[i], dp);
            }
            SB(2);
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.scale_log2, -lse2));
            if (masked) {                            // (a row that sees nothing has lse = -inf)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = j0 + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3);
                    p[i] = j >= lo && j < hi ? p[i] : 0.f;
                }
            }
            uintx4 df[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2)
                df[i >> 3][(i & 7) >> 1] =
                    pack16<BF>(p[i] * (dp[i] - delta), p[i + 1] * (dp[i + 1] - delta));
            SB(4);
#pragma unroll
            for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    acc[c] = mfma16<BF>(rd.columns(kt, 32 * b + 16 * i, c), df[i], acc[c]);
        }
    };
    for (int j0 = begin; j0 < end; j0 += 2 * kKeyTile) {
        step(j0, kt0, vt0, kt1, vt1);
        if (j0 + kKeyTile < end) step(j0 + kKeyTile, kt1, vt1, kt0, vt0);
    }
    if (!mine) return;
    char* out = a.dq.p + at * a.dq.row + head * a.dq.head;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + 2 * i + 4 * half;
            if (d < a.dim)
                *reinterpret_cast<uintx2*>(out + 2 * d) =
                    uintx2{pack16<BF>(acc[b][i] * a.scale, acc[b][i + 1] * a.scale),
                           pack16<BF>(acc[b][i + 2] * a.scale, acc[b][i + 3] * a.scale)};
        }
}

// A wave owns 32 keys, whose rows of K and V stay in its registers as right
// operands. S = Q K^T and dP = dout V^T leave a lane 16 rows of ONE key, the
// order in which dv^T += dout^T P and dk^T += Q^T dS take them.
template <bool BF, int DP>
__global__ void __launch_bounds__(256, DP == 64 ? 2 : DKVOCC) attn_dkv_kernel(AttnArgs a) {
    constexpr int kQuads = DP / 8;
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    __shared__ uintx4 qt0[kStepRows * kQuads];
    __shared__ uintx4 qt1[kStepRows * kQuads];
    __shared__ uintx4 gt0[kStepRows * kQuads];
    __shared__ uintx4 gt1[kStepRows * kQuads];
    __shared__ float4 s_row0[2][kStepRows / 4];      // lse2, delta
    __shared__ float4 s_row1[2][kStepRows / 4];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5;
    int kvh, tile, tiles, first;
    head_and_tile(a.kv_heads, kvh, tile, tiles);     // (early keys have the most rows)
    Seq s;
    seq_bounds<kPacked>(a, find_seq(a.start_k, a.tokens_k, a.batch, 1, kKeyRange, tile, first), s);
    const int k0 = (tile - first) * kKeyRange;
    if (k0 < 0 || k0 >= s.m) return;
    const int k1 = min(k0 + kKeyRange, s.m) - 1;

    const int key = min(k0 + wave * 32 + (lane & 31), s.m - 1);
    const int64_t at = s.k0 + key;
    uintx4 kf[kSteps], vf[kSteps];
    {
        const char* kp = a.k.p + at * a.k.row + kvh * a.k.head;
        const char* vp = a.v.p + at * a.v.row + kvh * a.v.head;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int d = 16 * i + 8 * half;
            const uintx4 zero = {0, 0, 0, 0};
            kf[i] = d < a.dim ? *reinterpret_cast<const uintx4*>(kp + 2 * d) : zero;
            vf[i] = d < a.dim ? *reinterpret_cast<const uintx4*>(vp + 2 * d) : zero;
        }
    }
    auto from_row = [&](int j) { return seen_from(j, s.off, s.n, a.group, a.causal); };
    auto to_row = [&](int j) { return seen_to(j, s.off, s.n, a.group, a.window); };
    const int lo = from_row(key), hi = to_row(key);
    const int wk0 = min(k0 + wave * 32, s.m - 1), wk1 = min(k0 + wave * 32 + 31, s.m - 1);
    // (rows past the last are rows that see nothing)
    const int all_lo = from_row(wk1), all_hi = min(to_row(wk0), s.rows);
    const int begin = from_row(k0) / kStepRows * kStepRows, end = to_row(k1);

    const TileLoader<kQuads> l(lane, a.dim);
    TileReader<kQuads> rd(lane);
    auto fetch = [&](int i0, uintx4* qt, uintx4* gt, float4 (*rows)[kStepRows / 4]) {
        // the tile's first row is (tok0, rem0); a lane's rows follow it
        const int tok0 = row_token(a, i0), rem0 = i0 - tok0 * a.group;
        const int to = kWaveRows * kQuads * wave;
        const char* qp = a.q.p + (int64_t)(s.q0 + tok0) * a.q.row + kvh * a.group * a.q.head;
        const char* gp = a.dout.p + (int64_t)(s.q0 + tok0) * a.dout.row + kvh * a.group * a.dout.head;
        const int last = s.rows - 1 - i0;
#pragma unroll
        for (int i = 0; i < l.kLoads; ++i) {
            const int r = rem0 + min(kWaveRows * wave + l.row(i), last);
            const unsigned t = row_token(a, r), h = r - t * a.group;
            load_lds16(qp + (t * (uint64_t)a.q.row + h * (uint64_t)a.q.head) + l.quad(i), qt + to + 64 * i);
            load_lds16(gp + (t * (uint64_t)a.dout.row + h * (uint64_t)a.dout.head) + l.quad(i), gt + to + 64 * i);
        }
        if (wave < 2) {
            const int r = rem0 + min(lane, last);
            const unsigned t = row_token(a, r), h = r - t * a.group;
            const float* p = (wave == 0 ? a.lse2 : a.delta) + (s.q0 + tok0 + (int64_t)t) * a.heads +
                             kvh * a.group + h;
            load_lds4(p, reinterpret_cast<float*>(rows[wave]));
        }
    };
    if (begin < end) fetch(begin, qt0, gt0, s_row0);

    floatx16 dk[kBlocks], dv[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[b][i] = dv[b][i] = 0.f;

    // One tile of rows, in qt and gt; the next goes into qn and gn.
    auto step = [&](int i0, const uintx4* qt, const uintx4* gt, const float4 (*rows)[kStepRows / 4],
                    uintx4* qn, uintx4* gn, float4 (*rn)[kStepRows / 4]) {
        wg_barrier<0>();                             // qt and gt are there, qn and gn free
        rd.fresh();
        if (i0 + kStepRows < end) fetch(i0 + kStepRows, qn, gn, rn);
        const bool masked = i0 < all_lo || i0 + kStepRows > all_hi;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            SB(1);
            floatx16 sc, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                sc = mfma16<BF>(rd.rows(qt, 32 * b, i), kf[i], sc);
                dp = mfma16<BF>(rd.rows(gt, 32 * b, i), vf[i], dp);
            }
            SB(2);
            float p[16], ds[16];
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float4 l4 = rows[0][8 * b + 2 * (i >> 2) + half];
                p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.scale_log2, -l4.x));
                p[i + 1] = __builtin_amdgcn_exp2f(fmaf(sc[i + 1], a.scale_log2, -l4.y));
                p[i + 2] = __builtin_amdgcn_exp2f(fmaf(sc[i + 2], a.scale_log2, -l4.z));
                p[i + 3] = __builtin_amdgcn_exp2f(fmaf(sc[i + 3], a.scale_log2, -l4.w));
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = i0 + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3);
                    p[i] = r >= lo && r < hi && r < s.rows ? p[i] : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float4 d4 = rows[1][8 * b + 2 * (i >> 2) + half];
                ds[i] = p[i] * (dp[i] - d4.x);
                ds[i + 1] = p[i + 1] * (dp[i + 1] - d4.y);
                ds[i + 2] = p[i + 2] * (dp[i + 2] - d4.z);
                ds[i + 3] = p[i + 3] * (dp[i + 3] - d4.w);
            }
            uintx4 pf[2], df[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                pf[i >> 3][(i & 7) >> 1] = pack16<BF>(p[i], p[i + 1]);
                df[i >> 3][(i & 7) >> 1] = pack16<BF>(ds[i], ds[i + 1]);
            }
            SB(4);
#pragma unroll
            for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    dv[c] = mfma16<BF>(rd.columns(gt, 32 * b + 16 * i, c), pf[i], dv[c]);
                    dk[c] = mfma16<BF>(rd.columns(qt, 32 * b + 16 * i, c), df[i], dk[c]);
                }
        }
    };
    for (int i0 = begin; i0 < end; i0 += 2 * kStepRows) {
        step(i0, qt0, gt0, s_row0, qt1, gt1, s_row1);
        if (i0 + kStepRows < end) step(i0 + kStepRows, qt1, gt1, s_row1, qt0, gt0, s_row0);
    }
    if (k0 + wave * 32 + (lane & 31) >= s.m) return;
    char* kp = a.dk.p + at * a.dk.row + kvh * a.dk.head;
    char* vp = a.dv.p + at * a.dv.row + kvh * a.dv.head;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + 2 * i + 4 * half;
            if (d < a.dim) {
                *reinterpret_cast<uintx2*>(kp + 2 * d) =
                    uintx2{pack16<BF>(dk[b][i] * a.scale, dk[b][i + 1] * a.scale),
                           pack16<BF>(dk[b][i + 2] * a.scale, dk[b][i + 3] * a.scale)};
                *reinterpret_cast<uintx2*>(vp + 2 * d) =
                    uintx2{pack16<BF>(dv[b][i], dv[b][i + 1]), pack16<BF>(dv[b][i + 2], dv[b][i + 3])};
            }
        }
}

template <bool BF, int DP>
void launch(const AttnArgs& a, hipStream_t s) {
    const dim3 rows((unsigned)attn_groups(a.kv_heads, a.tokens_q * a.group, kRowTile, a.batch));
    const dim3 keys((unsigned)attn_groups(a.kv_heads, a.tokens_k, kKeyRange, a.batch));
    hipLaunchKernelGGL((attn_dq_kernel<BF, DP>), rows, dim3(256), 0, s, a);
    hipLaunchKernelGGL((attn_dkv_kernel<BF, DP>), keys, dim3(256), 0, s, a);
}

}  // namespace

hipError_t attn_backward_launch(const AttnArgs& a, bool bf, hipStream_t s) {
    if (a.dim > 64) {
        if (bf) launch<true, 128>(a, s);
        else launch<false, 128>(a, s);
    } else {
        if (bf) launch<true, 64>(a, s);
        else launch<false, 64>(a, s);
    }
    return hipGetLastError();
}

}  // namespace ep
