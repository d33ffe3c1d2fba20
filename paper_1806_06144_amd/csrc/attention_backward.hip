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
constexpr int kStepRows = 64;         // rows of a tile (dk, dv)
constexpr int kKeyRange = 128;        // keys of a workgroup (dk, dv): 32 per wave

template <bool BF, int DP>
__global__ void __launch_bounds__(256, 2) attn_dq_kernel(AttnArgs a) {
    constexpr int kQuads = DP / 8;
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    constexpr int kLoads = kKeyTile * kQuads / 256;
    __shared__ uintx4 kt[kKeyTile * kQuads];
    __shared__ uintx4 vt[kKeyTile * kQuads];

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
    if (mine && half == 0) a.delta[at * a.heads + head] = delta;
    const float lse2 = a.lse[at * a.heads + head] * kLog2e;

    const int w0 = min(r0 + wave * 32, s.rows - 1), w1 = min(r0 + wave * 32 + 31, s.rows - 1);
    const bool active = r0 + wave * 32 < s.rows;
    const int t0 = row_token(a, w0), t1 = row_token(a, w1);
    const int w_lo = key_lo(a, s, t0), w_hi = key_hi(a, s, t1);
    const int all_lo = key_lo(a, s, t1), all_hi = key_hi(a, s, t0);
    const int begin = key_lo(a, s, row_token(a, r0)) / kKeyTile * kKeyTile;
    const int end = key_hi(a, s, row_token(a, r1));

    floatx16 acc[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;

    const int last_quad = a.dim / 8 - 1;
    for (int j0 = begin; j0 < end; j0 += kKeyTile) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at_quad = tid + 256 * i;
            const int r = at_quad / kQuads;
            const int quad = min((at_quad % kQuads) ^ swizzle<kQuads>(r), last_quad);
            const int64_t j = s.k0 + min(j0 + r, s.m - 1);
            kt[at_quad] = *reinterpret_cast<const uintx4*>(a.k.p + j * a.k.row + kvh * a.k.head + quad * 16);
            vt[at_quad] = *reinterpret_cast<const uintx4*>(a.v.p + j * a.v.row + kvh * a.v.head + quad * 16);
        }
        __syncthreads();
        if (!active || j0 >= w_hi || j0 + kKeyTile <= w_lo) continue;
        const bool masked = j0 < all_lo || j0 + kKeyTile > all_hi;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            floatx16 sc, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                sc = mfma16<BF>(tile_rows<kQuads>(kt, 32 * b, i, lane), qf[i], sc);
                dp = mfma16<BF>(tile_rows<kQuads>(vt, 32 * b, i, lane), gf[i], dp);
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = j0 + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3);
                    if (j < lo || j >= hi) sc[i] = -__builtin_inff();
                }
            }
            uintx4 df[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                // (a row that sees nothing has no unmasked entry)
                float x = __builtin_amdgcn_exp2f(fmaf(sc[i], a.scale_log2, -lse2));
                float y = __builtin_amdgcn_exp2f(fmaf(sc[i + 1], a.scale_log2, -lse2));
                if (masked) {
                    x = sc[i] == -__builtin_inff() ? 0.f : x;
                    y = sc[i + 1] == -__builtin_inff() ? 0.f : y;
                }
                df[i >> 3][(i & 7) >> 1] = pack16<BF>(x * (dp[i] - delta), y * (dp[i + 1] - delta));
            }
#pragma unroll
            for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    acc[c] = mfma16<BF>(tile_columns<kQuads>(kt, 32 * b + 16 * i, c, lane), df[i], acc[c]);
        }
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
__global__ void __launch_bounds__(256, 2) attn_dkv_kernel(AttnArgs a) {
    constexpr int kQuads = DP / 8;
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    constexpr int kLoads = kStepRows * kQuads / 256;
    __shared__ uintx4 qt[kStepRows * kQuads];
    __shared__ uintx4 gt[kStepRows * kQuads];
    __shared__ float4 s_lse[kStepRows / 4];
    __shared__ float4 s_delta[kStepRows / 4];

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
    const bool active = k0 + wave * 32 < s.m;
    const int w_lo = from_row(wk0), w_hi = to_row(wk1);
    const int all_lo = from_row(wk1), all_hi = to_row(wk0);
    const int begin = from_row(k0) / kStepRows * kStepRows, end = to_row(k1);

    floatx16 dk[kBlocks], dv[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[b][i] = dv[b][i] = 0.f;

    const int last_quad = a.dim / 8 - 1;
    for (int i0 = begin; i0 < end; i0 += kStepRows) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at_quad = tid + 256 * i;
            const int r = at_quad / kQuads;
            const int quad = min((at_quad % kQuads) ^ swizzle<kQuads>(r), last_quad);
            const int row = min(i0 + r, s.rows - 1);
            const int tok = row_token(a, row);
            const int head = kvh * a.group + (row - tok * a.group);
            const int64_t q = s.q0 + tok;
            qt[at_quad] = *reinterpret_cast<const uintx4*>(a.q.p + q * a.q.row + head * a.q.head + quad * 16);
            gt[at_quad] = *reinterpret_cast<const uintx4*>(a.dout.p + q * a.dout.row + head * a.dout.head + quad * 16);
        }
        if (tid < kStepRows) {
            const int row = min(i0 + tid, s.rows - 1);
            const int tok = row_token(a, row);
            const int64_t q = (s.q0 + tok) * (int64_t)a.heads + kvh * a.group + (row - tok * a.group);
            reinterpret_cast<float*>(s_lse)[tid] = a.lse[q] * kLog2e;
            reinterpret_cast<float*>(s_delta)[tid] = a.delta[q];
        }
        __syncthreads();
        if (!active || i0 >= w_hi || i0 + kStepRows <= w_lo) continue;
        // (rows past the last are rows that see nothing)
        const bool masked = i0 < all_lo || i0 + kStepRows > min(all_hi, s.rows);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            floatx16 sc, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                sc = mfma16<BF>(tile_rows<kQuads>(qt, 32 * b, i, lane), kf[i], sc);
                dp = mfma16<BF>(tile_rows<kQuads>(gt, 32 * b, i, lane), vf[i], dp);
            }
            uintx4 pf[2], df[2];
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float4 l4 = s_lse[8 * b + 2 * (i >> 2) + half];
                const float4 d4 = s_delta[8 * b + 2 * (i >> 2) + half];
                const float l[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
                float p[4], ds[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(sc[i + e], a.scale_log2, -l[e]));
                    if (masked) {
                        const int r = i0 + 32 * b + 2 * i + 4 * half + e;
                        p[e] = r >= lo && r < hi && r < s.rows ? p[e] : 0.f;
                    }
                    ds[e] = p[e] * (dp[i + e] - dl[e]);
                }
                pf[i >> 3][(i & 7) >> 1] = pack16<BF>(p[0], p[1]);
                pf[i >> 3][((i & 7) >> 1) + 1] = pack16<BF>(p[2], p[3]);
                df[i >> 3][(i & 7) >> 1] = pack16<BF>(ds[0], ds[1]);
                df[i >> 3][((i & 7) >> 1) + 1] = pack16<BF>(ds[2], ds[3]);
            }
#pragma unroll
            for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    dv[c] = mfma16<BF>(tile_columns<kQuads>(gt, 32 * b + 16 * i, c, lane), pf[i], dv[c]);
                    dk[c] = mfma16<BF>(tile_columns<kQuads>(qt, 32 * b + 16 * i, c, lane), df[i], dk[c]);
                }
        }
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
