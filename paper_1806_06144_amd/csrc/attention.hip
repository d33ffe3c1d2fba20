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
// order in which a lane holds its keys (tile_columns).
//
// Scores, maximum, sum and output accumulate in float32. The probabilities
// are rounded to 16 bits for the second product (relative 2^-9 in bf16, as
// much as the output's own rounding); their sum is taken before that.
#include "attn.h"
#include "ep_internal.h"

namespace ep {

namespace {

constexpr int kKeys = 64;             // keys of a tile

template <bool BF, int DP, int SOURCE>
__global__ void __launch_bounds__(256, 2) attn_kernel(AttnArgs a) {
    constexpr int kQuads = DP / 8;
    constexpr int kSteps = DP / 16;
    constexpr int kBlocks = DP / 32;
    constexpr int kLoads = kKeys * kQuads / 256;
    __shared__ uintx4 kt[kKeys * kQuads];
    __shared__ uintx4 vt[kKeys * kQuads];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5;
    int kvh, tile, tiles, first;
    head_and_tile(a.kv_heads, kvh, tile, tiles);
    tile = tiles - 1 - tile;                         // long causal tiles first
    Seq s;
    seq_bounds<SOURCE>(a, find_seq(a.start_q, a.tokens_q, a.batch, a.group, kRowTile, tile, first), s);
    const int r0 = (tile - first) * kRowTile;
    if (r0 < 0 || r0 >= s.rows) return;
    const int r1 = min(r0 + kRowTile, s.rows) - 1;   // the last row

    // this lane's row
    const int row = min(r0 + wave * 32 + (lane & 31), s.rows - 1);
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
    // the wave's and the workgroup's ranges of keys
    const int w0 = min(r0 + wave * 32, s.rows - 1), w1 = min(r0 + wave * 32 + 31, s.rows - 1);
    const bool active = r0 + wave * 32 < s.rows;
    const int t0 = row_token(a, w0), t1 = row_token(a, w1);
    const int w_lo = key_lo(a, s, t0), w_hi = key_hi(a, s, t1);          // any row sees
    const int all_lo = key_lo(a, s, t1), all_hi = key_hi(a, s, t0);      // every row sees
    const int begin = key_lo(a, s, row_token(a, r0)) / kKeys * kKeys;
    const int end = key_hi(a, s, row_token(a, r1));

    floatx16 acc[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
    float top = -3.0e38f, sum = 0.f;                 // (top: in units of log 2)

    const int last_quad = a.dim / 8 - 1;
    for (int j0 = begin; j0 < end; j0 += kKeys) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at_quad = tid + 256 * i;
            const int r = at_quad / kQuads;
            const int quad = min((at_quad % kQuads) ^ swizzle<kQuads>(r), last_quad);
            const int j = min(j0 + r, s.m - 1);
            if constexpr (SOURCE == kPacked) {
                const int64_t row = s.k0 + j;
                kt[at_quad] = *reinterpret_cast<const uintx4*>(a.k.p + row * a.k.row + kvh * a.k.head + quad * 16);
                vt[at_quad] = *reinterpret_cast<const uintx4*>(a.v.p + row * a.v.row + kvh * a.v.head + quad * 16);
            } else {
                const int64_t row = page_row(a.table, a.cols, s.b, a.pages, a.page_shift, a.err, j);
                if constexpr (SOURCE == kPaged) {
                    kt[at_quad] = *reinterpret_cast<const uintx4*>(a.k.p + row * a.k.row + kvh * a.k.head + quad * 16);
                    vt[at_quad] = *reinterpret_cast<const uintx4*>(a.v.p + row * a.v.row + kvh * a.v.head + quad * 16);
                } else {
                    const int64_t sc = row * a.kv_heads + kvh;
                    kt[at_quad] = widen8<BF>(*reinterpret_cast<const uintx2*>(a.k.p + row * a.k.row + kvh * a.k.head + quad * 8), a.k_scale[sc]);
                    vt[at_quad] = widen8<BF>(*reinterpret_cast<const uintx2*>(a.v.p + row * a.v.row + kvh * a.v.head + quad * 8), a.v_scale[sc]);
                }
            }
        }
        __syncthreads();
        if (!active || j0 >= w_hi || j0 + kKeys <= w_lo) continue;
        floatx16 sc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                sc[b] = mfma16<BF>(tile_rows<kQuads>(kt, 32 * b, i, lane), qf[i], sc[b]);
        }
        if (j0 < all_lo || j0 + kKeys > all_hi) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = j0 + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3);
                    if (j < lo || j >= hi) sc[b][i] = -__builtin_inff();
                }
        }
        float mx = sc[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[b][i]);
        mx = pair_max(mx) * a.scale_log2;
        const float now = fmaxf(top, mx);
        const float shrink = __builtin_amdgcn_exp2f(top - now);
        top = now;
        sum *= shrink;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[b][i] *= shrink;
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
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                acc[b] = mfma16<BF>(tile_columns<kQuads>(vt, 16 * i, b, lane), pf[i], acc[b]);
    }
    if (r0 + wave * 32 + (lane & 31) >= s.rows) return;
    sum = pair_sum(sum);
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
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
    if (a.lse && half == 0)
        a.lse[at * a.heads + head] =
            sum == 0.f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <bool BF, int SOURCE>
void launch(const AttnArgs& a, dim3 grid, hipStream_t s) {
    if (a.dim > 64) hipLaunchKernelGGL((attn_kernel<BF, 128, SOURCE>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_kernel<BF, 64, SOURCE>), grid, dim3(256), 0, s, a);
}

}  // namespace

hipError_t attn_forward_launch(const AttnArgs& a, bool bf, int source, hipStream_t s) {
    const dim3 grid((unsigned)attn_groups(a.kv_heads, a.tokens_q * a.group, kRowTile, a.batch));
    switch (source * 2 + (bf ? 1 : 0)) {
    case 0: launch<false, kPacked>(a, grid, s); break;
    case 1: launch<true, kPacked>(a, grid, s); break;
    case 2: launch<false, kPaged>(a, grid, s); break;
    case 3: launch<true, kPaged>(a, grid, s); break;
    case 4: launch<false, kPaged8>(a, grid, s); break;
    default: launch<true, kPaged8>(a, grid, s); break;
    }
    return hipGetLastError();
}

}  // namespace ep
