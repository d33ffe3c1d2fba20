// A paged cache of keys and values: writing a sequence's new tokens into its
// pages, with or without rounding to 8 bits, and reading tokens back.
//
// An 8-bit row (one token, one key head) is e4m3 numbers times one power of
// two, 2^e with the smallest e that brings the row's largest finite value
// within 448. Dividing by a power of two is exact, so a value is rounded
// once (to nearest, at most 2^-4 of it above 2^(e-6)); multiplying back is
// exact in bf16 and fp16 alike, so attention reads the very values that a
// read back gives. A scale of amax / 448 would use up to twice the range but
// round twice and cost a multiplication per score and probability.
// Such scales, set elsewhere, are read as they are: widen8 (attn.h) multiplies
// in float32 and rounds.
// Values above 1.875 times the largest power of two of the type are stored as
// that (they would round up to a number the type does not have); infinities
// and NaN are stored as NaN.
//
// Both kernels are bound by memory: a row is held by a group of 16 (8 for
// dim <= 64) lanes, 16 bytes a lane, and a group takes up to four heads at once.
// e4m3 pages of 8 heads of 128: 9087 tokens in 17 us (3.3 TB/s), 40647 back in
// 43 (5.9 TB/s; 61 a head at a time).
#include "attn.h"
#include "ep_internal.h"
#include "launch.h"

#include <type_traits>

namespace ep {

namespace {

// The sequence of packed row t, and whether t belongs to one.
__device__ __forceinline__ int seq_of(const int* start, int batch, int t) {
    int lo = 0, hi = batch;                          // start[lo] <= t < start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= t) lo = mid;
        else hi = mid;
    }
    return t >= start[lo] && t < start[lo + 1] ? lo : -1;
}

template <bool BF, int LANES>
__device__ __forceinline__ uintx2 narrow8(uintx4 x, float& scale) {
    constexpr float kTop = BF ? 0x1.ep127f : 0x1.ep15f;
    constexpr int kLow = BF ? -110 : -15;
    float v[8], most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = lo16<BF>(x[i]);
        v[2 * i + 1] = hi16<BF>(x[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool finite = __builtin_isfinite(v[i]);
        v[i] = finite ? fminf(fmaxf(v[i], -kTop), kTop) : __builtin_nanf("");
        most = fmaxf(most, finite ? fabsf(v[i]) : 0.f);
    }
#pragma unroll
    for (int i = 1; i < LANES; i *= 2) most = fmaxf(most, __shfl_xor(most, i));
    // most = f 2^x, f in [1/2, 1): 448 = 7/8 2^9
    int x2 = 0;
    const float f = frexpf(most, &x2);
    const int e = max(f <= 0.875f ? x2 - 9 : x2 - 8, kLow);
    scale = most == 0.f ? 1.f : __builtin_bit_cast(float, (e + 127) << 23);
    const float inv = most == 0.f ? 1.f : __builtin_bit_cast(float, (127 - e) << 23);
    uintx2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
        r[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, w, true);
    }
    return r;
}

template <bool BF, bool E4M3, int LANES, int HEADS>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheArgs a) {
    const int chunks = a.kv_heads / HEADS;
    const int64_t rows = a.tokens * chunks;
    const int quad = threadIdx.x % LANES;
    const bool in = quad * 8 < a.dim;
    for (int64_t i = blockIdx.x * (256 / LANES) + threadIdx.x / LANES; i < rows;
         i += (int64_t)gridDim.x * (256 / LANES)) {
        const int t = (int)(i / chunks), h = (int)(i % chunks) * HEADS;
        uintx4 k[HEADS], v[HEADS];
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            k[u] = v[u] = uintx4{0, 0, 0, 0};
            if (in) {
                k[u] = *reinterpret_cast<const uintx4*>(a.k.p + t * a.k.row + (h + u) * a.k.head + quad * 16);
                v[u] = *reinterpret_cast<const uintx4*>(a.v.p + t * a.v.row + (h + u) * a.v.head + quad * 16);
            }
        }
        const int b = seq_of(a.start, a.batch, t);
        if (b < 0) continue;
        // the new tokens are the sequence's last
        int first, count;
        held_range(a.start[b], a.start[b + 1], (int)a.tokens, first, count);
        const int64_t j = (int64_t)a.lengths[b] - (first + count) + t;
        int page = -1;
        if (j >= 0 && j < a.cols << a.page_shift)
            page = page_of(a.table, a.cols, b, a.pages, a.page_shift, j);
        if (page < 0) {
            if (a.err) *a.err = 1;
            continue;
        }
        const int64_t to = page_slot(page, a.page_shift, j) * a.kv_heads + h;
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            if constexpr (E4M3) {
                float ks, vs;
                const uintx2 k8 = narrow8<BF, LANES>(k[u], ks), v8 = narrow8<BF, LANES>(v[u], vs);
                if (in) {
                    *reinterpret_cast<uintx2*>(a.kp + (to + u) * a.dim + quad * 8) = k8;
                    *reinterpret_cast<uintx2*>(a.vp + (to + u) * a.dim + quad * 8) = v8;
                }
                if (quad == 0) {
                    a.ks[to + u] = ks;
                    a.vs[to + u] = vs;
                }
            } else if (in) {
                *reinterpret_cast<uintx4*>(a.kp + (to + u) * a.dim * 2 + quad * 16) = k[u];
                *reinterpret_cast<uintx4*>(a.vp + (to + u) * a.dim * 2 + quad * 16) = v[u];
            }
        }
    }
}

template <bool BF, bool E4M3, int LANES, int HEADS>
__global__ void __launch_bounds__(256) cache_read_kernel(CacheArgs a) {
    const int chunks = a.kv_heads / HEADS;
    const int64_t rows = a.tokens * chunks;
    const int quad = threadIdx.x % LANES;
    if (quad * 8 >= a.dim) return;
    for (int64_t i = blockIdx.x * (256 / LANES) + threadIdx.x / LANES; i < rows;
         i += (int64_t)gridDim.x * (256 / LANES)) {
        const int t = (int)(i / chunks), h = (int)(i % chunks) * HEADS;
        const int b = seq_of(a.start, a.batch, t);
        if (b < 0) continue;
        const int j = t - clamp_i(a.start[b], 0, (int)a.tokens);
        const int length = a.lengths[b], held = held_length(length, a.cols, a.page_shift);
        const int page = j < held ? page_of(a.table, a.cols, b, a.pages, a.page_shift, j) : -1;
        if ((page < 0 || length != held) && a.err) *a.err = 1;
        if (page < 0) continue;
        const int64_t from = page_slot(page, a.page_shift, j) * a.kv_heads + h;
        typedef std::conditional_t<E4M3, uintx2, uintx4> Quad;
        Quad k[HEADS], v[HEADS];
        float ks[HEADS], vs[HEADS];
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            const int64_t at = (from + u) * a.dim / 8 + quad;
            k[u] = reinterpret_cast<const Quad*>(a.kp)[at];
            v[u] = reinterpret_cast<const Quad*>(a.vp)[at];
            if constexpr (E4M3) {
                ks[u] = a.ks[from + u];
                vs[u] = a.vs[from + u];
            }
        }
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            uintx4 x, y;
            if constexpr (E4M3) {
                x = widen8<BF>(k[u], ks[u], power_of_two(ks[u]));
                y = widen8<BF>(v[u], vs[u], power_of_two(vs[u]));
            } else {
                x = k[u];
                y = v[u];
            }
            *reinterpret_cast<uintx4*>(a.k.p + t * a.k.row + (h + u) * a.k.head + quad * 16) = x;
            *reinterpret_cast<uintx4*>(a.v.p + t * a.v.row + (h + u) * a.v.head + quad * 16) = y;
        }
    }
}

template <bool WRITE, bool BF, bool E4M3, int LANES, int HEADS>
void launch_one(const CacheArgs& a, hipStream_t s) {
    const int64_t blocks = ceil_div(a.tokens * (a.kv_heads / HEADS), 256 / LANES);
    const dim3 grid(stride_grid(blocks, 256));
    if constexpr (WRITE)
        hipLaunchKernelGGL((cache_write_kernel<BF, E4M3, LANES, HEADS>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((cache_read_kernel<BF, E4M3, LANES, HEADS>), grid, dim3(256), 0, s, a);
}

// Heads a group of lanes takes at once: their loads are on the way together
// and share the look-ups of sequence and page.
template <bool WRITE, bool BF, bool E4M3, int LANES>
void launch_lanes(const CacheArgs& a, hipStream_t s) {
    if (a.kv_heads % 4 == 0) launch_one<WRITE, BF, E4M3, LANES, 4>(a, s);
    else if (a.kv_heads % 2 == 0) launch_one<WRITE, BF, E4M3, LANES, 2>(a, s);
    else launch_one<WRITE, BF, E4M3, LANES, 1>(a, s);
}

template <bool WRITE, bool BF, bool E4M3>
void launch(const CacheArgs& a, hipStream_t s) {
    if (a.dim > 64) launch_lanes<WRITE, BF, E4M3, 16>(a, s);
    else launch_lanes<WRITE, BF, E4M3, 8>(a, s);
}

template <bool WRITE>
hipError_t pick(const CacheArgs& a, bool bf, bool e4m3, hipStream_t s) {
    if (bf) {
        if (e4m3) launch<WRITE, true, true>(a, s);
        else launch<WRITE, true, false>(a, s);
    } else {
        if (e4m3) launch<WRITE, false, true>(a, s);
        else launch<WRITE, false, false>(a, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t cache_write_launch(const CacheArgs& a, bool bf, bool e4m3, hipStream_t s) {
    return pick<true>(a, bf, e4m3, s);
}
hipError_t cache_read_launch(const CacheArgs& a, bool bf, bool e4m3, hipStream_t s) {
    return pick<false>(a, bf, e4m3, s);
}

}  // namespace ep
