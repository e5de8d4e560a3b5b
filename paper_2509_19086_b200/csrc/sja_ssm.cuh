// Selective state space scan with its short causal convolution: the recurrent half of a layer that forecasts job
// profiles from their histories.  Per job, token t, channel d of group g and state n:
//
//     row_t   = [x (D) | B (G x N) | C (G x N)],   u_t = silu(conv_b + sum_w conv_w[:, w] row_{t-W+1+w})
//     dt_t    = softplus(raw_t + dt_bias)
//     h_t     = exp(dt_t A[d, n]) h_{t-1} + dt_t u_t[d] B_t[g, n]
//     y_t     = (sum_n C_t[g, n] h_t[d, n] + skip[d] u_t[d]) silu(z_t[d])
//
// Everything between the loads and the stores is 32-bit: the convolved row is never rounded to the input type.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sja_common.cuh"

namespace sja {

constexpr int SSM_MAX_WIDTH = 4;
constexpr int SSM_MAX_STATE = 128;

struct SsmArgs {
    const void *xbc, *dt, *z;
    void* y;
    int64_t xbc_stride, dt_stride, z_stride, y_stride;   // elements between rows
    const float *A, *skip, *dt_bias, *conv_w, *conv_b;
    void* history;                // [n_slots, W - 1, rows] in the input type
    float* state;                 // [n_slots, D, N]
    const int32_t* slots;         // [S] or nullptr (job s keeps slot s)
    const uint64_t* off;          // [S + 1]
    uint64_t T;
    uint32_t S, n_slots, D, N, G, W, rows, resume;
    // split of the token axis (prompts)
    uint32_t n_seg, snap;
    uint64_t seg_len;
    uint32_t* seg_flag;           // [n_seg]
    float *seg_h, *seg_first, *seg_sdt;   // [n_seg, D, N], [n_seg, D, N], [n_seg, D]
};

// What the job across a segment's end did inside the segment.
enum : uint32_t { SEG_NONE = 0, SEG_STARTS = 1, SEG_PASSES = 2 };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float silu(float v) { return __fdividef(v, 1.0f + __expf(-v)); }
// log1p keeps the relative accuracy of small time steps (softplus(v) ~ e^v for very negative v)
__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.0f) + log1pf(__expf(-fabsf(v))); }

__device__ __forceinline__ float exp2_fast(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Two 32-bit values in one 64-bit register pair: one instruction issued for two multiply-adds.
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float a, float b) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void f2_split(F2 p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// First index in off[0 .. n) whose value is >= v (n if none): 32 probes at a time by the whole warp, so that
// 1024 jobs take two dependent loads.
__device__ __forceinline__ uint32_t warp_lower_bound(const uint64_t* __restrict__ off, uint32_t n, uint64_t v) {
    const uint32_t lane = threadIdx.x & 31u;
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t step = (hi - lo + 31u) / 32u;
        const uint64_t i = (uint64_t)lo + (uint64_t)lane * step;
        const bool below = i < hi && off[i] < v;
        const uint32_t c = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, below));
        if (c == 0u) break;
        const uint64_t top = (uint64_t)lo + (uint64_t)c * step;
        lo += (c - 1u) * step + 1u;
        hi = top < hi ? (uint32_t)top : hi;
    }
    return lo;
}

// Boundary k of the token axis: k * seg_len, moved to the nearest start of a job when one is within `snap`
// tokens.  A boundary between two jobs carries nothing over, so loads of jobs shorter than a segment never pay for
// the split.
__device__ __forceinline__ uint64_t segment_bound(const SsmArgs& a, uint32_t k) {
    if (k == 0u) return 0ull;
    if (k >= a.n_seg) return a.T;
    const uint64_t at = (uint64_t)k * a.seg_len;
    const uint32_t j = warp_lower_bound(a.off, a.S + 1u, at);
    uint64_t best = at, dist = (uint64_t)a.snap + 1ull;
    if (j <= a.S) {
        const uint64_t v = a.off[j];
        if (v - at < dist) { best = v; dist = v - at; }
    }
    if (j > 0u) {
        const uint64_t v = a.off[j - 1u];
        if (at - v < dist) best = v;
    }
    return best < a.T ? best : a.T;
}

__device__ __forceinline__ int64_t slot_of(const SsmArgs& a, uint32_t s) {
    const int64_t v = a.slots ? (int64_t)a.slots[s] : (int64_t)s;
    return v >= 0 && v < (int64_t)a.n_slots ? v : -1;     // outside the pool: starts from zero, nothing is kept
}

// Raw row value of column `col` at position `pos` (counted from the job's first token of this call; negative
// positions are the history).
template <typename T>
__device__ __forceinline__ float row_value(const SsmArgs& a, uint64_t first, int64_t pos, uint32_t col, int64_t slot) {
    if (pos >= 0) return to_f32(static_cast<const T*>(a.xbc)[(int64_t)(first + (uint64_t)pos) * a.xbc_stride + col]);
    if (!a.resume || slot < 0) return 0.0f;
    return to_f32(static_cast<const T*>(a.history)[(slot * (int64_t)(a.W - 1u) + (int64_t)(a.W - 1u) + pos) * a.rows + col]);
}

// One column of the short convolution, fed token by token; w[3] meets the newest value.  Taps the layer does not
// have are left out rather than multiplied by zero: an infinite value outside the window must not count.
struct Conv {
    float w[4], b, p1, p2, p3;
    __device__ __forceinline__ void load(const SsmArgs& a, uint32_t col) {
        w[0] = w[1] = w[2] = w[3] = b = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < (int)a.W) w[3 - k] = a.conv_w[(uint64_t)col * a.W + (a.W - 1u - (uint32_t)k)];
        if (a.W && a.conv_b) b = a.conv_b[col];
    }
    template <typename T>
    __device__ __forceinline__ void seek(const SsmArgs& a, uint64_t first, int64_t pos, uint32_t col, int64_t slot) {
        p1 = a.W > 1u ? row_value<T>(a, first, pos - 1, col, slot) : 0.0f;
        p2 = a.W > 2u ? row_value<T>(a, first, pos - 2, col, slot) : 0.0f;
        p3 = a.W > 3u ? row_value<T>(a, first, pos - 3, col, slot) : 0.0f;
    }
    __device__ __forceinline__ float next(uint32_t W, float v) {
        if (W == 0u) return v;
        float s = fmaf(w[3], v, b);
        if (W > 1u) s = fmaf(w[2], p1, s);
        if (W > 2u) s = fmaf(w[1], p2, s);
        if (W > 3u) s = fmaf(w[0], p3, s);
        p3 = p2; p2 = p1; p1 = v;
        return silu(s);
    }
};

__host__ __device__ constexpr int ssm_tile_tokens(int np) { return np <= 32 ? 32 : np <= 64 ? 16 : 8; }

// Prompts.  A thread owns CPT channels and K of their states (LPC lanes share a channel), walks its segment of the
// token axis and keeps the states in registers; B and C of a tile of tokens are convolved once per CTA into shared
// memory and read by broadcast.  CARRY = true is the first pass of a split: what the job that crosses the segment's
// end adds to its state inside the segment, and its sum of time steps (exp(A sum dt) is the decay over the segment).
template <typename T, int K, int LPC, int CPT, bool CARRY>
__global__ void __launch_bounds__(128) ssm_prompt_kernel(const SsmArgs a) {
    constexpr int NP = K * LPC, TT = ssm_tile_tokens(NP), CPW = 32 / LPC, U = 4;
    __shared__ __align__(16) float sB[TT * NP], sC[TT * NP];
    dep_wait();
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    const uint32_t Dg = a.D / a.G, span = (blockDim.x >> 5) * CPW * CPT;
    const uint32_t tiles = (Dg + span - 1u) / span;
    const uint32_t g = blockIdx.x / tiles, seg = blockIdx.y;
    const uint32_t in_group = (blockIdx.x % tiles) * span + warp * (CPW * CPT) + lane / LPC;
    const uint32_t n0 = (lane % LPC) * K;
    uint32_t ch[CPT];
    bool live[CPT];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        live[i] = in_group + i * CPW < Dg;
        ch[i] = g * Dg + (live[i] ? in_group + i * CPW : 0u);
    }
    const uint64_t b0 = segment_bound(a, seg), b1 = segment_bound(a, seg + 1u);
    uint64_t begin = b0;
    uint32_t s;
    if (CARRY) {
        s = warp_lower_bound(a.off, a.S + 1u, b1 + 1ull);
        s = s ? s - 1u : 0u;
        const uint64_t q = a.off[s];
        const uint32_t flag = (s >= a.S || q >= b1) ? SEG_NONE : q >= b0 ? SEG_STARTS : SEG_PASSES;
        if (blockIdx.x == 0u && tid == 0u) a.seg_flag[seg] = flag;
        if (flag == SEG_NONE) return;
        begin = q > b0 ? q : b0;
    } else {
        s = warp_lower_bound(a.off, a.S + 1u, b0 + 1ull);
        s = s ? s - 1u : 0u;
    }

    F2 A2[CPT][K / 2], h[CPT][K / 2];
    Conv cx[CPT];
    float skip[CPT], bias[CPT], sdt[CPT];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        cx[i].load(a, ch[i]);
        skip[i] = a.skip ? a.skip[ch[i]] : 0.0f;
        bias[i] = a.dt_bias ? a.dt_bias[ch[i]] : 0.0f;
        sdt[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < K / 2; ++k) {
            const uint32_t n = n0 + 2 * k;
            const float* r = a.A + (uint64_t)ch[i] * a.N;
            A2[i][k] = f2(n < a.N ? r[n] * 1.44269504f : 0.0f, n + 1u < a.N ? r[n + 1u] * 1.44269504f : 0.0f);
            h[i][k] = f2(0.0f, 0.0f);
        }
    }
    auto load_h = [&](const float* from) {
#pragma unroll
        for (int i = 0; i < CPT; ++i)
#pragma unroll
            for (int k = 0; k < K / 2; ++k) {
                const uint32_t n = n0 + 2 * k;
                const float* r = from + (uint64_t)ch[i] * a.N;
                h[i][k] = f2(n < a.N ? r[n] : 0.0f, n + 1u < a.N ? r[n + 1u] : 0.0f);
            }
    };
    auto store_h = [&](float* to) {
#pragma unroll
        for (int i = 0; i < CPT; ++i)
#pragma unroll
            for (int k = 0; k < K / 2; ++k) {
                const uint32_t n = n0 + 2 * k;
                float* r = to + (uint64_t)ch[i] * a.N;
                float v0, v1;
                f2_split(h[i][k], v0, v1);
                if (live[i] && n < a.N) r[n] = v0;
                if (live[i] && n + 1u < a.N) r[n + 1u] = v1;
            }
    };
    const uint64_t DN = (uint64_t)a.D * a.N;
    const T* xp = static_cast<const T*>(a.xbc);
    const T* dp = static_cast<const T*>(a.dt);
    const T* zp = static_cast<const T*>(a.z);
    T* yp = static_cast<T*>(a.y);

    uint64_t t = begin;
    for (; t < b1 && s < a.S; ++s) {
        const uint64_t q = a.off[s];
        uint64_t e = a.off[s + 1u];
        if (e <= t || q > t) continue;                 // an empty job (or offsets that are not ascending)
        const bool ends = e <= b1;
        if (!ends) e = b1;
        const int64_t slot = slot_of(a, s);
        // where the job's state comes from: the segment before, its slot, or nothing
        if (q < t) {
            if (!CARRY) load_h(a.seg_h + (uint64_t)(seg - 1u) * DN);
        } else if (a.resume && slot >= 0 && a.state) {
            // a job that goes on behind this segment may be stored by another CTA meanwhile: the first pass kept a copy
            if (CARRY || ends || a.n_seg == 1u) load_h(a.state + slot * (int64_t)DN);
            else load_h(a.seg_first + (uint64_t)seg * DN);
            if (CARRY) store_h(a.seg_first + (uint64_t)seg * DN);
        } else {
#pragma unroll
            for (int i = 0; i < CPT; ++i)
#pragma unroll
                for (int k = 0; k < K / 2; ++k) h[i][k] = f2(0.0f, 0.0f);
        }
#pragma unroll
        for (int i = 0; i < CPT; ++i) cx[i].template seek<T>(a, q, (int64_t)(t - q), ch[i], slot);

        while (t < e) {
            const uint32_t n_tok = e - t < (uint64_t)TT ? (uint32_t)(e - t) : (uint32_t)TT;
            __syncthreads();
            // convolve B (and C) of the tile: a thread takes one column and every fourth stretch of tokens
            const uint32_t cols = CARRY ? NP : 2 * NP;
            const uint32_t parts = blockDim.x / cols ? blockDim.x / cols : 1u, per = (n_tok + parts - 1u) / parts;
            for (uint32_t w = tid; w < cols * parts; w += blockDim.x) {
                const uint32_t col = w % cols, from = (w / cols) * per, to = min(from + per, n_tok);
                const uint32_t n = col % NP;
                float* dst = col < NP ? sB : sC;
                if (n >= a.N) {
                    for (uint32_t i = from; i < to; ++i) dst[i * NP + n] = 0.0f;
                } else if (from < to) {
                    const uint32_t rc = a.D + (col < NP ? 0u : a.G * a.N) + g * a.N + n;
                    Conv cv;
                    cv.load(a, rc);
                    cv.template seek<T>(a, q, (int64_t)(t - q) + from, rc, slot);
                    for (uint32_t i = from; i < to; ++i)
                        dst[i * NP + n] = cv.next(a.W, to_f32(xp[(int64_t)(t + i) * a.xbc_stride + rc]));
                }
            }
            __syncthreads();
            for (uint32_t i0 = 0; i0 < n_tok; i0 += U) {
                float xv[U][CPT], dv[U][CPT], zv[U][CPT];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    const uint64_t r = t + min(i0 + j, n_tok - 1u);
#pragma unroll
                    for (int i = 0; i < CPT; ++i) {
                        xv[j][i] = to_f32(xp[(int64_t)r * a.xbc_stride + ch[i]]);
                        dv[j][i] = to_f32(dp[(int64_t)r * a.dt_stride + ch[i]]);
                        zv[j][i] = !CARRY && zp ? to_f32(zp[(int64_t)r * a.z_stride + ch[i]]) : 0.0f;
                    }
                }
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    if (i0 + j >= n_tok) break;
                    F2 d2[CPT], du2[CPT], acc[CPT];
                    float u[CPT];
#pragma unroll
                    for (int i = 0; i < CPT; ++i) {
                        u[i] = cx[i].next(a.W, xv[j][i]);
                        const float d = softplus(dv[j][i] + bias[i]);
                        if (CARRY) sdt[i] += d;
                        d2[i] = f2(d, d);
                        du2[i] = f2(d * u[i], d * u[i]);
                        acc[i] = f2(0.0f, 0.0f);
                    }
                    const ulonglong2* pB = reinterpret_cast<const ulonglong2*>(sB + (i0 + j) * NP + n0);
                    const ulonglong2* pC = reinterpret_cast<const ulonglong2*>(sC + (i0 + j) * NP + n0);
#pragma unroll
                    for (int k = 0; k < K / 4; ++k) {
                        const ulonglong2 bq = pB[k];
                        ulonglong2 cq = {0ull, 0ull};
                        if (!CARRY) cq = pC[k];
                        const F2 b2[2] = {{bq.x}, {bq.y}}, c2[2] = {{cq.x}, {cq.y}};
#pragma unroll
                        for (int i = 0; i < CPT; ++i)
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                float e0, e1;
                                f2_split(f2_mul(d2[i], A2[i][2 * k + m]), e0, e1);
                                const F2 decay = f2(exp2_fast(e0), exp2_fast(e1));
                                F2& hh = h[i][2 * k + m];
                                hh = f2_fma(decay, hh, f2_mul(du2[i], b2[m]));
                                if (!CARRY) acc[i] = f2_fma(hh, c2[m], acc[i]);
                            }
                    }
                    if (!CARRY) {
#pragma unroll
                        for (int i = 0; i < CPT; ++i) {
                            float v0, v1;
                            f2_split(acc[i], v0, v1);
                            float v = v0 + v1;
#pragma unroll
                            for (int m = 1; m < LPC; m *= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
                            v = fmaf(skip[i], u[i], v);
                            if (zp) v *= silu(zv[j][i]);
                            if (live[i] && (lane % LPC) == (uint32_t)(i % LPC))
                                yp[(int64_t)(t + i0 + j) * a.y_stride + ch[i]] = from_f32<T>(v);
                        }
                    }
                }
            }
            t += n_tok;
        }
        if (!CARRY && ends && slot >= 0 && a.state) store_h(a.state + slot * (int64_t)DN);
    }
    if (CARRY) {
        store_h(a.seg_h + (uint64_t)seg * DN);
#pragma unroll
        for (int i = 0; i < CPT; ++i)
            if (live[i] && n0 == 0u) a.seg_sdt[(uint64_t)seg * a.D + ch[i]] = sdt[i];
    }
}

// Second pass of a split: the state at each segment's end, in order along the token axis, one thread per state.
__global__ void __launch_bounds__(256) ssm_carry_kernel(const SsmArgs a) {
    dep_wait();
    const uint64_t DN = (uint64_t)a.D * a.N, i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= DN) return;
    const uint32_t d = (uint32_t)(i / a.N);
    const float A2 = a.A[i] * 1.44269504f;
    float carry = 0.0f;
#pragma unroll 4
    for (uint32_t k = 0; k + 1u < a.n_seg; ++k) {
        const uint32_t flag = a.seg_flag[k];
        if (flag == SEG_NONE) continue;
        const float own = a.seg_h[k * DN + i];
        carry = flag == SEG_STARTS ? own : fmaf(exp2_fast(A2 * a.seg_sdt[(uint64_t)k * a.D + d]), carry, own);
        a.seg_h[k * DN + i] = carry;
    }
}

// What a prompt leaves behind beside the states: the last W - 1 rows of each job, and the zero state of a job without
// tokens.  Behind the scan in the stream, because the scan of any CTA may read the rows kept before.
template <typename T>
__global__ void __launch_bounds__(256) ssm_history_kernel(const SsmArgs a) {
    dep_wait();
    const uint32_t s = blockIdx.x;
    const int64_t slot = slot_of(a, s);
    if (slot < 0) return;
    const uint64_t q = a.off[s], e0 = a.off[s + 1u], e = e0 < a.T ? e0 : a.T;
    const int64_t len = e > q ? (int64_t)(e - q) : 0;
    if (a.W > 1u && a.history)
        for (uint32_t c = blockIdx.y * blockDim.x + threadIdx.x; c < a.rows; c += gridDim.y * blockDim.x) {
            float v[SSM_MAX_WIDTH - 1];
#pragma unroll
            for (int k = 0; k < SSM_MAX_WIDTH - 1; ++k)
                v[k] = k < (int)a.W - 1 ? row_value<T>(a, q, len - (int64_t)(a.W - 1u) + k, c, slot) : 0.0f;
#pragma unroll
            for (int k = 0; k < SSM_MAX_WIDTH - 1; ++k)
                if (k < (int)a.W - 1)
                    static_cast<T*>(a.history)[(slot * (int64_t)(a.W - 1u) + k) * a.rows + c] = from_f32<T>(v[k]);
        }
    if (len == 0 && !a.resume && a.state) {
        const uint64_t DN = (uint64_t)a.D * a.N;
        for (uint64_t i = blockIdx.y * blockDim.x + threadIdx.x; i < DN; i += (uint64_t)gridDim.y * blockDim.x)
            a.state[slot * (int64_t)DN + i] = 0.0f;
    }
}

constexpr int SSM_STEP_THREADS = 256;

// Single tokens: a cluster of CTAs per job, 4 states of one channel per thread.  The state is read and written once;
// every CTA convolves the job's B and C for itself, so the kept rows of B and C are replaced by the first CTA only
// after the cluster has read them.
template <typename T>
__global__ void __launch_bounds__(SSM_STEP_THREADS) ssm_step_kernel(const SsmArgs a, uint32_t lanes, uint32_t vec) {
    extern __shared__ __align__(16) float s_bc[];           // B of all groups, then C, each padded to 4 * lanes
    dep_wait();
    uint32_t rank, n_rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_rank));
    const uint32_t s = blockIdx.x / n_rank, tid = threadIdx.x, NP = 4u * lanes;
    const int64_t slot = slot_of(a, s);
    const T* row = static_cast<const T*>(a.xbc) + (int64_t)s * a.xbc_stride;
    T* hist = a.W > 1u && a.history && slot >= 0 ? static_cast<T*>(a.history) + slot * (int64_t)(a.W - 1u) * a.rows : nullptr;
    auto convolve = [&](uint32_t col, float v, float (&past)[3]) {
        if (a.W == 0u) return v;
        float acc = fmaf(a.conv_w[(uint64_t)col * a.W + a.W - 1u], v, a.conv_b ? a.conv_b[col] : 0.0f);
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < (int)a.W - 1) {
                past[k] = hist ? to_f32(hist[(uint64_t)k * a.rows + col]) : 0.0f;
                acc = fmaf(a.conv_w[(uint64_t)col * a.W + k], past[k], acc);
            }
        return silu(acc);
    };
    auto shift = [&](uint32_t col, float v, const float (&past)[3]) {
        if (!hist) return;
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < (int)a.W - 1)
                hist[(uint64_t)k * a.rows + col] = from_f32<T>(k + 1 < (int)a.W - 1 ? past[k + 1 < 3 ? k + 1 : 2] : v);
    };
    for (uint32_t i = tid; i < 2u * a.G * NP; i += SSM_STEP_THREADS) {
        const uint32_t n = i % NP, which = i / NP;          // which: B of group 0 .. G - 1, then C
        float v = 0.0f, past[3] = {0.0f, 0.0f, 0.0f};
        if (n < a.N) {
            const uint32_t col = a.D + which * a.N + n;
            v = convolve(col, to_f32(row[col]), past);
        }
        s_bc[i] = v;
    }
    __syncthreads();
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");

    const uint32_t per = SSM_STEP_THREADS / lanes, sub = tid % lanes, Dg = a.D / a.G;
    const uint32_t stride = per * n_rank;
    for (uint32_t d = rank * per + tid / lanes; d < (a.D + stride - 1u) / stride * stride; d += stride) {
        const bool live = d < a.D;
        const uint32_t c = live ? d : 0u, n = sub * 4u;
        float hv[4], av[4];
        float* hp = slot >= 0 && a.state ? a.state + (slot * (int64_t)a.D + c) * a.N + n : nullptr;
        const float* ap = a.A + (uint64_t)c * a.N + n;
        if (vec) {
            const float4 q = hp && n < a.N ? *reinterpret_cast<const float4*>(hp) : make_float4(0.f, 0.f, 0.f, 0.f);
            const float4 p = n < a.N ? *reinterpret_cast<const float4*>(ap) : make_float4(0.f, 0.f, 0.f, 0.f);
            hv[0] = q.x; hv[1] = q.y; hv[2] = q.z; hv[3] = q.w;
            av[0] = p.x; av[1] = p.y; av[2] = p.z; av[3] = p.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                hv[k] = hp && n + k < a.N ? hp[k] : 0.0f;
                av[k] = n + k < a.N ? ap[k] : 0.0f;
            }
        }
        const float xv = to_f32(row[c]);
        float past[3] = {0.0f, 0.0f, 0.0f};
        const float u = convolve(c, xv, past);
        const float dt = softplus(to_f32(static_cast<const T*>(a.dt)[(int64_t)s * a.dt_stride + c]) + (a.dt_bias ? a.dt_bias[c] : 0.0f));
        const float* bq = s_bc + (c / Dg) * NP + n;
        const float* cq = bq + a.G * NP;
        float acc = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            hv[k] = fmaf(exp2_fast(dt * (av[k] * 1.44269504f)), hv[k], dt * u * bq[k]);
            acc = fmaf(hv[k], cq[k], acc);
        }
        for (uint32_t m = 1; m < lanes; m *= 2) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, m);
        __syncwarp();                                       // all lanes have read the kept rows of their channel
        if (live) {
            if (hp) {
                if (vec) {
                    if (n < a.N) *reinterpret_cast<float4*>(hp) = make_float4(hv[0], hv[1], hv[2], hv[3]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (n + k < a.N) hp[k] = hv[k];
                }
            }
            if (sub == 0u) {
                float v = fmaf(a.skip ? a.skip[c] : 0.0f, u, acc);
                if (a.z) v *= silu(to_f32(static_cast<const T*>(a.z)[(int64_t)s * a.z_stride + c]));
                static_cast<T*>(a.y)[(int64_t)s * a.y_stride + c] = from_f32<T>(v);
                shift(c, xv, past);
            }
        }
    }
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (rank == 0u && hist)
        for (uint32_t i = tid; i < 2u * a.G * a.N; i += SSM_STEP_THREADS) {
            const uint32_t col = a.D + i;
            float past[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < (int)a.W - 1) past[k] = to_f32(hist[(uint64_t)k * a.rows + col]);
            shift(col, to_f32(row[col]), past);
        }
}

}  // namespace sja
