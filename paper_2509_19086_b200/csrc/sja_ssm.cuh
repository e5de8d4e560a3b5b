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

__device__ __forceinline__ float exp2_fast(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp_fast(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

constexpr float LN2 = 0.693147182f, LOG2E = 1.44269504f;

__device__ __forceinline__ float silu(float v) { return v * rcp_fast(1.0f + exp2_fast(-LOG2E * v)); }

// softplus(v) = max(v, 0) + log1p(e), e = exp(-|v|).  Time steps of 0.001 and less come from very negative v, where
// log(1 + e) would lose what 1 + e rounds away; log1p(e) = 2 atanh(q), q = e / (2 + e) in 0 .. 1/3, keeps it: the
// odd series in q, its even part fitted by a polynomial in q^2 on 0 .. 1/9 (relative error 8e-9).
__device__ __forceinline__ float softplus(float v) {
    const float e = exp2_fast(-LOG2E * fabsf(v)), q = e * rcp_fast(2.0f + e), w = q * q;
    float p = fmaf(w, 0.140873283f, 0.139807090f);
    p = fmaf(w, p, 0.200124264f);
    p = fmaf(w, p, 0.333331585f);
    p = fmaf(w, p, 1.0f);
    return fmaf(q + q, p, fmaxf(v, 0.0f));
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
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
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

constexpr uint32_t SSM_THREADS = 256;    // most threads of a prompt CTA
// Tokens whose B and C one CTA keeps at a time: a thread convolves a stretch of 8 tokens of one column (2 NP of them).
__host__ __device__ constexpr uint32_t ssm_tile_tokens(uint32_t np) { return 1024u / np; }

// Prompts.  A thread owns one channel and K of its states (LPC lanes share a channel), walks its segment of the token
// axis and keeps the states in registers.  B and C of a tile of tokens are convolved once per CTA into shared memory,
// one tile ahead of the walk, and read by broadcast; x, dt and z of the next four tokens are on their way while four
// are worked on.  CARRY = true is the first pass of a split: what the job that crosses the segment's end adds to its
// state inside the segment, and its sum of time steps (exp(A sum dt) is the decay over the segment).
template <typename T, int K, int LPC, bool CARRY>
__global__ void __launch_bounds__(SSM_THREADS, 2) ssm_prompt_kernel(const SsmArgs a) {
    constexpr uint32_t NP = K * LPC, TT = ssm_tile_tokens(NP), CPW = 32 / LPC, COLS = CARRY ? NP : 2 * NP;
    constexpr int U = 4, STRETCH = 8;
    __shared__ __align__(16) float s_bc[2][TT * 2 * NP];       // [buffer][token][B | C]
    dep_wait();
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    const uint32_t Dg = a.D / a.G, span = (blockDim.x >> 5) * CPW;
    const uint32_t tiles = (Dg + span - 1u) / span;
    const uint32_t g = blockIdx.x / tiles, seg = blockIdx.y;
    const uint32_t in_group = (blockIdx.x % tiles) * span + warp * CPW + lane / LPC;
    const uint32_t n0 = (lane % LPC) * K;
    const bool live = in_group < Dg;
    const uint32_t ch = g * Dg + (live ? in_group : 0u);
    const uint64_t b0 = segment_bound(a, seg), b1 = segment_bound(a, seg + 1u);
    uint64_t t = b0;
    uint32_t s;
    if (CARRY) {
        s = warp_lower_bound(a.off, a.S + 1u, b1 + 1ull);
        s = s ? s - 1u : 0u;
        const uint64_t q = a.off[s];
        const uint32_t flag = (s >= a.S || q >= b1) ? SEG_NONE : q >= b0 ? SEG_STARTS : SEG_PASSES;
        if (blockIdx.x == 0u && tid == 0u) a.seg_flag[seg] = flag;
        if (flag == SEG_NONE) return;
        t = q > b0 ? q : b0;
    } else {
        s = warp_lower_bound(a.off, a.S + 1u, b0 + 1ull);
        s = s ? s - 1u : 0u;
    }

    F2 A2[K / 2], h[K / 2];
    Conv cx;
    cx.load(a, ch);
    const float skip = a.skip ? a.skip[ch] : 0.0f, bias = a.dt_bias ? a.dt_bias[ch] : 0.0f;
    float sdt = 0.0f;
    auto load_states = [&](F2 (&to)[K / 2], const float* from, float scale) {
        const float* r = from + (uint64_t)ch * a.N;
#pragma unroll
        for (int k = 0; k < K / 2; ++k) {
            const uint32_t n = n0 + 2 * k;
            to[k] = f2(n < a.N ? r[n] * scale : 0.0f, n + 1u < a.N ? r[n + 1u] * scale : 0.0f);
        }
    };
    auto store_h = [&](float* to) {
        float* r = to + (uint64_t)ch * a.N;
#pragma unroll
        for (int k = 0; k < K / 2; ++k) {
            const uint32_t n = n0 + 2 * k;
            float v0, v1;
            f2_split(h[k], v0, v1);
            if (live && n < a.N) r[n] = v0;
            if (live && n + 1u < a.N) r[n + 1u] = v1;
        }
    };
    load_states(A2, a.A, LOG2E);
#pragma unroll
    for (int k = 0; k < K / 2; ++k) h[k] = f2(0.0f, 0.0f);
    const uint64_t DN = (uint64_t)a.D * a.N;
    const T* xp = static_cast<const T*>(a.xbc);

    // this thread's part in convolving B and C: column bc_col, tokens bc_from .. bc_from + 7 of a tile
    const uint32_t parts = max(blockDim.x / COLS, 1u), tile_tok = min(parts * (uint32_t)STRETCH, TT);
    auto stage = [&](uint32_t w, uint64_t q, int64_t slot, uint64_t at, uint32_t n_tok, float* to) {
        const uint32_t col = w % COLS, from = (w / COLS) * STRETCH, n = col % NP;
        if (from >= n_tok) return;
        const uint32_t cnt = min((uint32_t)STRETCH, n_tok - from);
        float* dst = to + from * (2 * NP) + (col < NP ? 0u : NP) + n;
        if (n >= a.N) {
#pragma unroll
            for (int i = 0; i < STRETCH; ++i) dst[i * (2 * NP)] = 0.0f;      // the tile has room for whole stretches
            return;
        }
        const uint32_t rc = a.D + (col < NP ? 0u : a.G * a.N) + g * a.N + n;
        Conv cv;
        cv.load(a, rc);
        cv.template seek<T>(a, q, (int64_t)(at - q) + from, rc, slot);
        const T* src = xp + (int64_t)(at + from) * a.xbc_stride + rc;
        float v[STRETCH];
#pragma unroll
        for (int i = 0; i < STRETCH; ++i) v[i] = (uint32_t)i < cnt ? to_f32(src[(int64_t)i * a.xbc_stride]) : 0.0f;
#pragma unroll
        for (int i = 0; i < STRETCH; ++i) dst[i * (2 * NP)] = cv.next(a.W, v[i]);
    };

    // what a job leaves behind beside its state: its last W - 1 rows.  With `resume` other CTAs may still have to read
    // the rows that these replace: then a kernel of its own stores them.
    const bool keeps = !CARRY && !a.resume;
    auto store_history = [&](uint64_t first, int64_t len, int64_t slot) {
        if (a.W <= 1u || !a.history || slot < 0) return;
        T* to = static_cast<T*>(a.history) + slot * (int64_t)(a.W - 1u) * a.rows;
        for (uint32_t k = 0; k + 1u < a.W; ++k) {
            const int64_t pos = len - (int64_t)(a.W - 1u) + k;
            if (live && n0 == 0u) to[(uint64_t)k * a.rows + ch] = from_f32<T>(row_value<T>(a, first, pos, ch, slot));
            if (blockIdx.x % tiles == 0u)
                for (uint32_t i = tid; i < 2u * a.N; i += blockDim.x) {
                    const uint32_t col = a.D + (i < a.N ? g * a.N + i : a.G * a.N + g * a.N + i - a.N);
                    to[(uint64_t)k * a.rows + col] = from_f32<T>(row_value<T>(a, first, pos, col, slot));
                }
        }
    };

    // a segment has the jobs that end behind its first token and up to its end, empty ones among them
    if (!CARRY && seg == 0u) s = 0u;
    for (; s < a.S; ++s) {
        const uint64_t q = a.off[s];
        uint64_t e = a.off[s + 1u];
        if (e == q && q <= b1) {
            if (keeps) {
                const int64_t slot = slot_of(a, s);
#pragma unroll
                for (int k = 0; k < K / 2; ++k) h[k] = f2(0.0f, 0.0f);
                if (slot >= 0 && a.state) store_h(a.state + slot * (int64_t)DN);
                store_history(q, 0, slot);
            }
            continue;
        }
        if (t >= b1 || q >= b1) break;
        if (e <= t || q > t) continue;                 // offsets that are not ascending
        const bool ends = e <= b1;
        if (!ends) e = b1;
        const int64_t slot = slot_of(a, s);
        // where the job's state comes from: the segment before, its slot, or nothing
        if (q < t) {
            if (!CARRY) load_states(h, a.seg_h + (uint64_t)(seg - 1u) * DN, 1.0f);
        } else if (a.resume && slot >= 0 && a.state) {
            // a job that goes on behind this segment may be stored by another CTA meanwhile: the first pass kept a copy
            if (CARRY || ends || a.n_seg == 1u) load_states(h, a.state + slot * (int64_t)DN, 1.0f);
            else load_states(h, a.seg_first + (uint64_t)seg * DN, 1.0f);
            if (CARRY) store_h(a.seg_first + (uint64_t)seg * DN);
        } else {
#pragma unroll
            for (int k = 0; k < K / 2; ++k) h[k] = f2(0.0f, 0.0f);
        }
        cx.template seek<T>(a, q, (int64_t)(t - q), ch, slot);
        const T* px = xp + (int64_t)t * a.xbc_stride + ch;
        const T* pd = static_cast<const T*>(a.dt) + (int64_t)t * a.dt_stride + ch;
        const T* pz = a.z && !CARRY ? static_cast<const T*>(a.z) + (int64_t)t * a.z_stride + ch : nullptr;
        T* py = static_cast<T*>(a.y) + (int64_t)t * a.y_stride + ch;
        uint64_t left = e - t;
        T xr[U], dr[U], zr[U];
        auto fetch = [&](uint64_t have) {              // rows behind the job's end are not touched
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if ((uint64_t)j < have) {
                    xr[j] = px[j * a.xbc_stride];
                    dr[j] = pd[j * a.dt_stride];
                    if (pz) zr[j] = pz[j * a.z_stride];
                }
            }
        };
#pragma unroll
        for (int j = 0; j < U; ++j) xr[j] = dr[j] = zr[j] = from_f32<T>(0.0f);
        fetch(left);
        uint32_t buf = 0;
        __syncthreads();
        for (uint32_t w = tid; w < COLS * parts; w += blockDim.x)
            stage(w, q, slot, t, (uint32_t)min((uint64_t)tile_tok, left), s_bc[0]);
        while (t < e) {
            const uint32_t n_tok = (uint32_t)min((uint64_t)tile_tok, left);
            __syncthreads();
            if (left > n_tok)
                for (uint32_t w = tid; w < COLS * parts; w += blockDim.x)
                    stage(w, q, slot, t + n_tok, (uint32_t)min((uint64_t)tile_tok, left - n_tok), s_bc[buf ^ 1u]);
            const float* bc = s_bc[buf] + n0;
            for (uint32_t i0 = 0; i0 < n_tok; i0 += U) {
                // convolution, time step and gate of the four tokens first: four independent chains (what follows a
                // job's last token is worked out too, and not used)
                float uv[U], dv[U], zv[U];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    uv[j] = cx.next(a.W, to_f32(xr[j]));
                    dv[j] = softplus(to_f32(dr[j]) + bias);
                    zv[j] = CARRY || !a.z ? 1.0f : silu(to_f32(zr[j]));
                }
                px += U * a.xbc_stride; pd += U * a.dt_stride;
                if (pz) pz += U * a.z_stride;
                if (left > i0 + U) fetch(left - i0 - U);
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    if (i0 + j >= n_tok) break;
                    const float u = uv[j], d = dv[j];
                    if (CARRY) sdt += d;
                    const F2 d2 = f2(d, d), du2 = f2(d * u, d * u);
                    F2 acc = f2(0.0f, 0.0f);
                    const ulonglong2* pB = reinterpret_cast<const ulonglong2*>(bc + (i0 + j) * (2 * NP));
#pragma unroll
                    for (int k = 0; k < K / 4; ++k) {
                        const ulonglong2 bq = pB[k];
                        ulonglong2 cq = {0ull, 0ull};
                        if (!CARRY) cq = pB[NP / 4 + k];
                        const F2 b2[2] = {{bq.x}, {bq.y}}, c2[2] = {{cq.x}, {cq.y}};
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            float e0, e1;
                            f2_split(f2_mul(d2, A2[2 * k + m]), e0, e1);
                            const F2 decay = f2(exp2_fast(e0), exp2_fast(e1));
                            F2& hh = h[2 * k + m];
                            hh = f2_fma(decay, hh, f2_mul(du2, b2[m]));
                            if (!CARRY) acc = f2_fma(hh, c2[m], acc);
                        }
                    }
                    if (!CARRY) {
                        float v0, v1;
                        f2_split(acc, v0, v1);
                        float v = v0 + v1;
#pragma unroll
                        for (int m = 1; m < LPC; m *= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
                        v = fmaf(skip, u, v);
                        v *= zv[j];
                        if (live && n0 == 0u) py[j * a.y_stride] = from_f32<T>(v);
                    }
                }
                py += U * a.y_stride;
            }
            // (a tile that is not a whole number of groups is the job's last one)
            t += n_tok;
            left -= n_tok;
            buf ^= 1u;
        }
        if (!CARRY && ends && slot >= 0 && a.state) store_h(a.state + slot * (int64_t)DN);
        if (keeps && ends) store_history(q, (int64_t)(e - q), slot);
    }
    if (CARRY) {
        store_h(a.seg_h + (uint64_t)seg * DN);
        if (live && n0 == 0u) a.seg_sdt[(uint64_t)seg * a.D + ch] = sdt;
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

// The last W - 1 rows of each job of a prompt that went on from its slots (or of one without any tokens, which also
// leaves zero states).  Behind the scan in the stream, because the scan of any CTA may read the rows kept before.
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

constexpr uint32_t SSM_STEP_THREADS = 256;

// Single tokens.  A CTA takes 256 channels of a job at a time: while their states are on the way (four 16-byte pieces
// a thread), each thread works out convolution, time step and gate of one channel; then the states are advanced,
// written back, and summed against C over the lanes of a channel.  The CTAs of a job form a cluster: each convolves
// the job's B and C for itself, so the kept rows of B and C are replaced only when the whole cluster has read them.
template <typename T>
__global__ void __launch_bounds__(SSM_STEP_THREADS, 4) ssm_step_kernel(const SsmArgs a, uint32_t lanes, uint32_t vec) {
    extern __shared__ __align__(16) float s_bc[];           // B of all groups, then C, each padded to 4 * lanes
    __shared__ float s_dt[SSM_STEP_THREADS], s_du[SSM_STEP_THREADS], s_y[SSM_STEP_THREADS];
    constexpr int U = 4;
    dep_wait();
    uint32_t rank, n_rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_rank));
    const uint32_t s = blockIdx.x / n_rank, tid = threadIdx.x, NP = 4u * lanes;
    const int64_t slot = slot_of(a, s);
    const T* row = static_cast<const T*>(a.xbc) + (int64_t)s * a.xbc_stride;
    const uint32_t H = a.W > 1u ? a.W - 1u : 0u;
    T* hist = H && a.history && slot >= 0 ? static_cast<T*>(a.history) + slot * (int64_t)H * a.rows : nullptr;
    float* state = slot >= 0 && a.state ? a.state + slot * (int64_t)a.D * a.N : nullptr;
    auto convolve = [&](uint32_t col, float v, float (&past)[3]) {
#pragma unroll
        for (uint32_t k = 0; k < 3u; ++k) past[k] = k < H && hist ? to_f32(hist[(uint64_t)k * a.rows + col]) : 0.0f;
        if (a.W == 0u) return v;
        const float* w = a.conv_w + (uint64_t)col * a.W;
        float acc = fmaf(w[H], v, a.conv_b ? a.conv_b[col] : 0.0f);
#pragma unroll
        for (uint32_t k = 0; k < 3u; ++k)
            if (k < H) acc = fmaf(w[k], past[k], acc);
        return silu(acc);
    };
    auto shift = [&](uint32_t col, float v, const float (&past)[3]) {
#pragma unroll
        for (uint32_t k = 0; k < 3u; ++k)
            if (k < H && hist) hist[(uint64_t)k * a.rows + col] = from_f32<T>(k + 1u < H ? past[k < 2u ? k + 1u : 2u] : v);
    };

    const uint32_t sub = tid % lanes, n = sub * 4u, per = SSM_STEP_THREADS / lanes, Dg = a.D / a.G;
    bool first = true;
    for (uint32_t base = rank * SSM_STEP_THREADS; base < a.D; base += n_rank * SSM_STEP_THREADS) {
        float4 hv[U], av[U];
        auto fetch = [&](uint32_t p0) {                     // passes p0 .. p0 + 3 over the 256 channels
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const uint32_t d = base + (p0 + j) * per + tid / lanes;
                hv[j] = av[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (p0 + j >= lanes || d >= a.D) continue;
                const uint64_t at = (uint64_t)d * a.N + n;
                if (vec) {
                    if (n < a.N) {
                        if (state) hv[j] = *reinterpret_cast<const float4*>(state + at);
                        av[j] = *reinterpret_cast<const float4*>(a.A + at);
                    }
                } else {
                    float* hq = &hv[j].x;
                    float* aq = &av[j].x;
#pragma unroll
                    for (uint32_t k = 0; k < 4u; ++k)
                        if (n + k < a.N) {
                            if (state) hq[k] = state[at + k];
                            aq[k] = a.A[at + k];
                        }
                }
            }
        };
        fetch(0);
        const uint32_t c = base + tid;
        float u = 0.0f, gate = 1.0f, skip = 0.0f;
        if (c < a.D) {
            const float xv = to_f32(row[c]);
            float past[3];
            u = convolve(c, xv, past);
            shift(c, xv, past);
            const float dt = softplus(to_f32(static_cast<const T*>(a.dt)[(int64_t)s * a.dt_stride + c]) + (a.dt_bias ? a.dt_bias[c] : 0.0f));
            s_dt[tid] = dt;
            s_du[tid] = dt * u;
            if (a.z) gate = silu(to_f32(static_cast<const T*>(a.z)[(int64_t)s * a.z_stride + c]));
            if (a.skip) skip = a.skip[c];
        }
        if (first)
            for (uint32_t i = tid; i < 2u * a.G * NP; i += SSM_STEP_THREADS) {
                const uint32_t m = i % NP, which = i / NP;  // which: B of group 0 .. G - 1, then C
                float v = 0.0f, past[3];
                if (m < a.N) {
                    const uint32_t col = a.D + which * a.N + m;
                    v = convolve(col, to_f32(row[col]), past);
                }
                s_bc[i] = v;
            }
        __syncthreads();
        if (first) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
        first = false;
        for (uint32_t p0 = 0; p0 < lanes; p0 += U) {
            if (p0) fetch(p0);
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (p0 + j >= lanes) break;
                const uint32_t local = (p0 + j) * per + tid / lanes, d = base + local;
                const bool live = d < a.D;
                const float dt = live ? s_dt[local] : 0.0f, du = live ? s_du[local] : 0.0f;
                const float* bq = s_bc + (live ? d / Dg : 0u) * NP + n;
                const float4 B = *reinterpret_cast<const float4*>(bq), C = *reinterpret_cast<const float4*>(bq + a.G * NP);
                const float dl = dt * LOG2E;
                hv[j].x = fmaf(exp2_fast(dl * av[j].x), hv[j].x, du * B.x);
                hv[j].y = fmaf(exp2_fast(dl * av[j].y), hv[j].y, du * B.y);
                hv[j].z = fmaf(exp2_fast(dl * av[j].z), hv[j].z, du * B.z);
                hv[j].w = fmaf(exp2_fast(dl * av[j].w), hv[j].w, du * B.w);
                float acc = fmaf(hv[j].x, C.x, hv[j].y * C.y) + fmaf(hv[j].z, C.z, hv[j].w * C.w);
                for (uint32_t m = 1; m < lanes; m *= 2) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, m);
                if (live) {
                    if (sub == 0u) s_y[local] = acc;
                    const uint64_t at = (uint64_t)d * a.N + n;
                    if (!state) continue;
                    if (vec) {
                        if (n < a.N) *reinterpret_cast<float4*>(state + at) = hv[j];
                    } else {
                        const float* hq = &hv[j].x;
#pragma unroll
                        for (uint32_t k = 0; k < 4u; ++k)
                            if (n + k < a.N) state[at + k] = hq[k];
                    }
                }
            }
        }
        __syncthreads();
        if (c < a.D)
            static_cast<T*>(a.y)[(int64_t)s * a.y_stride + c] = from_f32<T>(fmaf(skip, u, s_y[tid]) * gate);
        // (s_y is next written behind the next round's barrier, s_dt and s_du are not read any more)
    }
    if (first) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");   // a CTA without channels
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (rank == 0u && hist)
        for (uint32_t i = tid; i < 2u * a.G * a.N; i += SSM_STEP_THREADS) {
            const uint32_t col = a.D + i;
            float past[3];
#pragma unroll
            for (uint32_t k = 0; k < 3u; ++k) past[k] = k < H ? to_f32(hist[(uint64_t)k * a.rows + col]) : 0.0f;
            shift(col, to_f32(row[col]), past);
        }
}

}  // namespace sja
