// Statistics of rows of logits: log probability of a given token, entropy, and the most likely alternatives.
//
// One pass keeps the largest logit m, the sum s = sum 2^d and the weighted sum w = sum 2^d d over d = (x - m) scale log2(e):
// log p(v) = (x_v - m) scale - ln 2 log2 s, entropy = ln 2 (log2 s - w / s).  m is subtracted before anything is scaled,
// so that a mask of the type's lowest value stays a (very small) number and a row of nothing else is uniform.
#pragma once
#include "sja_ssm.cuh"

namespace sja {

constexpr uint32_t TOK_MAX_TOP = 32;

struct TokenArgs {
    const void* logits;
    int64_t row_stride;
    uint64_t R;
    uint32_t V, top;
    float scale, c;               // c = scale * log2(e)
    const int64_t* tokens;
    float *logp, *entropy, *top_logp;
    int32_t* top_ids;
};

// Order of the alternatives as one whole number: the larger logit first (NaN below -inf, -0 = 0), then the lower
// index.  All keys of a row are distinct and none is 0.
__device__ __forceinline__ uint32_t value_key(float v) {
    v += 0.0f;
    const uint32_t b = __float_as_uint(v);
    return v != v ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return k == 0u ? __uint_as_float(0x7FC00000u) : __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint64_t order_key(float v, uint32_t idx) {
    return ((uint64_t)value_key(v) << 32) | (uint32_t)~idx;
}

// Sums of a part of a row relative to m (its largest logit; -inf where nothing was seen but -inf).
struct Stat { float m, s, w; };

__device__ __forceinline__ Stat stat_join(const Stat& a, const Stat& b, float c) {
    Stat r;
    r.m = fmaxf(a.m, b.m);
    // an empty side has s = 0 (or NaN, which has to stay); inf - inf below is left to make NaN of a row with +inf
    const float da = a.m == -INFINITY ? 0.0f : (a.m - r.m) * c, db = b.m == -INFINITY ? 0.0f : (b.m - r.m) * c;
    const float fa = exp2_fast(da), fb = exp2_fast(db);
    r.s = a.s * fa + b.s * fb;
    r.w = fa * fmaf(a.s, fmaxf(da, -200.0f), a.w) + fb * fmaf(b.s, fmaxf(db, -200.0f), b.w);
    return r;
}

template <typename T> struct Vec { static constexpr int n = 16 / sizeof(T); };

// The elements of one 16-byte vector of the row (or fewer at its end), as 32-bit values.
template <typename T>
__device__ __forceinline__ void load_vec(const T* p, bool aligned, uint32_t count, float (&v)[Vec<T>::n]) {
    constexpr int n = Vec<T>::n;
    if (aligned && count >= (uint32_t)n) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        const T* e = reinterpret_cast<const T*>(&q);
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = to_f32(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = (uint32_t)i < count ? to_f32(p[i]) : -INFINITY;
    }
}

// Row log probabilities from the joined sums.
struct RowStat {
    float m, log_s, entropy;
    bool empty;
    __device__ __forceinline__ explicit RowStat(const Stat& t) {
        empty = t.m == -INFINITY && t.s == 0.0f;
        m = empty ? 0.0f : t.m;
        log_s = empty ? 0.0f : __log2f(t.s);
        entropy = empty ? 0.0f : LN2 * (log_s - t.w / t.s);
    }
    __device__ __forceinline__ float logp(float logit, float scale) const {
        if (logit == -INFINITY) return -INFINITY;
        return fmaf(logit - m, scale, -LN2 * log_s);
    }
};

constexpr int TOK_THREADS = 256, TOK_CAND = 2048;

// One CTA per row, any vocabulary.  The alternatives: every thread knows its largest element; the r-th largest of
// each warp's, r * warps >= top, bound the answer from below, so a second look at the row (which the cache still
// holds) keeps a few dozen candidates, ranked by counting.  Rows on which the bound fails to thin the candidates out
// take `top` rounds of a maximum instead.
template <typename T>
__global__ void __launch_bounds__(TOK_THREADS) token_stats_kernel(const TokenArgs a) {
    constexpr int n = Vec<T>::n, WARPS = TOK_THREADS / 32;
    __shared__ Stat s_stat[WARPS];
    __shared__ uint64_t s_bound[WARPS], s_cand[TOK_CAND], s_max[WARPS];
    __shared__ uint32_t s_count;
    dep_wait();
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    const uint64_t r = blockIdx.x;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.row_stride;
    const bool aligned = (reinterpret_cast<uintptr_t>(row) & 15u) == 0u;
    if (tid == 0u) s_count = 0u;

    Stat st = {-INFINITY, 0.0f, 0.0f};
    float best = -INFINITY;
    uint64_t key = 0ull;
    for (uint32_t i = tid * n; i < a.V; i += TOK_THREADS * n) {
        float v[n];
        const uint32_t count = min(a.V - i, (uint32_t)n);
        load_vec(row + i, aligned, count, v);
        float vm = v[0];
#pragma unroll
        for (int j = 1; j < n; ++j) vm = fmaxf(vm, v[j]);
        if (key == 0ull || vm > best) {
            uint64_t k = 0ull;
#pragma unroll
            for (int j = 0; j < n; ++j)
                if ((uint32_t)j < count) k = max(k, order_key(v[j], i + j));
            if (k > key) key = k;
            if (vm > best) {
                best = vm;
                const float d = st.m == -INFINITY ? 0.0f : (st.m - best) * a.c, f = exp2_fast(d);
                st.w = f * fmaf(st.s, fmaxf(d, -200.0f), st.w);
                st.s *= f;
                st.m = best;
            }
        }
        const float m = st.m == -INFINITY ? 0.0f : st.m;
#pragma unroll
        for (int j = 0; j < n; ++j) {
            const float d = (v[j] - m) * a.c, e = exp2_fast(d);
            st.s += e;
            st.w = fmaf(e, fmaxf(d, -200.0f), st.w);
        }
    }
    // a thread that has seen NaN only has best = -inf and a NaN sum: the sums carry it from here
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        Stat o;
        o.m = __shfl_xor_sync(0xFFFFFFFFu, st.m, m);
        o.s = __shfl_xor_sync(0xFFFFFFFFu, st.s, m);
        o.w = __shfl_xor_sync(0xFFFFFFFFu, st.w, m);
        st = stat_join(st, o, a.c);
    }
    if (lane == 0u) s_stat[warp] = st;
    const uint32_t top = min(a.top, a.V);
    if (top) {
        uint64_t left = key, bound = 0ull;
        for (uint32_t k = 0; k < (top + WARPS - 1u) / WARPS; ++k) {
            bound = warp_max_u64(left);
            if (left == bound) left = 0ull;
        }
        if (lane == 0u) s_bound[warp] = bound;
    }
    __syncthreads();
    st = s_stat[0];
    for (int w = 1; w < WARPS; ++w) st = stat_join(st, s_stat[w], a.c);
    const RowStat rs(st);
    if (tid == 0u) {
        if (a.entropy) a.entropy[r] = rs.entropy;
        if (a.logp) {
            const int64_t t = a.tokens[r];
            a.logp[r] = t < 0 ? 0.0f : t >= (int64_t)a.V ? __uint_as_float(0x7FC00000u) : rs.logp(to_f32(row[t]), a.scale);
        }
    }
    if (!a.top) return;
    auto put = [&](uint32_t k, uint64_t q) {
        const float v = key_value((uint32_t)(q >> 32));
        if (a.top_ids) a.top_ids[r * a.top + k] = q ? (int32_t)~(uint32_t)q : -1;
        if (a.top_logp) a.top_logp[r * a.top + k] = q ? rs.logp(v, a.scale) : -INFINITY;
    };
    for (uint32_t k = top + tid; k < a.top; k += TOK_THREADS) put(k, 0ull);
    uint64_t bound = s_bound[0];
    for (int w = 1; w < WARPS; ++w) bound = min(bound, s_bound[w]);
    for (uint32_t i = tid * n; i < a.V; i += TOK_THREADS * n) {
        float v[n];
        const uint32_t count = min(a.V - i, (uint32_t)n);
        load_vec(row + i, aligned, count, v);
#pragma unroll
        for (int j = 0; j < n; ++j) {
            const uint64_t k = order_key(v[j], i + j);
            if ((uint32_t)j < count && k >= bound) {
                const uint32_t at = atomicAdd(&s_count, 1u);
                if (at < TOK_CAND) s_cand[at] = k;
            }
        }
    }
    __syncthreads();
    const uint32_t count = s_count;
    if (count <= TOK_CAND) {
        for (uint32_t i = tid; i < count; i += TOK_THREADS) {
            const uint64_t k = s_cand[i];
            uint32_t rank = 0;
            for (uint32_t j = 0; j < count && rank < top; ++j) rank += s_cand[j] > k;
            if (rank < top) put(rank, k);
        }
        return;
    }
    uint64_t below = ~0ull;
    for (uint32_t k = 0; k < top; ++k) {
        uint64_t most = 0ull;
        for (uint32_t i = tid; i < a.V; i += TOK_THREADS) {
            const uint64_t q = order_key(to_f32(row[i]), i);
            if (q < below) most = max(most, q);
        }
        most = warp_max_u64(most);
        if (lane == 0u) s_max[warp] = most;
        __syncthreads();
        most = s_max[0];
        for (int w = 1; w < WARPS; ++w) most = max(most, s_max[w]);
        if (tid == 0u) put(k, most);
        below = most;
        __syncthreads();
    }
}

}  // namespace sja
