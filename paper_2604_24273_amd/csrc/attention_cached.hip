// Attention of new tokens over a paged key/value cache.
#include "common.hpp"

namespace brl {

namespace {

// element d of a row of the cache, widened
__device__ __forceinline__ float cache_value(const char* pool, const float* scales, int dtype, int row, long long idx, int d) {
    const size_t e = (size_t)idx * row + d;
    if (dtype == BRL_F32) return reinterpret_cast<const float*>(pool)[e];
    if (dtype == BRL_F16) return (float)reinterpret_cast<const _Float16*>(pool)[e];
    return (float)reinterpret_cast<const int8_t*>(pool)[e] * scales[idx];
}

__device__ __forceinline__ bool sees(const CachedAttention& a, const StateTokens& st, int i, int slot) {
    if (!a.tree) return slot <= st.base + i;
    const int j = slot - st.base;
    if (j < 0) return true;
    return (j >> 5) < a.mask_words && (a.tree[(size_t)(st.row0 + i) * a.mask_words + (j >> 5)] >> (j & 31) & 1u);
}

// One wavefront per token and query head; a lane per slot for the scores, per component for the sum.
__global__ __launch_bounds__(64) void cached_rows_kernel(CachedAttention a, float* lse) {
    __shared__ float q[128], p[64];
    __shared__ long long rows[64];
    const int lane = threadIdx.x, hq = blockIdx.x % a.n_heads;
    const int b = blockIdx.x / a.n_heads / a.t.max_new, i = blockIdx.x / a.n_heads % a.t.max_new;
    const StateTokens st = state_tokens(a.t, a.c, b);
    if (i >= st.n) return;
    const int dh = a.c.dh, half = dh / 2, h = hq / (a.n_heads / a.c.n_kv), row = st.row0 + i;
    const float* x = a.qkv + (size_t)row * ((a.n_heads + 2 * a.c.n_kv) * dh) + hq * dh;
    const int pos = rope_position(a.t, row, st.base + i);
    const float scale = (float)(1.0 / sqrt((double)dh)) * 1.4426950408889634f;
    if (lane < half) {
        const float c = a.t.cos_t[(size_t)pos * half + lane], s = a.t.sin_t[(size_t)pos * half + lane];
        q[lane] = (x[lane] * c - x[lane + half] * s) * scale;
        q[lane + half] = (x[lane + half] * c + x[lane] * s) * scale;
    }
    __syncthreads();
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int k0 = 0; k0 < st.len; k0 += 64) {
        const int slot = k0 + lane;
        const long long idx = slot < st.len ? kv_row_index(a.c, b, h, slot) : -1;
        float v = -INFINITY;
        if (idx >= 0 && sees(a, st, i, slot)) {
            v = 0.f;
            for (int d = 0; d < dh; ++d) v += q[d] * cache_value(a.c.k, a.c.ks, a.c.dtype, a.c.row, idx, d);
        }
        const float m_new = fmaxf(m, wave_max(v));
        if (m_new == -INFINITY) continue;
        const float e = __builtin_amdgcn_exp2f(v - m_new), alpha = __builtin_amdgcn_exp2f(m - m_new);
        p[lane] = e;
        rows[lane] = e > 0.f ? idx : -1;
        __syncthreads();
        l = l * alpha + wave_total(e);
        o0 *= alpha; o1 *= alpha;
        for (int k = 0; k < 64; ++k) {
            if (rows[k] < 0) continue;
            if (lane < dh) o0 += p[k] * cache_value(a.c.v, a.c.vs, a.c.dtype, a.c.row, rows[k], lane);
            if (lane + 64 < dh) o1 += p[k] * cache_value(a.c.v, a.c.vs, a.c.dtype, a.c.row, rows[k], lane + 64);
        }
        __syncthreads();
        m = m_new;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    float* o = a.out + (size_t)row * a.n_heads * dh + hq * dh;
    if (lane < dh) o[lane] = o0 * inv;
    if (lane + 64 < dh) o[lane + 64] = o1 * inv;
    if (lse && lane == 0) lse[(size_t)row * a.n_heads + hq] = l > 0.f ? m + __builtin_amdgcn_logf(l) : INFINITY;
}

// One thread per slot and k/v head: its weight summed over the rows that see it.
__global__ __launch_bounds__(64) void cached_weights_kernel(CachedAttention a, const float* lse, int chunks) {
    __shared__ float q[128];
    const int lane = threadIdx.x, h = blockIdx.x / chunks % a.c.n_kv, b = blockIdx.x / chunks / a.c.n_kv;
    const int slot = blockIdx.x % chunks * 64 + lane;
    const StateTokens st = state_tokens(a.t, a.c, b);
    const int dh = a.c.dh, half = dh / 2, group = a.n_heads / a.c.n_kv;
    const float scale = (float)(1.0 / sqrt((double)dh)) * 1.4426950408889634f;
    const long long idx = slot < st.len ? kv_row_index(a.c, b, h, slot) : -1;
    float sum = 0.f;
    for (int i = 0; i < st.n; ++i)
        for (int g = 0; g < group; ++g) {
            const int row = st.row0 + i, hq = h * group + g;
            const float* x = a.qkv + (size_t)row * ((a.n_heads + 2 * a.c.n_kv) * dh) + hq * dh;
            const int pos = rope_position(a.t, row, st.base + i);
            __syncthreads();
            if (lane < half) {
                const float c = a.t.cos_t[(size_t)pos * half + lane], s = a.t.sin_t[(size_t)pos * half + lane];
                q[lane] = (x[lane] * c - x[lane + half] * s) * scale;
                q[lane + half] = (x[lane + half] * c + x[lane] * s) * scale;
            }
            __syncthreads();
            if (idx < 0 || !sees(a, st, i, slot)) continue;
            float v = 0.f;
            for (int d = 0; d < dh; ++d) v += q[d] * cache_value(a.c.k, a.c.ks, a.c.dtype, a.c.row, idx, d);
            sum += __builtin_amdgcn_exp2f(v - lse[(size_t)row * a.n_heads + hq]);
        }
    if (idx >= 0) a.weights[((size_t)b * a.c.n_kv + h) * a.ld_weights + slot] += sum;
}

}  // namespace

size_t cached_attention_ws_bytes(const KvView& c, int n_heads, int T, int B, int max_new, int max_len, bool weights) {
    (void)c; (void)B; (void)max_new; (void)max_len;
    return weights ? (size_t)T * n_heads * 4 : 0;
}

int launch_cached_attention(const CachedAttention& a, void* workspace, hipStream_t s) {
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    float* lse = a.weights ? static_cast<float*>(workspace) : nullptr;
    hipLaunchKernelGGL(cached_rows_kernel, dim3((unsigned)a.t.B * a.t.max_new * a.n_heads), dim3(64), 0, s, a, lse);
    if (a.weights) {
        const int chunks = (a.t.max_len + 63) / 64;
        hipLaunchKernelGGL(cached_weights_kernel, dim3((unsigned)a.t.B * a.c.n_kv * chunks), dim3(64), 0, s, a, (const float*)lse, chunks);
    }
    BRL_LAUNCH_CHECK("cached_rows_kernel");
    return BRL_OK;
}

}  // namespace brl
