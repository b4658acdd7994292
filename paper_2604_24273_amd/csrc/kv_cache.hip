// The paged key/value cache apart from attention: storing new tokens, choosing which slots to keep, moving them together.
#include "common.hpp"

namespace brl {

namespace {

// ---- append ----
// A group of GS lanes stores one token of one k/v head: each lane holds VW rotary pairs (i, i + dh/2) of the key row and the
// same components of the value row.  k' = k R(pos): two products and a sum per component, each rounded once.
struct AppendArgs {
    KvView c;
    NewTokens t;
    const float* qkv;
    int n_heads;
    int chunks;               // workgroups of a state
};

template <int VW>
struct Floats {
    float x[VW];
};
template <int VW>
__device__ __forceinline__ Floats<VW> load_floats(const float* p) {
    Floats<VW> r;
    if constexpr (VW == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        r.x[0] = v.x; r.x[1] = v.y; r.x[2] = v.z; r.x[3] = v.w;
    } else {
        const float2 v = *reinterpret_cast<const float2*>(p);
        r.x[0] = v.x; r.x[1] = v.y;
    }
    return r;
}

// VW neighbouring elements of a row in the cache's type; s: 127 / a of an int8 row
template <int DT, int VW>
__device__ __forceinline__ void store_elements(char* row, int d, const Floats<VW>& v, float s) {
    if constexpr (DT == BRL_F32) {
        float* p = reinterpret_cast<float*>(row) + d;
        if constexpr (VW == 4) *reinterpret_cast<float4*>(p) = make_float4(v.x[0], v.x[1], v.x[2], v.x[3]);
        else *reinterpret_cast<float2*>(p) = make_float2(v.x[0], v.x[1]);
    } else if constexpr (DT == BRL_F16) {
        typedef _Float16 vh __attribute__((ext_vector_type(VW)));
        vh h;
#pragma unroll
        for (int e = 0; e < VW; ++e) h[e] = (_Float16)v.x[e];
        *reinterpret_cast<vh*>(reinterpret_cast<_Float16*>(row) + d) = h;
    } else {
        float four[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < VW; ++e) four[e] = v.x[e];
        const uint32_t q = quantise_four(four, s);
        if constexpr (VW == 4) *reinterpret_cast<uint32_t*>(row + d) = q;
        else *reinterpret_cast<uint16_t*>(row + d) = (uint16_t)q;
    }
}

template <int DT, int VW, int GS>
__device__ __forceinline__ void store_row(char* pool, float* scales, int idx, int rowlen, int dh, const Floats<VW>& a,
                                          const Floats<VW>& b, int lane) {
    const int half = dh / 2;
    const bool mine = lane * VW < half;
    float s = 0.f;
    if constexpr (DT == BRL_I8) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < VW; ++e) m = fmaxf(m, fmaxf(fabsf(a.x[e]), fabsf(b.x[e])));
        if (!mine) m = 0.f;
#pragma unroll
        for (int x = 1; x < GS; x <<= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
        m = fmaxf(m, 1e-30f);
        s = 127.f / m;
        if (lane == 0) scales[idx] = m / 127.f;
    }
    char* row = pool + (size_t)idx * rowlen * kv_bytes(DT);
    if (mine) {
        store_elements<DT, VW>(row, lane * VW, a, s);
        store_elements<DT, VW>(row, half + lane * VW, b, s);
    } else if (dh + (lane - half / VW) * VW < rowlen) {          // zeros behind head_dim
        Floats<VW> z;
#pragma unroll
        for (int e = 0; e < VW; ++e) z.x[e] = 0.f;
        store_elements<DT, VW>(row, dh + (lane - half / VW) * VW, z, 0.f);
    }
}

constexpr int AP_THREADS = 256;

template <int DT, int DH>
__global__ __launch_bounds__(AP_THREADS) void cache_append_kernel(AppendArgs a) {
    constexpr int VW = DH % 8 == 0 ? 4 : 2;
    constexpr int GS = DH == 128 ? 16 : DH == 64 ? 8 : DH == 32 ? 4 : DH == 16 ? 2 : 32;
    constexpr int half = DH / 2;
    static_assert(GS * VW >= half && (DH % 16 == 0 || GS * VW - half >= 16 - DH % 16), "a group covers half a row and the padding");
    const int b = blockIdx.x / a.chunks, lane = threadIdx.x % GS;
    const StateTokens st = state_tokens(a.t, a.c, b);
    const int item = blockIdx.x % a.chunks * (AP_THREADS / GS) + threadIdx.x / GS;
    const int i = item / a.c.n_kv, h = item % a.c.n_kv;
    if (i >= st.n) return;                                        // (whole groups leave)
    const int slot = st.base + i;
    if (slot < 0) return;
    const int idx = kv_row_index(a.c, b, h, slot);
    if (idx < 0) return;
    const int row = st.row0 + i, pos = rope_position(a.t, row, slot);
    const int d = lane * VW < half ? lane * VW : 0;
    const float* kp = a.qkv + (size_t)row * ((a.n_heads + 2 * a.c.n_kv) * DH) + (a.n_heads + h) * DH + d;
    const Floats<VW> x = load_floats<VW>(kp), y = load_floats<VW>(kp + half);
    const Floats<VW> v0 = load_floats<VW>(kp + a.c.n_kv * DH), v1 = load_floats<VW>(kp + a.c.n_kv * DH + half);
    const Floats<VW> c = load_floats<VW>(a.t.cos_t + (size_t)pos * half + d), s = load_floats<VW>(a.t.sin_t + (size_t)pos * half + d);
    Floats<VW> k0, k1;
#pragma unroll
    for (int e = 0; e < VW; ++e) {
        k0.x[e] = x.x[e] * c.x[e] - y.x[e] * s.x[e];
        k1.x[e] = y.x[e] * c.x[e] + x.x[e] * s.x[e];
    }
    store_row<DT, VW, GS>(a.c.k, a.c.ks, idx, a.c.row, DH, k0, k1, lane);
    store_row<DT, VW, GS>(a.c.v, a.c.vs, idx, a.c.row, DH, v0, v1, lane);
}

template <int DT>
int append_typed(AppendArgs a, hipStream_t s) {
    const int dh = a.c.dh;
    const int gs = dh == 128 ? 16 : dh == 64 ? 8 : dh == 32 ? 4 : dh == 16 ? 2 : 32;
    a.chunks = (a.t.max_new * a.c.n_kv + AP_THREADS / gs - 1) / (AP_THREADS / gs);
    const dim3 grid((unsigned)a.chunks * (unsigned)a.t.B), block(AP_THREADS);
    switch (dh) {
        case 16: hipLaunchKernelGGL((cache_append_kernel<DT, 16>), grid, block, 0, s, a); break;
        case 32: hipLaunchKernelGGL((cache_append_kernel<DT, 32>), grid, block, 0, s, a); break;
        case 64: hipLaunchKernelGGL((cache_append_kernel<DT, 64>), grid, block, 0, s, a); break;
        case 100: hipLaunchKernelGGL((cache_append_kernel<DT, 100>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((cache_append_kernel<DT, 128>), grid, block, 0, s, a); break;
    }
    BRL_LAUNCH_CHECK("cache_append_kernel");
    return BRL_OK;
}

// ---- select ----
// One workgroup per list.  The threshold (the key of the last slot that is taken) is found bit group by bit group: a histogram
// of the next bits of the keys that agree with the threshold so far, scanned from the top.  Then one pass in slot order takes
// what lies above it and the first of those equal to it.
constexpr int SEL_THREADS = 1024, SEL_BINS = 2048;

struct SelectArgs {
    const float* weights;
    size_t ld;
    const int32_t* lens;
    int n_kv, max_len, keep, first, recent;
    int32_t *kept, *counts;
};

// order of floats as order of unsigned numbers; NaN counts as -inf, -0 as 0
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (!(w == w)) w = -INFINITY;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// sum over the workgroup of what lies in front of this thread, and the total
__device__ __forceinline__ uint32_t scan_before(uint32_t v, uint32_t* waves, uint32_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d, 64);
        if (lane >= d) x += y;
    }
    if (lane == 63) waves[wave] = x;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < SEL_THREADS / 64; ++w) {
        if (w < wave) before += waves[w];
        sum += waves[w];
    }
    total = sum;
    __syncthreads();
    return before + x - v;
}

__global__ __launch_bounds__(SEL_THREADS) void cache_select_kernel(SelectArgs a) {
    __shared__ uint32_t hist[SEL_BINS];
    __shared__ uint32_t waves[SEL_THREADS / 64];
    __shared__ uint32_t s_bin, s_above;
    const int b = blockIdx.x / a.n_kv, tid = threadIdx.x;
    const int len = clampi(a.lens[b], 0, a.max_len);
    int32_t* kept = a.kept + (size_t)blockIdx.x * a.keep;
    if (blockIdx.x % a.n_kv == 0 && tid == 0) a.counts[b] = len < a.keep ? len : a.keep;
    if (len <= a.keep) {
        for (int i = tid; i < a.keep; i += SEL_THREADS) kept[i] = i < len ? i : -1;
        return;
    }
    const int mid = a.keep - a.first - a.recent;      // to be taken out of slots first .. len - recent - 1, more than mid of them
    const int lo = a.first, hi = len - a.recent;
    for (int i = tid; i < a.first; i += SEL_THREADS) kept[i] = i;
    for (int i = tid; i < a.recent; i += SEL_THREADS) kept[a.first + mid + i] = hi + i;
    if (mid == 0) return;
    const float* w = a.weights + (size_t)blockIdx.x * a.ld;
    uint32_t prefix = 0, want = mid;                  // still to be taken among the keys that begin with prefix
    int shift = 32;
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, above = shift;
        shift -= bits;
        for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[i] = 0;
        __syncthreads();
        for (int i = lo + tid; i < hi; i += SEL_THREADS) {
            const uint32_t k = weight_key(w[i]);
            if (above == 32 || (k >> above) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        // bins from the top: thread t has bins top - 2 t and top - 2 t - 1
        const int top = (1 << bits) - 1, b0 = top - 2 * tid, b1 = b0 - 1;
        const uint32_t h0 = b0 >= 0 ? hist[b0] : 0, h1 = b1 >= 0 ? hist[b1] : 0;
        uint32_t total;
        const uint32_t before = scan_before(h0 + h1, waves, total);
        if (before < want && want <= before + h0) { s_bin = b0; s_above = before; }
        else if (before + h0 < want && want <= before + h0 + h1) { s_bin = b1; s_above = before + h0; }
        __syncthreads();
        prefix = (prefix << bits) | s_bin;
        want -= s_above;
        __syncthreads();
    }
    // in slot order: all above the threshold, the first `want` equal to it
    uint32_t greater = 0, equal = 0;                  // so far
    for (int i0 = lo; i0 < hi; i0 += SEL_THREADS) {
        const int i = i0 + tid;
        const uint32_t k = i < hi ? weight_key(w[i]) : 0;
        const bool g = i < hi && k > prefix, e = i < hi && k == prefix;
        uint32_t total;
        const uint32_t before = scan_before((g ? 1u : 0u) | (e ? 0x10000u : 0u), waves, total);
        const uint32_t eb = equal + (before >> 16), gb = greater + (before & 0xffffu);
        if (g || (e && eb < want)) kept[a.first + gb + (eb < want ? eb : want)] = i;
        greater += total & 0xffffu;
        equal += total >> 16;
    }
}

// ---- compact ----
// Rows move to lower slots of the same pages (kept[i] >= start + i).  One workgroup owns one column slice of the rows of one
// head and walks them in ascending order, a chunk at a time: what a chunk overwrites lies below the sources of every later
// chunk, so the only order needed is that all of a chunk has been read before any of it is written.
constexpr int CP_THREADS = 256, CP_ITEMS = 8, CP_INFLIGHT = CP_THREADS * CP_ITEMS;

template <class T>
__device__ __forceinline__ void move_rows(const CompactArgs& a, T* pool, size_t row_units, int first_unit, int units, int b, int h, int len,
                                          int start, int count, bool paged) {
    const int32_t* kept = a.kept + ((size_t)b * a.kept_heads + (a.kept_heads == 1 ? 0 : h)) * a.ld_kept;
    const int rows = CP_INFLIGHT / units;             // of a chunk
    for (int r0 = 0; r0 < count; r0 += rows) {
        T v[CP_ITEMS];
        long long to[CP_ITEMS];
#pragma unroll
        for (int e = 0; e < CP_ITEMS; ++e) {
            const int item = e * CP_THREADS + threadIdx.x, r = r0 + item / units, u = first_unit + item % units;
            to[e] = -1;
            if (item >= rows * units || r >= count) continue;
            const int src = kept[r], dst = start + r;
            if (src <= dst || src >= len) continue;
            const int from = paged ? kv_row_index(a.c, b, h, src) : src;
            const int at = paged ? kv_row_index(a.c, b, h, dst) : dst;
            if (from < 0 || at < 0) continue;
            v[e] = pool[(size_t)from * row_units + u];
            to[e] = (long long)at * (long long)row_units + u;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // read, not only requested
        __syncthreads();
#pragma unroll
        for (int e = 0; e < CP_ITEMS; ++e)
            if (to[e] >= 0) pool[to[e]] = v[e];
    }
}

__global__ __launch_bounds__(CP_THREADS) void cache_compact_kernel(CompactArgs a, int slices, int units, int row_units) {
    const int parts = 2 * slices + 1;
    const int part = blockIdx.x % parts, h = blockIdx.x / parts % a.c.n_kv, b = blockIdx.x / (parts * a.c.n_kv);
    const int len = clampi(a.lens[b], 0, a.max_len);
    const int start = a.start ? clampi(a.start[b], 0, len) : 0;
    const int most = len - start < a.ld_kept ? len - start : a.ld_kept;
    const int count = clampi(a.counts[b], 0, most);
    if (part < 2 * slices) {
        const int first = part % slices * units;
        const int n = row_units - first < units ? row_units - first : units;
        move_rows(a, reinterpret_cast<uint4*>(part < slices ? a.c.k : a.c.v), (size_t)row_units, first, n, b, h, len, start, count, true);
        return;
    }
    if (a.c.dtype == BRL_I8) {
        move_rows(a, a.c.ks, 1, 0, 1, b, h, len, start, count, true);
        move_rows(a, a.c.vs, 1, 0, 1, b, h, len, start, count, true);
    }
    if (a.weights) move_rows(a, a.weights + ((size_t)b * a.c.n_kv + h) * a.ld_weights, 1, 0, 1, b, h, len, start, count, false);
}

}  // namespace

int launch_cache_append(const KvView& c, const NewTokens& t, const float* qkv, int n_heads, hipStream_t s) {
    AppendArgs a;
    a.c = c; a.t = t; a.qkv = qkv; a.n_heads = n_heads;
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    return c.dtype == BRL_F32 ? append_typed<BRL_F32>(a, s) : c.dtype == BRL_F16 ? append_typed<BRL_F16>(a, s) : append_typed<BRL_I8>(a, s);
}

int launch_cache_select(const float* weights, size_t ld_weights, int B, int n_kv, const int32_t* lens, int max_len, int keep,
                        int first, int recent, int32_t* kept, int32_t* counts, hipStream_t s) {
    SelectArgs a;
    a.weights = weights; a.ld = ld_weights; a.lens = lens; a.n_kv = n_kv; a.max_len = max_len; a.keep = keep;
    a.first = first; a.recent = recent; a.kept = kept; a.counts = counts;
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    hipLaunchKernelGGL(cache_select_kernel, dim3((unsigned)(B * n_kv)), dim3(SEL_THREADS), 0, s, a);
    BRL_LAUNCH_CHECK("cache_select_kernel");
    return BRL_OK;
}

int launch_cache_compact(const CompactArgs& a, hipStream_t s) {
    const int row_units = a.c.row * kv_bytes(a.c.dtype) / 16;
    const int units = row_units < 4 ? row_units : 4, slices = (row_units + units - 1) / units;
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    hipLaunchKernelGGL(cache_compact_kernel, dim3((unsigned)(a.B * a.c.n_kv * (2 * slices + 1))), dim3(CP_THREADS), 0, s, a, slices, units,
                       row_units);
    BRL_LAUNCH_CHECK("cache_compact_kernel");
    return BRL_OK;
}

}  // namespace brl
