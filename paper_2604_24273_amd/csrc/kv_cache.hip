// The paged key/value cache apart from attention: storing new tokens, choosing which slots to keep, moving them together.
#include <type_traits>

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
__device__ __forceinline__ void store_row(char* pool, float* scales, int idx, int rowlen, int dh, Floats<VW> a, Floats<VW> b, int lane) {
    const int half = dh / 2;
    const bool mine = lane * VW < half;
    float s = 0.f;
    if constexpr (DT == BRL_I8) {
        // |x| in the order of its bits: a NaN is above infinity and so becomes the row's scale
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            const uint32_t x = __float_as_uint(a.x[e]) & 0x7fffffffu, y = __float_as_uint(b.x[e]) & 0x7fffffffu;
            top = top > x ? top : x;
            top = top > y ? top : y;
        }
        if (!mine) top = 0;
#pragma unroll
        for (int x = 1; x < GS; x <<= 1) {
            const uint32_t y = __shfl_xor(top, x, 64);
            top = top > y ? top : y;
        }
        float m = __uint_as_float(top);
        m = m < 1e-30f ? 1e-30f : m;
        s = 127.f / m;
        if (lane == 0) scales[idx] = m / 127.f;
        if (!(m < INFINITY)) {                                    // no numbers in this row: codes of zero
#pragma unroll
            for (int e = 0; e < VW; ++e) a.x[e] = b.x[e] = 0.f;
            s = 0.f;
        }
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
constexpr int SEL_THREADS = 1024, SEL_BINS = 2048, PARTS = SEL_THREADS / 64;

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

// inclusive sum over a wavefront: rows of 16 lanes, then across them (data-parallel primitives, no trip through LDS)
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);       // from 1, 2, 4, 8 lanes below, inside a row
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);       // row 0's sum to row 1, row 2's to row 3
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);       // lane 31's to rows 2 and 3
    return v;
}
// sum over the workgroup of what lies in front of this thread
__device__ __forceinline__ uint32_t scan_before(uint32_t a, uint32_t* waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t x = wave_scan(a);
    if (lane == 63) waves[wave] = x;
    __syncthreads();
    const uint32_t p = wave_scan(lane < PARTS ? waves[lane % PARTS] : 0u);     // every wavefront scans the wavefronts' totals itself
    return x - a + (wave ? lane_value(p, wave - 1) : 0u);
}

// HELD: quads of weights that a thread keeps in registers, every 4096 slots one (all of a list in 4096 HELD slots); 0: the list is read
// again for each pass, 4096 slots at a time.  8000 slots, 320 lists: 20.4 us when every list was read four times.  60000 slots, 20 lists:
// 40 us when a thread had 64 neighbouring slots, 28 now.
// WHOLE: rows of weights start on 16 bytes.
template <int HELD, bool WHOLE>
__global__ __launch_bounds__(SEL_THREADS) void cache_select_kernel(SelectArgs a) {
    // Weights crowd into few bins of the first pass (their exponents): copies of each bin, side by side in neighbouring banks, so that a
    // wavefront's lanes do not queue for one address.
    constexpr int COPIES = HELD > 4 ? 16 : 8;         // (a list of many slots has the compute unit to itself)
    __shared__ __attribute__((aligned(16))) uint32_t hist[SEL_BINS * COPIES];
    __shared__ uint32_t waves[PARTS];
    __shared__ uint32_t s_bin, s_above;
    constexpr int Q = HELD ? HELD : 1, STEP = 4 * SEL_THREADS;
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
    const float* w = a.weights + (size_t)blockIdx.x * a.ld;
    uint32_t key[4 * Q];                              // 0 (below every key of a weight) outside lo .. hi - 1
    // (loads past the list read its row's end, not used: a load that might not happen is waited for before the next)
    const int row_end = a.ld < (size_t)hi + 3 ? (int)a.ld : hi + 3;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto quads = [&](int step) {                      // how many of this wavefront's hold any slot of the list
        const int n = (hi - step * STEP - wave * 256 + STEP - 1) / STEP;
        return n < Q ? n : Q;
    };
    auto read = [&](int step) {                       // quads 4096 slots apart
        const int i0 = step * STEP + tid * 4;
        if constexpr (WHOLE) {
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                const int i = i0 + j * STEP, at = i + 4 <= row_end ? i : (row_end & ~3) - 4;
                const float4 x = *reinterpret_cast<const float4*>(w + (at < 0 ? 0 : at));
                key[4 * j] = __float_as_uint(x.x); key[4 * j + 1] = __float_as_uint(x.y);
                key[4 * j + 2] = __float_as_uint(x.z); key[4 * j + 3] = __float_as_uint(x.w);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4 * Q; ++e) {
                const int i = i0 + e / 4 * STEP + e % 4;
                key[e] = __float_as_uint(w[i < hi ? i : hi - 1]);
            }
        }
        const int n = quads(step);
#pragma unroll
        for (int j = 0; j < Q; ++j) {
            if (j >= n) continue;                     // (its keys are not looked at)
#pragma unroll
            for (int e = 4 * j; e < 4 * j + 4; ++e) {
                const int i = i0 + j * STEP + e % 4;
                key[e] = weight_key(__uint_as_float(key[e])) & ((unsigned)(i - lo) < (unsigned)(hi - lo) ? ~0u : 0u);
            }
        }
    };
    const int steps = HELD ? 1 : (hi + STEP - 1) / STEP;
    if (HELD) read(0);
    for (int i = tid; i < a.first; i += SEL_THREADS) kept[i] = i;
    for (int i = tid; i < a.recent; i += SEL_THREADS) kept[a.first + mid + i] = hi + i;
    if (mid == 0) return;
    uint32_t prefix = 0, want = mid;                  // still to be taken among the keys that begin with prefix
    auto pass = [&](auto number) __attribute__((always_inline)) {
        constexpr int P = decltype(number)::value, BITS = P < 2 ? 11 : 10, SHIFT = P == 0 ? 21 : P == 1 ? 10 : 0;
        for (int i = tid; i < SEL_BINS * COPIES / 4; i += SEL_THREADS) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        uint32_t* const mine = hist + tid % COPIES;
        for (int step = 0; step < steps; ++step) {
            if (!HELD) read(step);
            const int n = quads(step);
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                if (j >= n) continue;                 // (a loop with an end of its own would have the keys in memory)
#pragma unroll
                for (int e = 4 * j; e < 4 * j + 4; ++e) {
                    // (0, no slot's key, falls into bin 0 of the first pass, far below the threshold: -inf is in bin 3)
                    const bool in = P == 0 || key[e] - (prefix << (SHIFT + BITS & 31)) < (1u << (SHIFT + BITS & 31));
                    if (in) atomicAdd(mine + (key[e] >> SHIFT & ((1u << BITS) - 1)) * COPIES, 1u);
                }
            }
        }
        __syncthreads();
        // bins from the top: thread t has bins top - 2 t and top - 2 t - 1, neighbours in LDS.  (Their copies sixteen bytes at a time, each
        // lane from another place on, so that sixteen lanes are on all banks.)
        constexpr int TOP = (1 << BITS) - 1, CHUNKS = COPIES / 2;
        const int b0 = TOP - 2 * tid, b1 = b0 - 1;
        uint32_t h0 = 0, h1 = 0;
        if (b1 >= 0) {
#pragma unroll
            for (int x = 0; x < CHUNKS; ++x) {
                const int at = (x + tid / (16 / CHUNKS)) % CHUNKS;
                const uint4 f = reinterpret_cast<const uint4*>(hist)[CHUNKS / 2 * b1 + at];
                const uint32_t n = f.x + f.y + f.z + f.w;
                h0 += at < CHUNKS / 2 ? 0u : n;
                h1 += at < CHUNKS / 2 ? n : 0u;
            }
        }
        const uint32_t before = scan_before(h0 + h1, waves);
        if (before < want && want <= before + h0) { s_bin = b0; s_above = before; }
        else if (before + h0 < want && want <= before + h0 + h1) { s_bin = b1; s_above = before + h0; }
        __syncthreads();
        prefix = (prefix << BITS) | s_bin;
        want -= s_above;
    };
    pass(std::integral_constant<int, 0>());
    pass(std::integral_constant<int, 1>());
    pass(std::integral_constant<int, 2>());
    // in slot order: all above the threshold, the first `want` equal to it.  What lies in front of a quad: in its wavefront's part of the
    // step (above | equal << 16), in front of that part.
    __shared__ uint32_t part[Q * PARTS];
    __shared__ uint2 front[Q * PARTS];
    uint32_t greater = 0, equal = 0;                  // in front of the step
    for (int step = 0; step < steps; ++step) {
        int i0 = step * STEP + tid * 4;
        if (!HELD) read(step);
        asm volatile("" : "+v"(i0));                  // (opaque: or all slots' numbers are kept in registers from the first read on)
        uint32_t mine[Q];
        const int live = quads(step);
#pragma unroll
        for (int j = 0; j < Q; ++j) {
            mine[j] = 0;
            if (j >= live) {
                if (lane == 0) part[j * PARTS + wave] = 0;
                continue;
            }
            uint32_t over = 0, least = 0;             // above the threshold; not below it
#pragma unroll
            for (int e = 4 * j; e < 4 * j + 4; ++e) {
                over += key[e] > prefix;
                least += key[e] >= prefix;
            }
            const uint32_t n = over | (least - over) << 16;
            const uint32_t x = wave_scan(n);
            if (lane == 63) part[j * PARTS + wave] = x;
            mine[j] = x - n;
        }
        __syncthreads();
        uint32_t all_g, all_q;
        if (wave == 0) {
            constexpr int PER = (Q * PARTS + 63) / 64;
            uint32_t g[PER], q[PER], sum_g = 0, sum_q = 0;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const uint32_t n = lane * PER + x < Q * PARTS ? part[lane * PER + x] : 0u;
                g[x] = n & 0xffffu; q[x] = n >> 16;
                sum_g += g[x]; sum_q += q[x];
            }
            uint32_t at_g = wave_scan(sum_g), at_q = wave_scan(sum_q);
            all_g = lane_value(at_g, 63); all_q = lane_value(at_q, 63);
            at_g -= sum_g; at_q -= sum_q;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                if (lane * PER + x < Q * PARTS) front[lane * PER + x] = make_uint2(greater + at_g, equal + at_q);
                at_g += g[x]; at_q += q[x];
            }
            greater += all_g;                         // (of wavefront 0, which counts on)
            equal += all_q;
        }
        __syncthreads();
        // Through LDS, so that they leave in whole lines (320 times 2048 of 4000 - 8000 slots: 11.8 us, 12.1 without).
        constexpr uint32_t ROOM = SEL_BINS * COPIES;
        for (uint32_t from = 0; from < (uint32_t)mid; from += ROOM) {
            asm volatile("" : "+v"(i0));              // (opaque: see above)
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                if (j >= live) continue;
                const uint2 f = front[j * PARTS + wave];
                uint32_t qb = f.y + (mine[j] >> 16);
                uint32_t at = f.x + (mine[j] & 0xffffu) + (qb < want ? qb : want) - from;
#pragma unroll
                for (int e = 4 * j; e < 4 * j + 4; ++e) {
                    const bool same = key[e] == prefix, take = key[e] > prefix || (same && qb < want);
                    const int slot = i0 + j * STEP + e % 4;
                    if constexpr (HELD) {
                        if (take && at < ROOM) hist[at] = slot;
                    } else {
                        if (take) kept[a.first + at] = slot;
                    }
                    at += take;
                    qb += same;
                }
            }
            if (!HELD) break;
            __syncthreads();
            const uint32_t n = mid - from < ROOM ? mid - from : ROOM;
            for (uint32_t i = tid; i < n; i += SEL_THREADS) kept[a.first + from + i] = hist[i];
            __syncthreads();
        }
    }
}

// ---- compact ----
// Rows move to lower slots of the same pages (kept[i] >= start + i).  One workgroup owns one column slice of the rows of one
// head and walks them in ascending order, a chunk at a time: what a chunk overwrites lies below the sources of every later
// chunk, so the only order needed is that all of a chunk has been read before any of it is written.  While a chunk's rows are
// on their way the places of the next chunk's are looked up (list, then page table).
constexpr int CP_ITEMS = 8;                           // sixteen bytes of a thread in a chunk

typedef uint32_t chunk16 __attribute__((ext_vector_type(4)));

struct Move {
    const CompactArgs& a;
    const int32_t* kept;
    int b, h, len, start, count;
    bool paged;
    // row indices of entry r's source and target, from = -1: nothing moves
    __device__ __forceinline__ int2 place(int r) const {
        if (r >= count) return make_int2(-1, -1);
        const int src = kept[r], dst = start + r;
        if (src <= dst || src >= len) return make_int2(-1, -1);
        if (!paged) return make_int2(src, dst);
        const int from = kv_row_index(a.c, b, h, src), at = kv_row_index(a.c, b, h, dst);
        return at < 0 ? make_int2(-1, -1) : make_int2(from, at);
    }
};

// units `first` .. first + units - 1 of every row, rows of `row_units` units of type T
template <int THREADS, class T>
__device__ __forceinline__ void move_rows(const Move& m, T* pool, int row_units, int first, int units, int2* places) {
    constexpr int INFLIGHT = THREADS * CP_ITEMS;
    const int rows = INFLIGHT / units;             // of a chunk
    const int tid = threadIdx.x, q = THREADS / units, rem = THREADS % units;
    for (int i = tid; i < rows; i += THREADS) places[i] = m.place(i);
    __syncthreads();
    int buf = 0;
    for (int r0 = 0; r0 < m.count; r0 += rows) {
        T v[CP_ITEMS];
        size_t to[CP_ITEMS];
        bool moves[CP_ITEMS];
        int r = tid / units, u = tid % units;
#pragma unroll
        for (int e = 0; e < CP_ITEMS; ++e) {
            // (what does not move reads row 0: loads that might not happen would each be waited for)
            const int2 x = r < rows ? places[buf * INFLIGHT + r] : make_int2(-1, -1);
            moves[e] = x.x >= 0;
            v[e] = pool[(size_t)(moves[e] ? x.x : 0) * row_units + first + u];
            to[e] = (size_t)(moves[e] ? x.y : 0) * row_units + first + u;
            r += q;
            u += rem;
            if (u >= units) {
                u -= units;
                ++r;
            }
        }
        buf ^= 1;
        if (r0 + rows < m.count)
            for (int i = tid; i < rows; i += THREADS) places[buf * INFLIGHT + i] = m.place(r0 + rows + i);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // read, not only requested
        __syncthreads();
#pragma unroll
        for (int e = 0; e < CP_ITEMS; ++e)
            if (moves[e]) pool[to[e]] = v[e];
    }
    __syncthreads();
}

// How a row of k or v is cut into slices of `units` times 16 bytes.  Slices that share 128 bytes (`near` of them) are workgroups whose
// numbers differ by multiples of 8: they run on one die, whose L2 so fetches the line once.
struct Slices {
    int units, row_units, count, near, lines;         // lines: of a row, count / near rounded up
    int main_blocks;                                  // workgroups for k and v; behind them one per list for scales and weights
};
template <int THREADS>
__global__ __launch_bounds__(THREADS) void cache_compact_kernel(CompactArgs a, Slices sl) {
    __shared__ int2 places[2 * THREADS * CP_ITEMS];
    int list, slice = 0, line = 0;
    const bool rows = blockIdx.x < (unsigned)sl.main_blocks;
    if (rows) {
        const int many = 8 * sl.near, r = blockIdx.x % many;
        line = blockIdx.x / many * 8 + r % 8;         // of all lists' keys and values
        list = line / (2 * sl.lines);
        slice = line % sl.lines * sl.near + r / 8;
        if (list >= a.B * a.c.n_kv || slice >= sl.count) return;
    } else {
        list = blockIdx.x - sl.main_blocks;
    }
    const int h = list % a.c.n_kv, b = list / a.c.n_kv;
    const int len = clampi(a.lens[b], 0, a.max_len);
    const int start = a.start ? clampi(a.start[b], 0, len) : 0;
    const int most = len - start < a.ld_kept ? len - start : a.ld_kept;
    Move m = {a, a.kept + ((size_t)b * a.kept_heads + (a.kept_heads == 1 ? 0 : h)) * a.ld_kept, b, h, len, start, clampi(a.counts[b], 0, most), true};
    if (rows) {
        const int first = slice * sl.units;
        move_rows<THREADS>(m, reinterpret_cast<chunk16*>(line / sl.lines % 2 ? a.c.v : a.c.k), sl.row_units, first,
                  sl.row_units - first < sl.units ? sl.row_units - first : sl.units, places);
        return;
    }
    if (a.c.dtype == BRL_I8) {
        move_rows<THREADS>(m, a.c.ks, 1, 0, 1, places);
        move_rows<THREADS>(m, a.c.vs, 1, 0, 1, places);
    }
    m.paged = false;
    if (a.weights) move_rows<THREADS>(m, a.weights + ((size_t)b * a.c.n_kv + h) * a.ld_weights, 1, 0, 1, places);
}

}  // namespace

int launch_cache_append(const KvView& c, const NewTokens& t, const float* qkv, int n_heads, hipStream_t s) {
    AppendArgs a;
    a.c = c; a.t = t; a.qkv = qkv; a.n_heads = n_heads;
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    return c.dtype == BRL_F32 ? append_typed<BRL_F32>(a, s) : c.dtype == BRL_F16 ? append_typed<BRL_F16>(a, s) : append_typed<BRL_I8>(a, s);
}

template <bool WHOLE>
static void select_held(const SelectArgs& a, int lists, hipStream_t s) {
    const dim3 grid((unsigned)lists), block(SEL_THREADS);
    constexpr int ONE = 4 * SEL_THREADS;
    if (a.max_len <= ONE) hipLaunchKernelGGL((cache_select_kernel<1, WHOLE>), grid, block, 0, s, a);
    else if (a.max_len <= 2 * ONE) hipLaunchKernelGGL((cache_select_kernel<2, WHOLE>), grid, block, 0, s, a);
    else if (a.max_len <= 4 * ONE) hipLaunchKernelGGL((cache_select_kernel<4, WHOLE>), grid, block, 0, s, a);
    else if (a.max_len <= 16 * ONE) hipLaunchKernelGGL((cache_select_kernel<16, WHOLE>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((cache_select_kernel<0, WHOLE>), grid, block, 0, s, a);
}

int launch_cache_select(const float* weights, size_t ld_weights, int B, int n_kv, const int32_t* lens, int max_len, int keep,
                        int first, int recent, int32_t* kept, int32_t* counts, hipStream_t s) {
    SelectArgs a;
    a.weights = weights; a.ld = ld_weights; a.lens = lens; a.n_kv = n_kv; a.max_len = max_len; a.keep = keep;
    a.first = first; a.recent = recent; a.kept = kept; a.counts = counts;
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    const bool whole = ((ld_weights | (size_t)(reinterpret_cast<uintptr_t>(weights) >> 2)) & 3) == 0;
    whole ? select_held<true>(a, B * n_kv, s) : select_held<false>(a, B * n_kv, s);
    BRL_LAUNCH_CHECK("cache_select_kernel");
    return BRL_OK;
}

int launch_cache_compact(const CompactArgs& a, hipStream_t s) {
    const int row_units = a.c.row * kv_bytes(a.c.dtype) / 16;
    // A workgroup has 8 x 16 bytes per thread under way and pays a chunk's way from memory each time (5 us): where lists are few they take
    // 1024 threads, which fill a compute unit, and rows are cut, down to 32 bytes, into as many slices as there are units.  Keys and values
    // of fp16, us with 256 threads and up to 512 workgroups / so: 20 lists of 7000 slots 69 / 48, 6 heads of 64, 24000 slots 92 / 58,
    // 65 of 1000 19 / 18; fp32, 50 of 11000 173 / 160.  More than 256 workgroups: 205 lists of 500 slots 18 / 24.
    int slices = 1;
    while ((long long)a.B * a.c.n_kv * 4 * slices <= 256 && row_units / (2 * slices) >= 2) slices *= 2;
    Slices sl;
    sl.row_units = row_units;
    sl.units = (row_units + slices - 1) / slices;
    sl.count = (row_units + sl.units - 1) / sl.units;
    sl.near = sl.units >= 8 ? 1 : 8 / sl.units < sl.count ? 8 / sl.units : sl.count;
    sl.lines = (sl.count + sl.near - 1) / sl.near;
    sl.main_blocks = (a.B * a.c.n_kv * 2 * sl.lines + 7) / 8 * 8 * sl.near;
    const int others = a.c.dtype == BRL_I8 || a.weights ? a.B * a.c.n_kv : 0;
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    const dim3 grid((unsigned)(sl.main_blocks + others));
    const bool large = (long long)a.B * a.c.n_kv * 2 * sl.count <= 256 && a.ld_kept > 256 * CP_ITEMS / sl.units;      // (and several chunks)
    if (large) hipLaunchKernelGGL(cache_compact_kernel<1024>, grid, dim3(1024), 0, s, a, sl);
    else hipLaunchKernelGGL(cache_compact_kernel<256>, grid, dim3(256), 0, s, a, sl);
    BRL_LAUNCH_CHECK("cache_compact_kernel");
    return BRL_OK;
}

}  // namespace brl
