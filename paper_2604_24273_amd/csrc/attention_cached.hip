// Attention of new tokens over a paged key/value cache, on the matrix cores.
//
// Rows: the new tokens of a state times the query heads of one k/v head, row r = token r / group, head r % group.  Every
// row of a state reads the same keys and values, so 16 rows are one column block of v_mfma_f32_16x16x32_f16:
//   S^T (16 keys x 16 rows) = K (16 x 32 components) Q^T,   O^T (16 components x 16 rows) += V^T (16 x 32 keys) P^T.
// fp32 operands are carried as fp16 hi + lo pairs (the query rows and the probabilities always, keys and values of an fp32 cache):
// products with one such operand take two matrix instructions, with two three (lo * lo is dropped).  int8 codes are exact
// in fp16; a key's scale multiplies its scores, a value's scale its probabilities.
//
// Order of the keys.  A block of 32 keys is two key tiles; row 4 a + r of tile t is key 8 a + 4 t + r.  Lane l = 16 g + c of
// S^T then holds row c's scores of the keys 8 g .. 8 g + 7, and those are the eight contraction slots that lane has to
// fill as operand P of the second product: the probabilities never leave their lane.
#include <cstring>

#include "common.hpp"

namespace brl {

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __fp16 v4fp __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
// Probabilities are carried as 2^(s - m + P_SHIFT) with m the running maximum, which follows the true one only once that is
// P_SLACK ahead: at most 2^14, inside fp16, while parts down to 2^-38 of the largest keep their hi and lo planes apart.
constexpr float P_SHIFT = 6.f, P_SLACK = 8.f;

// fp16 hi and lo of two values, each rounded once (x - hi is exact; the multiply-add rounds it to fp16 directly)
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t& hi, uint32_t& lo) {
    v2h h = {(_Float16)x0, (_Float16)x1};
    hi = __builtin_bit_cast(uint32_t, h);
    float one = 1.0f;                                // (opaque, or the compiler takes the steps apart into more instructions)
    asm("" : "+s"(one));
    asm("" : "+v"(hi));
    h = __builtin_bit_cast(v2h, hi);
    const v2h l = {(_Float16)__builtin_fmaf(x0, one, -(float)h[0]), (_Float16)__builtin_fmaf(x1, one, -(float)h[1])};
    lo = __builtin_bit_cast(uint32_t, l);
}

// four int8 codes to fp16: byte u = code ^ 0x80 under the exponent of 1024 is 1024 + u = 1152 + code
__device__ __forceinline__ void widen_codes(uint32_t q, uint32_t& h01, uint32_t& h23) {
    const uint32_t u = q ^ 0x80808080u;
    const v2h off = {(_Float16)1152.f, (_Float16)1152.f};
    h01 = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off);
    h23 = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off);
}

template <int DT_, int DH_>
struct Shape {
    static constexpr int DT = DT_, DH = DH_;
    static constexpr int SZ = DT == BRL_F32 ? 4 : DT == BRL_F16 ? 2 : 1;
    static constexpr int ROW = (DH + 15) / 16 * 16, RB = ROW * SZ;     // a row of the cache: elements, bytes
    static constexpr int CPR = RB / 16;                                // 16-byte chunks
    static constexpr int KS = (DH + 31) / 32, DTL = ROW / 16;          // contraction steps of a score, component tiles of a sum
    static constexpr int PL = DT == BRL_F32 ? 2 : 1;                   // planes of keys and values
    static constexpr int NCH = ROW / 8 <= 8 ? ROW / 8 : 16;            // 16-byte chunks of a row of halfs in LDS
    static constexpr int LS = NCH * 16, PLANE = 32 * LS;               // bytes of such a row, of a block's plane
    static constexpr int LDS = PL * PLANE;
    static constexpr int NV = (32 * CPR + 63) / 64;                    // loads of a wavefront for a block of rows
    static constexpr int KL = DT == BRL_F32 ? 2 : 1;                   // 16-byte (int8: 8-byte) loads of a key fragment
};

// Where chunk c of a key's row lies in LDS.  The chunks of a row are permuted by bits of the key such that both the 16 rows
// x 16 bytes of a key fragment and the 16 rows x 32 bytes of a transposing read fall on all banks.
template <class S>
__device__ __forceinline__ int lds_chunk(int key, int c) {
    int f;
    if constexpr (S::NCH == 16) f = (key & 3) | ((key >> 1) & 12);
    else if constexpr (S::NCH == 8) f = ((key >> 1) & 1) | ((key >> 2) & 6);
    else if constexpr (S::NCH == 4) f = (key >> 3) & 3;
    else f = (key >> 3) & 1;
    return key * S::LS + ((c ^ f) << 4);
}

// ---- a state's block of 32 slots: where its two halves of 16 lie (pages hold 16 at least) ----
struct Block {
    long long lo, hi;         // rows of the pool, -1: not there
};

template <int DT>
struct Raw { typedef uint4 type; };
template <>
struct Raw<BRL_I8> { typedef uint2 type; };

// Fragments of the keys straight from the pool: lane 16 g + c reads, of the key in row c of each tile, components 32 s + 8 g on.
template <class S>
struct KeyLoads {
    typename Raw<S::DT>::type raw[2][S::KS][S::KL];
    __device__ __forceinline__ void request(const char* pool, const Block& b, int lane) {
        const int c = lane & 15, g = lane >> 4;
        const long long row = (c >> 3) ? b.hi : b.lo;
        const char* p = pool + (row < 0 ? 0 : row) * (long long)S::RB + (((c >> 2) & 1) * 8 + (c & 3)) * S::RB + 8 * g * S::SZ;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < S::KS; ++s) {
                const char* q = p + t * 4 * S::RB + s * 32 * S::SZ;
                if (S::KS * 32 > S::ROW && s == S::KS - 1 && 32 * s + 8 * g + 8 > S::ROW) q = p;      // (a row ends inside the step)
#pragma unroll
                for (int i = 0; i < S::KL; ++i) raw[t][s][i] = reinterpret_cast<const typename Raw<S::DT>::type*>(q)[i];
            }
    }
    __device__ __forceinline__ void fragment(int t, int s, int lane, v8h (&f)[S::PL]) const {
        uint32_t w[S::PL][4];
        if constexpr (S::DT == BRL_F32) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 r = raw[t][s][i];
                split_pair(__uint_as_float(r.x), __uint_as_float(r.y), w[0][2 * i], w[1][2 * i]);
                split_pair(__uint_as_float(r.z), __uint_as_float(r.w), w[0][2 * i + 1], w[1][2 * i + 1]);
            }
        } else if constexpr (S::DT == BRL_F16) {
            const uint4 r = raw[t][s][0];
            w[0][0] = r.x; w[0][1] = r.y; w[0][2] = r.z; w[0][3] = r.w;
        } else {
            const uint2 r = raw[t][s][0];
            widen_codes(r.x, w[0][0], w[0][1]);
            widen_codes(r.y, w[0][2], w[0][3]);
        }
        if (S::KS * 32 > S::DH && s == S::KS - 1) {                    // what lies behind head_dim is not a number
            const int valid = S::DH - (32 * s + 8 * (lane >> 4));
#pragma unroll
            for (int p = 0; p < S::PL; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[p][j] = 2 * j < valid ? w[p][j] : 0u;
        }
#pragma unroll
        for (int p = 0; p < S::PL; ++p) f[p] = __builtin_bit_cast(v8h, make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]));
    }
};

// Rows of the values, 16 bytes per lane in the order of the pool, and from there as halfs into LDS.
template <class S>
struct ValueLoads {
    uint4 raw[S::NV];
    __device__ __forceinline__ void request(const char* pool, const Block& b, int lane) {
        const char* lo = pool + (b.lo < 0 ? 0 : b.lo) * (long long)S::RB;
        const char* hi = pool + (b.hi < 0 ? 0 : b.hi) * (long long)S::RB - 16 * S::RB;
#pragma unroll
        for (int i = 0; i < S::NV; ++i) {
            const int idx = i * 64 + lane;
            if (S::NV * 64 > 32 * S::CPR && idx >= 32 * S::CPR) continue;
            raw[i] = *reinterpret_cast<const uint4*>((idx >= 16 * S::CPR ? hi : lo) + idx * 16);
        }
    }
    // there: keys first .. last - 1 of the block hold numbers (the others are stored as zeros)
    template <bool MASK>
    __device__ __forceinline__ void store(char* lds, int lane, uint32_t there) const {
#pragma unroll
        for (int i = 0; i < S::NV; ++i) {
            const int idx = i * 64 + lane, key = idx / S::CPR, c = idx % S::CPR;
            if (S::NV * 64 > 32 * S::CPR && idx >= 32 * S::CPR) continue;
            uint4 r = raw[i];
            if (MASK && !(there >> key & 1u)) r = make_uint4(0, 0, 0, 0);
            if constexpr (S::DT == BRL_F16) {
                *reinterpret_cast<uint4*>(lds + lds_chunk<S>(key, c)) = r;
            } else if constexpr (S::DT == BRL_F32) {
                uint2 h, l;
                split_pair(__uint_as_float(r.x), __uint_as_float(r.y), h.x, l.x);
                split_pair(__uint_as_float(r.z), __uint_as_float(r.w), h.y, l.y);
                char* p = lds + lds_chunk<S>(key, c >> 1) + (c & 1) * 8;
                *reinterpret_cast<uint2*>(p) = h;
                *reinterpret_cast<uint2*>(p + S::PLANE) = l;
            } else {
                uint4 a, b;
                widen_codes(r.x, a.x, a.y);
                widen_codes(r.y, a.z, a.w);
                widen_codes(r.z, b.x, b.y);
                widen_codes(r.w, b.z, b.w);
                *reinterpret_cast<uint4*>(lds + lds_chunk<S>(key, 2 * c)) = a;
                *reinterpret_cast<uint4*>(lds + lds_chunk<S>(key, 2 * c + 1)) = b;
            }
        }
    }
};

// Transposed value fragment: of components 16 d + (lane & 15) the keys 8 g .. 8 g + 7.  A transposing read gives each lane
// of 16 one column of 4 rows x 16 halfs whose row i the lanes 4 i .. 4 i + 3 address.
template <class S>
__device__ __forceinline__ v8h value_fragment(const char* lds, int d, int lane) {
    const int c = lane & 15, g = lane >> 4;
    uint2 r[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int key = 8 * g + 4 * u + (c >> 2);
        const char* p = lds + lds_chunk<S>(key, 2 * d + ((c & 3) >> 1)) + (c & 1) * 8;
        typedef __attribute__((address_space(3))) v4fp* lds_ptr;
        const v4fp x = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_ptr)(p));
        r[u] = __builtin_bit_cast(uint2, x);
    }
    return __builtin_bit_cast(v8h, make_uint4(r[0].x, r[0].y, r[1].x, r[1].y));
}

// the 16 query rows of a tile, rotated, scaled and split: lane 16 g + c holds components 32 s + 8 g .. of row c
template <class S>
struct QueryTile {
    v8h hi[S::KS], lo[S::KS];
    __device__ __forceinline__ void load(const CachedAttention& a, const StateTokens& st, int h, int group, int r, int rows, int lane) {
        constexpr int DH = S::DH, half = DH / 2;
        const int g = lane >> 4;
        const float scale = (float)(1.0 / sqrt((double)DH)) * LOG2E;
        const bool live = r < rows;
        const int i = live ? r / group : 0, head = h * group + (live ? r % group : 0);
        const int row = st.row0 + i, pos = rope_position(a.t, row, st.base + i);
        const float* x = a.qkv + (size_t)row * ((a.n_heads + 2 * a.c.n_kv) * DH) + head * DH;
        const float *ct = a.t.cos_t + (size_t)pos * half, *sn = a.t.sin_t + (size_t)pos * half;
#pragma unroll
        for (int s = 0; s < S::KS; ++s) {
            float y[8];
            const int d0 = 32 * s + 8 * g;
            if constexpr (DH % 16 == 0) {                              // eight components lie in one half
                const bool in = live && d0 < DH;
                const int d = d0 < DH ? d0 : 0, f = d < half ? d : d - half, partner = d < half ? d + half : d - half;
                float u[8], v[8], c[8], w[8];
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    *reinterpret_cast<float4*>(u + e) = *reinterpret_cast<const float4*>(x + d + e);
                    *reinterpret_cast<float4*>(v + e) = *reinterpret_cast<const float4*>(x + partner + e);
                    *reinterpret_cast<float4*>(c + e) = *reinterpret_cast<const float4*>(ct + f + e);
                    *reinterpret_cast<float4*>(w + e) = *reinterpret_cast<const float4*>(sn + f + e);
                }
                const float sign = d < half ? -1.f : 1.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = in ? (u[e] * c[e] + sign * (v[e] * w[e])) * scale : 0.f;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = live && d0 + e < DH;
                    const int d = d0 + e < DH ? d0 + e : 0, f = d < half ? d : d - half, partner = d < half ? d + half : d - half;
                    const float p = x[partner] * sn[f];
                    y[e] = in ? (x[d] * ct[f] + (d < half ? -p : p)) * scale : 0.f;
                }
            }
            uint32_t a4[4], b4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) split_pair(y[2 * e], y[2 * e + 1], a4[e], b4[e]);
            hi[s] = __builtin_bit_cast(v8h, make_uint4(a4[0], a4[1], a4[2], a4[3]));
            lo[s] = __builtin_bit_cast(v8h, make_uint4(b4[0], b4[1], b4[2], b4[3]));
        }
    }
};

// which of the keys 8 g + e of a block row (token i) sees, for blocks that not every row sees whole
__device__ __forceinline__ uint32_t visible_bits(const CachedAttention& a, const StateTokens& st, int i, int slot0) {
    if (!a.tree) {
        const int n = st.base + i + 1 - slot0;                         // keys from slot0 on that are seen
        return n >= 8 ? 0xffu : n <= 0 ? 0u : (1u << n) - 1u;
    }
    uint32_t bits = 0;
    const uint32_t* mask = a.tree + (size_t)(st.row0 + i) * a.mask_words;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int j = slot0 + e - st.base;
        const bool see = j < 0 || ((j >> 5) < a.mask_words && (mask[j >> 5] >> (j & 31) & 1u));
        bits |= see ? 1u << e : 0u;
    }
    return bits;
}

// ---- running softmax and sum of one tile of 16 rows ----
template <class S>
struct RowState {
    v4f o[S::DTL];
    float m, ref, l;          // maximum that is followed (-inf: none yet), what scores are taken relative to, this lane's sum
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int d = 0; d < S::DTL; ++d) o[d] = v4f{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY; ref = 0.f; l = 0.f;
    }
    __device__ __forceinline__ void scale(float f) {
#pragma unroll
        for (int d = 0; d < S::DTL; ++d) o[d] *= f;
    }
    // s: scores of keys 8 g + e; on return their probabilities
    __device__ __forceinline__ void probabilities(float (&s)[8]) {
        float top = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
        if (__any(top > m + P_SLACK)) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(m, top), ref_new = m_new == -INFINITY ? 0.f : m_new - P_SHIFT;
            const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - ref_new);
            l *= alpha;
            scale(alpha);
            m = m_new;
            ref = ref_new;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[e] = __builtin_amdgcn_exp2f(s[e] - ref);
            l += s[e];
        }
    }
};

// One wavefront's pass over a block: scores of RT row tiles against the block's 32 keys
template <class S, int RT>
__device__ __forceinline__ void block_scores(const KeyLoads<S>& k, const QueryTile<S> (&q)[RT], int lane, float (&s)[RT][8]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        v4f acc[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < S::KS; ++st) {
            v8h f[S::PL];
            k.fragment(t, st, lane, f);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if constexpr (S::PL == 2) acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[1], q[r].hi[st], acc[r], 0, 0, 0);
                acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0], q[r].lo[st], acc[r], 0, 0, 0);
                acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0], q[r].hi[st], acc[r], 0, 0, 0);
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[r][4 * t + j] = acc[r][j];
    }
}

template <class S, int RT>
__device__ __forceinline__ void block_values(const char* lds, const float (&p)[RT][8], RowState<S> (&st)[RT], int lane) {
    v8h ph[RT], pl[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_pair(p[r][2 * e], p[r][2 * e + 1], h[e], l[e]);
        ph[r] = __builtin_bit_cast(v8h, make_uint4(h[0], h[1], h[2], h[3]));
        pl[r] = __builtin_bit_cast(v8h, make_uint4(l[0], l[1], l[2], l[3]));
    }
#pragma unroll
    for (int d = 0; d < S::DTL; ++d) {
        v8h f[S::PL];
#pragma unroll
        for (int x = 0; x < S::PL; ++x) f[x] = value_fragment<S>(lds + x * S::PLANE, d, lane);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if constexpr (S::PL == 2) st[r].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[1], ph[r], st[r].o[d], 0, 0, 0);
            st[r].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0], pl[r], st[r].o[d], 0, 0, 0);
            st[r].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0], ph[r], st[r].o[d], 0, 0, 0);
        }
    }
}

struct Plan {
    int group, rows_max;      // query heads per k/v head; rows of a state at most
    int row_blocks, splits;   // workgroups per (state, k/v head): blocks of rows, parts of the keys
    int rows_pad;             // rows reserved per (state, k/v head) in the scratch space
    float* part_o;            // [B][n_kv][rows_pad][splits][dh], relative to part_ml's reference
    float2* part_ml;          // [B][n_kv][rows_pad][splits]: reference and sum
    float* scores;            // [B][n_kv][rows_pad][ld_scores] or nullptr
    size_t ld_scores;
};

__device__ __forceinline__ float* out_row(const CachedAttention& a, const StateTokens& st, int h, int group, int r) {
    return a.out + ((size_t)(st.row0 + r / group) * a.n_heads + h * group + r % group) * a.c.dh;
}

// ---- few rows: every wavefront of a workgroup walks its own blocks of the workgroup's part of the keys ----
// Nothing is shared between wavefronts before the end: keys go from memory into operand registers, values through a region of LDS of the
// wavefront's own, where the transposing reads turn them.  The next block's keys are requested as soon as the scores have been
// taken, its values as soon as this block's have been stored, so that loads are in flight all the time.
template <int DT, int DH, int RT>
__global__ __launch_bounds__(512, 2) void cached_stream_kernel(CachedAttention a, Plan p) {
    typedef Shape<DT, DH> S;
    extern __shared__ __attribute__((aligned(16))) char lds_all[];
    __shared__ float2 s_ml[8][RT * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int split = blockIdx.x % p.splits, h = blockIdx.x / p.splits % a.c.n_kv, b = blockIdx.x / p.splits / a.c.n_kv;
    const StateTokens st = state_tokens(a.t, a.c, b);
    const int rows = st.n * p.group;
    if (rows == 0) return;
    const int c = lane & 15, g = lane >> 4;
    char* lds = lds_all + wave * S::LDS;
    const int seen = st.len;                                           // (the last token sees them all, or bits of the mask)
    const int blocks = (seen + 31) >> 5, per = (blocks + p.splits - 1) / p.splits;
    const int first = split * per, last = first + per < blocks ? first + per : blocks;

    QueryTile<S> q[RT];
    RowState<S> row[RT];
    float unit = 0x1p126f;                                             // int8: power of two that the sums are multiplied by
    // the first token of each row tile decides up to where all of its rows see everything
    int token[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        row[r].clear();
        token[r] = (r * 16 + c < rows ? r * 16 + c : rows - 1) / p.group;
    }
    const int all_see = st.base + (a.tree ? 0 : 1);                    // slots below are seen by every row (causal: by token 0)

    long long page_lo = -1, page_hi = -1;                              // of the lane-th block ahead
    auto pages = [&](int t0) {
        const int slot = (t0 + lane * waves) * 32;
        page_lo = slot < seen ? kv_row_index(a.c, b, h, slot) : -1;
        page_hi = slot + 16 < seen ? kv_row_index(a.c, b, h, slot + 16) : -1;
    };
    auto block_at = [&](int i) {
        Block x;
        x.lo = lane_value(page_lo, i);
        x.hi = lane_value(page_hi, i);
        return x;
    };
    KeyLoads<S> keys;
    ValueLoads<S> values;
    Block cur;
    float4 ks[2], vs[2];                                               // int8: scales of keys 8 g .. 8 g + 7
    auto key_scales = [&](const Block& x) {
        const long long r = (g >> 1) ? x.hi : x.lo;
        const float* f = a.c.ks + (r < 0 ? 0 : r) + (g & 1) * 8;
        ks[0] = reinterpret_cast<const float4*>(f)[0];
        ks[1] = reinterpret_cast<const float4*>(f)[1];
    };
    auto value_scales = [&](const Block& x) {
        const long long r = (g >> 1) ? x.hi : x.lo;
        const float* f = a.c.vs + (r < 0 ? 0 : r) + (g & 1) * 8;
        vs[0] = reinterpret_cast<const float4*>(f)[0];
        vs[1] = reinterpret_cast<const float4*>(f)[1];
    };
    int t = first + wave, ahead = 0;
    if (t < last) {
        pages(t);
        cur = block_at(0);
        keys.request(a.c.k, cur, lane);
        if constexpr (DT == BRL_I8) key_scales(cur);
        values.request(a.c.v, cur, lane);
        if constexpr (DT == BRL_I8) value_scales(cur);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) q[r].load(a, st, h, p.group, r * 16 + c, rows, lane);
    for (; t < last; t += waves) {
        const int slot0 = t * 32;
        float s[RT][8];
        block_scores<S, RT>(keys, q, lane, s);
        if constexpr (DT == BRL_I8) {
            const float f[8] = {ks[0].x, ks[0].y, ks[0].z, ks[0].w, ks[1].x, ks[1].y, ks[1].z, ks[1].w};
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[r][e] *= f[e];
        }
        // the next block's keys
        Block next = cur;
        const bool more = t + waves < last;
        if (more) {
            if (++ahead == 64) {
                ahead = 0;
                pages(t + waves);
            }
            next = block_at(ahead);
            keys.request(a.c.k, next, lane);
            if constexpr (DT == BRL_I8) key_scales(next);
        }
        __builtin_amdgcn_sched_barrier(0);
        const bool whole = slot0 + 32 <= all_see && cur.lo >= 0 && cur.hi >= 0;
        float vf[8];
        if constexpr (DT == BRL_I8) {
            const float f[8] = {vs[0].x, vs[0].y, vs[0].z, vs[0].w, vs[1].x, vs[1].y, vs[1].z, vs[1].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) vf[e] = f[e];
        }
        if (whole) {
            values.template store<false>(lds, lane, 0);
        } else {
            const int n = seen - slot0;
            uint32_t there = n >= 32 ? 0xffffffffu : (1u << n) - 1u;
            if (cur.lo < 0) there &= 0xffff0000u;
            if (cur.hi < 0) there &= 0x0000ffffu;
            values.template store<true>(lds, lane, there);
            const uint32_t mine = there >> (8 * g) & 0xffu;
            if constexpr (DT == BRL_I8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) vf[e] = mine >> e & 1u ? vf[e] : 0.f;
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const uint32_t bits = mine & visible_bits(a, st, token[r], slot0 + 8 * g);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[r][e] = bits >> e & 1u ? s[r][e] : -INFINITY;
            }
        }
        if (more) {
            values.request(a.c.v, next, lane);
            if constexpr (DT == BRL_I8) value_scales(next);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (p.scores) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
                if (r * 16 + c < rows) {
                    float* f = p.scores + (((size_t)b * a.c.n_kv + h) * p.rows_pad + r * 16 + c) * p.ld_scores + slot0 + 8 * g;
                    reinterpret_cast<float4*>(f)[0] = make_float4(s[r][0], s[r][1], s[r][2], s[r][3]);
                    reinterpret_cast<float4*>(f)[1] = make_float4(s[r][4], s[r][5], s[r][6], s[r][7]);
                }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) row[r].probabilities(s[r]);
        if constexpr (DT == BRL_I8) {
            // scales relative to the largest so far, a power of two that only falls: fp16 holds the products
            float top = vf[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, vf[e]);
            if (__any(top * unit > 1.f)) {
                const float now = __builtin_amdgcn_exp2f(-ceilf(__builtin_amdgcn_logf(wave_max(top))) - 1.f);
                const float f = now / unit;
#pragma unroll
                for (int r = 0; r < RT; ++r) row[r].scale(f);
                unit = now;
            }
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[r][e] *= vf[e] * unit;
        }
        __builtin_amdgcn_wave_barrier();
        block_values<S, RT>(lds, s, row, lane);
        __builtin_amdgcn_wave_barrier();
        cur = next;
    }
    // the wavefronts' parts meet: sums to the largest reference, then O over LDS, a row tile at a time
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        row[r].l += __shfl_xor(row[r].l, 16, 64);
        row[r].l += __shfl_xor(row[r].l, 32, 64);
        if (g == 0) s_ml[wave][r * 16 + c] = make_float2(row[r].l > 0.f ? row[r].ref : -INFINITY, row[r].l);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float top = -INFINITY;
        for (int w = 0; w < waves; ++w) top = fmaxf(top, s_ml[w][r * 16 + c].x);
        float f = row[r].l > 0.f ? __builtin_amdgcn_exp2f(row[r].ref - top) : 0.f;
        if constexpr (DT == BRL_I8) f /= unit;
        float* o = reinterpret_cast<float*>(lds);                      // [16 rows][ROW]
#pragma unroll
        for (int d = 0; d < S::DTL; ++d) *reinterpret_cast<v4f*>(o + c * S::ROW + 16 * d + 4 * g) = row[r].o[d] * f;
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * S::ROW / 4; i += blockDim.x) {
            const int x = i / (S::ROW / 4), d = i % (S::ROW / 4) * 4, rr = r * 16 + x;
            if (rr >= rows || d >= DH) continue;
            float ref = -INFINITY, l = 0.f;
            for (int w = 0; w < waves; ++w) ref = fmaxf(ref, s_ml[w][rr].x);
            v4f sum = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < waves; ++w) {
                const float2 ml = s_ml[w][rr];
                if (ml.y > 0.f) l += ml.y * __builtin_amdgcn_exp2f(ml.x - ref);
                sum += *reinterpret_cast<const v4f*>(reinterpret_cast<const float*>(lds_all + w * S::LDS) + x * S::ROW + d);
            }
            const size_t at = (((size_t)b * a.c.n_kv + h) * p.rows_pad + rr) * p.splits + split;
            if (p.part_ml && d == 0) p.part_ml[at] = make_float2(ref, l);
            if (p.splits > 1) *reinterpret_cast<v4f*>(p.part_o + at * DH + d) = sum;
            else *reinterpret_cast<v4f*>(out_row(a, st, h, p.group, rr) + d) = sum * (l > 0.f ? 1.f / l : 0.f);
        }
        __syncthreads();
    }
}

// ---- the parts of the keys joined: a wavefront per row ----
__global__ __launch_bounds__(256) void cached_join_kernel(CachedAttention a, Plan p) {
    const int lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r = (int)(unit % p.rows_max), h = (int)(unit / p.rows_max % a.c.n_kv);
    const long long b = unit / p.rows_max / a.c.n_kv;
    if (b >= a.t.B) return;
    const StateTokens st = state_tokens(a.t, a.c, (int)b);
    if (r >= st.n * p.group) return;
    const size_t at = (((size_t)b * a.c.n_kv + h) * p.rows_pad + r) * p.splits;
    float ref = -INFINITY;
    for (int s = lane; s < p.splits; s += 64) ref = fmaxf(ref, p.part_ml[at + s].x);
    ref = wave_max(ref);
    float l = 0.f, o[2] = {0.f, 0.f};
    const int dh = a.c.dh;
    for (int s = 0; s < p.splits; ++s) {
        const float2 ml = p.part_ml[at + s];
        if (!(ml.y > 0.f)) continue;
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        l += ml.y * f;
        const float* x = p.part_o + (at + s) * dh;
        if (lane < dh) o[0] += x[lane] * f;
        if (lane + 64 < dh) o[1] += x[lane + 64] * f;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    float* y = out_row(a, st, h, p.group, r);
    if (lane < dh) y[lane] = o[0] * inv;
    if (lane + 64 < dh) y[lane + 64] = o[1] * inv;
}

// ---- weights of slots from the stored scores: a thread per four slots ----
__global__ __launch_bounds__(256) void cached_weights_kernel(CachedAttention a, Plan p, int chunks) {
    __shared__ float s_lse[32];
    const int h = blockIdx.x / chunks % a.c.n_kv, b = blockIdx.x / chunks / a.c.n_kv;
    const StateTokens st = state_tokens(a.t, a.c, b);
    const int rows = st.n * p.group, slot = (blockIdx.x % chunks * 256 + threadIdx.x) * 4;
    const size_t unit = ((size_t)b * a.c.n_kv + h) * p.rows_pad;
    if (rows == 0) return;
    if (threadIdx.x < 32 && (int)threadIdx.x < rows) {
        float ref = -INFINITY, l = 0.f;
        for (int s = 0; s < p.splits; ++s) ref = fmaxf(ref, p.part_ml[(unit + threadIdx.x) * p.splits + s].x);
        for (int s = 0; s < p.splits; ++s) {
            const float2 ml = p.part_ml[(unit + threadIdx.x) * p.splits + s];
            if (ml.y > 0.f) l += ml.y * __builtin_amdgcn_exp2f(ml.x - ref);
        }
        s_lse[threadIdx.x] = l > 0.f ? ref + __builtin_amdgcn_logf(l) : INFINITY;
    }
    __syncthreads();
    if (slot >= st.len) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < rows; ++r) {
        const float4 s = *reinterpret_cast<const float4*>(p.scores + (unit + r) * p.ld_scores + slot);
        const float lse = s_lse[r];
        w[0] += __builtin_amdgcn_exp2f(s.x - lse);
        w[1] += __builtin_amdgcn_exp2f(s.y - lse);
        w[2] += __builtin_amdgcn_exp2f(s.z - lse);
        w[3] += __builtin_amdgcn_exp2f(s.w - lse);
    }
    float* y = a.weights + ((size_t)b * a.c.n_kv + h) * a.ld_weights + slot;
    for (int e = 0; e < 4; ++e)
        if (slot + e < st.len) y[e] += w[e];
}

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
__global__ __launch_bounds__(64) void simple_weights_kernel(CachedAttention a, const float* lse, int chunks) {
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

int launch_simple(const CachedAttention& a, void* workspace, hipStream_t s) {
    float* lse = a.weights ? static_cast<float*>(workspace) : nullptr;
    hipLaunchKernelGGL(cached_rows_kernel, dim3((unsigned)a.t.B * a.t.max_new * a.n_heads), dim3(64), 0, s, a, lse);
    if (a.weights) {
        const int chunks = (a.t.max_len + 63) / 64;
        hipLaunchKernelGGL(simple_weights_kernel, dim3((unsigned)a.t.B * a.c.n_kv * chunks), dim3(64), 0, s, a, (const float*)lse, chunks);
    }
    BRL_LAUNCH_CHECK("cached_rows_kernel");
    return BRL_OK;
}


struct Layout {
    Plan p;
    int waves, rt;
    size_t o_off, ml_off, scores_off, total;
};

Layout plan_cached(const KvView& c, int n_heads, int T, int B, int max_new, int max_len, bool weights) {
    Layout L;
    memset(&L, 0, sizeof(L));
    Plan& p = L.p;
    p.group = n_heads / c.n_kv;
    p.rows_max = max_new * p.group;
    const int units = B * c.n_kv, blocks = (max_len + 31) / 32;
    if (p.rows_max <= 32) {
        L.rt = p.rows_max <= 16 ? 1 : 2;
        p.row_blocks = 1;
        L.waves = 4;
        int s = (1536 + units - 1) / units;
        const int most = (blocks + L.waves * 2 - 1) / (L.waves * 2);
        if (s > most) s = most;
        p.splits = s < 1 ? 1 : s;
        p.rows_pad = L.rt * 16;
        const size_t rows = (size_t)units * p.rows_pad;
        size_t off = 0;
        if (p.splits > 1) { L.o_off = off; off += round_up_sz(rows * p.splits * c.dh * 4, 256); }
        if (p.splits > 1 || weights) { L.ml_off = off; off += round_up_sz(rows * p.splits * 8, 256); }
        if (weights) {
            p.ld_scores = (size_t)blocks * 32;
            L.scores_off = off;
            off += round_up_sz(rows * p.ld_scores * 4, 256);
        }
        L.total = off;
    } else {
        L.total = weights ? (size_t)T * n_heads * 4 : 0;
    }
    return L;
}

template <int DT, int DH>
int launch_stream(const CachedAttention& a, const Layout& L, hipStream_t s) {
    const dim3 grid((unsigned)(a.t.B * a.c.n_kv * L.p.splits)), block(L.waves * 64);
    const size_t lds = (size_t)L.waves * Shape<DT, DH>::LDS;
    if (L.rt == 1) hipLaunchKernelGGL((cached_stream_kernel<DT, DH, 1>), grid, block, lds, s, a, L.p);
    else hipLaunchKernelGGL((cached_stream_kernel<DT, DH, 2>), grid, block, lds, s, a, L.p);
    BRL_LAUNCH_CHECK("cached_stream_kernel");
    return BRL_OK;
}

template <int DT>
int launch_stream_dh(const CachedAttention& a, const Layout& L, hipStream_t s) {
    switch (a.c.dh) {
        case 16: return launch_stream<DT, 16>(a, L, s);
        case 32: return launch_stream<DT, 32>(a, L, s);
        case 64: return launch_stream<DT, 64>(a, L, s);
        case 100: return launch_stream<DT, 100>(a, L, s);
        default: return launch_stream<DT, 128>(a, L, s);
    }
}

}  // namespace

size_t cached_attention_ws_bytes(const KvView& c, int n_heads, int T, int B, int max_new, int max_len, bool weights) {
    return plan_cached(c, n_heads, T, B, max_new, max_len, weights).total;
}

int launch_cached_attention(const CachedAttention& a, void* workspace, hipStream_t s) {
    Layout L = plan_cached(a.c, a.n_heads, a.t.T, a.t.B, a.t.max_new, a.t.max_len, a.weights != nullptr);
    char* base = static_cast<char*>(workspace);
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    if (L.p.rows_max <= 32) {
        Plan& p = L.p;
        if (p.splits > 1) p.part_o = reinterpret_cast<float*>(base + L.o_off);
        if (p.splits > 1 || a.weights) p.part_ml = reinterpret_cast<float2*>(base + L.ml_off);
        if (a.weights) p.scores = reinterpret_cast<float*>(base + L.scores_off);
        const int rc = a.c.dtype == BRL_F32 ? launch_stream_dh<BRL_F32>(a, L, s) : a.c.dtype == BRL_F16 ? launch_stream_dh<BRL_F16>(a, L, s)
                                                                                                   : launch_stream_dh<BRL_I8>(a, L, s);
        if (rc) return rc;
        if (p.splits > 1) {
            const long long rows = (long long)a.t.B * a.c.n_kv * p.rows_max;
            hipLaunchKernelGGL(cached_join_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a, p);
            BRL_LAUNCH_CHECK("cached_join_kernel");
        }
        if (a.weights) {
            const int chunks = (a.t.max_len + 1023) / 1024;
            hipLaunchKernelGGL(cached_weights_kernel, dim3((unsigned)(a.t.B * a.c.n_kv * chunks)), dim3(256), 0, s, a, p, chunks);
            BRL_LAUNCH_CHECK("cached_weights_kernel");
        }
        return BRL_OK;
    }
    return launch_simple(a, workspace, s);
}

}  // namespace brl
