// Attention of new tokens over a paged key/value cache, on the matrix cores.
//
// Rows: the new tokens of a state times the query heads of one k/v head, row r = token r / group, head r % group.  Every
// row of a state reads the same keys and values, so 16 rows are one column block of v_mfma_f32_16x16x32_f16:
//   S^T (16 keys x 16 rows) = K (16 x 32 components) Q^T,   O^T (16 components x 16 rows) += V^T (16 x 32 keys) P^T.
// fp32 operands are carried as fp16 hi + lo pairs (the query rows and the probabilities always, keys and values of an fp32 cache):
// products with one such operand take two matrix instructions, with two three (lo * lo is dropped).  int8 codes are exact
// in fp16; a key's scale multiplies its scores, a value's scale its probabilities.
//
// Order of the keys.  A block of 32 keys is two key tiles of 16.  Lane l = 16 g + c of S^T holds row c's scores of the keys 4 g ..
// 4 g + 3 of both tiles.  The contraction of the second product may run over the keys in any order: with those eight as the
// slots that lane has to fill of operand P, the probabilities never leave their lane.
#include <cstring>
#include <type_traits>

#include "common.hpp"

namespace brl {

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __fp16 v4fp __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
// Probabilities are carried as 2^(s - m + SHIFT), m the running maximum rounded up to a whole number (so that going over to another one
// multiplies by powers of two), which follows the true one only once that is SLACK ahead: at most 2^15, inside fp16.  The smallest step of
// the lo plane is 2^-24, so each is carried to 2^-22 of itself or to 2^(-24 - SHIFT) of the row's largest, which is 2^(SHIFT - 1) or more.
// A smaller SLACK has sums rescaled more often: 4 prompts of 4096 tokens, 20 heads of 128, SHIFT 6 / 12 / 13 / 14 of an fp16 cache 621 / 620 /
// 621 / 633 us, 11 / 13 of an int8 cache 662 / 684 (whose values are rounded to 2^-8 of a row's largest anyway).
template <int DT>
struct Reference {
    static constexpr float SHIFT = DT == BRL_I8 ? 11.f : 13.f, SLACK = 15.f - SHIFT;
};

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
    // Key fragments straight from memory: which components a lane of group g holds in step s is free as long as the queries go along.
    // Chosen such that four lanes read 64 bytes of a row with each load: 32 s + 8 g .. + 7 of fp16 rows; 32 s + 4 g .. + 3 and sixteen
    // further on of fp32 rows (two loads a step); of int8 rows 64 u + 16 g .. + 15 with one load for the steps 2 u and 2 u + 1 (8 bytes
    // a lane where a row is shorter than that).
    static constexpr bool PAIRED = DT == BRL_I8 && ROW > 32;
    static constexpr int KL = DT == BRL_F32 ? 2 * KS : PAIRED ? KS / 2 : KS;      // loads of a tile
    static_assert(!PAIRED || KS % 2 == 0, "whole pairs of steps");
};

// Where chunk c of a key's row lies in LDS.  The chunks of a row are permuted by bits of the key such that both the 16 rows
// x 16 bytes of a key fragment and the 16 rows x 32 bytes of a transposing read fall on all banks.
template <class S>
__device__ __forceinline__ unsigned lds_chunk(unsigned key, unsigned c) {      // (unsigned: shifts and masks, no corrections for signs)
    constexpr int SKIP = S::NCH == 16 ? 0 : S::NCH == 8 ? 1 : S::NCH == 4 ? 2 : 3;   // rows that lie side by side in 256 bytes
    return key * S::LS + ((c ^ ((key & 15) >> SKIP)) << 4);
}

// A block of 32 slots lies in two halves of 16 (pages hold 16 at least): lo and hi are their first rows in the pool, -1 where
// there is none.

// The keys of a block, lane 16 g + c those of row c of both tiles.
template <class S>
struct KeyLoads {
    static constexpr bool WIDE = S::DT != BRL_I8 || S::PAIRED;         // 16 bytes a lane, else 8
    static constexpr int STEP = WIDE ? 64 : 32;                        // bytes of a row that a load covers
    typedef typename std::conditional<WIDE, uint4, uint2>::type raw_t;
    raw_t raw[2][S::KL];
    __device__ __forceinline__ void request(const char* pool, int lo, int hi, unsigned lane) {
        const unsigned c = lane & 15, g = lane >> 4, mine = g * (STEP / 4);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = t ? hi : lo;
            const char* p = pool + (size_t)(row < 0 ? 0 : row) * S::RB;          // (the same for all lanes)
#pragma unroll
            for (int i = 0; i < S::KL; ++i) {
                unsigned at = c * S::RB;                               // (past the end of a row: its beginning, not used)
                if ((i + 1) * STEP <= S::RB || i * STEP + mine < (unsigned)S::RB) at += i * STEP + mine;
                raw[t][i] = *reinterpret_cast<const raw_t*>(p + at);
            }
        }
    }
    // the operand of step s
    __device__ __forceinline__ void fragment(int t, int s, unsigned lane, v8h (&f)[S::PL]) const {
        uint32_t w[S::PL][4];
        const int g = (int)(lane >> 4);
        int first, second;                                             // components of the first and the second four
        if constexpr (S::DT == BRL_F32) {
            first = 32 * s + 4 * g;
            second = first + 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 r = raw[t][2 * s + i];
                split_pair(__uint_as_float(r.x), __uint_as_float(r.y), w[0][2 * i], w[1][2 * i]);
                split_pair(__uint_as_float(r.z), __uint_as_float(r.w), w[0][2 * i + 1], w[1][2 * i + 1]);
            }
        } else if constexpr (S::DT == BRL_F16) {
            first = 32 * s + 8 * g;
            second = first + 4;
            const uint4 r = raw[t][s];
            w[0][0] = r.x; w[0][1] = r.y; w[0][2] = r.z; w[0][3] = r.w;
        } else if constexpr (S::PAIRED) {
            first = 64 * (s / 2) + 16 * g + 8 * (s % 2);
            second = first + 4;
            const uint4 r = raw[t][s / 2];
            widen_codes(s % 2 ? r.z : r.x, w[0][0], w[0][1]);
            widen_codes(s % 2 ? r.w : r.y, w[0][2], w[0][3]);
        } else {
            first = 32 * s + 8 * g;
            second = first + 4;
            widen_codes(raw[t][s].x, w[0][0], w[0][1]);
            widen_codes(raw[t][s].y, w[0][2], w[0][3]);
        }
        // what lies behind head_dim is not a number (four components are on one side of it or the other)
        static_assert(S::DH % 4 == 0, "whole fours");
        if (S::DH % (S::PAIRED ? 64 : 32) && s >= S::KS - (S::PAIRED ? 2 : 1)) {
#pragma unroll
            for (int p = 0; p < S::PL; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[p][j] = (j < 2 ? first : second) < S::DH ? w[p][j] : 0u;
        }
#pragma unroll
        for (int p = 0; p < S::PL; ++p) f[p] = __builtin_bit_cast(v8h, make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]));
    }
};
// Components 32 s + 8 g .. + 7 of the rows of a query tile (lane 16 g + c has them of row c) to where the operand of KeyLoads' fragments
// wants them, in [step][hi, lo][64 lanes].
template <class S>
__device__ __forceinline__ void store_query(uint4* to, int s, int lane, const uint4& hi, const uint4& lo) {
    const int c = lane & 15, g = lane >> 4;
    if constexpr (S::DT == BRL_F32) {
        uint2* f = reinterpret_cast<uint2*>(to) + (s * 2 * 64 + 16 * (2 * (g & 1)) + c) * 2 + (g >> 1);
        f[0] = make_uint2(hi.x, hi.y);
        f[32] = make_uint2(hi.z, hi.w);                                // sixteen lanes on
        f[128] = make_uint2(lo.x, lo.y);
        f[160] = make_uint2(lo.z, lo.w);
    } else {
        const int n = 4 * s + g;                                       // which eight components of the row
        const int step = S::PAIRED ? 2 * (n >> 3) + (n & 1) : s, group = S::PAIRED ? (n & 7) >> 1 : g;
        to[step * 128 + 16 * group + c] = hi;
        to[step * 128 + 64 + 16 * group + c] = lo;
    }
}

// ---- values that are no numbers, in blocks that some rows do not see whole ----
// Zero times infinity is NaN, so such a value would reach rows that do not see its slot.  In blocks that hold new tokens these values
// go into LDS as zeros; the rows that see their slots have them added in fp32 by add_strange.  (In older blocks every row sees them.)
// fp32: what hi + lo do not hold counts as such, too.  int8: the value's scale.
template <int DT>
__device__ __forceinline__ bool strange_word(uint32_t w) {             // one float, or either of two halfs
    if constexpr (DT == BRL_F32) return (w & 0x7fffffffu) >= 0x477ff000u;          // 65520, from where on hi is infinite
    return (((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u) != 0;
}
template <int DT>
__device__ __forceinline__ uint32_t plain_word(uint32_t w) {
    if constexpr (DT == BRL_F32) return strange_word<DT>(w) ? 0u : w;
    return ((w & 0x7c00u) == 0x7c00u ? 0u : w & 0xffffu) | ((w & 0x7c000000u) == 0x7c000000u ? 0u : w & 0xffff0000u);
}
template <int DT>
__device__ __forceinline__ bool strange(const uint4& r) {
    return strange_word<DT>(r.x) || strange_word<DT>(r.y) || strange_word<DT>(r.z) || strange_word<DT>(r.w);
}
// Whether there may be any among several words, in one instruction a word: a sum that such a value leaves infinite or NaN.
template <int DT>
struct Suspicion {
    typedef typename std::conditional<DT == BRL_F32, float, v2h>::type sum_t;
    sum_t sum = {};
    __device__ __forceinline__ void word(uint32_t w) {
        if constexpr (DT == BRL_F32) sum = __builtin_fmaf(__uint_as_float(w), 0x1p113f, sum);          // (overflows from 2^15 on)
        else sum = __builtin_elementwise_fma(__builtin_bit_cast(v2h, w), v2h{(_Float16)0.f, (_Float16)0.f}, sum);
    }
    __device__ __forceinline__ void words(const uint4& r) { word(r.x); word(r.y); word(r.z); word(r.w); }
    __device__ __forceinline__ bool any() const {                      // of the wavefront's
        if constexpr (DT == BRL_F32) return __any(!(fabsf(sum) < INFINITY));
        else return __any(sum[0] != sum[0] || sum[1] != sum[1]);
    }
};
template <int DT>
__device__ __forceinline__ uint4 plain(const uint4& r) {
    return make_uint4(plain_word<DT>(r.x), plain_word<DT>(r.y), plain_word<DT>(r.z), plain_word<DT>(r.w));
}
__device__ __forceinline__ bool strange_scale(float s) { return (__float_as_uint(s) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t any_lane(uint32_t x) {              // bits that any lane of the wavefront has
    if (!__any(x != 0)) return 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x |= __shfl_xor(x, d, 64);
    return __builtin_amdgcn_readfirstlane(x);
}

// Rows of the values, 16 bytes per lane in the order of the pool, and from there as halfs into LDS.
template <class S>
struct ValueLoads {
    uint4 raw[S::NV];
    __device__ __forceinline__ void request(const char* pool, int lo_row, int hi_row, int lane) {
        const char* lo = pool + (size_t)(lo_row < 0 ? 0 : lo_row) * S::RB;
        const char* hi = pool + (size_t)(hi_row < 0 ? 0 : hi_row) * S::RB;
        constexpr int HALF = 16 * S::CPR;                              // chunks of 16 rows
#pragma unroll
        for (int i = 0; i < S::NV; ++i) {
            int idx = i * 64 + lane;
            // past the end: the last chunk again, not stored (a load that might not happen is waited for before its registers'
            // next use, which is the load of the next block)
            if (S::NV * 64 > 32 * S::CPR && idx >= 32 * S::CPR) idx = 32 * S::CPR - 1;
            if ((i + 1) * 64 <= HALF) raw[i] = *reinterpret_cast<const uint4*>(lo + (unsigned)(idx * 16));
            else if (i * 64 >= HALF) raw[i] = *reinterpret_cast<const uint4*>(hi + (unsigned)((idx - HALF) * 16));
            else raw[i] = *reinterpret_cast<const uint4*>(idx >= HALF ? hi + (unsigned)((idx - HALF) * 16) : lo + (unsigned)(idx * 16));
        }
    }
    __device__ __forceinline__ bool suspicious() const {
        Suspicion<S::DT> x;
#pragma unroll
        for (int i = 0; i < S::NV; ++i) x.words(raw[i]);
        return x.any();
    }
    __device__ __forceinline__ void store(char* lds, unsigned lane) const {
#pragma unroll
        for (int i = 0; i < S::NV; ++i) {
            const unsigned idx = i * 64 + lane, key = idx / S::CPR, c = idx % S::CPR;
            if (S::NV * 64 > 32 * S::CPR && idx >= 32u * S::CPR) continue;
            const uint4 r = raw[i];
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
// rows of a stored block that hold no numbers: zeros (bit `key` of there is clear)
template <class S>
__device__ __forceinline__ void clear_rows(char* lds, int lane, uint32_t there) {
#pragma unroll 1
    for (int i = lane; i < S::PL * 32 * S::NCH; i += 64)
        if (!(there >> (i / S::NCH % 32) & 1u)) reinterpret_cast<uint4*>(lds)[i] = make_uint4(0, 0, 0, 0);
}

// Strange values of a stored block to zeros; the keys whose rows had some.
template <class S>
__device__ __forceinline__ uint32_t take_strange(char* lds, int lane) {
    uint32_t keys = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");             // (other lanes' stores)
#pragma unroll 1
    for (int i = lane; i < 32 * S::NCH; i += 64) {
        uint4* hi = reinterpret_cast<uint4*>(lds) + i;
        if (!strange<BRL_F16>(*hi)) continue;
        keys |= 1u << (i / S::NCH);
        if constexpr (S::PL == 2) {
            uint4* lo = hi + S::PLANE / 16;                            // (infinite or NaN as well, where hi is)
            *lo = plain<BRL_F16>(*lo);
        }
        *hi = plain<BRL_F16>(*hi);
    }
    return any_lane(keys);
}

// Transposed value fragment: of components 16 d + (lane & 15) the keys 4 g .. 4 g + 3 of both tiles.  A transposing read gives
// each lane of 16 one column of 4 rows x 16 halfs whose row i the lanes 4 i .. 4 i + 3 address.  (Keys sixteen apart have their
// chunks permuted alike, so the second read is the first one's address and a constant.)
template <class S>
struct ValueReads {
    const char* base;
    unsigned x;
    __device__ __forceinline__ ValueReads(const char* lds, unsigned lane) {
        const unsigned c = lane & 15, key = 4 * (lane >> 4) + (c >> 2);
        const unsigned at = lds_chunk<S>(key, (c & 3) >> 1);
        base = lds + key * S::LS + (c & 1) * 8;
        x = at - key * S::LS;
    }
    __device__ __forceinline__ v8h fragment(int d, int plane) const {
        uint2 r[2];
        const char* p = base + (x ^ (unsigned)(d << 5));
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            typedef __attribute__((address_space(3))) v4fp* lds_ptr;
            const v4fp v = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_ptr)(p + plane * S::PLANE + u * 16 * S::LS));
            r[u] = __builtin_bit_cast(uint2, v);
        }
        return __builtin_bit_cast(v8h, make_uint4(r[0].x, r[0].y, r[1].x, r[1].y));
    }
};

// Query heads per k/v head.  Rows are divided by them often enough to multiply by the inverse instead: ceil(2^32 / n), right for
// rows below 2^32 / n, which the entry point sees to; 0 stands for one head.
struct Group {
    int n;
    uint32_t inverse;
    __device__ __forceinline__ int token(int r) const { return inverse ? (int)__umulhi((uint32_t)r, inverse) : r; }
};

struct QueryRow {
    const float *x, *ct, *sn;          // a query row, the cosines and sines of its position
    __device__ __forceinline__ QueryRow(const CachedAttention& a, const StateTokens& st, int h, const Group& group, int r, int token, int pos) {
        const int row = st.row0 + token, dh = a.c.dh;
        x = a.qkv + (size_t)row * ((a.n_heads + 2 * a.c.n_kv) * dh) + (h * group.n + r - token * group.n) * dh;
        ct = a.t.cos_t + (size_t)pos * (dh / 2);
        sn = a.t.sin_t + (size_t)pos * (dh / 2);
    }
};
// Four components d0 .. of a query row, rotated, scaled and split into an operand's hi and lo words.
template <class S>
struct QueryFour {
    float x[4], y[4], c[4], w[4];      // components, their partners, cosines, sines
    __device__ __forceinline__ void request(const QueryRow& q, int d0) {
        constexpr int DH = S::DH, half = DH / 2;
        if constexpr (DH % 8 == 0) {                                   // four components lie in one half
            const int d = d0 < DH ? d0 : 0, f = d < half ? d : d - half, partner = d < half ? d + half : d - half;
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(q.x + d);
            *reinterpret_cast<float4*>(y) = *reinterpret_cast<const float4*>(q.x + partner);
            *reinterpret_cast<float4*>(c) = *reinterpret_cast<const float4*>(q.ct + f);
            *reinterpret_cast<float4*>(w) = *reinterpret_cast<const float4*>(q.sn + f);
        } else {                                                       // two do
            static_assert(DH % 4 == 0, "pairs do not straddle the halves");
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const int d = d0 + e < DH ? d0 + e : 0, f = d < half ? d : d - half, partner = d < half ? d + half : d - half;
                *reinterpret_cast<float2*>(x + e) = *reinterpret_cast<const float2*>(q.x + d);
                *reinterpret_cast<float2*>(y + e) = *reinterpret_cast<const float2*>(q.x + partner);
                *reinterpret_cast<float2*>(c + e) = *reinterpret_cast<const float2*>(q.ct + f);
                *reinterpret_cast<float2*>(w + e) = *reinterpret_cast<const float2*>(q.sn + f);
            }
        }
    }
    __device__ __forceinline__ void split(bool live, int d0, uint2& hi, uint2& lo) const {
        constexpr int DH = S::DH, half = DH / 2;
        const float scale = (float)(1.0 / sqrt((double)DH)) * LOG2E;
        float z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = y[e] * w[e];
            z[e] = live && d0 + e < DH ? (x[e] * c[e] + (d0 + e < half ? -p : p)) * scale : 0.f;
        }
        split_pair(z[0], z[1], hi.x, lo.x);
        split_pair(z[2], z[3], hi.y, lo.y);
    }
};
// Components 32 s + 8 g .. + 7 of the rows of a query tile, for lane 16 g + c of row c.  ONE_BY_ONE: four and four, in half the registers.
template <class S, bool ONE_BY_ONE>
struct QueryPart {
    QueryFour<S> q[ONE_BY_ONE ? 1 : 2];
    __device__ __forceinline__ void request(const QueryRow& from, int d0) {
        q[0].request(from, d0);
        if constexpr (!ONE_BY_ONE) q[1].request(from, d0 + 4);
    }
    __device__ __forceinline__ void split(const QueryRow& from, bool live, int d0, uint4& hi, uint4& lo) {
        uint2 a, b, c, d;
        q[0].split(live, d0, a, b);
        if constexpr (ONE_BY_ONE) {
            __builtin_amdgcn_sched_barrier(0);
            q[0].request(from, d0 + 4);
            q[0].split(live, d0 + 4, c, d);
        } else {
            q[1].split(live, d0 + 4, c, d);
        }
        hi = make_uint4(a.x, a.y, c.x, c.y);
        lo = make_uint4(b.x, b.y, d.x, d.y);
    }
};

// which of the slots slot0 .. slot0 + 31 token i sees, for blocks that not every row sees whole
__device__ __forceinline__ uint32_t visible_bits(const CachedAttention& a, const StateTokens& st, int i, int slot0) {
    if (!a.tree) {
        const int n = st.base + i + 1 - slot0;                         // from slot0 on
        return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
    }
    const int j = slot0 - st.base, w = j >> 5;                         // bits j .. j + 31, set in front of the mask, clear behind it
    const uint32_t* mask = a.tree + (size_t)(st.row0 + i) * a.mask_words;
    const uint32_t lo = w < 0 ? 0xffffffffu : w < a.mask_words ? mask[w] : 0u;
    const uint32_t hi = w + 1 < 0 ? 0xffffffffu : w + 1 < a.mask_words ? mask[w + 1] : 0u;
    return (uint32_t)((((uint64_t)hi << 32) | lo) >> (j & 31));
}
// the bits of the keys that lanes of group g hold, in the order of their scores
__device__ __forceinline__ uint32_t bits_of_group(uint32_t bits, int g) { return (bits >> (4 * g) & 0xfu) | (bits >> (16 + 4 * g) & 0xfu) << 4; }
// where score e of group g stands in its block
__device__ __forceinline__ constexpr int key_of_score(int g, int e) { return 16 * (e >> 2) + 4 * g + (e & 3); }

// log2 of l 2^ref, as exact as its own size allows (ref is a whole number); +inf where nothing was summed up
__device__ __forceinline__ float log_sum(float ref, float l) {
    return l > 0.f ? ref + (float)__builtin_amdgcn_frexp_expf(l) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l)) : INFINITY;
}

// int8: what multiplies the codes is a probability times its slot's scale, and scales are of any size.  So the maximum that is followed is
// that of s + log2(scale) over the slots that the row sees: the products have the bounds that probabilities have otherwise, whatever the
// scales of slots that the row does not see or hardly weighs.  (Scales count as LEAST_SCALE at least, which keeps the probabilities
// themselves below 2^90, and parts that meet comparable; values below 1e-25 have fewer digits for it.  Those of values that are no
// numbers count as that.)
constexpr float LEAST_SCALE = 0x1p-75f;
// log2 of x from its bits, at most 0.09 below: exponent and, for the logarithm of a mantissa 1 + f, f
__device__ __forceinline__ float rough_log2(float x) { return (float)__float_as_uint(x) * 0x1p-23f - 127.f; }
__device__ __forceinline__ float scale_bits(float x) { return rough_log2(fabsf(x) < INFINITY ? fmaxf(fabsf(x), LEAST_SCALE) : LEAST_SCALE); }

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
    // s: a lane's scores; on return their probabilities.  scales (int8): of the slots' values.
    __device__ __forceinline__ void probabilities(float (&s)[8], const float (&scales)[8]) {
        float top = s[0], most = LEAST_SCALE;
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
        if constexpr (S::DT == BRL_I8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(scales[e]));
        }
        // (int8: may be above; the largest scale need not be the likeliest slot's)
        if (__any((S::DT == BRL_I8 ? top + rough_log2(most) : top) > m + Reference<S::DT>::SLACK)) {
            if constexpr (S::DT == BRL_I8) {
                top = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = scales[e];
                    asm volatile("" : "+v"(x));       // (opaque: or this is computed in front of the branch, every time)
                    top = fmaxf(top, s[e] + scale_bits(x));
                }
            }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(m, ceilf(top)), ref_new = m_new == -INFINITY ? 0.f : m_new - Reference<S::DT>::SHIFT;
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

// The strange values of some of a block's keys (its halves' first rows in the pool: lo, hi) for the rows that see them.  p: a lane's
// probabilities, 0 where its row does not see the key.
template <class S>
__device__ __forceinline__ void add_strange(const KvView& kv, int lo, int hi, uint32_t keys, const float (&p)[8], RowState<S>& row, int lane) {
    const int c = lane & 15, g = lane >> 4;
#pragma unroll 1
    for (; keys; keys &= keys - 1) {
        const int key = __builtin_ctz(keys), at = (key < 16 ? lo : hi) + (key & 15);
        float x = p[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) x = (key >> 4) * 4 + (key & 3) == e ? p[e] : x;
        x = __shfl(x, 16 * (key >> 2 & 3) + c, 64);
        const char* from = kv.v + (size_t)at * S::RB;
#pragma unroll
        for (int d = 0; d < S::DTL; ++d) {
            __builtin_amdgcn_sched_barrier(0);
            const int first = 16 * d + 4 * g;
            if (first >= S::DH) continue;
            float v[4];
            if constexpr (S::DT == BRL_F32) {
                *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(from + first * 4);
            } else if constexpr (S::DT == BRL_F16) {
                const v4h f = *reinterpret_cast<const v4h*>(from + first * 2);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = (float)f[j];
            } else {
                const uint32_t f = *reinterpret_cast<const uint32_t*>(from + first);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = (float)(int8_t)(f >> (8 * j)) * kv.vs[at];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool other = S::DT == BRL_I8 || strange_word<BRL_F32>(__float_as_uint(v[j]));
                row.o[d][j] += other && x != 0.f ? x * v[j] : 0.f;
            }
        }
    }
}

// One wavefront's pass over a block: scores of 16 rows against the block's 32 keys.  A step at a time: left to itself the compiler
// reads all query fragments and widens all keys first.
template <class S>
__device__ __forceinline__ void block_scores(const KeyLoads<S>& k, const uint4* q, unsigned lane, float (&s)[8]) {
    v4f acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int st = 0; st < S::KS; ++st) {
        v8h f[2][S::PL];
#pragma unroll
        for (int t = 0; t < 2; ++t) k.fragment(t, st, lane, f[t]);
        const v8h qh = __builtin_bit_cast(v8h, q[(st * 2) * 64 + lane]), ql = __builtin_bit_cast(v8h, q[(st * 2 + 1) * 64 + lane]);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (S::PL == 2) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[t][1], qh, acc[t], 0, 0, 0);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[t][0], ql, acc[t], 0, 0, 0);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[t][0], qh, acc[t], 0, 0, 0);
        }
        if (st % 2) __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = acc[e >> 2][e & 3];
}

template <class S, int RT>
__device__ __forceinline__ void block_values(const char* lds, const float (*p)[8], RowState<S>* st, unsigned lane) {
    v8h ph[RT], pl[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_pair(p[r][2 * e], p[r][2 * e + 1], h[e], l[e]);
        ph[r] = __builtin_bit_cast(v8h, make_uint4(h[0], h[1], h[2], h[3]));
        pl[r] = __builtin_bit_cast(v8h, make_uint4(l[0], l[1], l[2], l[3]));
    }
    const ValueReads<S> v(lds, lane);
#pragma unroll
    for (int d = 0; d < S::DTL; ++d) {
        v8h f[S::PL];
#pragma unroll
        for (int x = 0; x < S::PL; ++x) f[x] = v.fragment(d, x);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if constexpr (S::PL == 2) st[r].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[1], ph[r], st[r].o[d], 0, 0, 0);
            st[r].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0], pl[r], st[r].o[d], 0, 0, 0);
            st[r].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0], ph[r], st[r].o[d], 0, 0, 0);
        }
    }
}

struct Plan {
    Group group;
    int rows_max;             // rows of a state at most
    int row_blocks, splits;   // many rows: blocks of rows of a (state, k/v head), parts of the keys
    uint4* q;                 // many rows with weights: [B][n_kv][rows_pad / 16][steps][hi, lo][64] query fragments
    int rows_pad;             // rows reserved per (state, k/v head) in the scratch space
    int groups;               // workgroups that share all blocks evenly, 0: one workgroup per (state, k/v head)
    int least;                // blocks a workgroup takes at least
    float* part_o;            // [2 groups][rows_pad][dh]: sums relative to part_ml's reference
    float2* part_ml;          // [2 groups][rows_pad]: reference and sum of probabilities
    float* lse;               // [B][n_kv][rows_pad] or nullptr: log2 of a row's sum, +inf where it sees nothing
    float* scores;            // few rows with weights: [B][n_kv][rows_max][ld_scores], else nullptr
    size_t ld_scores;
    int w_parts;              // many rows with weights: parts of the rows whose sums are added up by a second kernel (1: none)
    float* part_w;            // [w_parts][B][n_kv][ld_scores] or nullptr
};

__device__ __forceinline__ float* out_row(const CachedAttention& a, const StateTokens& st, int h, const Group& group, int r) {
    const int token = group.token(r);
    return a.out + ((size_t)(st.row0 + token) * a.n_heads + h * group.n + r - token * group.n) * a.c.dh;
}

// ---- sharing the work ----
// The blocks of 32 slots of all (state, k/v head) pairs, in that order, are one list; workgroup w takes the entries
// w share .. (w + 1) share - 1.  States of different length so cost every workgroup the same.
__device__ __forceinline__ int blocks_of(const StateTokens& st) { return st.n ? (st.len + 31) >> 5 : 0; }
__device__ __forceinline__ int state_blocks(const CachedAttention& a, int b) { return blocks_of(state_tokens(a.t, a.c, b)); }
// Per wavefront: blocks of the states in front of this lane's stretch of states, and of all.
struct Prefix {
    int stretch;              // states per lane
    int before, total;
    StateTokens own;          // the last of this lane's states (where there are at most 64: state `lane`)
};
__device__ __forceinline__ Prefix prefix_blocks(const CachedAttention& a, int lane) {
    Prefix p;
    p.stretch = (a.t.B + 63) / 64;
    int mine = 0;
    p.own = StateTokens{0, 0, 0, 0};
    for (int b = lane * p.stretch; b < (lane + 1) * p.stretch && b < a.t.B; ++b) {
        p.own = state_tokens(a.t, a.c, b);
        mine += blocks_of(p.own);
    }
    int x = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d, 64);
        if (lane >= d) x += y;
    }
    p.before = x - mine;
    p.total = lane_value(x, 63);
    return p;
}
__device__ __forceinline__ unsigned share_of(const Plan& p, unsigned entries) {       // (the list has fewer than 2^31)
    const unsigned s = (entries + p.groups - 1) / p.groups;
    return s < (unsigned)p.least ? p.least : s;
}

// ---- few rows: every wavefront of a workgroup walks its own blocks ----
// Nothing is shared between wavefronts but the query rows: keys go from memory into operand registers, values through a region of
// LDS of the wavefront's own, where the transposing reads turn them.  The next block's keys are requested as soon as the scores
// have been taken, its values as soon as this block's have been stored, so that loads are in flight all the time.
// A workgroup may have to finish one (state, k/v head) and go on with the next: the wavefronts' first blocks of the next segment are
// requested like any next block, so that the end of a segment (6 us: sums joined, queries of the next read) has loads in flight.
template <int DT, int DH>
struct StreamShape {
    typedef Shape<DT, DH> S;
    static constexpr int OS = S::ROW + 4;                              // floats of a row of O in LDS: rows start on different banks
    static constexpr int LDS = S::LDS > 16 * OS * 4 ? S::LDS : 16 * OS * 4;
};

template <int DT, int DH>
__global__ __launch_bounds__(512, 2) void cached_stream_kernel(CachedAttention a, Plan p) {
    typedef Shape<DT, DH> S;
    constexpr int OS = StreamShape<DT, DH>::OS, LDS = StreamShape<DT, DH>::LDS;
    extern __shared__ __attribute__((aligned(16))) char lds_all[];
    __shared__ uint4 s_q[S::KS * 2 * 64];                              // query fragments: [step][hi, lo][64 lanes]
    __shared__ float2 s_ml[8][16];                                     // per wavefront and row: reference and sum
    __shared__ float s_l[8][16];                                       // sums relative to the largest reference
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int c = lane & 15, g = lane >> 4;
    char* lds = lds_all + wave * LDS;

    // this workgroup's entries: left of them, the state and head they begin in, the block in it
    int b, h, first, left;
    StateTokens st;
    Prefix pre;
    pre.stretch = 0;
    auto tokens_of = [&](int x) {                                      // of state x
        StateTokens t;
        if (pre.stretch == 1) {
            t.row0 = lane_value(pre.own.row0, x);
            t.n = lane_value(pre.own.n, x);
            t.len = lane_value(pre.own.len, x);
            t.base = lane_value(pre.own.base, x);
        } else {
            t = state_tokens(a.t, a.c, x);
        }
        return t;
    };
    if (p.groups == 0) {
        h = blockIdx.x % a.c.n_kv; b = blockIdx.x / a.c.n_kv; first = 0;
        left = 0x7fffffff;
        st = tokens_of(b);
    } else {
        pre = prefix_blocks(a, lane);
        const unsigned entries = (unsigned)pre.total * a.c.n_kv, share = share_of(p, entries);
        if (entries == 0 || blockIdx.x > (entries - 1) / share) return;
        unsigned at = blockIdx.x * share;
        left = (int)(entries - at < share ? entries - at : share);
        const unsigned long long in = __ballot((unsigned)pre.before * a.c.n_kv <= at);
        const int l = 63 - __builtin_clzll(in);                         // the last stretch that begins at or before the entry
        at -= (unsigned)lane_value(pre.before, l) * a.c.n_kv;
        b = l * pre.stretch;
        st = tokens_of(b);
        unsigned n = blocks_of(st);
        while (at >= n * a.c.n_kv) {
            at -= n * a.c.n_kv;
            st = tokens_of(++b);
            n = blocks_of(st);
        }
        h = at / n;
        first = at % n;
    }
    if (st.n == 0) return;                                             // (one workgroup per (state, k/v head), nothing new)
    auto next_segment = [&](int& x, int& y, StateTokens& t) {          // (there is one: entries are left)
        if (++y < a.c.n_kv) return;
        y = 0;
        do t = tokens_of(++x);
        while (blocks_of(t) == 0);
    };
    int blocks = blocks_of(st);
    int last = left < blocks - first ? first + left : blocks;

    KeyLoads<S> keys;
    ValueLoads<S> values;
    float4 ks[2], vs[2];                                               // int8: scales of this lane's keys
    auto scales = [&](const float* pool, int x_lo, int x_hi, float4 (&f)[2]) {
        f[0] = *reinterpret_cast<const float4*>(pool + (x_lo < 0 ? 0 : x_lo) + (unsigned)(4 * g));
        f[1] = *reinterpret_cast<const float4*>(pool + (x_hi < 0 ? 0 : x_hi) + (unsigned)(4 * g));
    };
    int page_lo = -1, page_hi = -1;                                    // rows of the lane-th block ahead
    auto pages = [&](int t0, int from) {                               // from: this lane
        const int block = t0 + from * waves, slot = block * 32;
        page_lo = block < last && slot < st.len ? kv_row_index(a.c, b, h, slot) : -1;
        page_hi = block < last && slot + 16 < st.len ? kv_row_index(a.c, b, h, slot + 16) : -1;
    };
    constexpr int JOBS = S::KS * 64;                                   // query fragments: a lane of a step each, of the first threads
    static_assert(JOBS <= 256, "every workgroup has the threads");
    auto query_row = [&](int c) { return c < st.n * p.group.n ? c : st.n * p.group.n - 1; };
    auto position = [&](int token) { return rope_position(a.t, st.row0 + token, st.base + token); };
    int token = p.group.token(query_row(c)), pos = position(token);
    pages(first + wave, lane);
    int lo = lane_value(page_lo, 0), hi = lane_value(page_hi, 0);      // where the block under way lies
    keys.request(a.c.k, lo, hi, lane);
    if constexpr (DT == BRL_I8) scales(a.c.ks, lo, hi, ks);
    values.request(a.c.v, lo, hi, lane);
    if constexpr (DT == BRL_I8) scales(a.c.vs, lo, hi, vs);
    bool before = true;                                                // nothing but this segment's beginning lies in front
    for (;;) {
        int here = lane;                                               // (opaque: nothing that a segment needs is kept from one to the next)
        asm volatile("" : "+v"(here));
        const int c = here & 15, g = here >> 4, d0 = 32 * wave + 8 * g;
        const int rows = st.n * p.group.n, seen = st.len;                // (the last token sees them all, or bits of the mask)
        const bool all = first == 0 && last == blocks, live = c < rows;
        const QueryRow from(a, st, h, p.group, query_row(c), token, pos);
        QueryPart<S, DT == BRL_F32> q;                                 // (fp32: the blocks under way leave no registers for all of it)
        if (threadIdx.x < JOBS) q.request(from, d0);
        // where this wavefront's first block of the next segment lies
        left -= last - first;
        if (p.groups == 0) left = 0;
        int after_lo = -1, after_hi = -1;
        if (left > 0) {
            int x = b, y = h;
            StateTokens next = st;
            next_segment(x, y, next);
            const int n = blocks_of(next), slot = wave * 32;
            if (wave < (left < n ? left : n)) {
                after_lo = kv_row_index(a.c, x, y, slot);
                after_hi = slot + 16 < next.len ? kv_row_index(a.c, x, y, slot + 16) : -1;
            }
        }
        RowState<S> row;
        row.clear();
        const int all_see = st.base + (a.tree ? 0 : 1);                // slots below are seen by every row (causal: by token 0)
        if (threadIdx.x < JOBS) {
            uint4 x, y;
            q.split(from, live, d0, x, y);
            store_query<S>(s_q, wave, here, x, y);
        }
        after_lo = __builtin_amdgcn_readfirstlane(after_lo);
        after_hi = __builtin_amdgcn_readfirstlane(after_hi);
        __syncthreads();
        int t = first + wave, ahead = 0;
        // A wavefront without a block takes a turn, too: for the requests, nothing else.  (A branch around it costs the loop registers.)
        const bool mine = t < last;
        do {
            const int slot0 = t * 32;
            unsigned at = lane;                                        // (opaque: or the compiler keeps all of LDS in registers)
            asm volatile("" : "+v"(at));
            float s[8];
            block_scores<S>(keys, s_q, at, s);
            if constexpr (DT == BRL_I8) {
                const float f[8] = {ks[0].x, ks[0].y, ks[0].z, ks[0].w, ks[1].x, ks[1].y, ks[1].z, ks[1].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] *= f[e];
            }
            __builtin_amdgcn_sched_barrier(0);                         // (the old keys' registers are free from here on)
            // Behind the very last block, rows 0 of the pool are requested and never used: a request that might not be made would
            // have every wait in the loop wait for all of them.
            if (++ahead == 64) {
                ahead = 0;
                pages(t + waves, at);
            }
            const bool more = t + waves < last;
            const int next_lo = more ? lane_value(page_lo, ahead) : after_lo, next_hi = more ? lane_value(page_hi, ahead) : after_hi;
            keys.request(a.c.k, next_lo, next_hi, lane);
            if constexpr (DT == BRL_I8) scales(a.c.ks, next_lo, next_hi, ks);
            __builtin_amdgcn_sched_barrier(0);
            const bool whole = slot0 + 32 <= all_see && mine && lo >= 0 && hi >= 0;
            float vf[8];
            if constexpr (DT == BRL_I8) {
                const float f[8] = {vs[0].x, vs[0].y, vs[0].z, vs[0].w, vs[1].x, vs[1].y, vs[1].z, vs[1].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) vf[e] = f[e];
            }
            uint32_t odd = 0;                                          // keys with strange values
            values.store(lds, at);
            if (!whole) {
                const int n = mine ? seen - slot0 : 0;
                uint32_t there = n >= 32 ? 0xffffffffu : n > 0 ? (1u << n) - 1u : 0u;
                if (lo < 0) there &= 0xffff0000u;
                if (hi < 0) there &= 0x0000ffffu;
                if (there != 0xffffffffu) clear_rows<S>(lds, lane, there);
                const uint32_t own = bits_of_group(there, g);
                if constexpr (DT == BRL_I8) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (own >> e & 1u && strange_scale(vf[e])) odd |= 1u << key_of_score(g, e);
                        vf[e] = own >> e & 1u && !strange_scale(vf[e]) ? vf[e] : 0.f;
                    }
                    odd = any_lane(odd);
                } else if (values.suspicious()) {
                    odd = take_strange<S>(lds, lane);
                }
                odd &= there;
                const uint32_t bits = own & bits_of_group(visible_bits(a, st, token, slot0), g);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = bits >> e & 1u ? s[e] : -INFINITY;
            }
            __builtin_amdgcn_sched_barrier(0);
            values.request(a.c.v, next_lo, next_hi, lane);
            if constexpr (DT == BRL_I8) scales(a.c.vs, next_lo, next_hi, vs);
            __builtin_amdgcn_sched_barrier(0);
            const int here_lo = lo, here_hi = hi;
            lo = next_lo;
            hi = next_hi;
            if (!mine) break;
            if (p.scores && live) {
                float* f = p.scores + (((size_t)b * a.c.n_kv + h) * p.rows_max + c) * p.ld_scores + slot0 + 4 * g;
                reinterpret_cast<float4*>(f)[0] = make_float4(s[0], s[1], s[2], s[3]);
                reinterpret_cast<float4*>(f)[4] = make_float4(s[4], s[5], s[6], s[7]);
            }
            row.probabilities(s, vf);
            if (odd) add_strange<S>(a.c, here_lo, here_hi, odd, s, row, at);
            if constexpr (DT == BRL_I8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] *= vf[e];
            }
            __builtin_amdgcn_wave_barrier();
            block_values<S, 1>(lds, &s, &row, at);
            __builtin_amdgcn_wave_barrier();
            t += waves;
        } while (t < last);
        // the wavefronts' parts meet: sums to the largest reference, then O over LDS
        row.l += __shfl_xor(row.l, 16, 64);
        row.l += __shfl_xor(row.l, 32, 64);
        if (g == 0) s_ml[wave][c] = make_float2(row.l > 0.f ? row.ref : -INFINITY, row.l);
        __syncthreads();
        float top = -INFINITY;
#pragma unroll 4
        for (int w = 0; w < waves; ++w) top = fmaxf(top, s_ml[w][c].x);
        const float f = row.l > 0.f ? __builtin_amdgcn_exp2f(row.ref - top) : 0.f;
        if (g == 0) s_l[wave][c] = row.l * f;
        float* o = reinterpret_cast<float*>(lds);                      // [16 rows][OS]
#pragma unroll
        for (int d = 0; d < S::DTL; ++d) *reinterpret_cast<v4f*>(o + c * OS + 16 * d + 4 * g) = row.o[d] * f;
        __syncthreads();
        const size_t slot = (2 * (size_t)blockIdx.x + (before ? 0 : 1)) * p.rows_pad;
        for (int i = threadIdx.x; i < rows * (S::ROW / 4); i += blockDim.x) {
            const int r = i / (S::ROW / 4), d = i % (S::ROW / 4) * 4;
            if (d >= DH) continue;
            float ref = -INFINITY, l = 0.f;
            v4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int w = 0; w < waves; ++w) {
                ref = fmaxf(ref, s_ml[w][r].x);
                l += s_l[w][r];
                sum += *reinterpret_cast<const v4f*>(reinterpret_cast<const float*>(lds_all + w * LDS) + r * OS + d);
            }
            if (all) {
                *reinterpret_cast<v4f*>(out_row(a, st, h, p.group, r) + d) = sum * (l > 0.f ? 1.f / l : 0.f);
                if (p.lse && d == 0) p.lse[((size_t)b * a.c.n_kv + h) * p.rows_pad + r] = log_sum(ref, l);
            } else {
                *reinterpret_cast<v4f*>(p.part_o + (slot + r) * DH + d) = sum;
                if (d == 0) p.part_ml[slot + r] = make_float2(ref, l);
            }
        }
        if (left <= 0) return;
        __syncthreads();
        before = false;
        next_segment(b, h, st);
        blocks = blocks_of(st);
        first = 0;
        last = left < blocks ? left : blocks;
        pages(wave, here);
        token = p.group.token(query_row(c));
        pos = position(token);
    }
}

// ---- parts of a row's keys joined ----
// 256 threads: four components of the row each, LANES of them; the rest of the threads share the parts, or are other rows.
template <int DH, int GROUPS>
struct Joiner {
    static constexpr int LANES = DH == 100 ? 32 : DH / 4, PER = 256 / LANES;
    static_assert(GROUPS == 1 || GROUPS == PER, "all on one row, or each on its own");
    // parts w0 .. w1 at place(w) of part_ml and part_o
    template <class Place>
    static __device__ __forceinline__ void run(const Plan& p, unsigned w0, unsigned w1, Place place, float* y, float* lse) {
        __shared__ __attribute__((aligned(16))) float s_o[PER][DH];
        __shared__ float s_l[PER];
        const int d = threadIdx.x % LANES * 4, part = threadIdx.x / LANES;
        float ref = -INFINITY;
        if constexpr (GROUPS == 1) {
            for (unsigned w = w0 + (threadIdx.x & 63); w <= w1; w += 64) ref = fmaxf(ref, p.part_ml[place(w)].x);
            ref = wave_max(ref);
        } else {
            for (unsigned w = w0; w <= w1; ++w) ref = fmaxf(ref, p.part_ml[place(w)].x);
        }
        float l = 0.f;
        v4f o = {0.f, 0.f, 0.f, 0.f};
        constexpr unsigned STEP = GROUPS == 1 ? PER : 1;
#pragma unroll 4
        for (unsigned w = w0 + (GROUPS == 1 ? part : 0); w <= w1; w += STEP) {
            const float2 ml = p.part_ml[place(w)];
            const v4f x = d < DH ? *reinterpret_cast<const v4f*>(p.part_o + place(w) * DH + d) : v4f{0.f, 0.f, 0.f, 0.f};
            const float f = ml.y > 0.f ? __builtin_amdgcn_exp2f(ml.x - ref) : 0.f;
            l += ml.y * f;
            o += x * f;
        }
        if constexpr (GROUPS == 1) {
            if (d < DH) *reinterpret_cast<v4f*>(&s_o[part][d]) = o;
            if (d == 0) s_l[part] = l;
            __syncthreads();
            if (part != 0) return;
            l = 0.f;
            o = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                l += s_l[x];
                if (d < DH) o += *reinterpret_cast<const v4f*>(&s_o[x][d]);
            }
        }
        if (d < DH) *reinterpret_cast<v4f*>(y + d) = o * (l > 0.f ? 1.f / l : 0.f);
        if (lse && d == 0) *lse = log_sum(ref, l);
    }
};

// few rows: the parts that workgroups of the shared list took, a workgroup per row
template <int DH>
__global__ __launch_bounds__(256) void cached_join_kernel(CachedAttention a, Plan p) {
    const int r = blockIdx.x % p.rows_max, h = blockIdx.x / p.rows_max % a.c.n_kv, b = blockIdx.x / p.rows_max / a.c.n_kv;
    const StateTokens st = state_tokens(a.t, a.c, b);
    if (r >= st.n * p.group.n) return;
    const int lane = threadIdx.x & 63;
    const Prefix pre = prefix_blocks(a, lane);
    const unsigned share = share_of(p, (unsigned)pre.total * a.c.n_kv);
    unsigned start = lane_value(pre.before, b / pre.stretch);
    for (int x = b / pre.stretch * pre.stretch; x < b; ++x) start += state_blocks(a, x);
    const int blocks = (st.len + 31) >> 5;
    start = start * a.c.n_kv + (unsigned)h * blocks;
    float* y = out_row(a, st, h, p.group, r);
    float* lse = p.lse ? p.lse + ((size_t)b * a.c.n_kv + h) * p.rows_pad + r : nullptr;
    if (blocks == 0) {                                                 // no workgroup of the list comes by
        if (threadIdx.x < DH) y[threadIdx.x] = 0.f;
        if (lse && threadIdx.x == 0) *lse = INFINITY;
        return;
    }
    const unsigned w0 = start / share, w1 = (start + blocks - 1) / share;
    if (w0 == w1) return;                                              // written by that workgroup
    Joiner<DH, 1>::run(p, w0, w1, [&](unsigned w) { return (2 * (size_t)w + (w == w0 && start > w * share ? 1 : 0)) * p.rows_pad + r; }, y, lse);
}

// many rows: a fixed number of parts; a workgroup for several rows where they are few
template <int DH, int GROUPS>
__global__ __launch_bounds__(256) void cached_join_splits_kernel(CachedAttention a, Plan p) {
    const long long i = (long long)blockIdx.x * GROUPS + (GROUPS == 1 ? 0 : threadIdx.x / Joiner<DH, GROUPS>::LANES);
    const int r = (int)(i % p.rows_max), unit = (int)(i / p.rows_max), h = unit % a.c.n_kv, b = unit / a.c.n_kv;
    if (b >= a.t.B) return;
    const StateTokens st = state_tokens(a.t, a.c, b);
    if (r >= st.n * p.group.n) return;
    const size_t at = ((size_t)unit * p.rows_pad + r) * p.splits;
    Joiner<DH, GROUPS>::run(p, 0u, (unsigned)p.splits - 1, [&](unsigned w) { return at + w; }, out_row(a, st, h, p.group, r),
                            p.lse ? p.lse + (size_t)unit * p.rows_pad + r : nullptr);
}

// ---- weights of slots from the stored scores: a thread per four slots ----
__global__ __launch_bounds__(256) void cached_weights_kernel(CachedAttention a, Plan p, int chunks) {
    const int h = blockIdx.x / chunks % a.c.n_kv, b = blockIdx.x / chunks / a.c.n_kv;
    const StateTokens st = state_tokens(a.t, a.c, b);
    const int rows = st.n * p.group.n, slot = (blockIdx.x % chunks * 256 + threadIdx.x) * 4;
    const size_t unit = (size_t)b * a.c.n_kv + h;
    if (slot >= st.len) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
        const float4 s = *reinterpret_cast<const float4*>(p.scores + (unit * p.rows_max + r) * p.ld_scores + slot);
        const float lse = p.lse[unit * p.rows_pad + r];
        w[0] += __builtin_amdgcn_exp2f(s.x - lse);
        w[1] += __builtin_amdgcn_exp2f(s.y - lse);
        w[2] += __builtin_amdgcn_exp2f(s.z - lse);
        w[3] += __builtin_amdgcn_exp2f(s.w - lse);
    }
    float* y = a.weights + ((size_t)b * a.c.n_kv + h) * a.ld_weights + slot;
    for (int e = 0; e < 4; ++e)
        if (slot + e < st.len) y[e] += w[e];
}

// ---- many rows: the wavefronts of a workgroup share every block of keys and values through LDS ----
// A wavefront owns RT tiles of 16 rows, whose operands stay in its registers.  While a block is worked on, the next one is on its way
// into registers; it goes to the other half of LDS at the end, so that one barrier per block is enough.
template <class S>
struct SharedLoads {
    static constexpr int N = (32 * S::CPR + 255) / 256;
    uint4 k[N], v[N];
    float scale;
    __device__ __forceinline__ void request(const KvView& c, int lo, int hi, unsigned tid) {
        const size_t lo_at = (size_t)(lo < 0 ? 0 : lo) * S::RB, hi_at = (size_t)(hi < 0 ? 0 : hi) * S::RB;
        constexpr int HALF = 16 * S::CPR;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            unsigned idx = i * 256 + tid;                              // (past the end: the last chunk again, see ValueLoads)
            if (N * 256 > 32 * S::CPR && idx >= 32u * S::CPR) idx = 32 * S::CPR - 1;
            const size_t at = idx >= (unsigned)HALF ? hi_at + (size_t)((idx - HALF) * 16) : lo_at + (size_t)(idx * 16);
            k[i] = *reinterpret_cast<const uint4*>(c.k + at);
            v[i] = *reinterpret_cast<const uint4*>(c.v + at);
        }
        if constexpr (S::DT == BRL_I8) {
            const int key = tid & 31, r = key < 16 ? lo : hi;
            scale = (tid & 32 ? c.vs : c.ks)[(r < 0 ? 0 : r) + (key & 15)];
        }
    }
    // there: bit per key whose row holds numbers.  look: strange values are taken out; returns the keys of such rows (in an int8 cache:
    // scales) among what this wavefront has stored.
    template <bool LOOK>
    __device__ __forceinline__ uint32_t store(char* lds, float* scales, unsigned tid, uint32_t there, bool look) {
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const unsigned idx = i * 256 + tid, key = idx / S::CPR, ch = idx % S::CPR;
            if (N * 256 > 32 * S::CPR && idx >= 32u * S::CPR) continue;
            uint4 x = k[i], y = v[i];
            if (there != 0xffffffffu && !(there >> key & 1u)) y = make_uint4(0, 0, 0, 0);
            if constexpr (LOOK && S::DT != BRL_I8) {
                if (look) {
                    odd |= strange<S::DT>(y) ? 1u << key : 0u;
                    y = plain<S::DT>(y);
                }
            }
            if constexpr (S::ROW > S::DH) {                            // what lies behind head_dim is not a number
                constexpr int PER = 16 / S::SZ;
                const int valid = S::DH - (int)ch * PER;                    // elements of this chunk
                uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = j * (4 / S::SZ) < valid ? w[j] : 0u;
                x = make_uint4(w[0], w[1], w[2], w[3]);
            }
            put(lds, key, ch, x);
            put(lds + S::LDS, key, ch, y);
        }
        if constexpr (S::DT == BRL_I8) {
            if (tid < 64) {
                const bool mine = there >> (tid & 31) & 1u, other = LOOK && look && tid >= 32 && strange_scale(scale);
                scales[tid] = mine && !other ? scale : 0.f;
                odd = mine && other ? 1u << (tid & 31) : 0u;
            }
        }
        return LOOK ? any_lane(odd) : 0;
    }
    static __device__ __forceinline__ void put(char* lds, unsigned key, unsigned ch, const uint4& r) {
        if constexpr (S::DT == BRL_F16) {
            *reinterpret_cast<uint4*>(lds + lds_chunk<S>(key, ch)) = r;
        } else if constexpr (S::DT == BRL_F32) {
            uint2 h, l;
            split_pair(__uint_as_float(r.x), __uint_as_float(r.y), h.x, l.x);
            split_pair(__uint_as_float(r.z), __uint_as_float(r.w), h.y, l.y);
            char* p = lds + lds_chunk<S>(key, ch >> 1) + (ch & 1) * 8;
            *reinterpret_cast<uint2*>(p) = h;
            *reinterpret_cast<uint2*>(p + S::PLANE) = l;
        } else {
            uint4 a, b;
            widen_codes(r.x, a.x, a.y);
            widen_codes(r.y, a.z, a.w);
            widen_codes(r.z, b.x, b.y);
            widen_codes(r.w, b.z, b.w);
            *reinterpret_cast<uint4*>(lds + lds_chunk<S>(key, 2 * ch)) = a;
            *reinterpret_cast<uint4*>(lds + lds_chunk<S>(key, 2 * ch + 1)) = b;
        }
    }
};

// the slots that rows r0 .. r1 of a state can see at all end here
__device__ __forceinline__ int end_of_sight(const CachedAttention& a, const StateTokens& st, const Group& group, int r1) {
    const int n = a.tree ? st.len : st.base + group.token(r1) + 1;
    return n < 0 ? 0 : n;
}

template <int DT, int DH, int RT>
__global__ __launch_bounds__(256, 2) void cached_tiles_kernel(CachedAttention a, Plan p) {
    typedef Shape<DT, DH> S;
    constexpr int ROWS = 64 * RT;                                      // of a workgroup
    __shared__ __attribute__((aligned(16))) char s_kv[2][2 * S::LDS];   // keys, values; two blocks
    __shared__ float s_scale[2][64];
    __shared__ uint4 s_odd[2];                                         // keys with strange values, per wavefront that stored them
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    // blocks of rows from the last to the first: with causal masks the last see most keys
    const int units = a.t.B * a.c.n_kv, unit = blockIdx.x % units, split = blockIdx.x / units % p.splits;
    const int rb = p.row_blocks - 1 - (int)(blockIdx.x / units) / p.splits, h = unit % a.c.n_kv, b = unit / a.c.n_kv;
    const StateTokens st = state_tokens(a.t, a.c, b);
    const int rows = st.n * p.group.n, r0 = rb * ROWS;
    if (r0 >= rows) return;
    const int r1 = (r0 + ROWS < rows ? r0 + ROWS : rows) - 1;
    const int blocks = (end_of_sight(a, st, p.group, r1) + 31) >> 5, per = (blocks + p.splits - 1) / p.splits;
    const int first = split * per, last = first + per < blocks ? first + per : blocks;

    int page_lo = -1, page_hi = -1;
    auto pages = [&](int t0) {
        const int slot = (t0 + lane) * 32;
        page_lo = slot < st.len ? kv_row_index(a.c, b, h, slot) : -1;
        page_hi = slot + 16 < st.len ? kv_row_index(a.c, b, h, slot + 16) : -1;
    };
    auto there_of = [&](int t, int lo, int hi) {
        const int n = st.len - t * 32;
        uint32_t x = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
        if (lo < 0) x &= 0xffff0000u;
        if (hi < 0) x &= 0x0000ffffu;
        return x;
    };
    // Blocks under way in registers.  One row tile per wavefront is less work on a block than the way from memory takes: two.
    constexpr int DEPTH = RT == 1 ? 2 : 1;
    SharedLoads<S> load[DEPTH];
    int lo[DEPTH + 1], hi[DEPTH + 1];                                  // of the block worked on and of those under way
    int ahead;
    auto locate = [&](int t, int i) {
        lo[i] = t < last ? lane_value(page_lo, ahead) : -1;
        hi[i] = t < last ? lane_value(page_hi, ahead) : -1;
    };
    auto begin = [&]() {
        ahead = 0;
        if (first < last) pages(first);
        locate(first, 0);
        load[0].request(a.c, lo[0], hi[0], tid);
    };
    begin();
    // this wavefront's rows
    const int w0 = r0 + wave * 16 * RT, w1 = w0 + 16 * RT - 1 < r1 ? w0 + 16 * RT - 1 : r1;
    const bool busy = w0 <= r1;
    const int wave_blocks = busy ? (end_of_sight(a, st, p.group, w1) + 31) >> 5 : 0;
    const int all_see = st.base + (a.tree ? 0 : p.group.token(w0) + 1);
    RowState<S> row[RT];
    v8h qh[RT][S::KS], ql[RT][S::KS];
    int token[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int rr = w0 + r * 16 + c;
        token[r] = p.group.token(rr < rows ? rr : rows - 1);
        const QueryRow from(a, st, h, p.group, rr < rows ? rr : rows - 1, token[r], rope_position(a.t, st.row0 + token[r], st.base + token[r]));
#pragma unroll
        for (int s = 0; s < S::KS; ++s) {
            QueryPart<S, false> q;
            q.request(from, 32 * s + 8 * g);
            uint4 x, y;
            q.split(from, rr < rows, 32 * s + 8 * g, x, y);
            qh[r][s] = __builtin_bit_cast(v8h, x);
            ql[r][s] = __builtin_bit_cast(v8h, y);
            if (p.q && split == 0 && w0 + r * 16 <= r1)
                store_query<S>(p.q + ((size_t)unit * p.rows_pad + w0 + r * 16) / 16 * S::KS * 128, s, lane, x, y);
        }
    }
    if constexpr (S::NCH * 8 > S::ROW) {                               // components of the last step that no row has
        for (int i = tid; i < 2 * S::PL * 32 * (S::NCH - S::ROW / 8); i += 256) {
            const int x = i % (S::NCH - S::ROW / 8), key = i / (S::NCH - S::ROW / 8) % 32, plane = i / (S::NCH - S::ROW / 8) / 32;
            *reinterpret_cast<uint4*>(s_kv[plane / S::PL] + plane % S::PL * S::PLANE + lds_chunk<S>(key, S::ROW / 8 + x)) = make_uint4(0, 0, 0, 0);
        }
    }
    // LOOK: strange values are looked for in the blocks with new tokens, which not every row sees.
    auto pass = [&](auto looks) __attribute__((always_inline)) {
        constexpr bool LOOK = decltype(looks)::value;
        auto has_new = [&](int t) { return LOOK && t * 32 + 32 > st.base; };
        auto store = [&](SharedLoads<S>& from, int t, int to) {
            const uint32_t odd = from.template store<LOOK>(s_kv[to], s_scale[to], tid, there_of(t, lo[0], hi[0]), has_new(t));
            if (LOOK && lane == 0) reinterpret_cast<uint32_t*>(&s_odd[to])[wave] = odd;
        };
#pragma unroll
        for (int r = 0; r < RT; ++r) row[r].clear();
        store(load[0], first, 0);
        if constexpr (DEPTH == 2) {
            ++ahead;
            locate(first + 1, 1);
            load[1].request(a.c, lo[1], hi[1], tid);
        }
        __syncthreads();
        int buf = 0;
        for (int t0 = first; t0 < last; t0 += DEPTH) {
#pragma unroll
            for (int turn = 0; turn < DEPTH; ++turn) {
                const int t = t0 + turn;
                if (DEPTH > 1 && t >= last) break;
                if (++ahead == 64) {
                    ahead = 0;
                    pages(t + DEPTH);
                }
                // (block t was in load[turn])
                locate(t + DEPTH, DEPTH);
                load[turn].request(a.c, lo[DEPTH], hi[DEPTH], tid);
                __builtin_amdgcn_sched_barrier(0);
                if (t < wave_blocks) {
                    const char* keys = s_kv[buf];
                    const char* vals = keys + S::LDS;
                    float s[RT][8];
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) {
                        v4f acc[RT];
#pragma unroll
                        for (int r = 0; r < RT; ++r) acc[r] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int x = 0; x < S::KS; ++x) {
                            const char* f = keys + lds_chunk<S>(16 * kt + c, (4 * x + g) & (S::NCH - 1));
                            const v8h kh = __builtin_bit_cast(v8h, *reinterpret_cast<const uint4*>(f));
                            v8h kl;
                            if constexpr (S::PL == 2) kl = __builtin_bit_cast(v8h, *reinterpret_cast<const uint4*>(f + S::PLANE));
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                if constexpr (S::PL == 2) acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl, qh[r][x], acc[r], 0, 0, 0);
                                acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, ql[r][x], acc[r], 0, 0, 0);
                                acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, qh[r][x], acc[r], 0, 0, 0);
                            }
                        }
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int j = 0; j < 4; ++j) s[r][4 * kt + j] = acc[r][j];
                    }
                    float vf[8];
                    if constexpr (DT == BRL_I8) {
                        float kf[8];
#pragma unroll
                        for (int e = 0; e < 8; e += 4) {
                            *reinterpret_cast<float4*>(kf + e) = *reinterpret_cast<const float4*>(&s_scale[buf][key_of_score(0, e) + 4 * g]);
                            *reinterpret_cast<float4*>(vf + e) = *reinterpret_cast<const float4*>(&s_scale[buf][32 + key_of_score(0, e) + 4 * g]);
                        }
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int e = 0; e < 8; ++e) s[r][e] *= kf[e];
                    }
                    if (t * 32 + 32 > all_see || lo[0] < 0 || hi[0] < 0) {
                        const uint32_t mine = bits_of_group(there_of(t, lo[0], hi[0]), g);
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const uint32_t bits = mine & bits_of_group(visible_bits(a, st, token[r], t * 32), g);
#pragma unroll
                            for (int e = 0; e < 8; ++e) s[r][e] = bits >> e & 1u ? s[r][e] : -INFINITY;
                        }
                    }
#pragma unroll
                    for (int r = 0; r < RT; ++r) row[r].probabilities(s[r], vf);
                    if (LOOK && has_new(t)) {
                        const uint4 x = s_odd[buf];
                        const uint32_t odd = __builtin_amdgcn_readfirstlane(x.x | x.y | x.z | x.w);
                        if (odd) {
#pragma unroll
                            for (int r = 0; r < RT; ++r) add_strange<S>(a.c, lo[0], hi[0], odd, s[r], row[r], lane);
                        }
                    }
                    if constexpr (DT == BRL_I8) {
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int e = 0; e < 8; ++e) s[r][e] *= vf[e];
                    }
                    block_values<S, RT>(vals, s, row, lane);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < DEPTH; ++i) {
                    lo[i] = lo[i + 1];
                    hi[i] = hi[i + 1];
                }
                store(load[(turn + 1) % DEPTH], t + 1, buf ^ 1);
                buf ^= 1;
                __syncthreads();
            }
        }
    };
    pass(std::false_type());
    // Sums that came out infinite or NaN: once more, with a look at the values.  (Always with it, 4 prompts of 4096 tokens and 20 heads of
    // 128, fp16: 697 us instead of 640.)
    float zero = 0.f;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int d = 0; d < S::DTL; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) zero = __builtin_fmaf(row[r].o[d][j], 0.f, zero);
    if (__syncthreads_or(zero != 0.f)) {                               // (NaN is not equal to anything)
        begin();
        pass(std::true_type());
    }
    if (!busy) return;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float l = row[r].l;
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        const int rr = w0 + r * 16 + c;
        if (rr > r1) continue;
        float f = 1.f;
        float* y;
        if (p.splits == 1) {
            f *= l > 0.f ? 1.f / l : 0.f;
            y = out_row(a, st, h, p.group, rr);
            if (p.lse && g == 0) p.lse[(size_t)unit * p.rows_pad + rr] = log_sum(row[r].ref, l);
        } else {
            const size_t at = ((size_t)unit * p.rows_pad + rr) * p.splits + split;
            y = p.part_o + at * DH;
            if (g == 0) p.part_ml[at] = make_float2(l > 0.f ? row[r].ref : -INFINITY, l);
        }
#pragma unroll
        for (int d = 0; d < S::DTL; ++d)
            if (16 * d + 4 * g < DH) *reinterpret_cast<v4f*>(y + 16 * d + 4 * g) = row[r].o[d] * f;
    }
}

// Weights of slots, many rows: the scores once more.  A wavefront keeps a block of 32 keys in registers and walks the row tiles that
// can see it (the next tile's queries on their way meanwhile); each lane sums its eight keys over its row of every tile, the sixteen rows
// meet at the end.  Where blocks are few the row tiles go round among w_parts wavefronts.
// Blocks per wavefront: every tile's queries come from the caches for each wavefront, 8 KB at heads of 128, so two where the keys' operands
// leave the registers (80 heads, 2000 slots, 4000 rows, fp16: 970 us a call with two, 1250 with one).
template <int DT>
struct WeightBlocks {
    static constexpr int N = DT == BRL_F32 ? 1 : 2;
};
template <int DT, int DH>
__global__ __launch_bounds__(256, 2) void cached_tile_weights_kernel(CachedAttention a, Plan p, int chunks) {
    typedef Shape<DT, DH> S;
    constexpr int NB = WeightBlocks<DT>::N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int units = a.t.B * a.c.n_kv, unit = blockIdx.x / chunks % units, part = blockIdx.x / chunks / units;
    const int h = unit % a.c.n_kv, b = unit / a.c.n_kv;
    const StateTokens st = state_tokens(a.t, a.c, b);
    const int rows = st.n * p.group.n, slot0 = (blockIdx.x % chunks * 4 + wave) * 32 * NB;
    if (rows == 0 || slot0 >= st.len) return;
    v8h key[NB][2][S::KS][S::PL];
    float kf[NB][8];
    uint32_t mine[NB];                                                 // which of this lane's keys there are
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int slot = slot0 + 32 * n, left = st.len - slot;
        const int lo = left > 0 ? kv_row_index(a.c, b, h, slot) : -1, hi = left > 16 ? kv_row_index(a.c, b, h, slot + 16) : -1;
        uint32_t there = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u;
        if (lo < 0) there &= 0xffff0000u;
        if (hi < 0) there &= 0x0000ffffu;
        mine[n] = bits_of_group(there, g);
        KeyLoads<S> raw;
        raw.request(a.c.k, lo, hi, lane);
        if constexpr (DT == BRL_I8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) kf[n][e] = a.c.ks[((e < 4 ? lo : hi) < 0 ? 0 : (e < 4 ? lo : hi)) + 4 * g + (e & 3)];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < S::KS; ++s) raw.fragment(t, s, lane, key[n][t][s]);
    }
    float sum[NB][8] = {};
    const int token0 = a.tree || slot0 <= st.base ? 0 : slot0 - st.base;          // the first token that sees the first slot
    const int tiles = (rows + 15) / 16;
    int rt = token0 * p.group.n / 16 + part;
    v8h qh[2][S::KS], ql[2][S::KS];                                    // of the tile worked on and of the next
    float lse[2];
    auto request = [&](int t, int i) __attribute__((always_inline)) {
        if (t >= tiles) t = tiles - 1;                                 // (not used)
        const uint4* q = p.q + (((size_t)unit * p.rows_pad / 16 + t) * S::KS * 2) * 64 + lane;
#pragma unroll
        for (int s = 0; s < S::KS; ++s) {
            qh[i][s] = __builtin_bit_cast(v8h, q[s * 128]);
            ql[i][s] = __builtin_bit_cast(v8h, q[s * 128 + 64]);
        }
        const int r = t * 16 + c;
        lse[i] = p.lse[(size_t)unit * p.rows_pad + (r < rows ? r : rows - 1)];
    };
    auto add = [&](int t, int i) __attribute__((always_inline)) {
        const int r = t * 16 + c, token = p.group.token(r < rows ? r : rows - 1);
        const int all_see = st.base + (a.tree ? 0 : p.group.token(t * 16) + 1);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            v4f acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int s = 0; s < S::KS; ++s) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if constexpr (S::PL == 2) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[n][t][s][1], qh[i][s], acc[t], 0, 0, 0);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[n][t][s][0], ql[i][s], acc[t], 0, 0, 0);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[n][t][s][0], qh[i][s], acc[t], 0, 0, 0);
                }
            }
            uint32_t bits = r < rows ? mine[n] : 0u;
            if (slot0 + 32 * n + 32 > all_see) bits &= bits_of_group(visible_bits(a, st, token, slot0 + 32 * n), g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float x = acc[e >> 2][e & 3];
                if constexpr (DT == BRL_I8) x *= kf[n][e];
                sum[n][e] += bits >> e & 1u ? __builtin_amdgcn_exp2f(x - lse[i]) : 0.f;
            }
        }
    };
    request(rt, 0);
    for (; rt < tiles; rt += 2 * p.w_parts) {
        request(rt + p.w_parts, 1);
        __builtin_amdgcn_sched_barrier(0);
        add(rt, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (rt + p.w_parts >= tiles) break;
        request(rt + 2 * p.w_parts, 0);
        __builtin_amdgcn_sched_barrier(0);
        add(rt + p.w_parts, 1);
        __builtin_amdgcn_sched_barrier(0);
    }
    float* y = p.w_parts == 1 ? a.weights + (size_t)unit * a.ld_weights + slot0 : p.part_w + ((size_t)part * units + unit) * p.ld_scores + slot0;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x = sum[n][e];
            x += lane_exchange<DPP_XOR1>(x);
            x += lane_exchange<DPP_XOR2>(x);
            x += lane_exchange<DPP_HALF_MIRROR>(x);
            x += lane_exchange<DPP_MIRROR>(x);
            if (c != 0) continue;
            if (p.w_parts > 1) y[32 * n + key_of_score(g, e)] = x;
            else if (mine[n] >> e & 1u) y[32 * n + key_of_score(g, e)] += x;
        }
    }
}
// the parts of the rows added up, in their order: a thread per slot
__global__ __launch_bounds__(256) void cached_sum_weights_kernel(CachedAttention a, Plan p, int chunks) {
    const int unit = blockIdx.x / chunks, slot = blockIdx.x % chunks * 256 + threadIdx.x;
    const StateTokens st = state_tokens(a.t, a.c, unit / a.c.n_kv);
    if (st.n == 0 || slot >= st.len) return;
    const float* x = p.part_w + (size_t)unit * p.ld_scores + slot;
    float w = 0.f;
#pragma unroll 8
    for (int i = 0; i < p.w_parts; ++i) w += x[(size_t)i * a.t.B * a.c.n_kv * p.ld_scores];
    a.weights[(size_t)unit * a.ld_weights + slot] += w;
}

struct Layout {
    Plan p;
    bool tiles;               // many rows
    int waves, rt;            // few rows: wavefronts of a workgroup; many: row tiles of a wavefront
    size_t o_off, ml_off, lse_off, scores_off, q_off, w_off, total;
};

Layout plan_cached(const KvView& c, int n_heads, int B, int max_new, int max_len, bool weights) {
    Layout L;
    memset(&L, 0, sizeof(L));
    Plan& p = L.p;
    p.group.n = n_heads / c.n_kv;
    p.group.inverse = p.group.n == 1 ? 0u : (uint32_t)(((1ull << 32) + p.group.n - 1) / p.group.n);
    p.rows_max = max_new * p.group.n;
    p.splits = 1;
    const int units = B * c.n_kv, blocks = (max_len + 31) / 32;
    // 16 rows fill one column block of the matrix instructions; more would have a wavefront of the first form hold two.  64 states of 1000-2000
    // slots, 5 heads of 128, first form / second, us: 4 rows fp32 105 / 114, fp16 58 / 71, int8 41 / 62; 16 rows 117 / 120, 70 / 75, 51 / 64.
    L.tiles = p.rows_max > 16;
    size_t parts;
    if (!L.tiles) {
        p.rows_pad = 16;
        // A workgroup per (state, k/v head) needs no second launch (about 7 us) but takes all of a state's keys through one compute unit:
        // up to two turns of its eight wavefronts of an fp32 cache, four of the others, which are half the work, twice that
        // where there are workgroups to fill every unit.  Heads of 128, this form / shared, us, fp32, fp16 and int8: 5 of 300 slots 16.2 / 20.8,
        // 10.3 / 16.2, 10.4 / 17.3; 5 of 500 19.3 / 15.0, 11.5 / 12.4, 11.4 / 12.8; 5 of 1000 29.0 / 15.1, 16.5 / 12.3, 15.0 / 12.9; 255 of 1000
        // 52 / 58, 28.3 / 33.4, 18.3 / 23.3; 320 of 1000 76 / 72, 40 / 43, 25 / 30; 550 of 1800 204 / 193, 105 / 108, 71 / 74.
        const int whole = c.dtype == BRL_F32 ? 16 : 32;
        if (blocks <= whole || (units >= 512 && blocks <= 64) || (long long)units * p.rows_max > (1 << 22) ||
            (long long)units * blocks >= (1ll << 31)) {
            // Eight wavefronts where a workgroup has a compute unit to itself and blocks for them, else four, so that two workgroups share
            // a unit.  4 / 8, us: 5 of 120 slots fp32 11.0 / 15.4, fp16 8.9 / 9.5; 5 of 1000 int8 17.7 / 15.0; 255 of 1800 fp32 89 / 85, fp16 47 / 45,
            // int8 31 / 28; 320 of 300 fp16 16.3 / 22.1, of 1000 40 / 45; 1280 of 300 fp32 82 / 105, fp16 47 / 63; 4000 of 1000 355 / 379.
            L.waves = blocks <= 4 || units > 256 ? 4 : 8;
        } else {
            L.waves = 4;
            p.groups = 512;                           // as many as run at a time
            p.least = 4;
        }
        parts = 2 * (size_t)p.groups * p.rows_pad;
    } else {
        L.rt = p.rows_max <= 64 ? 1 : 2;
        p.row_blocks = (p.rows_max + 64 * L.rt - 1) / (64 * L.rt);
        p.rows_pad = p.row_blocks * 64 * L.rt;
        // (512 workgroups run at a time.)
        const long long groups = (long long)units * p.row_blocks;
        const int new_blocks = (max_new + 31) / 32, most = blocks / 8 < 64 ? blocks / 8 : 64;
        if (4 * new_blocks < blocks) {
            // Long keys.  A workgroup costs its blocks and about four more (queries, first loads, end), parts that have to be joined another
            // four; the split with the shortest sum of rounds.  This / the other rule's number of parts, heads of 128, fp16 and fp32, us: 80
            // workgroups (8 x 48 tokens on 2000 slots) 44 / 57 and 60 / 73; 140 (4 x 200 on 2000) 67 / 78 and 91 / 108; 190 (38 x 7 on 5000) 121 /
            // 113 and 199 / 243; 320 (64 x 7 on 2000) 89 / 83 and 147 / 130, int8 77 / 90; 640 (128 x 7 on 5000) 351 / 315 and 620 / 684, int8 288 / 353.
            // With a quarter of the slots new and more, or few workgroups, both rules choose alike or nearly so.
            long long best = 0;
            for (int s = 1; s == 1 || s <= most; ++s) {
                const long long cost = (groups * s + 511) / 512 * ((blocks + s - 1) / s + 4) + (s > 1 ? 4 + s / 8 : 0);
                if (s == 1 || cost < best) { best = cost; p.splits = s; }
            }
        } else {
            // Mostly new tokens: workgroups of every length, the longest first, fill the rounds by themselves, and there are many rows
            // to be joined: only until all units have work.  1 / 2 / 3 / 4 parts, us: 650 workgroups (2 x 2000 tokens, 5 groups of 4 heads of
            // 128, fp16) 115 / 144 / 171 / 184; 640 205 / 225 / 250 / 251; 512 (heads of 100) 105 / 128 / 139 / 152; 256 (fp32) 80 / 68 /
            // 80 / 85; 235 (fp32) 107 / 84 / 81 / 90; 136 (heads of 64) 64 / 46 / 39 / 37.  160 (1 x 1000, fp16): 44 with 3, 54 with 4; 188 (heads
            // of 16): 39 with 2, 32 with 3.  320 (2 x 1000): fp16 56 / 62 / 74 / 88, fp32 81 / 71 / 87 / 101.
            const long long s = 576 / groups;
            p.splits = s < 1 || most < 1 ? 1 : s < most ? (int)s : most;
        }
        parts = p.splits > 1 ? (size_t)units * p.rows_pad * p.splits : 0;
    }
    const size_t rows = (size_t)units * p.rows_pad;
    size_t off = 0;
    auto take = [&off](size_t bytes) {
        const size_t at = off;
        off += round_up_sz(bytes, 256);
        return at;
    };
    L.o_off = take(parts * c.dh * 4);
    L.ml_off = take(parts * 8);
    if (weights) {
        L.lse_off = take(rows * 4);
        if (L.tiles) {
            L.q_off = take(rows * ((c.dh + 31) / 32) * 32 * 4);
            // A block's wavefront walks the row tiles one after the other: parts until there are four wavefronts per SIMD, of four tiles at
            // least.  us of a call, one part / so: 2 heads of 16, 1800 slots, 7600 rows 239 / 42; 10 of 128, 2800 slots, int8, 5900
            // rows 1076 / 328; 5 of 128, 512 slots, fp32, 2048 rows 190 / 52.
            const int own = c.dtype == BRL_F32 ? WeightBlocks<BRL_F32>::N : WeightBlocks<BRL_F16>::N;
            const int row_blocks = (blocks + own - 1) / own;             // wavefronts that it takes for a unit's keys
            const long long want = 4096 / ((long long)units * row_blocks), most = (p.rows_max + 63) / 64;
            p.w_parts = want > most ? (int)most : want > 1 ? (int)want : 1;
            if (p.w_parts > 32) p.w_parts = 32;
            p.ld_scores = (size_t)row_blocks * own * 32;
            if (p.w_parts > 1) L.w_off = take((size_t)p.w_parts * units * p.ld_scores * 4);
        } else {
            p.ld_scores = (size_t)blocks * 32;
            L.scores_off = take((size_t)units * p.rows_max * p.ld_scores * 4);
        }
    }
    L.total = off;
    return L;
}

template <int DT, int DH>
int launch_few(const CachedAttention& a, const Layout& L, hipStream_t s) {
    const Plan& p = L.p;
    const dim3 grid((unsigned)(p.groups ? p.groups : a.t.B * a.c.n_kv)), block(L.waves * 64);
    const size_t lds = (size_t)L.waves * StreamShape<DT, DH>::LDS;
    hipLaunchKernelGGL((cached_stream_kernel<DT, DH>), grid, block, lds, s, a, p);
    BRL_LAUNCH_CHECK("cached_stream_kernel");
    if (p.groups) {
        hipLaunchKernelGGL(cached_join_kernel<DH>, dim3((unsigned)(a.t.B * a.c.n_kv * p.rows_max)), dim3(256), 0, s, a, p);
        BRL_LAUNCH_CHECK("cached_join_kernel");
    }
    if (a.weights) {
        const int chunks = (a.t.max_len + 1023) / 1024;
        hipLaunchKernelGGL(cached_weights_kernel, dim3((unsigned)(a.t.B * a.c.n_kv * chunks)), dim3(256), 0, s, a, p, chunks);
        BRL_LAUNCH_CHECK("cached_weights_kernel");
    }
    return BRL_OK;
}

template <int DT, int DH>
int launch_many(const CachedAttention& a, const Layout& L, hipStream_t s) {
    const Plan& p = L.p;
    const int units = a.t.B * a.c.n_kv;
    const dim3 grid((unsigned)(units * p.row_blocks * p.splits)), block(256);
    if (L.rt == 1) hipLaunchKernelGGL((cached_tiles_kernel<DT, DH, 1>), grid, block, 0, s, a, p);
    else hipLaunchKernelGGL((cached_tiles_kernel<DT, DH, 2>), grid, block, 0, s, a, p);
    BRL_LAUNCH_CHECK("cached_tiles_kernel");
    if (p.splits > 1) {
        constexpr int PER = Joiner<DH, 1>::PER;
        const unsigned rows = (unsigned)(units * p.rows_max);
        // (a workgroup for several rows where the parts are few or the rows many: 1 x 2000 tokens, 8 heads of 32, 5 parts: 24 us a call, 33 with
        // one for each)
        if (p.splits <= 4 || rows > 4096) hipLaunchKernelGGL((cached_join_splits_kernel<DH, PER>), dim3((rows + PER - 1) / PER), dim3(256), 0, s, a, p);
        else hipLaunchKernelGGL((cached_join_splits_kernel<DH, 1>), dim3(rows), dim3(256), 0, s, a, p);
        BRL_LAUNCH_CHECK("cached_join_splits_kernel");
    }
    if (a.weights) {
        constexpr int SLOTS = 128 * WeightBlocks<DT>::N;               // of a workgroup
        const int chunks = (a.t.max_len + SLOTS - 1) / SLOTS;
        hipLaunchKernelGGL((cached_tile_weights_kernel<DT, DH>), dim3((unsigned)(units * chunks * p.w_parts)), block, 0, s, a, p, chunks);
        BRL_LAUNCH_CHECK("cached_tile_weights_kernel");
        if (p.w_parts > 1) {
            const int all = (a.t.max_len + 255) / 256;
            hipLaunchKernelGGL(cached_sum_weights_kernel, dim3((unsigned)(units * all)), dim3(256), 0, s, a, p, all);
            BRL_LAUNCH_CHECK("cached_sum_weights_kernel");
        }
    }
    return BRL_OK;
}

template <int DT>
int launch_typed(const CachedAttention& a, const Layout& L, hipStream_t s) {
    switch (a.c.dh) {
        case 16: return L.tiles ? launch_many<DT, 16>(a, L, s) : launch_few<DT, 16>(a, L, s);
        case 32: return L.tiles ? launch_many<DT, 32>(a, L, s) : launch_few<DT, 32>(a, L, s);
        case 64: return L.tiles ? launch_many<DT, 64>(a, L, s) : launch_few<DT, 64>(a, L, s);
        case 100: return L.tiles ? launch_many<DT, 100>(a, L, s) : launch_few<DT, 100>(a, L, s);
        default: return L.tiles ? launch_many<DT, 128>(a, L, s) : launch_few<DT, 128>(a, L, s);
    }
}

}  // namespace

size_t cached_attention_ws_bytes(const KvView& c, int n_heads, int B, int max_new, int max_len, bool weights) {
    return plan_cached(c, n_heads, B, max_new, max_len, weights).total;
}

int launch_cached_attention(const CachedAttention& a, void* workspace, hipStream_t s) {
    Layout L = plan_cached(a.c, a.n_heads, a.t.B, a.t.max_new, a.t.max_len, a.weights != nullptr);
    char* base = static_cast<char*>(workspace);
    Plan& p = L.p;
    p.part_o = reinterpret_cast<float*>(base + L.o_off);
    p.part_ml = reinterpret_cast<float2*>(base + L.ml_off);
    if (a.weights) {
        p.lse = reinterpret_cast<float*>(base + L.lse_off);
        if (L.tiles) {
            p.q = reinterpret_cast<uint4*>(base + L.q_off);
            p.part_w = reinterpret_cast<float*>(base + L.w_off);
        } else p.scores = reinterpret_cast<float*>(base + L.scores_off);
    }
    LaunchTimer tm(BRL_KC_ATTENTION, s);
    return a.c.dtype == BRL_F32 ? launch_typed<BRL_F32>(a, L, s) : a.c.dtype == BRL_F16 ? launch_typed<BRL_F16>(a, L, s)
                                                                                       : launch_typed<BRL_I8>(a, L, s);
}

}  // namespace brl
