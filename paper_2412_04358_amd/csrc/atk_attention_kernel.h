// Attention over a paged cache whose first keys all sequences of a batch share: one range of keys against a block of queries.
//
// Softmax over keys in any number of ranges: a range keeps m = max s, l = sum 2^(c (s - m)), o = sum 2^(c (s - m)) v (s = q.k, c = scale * log2(e)), and
// ranges join by M = max m, l = sum 2^(c (m_i - M)) l_i, o likewise.  So a range can be any workgroup's: the shared keys are cut for all rows
// of all sequences together, a sequence's own keys for its rows, and attn_join_kernel joins what a row has.
//
// A wavefront takes 32 keys at a time and keeps everything in registers, without LDS between the products:
//   S^T = K Q^T by 16x16 matrix instructions: K is read as it lies (a lane has 16 bytes of one key), and a lane ends up with one query
//   (lane % 16) and eight keys, 4 * (lane / 16) + 0..3 of both halves of the 32.  Maximum and sum of a query are over its own registers and two
//   exchanges.
//   O^T = V^T P^T: P^T's operand is wanted as (query, eight keys) in a lane: what the lane already has, when these keys are taken in its order.  V's is
//   (d, the same eight keys): the lane reads DP/16 elements of each of the eight keys (a row of V over 16 lanes, whole lines) and
//   pairs them up with one v_perm for two elements; element i of a lane's piece goes to product i, so 16 lanes' pieces make the d's of a product
//   DP/16 apart, and a lane's results are contiguous in d again.
#pragma once

#include <type_traits>

#include "atk_decode_common.h"

namespace atk {

constexpr float kNoMax = -__builtin_inff();
constexpr int kAttnWaves = 4;      // of a workgroup of attn_range_kernel: they take turns at the tiles of its range and join through LDS
constexpr int kTileKeys = 32;      // keys of a wavefront that ranges are cut by
// Halves of 16 keys that a wavefront takes at a time: two, whose keys are the 32 of a 16-bit product; one in f32, whose products take a key of each lane group, where K and V of 32 keys would
// leave a SIMD one wavefront (12 sequences of 16 heads on 2047 + 191 keys of 128: 29 us with two halves, 26 with one).
constexpr int attn_halves(int elt) { return elt == ATK_F32 ? 1 : 2; }
constexpr float kLazyMax = 8.0f;   // the maximum that weights are taken relative to follows the true one when that is 2^8 above it: 2^8 times the largest weight is
                                   // far from f32's and bf16's range, and rescaling is rare

struct AttnDev {
    const void *q, *k, *v;
    void *out;
    float *lse;
    const int32_t *table, *lens, *seqs;
    int32_t *status;
    float *parts_o;    // [row][part][dim]
    float2 *parts_ml;  // [row][part]
    int64_t table_stride;
    int64_t qs[3], os[3], ks[3], vs[3];
    int batch, tokens, heads, kv_heads, group, dim;
    int rows, row_pages, n_pages;
    int prefix_len;
    int prefix_splits, prefix_blocks, prefix_keys;  // ranges of the shared keys, row blocks, keys of a range (a multiple of a workgroup's tiles)
    int own_splits, own_blocks;
    int n_prefix, prefix_grid, n_own;  // units of the shared keys and workgroups for them, which come first; units of own keys
    int own_from;                      // where own keys begin: prefix_len, or 0 where a sequence's workgroups take the shared ones as well
    int masked_grid, block_rows;       // workgroups that look for attn_block_kernel's units with masks; rows of such a unit
    int parts;         // prefix_splits + own_splits
    bool around;       // own keys past the caches
    bool direct;       // one part, attn_range's: it is the result, and no join follows
    FastDiv page;
    float scale, scale2;  // scale2: scale * log2(e)
};

// Element types: a 16-byte piece of a row, its products, and a lane's weights as the second product takes them.
template <int ELT>
struct AttnElt;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <>
struct AttnElt<ATK_BF16> {
    static constexpr int kBytes = 2;
    static constexpr float kBias = 0.0f;  // weights are 2^(s - m + kBias)
    static constexpr uint32_t kExp = 0x7f807f80u;
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    }
};
template <>
struct AttnElt<ATK_F16> {
    static constexpr int kBytes = 2;
    // f16 has no exponents below -24: many weights of 2^-25 beside one of 1 would vanish, and their sum need not be small.  2^7 above them, and at most 2^15 with
    // the lazy maximum, weights down to 2^-31 count.
    static constexpr float kBias = 7.0f;
    static constexpr uint32_t kExp = 0x7c007c00u;
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
    }
};
template <>
struct AttnElt<ATK_F32> {
    static constexpr int kBytes = 4;
    static constexpr float kBias = 0.0f;
    static constexpr uint32_t kExp = 0x7f800000u;
    // a piece is four elements: four products of one k each per lane group
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
};

template <int ELT>
__device__ __forceinline__ bool not_finite(uint32_t w) {
    if (ELT == ATK_F32) return (w & 0x7f800000u) == 0x7f800000u;
    constexpr uint32_t lo = AttnElt<ELT>::kExp & 0xffffu, hi = AttnElt<ELT>::kExp & 0xffff0000u;
    return (w & lo) == lo || (w & hi) == hi;
}

// AROUND: past the caches, for keys that are read once and are more than the caches hold.
template <bool AROUND, typename T>
__device__ __forceinline__ T fetch(const void *p) {
    return AROUND ? __builtin_nontemporal_load((const T *)p) : *(const T *)p;
}

// The rows of V that a lane has, four of each half: kDvl elements each.
template <int ELT, int DP>
struct VRows {
    static constexpr int kDvl = DP / 16;                                    // elements of a lane's piece of a row
    static constexpr int kWords = kDvl * AttnElt<ELT>::kBytes / 4;          // 32-bit words of it
    static constexpr int kVec = kWords % 4 == 0 ? 4 : 2;                    // words of a load
    static constexpr int kRows = 4 * attn_halves(ELT);
    uint32_t w[kRows][kWords];

    template <bool AROUND>
    __device__ __forceinline__ void load(int j, const char *row, int n, int dim) {
#pragma unroll
        for (int x = 0; x < kWords; x += kVec) {
            const int word = n * kWords + x;
            if (DP * AttnElt<ELT>::kBytes / 4 == kVec || word * 4 < dim * AttnElt<ELT>::kBytes) {
                if (kVec == 4) {
                    const u32x4 t = fetch<AROUND, u32x4>(row + word * 4);
#pragma unroll
                    for (int y = 0; y < 4; ++y) w[j][x + y] = t[y];
                } else {
                    const u32x2 t = fetch<AROUND, u32x2>(row + word * 4);
                    w[j][x] = t[0], w[j][x + 1] = t[1];
                }
            } else {
#pragma unroll
                for (int y = 0; y < kVec; ++y) w[j][x + y] = 0;
            }
        }
    }
    // the operand of product i in 16 bits: element i of all eight keys
    __device__ __forceinline__ u32x4 operand(int i) const {
        u32x4 r;
#pragma unroll
        for (int p = 0; p < 4; ++p)
            r[p] = __builtin_amdgcn_perm(w[2 * p + 1][i / 2], w[2 * p][i / 2], (i & 1) ? 0x07060302u : 0x05040100u);
        return r;
    }
    __device__ __forceinline__ bool any_not_finite() const {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int x = 0; x < kWords; ++x) bad |= not_finite<ELT>(w[j][x]);
        return bad;
    }
};

// A lane's weights as operands, four of each half.  In 16 bits they are rounded to the type, since its products take nothing wider, and f32 products are a seventh as fast: each weight is
// off by half a step at most, as the result's own rounding is, and the two together by 1.4 times that on average (64 samples on 8192 + 384 keys in bf16: 2.3e-3 of the result, rounded
// once 1.7e-3).  Their sum l is taken before, in f32.
template <int ELT>
struct Weights {
    u32x4 w;
    __device__ __forceinline__ void set(const f32x4 *s) {
        const f32x4 a = s[0];
        if constexpr (ELT == ATK_F32) {
            w = __builtin_bit_cast(u32x4, a);
        } else {
            const f32x4 b = s[1];
            w = u32x4{AttnElt<ELT>::pack(a[0], a[1]), AttnElt<ELT>::pack(a[2], a[3]), AttnElt<ELT>::pack(b[0], b[1]), AttnElt<ELT>::pack(b[2], b[3])};
        }
    }
};

template <int ELT, int DP>
__device__ __forceinline__ f32x4 mma_pv(const VRows<ELT, DP> &v, int i, const Weights<ELT> &p, f32x4 c) {
    if constexpr (ELT == ATK_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v.w[j][i]), __uint_as_float(p.w[j]), c, 0, 0, 0);
        return c;
    } else {
        return AttnElt<ELT>::mma(v.operand(i), p.w, c);
    }
}

// What becomes of a row: the log of the sum of exponentials from its maximum and sum, four elements of its result.
template <int ELT>
__device__ __forceinline__ float row_lse(const AttnDev &a, float m, float l) {
    if (l == 0.0f) return kNoMax;
    return m == kNoMax ? l : fmaf(m, a.scale, (log2f(l) - AttnElt<ELT>::kBias) * 0.6931471805599453f);
}
template <int ELT>
__device__ __forceinline__ void store_out(char *out, const f32x4 &o) {
    if constexpr (ELT == ATK_F32)
        *(f32x4 *)out = o;
    else
        *(u32x2 *)out = u32x2{AttnElt<ELT>::pack(o[0], o[1]), AttnElt<ELT>::pack(o[2], o[3])};
}

// Row r of the rows that read head h of a range: where its query lies, and how many keys it sees.
struct AttnRow {
    int b, t, head;
};
__device__ __forceinline__ AttnRow attn_row(const AttnDev &a, int h, int r, int own_b) {
    AttnRow x;
    const int g = r % a.group, bt = r / a.group;
    x.head = h * a.group + g;
    if (own_b >= 0) {
        x.b = own_b, x.t = bt;
    } else {
        x.b = bt / a.tokens, x.t = bt - x.b * a.tokens;
    }
    return x;
}
// keys of sequence b (0 for a row number or a length that is out of range)
__device__ __forceinline__ int seq_row(const AttnDev &a, int b, bool *bad) {
    const int s = a.seqs ? a.seqs[b] : b;
    if ((unsigned)s < (unsigned)a.rows) return s;
    *bad = true;
    return -1;
}
__device__ __forceinline__ int seq_len(const AttnDev &a, int row, bool *bad) {
    if (row < 0) return 0;
    const int len = a.lens[row];
    const int64_t most = (int64_t)a.row_pages * a.page.d;
    if (len >= 0 && len <= most) return len;
    *bad = true;
    return len < 0 ? 0 : (int)most;
}

// Rows r0 .. r0 + 16 * RT - 1 of the n_rows that read head h (own_b: those of that sequence; -1: of all) against keys ka .. kb - 1.  Keys below `shared` are looked up in
// the row `first` of the table.
template <int ELT, int DP, int RT, int NW, bool AROUND = false>
__device__ __forceinline__ void attn_range(const AttnDev &a, int h, int r0, int n_rows, int own_b, const int32_t *table_row, int ka, int kb, int part, char *lds,
                                           const int32_t *first = nullptr, int shared = 0) {
    typedef AttnElt<ELT> E;
    constexpr int kPiece = 16 / E::kBytes;            // elements of 16 bytes
    constexpr int NC = DP / (4 * kPiece);             // 16-byte pieces of a row that a lane has
    constexpr int NT = DP / 16;                       // products along d
    constexpr int NX = attn_halves(ELT), TK = 16 * NX;
    constexpr uint32_t kAll = (uint32_t)((1ull << TK) - 1);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = lane & 15, g = lane >> 4;

    u32x4 q[RT][NC];
    int lim[RT];
    int min_lim = kb;
    bool bad_len = false, bad_seq = false, bad_page = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + rt * 16 + n;
        const bool real = r < n_rows;
        const AttnRow x = attn_row(a, h, real ? r : 0, own_b);
        const int len = seq_len(a, seq_row(a, x.b, &bad_seq), &bad_len);
        // rows past the end are computed as if they saw all keys, and not written: they must not make tiles masked
        lim[rt] = real ? min(kb, len - (a.tokens - 1 - x.t)) : kb;
        min_lim = min(min_lim, lim[rt]);
        const char *p = (const char *)a.q + (x.b * a.qs[0] + x.t * a.qs[1] + x.head * a.qs[2]) * E::kBytes;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * 4 + g) * 16;
            q[rt][c] = at < a.dim * E::kBytes ? *(const u32x4 *)(p + at) : u32x4{0, 0, 0, 0};
        }
    }
    for (int w = 1; w < 16; w <<= 1) min_lim = min(min_lim, __shfl_xor(min_lim, w, 64));

    float m[RT], l[RT];  // maximum, in units of s: c * s need not be finite where s is
    bool far = false;    // ... and is not for some query of the wavefront
    f32x4 acc[RT][NT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = kNoMax, l[rt] = 0.0f;
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[rt][i] = f32x4{0, 0, 0, 0};
    }
    const char *kh = (const char *)a.k + h * a.ks[2] * E::kBytes, *vh = (const char *)a.v + h * a.vs[2] * E::kBytes;

    // lane j (and those TK apart) looks key k0 + j up, a tile ahead; keys past the end are read as the last one and masked
    auto page_of = [&](int k0) {
        const int key = min(k0 + (lane & (TK - 1)), kb - 1);
        return (key < shared ? first : table_row)[a.page.div(key)];
    };
    int page_next = ka < kb ? page_of(ka + wave * TK) : 0;
    for (int k0 = ka + wave * TK; k0 < kb; k0 += NW * TK) {
        int page = page_next;
        page_next = page_of(min(k0 + NW * TK, kb - 1));
        const bool good = (unsigned)page < (unsigned)a.n_pages;
        bad_page |= !good;
        if (!good) page = 0;
        const uint32_t valid = (uint32_t)__ballot(good) & kAll;

        u32x4 kf[NX][NC];
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const int key = min(k0 + x * 16 + n, kb - 1);
            const char *row = kh + (__shfl(page, x * 16 + n, 64) * a.ks[0] + a.page.mod(key) * a.ks[1]) * E::kBytes;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int at = (c * 4 + g) * 16;
                kf[x][c] = at < a.dim * E::kBytes ? fetch<AROUND, u32x4>(row + at) : u32x4{0, 0, 0, 0};
            }
        }
        VRows<ELT, DP> v;
#pragma unroll
        for (int j = 0; j < 4 * NX; ++j) {
            const int at = (j / 4) * 16 + g * 4 + j % 4;
            const int key = min(k0 + at, kb - 1);
            const char *row = vh + (__shfl(page, at, 64) * a.vs[0] + a.page.mod(key) * a.vs[1]) * E::kBytes;
            v.template load<AROUND>(j, row, n, a.dim);
        }
        f32x4 s[RT][NX];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                s[rt][x] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < NC; ++c) s[rt][x] = E::mma(kf[x][c], q[rt][c], s[rt][x]);
            }
        const bool masked = k0 + TK > min_lim || valid != kAll;
        bool apart = false;  // a value that is not finite beside a mask: 0 * it would not be 0
        if (masked) {
            asm volatile("");  // (a branch, no selections)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int x = 0; x < NX; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at = x * 16 + g * 4 + j;
                        if (k0 + at >= lim[rt] || !(valid >> at & 1)) s[rt][x][j] = kNoMax;
                    }
            apart = __any(v.any_not_finite());
        }
        float top[RT];
        bool raise = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float t = s[rt][0][0];
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) t = fmaxf(t, s[rt][x][j]);
            t = fmaxf(t, __shfl_xor(t, 16, 64));
            t = fmaxf(t, __shfl_xor(t, 32, 64));
            top[rt] = t;
            raise |= (t - m[rt]) * a.scale2 > kLazyMax;
        }
        if (__any(raise)) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float to = fmaxf(m[rt], top[rt]);
                const float f = __builtin_amdgcn_exp2f((m[rt] - to) * a.scale2);
                if (m[rt] != kNoMax) {  // (else nothing is kept yet)
                    l[rt] *= f;
#pragma unroll
                    for (int i = 0; i < NT; ++i) acc[rt][i] *= f;
                }
                m[rt] = to;
                far |= fabsf(to) < __builtin_inff() && !(fabsf(to * a.scale2) < __builtin_inff());
            }
            far = __any(far);
        }
        Weights<ELT> p[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float zero = m[rt] == kNoMax ? 0.0f : m[rt];
            const float ref = zero * a.scale2 - E::kBias;
            float sum = 0.0f;
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = __builtin_amdgcn_exp2f(far ? fmaf(s[rt][x][j] - zero, a.scale2, E::kBias) : fmaf(s[rt][x][j], a.scale2, -ref));
                    s[rt][x][j] = e;
                    sum += e;
                }
            l[rt] += sum;
            p[rt].set(s[rt]);
        }
        if (!apart) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) acc[rt][i] = mma_pv<ELT, DP>(v, i, p[rt], acc[rt][i]);
        } else {
            // query by query, with the values it does not see at 0; a product's columns are queries of their own
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                for (int c = 0; c < 16; ++c) {
                    const int limit = __shfl(lim[rt], c, 64);
                    VRows<ELT, DP> u = v;
#pragma unroll
                    for (int j = 0; j < 4 * NX; ++j) {
                        const int at = (j / 4) * 16 + g * 4 + j % 4;
                        if (k0 + at >= limit || !(valid >> at & 1))
#pragma unroll
                            for (int x = 0; x < VRows<ELT, DP>::kWords; ++x) u.w[j][x] = 0;
                    }
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const f32x4 t = mma_pv<ELT, DP>(u, i, p[rt], acc[rt][i]);
                        if (n == c) acc[rt][i] = t;
                    }
                }
        }
    }
    const int bad = (bad_page ? ATK_STATUS_BAD_PAGE : 0) | (bad_seq ? ATK_STATUS_BAD_SEQ : 0) | (bad_len ? ATK_STATUS_BAD_LEN : 0);
    if (bad && a.status) atomicOr(a.status, bad);

    // the wavefronts' ranges join in LDS, in their order
    float *ls_m = (float *)lds, *ls_l = ls_m + NW * RT * 16, *ls_o = ls_l + NW * RT * 16;
    constexpr int kPitch = DP + 4;
    float total[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16, 64);
        l[rt] += __shfl_xor(l[rt], 32, 64);
        if (g == 0) ls_m[(wave * RT + rt) * 16 + n] = m[rt], ls_l[(wave * RT + rt) * 16 + n] = l[rt];
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float to = kNoMax;
        for (int w = 0; w < NW; ++w) to = fmaxf(to, ls_m[(w * RT + rt) * 16 + n]);
        total[rt] = 0.0f;
        for (int w = 0; w < NW; ++w) {
            const float mw = ls_m[(w * RT + rt) * 16 + n];
            total[rt] += ls_l[(w * RT + rt) * 16 + n] * (mw == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((mw - to) * a.scale2));
        }
        if (m[rt] != kNoMax) {
            const float f = __builtin_amdgcn_exp2f((m[rt] - to) * a.scale2);
#pragma unroll
            for (int i = 0; i < NT; ++i) acc[rt][i] *= f;
        }
        m[rt] = to;
    }
    for (int w = 0; w < NW; ++w) {
        if (wave == w) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float *o = ls_o + (rt * 16 + n) * kPitch + (g * 4 + j) * NT + i;
                        if (w > 0) acc[rt][i][j] += *o;
                        if (w < NW - 1) *o = acc[rt][i][j];
                    }
        }
        __syncthreads();
    }
    if (wave != NW - 1) return;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + rt * 16 + n;
        if (r >= n_rows) continue;
        const AttnRow x = attn_row(a, h, r, own_b);
        const int64_t row = ((int64_t)x.b * a.tokens + x.t) * a.heads + x.head;
        if (a.direct) {  // nothing to join
            if (g == 0 && a.lse) a.lse[row] = row_lse<ELT>(a, m[rt], total[rt]);
            const float f = 1.0f / total[rt];
            const bool none = total[rt] == 0.0f;  // no key, or scores of -inf alone, whose values do not count even if they are NaN
            char *out = (char *)a.out + (x.b * a.os[0] + x.t * a.os[1] + x.head * a.os[2]) * E::kBytes;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < NT; i += 4) {
                    const int d = (g * 4 + j) * NT + i;
                    f32x4 o = f32x4{acc[rt][i][j] * f, acc[rt][i + 1][j] * f, acc[rt][i + 2][j] * f, acc[rt][i + 3][j] * f};
                    if (none) o = f32x4{0, 0, 0, 0};
                    if (d < a.dim) store_out<ELT>(out + d * E::kBytes, o);
                }
            continue;
        }
        if (g == 0) a.parts_ml[row * a.parts + part] = float2{m[rt], total[rt]};
        float *o = a.parts_o + (row * a.parts + part) * a.dim;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < NT; i += 4) {
                const int d = (g * 4 + j) * NT + i;
                if (d < a.dim) *(f32x4 *)(o + d) = f32x4{acc[rt][i][j], acc[rt][i + 1][j], acc[rt][i + 2][j], acc[rt][i + 3][j]};
            }
    }
}


// ------------------------------------------------------------------------------------ many rows on shared keys, 16-bit types
//
// With more rows than a tile or two the shared keys are bound by the matrix units and the exponentials, so a key's data should come to a wavefront once for
// 32 rows and to a CU once for all of its rows: a workgroup's NW wavefronts have 32 rows each, and 64 keys at a time pass through LDS.
//   S^T = K Q^T and O^T = V^T P^T by 32x32x16 matrix instructions, half the operands' reads of 16x16x32 for a product.  A lane has one query (lane % 32) and of
//   each 32 keys those with 8 * i + 4 * (lane / 32) + 0..3; step x of the second product takes i = 2 x and 2 x + 1.
//   A tile is a phase of products (those of the tile before with V, this one's with K) and one of vector instructions (maximum, exponentials, packing, the next
//   tiles' loads), and with eight wavefronts each SIMD has two of them, one of each half: the second half is a phase late, so that one of the two has the matrix
//   units while the other one has the vector unit.  128 samples of 32 heads on 65536 keys: 139 us by itself (0.99 PFLOP/s where a
//   large matrix product reaches 1.1), 148 to 151 right after other launches; the matrix units are busy for
//   55 % of the cycles, and the clock is down to 1.7 GHz, as it is under matrix products of such data alone.  With one meeting of the wavefronts a tile in place of two: 160 us.
//   K and V come from memory into LDS without passing through registers, row by row, 1 KB an instruction, a tile ahead.  (By way of registers, with V transposed there, the loads' and
//   stores' instructions were half of the vector phase: 128 samples' 65536 keys took 184 us, and take 139.)  V is transposed on the way out, by
//   the transposing reads: 16 lanes get 16 d's of four keys.
//   Rows lie in LDS without gaps, so a row's 16-byte pieces are permuted (piece ^ a few bits of the key) for lanes a row apart to meet in different banks; the lane that brings a
//   piece in takes its place's piece from memory.
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int ELT>
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (ELT == ATK_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 16 bytes of each lane from base + off to LDS at `lds` + 16 * lane.  (Nothing but vmcnt waits for it, and no wait that the compiler inserts, which by the builtin are for all of them
// in front of every read from LDS.  m0 holds the place; as an operand it is the compiler's, which keeps track of it.)
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(const char *address, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(lds), "v"(address) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {  // until all but the last N are there
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

constexpr int kBlockKeys = 64;
template <int DP, int NW>
struct BlockLds {
    static constexpr int kRow = DP * 2;                    // bytes of a key's row
    static constexpr int kTile = kBlockKeys * kRow;
    static constexpr int kBuffers = NW == 8 ? 3 : 2;       // of K and of V: wavefronts a phase apart hold one longer
    static constexpr int kRing = 64;                       // tiles whose addresses are at hand
    static constexpr int kData = 2 * kBuffers * kTile;
    static constexpr int kBytes = kData + 2 * kRing * 16 * 4;
};

// Rows r0 .. r0 + 32 * NW - 1 of head h against keys ka .. kb - 1 (one at least), all of which every one of these rows has to see: nothing is written if one does not, or if a
// key's page is none (attn_rest then does the rows, with masks).
// FULL: dim == DP.
template <int ELT, int DP, int NW, bool FULL>
__device__ __forceinline__ void attn_block(const AttnDev &a, int h, int r0, int n_rows, const int32_t *table_row, int ka, int kb, int part, char *lds) {
    typedef AttnElt<ELT> E;
    typedef BlockLds<DP, NW> L;
    constexpr int NS = DP / 16;                            // steps of the first product
    constexpr int ND = DP / 32;                            // tiles of d
    constexpr int kPieces = DP / 8;                        // 16-byte pieces of a row
    constexpr int kLoads = L::kTile / 1024 / NW;           // of K, and of V, of a wavefront and tile
    constexpr int kLoadKeys = 64 / kPieces;                // keys of one
    constexpr bool kHalves = kLoadKeys == 8;               // two times four keys
    static_assert(kLoads >= 1 && (DP == 64 || DP == 128 || DP == 256), "every wavefront has its share");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;
    const char *kh = (const char *)a.k + h * a.ks[2] * 2, *vh = (const char *)a.v + h * a.vs[2] * 2;
    const int tiles = (kb - ka + kBlockKeys - 1) / kBlockKeys;

    // the query of a lane
    const int r = r0 + wave * 32 + n;
    const bool real = r < n_rows;
    const AttnRow x = attn_row(a, h, real ? r : 0, -1);
    bool bad = false;  // (told by attn_rest)
    const int sees = seq_len(a, seq_row(a, x.b, &bad), &bad) - (a.tokens - 1 - x.t);

    // What comes in.  Four keys that begin at a multiple of four lie in one page (page_size % 4 == 0, and so ka): a load has the address of its four keys, a scalar that a
    // wavefront finds in LDS, and offsets that stay the same.  Addresses are looked up by all threads together, for 64 tiles and then 32 at a time, in units of 16 bytes.  (Looked up
    // by every wavefront for each tile, with 64-bit products, they took as long as the tile's exponentials: 128 samples' 65536 keys 152 us.)
    // Load c of a wavefront brings keys first_key(c) + lane / kPieces, place lane % kPieces of the row.
    auto first_key = [&](int c) { return (c * NW + wave) * kLoadKeys; };
    const int in_load = lane / kPieces, place = lane % kPieces;
    auto k_swizzle = [](int key) { return DP == 64 ? key & 7 : key & 15; };
    auto v_swizzle = [](int key) { return DP == 64 ? (key & 2) << 1 : (key & 3) << 2; };  // (half a wavefront reads 64 bytes of four keys at once)
    // (the same for all c but for K's with 256: loads are eight keys apart there)
    const int k_piece = place ^ k_swizzle(first_key(0) + in_load), v_piece = place ^ v_swizzle(first_key(0) + in_load);
    const uint32_t in_group = kHalves ? in_load & 3 : in_load;  // key of the four (from first_key(c) & 3 on)
    const uint32_t k_step = (uint32_t)a.ks[1] * 2, v_step = (uint32_t)a.vs[1] * 2;
    bool bad_page = false;
    uint32_t *const k_ring = (uint32_t *)(lds + L::kData), *const v_ring = k_ring + L::kRing * 16;
    // tiles past the last are that one once more (brought in and not used: no branches), keys past the end the last four
    auto look_up = [&](int t0, int count) {
        for (int i = threadIdx.x; i < count * 16; i += NW * 64) {
            const int t = t0 + i / 16, key = min(ka + min(t, tiles - 1) * kBlockKeys + i % 16 * 4, (kb - 1) & ~3);
            int page = table_row[a.page.div(key)];
            if ((unsigned)page >= (unsigned)a.n_pages) bad_page = true, page = 0;
            const int64_t slot = a.page.mod(key);
            const int at = t % L::kRing * 16 + i % 16;
            k_ring[at] = (uint32_t)((page * a.ks[0] + slot * a.ks[1]) >> 3);
            v_ring[at] = (uint32_t)((page * a.vs[0] + slot * a.vs[1]) >> 3);
        }
    };
    const uint32_t k_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds, v_lds = k_lds + L::kBuffers * L::kTile;
    struct Bases {
        uint32_t at[kLoads * (kHalves ? 2 : 1)];  // of the four keys of each load, 16 bytes
    };
    auto bases_of = [&](const uint32_t *ring, int t) {
        Bases y;
        ring += t % L::kRing * 16;
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
            if constexpr (kHalves) {
                y.at[2 * c] = ring[first_key(c) / 4], y.at[2 * c + 1] = ring[first_key(c) / 4 + 1];
            } else {
                y.at[c] = ring[first_key(c) / 4];
            }
        }
        return y;
    };
    auto load = [&](const char *head, const Bases &y, uint32_t step, int piece, bool k, uint32_t to) {
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
            const int first = first_key(c);
            const int p = DP == 256 && k ? piece ^ (first & 8) ^ (first_key(0) & 8) : piece;
            const uint32_t off = in_group * step + p * 16;
            const uint32_t at = to + (uint32_t)(c * NW + wave) * 1024;
            if (FULL || p * 8 < a.dim) {
                if constexpr (kHalves) {
                    load_to_lds(head + ((uint64_t)(lane < 32 ? y.at[2 * c] : y.at[2 * c + 1]) << 4) + off, at);
                } else {
                    const uint32_t base = __builtin_amdgcn_readfirstlane(y.at[c]);
                    load_to_lds(head + ((uint64_t)base << 4), DP == 256 ? off + (first & 3) * step : off, at);
                }
            }
        }
    };
    auto buffer = [&](int t) { return (uint32_t)(t % L::kBuffers) * L::kTile; };
    auto load_k = [&](int t, const Bases &y) { load(kh, y, k_step, k_piece, true, k_lds + buffer(t)); };
    auto load_v = [&](int t, const Bases &y) { load(vh, y, v_step, v_piece, false, v_lds + buffer(t)); };

    // The phases bring in K two tiles ahead and V one; the second half of the wavefronts, a phase late, one more.
    const int late = NW == 8 ? wave >> 2 : 0;
    look_up(0, min(L::kRing, tiles + 4));
    if constexpr (!FULL) {  // pieces past dim stay 0
        for (int i = threadIdx.x; i < L::kData / 16; i += NW * 64) ((u32x4 *)lds)[i] = u32x4{0, 0, 0, 0};
    }
    if (!__syncthreads_and(!real || sees >= kb)) return;
    load_k(0, bases_of(k_ring, 0));
    load_k(1, bases_of(k_ring, 1));
    load_v(0, bases_of(v_ring, 0));
    // What lies behind the last key has weight 0, which NaN in V would not heed: a wavefront clears it in what it has brought in, before the first products that read it.
    auto clear_tail = [&]() {
        const int left = kb - ka - (tiles - 1) * kBlockKeys;
        if (left == kBlockKeys) return;
#pragma unroll
        for (int c = 0; c < kLoads; ++c)
            if (first_key(c) + in_load >= left)
                *(__attribute__((address_space(3))) u32x4 *)(uintptr_t)(v_lds + buffer(tiles - 1) + (c * NW + wave) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    };
    if (late) {
        load_k(2, bases_of(k_ring, 2));
        load_v(1, bases_of(v_ring, 1));
    }
    u32x4 q[NS];
    {
        const char *p = (const char *)a.q + (x.b * a.qs[0] + x.t * a.qs[1] + x.head * a.qs[2]) * 2;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int at = (s * 2 + g) * 16;
            q[s] = FULL || at < a.dim * 2 ? *(const u32x4 *)(p + at) : u32x4{0, 0, 0, 0};
        }
    }
    wait_loads<0>();
    if (tiles == 1) clear_tail();
    __syncthreads();

    float m = kNoMax, l = 0.0f;
    bool far = false;
    f32x16 acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;
    f32x16 s[2];
    u32x4 p[2][2];
    auto barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    // Products of tile t with V and of tile t + 1 with K (either may be left out).  Reads from LDS run kAhead in front: one takes four products' time.
    const int q16 = lane >> 4, i16 = lane & 15, v_key = 4 * (q16 >> 1) + i16 / 4;
    const uint32_t k_at = n * L::kRow + ((g ^ k_swizzle(n)) << 4);
    const uint32_t v_at = v_key * L::kRow + ((((q16 & 1) * 2 + (i16 & 3) / 2) ^ v_swizzle(v_key)) << 4) + (i16 & 1) * 8;
    typedef const __attribute__((address_space(3))) u32x4 *Lds16;
    typedef __attribute__((address_space(3))) s16x4 *Lds8;
    auto products = [&](auto second, auto first, int t) {
        constexpr bool kSecond = decltype(second)::value, kFirst = decltype(first)::value;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        if constexpr (kSecond) {
            const uint32_t v = v_lds + buffer(t) + v_at;
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        const uint32_t at = (v ^ (i << 6)) + (y * 2 + z) * 16 * L::kRow;
                        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds8)(uintptr_t)at);
                        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds8)(uintptr_t)(at + 8 * L::kRow));
                        const u32x2 lw = __builtin_bit_cast(u32x2, lo), hw = __builtin_bit_cast(u32x2, hi);
                        acc[i] = mma32<ELT>(u32x4{lw[0], lw[1], hw[0], hw[1]}, p[y][z], acc[i]);
                    }
        }
        if constexpr (kFirst) {
            const uint32_t k = k_lds + buffer(t + 1) + k_at;
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[y][j] = 0.0f;
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int y = 0; y < 2; ++y) s[y] = mma32<ELT>(*(Lds16)(uintptr_t)((k ^ (i << 5)) + y * 32 * L::kRow), q[i], s[y]);
        }
        // (of the second product, two reads each)
        constexpr int kReads = (kSecond ? 8 * ND : 0) + (kFirst ? 2 * NS : 0), kAhead = 8;
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);  // reads from LDS
        int reads = kAhead;
        if constexpr (kSecond) {
#pragma unroll
            for (int i = 0; i < 4 * ND; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);  // a product
                if (reads < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                reads += 2;
            }
        }
        if constexpr (kFirst) {
#pragma unroll
            for (int i = 0; i < 2 * NS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                if (reads < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                reads += 1;
            }
        }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    };
    typedef std::true_type Yes;
    typedef std::false_type No;
    auto softmax = [&](int t) {
        const int left = kb - ka - t * kBlockKeys;  // keys of the tile
        if (left < kBlockKeys) {
            asm volatile("");  // (a branch: as selections these instructions are every tile's)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (y * 32 + 8 * (j >> 2) + 4 * g + (j & 3) >= left) s[y][j] = kNoMax;
        }
        float top = s[0][0];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[y][j]);
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
        if (__any((top - m) * a.scale2 > kLazyMax)) {
            const float to = fmaxf(m, top);
            const float f = __builtin_amdgcn_exp2f((m - to) * a.scale2);
            if (m != kNoMax) {
                l *= f;
#pragma unroll
                for (int i = 0; i < ND; ++i) acc[i] *= f;
            }
            m = to;
            far = __any(fabsf(to) < __builtin_inff() && !(fabsf(to * a.scale2) < __builtin_inff()));
        }
        const float zero = m == kNoMax ? 0.0f : m;
        const float ref = zero * a.scale2 - E::kBias;
        if (far) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[y][j] = fmaf(s[y][j] - zero, a.scale2, E::kBias);
        } else {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[y][j] = fmaf(s[y][j], a.scale2, -ref);
        }
        float sum = 0.0f;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                s[y][j] = __builtin_amdgcn_exp2f(s[y][j]);
                sum += s[y][j];
            }
#pragma unroll
            for (int z = 0; z < 2; ++z)
                p[y][z] = u32x4{E::pack(s[y][8 * z], s[y][8 * z + 1]), E::pack(s[y][8 * z + 2], s[y][8 * z + 3]), E::pack(s[y][8 * z + 4], s[y][8 * z + 5]),
                                E::pack(s[y][8 * z + 6], s[y][8 * z + 7])};
        }
        l += sum;
    };
    if (late) barrier();
    products(No{}, Yes{}, -1);
    barrier();
    for (int t = 0; t < tiles - 1; ++t) {
        if (tiles > L::kRing && t > 0 && t % (L::kRing / 2) == 0) look_up(t + L::kRing / 2, L::kRing / 2);  // over the addresses of tiles that are there
        const Bases next_k = bases_of(k_ring, t + 2 + late), next_v = bases_of(v_ring, t + 1 + late);
        load_k(t + 2 + late, next_k);
        load_v(t + 1 + late, next_v);
        softmax(t);
        wait_loads<2 * kLoads>();
        if (late && t == tiles - 2) clear_tail();  // (the first half of the wavefronts comes to the last tile's V a phase sooner)
        barrier();
        products(Yes{}, Yes{}, t);
        barrier();
    }
    softmax(tiles - 1);
    wait_loads<0>();
    if (!late && tiles > 1) clear_tail();
    barrier();
    products(Yes{}, No{}, tiles - 1);
    if (!late && NW == 8) barrier();
    if (__syncthreads_or(bad_page)) return;
    l += __shfl_xor(l, 32, 64);
    if (!real) return;
    const int64_t row = ((int64_t)x.b * a.tokens + x.t) * a.heads + x.head;
    if (g == 0) a.parts_ml[row * a.parts + part] = float2{m, l};
    float *o = a.parts_o + (row * a.parts + part) * a.dim;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = i * 32 + j * 8 + g * 4;
            if (FULL || d < a.dim) *(f32x4 *)(o + d) = f32x4{acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2], acc[i][4 * j + 3]};
        }
}

// Workgroup `id` of 8 * ceil(n / 8) in the order of units 0 .. n - 1 that gives each XCD (id % 8) units in a row; -1: none.  Units with the same keys, and the heads of the
// same tokens, are neighbours, and so meet in one L2 (against an XCD for each head: level, and no less so with a number of heads that is not a multiple of eight).
__device__ __forceinline__ int xcd_unit(int id, int n) {
    const int per = (n + 7) / 8, u = (id & 7) * per + (id >> 3);
    return (id >> 3) < per && u < n ? u : -1;
}

// Own keys of a sequence, or (own_from 0) all of them: workgroup y of those.
template <int ELT, int DP, int NW, bool AROUND>
__device__ __forceinline__ void attn_own(const AttnDev &a, int y, char *lds) {
    bool bad = false;  // (told by attn_range)
    y = xcd_unit(y, a.n_own);
    if (y < 0) return;
    const int block = y % a.own_blocks;
    int x = y / a.own_blocks;
    const int h = x % a.kv_heads;
    x /= a.kv_heads;
    const int split = x % a.own_splits, b = x / a.own_splits;
    const int row = seq_row(a, b, &bad), len = seq_len(a, row, &bad);
    int from0 = a.own_from;
    const int32_t *first = a.table;
    if (from0 < a.prefix_len) {
        const int s = seq_row(a, 0, &bad);
        first += s * a.table_stride;
        if (s < 0) from0 = a.prefix_len;
    }
    const int keys = max(0, len - from0);
    constexpr int kStep = NW * kTileKeys;
    const int per = (int)(((int64_t)keys + a.own_splits * kStep - 1) / (a.own_splits * kStep)) * kStep;
    const int64_t from = from0 + (int64_t)split * per;
    const int ka = (int)min((int64_t)len, from), kb = (int)min((int64_t)len, from + per);
    attn_range<ELT, DP, 1, NW, AROUND>(a, h, block * 16, a.tokens * a.group, b, a.table + row * a.table_stride, ka, max(ka, kb), a.prefix_splits + split, lds, first, a.prefix_len);
}

template <int DP, int RT, int NW>
constexpr int attn_lds_bytes() { return 2 * NW * RT * 16 * 4 + RT * 16 * (DP + 4) * 4; }

// A unit of the shared keys: head, rows and keys.
struct SharedUnit {
    int h, block, split, row, ka, kb;
    __device__ __forceinline__ SharedUnit(const AttnDev &a, int u) {
        bool bad = false;  // (told by attn_range)
        block = u % a.prefix_blocks, h = u / a.prefix_blocks % a.kv_heads, split = u / (a.prefix_blocks * a.kv_heads);
        row = seq_row(a, 0, &bad);
        ka = split * a.prefix_keys, kb = row < 0 ? ka : min(a.prefix_len, ka + a.prefix_keys);
    }
};

// Of attn_block_kernel's units (the first masked_grid workgroups), those with a row that sees only a part of the keys - a sequence that ends before them, a page that is none: tile by
// tile, with masks, 16 rows after the other, and each time K and V again.  That is the way of few rows, and slow for many: one sequence of length 0 among 64 on 8192 + 384 keys makes 176 us of
// 49, 32 of them 209; among 128 on 65536 + 1125 keys 1500 of 270.  Then own keys.
template <int ELT, int DP, bool AROUND>
__device__ __forceinline__ void attn_rest(const AttnDev &a, int id, char *lds) {
    if (id >= a.masked_grid) {
        attn_own<ELT, DP, kAttnWaves, AROUND>(a, id - a.masked_grid, lds);
        return;
    }
    const int u = xcd_unit(id, a.n_prefix), n_rows = a.batch * a.tokens * a.group;
    if (u < 0) return;
    const SharedUnit s(a, u);
    const int r0 = s.block * a.block_rows;
    bool all = s.ka < s.kb, bad_len = false;
    for (int r = r0 + threadIdx.x; r < min(n_rows, r0 + a.block_rows); r += kAttnWaves * 64) {
        const AttnRow x = attn_row(a, s.h, r, -1);
        bool bad_seq = false;  // (sees nothing: attn_range tells)
        if (seq_len(a, seq_row(a, x.b, &bad_seq), &bad_len) - (a.tokens - 1 - x.t) < s.kb) all = false;
    }
    if (bad_len && a.status) atomicOr(a.status, ATK_STATUS_BAD_LEN);
    const int32_t *table_row = a.table + s.row * a.table_stride;
    if (s.ka < s.kb)
        for (int j = a.page.div(s.ka) + threadIdx.x, to = a.page.div(s.kb - 1); j <= to; j += kAttnWaves * 64)
            if ((unsigned)table_row[j] >= (unsigned)a.n_pages) all = false;
    if (__syncthreads_and(all)) return;
    for (int r = r0; r < min(n_rows, r0 + a.block_rows); r += 16) {
        attn_range<ELT, DP, 1, kAttnWaves>(a, s.h, r, n_rows, -1, table_row, s.ka, s.kb, s.split, lds);
        __syncthreads();
    }
}

// Few rows on the shared keys: the wavefronts of a workgroup share its keys out.  And the rest.
template <int ELT, int DP, int RT, bool AROUND>
__global__ __launch_bounds__(kAttnWaves * 64, RT == 1 && DP <= 128 ? 2 : 1) void attn_range_kernel(const AttnDev a) {
    __shared__ __align__(16) char lds[attn_lds_bytes<DP, RT, kAttnWaves>()];
    int id = blockIdx.x;
    if (id < a.prefix_grid) {
        const int u = xcd_unit(id, a.n_prefix);
        if (u < 0) return;
        const SharedUnit s(a, u);
        attn_range<ELT, DP, RT, kAttnWaves>(a, s.h, s.block * RT * 16, a.batch * a.tokens * a.group, -1, a.table + s.row * a.table_stride, s.ka, s.kb, s.split, lds);
        return;
    }
    id -= a.prefix_grid;
    if constexpr (RT == 1)
        attn_rest<ELT, DP, AROUND>(a, id, lds);
    else
        attn_own<ELT, DP, kAttnWaves, AROUND>(a, id, lds);
}

// Many: its wavefronts share its rows out.
template <int ELT, int DP, int NW, bool FULL>
__device__ __forceinline__ void attn_block_unit(const AttnDev &a, int id, char *lds) {
    const int u = xcd_unit(id, a.n_prefix);
    if (u < 0) return;
    const SharedUnit s(a, u);
    if (s.ka < s.kb) attn_block<ELT, DP, NW, FULL>(a, s.h, s.block * NW * 32, a.batch * a.tokens * a.group, a.table + s.row * a.table_stride, s.ka, s.kb, s.split, lds);
}
template <int ELT, int DP, int NW, bool FULL>
__global__ __launch_bounds__(NW * 64, DP <= 128 ? 2 : 1) void attn_block_kernel(const AttnDev a) {
    __shared__ __align__(1024) char lds[BlockLds<DP, NW>::kBytes];
    attn_block_unit<ELT, DP, NW, FULL>(a, blockIdx.x, lds);
}

// Many rows and the rest in one launch: a workgroup of each to a CU (plan_blocks), so that the matrix units and memory work side by side.  The workgroups come in the order of their
// numbers, so all of the first kind are there when the others begin; in turns, 64 samples on 8192 + 384 keys took 58 us and not 50.
template <int ELT, int DP, bool FULL, bool AROUND>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void attn_mixed_kernel(const AttnDev a) {
    static_assert(BlockLds<DP, kAttnWaves>::kBytes >= attn_lds_bytes<DP, 1, kAttnWaves>(), "LDS of either kind");
    __shared__ __align__(1024) char lds[BlockLds<DP, kAttnWaves>::kBytes];
    const int id = blockIdx.x;
    if (id < a.prefix_grid)
        attn_block_unit<ELT, DP, kAttnWaves, FULL>(a, id, lds);
    else
        attn_rest<ELT, DP, AROUND>(a, id - a.prefix_grid, lds);
}

// rt: 16-row tiles of a workgroup of attn_range_kernel; 0: attn_block_kernel on the shared keys, waves of 32 rows, and own keys in a launch of their own; kMixed: both in one
hipError_t launch_attn_bf16(const AttnDev &a, int dp, int rt, int waves, hipStream_t stream);
hipError_t launch_attn_f16(const AttnDev &a, int dp, int rt, int waves, hipStream_t stream);
hipError_t launch_attn_f32(const AttnDev &a, int dp, int rt, int waves, hipStream_t stream);

constexpr int kMixed = -1;
// 16-row tiles of a workgroup's rows that attn_range_kernel is built for: registers hold Q, K, V and O of RT tiles, up to 512 words of a lane
constexpr int attn_max_rt(int elt, int dp) { return dp > 128 ? 1 : 2; }
// wavefronts of a workgroup of attn_block_kernel: eight at 256 words of a lane, or four at up to 512
constexpr int attn_max_waves(int dp) { return dp > 128 ? 4 : 8; }

template <int ELT, int DP>
hipError_t launch_attn_dp(AttnDev a, int rt, int waves, hipStream_t stream) {
    if constexpr (ELT != ATK_F32 && attn_max_waves(DP) >= 8) {
        if (rt == kMixed) {
            const dim3 g((uint32_t)(2 * a.prefix_grid + (a.n_own + 7) / 8 * 8)), threads(kAttnWaves * 64);
            a.masked_grid = a.prefix_grid;
            if (a.dim < DP)  // (rare: without the instance past the caches)
                hipLaunchKernelGGL((attn_mixed_kernel<ELT, DP, false, false>), g, threads, 0, stream, a);
            else if (a.around)
                hipLaunchKernelGGL((attn_mixed_kernel<ELT, DP, true, true>), g, threads, 0, stream, a);
            else
                hipLaunchKernelGGL((attn_mixed_kernel<ELT, DP, true, false>), g, threads, 0, stream, a);
            return hipGetLastError();
        }
    }
    if constexpr (ELT != ATK_F32) {
        if (rt == 0) {
            const dim3 g((uint32_t)a.prefix_grid);
            const bool full = a.dim == DP;
            if (waves == 8 && attn_max_waves(DP) >= 8) {
                if constexpr (attn_max_waves(DP) >= 8) {
                    if (full)
                        hipLaunchKernelGGL((attn_block_kernel<ELT, DP, 8, true>), g, dim3(512), 0, stream, a);
                    else
                        hipLaunchKernelGGL((attn_block_kernel<ELT, DP, 8, false>), g, dim3(512), 0, stream, a);
                }
            } else if (full) {
                hipLaunchKernelGGL((attn_block_kernel<ELT, DP, 4, true>), g, dim3(256), 0, stream, a);
            } else {
                hipLaunchKernelGGL((attn_block_kernel<ELT, DP, 4, false>), g, dim3(256), 0, stream, a);
            }
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            a.masked_grid = a.prefix_grid, a.prefix_grid = 0;
        }
    }
    const dim3 g((uint32_t)(a.prefix_grid + a.masked_grid + (a.n_own + 7) / 8 * 8)), threads(kAttnWaves * 64);
    if constexpr (attn_max_rt(ELT, DP) >= 2) {
        if (rt == 2) {
            hipLaunchKernelGGL((attn_range_kernel<ELT, DP, 2, false>), g, threads, 0, stream, a);
            return hipGetLastError();
        }
    }
    if (a.around)
        hipLaunchKernelGGL((attn_range_kernel<ELT, DP, 1, true>), g, threads, 0, stream, a);
    else
        hipLaunchKernelGGL((attn_range_kernel<ELT, DP, 1, false>), g, threads, 0, stream, a);
    return hipGetLastError();
}
template <int ELT>
hipError_t launch_attn(const AttnDev &a, int dp, int rt, int waves, hipStream_t stream) {
    if (dp == 64) return launch_attn_dp<ELT, 64>(a, rt, waves, stream);
    if (dp == 128) return launch_attn_dp<ELT, 128>(a, rt, waves, stream);
    return launch_attn_dp<ELT, 256>(a, rt, waves, stream);
}

}  // namespace atk
