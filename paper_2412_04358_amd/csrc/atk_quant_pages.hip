// append_quantized and read_quantized: tokens go into pools of few bits, and come back (include/atk_quant.h).
//
// Bound by memory: an element is read and written once, four lanes have a block of 32 (eight elements each, 16 bytes of a 16-bit type) and find its largest magnitude by two exchanges.
// append is atk_pages.hip's append with the conversion on the way, and a sequence's tokens cut into pieces, so that one long prompt fills the chip.
// Two prompts of 4000 tokens into 24 pools, 497 MB: 101 to 107 us, and read back, as much again, 76 to 81; eight sequences of 8192 tokens out of two pools, 407 MB: 77 us (5.3 TB/s); four tokens into
// two pools: 7 us, the chain of numbers, pages, values, and the tables behind them.  f32, whose lanes have 32 bytes in two pieces, goes at half the rate: 4000 tokens into 12 pools and back 291 us, eight
// sequences out of two 240.
#include "atk_mx.h"
#include "atk_pages_kernel.h"

namespace atk {

constexpr int kPieceUnits = 2048;  // units (of eight elements) of a workgroup's piece, about: 32 KB of a 16-bit type (with 8192, two prompts of 4000 tokens into 24 pools and back 245 us, 234)

struct QuantShape {
    FastDiv token;         // units of a token
    uint32_t code_bytes;   // of a token
    int64_t token_bytes;
    int piece, pieces;     // tokens of a piece, pieces of a sequence
};
struct QuantValues {
    const char *p[kPools];
    int64_t seq[kPools], token[kPools];  // bytes from one sequence's, one token's to the next one's
};

// Eight values, past the caches: they are read once (the same two prompts 234 us -> 224).
template <int ELT>
struct Eight;
template <>
struct Eight<ATK_F32> {
    mx_u32x4 a, b;
    __device__ __forceinline__ void load(const char *p) { a = __builtin_nontemporal_load((const mx_u32x4 *)p), b = __builtin_nontemporal_load((const mx_u32x4 *)p + 1); }
    __device__ __forceinline__ void get(float *x) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(a[i]), x[i + 4] = __uint_as_float(b[i]);
    }
};
template <>
struct Eight<ATK_BF16> {
    mx_u32x4 a;
    __device__ __forceinline__ void load(const char *p) { a = __builtin_nontemporal_load((const mx_u32x4 *)p); }
    __device__ __forceinline__ void get(float *x) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(a[i] << 16), x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
};
template <>
struct Eight<ATK_F16> {
    mx_u32x4 a;
    __device__ __forceinline__ void load(const char *p) { a = __builtin_nontemporal_load((const mx_u32x4 *)p); }
    __device__ __forceinline__ void get(float *x) const {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = a[i];  // (bit_cast of a vector's element takes element 0)
            const f16x2 h = __builtin_bit_cast(f16x2, w);
            x[2 * i] = (float)h[0], x[2 * i + 1] = (float)h[1];
        }
    }
};
constexpr int eight_bytes(int elt) { return elt == ATK_F32 ? 32 : 16; }

// Largest over the four lanes of a block.
__device__ __forceinline__ uint32_t most_of_four(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));
}

// to[x]: byte of token x in a pool, -1 for none.  `units` units of the tokens from `from`, which lie `stride` bytes apart.
template <int ELT, int BITS>
__device__ __forceinline__ void quantise_tokens(char *pool, const char *from, int64_t stride, const int64_t *to, int units, const QuantShape &q) {
    constexpr int kAtOnce = ELT == ATK_F32 ? 2 : 4;
    for (int u0 = threadIdx.x; u0 < units; u0 += kAtOnce * kThreads) {  // (units are a multiple of four: a block's lanes stay together)
        Eight<ELT> v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int u = min(u0 + j * kThreads, units - 1), x = q.token.div(u);
            v[j].load(from + x * stride + (int64_t)(u - x * (int)q.token.d) * eight_bytes(ELT));
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int u = u0 + j * kThreads, x = q.token.div(min(u, units - 1)), r = u - x * (int)q.token.d;
            float y[8];
            v[j].get(y);
            uint32_t amax = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(y[i]) & 0x7fffffffu);
            const uint32_t byte = mx_exponent<BITS>(most_of_four(amax));
            uint32_t w[Mx<BITS>::kWords];
            mx_encode<BITS>(y, byte, w);
            const int64_t at = to[x];
            if (u < units && at >= 0) {
                char *row = pool + at;
                if constexpr (BITS == 4)
                    *(uint32_t *)(row + r * 4) = w[0];
                else
                    *(mx_u32x2 *)(row + r * 8) = mx_u32x2{w[0], w[1]};
                if ((r & 3) == 0) row[q.code_bytes + r / 4] = (char)byte;
            }
        }
    }
}

template <int ELT, int BITS>
__global__ __launch_bounds__(kThreads) void quant_append_kernel(const PagesDev t, const Pools pools, const QuantValues values, int n_pools, const QuantShape q, const int32_t *seqs, int64_t n,
                                                                int64_t tokens, int shares, bool tables) {
    __shared__ int64_t to[kThreads];
    const int64_t i = blockIdx.x / shares;
    const int share = (int)(blockIdx.x % shares);
    int total = 0, before = 0, bad = 0;
    const int n_free = *t.n_free;
    for (int64_t j = threadIdx.x; j < n; j += kThreads) {
        const AppendSeq s = append_seq(t, seqs, j, tokens);
        bad |= s.bad;
        total += s.takes();
        if (j < i) before += s.takes();
    }
    meet_threads(&total, &before, &bad);
    if (total > n_free) bad |= ATK_STATUS_NO_PAGES;
    if (!bad) {
        const AppendSeq s = append_seq(t, seqs, i, tokens);
        const int top = n_free - 1 - before;
        const int64_t page_bytes = (int64_t)t.page.d * q.token_bytes;
        const int fresh = s.copy ? t.free_at(top) : -1;
        for (int64_t item = share; item < (int64_t)n_pools * q.pieces; item += shares) {
            const int p = (int)(item / q.pieces), x0 = (int)(item % q.pieces) * q.piece, count = (int)min((int64_t)q.piece, tokens - x0);
            if (x0 == 0 && s.copy && t.is_page(fresh))  // the old page's tokens
                copy_bytes<16>(pools.p[p] + fresh * page_bytes, pools.p[p] + s.old * page_bytes, t.page.mod(s.len) * q.token_bytes);
            __syncthreads();  // (to[] of the piece before is not read any more)
            if ((int)threadIdx.x < count) {
                const int at = s.len + x0 + (int)threadIdx.x, place = t.page.div(at);
                const int page = place >= s.used ? t.free_at((int64_t)top - (s.copy ? 1 : 0) - (place - s.used)) : s.copy ? fresh : s.old;
                to[threadIdx.x] = t.is_page(page) ? page * page_bytes + t.page.mod(at) * q.token_bytes : -1;
                if (!t.is_page(page)) t.tell(ATK_STATUS_BAD_PAGE);
            }
            __syncthreads();
            quantise_tokens<ELT, BITS>(pools.p[p], values.p[p] + i * values.seq[p] + x0 * values.token[p], values.token[p], to, count * (int)q.token.d, q);
        }
    }
    if (!tables || !last_workgroup(t.ticket)) return;
    if (bad) {
        if (threadIdx.x == 0) t.tell(bad);
        return;
    }
    append_tables(t, seqs, n, tokens, n_free);
}

// ---------------------------------------------------------------------------------------------------------------- read
struct Outs {
    char *p[kPools];
};

// What comes out is past the caches where it is more than half of what those hold: whoever reads it next would not find it there (eight sequences of 8192 tokens of two pools, 268 MB, 87 us -> 80).
constexpr int64_t kAroundBytes = INT64_C(128) << 20;
template <bool AROUND, typename T>
__device__ __forceinline__ void put(T v, T *to) {
    if (AROUND)
        __builtin_nontemporal_store(v, to);
    else
        *to = v;
}

template <int ELT, int BITS, bool AROUND>
__device__ __forceinline__ void store_eight(char *out, const uint32_t *w, float unit) {
    if constexpr (ELT == ATK_F32) {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        const mx_f32x2 a = mx_pair_f32<BITS, 0>(w, unit), b = mx_pair_f32<BITS, 1>(w, unit), c = mx_pair_f32<BITS, 2>(w, unit), d = mx_pair_f32<BITS, 3>(w, unit);
        put<AROUND>(f32x4{a[0], a[1], b[0], b[1]}, (f32x4 *)out);
        put<AROUND>(f32x4{c[0], c[1], d[0], d[1]}, (f32x4 *)out + 1);
    } else {
        put<AROUND>(mx_eight<ELT, BITS>(w, unit), (mx_u32x4 *)out);
    }
}

template <int ELT, int BITS, bool AROUND>
__global__ __launch_bounds__(kThreads) void quant_read_kernel(const PagesDev t, const Pools pools, const Outs outs, int n_pools, const QuantShape q, const int32_t *seqs, const int32_t *starts,
                                                              int64_t n, int64_t tokens) {
    __shared__ int64_t from[kThreads];
    constexpr int kAtOnce = 4;
    const int64_t items = n * n_pools * q.pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t of = item / q.pieces, i = of / n_pools;
        const int p = (int)(of % n_pools);
        const int64_t x0 = item % q.pieces * q.piece;
        const int count = (int)min((int64_t)q.piece, tokens - x0);
        __syncthreads();
        if ((int)threadIdx.x < count) {
            const int s = seqs[i];
            int64_t at = -1;
            int bad = 0;
            if (t.is_row(s)) {
                int64_t len = t.lens[s];
                const int64_t most = t.row_pages * t.page.d;
                if (len < 0 || len > most) bad = ATK_STATUS_BAD_LEN, len = len < 0 ? 0 : most;
                const int64_t key = (starts ? starts[i] : 0) + x0 + threadIdx.x;
                if (key >= 0 && key < len) {
                    const int page = t.table[s * t.row_pages + t.page.div((int)key)];
                    if (t.is_page(page))
                        at = ((int64_t)page * t.page.d + t.page.mod((int)key)) * q.token_bytes;
                    else
                        bad |= ATK_STATUS_BAD_PAGE;
                }
            } else {
                bad = ATK_STATUS_BAD_SEQ;
            }
            if (bad) t.tell(bad);
            from[threadIdx.x] = at;
        }
        __syncthreads();
        const char *pool = pools.p[p];
        char *out = outs.p[p] + (i * tokens + x0) * q.token.d * eight_bytes(ELT);
        const int units = count * (int)q.token.d;
        for (int u0 = threadIdx.x; u0 < units; u0 += kAtOnce * kThreads) {
            uint32_t w[kAtOnce][Mx<BITS>::kWords], byte[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int u = min(u0 + j * kThreads, units - 1), x = q.token.div(u), r = u - x * (int)q.token.d;
                const int64_t at = from[x];
                const char *row = pool + max(at, (int64_t)0);  // (there is a first row; what is read there in place of none is dropped)
                if constexpr (BITS == 4) {
                    w[j][0] = *(const uint32_t *)(row + r * 4);
                } else {
                    const mx_u32x2 c = *(const mx_u32x2 *)(row + r * 8);
                    w[j][0] = c[0], w[j][1] = c[1];
                }
                byte[j] = (uint8_t)row[q.code_bytes + r / 4];
                if (at < 0) {
                    byte[j] = 0;
#pragma unroll
                    for (int k = 0; k < Mx<BITS>::kWords; ++k) w[j][k] = 0;
                }
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int u = u0 + j * kThreads;
                if (u < units) store_eight<ELT, BITS, AROUND>(out + (int64_t)u * eight_bytes(ELT), w[j], mx_unit(byte[j]));
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------- host
static int check_shape(int64_t kv_heads, int64_t dim, int bits) {
    const int64_t bytes = atk_quant_token_bytes(kv_heads, dim, bits);
    return bytes < 0 ? (int)bytes : ATK_OK;
}

static QuantShape quant_shape(int64_t kv_heads, int64_t dim, int bits, int64_t tokens) {
    QuantShape q;
    q.token.set((uint32_t)(kv_heads * dim / 8));
    q.code_bytes = (uint32_t)(kv_heads * dim * bits / 8);
    q.token_bytes = mx_token_bytes(kv_heads, dim, bits);
    q.piece = (int)std::min<int64_t>(std::max<int64_t>(1, std::min<int64_t>(kThreads, kPieceUnits / q.token.d)), tokens);
    q.pieces = (int)((tokens + q.piece - 1) / q.piece);
    return q;
}

#define ATK_QUANT(elt, bits, call)                                                                  \
    do {                                                                                            \
        if ((bits) == 4) {                                                                          \
            constexpr int B = 4;                                                                    \
            if ((elt) == ATK_F32) { constexpr int E = ATK_F32; call; }                              \
            else if ((elt) == ATK_BF16) { constexpr int E = ATK_BF16; call; }                       \
            else { constexpr int E = ATK_F16; call; }                                               \
        } else {                                                                                    \
            constexpr int B = 8;                                                                    \
            if ((elt) == ATK_F32) { constexpr int E = ATK_F32; call; }                              \
            else if ((elt) == ATK_BF16) { constexpr int E = ATK_BF16; call; }                       \
            else { constexpr int E = ATK_F16; call; }                                               \
        }                                                                                           \
    } while (0)

}  // namespace atk

using namespace atk;

extern "C" {

int64_t atk_quant_token_bytes(int64_t kv_heads, int64_t dim, int bits) {
    if (bits != 4 && bits != 8) return ATK_ERR_UNSUPPORTED;
    if (kv_heads < 1 || dim < kMxBlock || dim > 256 || dim % kMxBlock || kv_heads > (1 << 20) / dim) return ATK_ERR_ARGS;
    return mx_token_bytes(kv_heads, dim, bits);
}

int atk_append_quantized(const atk_page_tables *t, void *const *pools, const void *const *values, const int64_t *value_strides, int64_t n_pools, int64_t kv_heads, int64_t dim, int bits,
                         int dtype, const int32_t *seqs, int64_t n, int64_t tokens, void *stream) {
    int rc = check_tables(t);
    if (rc == ATK_OK) rc = check_shape(kv_heads, dim, bits);
    if (rc != ATK_OK) return rc;
    if (dtype != ATK_F32 && dtype != ATK_BF16 && dtype != ATK_F16) return ATK_ERR_DTYPE;
    if (n < 0 || n > t->rows || !launches(n, kThreads) || tokens < 0 || tokens > (1 << 30)) return ATK_ERR_ARGS;
    uintptr_t address = 0;
    rc = check_pools(pools, n_pools, 1, &address);
    if (rc == ATK_OK && n * tokens > 0) rc = check_pools(values, n_pools, 1, &address);
    if (rc != ATK_OK) return rc;
    if (n == 0 || tokens == 0) return ATK_OK;
    // pages that the call could take, which its workgroups count in 31 bits (and no cache has: 2^28 at most)
    if (n * ((tokens + t->page_size - 1) / t->page_size + 1) > INT32_MAX) return ATK_ERR_ARGS;
    if (!seqs || (n_pools > 0 && !value_strides)) return ATK_ERR_NULL_PTR;
    if ((uintptr_t)seqs & 3) return ATK_ERR_ALIGN;
    const int64_t one[2] = {n, tokens};
    for (int64_t i = 0; i < 2 * n_pools; ++i) {
        if (value_strides[i] < 0) return ATK_ERR_ARGS;
        if (one[i & 1] > 1) address |= (uintptr_t)value_strides[i];
    }
    if (address & 15) return ATK_ERR_ALIGN;
    const PagesDev d = tables_dev(t);
    const QuantShape q = quant_shape(kv_heads, dim, bits, tokens);
    for (int64_t first = 0;; first += kPools) {  // the tables change with the last pools, and not before
        const int count = (int)std::min<int64_t>(kPools, n_pools - first);
        const bool last = first + count >= n_pools;
        Pools pp = {};
        QuantValues vv = {};
        for (int i = 0; i < count; ++i) {
            pp.p[i] = (char *)pools[first + i], vv.p[i] = (const char *)values[first + i];
            vv.seq[i] = n > 1 ? value_strides[2 * (first + i)] : 0, vv.token[i] = tokens > 1 ? value_strides[2 * (first + i) + 1] : 0;
        }
        const int shares = (int)std::max<int64_t>(1, std::min<int64_t>((int64_t)count * q.pieces, kCopyGrid / n));
        ATK_QUANT(dtype, bits, hipLaunchKernelGGL((quant_append_kernel<E, B>), dim3((uint32_t)(n * shares)), dim3(kThreads), 0, (hipStream_t)stream, d, pp, vv, count, q, seqs, n, tokens,
                                                  shares, last));
        rc = done();
        if (rc != ATK_OK || last) return rc;
    }
}

int atk_read_quantized(const atk_page_tables *t, const void *const *pools, void *const *outs, int64_t n_pools, int64_t kv_heads, int64_t dim, int bits, int dtype, const int32_t *seqs,
                       const int32_t *starts, int64_t n, int64_t tokens, void *stream) {
    int rc = check_tables(t);
    if (rc == ATK_OK) rc = check_shape(kv_heads, dim, bits);
    if (rc != ATK_OK) return rc;
    if (dtype != ATK_F32 && dtype != ATK_BF16 && dtype != ATK_F16) return ATK_ERR_DTYPE;
    if (n < 0 || n > (1 << 30) || tokens < 0 || tokens > (1 << 30) || n * tokens > (INT64_C(1) << 40)) return ATK_ERR_ARGS;
    uintptr_t address = 0;
    rc = check_pools(pools, n_pools, 1, &address);
    if (rc == ATK_OK && n * tokens > 0) rc = check_pools(outs, n_pools, 1, &address);
    if (rc != ATK_OK) return rc;
    if (n == 0 || tokens == 0 || n_pools == 0) return ATK_OK;
    if (!seqs) return ATK_ERR_NULL_PTR;
    if (address & 15) return ATK_ERR_ALIGN;
    if (((uintptr_t)seqs | (uintptr_t)starts) & 3) return ATK_ERR_ALIGN;
    const PagesDev d = tables_dev(t);
    const QuantShape q = quant_shape(kv_heads, dim, bits, tokens);
    for (int64_t first = 0; first < n_pools; first += kPools) {
        const int count = (int)std::min<int64_t>(kPools, n_pools - first);
        Pools pp = {};
        Outs oo = {};
        for (int i = 0; i < count; ++i) pp.p[i] = (char *)pools[first + i], oo.p[i] = (char *)outs[first + i];
        const uint32_t grid = (uint32_t)std::min<int64_t>(kCopyGrid, n * count * q.pieces);
        if (n * tokens * n_pools > kAroundBytes / (kv_heads * dim * (dtype == ATK_F32 ? 4 : 2)))
            ATK_QUANT(dtype, bits, hipLaunchKernelGGL((quant_read_kernel<E, B, true>), dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, d, pp, oo, count, q, seqs, starts, n, tokens));
        else
            ATK_QUANT(dtype, bits, hipLaunchKernelGGL((quant_read_kernel<E, B, false>), dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, d, pp, oo, count, q, seqs, starts, n, tokens));
        rc = done();
        if (rc != ATK_OK) return rc;
    }
    return ATK_OK;
}

}  // extern "C"
