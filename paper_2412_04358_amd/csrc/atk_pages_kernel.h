// The tables of a cache's pages on the device: what the kernels of atk_pages.hip and atk_quant_pages.hip share.
#pragma once

#include "atk_decode_common.h"

namespace atk {

constexpr int kPools = 64;       // pools of one launch: their addresses are kernel arguments
constexpr int kThreads = 256;
// Units (of 16 bytes, mostly) of a pool up to which a workgroup copies four pools at once, so as to wait for memory a quarter as often: four samples of two pools 7.8 -> 6.9 us.  With more
// of them pools one after the other are faster (512 samples of 24 pools, 1920 units: 77 us against 117): that many pools side by side are more addresses than the translation holds.
constexpr int kFlat = kThreads;
constexpr int kCopyGrid = 2048;  // workgroups of a launch that moves much: eight per CU

struct Pools {
    char *p[kPools];
};
struct Values {
    const char *p[kPools];
    int64_t stride[kPools];  // bytes from one sequence's to the next one's
};

struct PagesDev {
    int32_t *table, *lens, *refs, *free_pages, *n_free, *status;
    uint32_t *ticket;     // first words of the work area
    uint32_t *given;      // behind them: a bit for each page that was given back,
    uint32_t *left;       // ... a bit for each page that append copied,
    int32_t *leaving;     // ... and how many rows left such a page
    int64_t row_pages;
    int rows, n_pages;
    FastDiv page;         // tokens of a page
    __device__ __forceinline__ bool is_row(int s) const { return (unsigned)s < (unsigned)rows; }
    __device__ __forceinline__ bool is_page(int p) const { return (unsigned)p < (unsigned)n_pages; }
    __device__ __forceinline__ int pages(int64_t len) const { return page.div((int)(len + page.d - 1)); }
    // page i of the stack, from its bottom; -1 outside it (a count or a list of sequences that is not as the calls ask for)
    __device__ __forceinline__ int free_at(int64_t i) const { return i >= 0 && i < n_pages ? free_pages[i] : -1; }
    __device__ __forceinline__ void tell(int bits) const {
        if (status) atomicOr(status, bits);
    }
};
constexpr int kWorkHead = 64;    // bytes in front of the bits

// Copies `bytes` (a multiple of UNIT) with the workgroup's threads; both addresses are on UNIT bytes.
template <int UNIT>
struct Unit;
template <>
struct Unit<16> { typedef uint32_t T __attribute__((ext_vector_type(4))); };
template <>
struct Unit<4> { typedef uint32_t T; };
template <>
struct Unit<1> { typedef uint8_t T; };
// AROUND: around the caches, for whole pages, more of them than the caches hold (500 pages of 295 MB in all: 68 us -> 59, and 55 with 32-bit quotients in for_units; not for what the next call reads again: fork would be slower).
template <int UNIT, bool AROUND = false>
__device__ __forceinline__ void copy_bytes(char *dst, const char *src, int64_t bytes) {
    typedef typename Unit<UNIT>::T T;
    const int64_t n = bytes / UNIT;
    int64_t i = threadIdx.x;
    for (; i + 3 * kThreads < n; i += 4 * kThreads) {
        T t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = AROUND ? __builtin_nontemporal_load((const T *)src + i + j * kThreads) : ((const T *)src)[i + j * kThreads];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (AROUND)
                __builtin_nontemporal_store(t[j], (T *)dst + i + j * kThreads);
            else
                ((T *)dst)[i + j * kThreads] = t[j];
        }
    }
    for (; i < n; i += kThreads) ((T *)dst)[i] = ((const T *)src)[i];
}

// Whether this workgroup is the last of the launch to come here; the ticket is back at 0 then.  All that the others have read has been read, and their atomics have been done;
// their plain stores need not be visible (a release to the whole device writes the L2 back: 2048 of them made a launch that moves 380 MB four times as long).
__device__ __forceinline__ bool last_workgroup(uint32_t *ticket) {
    __shared__ uint32_t seen;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (threadIdx.x == 0) {
        seen = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (seen == gridDim.x - 1) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return seen == gridDim.x - 1;
}

// Sum of v over the workgroup; *before: over the threads in front of this one.
__device__ __forceinline__ int scan_threads(int v, int *before) {
    __shared__ int waves[kThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int up = v;
    for (int w = 1; w < 64; w <<= 1) {
        const int o = __shfl_up(up, w, 64);
        if (lane >= w) up += o;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = up;
    __syncthreads();
    int all = 0, front = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) front += waves[w];
        all += waves[w];
    }
    *before = front + up - v;
    return all;
}

// Sums of a and b and all bits of c over the workgroup.
__device__ __forceinline__ void meet_threads(int *a, int *b, int *c) {
    __shared__ int waves[3][kThreads / 64];
    for (int w = 1; w < 64; w <<= 1) *a += __shfl_xor(*a, w, 64), *b += __shfl_xor(*b, w, 64), *c |= __shfl_xor(*c, w, 64);
    if ((threadIdx.x & 63) == 0) waves[0][threadIdx.x >> 6] = *a, waves[1][threadIdx.x >> 6] = *b, waves[2][threadIdx.x >> 6] = *c;
    __syncthreads();
    *a = *b = *c = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) *a += waves[0][w], *b += waves[1][w], *c |= waves[2][w];
}

// Pushes the pages whose bits are set, the lowest last, and clears the bits.  By one workgroup.
__device__ __forceinline__ void push_given(const PagesDev &t) {
    const int words = (t.n_pages + 31) / 32;
    const int each = (words + kThreads - 1) / kThreads;
    const int from = min(words, (int)threadIdx.x * each), to = min(words, from + each);
    int mine = 0, before;
    for (int i = from; i < to; ++i) mine += __popc(__hip_atomic_load(&t.given[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    const int all = scan_threads(mine, &before);
    const int n = *t.n_free;
    // (a table that is at odds with its references could give back more than the stack has room for)
    const bool fits = n >= 0 && n <= t.n_pages - all;
    int at = n + all - 1 - before;
    for (int i = from; i < to; ++i) {
        uint32_t bits = __hip_atomic_load(&t.given[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (bits) t.given[i] = 0;
        for (; fits && bits; bits &= bits - 1) t.free_pages[at--] = i * 32 + __builtin_ctz(bits);
    }
    __syncthreads();
    if (threadIdx.x == 0 && all > 0) {
        if (fits)
            *t.n_free = n + all;
        else
            t.tell(ATK_STATUS_BAD_PAGE);
    }
}

// ------------------------------------------------------------------------------------------------------------- append
struct AppendSeq {
    int seq, len, used, after, old;  // old: a part-filled last page, -1 if there is none
    bool copy;                       // that other rows hold as well
    int bad;
    __device__ __forceinline__ int takes() const { return after - used + (copy ? 1 : 0); }
};
__device__ __forceinline__ AppendSeq append_seq(const PagesDev &t, const int32_t *seqs, int64_t i, int64_t tokens) {
    AppendSeq s;
    s.bad = 0, s.copy = false, s.old = -1, s.used = s.after = s.len = 0;
    s.seq = seqs[i];
    if (!t.is_row(s.seq)) {
        s.bad = ATK_STATUS_BAD_SEQ;
        return s;
    }
    const int len = t.lens[s.seq];
    if (len < 0 || len + tokens > t.row_pages * t.page.d) {
        s.bad = ATK_STATUS_BAD_LEN;
        return s;
    }
    s.len = len, s.used = t.pages(len), s.after = t.pages(len + tokens);
    if (t.page.mod(len)) {
        s.old = t.table[s.seq * t.row_pages + s.used - 1];
        if (t.is_page(s.old))
            s.copy = t.refs[s.old] > 1;
        else
            s.bad = ATK_STATUS_BAD_PAGE;
    }
    return s;
}

// What becomes of the tables when `tokens` tokens have gone to each of the sequences.  By one workgroup, the last to end; n_free: pages of the stack at the call.
__device__ __forceinline__ void append_tables(const PagesDev &t, const int32_t *seqs, int64_t n, int64_t tokens, int n_free) {
    // Rows, lengths and references, 256 sequences at a time.  Whether a page is copied goes by the references at the call, so the pages that
    // were copied only lose theirs afterwards.  Pages in their order over all threads: one thread for a sequence's took as long as all the rest of a prompt of 4000 tokens (250 pages).
    __shared__ int fronts[kThreads], places[kThreads], rows[kThreads];
    int base = n_free;
    bool copied = false;
    for (int64_t j0 = 0; j0 < n; j0 += kThreads) {
        const int64_t j = j0 + threadIdx.x;
        AppendSeq s;
        int takes = 0, front;
        if (j < n) {
            s = append_seq(t, seqs, j, tokens);
            takes = s.takes();
        }
        const int all = scan_threads(takes, &front);
        fronts[threadIdx.x] = front;
        if (j < n && !s.bad) {
            places[threadIdx.x] = s.copy ? s.used - 1 : s.used, rows[threadIdx.x] = s.seq;
            if (s.copy) {
                copied = true;
                atomicOr(&t.left[s.old >> 5], 1u << (s.old & 31));
                atomicAdd(&t.leaving[s.old], 1);
            }
            t.lens[s.seq] = (int)(s.len + tokens);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < all; e += kThreads) {
            int i = 0;  // the last sequence in front of which there are e pages at most: the one that takes page e
            for (int w = kThreads / 2; w > 0; w /= 2)
                if (fronts[i + w] <= e) i += w;
            const int fresh = t.free_at((int64_t)base - 1 - e);
            t.table[rows[i] * t.row_pages + places[i] + (e - fronts[i])] = fresh;
            if (t.is_page(fresh)) atomicAdd(&t.refs[fresh], 1);
        }
        __syncthreads();
        base -= all;
    }
    if (threadIdx.x == 0) *t.n_free = base;
    __builtin_amdgcn_s_waitcnt(0);
    if (!__syncthreads_or(copied)) return;
    for (int w = threadIdx.x; w < (t.n_pages + 31) / 32; w += kThreads) {
        uint32_t bits = __hip_atomic_load(&t.left[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), empty = 0;
        if (!bits) continue;
        t.left[w] = 0;
        for (; bits; bits &= bits - 1) {
            const int page = w * 32 + __builtin_ctz(bits);
            const int rows = atomicExch(&t.leaving[page], 0);
            if (atomicSub(&t.refs[page], rows) == rows) empty |= bits & -bits;
        }
        if (empty) atomicOr(&t.given[w], empty);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    push_given(t);
}

// ---------------------------------------------------------------------------------------------------------------- host
inline int64_t pages_words(int64_t n_pages) { return (n_pages + 31) / 32; }

inline int check_tables(const atk_page_tables *t) {
    if (!t) return ATK_ERR_NULL_PTR;
    const int64_t most = INT64_C(1) << 30;
    if (t->rows < 1 || t->row_pages < 1 || t->n_pages < 1 || t->page_size < 1 || t->rows > most || t->row_pages > most || t->n_pages > (1 << 28) || t->page_size > most)
        return ATK_ERR_ARGS;
    if (t->row_pages * t->page_size > most) return ATK_ERR_ARGS;
    if (!t->page_table || !t->lens || !t->refs || !t->free_pages || !t->n_free || !t->work) return ATK_ERR_NULL_PTR;
    if (((uintptr_t)t->page_table | (uintptr_t)t->lens | (uintptr_t)t->refs | (uintptr_t)t->free_pages | (uintptr_t)t->n_free | (uintptr_t)t->status) & 3) return ATK_ERR_ALIGN;
    if ((uintptr_t)t->work & 15) return ATK_ERR_ALIGN;
    if (t->work_bytes < atk_pages_work_bytes(t->n_pages)) return ATK_ERR_WORKSPACE;
    return ATK_OK;
}

inline int32_t *work_moves(const atk_page_tables *t) { return (int32_t *)((char *)t->work + kWorkHead + 8 * pages_words(t->n_pages) + 4 * t->n_pages); }

inline PagesDev tables_dev(const atk_page_tables *t) {
    PagesDev d;
    d.table = t->page_table, d.lens = t->lens, d.refs = t->refs, d.free_pages = t->free_pages, d.n_free = t->n_free, d.status = t->status;
    d.ticket = (uint32_t *)t->work;
    d.given = (uint32_t *)((char *)t->work + kWorkHead);
    d.left = d.given + pages_words(t->n_pages);
    d.leaving = (int32_t *)(d.left + pages_words(t->n_pages));
    d.row_pages = t->row_pages, d.rows = (int)t->rows, d.n_pages = (int)t->n_pages;
    d.page.set((uint32_t)t->page_size);
    return d;
}

inline int check_pools(const void *const *pools, int64_t n, int64_t bytes, uintptr_t *bits) {
    if (n < 0 || n > 65536 || bytes < 1 || bytes > (INT64_C(1) << 40)) return ATK_ERR_ARGS;
    if (n > 0 && !pools) return ATK_ERR_NULL_PTR;
    for (int64_t i = 0; i < n; ++i) {
        if (!pools[i]) return ATK_ERR_NULL_PTR;
        *bits |= (uintptr_t)pools[i];
    }
    return ATK_OK;
}
inline int done() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // namespace atk
