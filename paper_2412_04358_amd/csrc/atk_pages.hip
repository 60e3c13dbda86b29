// The pages of a cache: copy, fork, append, free, compact (include/atk_decode.h).
//
// These calls move whole tokens (bound by memory: every byte read once and written once) and change a few words of the tables (bound by launches and the
// chain of dependent reads), so each is one launch where it can be: a workgroup finds out by itself what the sequences in front of its own take from
// the stack (a sum over the call's sequences), moves its share of the data, and the last workgroup to end - by a ticket - changes what the others read.
// Nothing depends on the order of workgroups: pages are taken by rank and given back by number.  That each workgroup of fork and append reads all of the call's sequences
// is little for hundreds of them and quadratic past some thousands (one pool, fork and free: 512 sequences 31 us, 2048 85, 8192 263, 32768 1690).
// 16 sequences forked to 512 in 24 pools of 32 KB pages: fork 57 us, append of five tokens 69, free 17; compaction that moves
// 1500 pages of 16 pools, 1.57 GB read and written, 310 us (5.1 TB/s, a large copy's rate); 500 pages of 8 pools, 295 MB, in 55 us (5.4 TB/s, part of it out of the caches); one sequence: 6, 8 and 5 us.
#include "atk_pages_kernel.h"

namespace atk {

struct PoolPairs {
    const char *src[kPools];
    char *dst[kPools];
};
// The same for several pools, four at once: short pieces one after the other would wait for memory each time.  Unit u of src(x) goes to the
// byte where(u) of dst(x), x < n.
template <int UNIT, typename DST, typename SRC, typename WHERE>
__device__ __forceinline__ void copy_pools(int n, int units, DST dst, SRC src, WHERE where) {
    typedef typename Unit<UNIT>::T T;
    for (int x = 0; x < n; x += 4) {
        const T *from[4];
        char *into[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) from[j] = (const T *)src(min(x + j, n - 1)), into[j] = dst(min(x + j, n - 1));
        for (int u = threadIdx.x; u < units; u += kThreads) {
            const int64_t to = where(u);
            T t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (x + j < n) t[j] = from[j][u];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (x + j < n) *(T *)(into[j] + to) = t[j];
        }
    }
}

// One pool: unit u goes to the byte where(u) of dst.  Around the caches (512 samples' five tokens in 24 pools, fork and append: 185 us -> 179).
template <int UNIT, typename WHERE>
__device__ __forceinline__ void copy_pool(char *dst, const char *src, int units, WHERE where) {
    typedef typename Unit<UNIT>::T T;
    for (int u0 = threadIdx.x; u0 < units; u0 += 4 * kThreads) {
        T t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = __builtin_nontemporal_load((const T *)src + min(u0 + j * kThreads, units - 1));
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (u0 + j * kThreads < units) __builtin_nontemporal_store(t[j], (T *)(dst + where(u0 + j * kThreads)));
    }
}

// One row less holds the page.
__device__ __forceinline__ void give_back(const PagesDev &t, int page) {
    const int was = atomicSub(&t.refs[page], 1);
    if (was == 1) {
        atomicOr(&t.given[page >> 5], 1u << (page & 31));
    } else if (was < 1) {
        atomicAdd(&t.refs[page], 1);
        t.tell(ATK_STATUS_BAD_PAGE);
    }
}

// ---------------------------------------------------------------------------------------------------------------- copy
// f(page i, pool, piece of the page) for this workgroup's share of all of them.  (Their number mostly fits 32 bits, whose quotients take a tenth of 64 bits'.)
template <typename F>
__device__ __forceinline__ void for_units(int64_t n, int n_pools, int pieces, F f) {
    const int64_t units = n * n_pools * pieces;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        if (units <= 0xffffffffu) {
            const uint32_t y = (uint32_t)u / (uint32_t)pieces, i = y / (uint32_t)n_pools;
            f(i, (int)(y - i * n_pools), (int)((uint32_t)u - y * pieces));
        } else {
            const int64_t y = u / pieces, i = y / n_pools;
            f(i, (int)(y - i * n_pools), (int)(u - y * pieces));
        }
    }
}
template <int UNIT>
__global__ __launch_bounds__(kThreads) void pages_copy_kernel(const PoolPairs pools, int n_pools, int64_t page_bytes, int64_t piece, int pieces, int src_pages,
                                                              int dst_pages, const int32_t *src_ids, const int32_t *dst_ids, int64_t n, int32_t *status) {
    for_units(n, n_pools, pieces, [&](int64_t i, int pool, int x) {
        const int src = src_ids[i], dst = dst_ids[i];
        if ((unsigned)src >= (unsigned)src_pages || (unsigned)dst >= (unsigned)dst_pages) {
            if (threadIdx.x == 0 && status) atomicOr(status, ATK_STATUS_BAD_PAGE);
            return;
        }
        const int64_t at = x * piece;
        copy_bytes<UNIT, true>(pools.dst[pool] + dst * page_bytes + at, pools.src[pool] + src * page_bytes + at, min(piece, page_bytes - at));
    });
}

// ---------------------------------------------------------------------------------------------------------------- fork
struct ForkNeed {
    int total;   // pages that the call takes
    int before;  // ... for sequences in front of `mine`
    int bad;
};
// mine: the sequence that the workgroup works on
__device__ __forceinline__ ForkNeed fork_need(const PagesDev &t, const int32_t *parents, const int32_t *children, int64_t n, int64_t mine) {
    int total = 0, before = 0, bad = 0;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
        const int p = parents[i], c = children[i];
        if (!t.is_row(p) || !t.is_row(c)) {
            bad |= ATK_STATUS_BAD_SEQ;
            continue;
        }
        const int len = t.lens[p];
        if (len < 0 || len > t.row_pages * t.page.d) bad |= ATK_STATUS_BAD_LEN;  // (before any quotient: those are of 31 bits)
        else if (t.page.mod(len)) ++total, before += i < mine;
        if (t.lens[c] != 0) bad |= ATK_STATUS_BAD_SEQ;
    }
    const int n_free = *t.n_free;
    meet_threads(&total, &before, &bad);
    if (total > n_free) bad |= ATK_STATUS_NO_PAGES;
    return ForkNeed{total, before, bad};
}

template <int UNIT>
__global__ __launch_bounds__(kThreads) void pages_fork_kernel(const PagesDev t, const Pools pools, int n_pools, int64_t token_bytes, const int32_t *parents,
                                                              const int32_t *children, int64_t n, int shares, bool tables) {
    const int64_t i = blockIdx.x / shares;
    const int share = (int)(blockIdx.x % shares);
    const ForkNeed need = fork_need(t, parents, children, n, i);
    if (!need.bad) {
        const int parent = parents[i], child = children[i];
        const int len = t.lens[parent], part = t.page.mod(len), used = t.pages(len);
        const int32_t *row = t.table + parent * t.row_pages;
        int fresh = -1;
        if (part) {
            const int old = row[used - 1];
            fresh = t.free_at((int64_t)*t.n_free - 1 - need.before);
            if (t.is_page(old) && t.is_page(fresh)) {
                const int64_t to = (int64_t)fresh * t.page.d * token_bytes, from = (int64_t)old * t.page.d * token_bytes, units = part * token_bytes / UNIT;
                if (units <= kFlat) {
                    copy_pools<UNIT>((n_pools - share + shares - 1) / shares, (int)units, [&](int x) { return pools.p[share + x * shares] + to; },
                                     [&](int x) { return pools.p[share + x * shares] + from; }, [&](int u) { return (int64_t)u * UNIT; });
                } else {
                    for (int p = share; p < n_pools; p += shares) copy_bytes<UNIT>(pools.p[p] + to, pools.p[p] + from, part * token_bytes);
                }
            } else if (threadIdx.x == 0) {
                t.tell(ATK_STATUS_BAD_PAGE);
            }
        }
        if (tables && share == 0) {
            int32_t *to = t.table + child * t.row_pages;
            for (int64_t j = threadIdx.x; j < t.row_pages; j += kThreads) {
                const int page = j < used ? (part && j == used - 1 ? fresh : row[j]) : -1;
                to[j] = page;
                if (j < used) {
                    if (t.is_page(page))
                        atomicAdd(&t.refs[page], 1);
                    else
                        t.tell(ATK_STATUS_BAD_PAGE);
                }
            }
        }
    }
    if (!tables || !last_workgroup(t.ticket)) return;
    if (need.bad) {
        if (threadIdx.x == 0) t.tell(need.bad);
        return;
    }
    // Lengths as they were at the call, also where a parent is a child of another pair: children were empty, so a parent's length that is a new one by now - which are
    // stored as their complements until all have been read - was 0.
    for (int64_t j = threadIdx.x; j < n; j += kThreads) t.lens[children[j]] = ~max(0, t.lens[parents[j]]);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int64_t j = threadIdx.x; j < n; j += kThreads) {
        const int len = t.lens[children[j]];
        if (len < 0) t.lens[children[j]] = ~len;
    }
    if (threadIdx.x == 0) *t.n_free -= need.total;
}

// -------------------------------------------------------------------------------------------------------------- append
template <int UNIT>
__global__ __launch_bounds__(kThreads) void pages_append_kernel(const PagesDev t, const Pools pools, const Values values, int n_pools, int64_t token_bytes,
                                                                const int32_t *seqs, int64_t n, int64_t tokens, int shares, bool tables) {
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
    const int64_t page_bytes = (int64_t)t.page.d * token_bytes;
    if (!bad) {
        const AppendSeq s = append_seq(t, seqs, i, tokens);
        const int top = n_free - 1 - before;
        const int part = t.page.mod(s.len);
        const int fresh = s.copy ? t.free_at(top) : -1;
        // the page that new token x goes to
        auto page_of = [&](int64_t x) {
            const int place = t.page.div((int)(s.len + x));
            return place >= s.used ? t.free_at((int64_t)top - (s.copy ? 1 : 0) - (place - s.used)) : s.copy ? fresh : s.old;
        };
        const int mine = (n_pools - share + shares - 1) / shares;
        if (s.copy && t.is_page(fresh))
            for (int p = share; p < n_pools; p += shares) copy_bytes<UNIT>(pools.p[p] + fresh * page_bytes, pools.p[p] + s.old * page_bytes, part * token_bytes);
        const int64_t token_units = token_bytes / UNIT;
        if (tokens <= kThreads && token_units < (1 << 20)) {
            // where each token goes, once for all pools
            __shared__ int64_t to[kThreads];
            if (threadIdx.x < tokens) {
                const int page = page_of(threadIdx.x);
                to[threadIdx.x] = t.is_page(page) ? page * page_bytes + t.page.mod((int)(s.len + threadIdx.x)) * token_bytes : -1;
                if (!t.is_page(page)) t.tell(ATK_STATUS_BAD_PAGE);
            }
            if (__syncthreads_and(threadIdx.x >= tokens || to[threadIdx.x] >= 0)) {
                const int units = (int)(tokens * token_units);
                auto where = [&](int u) {
                    const int x = u / (int)token_units;
                    return to[x] + (int64_t)(u - x * (int)token_units) * UNIT;
                };
                if (units <= kFlat)
                    copy_pools<UNIT>(mine, units, [&](int x) { return pools.p[share + x * shares]; },
                                     [&](int x) { return values.p[share + x * shares] + i * values.stride[share + x * shares]; }, where);
                else
                    for (int p = share; p < n_pools; p += shares) copy_pool<UNIT>(pools.p[p], values.p[p] + i * values.stride[p], units, where);
            }
        } else {
            for (int p = share; p < n_pools; p += shares) {
                const char *value = values.p[p] + i * values.stride[p];
                for (int64_t done = 0; done < tokens;) {  // page by page
                    const int slot = t.page.mod((int)(s.len + done));
                    const int64_t now = min(tokens - done, (int64_t)(t.page.d - slot));
                    const int page = page_of(done);
                    if (t.is_page(page))
                        copy_bytes<UNIT>(pools.p[p] + page * page_bytes + slot * token_bytes, value + done * token_bytes, now * token_bytes);
                    else if (threadIdx.x == 0)
                        t.tell(ATK_STATUS_BAD_PAGE);
                    done += now;
                }
            }
        }
    }
    if (!tables || !last_workgroup(t.ticket)) return;
    if (bad) {
        if (threadIdx.x == 0) t.tell(bad);
        return;
    }
    append_tables(t, seqs, n, tokens, n_free);
}

// ---------------------------------------------------------------------------------------------------------------- free
__global__ __launch_bounds__(kThreads) void pages_free_kernel(const PagesDev t, const int32_t *seqs, const int32_t *drop, int64_t n) {
    __shared__ int length;
    const int seq = seqs[blockIdx.x];
    if (t.is_row(seq)) {
        if (threadIdx.x == 0) length = t.lens[seq];
        __syncthreads();
        int len = length;
        if (len < 0 || len > t.row_pages * t.page.d) {
            if (threadIdx.x == 0) t.tell(ATK_STATUS_BAD_LEN);
            len = len < 0 ? 0 : (int)(t.row_pages * t.page.d);
        }
        const int keep = drop ? max(0, len - max(0, drop[blockIdx.x])) : 0;
        int32_t *row = t.table + seq * t.row_pages;
        const int used = t.pages(len);
        for (int j = t.pages(keep) + threadIdx.x; j < used; j += kThreads) {
            const int page = atomicExch(&row[j], -1);  // (a row given twice gives its pages back once)
            if (t.is_page(page))
                give_back(t, page);
            else if (page != -1)
                t.tell(ATK_STATUS_BAD_PAGE);
        }
        if (threadIdx.x == 0) t.lens[seq] = keep;
    } else if (threadIdx.x == 0) {
        t.tell(ATK_STATUS_BAD_SEQ);
    }
    if (last_workgroup(t.ticket)) push_given(t);
}

// ------------------------------------------------------------------------------------------------------------- compact
// The plan: how many pages are held, the new number of each, the list of moves (behind the work area's bits: sources, then destinations, as many as there
// are pages at most) and the stack.  One workgroup of 1024, which goes over the pages twice, 1024 at a time: 11 us for a call with 6000 pages and nothing to move, 35 with 30000, 100 with 100000,
// 1210 with a million.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void pages_plan_kernel(const PagesDev t, int32_t *remap, int32_t *moves, int32_t *n_moves) {
    __shared__ int waves[3][kPlanThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int carry[3] = {0, 0, 0};  // held; holes; movers
    const int P = t.n_pages;
    int held = 0;
    for (int p = threadIdx.x; p < P; p += kPlanThreads) held += t.refs[p] > 0;
    for (int w = 1; w < 64; w <<= 1) held += __shfl_xor(held, w, 64);
    if (lane == 0) waves[0][wave] = held;
    __syncthreads();
    int live = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) live += waves[0][w];
    __syncthreads();
    for (int p0 = 0; p0 < P; p0 += kPlanThreads) {
        const int p = p0 + threadIdx.x;
        const bool is_held = p < P && t.refs[p] > 0;
        const bool hole = p < live && !is_held, mover = is_held && p >= live;
        const uint64_t holes = __ballot(hole), movers = __ballot(mover);
        if (lane == 0) waves[1][wave] = __popcll(holes), waves[2][wave] = __popcll(movers);
        __syncthreads();
        int front[3], all[3];
#pragma unroll
        for (int k = 1; k < 3; ++k) {
            front[k] = carry[k], all[k] = 0;
            for (int w = 0; w < kPlanThreads / 64; ++w) {
                if (w < wave) front[k] += waves[k][w];
                all[k] += waves[k][w];
            }
            carry[k] += all[k];
        }
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        if (hole) moves[P + front[1] + __popcll(holes & below)] = p;
        if (mover) moves[front[2] + __popcll(movers & below)] = p;
        if (p < P) remap[p] = is_held && p < live ? p : -1;
        if (p < P - live) t.free_pages[p] = P - 1 - p;
        __syncthreads();
    }
    // (this workgroup's own stores: visible to it behind the barrier)
    for (int i = threadIdx.x; i < carry[2]; i += kPlanThreads) remap[moves[i]] = moves[P + i];
    if (threadIdx.x == 0) *n_moves = carry[2], *t.n_free = P - live;
}

template <int UNIT>
__global__ __launch_bounds__(kThreads) void pages_move_kernel(const PagesDev t, const Pools pools, int n_pools, int64_t page_bytes, int64_t piece, int pieces,
                                                              const int32_t *remap, const int32_t *moves, const int32_t *n_moves, bool tables) {
    const int n = *n_moves;
    for_units(n, n_pools, pieces, [&](int64_t i, int pool, int x) {
        const int64_t at = x * piece;
        copy_bytes<UNIT, true>(pools.p[pool] + moves[t.n_pages + i] * page_bytes + at, pools.p[pool] + moves[i] * page_bytes + at, min(piece, page_bytes - at));
    });
    if (!tables) return;
    const int64_t threads = (int64_t)gridDim.x * kThreads, me = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    for (int64_t i = me; i < n; i += threads) {
        t.refs[moves[t.n_pages + i]] = t.refs[moves[i]];
        t.refs[moves[i]] = 0;
    }
    const int64_t entries = t.rows * t.row_pages;
    for (int64_t j = me; j < entries; j += threads) {
        const int page = t.table[j];
        if (page < 0) continue;
        const int to = t.is_page(page) ? remap[page] : -1;
        if (to != page) t.table[j] = to;
        if (to < 0) t.tell(ATK_STATUS_BAD_PAGE);
    }
}

// ---------------------------------------------------------------------------------------------------------------- host
// the widest unit that all addresses and sizes are multiples of
static int unit_of(uintptr_t bits) { return bits & 15 ? (bits & 3 ? 1 : 4) : 16; }

#define ATK_UNIT(unit, call)                    \
    do {                                        \
        if ((unit) == 16) { constexpr int U = 16; call; } \
        else if ((unit) == 4) { constexpr int U = 4; call; } \
        else { constexpr int U = 1; call; }     \
    } while (0)

// workgroups that a sequence's data is shared out to: no more than there are pools, and no more than fill the chip
static int shares_of(int64_t n, int64_t pools) { return (int)std::max<int64_t>(1, std::min<int64_t>(pools, kCopyGrid / n)); }

}  // namespace atk

using namespace atk;

extern "C" {

int64_t atk_pages_work_bytes(int64_t n_pages) {
    if (n_pages < 1 || n_pages > (1 << 28)) return ATK_ERR_ARGS;
    return kWorkHead + 8 * pages_words(n_pages) + 12 * n_pages + 16;
}

int atk_copy_pages(const void *const *src_pools, void *const *dst_pools, int64_t n_pools, int64_t page_bytes, int64_t src_pages, int64_t dst_pages, const int32_t *src_ids,
                   const int32_t *dst_ids, int64_t n, int32_t *status, void *stream) {
    uintptr_t bits = (uintptr_t)page_bytes;
    int rc = check_pools(src_pools, n_pools, page_bytes, &bits);
    if (rc == ATK_OK) rc = check_pools(dst_pools, n_pools, page_bytes, &bits);
    if (rc != ATK_OK) return rc;
    if (src_pages < 1 || dst_pages < 1 || src_pages > (1 << 28) || dst_pages > (1 << 28) || n < 0 || n > (1 << 28)) return ATK_ERR_ARGS;
    if (n == 0 || n_pools == 0) return ATK_OK;
    if (!src_ids || !dst_ids) return ATK_ERR_NULL_PTR;
    if (((uintptr_t)src_ids | (uintptr_t)dst_ids | (uintptr_t)status) & 3) return ATK_ERR_ALIGN;
    const int64_t piece = 16384;
    const int pieces = (int)((page_bytes + piece - 1) / piece);
    for (int64_t first = 0; first < n_pools; first += kPools) {
        const int count = (int)std::min<int64_t>(kPools, n_pools - first);
        PoolPairs pp = {};
        for (int i = 0; i < count; ++i) pp.src[i] = (const char *)src_pools[first + i], pp.dst[i] = (char *)dst_pools[first + i];
        const uint32_t grid = (uint32_t)std::min<int64_t>(kCopyGrid, n * count * pieces);
        ATK_UNIT(unit_of(bits), hipLaunchKernelGGL((pages_copy_kernel<U>), dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, pp, count, page_bytes, piece, pieces, (int)src_pages,
                                                   (int)dst_pages, src_ids, dst_ids, n, status));
        rc = done();
        if (rc != ATK_OK) return rc;
    }
    return ATK_OK;
}

int atk_fork_sequences(const atk_page_tables *t, void *const *pools, int64_t n_pools, int64_t token_bytes, const int32_t *parents, const int32_t *children, int64_t n, void *stream) {
    int rc = check_tables(t);
    uintptr_t bits = (uintptr_t)token_bytes;
    if (rc == ATK_OK) rc = check_pools(pools, n_pools, token_bytes, &bits);
    if (rc != ATK_OK) return rc;
    if (n < 0 || n > t->rows || !launches(n, kThreads)) return ATK_ERR_ARGS;
    if (n == 0) return ATK_OK;
    if (!parents || !children) return ATK_ERR_NULL_PTR;
    if (((uintptr_t)parents | (uintptr_t)children) & 3) return ATK_ERR_ALIGN;
    const PagesDev d = tables_dev(t);
    // the tables change with the last pools, and not before
    for (int64_t first = 0;; first += kPools) {
        const int count = (int)std::min<int64_t>(kPools, n_pools - first);
        const bool last = first + count >= n_pools;
        Pools pp = {};
        for (int i = 0; i < count; ++i) pp.p[i] = (char *)pools[first + i];
        const int shares = shares_of(n, count);
        ATK_UNIT(unit_of(bits), hipLaunchKernelGGL((pages_fork_kernel<U>), dim3((uint32_t)(n * shares)), dim3(kThreads), 0, (hipStream_t)stream, d, pp, count, token_bytes, parents, children,
                                                   n, shares, last));
        rc = done();
        if (rc != ATK_OK || last) return rc;
    }
}

int atk_append_tokens(const atk_page_tables *t, void *const *pools, const void *const *values, const int64_t *value_strides, int64_t n_pools, int64_t token_bytes, const int32_t *seqs,
                      int64_t n, int64_t tokens, void *stream) {
    int rc = check_tables(t);
    uintptr_t bits = (uintptr_t)token_bytes;
    if (rc == ATK_OK) rc = check_pools(pools, n_pools, token_bytes, &bits);
    if (rc == ATK_OK && n * tokens > 0) rc = check_pools(values, n_pools, token_bytes, &bits);
    if (rc != ATK_OK) return rc;
    if (n < 0 || n > t->rows || !launches(n, kThreads) || tokens < 0 || tokens > (1 << 30)) return ATK_ERR_ARGS;
    if (n == 0 || tokens == 0) return ATK_OK;
    // pages that the call could take, which its workgroups count in 31 bits (and no cache has: 2^28 at most)
    if (n * ((tokens + t->page_size - 1) / t->page_size + 1) > INT32_MAX) return ATK_ERR_ARGS;
    if (!seqs || (n_pools > 0 && !value_strides)) return ATK_ERR_NULL_PTR;
    if ((uintptr_t)seqs & 3) return ATK_ERR_ALIGN;
    for (int64_t i = 0; i < n_pools; ++i) {
        if (value_strides[i] < 0) return ATK_ERR_ARGS;
        bits |= (uintptr_t)value_strides[i];
    }
    const PagesDev d = tables_dev(t);
    for (int64_t first = 0;; first += kPools) {
        const int count = (int)std::min<int64_t>(kPools, n_pools - first);
        const bool last = first + count >= n_pools;
        Pools pp = {};
        Values vv = {};
        for (int i = 0; i < count; ++i) pp.p[i] = (char *)pools[first + i], vv.p[i] = (const char *)values[first + i], vv.stride[i] = value_strides[first + i];
        const int shares = shares_of(n, count);
        ATK_UNIT(unit_of(bits), hipLaunchKernelGGL((pages_append_kernel<U>), dim3((uint32_t)(n * shares)), dim3(kThreads), 0, (hipStream_t)stream, d, pp, vv, count, token_bytes, seqs, n,
                                                   tokens, shares, last));
        rc = done();
        if (rc != ATK_OK || last) return rc;
    }
}

int atk_free_sequences(const atk_page_tables *t, const int32_t *seqs, const int32_t *drop, int64_t n, void *stream) {
    int rc = check_tables(t);
    if (rc != ATK_OK) return rc;
    if (n < 0 || n > t->rows || !launches(n, kThreads)) return ATK_ERR_ARGS;
    if (n == 0) return ATK_OK;
    if (!seqs) return ATK_ERR_NULL_PTR;
    if (((uintptr_t)seqs | (uintptr_t)drop) & 3) return ATK_ERR_ALIGN;
    hipLaunchKernelGGL(pages_free_kernel, dim3((uint32_t)n), dim3(kThreads), 0, (hipStream_t)stream, tables_dev(t), seqs, drop, n);
    return done();
}

int atk_compact_pages(const atk_page_tables *t, void *const *pools, int64_t n_pools, int64_t token_bytes, int32_t *remap, void *stream) {
    int rc = check_tables(t);
    uintptr_t bits = (uintptr_t)token_bytes;
    if (rc == ATK_OK) rc = check_pools(pools, n_pools, token_bytes, &bits);
    if (rc != ATK_OK) return rc;
    if (!remap) return ATK_ERR_NULL_PTR;
    if ((uintptr_t)remap & 3) return ATK_ERR_ALIGN;
    if (token_bytes > (INT64_C(1) << 40) / t->page_size) return ATK_ERR_ARGS;
    const PagesDev d = tables_dev(t);
    int32_t *moves = work_moves(t), *n_moves = (int32_t *)t->work + 1;
    hipLaunchKernelGGL(pages_plan_kernel, dim3(1), dim3(kPlanThreads), 0, (hipStream_t)stream, d, remap, moves, n_moves);
    rc = done();
    const int64_t page_bytes = token_bytes * t->page_size, piece = 16384;
    const int pieces = (int)((page_bytes + piece - 1) / piece);
    for (int64_t first = 0; rc == ATK_OK; first += kPools) {
        const int count = (int)std::min<int64_t>(kPools, n_pools - first);
        const bool last = first + count >= n_pools;
        Pools pp = {};
        for (int i = 0; i < count; ++i) pp.p[i] = (char *)pools[first + i];
        // at most half of the pages move
        const int64_t most = std::max<int64_t>(t->n_pages / 2 * count * pieces, (t->rows * t->row_pages + 1023) / 1024);
        const uint32_t grid = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(kCopyGrid, most));
        ATK_UNIT(unit_of(bits), hipLaunchKernelGGL((pages_move_kernel<U>), dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, d, pp, count, page_bytes, piece, pieces, remap, moves, n_moves,
                                                   last));
        rc = done();
        if (last) break;
    }
    return rc;
}

}  // extern "C"
