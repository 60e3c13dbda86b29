// verify_drafts: accepted drafts, and one token drawn from what is left of the target's probabilities (include/atk_decode.h).
//
// 64 requests of 5 drafts over 128256 tokens in bf16: 33 MB at the least, 11 + 8 us; one request over 32000 f32: 9 us, one launch.
//
// Only one row of the target's probabilities is needed whole, and after a rejection one of the draft's: those of the first rejected
// token.  verify_sums_kernel finds it (a few gathers, done again by every workgroup of the request), and sums the weights of tiles of that row;
// verify_draw_kernel finds the tile, then a lane's eight elements, then the element at which the running sum passes the goal.
// verify_row_kernel does both for short rows.  Sums are f64: an index is what comes out, and the running sum of 10^5 f32 would be off by more than the weights.
#include "atk_decode_common.h"

namespace atk {

struct VerifyDev {
    const void *target, *draft;
    const int32_t *draft_tokens, *n_drafts;
    const float *u, *r;
    int32_t *accepted, *tokens;
    double2 *sums;  // [request][tile]: residual weights, target's weights
    int64_t ts[2], ds[2];
    int64_t vocab;
    int drafts, tiles, groups;  // tiles of a row, workgroups that share them
};

template <int ELT>
__device__ __forceinline__ double prob(const void *p, int64_t i) {
    if (ELT == ATK_F32) return (double)((const float *)p)[i];
    if (ELT == ATK_F16) return (double)(float)((const _Float16 *)p)[i];
    return (double)__uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16);
}
template <int ELT>
__device__ __forceinline__ const void *at(const void *p, int64_t i) { return (const char *)p + i * (ELT == ATK_F32 ? 4 : 2); }

// The row that the last token of a request is drawn from.
template <int ELT>
struct VerifyRow {
    const void *p, *q;   // q: NULL for no subtraction
    int64_t certain;     // element that a draft without probabilities had for sure, -1 if none
    int accepted;

    // found: how many were accepted, where that is known
    __device__ __forceinline__ VerifyRow(const VerifyDev &a, int64_t b, int found = -1) {
        const int lane = threadIdx.x & 63;
        const int n = a.n_drafts ? min(max(a.n_drafts[b], 0), a.drafts) : a.drafts;
        int first = n;
        if (found >= 0) first = found;
        for (int i0 = 0; found < 0 && i0 < n && first == n; i0 += 64) {
            const int i = i0 + lane;
            bool no = false;
            if (i < n) {
                const int64_t d = a.draft_tokens[b * a.drafts + i];
                no = true;
                if (d >= 0 && d < a.vocab) {
                    const double pd = prob<ELT>(a.target, b * a.ts[0] + i * a.ts[1] + d);
                    const double qd = a.draft ? prob<ELT>(a.draft, b * a.ds[0] + i * a.ds[1] + d) : 1.0;
                    no = !((double)a.u[b * a.drafts + i] * qd < pd);
                }
            }
            const uint64_t votes = __ballot(no);
            if (votes) first = i0 + __builtin_ctzll(votes);
        }
        accepted = first;
        p = at<ELT>(a.target, b * a.ts[0] + first * a.ts[1]);
        q = first < n && a.draft ? at<ELT>(a.draft, b * a.ds[0] + first * a.ds[1]) : nullptr;
        certain = first < n && !a.draft ? a.draft_tokens[b * a.drafts + first] : -1;
    }
    // weights of element v: x what is left of p over q, y p itself
    __device__ __forceinline__ double2 weights(int64_t v) const {
        const double pv = prob<ELT>(p, v);
        const double left = q ? pv - prob<ELT>(q, v) : v == certain ? pv - 1.0 : pv;
        return double2{left > 0 ? left : 0.0, pv > 0 ? pv : 0.0};
    }
};

// A thread's eight elements of a tile of kTile, from v on; those past `to` weigh nothing.
constexpr int kEach = 8, kTile = 256 * kEach;

// (rows begin where their strides put them: 16-byte loads at the elements' own alignment)
typedef uint32_t WordsOn4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t WordsOn2 __attribute__((ext_vector_type(4), aligned(2)));
template <int ELT>
struct Raw8 {  // eight elements as they lie in memory
    uint32_t w[ELT == ATK_F32 ? 8 : 4];
    __device__ __forceinline__ void load(const void *p, int64_t v) {
        if constexpr (ELT == ATK_F32) {
            const WordsOn4 a = *(const WordsOn4 *)((const float *)p + v), b = *(const WordsOn4 *)((const float *)p + v + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = a[e], w[4 + e] = b[e];
        } else {
            const WordsOn2 a = *(const WordsOn2 *)((const uint16_t *)p + v);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = a[e];
        }
    }
    __device__ __forceinline__ double value(int e) const {
        if constexpr (ELT == ATK_F32) return (double)__uint_as_float(w[e]);
        const uint32_t x = w[e / 2];
        if constexpr (ELT == ATK_BF16) return (double)__uint_as_float(e & 1 ? x & 0xffff0000u : x << 16);
        return (double)(float)__builtin_bit_cast(_Float16, (uint16_t)(e & 1 ? x >> 16 : x & 0xffffu));
    }
};

// w[e]: what is left of the target's probability over the draft's, or (of_target) that itself; all[e]: that itself
template <int ELT>
__device__ __forceinline__ void weights8(const VerifyRow<ELT> &row, int64_t v, int64_t to, double *left, double *all) {
    if (v + kEach <= to) {
        Raw8<ELT> p;
        p.load(row.p, v);
        if (row.q) {
            Raw8<ELT> q;
            q.load(row.q, v);
#pragma unroll
            for (int e = 0; e < kEach; ++e) left[e] = p.value(e) - q.value(e);
        } else {
#pragma unroll
            for (int e = 0; e < kEach; ++e) left[e] = v + e == row.certain ? p.value(e) - 1.0 : p.value(e);
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const double x = p.value(e);
            left[e] = left[e] > 0 ? left[e] : 0.0, all[e] = x > 0 ? x : 0.0;
        }
    } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            left[e] = all[e] = 0.0;
            if (v + e < to) {
                const double2 w = row.weights(v + e);
                left[e] = w.x, all[e] = w.y;
            }
        }
    }
}

__device__ __forceinline__ double wave_sum(double v) {
    for (int w = 1; w < 64; w <<= 1) v += __shfl_xor(v, w, 64);
    return v;
}

// Tiles of a workgroup: enough that a request's accepted drafts, a chain of three dependent reads, are not looked for too often (64 requests of 128256: 11.7 us with one tile, 10.0 with two).
constexpr int kMostTiles = 4;

template <int ELT>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyDev a) {
    __shared__ double2 waves[kMostTiles][4];
    const int64_t b = blockIdx.x / a.groups;
    const int group = (int)(blockIdx.x % a.groups), each = (a.tiles + a.groups - 1) / a.groups, lane = threadIdx.x & 63;
    const VerifyRow<ELT> row(a, b);
    double2 s[kMostTiles];
#pragma unroll
    for (int k = 0; k < kMostTiles; ++k) {
        s[k] = double2{0, 0};
        const int64_t v = ((int64_t)group * each + k) * kTile + threadIdx.x * kEach;
        if (k < each && v < a.vocab) {
            double left[kEach], all[kEach];
            weights8<ELT>(row, v, a.vocab, left, all);
#pragma unroll
            for (int e = 0; e < kEach; ++e) s[k].x += left[e], s[k].y += all[e];
        }
    }
#pragma unroll
    for (int k = 0; k < kMostTiles; ++k) {
        if (k >= each) break;
        s[k].x = wave_sum(s[k].x), s[k].y = wave_sum(s[k].y);
        if (lane == 0) waves[k][threadIdx.x >> 6] = s[k];
    }
    __syncthreads();
    const int k = threadIdx.x, tile = group * each + k;
    if (k < each && tile < a.tiles)
        a.sums[b * a.tiles + tile] = double2{(waves[k][0].x + waves[k][1].x) + (waves[k][2].x + waves[k][3].x), (waves[k][0].y + waves[k][1].y) + (waves[k][2].y + waves[k][3].y)};
    if (threadIdx.x == 0 && group == 0) a.accepted[b] = row.accepted;
}

// The first lane whose running sum of weights (from *run on) passes the goal, -1 if none, and *run is behind them all then; *before: a lane's running sum without its own;
// *last: the last lane with a weight, if there is one - where rounding lets no running sum pass, it is the one.
__device__ __forceinline__ int find64(double w, double goal, double *run, int *last, double *before) {
    const int lane = threadIdx.x & 63;
    double upto = w;
    for (int o = 1; o < 64; o <<= 1) {
        const double v = __shfl_up(upto, o, 64);
        if (lane >= o) upto += v;
    }
    *before = *run + (upto - w);
    const uint64_t some = __ballot(w > 0), passes = __ballot(w > 0 && *before + w > goal);
    if (some) *last = 63 - __builtin_clzll(some);
    *run += __shfl(upto, 63, 64);
    return passes ? __builtin_ctzll(passes) : -1;
}

// The element of a chunk of 64 * kEach from v0 on at which the running sum, `start` in front of it, passes the goal; where rounding lets none pass, the last one with a weight (-1: there
// is none).  By one wavefront.
constexpr int kChunk = 64 * kEach;
template <int ELT>
__device__ __forceinline__ int find_element(const VerifyRow<ELT> &row, int64_t v0, int64_t vocab, bool of_target, double goal, double start) {
    double w[kEach], t[kEach], sum = 0, run = start, before;
    weights8<ELT>(row, v0 + (threadIdx.x & 63) * kEach, vocab, w, t);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (of_target) w[e] = t[e];
        sum += w[e];
    }
    int last = -1;
    const int got = find64(sum, goal, &run, &last, &before);
    const int who = got >= 0 ? got : last;
    int at = -1;
    bool done = false;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (done || !(w[e] > 0)) continue;
        at = e;
        before += w[e];
        done = before > goal;
    }
    return who < 0 ? -1 : (int)v0 + who * kEach + __shfl(at, who, 64);
}

template <int ELT>
__device__ __forceinline__ void write_tokens(const VerifyDev &a, int64_t b, int accepted, int token) {
    for (int i = threadIdx.x & 63; i <= a.drafts; i += 64)
        a.tokens[b * (a.drafts + 1) + i] = i < accepted ? a.draft_tokens[b * a.drafts + i] : i == accepted ? token : -1;
}

// One wavefront a request: what is left to do is a chain of dependent steps, and four wavefronts that meet at barriers took 9 us where this takes 6.
template <int ELT>
__global__ __launch_bounds__(64) void verify_draw_kernel(const VerifyDev a) {
    const int lane = threadIdx.x;
    const int64_t b = blockIdx.x;
    const double2 *s = a.sums + b * a.tiles;
    const double r = (double)a.r[b];
    const double2 mine = lane < a.tiles ? s[lane] : double2{0, 0};
    const VerifyRow<ELT> row(a, b, a.accepted[b]);
    double left = mine.x, all = mine.y;
    for (int i = lane + 64; i < a.tiles; i += 64) left += s[i].x, all += s[i].y;
    left = wave_sum(left), all = wave_sum(all);
    const bool of_target = !(left > 0);  // nothing left (or sums that are no numbers): p itself
    const double goal = r * (of_target ? all : left);
    // the tile, ...
    int pick = -1, token = -1;
    double run = 0, start = 0, before;
    for (int i0 = 0; i0 < a.tiles; i0 += 64) {
        const double2 x = i0 == 0 ? mine : i0 + lane < a.tiles ? s[i0 + lane] : double2{0, 0};
        int last = -1;
        const int got = find64(of_target ? x.y : x.x, goal, &run, &last, &before);
        const int who = got >= 0 ? got : last;
        if (who >= 0) pick = i0 + who, start = __shfl(before, who, 64);
        if (got >= 0) break;
    }
    if (pick >= 0) {
        // ... the lane's eight elements of a quarter of it, and the one among them
        const int64_t v0 = (int64_t)pick * kTile;
        constexpr int kQuarter = 64 * kEach;
        double w[4][kEach], sum[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t v = v0 + k * kQuarter + lane * kEach;
            double t[kEach];
            weights8<ELT>(row, v, a.vocab, w[k], t);
            sum[k] = 0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                if (of_target) w[k][e] = t[e];
                sum[k] += w[k][e];
            }
        }
        run = start;
        bool found = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (found) continue;
            int last = -1;
            const int got = find64(sum[k], goal, &run, &last, &before);
            const int who = got >= 0 ? got : last;
            found = got >= 0;
            if (who < 0) continue;
            int at = -1;
            bool done = false;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                if (done || !(w[k][e] > 0)) continue;
                at = e;
                before += w[k][e];
                done = before > goal;
            }
            token = (int)(v0 + k * kQuarter) + who * kEach + __shfl(at, who, 64);
        }
    }
    write_tokens<ELT>(a, b, row.accepted, token);
}

// The whole request by one workgroup: its wavefronts have a sixteenth of the row each, then a chunk of the sixteenth that the goal lies in, then one has the chunk.
// (1024 threads leave 128 registers each: 84 words a lane are spilled to scratch, in all three types.)
constexpr int kRowBytes = 128 << 10;  // of a row at most
constexpr int kRowWaves = 16, kRowChunks = kRowBytes / 2 / (kRowWaves * kChunk);  // chunks of a sixteenth at most: eight, four in f32
static_assert(kRowChunks * kRowWaves * kChunk * 2 == kRowBytes && kRowChunks <= kRowWaves, "a wavefront for each chunk of a sixteenth");
template <int ELT>
__global__ __launch_bounds__(kRowWaves * 64) void verify_row_kernel(const VerifyDev a) {
    __shared__ double2 wave_sums[kRowWaves];
    __shared__ double chunk_sums[kRowChunks];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t b = blockIdx.x;
    const double r = (double)a.r[b];
    const VerifyRow<ELT> row(a, b);
    const int chunks = (int)((a.vocab + kRowWaves * kChunk - 1) / (kRowWaves * kChunk));  // of a wavefront
    double2 s = {0, 0};
    const int64_t first = (int64_t)wave * chunks * kChunk, end = min(a.vocab, first + (int64_t)chunks * kChunk);
    int64_t v0 = first;
    if (row.q) {  // eight 16-byte loads (f32: sixteen) on their way at once
        for (; v0 + 4 * kChunk <= end; v0 += 4 * kChunk) {
            Raw8<ELT> p[4], q[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) p[c].load(row.p, v0 + c * kChunk + lane * kEach), q[c].load(row.q, v0 + c * kChunk + lane * kEach);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const double x = p[c].value(e), y = x - q[c].value(e);
                    s.x += y > 0 ? y : 0.0, s.y += x > 0 ? x : 0.0;
                }
        }
    }
    for (; v0 < end; v0 += kChunk) {
        double left[kEach], all[kEach];
        weights8<ELT>(row, v0 + lane * kEach, end, left, all);
#pragma unroll
        for (int e = 0; e < kEach; ++e) s.x += left[e], s.y += all[e];
    }
    s.x = wave_sum(s.x), s.y = wave_sum(s.y);
    if (lane == 0) wave_sums[wave] = s;
    __syncthreads();
    const double2 mine = lane < kRowWaves ? wave_sums[lane] : double2{0, 0};
    const double left = wave_sum(mine.x), all = wave_sum(mine.y);
    const bool of_target = !(left > 0);
    const double goal = r * (of_target ? all : left);
    double run = 0, before;
    int last = -1;
    const int got = find64(of_target ? mine.y : mine.x, goal, &run, &last, &before);
    const int pick = got >= 0 ? got : last;
    int token = -1;
    if (pick >= 0) {
        run = __shfl(before, pick, 64);
        if (wave < chunks) {
            double w[kEach], t[kEach], sum = 0;
            weights8<ELT>(row, ((int64_t)pick * chunks + wave) * kChunk + lane * kEach, a.vocab, w, t);
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum += of_target ? t[e] : w[e];
            sum = wave_sum(sum);
            if (lane == 0) chunk_sums[wave] = sum;
        }
        __syncthreads();
        if (wave != 0) return;
        last = -1;
        const int found = find64(lane < chunks ? chunk_sums[lane] : 0.0, goal, &run, &last, &before);
        const int which = found >= 0 ? found : last;
        if (which >= 0) token = find_element<ELT>(row, ((int64_t)pick * chunks + which) * kChunk, a.vocab, of_target, goal, __shfl(before, which, 64));
    }
    if (wave != 0) return;
    write_tokens<ELT>(a, b, row.accepted, token);
    if (lane == 0) a.accepted[b] = row.accepted;
}

static int64_t verify_tiles(int64_t vocab) { return (vocab + kTile - 1) / kTile; }
// Workgroups of a request: a tile each, or as many tiles as keep all requests at about eight workgroups a CU.
static int64_t verify_groups(int64_t batch, int64_t vocab) {
    const int64_t tiles = verify_tiles(vocab), each = (batch * tiles + 8 * kNumCU - 1) / (8 * kNumCU);
    return (tiles + std::min<int64_t>(each, kMostTiles) - 1) / std::min<int64_t>(each, kMostTiles);
}

// Rows of up to 128 KB by one workgroup each: 9.1 us -> 6.9 for one request of 4000 f32, 13.1 -> 11.2 for 64 of 32000, 16.0 -> 11.3 for 128 of 32000 bf16; one of 128256 bf16 would
// take 16 us so and takes 8.4 in two launches, 64 of them 25 and 20.
static bool verify_by_row(int64_t vocab, int elt) { return vocab * (elt == ATK_F32 ? 4 : 2) <= kRowBytes; }
static bool verify_fits(int64_t batch, int64_t vocab, int elt) { return verify_by_row(vocab, elt) ? launches(batch, kRowWaves * 64) : launches(batch * verify_groups(batch, vocab), 256); }

template <int ELT>
static hipError_t launch_verify(const VerifyDev &a, int64_t batch, hipStream_t s) {
    if (verify_by_row(a.vocab, ELT)) {
        hipLaunchKernelGGL((verify_row_kernel<ELT>), dim3((uint32_t)batch), dim3(kRowWaves * 64), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((verify_sums_kernel<ELT>), dim3((uint32_t)(batch * a.groups)), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_draw_kernel<ELT>), dim3((uint32_t)batch), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace atk

using namespace atk;

extern "C" {

int64_t atk_verify_workspace_bytes(int64_t batch, int64_t drafts, int64_t vocab) {
    if (batch < 1 || batch > (1 << 24) || drafts < 0 || drafts > (1 << 20) || vocab < 1 || vocab >= (INT64_C(1) << 30)) return ATK_ERR_ARGS;
    if (!verify_fits(batch, vocab, ATK_F32) && !verify_fits(batch, vocab, ATK_BF16)) return ATK_ERR_ARGS;
    return batch * verify_tiles(vocab) * (int64_t)sizeof(double2);
}

int atk_verify_drafts(const void *target_probs, const int64_t target_stride[2], const void *draft_probs, const int64_t draft_stride[2],
                      const int32_t *draft_tokens, const float *accept_random, const float *final_random, const int32_t *n_drafts, int64_t batch,
                      int64_t drafts, int64_t vocab, int dtype, int32_t *accepted, int32_t *tokens, void *work, int64_t work_bytes, void *stream) {
    const int64_t need = atk_verify_workspace_bytes(batch, drafts, vocab);
    if (need < 0) return (int)need;
    if (dtype != ATK_F32 && dtype != ATK_BF16 && dtype != ATK_F16) return ATK_ERR_DTYPE;
    if (!verify_fits(batch, vocab, dtype)) return ATK_ERR_ARGS;
    if (!target_probs || !target_stride || (draft_probs && !draft_stride) || !final_random || !accepted || !tokens || !work) return ATK_ERR_NULL_PTR;
    if (drafts > 0 && (!draft_tokens || !accept_random)) return ATK_ERR_NULL_PTR;
    const int es = dtype == ATK_F32 ? 4 : 2;
    if (((uintptr_t)target_probs | (uintptr_t)draft_probs) & (es - 1)) return ATK_ERR_ALIGN;
    if (((uintptr_t)draft_tokens | (uintptr_t)accept_random | (uintptr_t)final_random | (uintptr_t)n_drafts | (uintptr_t)accepted | (uintptr_t)tokens) & 3) return ATK_ERR_ALIGN;
    if ((uintptr_t)work & 15) return ATK_ERR_ALIGN;
    if (work_bytes < need) return ATK_ERR_WORKSPACE;
    VerifyDev a;
    a.target = target_probs, a.draft = drafts > 0 ? draft_probs : nullptr, a.draft_tokens = draft_tokens, a.n_drafts = n_drafts;
    a.u = accept_random, a.r = final_random, a.accepted = accepted, a.tokens = tokens, a.sums = (double2 *)work;
    for (int i = 0; i < 2; ++i) {
        a.ts[i] = target_stride[i], a.ds[i] = draft_probs ? draft_stride[i] : 0;
        if (a.ts[i] < 0 || a.ds[i] < 0) return ATK_ERR_ARGS;
    }
    a.vocab = vocab, a.drafts = (int)drafts, a.tiles = (int)verify_tiles(vocab), a.groups = (int)verify_groups(batch, vocab);
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t e = dtype == ATK_F32 ? launch_verify<ATK_F32>(a, batch, s) : dtype == ATK_BF16 ? launch_verify<ATK_BF16>(a, batch, s) : launch_verify<ATK_F16>(a, batch, s);
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // extern "C"
