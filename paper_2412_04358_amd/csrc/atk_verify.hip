// verify_drafts: accepted drafts, and one token drawn from what is left of the target's probabilities (include/atk_decode.h).
//
// Only one row of the target's probabilities is needed whole, and after a rejection one of the draft's: those of the first rejected
// token.  verify_sums_kernel finds it (a few gathers, done again by every workgroup of the request), and sums the weights of a part of that row;
// verify_draw_kernel finds the part, then the thread's eight elements, then the element at which the running sum passes the goal.  Sums are f64: an index is what comes out, and the
// running sum of 10^5 f32 would be off by more than the weights.
#include "atk_decode_common.h"

namespace atk {

struct VerifyDev {
    const void *target, *draft;
    const int32_t *draft_tokens, *n_drafts;
    const float *u, *r;
    int32_t *accepted, *tokens;
    double2 *sums;  // [request][part]: residual weights, target's weights
    int64_t ts[2], ds[2];
    int64_t vocab, part;
    int drafts, parts;
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
__device__ __forceinline__ void probs8(const void *p, int64_t v, double *out) {
    if constexpr (ELT == ATK_F32) {
        const WordsOn4 a = *(const WordsOn4 *)((const float *)p + v), b = *(const WordsOn4 *)((const float *)p + v + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = (double)__uint_as_float(a[e]), out[4 + e] = (double)__uint_as_float(b[e]);
    } else {
        const WordsOn2 a = *(const WordsOn2 *)((const uint16_t *)p + v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t w = a[e];
            if constexpr (ELT == ATK_BF16) {
                out[2 * e] = (double)__uint_as_float(w << 16), out[2 * e + 1] = (double)__uint_as_float(w & 0xffff0000u);
            } else {
                out[2 * e] = (double)(float)__builtin_bit_cast(_Float16, (uint16_t)(w & 0xffffu));
                out[2 * e + 1] = (double)(float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
            }
        }
    }
}

// w[e]: what is left of the target's probability over the draft's, or (of_target) that itself; all[e]: that itself
template <int ELT>
__device__ __forceinline__ void weights8(const VerifyRow<ELT> &row, int64_t v, int64_t to, double *left, double *all) {
    if (v + kEach <= to) {
        probs8<ELT>(row.p, v, all);
        if (row.q) {
            probs8<ELT>(row.q, v, left);
#pragma unroll
            for (int e = 0; e < kEach; ++e) left[e] = all[e] - left[e];
        } else {
#pragma unroll
            for (int e = 0; e < kEach; ++e) left[e] = v + e == row.certain ? all[e] - 1.0 : all[e];
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) left[e] = left[e] > 0 ? left[e] : 0.0, all[e] = all[e] > 0 ? all[e] : 0.0;
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

__device__ __forceinline__ void sum256(double *a, double *b) {
    __shared__ double2 waves[4];
    *a = wave_sum(*a), *b = wave_sum(*b);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = double2{*a, *b};
    __syncthreads();
    *a = (waves[0].x + waves[1].x) + (waves[2].x + waves[3].x), *b = (waves[0].y + waves[1].y) + (waves[2].y + waves[3].y);
}

template <int ELT>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyDev a) {
    const int64_t b = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const VerifyRow<ELT> row(a, b);
    const int64_t from = part * a.part, to = min(a.vocab, from + a.part);
    double2 s = {0, 0};
    for (int64_t v = from + threadIdx.x * kEach; v < to; v += kTile) {
        double left[kEach], all[kEach];
        weights8<ELT>(row, v, to, left, all);
#pragma unroll
        for (int e = 0; e < kEach; ++e) s.x += left[e], s.y += all[e];
    }
    sum256(&s.x, &s.y);
    if (threadIdx.x == 0 && part == 0) a.accepted[b] = row.accepted;
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
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

// One wavefront a request: what is left to do is a chain of dependent steps, and four wavefronts that meet at barriers took 9 us where this takes 6.
template <int ELT>
__global__ __launch_bounds__(64) void verify_draw_kernel(const VerifyDev a) {
    const int lane = threadIdx.x;
    const int64_t b = blockIdx.x;
    const double2 *s = a.sums + b * a.parts;
    const double r = (double)a.r[b];
    const double2 mine = lane < a.parts ? s[lane] : double2{0, 0};
    const VerifyRow<ELT> row(a, b, a.accepted[b]);
    double left = mine.x, all = mine.y;
    for (int i = lane + 64; i < a.parts; i += 64) left += s[i].x, all += s[i].y;
    left = wave_sum(left), all = wave_sum(all);
    const bool of_target = !(left > 0);  // nothing left (or sums that are no numbers): p itself
    const double goal = r * (of_target ? all : left);
    // the part, ...
    int pick = -1, token = -1;
    double run = 0, start = 0, before;
    for (int i0 = 0; i0 < a.parts; i0 += 64) {
        const double2 x = i0 == 0 ? mine : i0 + lane < a.parts ? s[i0 + lane] : double2{0, 0};
        int last = -1;
        const int got = find64(of_target ? x.y : x.x, goal, &run, &last, &before);
        const int who = got >= 0 ? got : last;
        if (who >= 0) pick = i0 + who, start = __shfl(before, who, 64);
        if (got >= 0) break;
    }
    if (pick >= 0) {
        // ... the lane's eight elements of a quarter of a tile, and the one among them
        const int64_t from = (int64_t)pick * a.part, to = min(a.vocab, from + a.part);
        constexpr int kQuarter = 64 * kEach;
        run = start;
        bool found = false;
        for (int64_t v0 = from; v0 < to && !found; v0 += kTile) {
            double w[4][kEach], sum[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t v = v0 + k * kQuarter + lane * kEach;
                double t[kEach];
                weights8<ELT>(row, v, to, w[k], t);
                sum[k] = 0;
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    if (of_target) w[k][e] = t[e];
                    sum[k] += w[k][e];
                }
            }
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
    }
    for (int i = lane; i <= a.drafts; i += 64)
        a.tokens[b * (a.drafts + 1) + i] = i < row.accepted ? a.draft_tokens[b * a.drafts + i] : i == row.accepted ? token : -1;
}

// Elements of a part: a tile, or as many tiles as keep the parts of all requests at about eight workgroups a CU.
static int64_t verify_part(int64_t batch, int64_t vocab) {
    const int64_t tiles = (vocab + kTile - 1) / kTile, each = batch * tiles / (8 * kNumCU);
    return kTile * std::max<int64_t>(1, std::min<int64_t>(4, each));
}
static int64_t verify_parts(int64_t batch, int64_t vocab) {
    const int64_t part = verify_part(batch, vocab);
    return (vocab + part - 1) / part;
}

template <int ELT>
static hipError_t launch_verify(const VerifyDev &a, int64_t batch, hipStream_t s) {
    hipLaunchKernelGGL((verify_sums_kernel<ELT>), dim3((uint32_t)(batch * a.parts)), dim3(256), 0, s, a);
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
    if (batch * verify_parts(batch, vocab) >= (INT64_C(1) << 31)) return ATK_ERR_ARGS;  // workgroups
    return batch * verify_parts(batch, vocab) * (int64_t)sizeof(double2);
}

int atk_verify_drafts(const void *target_probs, const int64_t target_stride[2], const void *draft_probs, const int64_t draft_stride[2],
                      const int32_t *draft_tokens, const float *accept_random, const float *final_random, const int32_t *n_drafts, int64_t batch,
                      int64_t drafts, int64_t vocab, int dtype, int32_t *accepted, int32_t *tokens, void *work, int64_t work_bytes, void *stream) {
    const int64_t need = atk_verify_workspace_bytes(batch, drafts, vocab);
    if (need < 0) return (int)need;
    if (dtype != ATK_F32 && dtype != ATK_BF16 && dtype != ATK_F16) return ATK_ERR_DTYPE;
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
    a.vocab = vocab, a.drafts = (int)drafts, a.parts = (int)verify_parts(batch, vocab);
    a.part = verify_part(batch, vocab);
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t e = dtype == ATK_F32 ? launch_verify<ATK_F32>(a, batch, s) : dtype == ATK_BF16 ? launch_verify<ATK_BF16>(a, batch, s) : launch_verify<ATK_F16>(a, batch, s);
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // extern "C"
