// verify_drafts: accepted drafts, and one token drawn from what is left of the target's probabilities (include/atk_decode.h).
//
// Only one row of the target's probabilities is needed whole, and after a rejection one of the draft's: those of the first rejected
// token.  verify_sums_kernel finds it (a few gathers, done again by every workgroup of the request), and sums the weights of a part of that row;
// verify_draw_kernel finds the part, then the element, at which the running sum passes the target.  Sums are f64: an index is what comes out, and the
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

    __device__ __forceinline__ VerifyRow(const VerifyDev &a, int64_t b) {
        const int lane = threadIdx.x & 63;
        const int n = a.n_drafts ? min(max(a.n_drafts[b], 0), a.drafts) : a.drafts;
        int first = n;
        for (int i0 = 0; i0 < n && first == n; i0 += 64) {
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

__device__ __forceinline__ double wave_sum(double v) {
    for (int w = 1; w < 64; w <<= 1) v += __shfl_xor(v, w, 64);
    return v;
}

template <int ELT>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyDev a) {
    __shared__ double2 waves[4];
    const int64_t b = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const VerifyRow<ELT> row(a, b);
    const int64_t from = part * a.part, to = min(a.vocab, from + a.part);
    double2 s = {0, 0};
    for (int64_t v = from + threadIdx.x; v < to; v += 256) {
        const double2 w = row.weights(v);
        s.x += w.x, s.y += w.y;
    }
    s.x = wave_sum(s.x), s.y = wave_sum(s.y);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[blockIdx.x] = double2{(waves[0].x + waves[1].x) + (waves[2].x + waves[3].x), (waves[0].y + waves[1].y) + (waves[2].y + waves[3].y)};
}

template <int ELT>
__global__ __launch_bounds__(256) void verify_draw_kernel(const VerifyDev a) {
    __shared__ double before[256];
    __shared__ int found, fallback, chosen;
    __shared__ double base;
    const int64_t b = blockIdx.x;
    const VerifyRow<ELT> row(a, b);
    bool of_target = false;
    if (threadIdx.x == 0) {
        const double2 *s = a.sums + b * a.parts;
        double left = 0, all = 0;
        for (int i = 0; i < a.parts; ++i) left += s[i].x, all += s[i].y;
        of_target = !(left > 0);  // nothing left (or sums that are no numbers): p itself
        const double goal = (double)a.r[b] * (of_target ? all : left);
        // the first part whose running sum passes the goal; rounding may leave none: the last one with a weight
        double run = 0, start = 0;
        int pick = -1;
        for (int i = 0; i < a.parts; ++i) {
            const double w = of_target ? s[i].y : s[i].x;
            if (!(w > 0)) continue;
            pick = i, start = run;
            run += w;
            if (run > goal) break;
        }
        chosen = pick | (of_target ? 1 << 30 : 0);
        if (pick < 0) chosen = -1;
        base = start;
        before[0] = goal;
        found = 256, fallback = -1;
    }
    __syncthreads();
    const int pick = chosen;
    const double goal = before[0], start = base;
    __syncthreads();
    int token = -1;
    if (pick >= 0) {
        of_target = pick >> 30;
        const int64_t from = (pick & ((1 << 30) - 1)) * a.part, to = min(a.vocab, from + a.part);
        const int64_t each = (to - from + 255) / 256;
        const int64_t mine = min(to, from + threadIdx.x * each), end = min(to, mine + each);
        double sum = 0;
        for (int64_t v = mine; v < end; ++v) {
            const double2 w = row.weights(v);
            sum += of_target ? w.y : w.x;
        }
        // running sums in front of each thread's elements, in order
        before[threadIdx.x] = sum;
        __syncthreads();
        if (threadIdx.x < 64) {
            double t[4], run = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = before[threadIdx.x * 4 + j], run += t[j];
            double upto = run;
            for (int w = 1; w < 64; w <<= 1) {
                const double o = __shfl_up(upto, w, 64);
                if ((int)threadIdx.x >= w) upto += o;
            }
            double x = start + (upto - run);
#pragma unroll
            for (int j = 0; j < 4; ++j) before[threadIdx.x * 4 + j] = x, x += t[j];
        }
        __syncthreads();
        const double x = before[threadIdx.x];
        if (sum > 0) {
            atomicMax(&fallback, (int)threadIdx.x);
            if (x + sum > goal) atomicMin(&found, (int)threadIdx.x);
        }
        __syncthreads();
        const int who = found < 256 ? found : fallback;
        if ((int)threadIdx.x == who) {
            double run = x;
            for (int64_t v = mine; v < end; ++v) {
                const double2 w2 = row.weights(v);
                const double w = of_target ? w2.y : w2.x;
                if (!(w > 0)) continue;
                token = (int)v;
                run += w;
                if (run > goal) break;
            }
            chosen = token;
        }
        __syncthreads();
        token = chosen;
    }
    for (int i = threadIdx.x; i <= a.drafts; i += 256)
        a.tokens[b * (a.drafts + 1) + i] = i < row.accepted ? a.draft_tokens[b * a.drafts + i] : i == row.accepted ? token : -1;
    if (threadIdx.x == 0) a.accepted[b] = row.accepted;
}

// Parts of a row: enough for the chip's workgroups, of 2048 elements at least.
static int64_t verify_parts(int64_t batch, int64_t vocab) {
    const int64_t wanted = std::max<int64_t>(1, 4 * kNumCU / batch);
    return std::max<int64_t>(1, std::min(wanted, (vocab + 2047) / 2048));
}

template <int ELT>
static hipError_t launch_verify(const VerifyDev &a, int64_t batch, hipStream_t s) {
    hipLaunchKernelGGL((verify_sums_kernel<ELT>), dim3((uint32_t)(batch * a.parts)), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_draw_kernel<ELT>), dim3((uint32_t)batch), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace atk

using namespace atk;

extern "C" {

int64_t atk_verify_workspace_bytes(int64_t batch, int64_t drafts, int64_t vocab) {
    if (batch < 1 || batch > (1 << 24) || drafts < 0 || drafts > (1 << 20) || vocab < 1 || vocab >= (INT64_C(1) << 30)) return ATK_ERR_ARGS;
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
    a.part = (vocab + a.parts - 1) / a.parts;
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t e = dtype == ATK_F32 ? launch_verify<ATK_F32>(a, batch, s) : dtype == ATK_BF16 ? launch_verify<ATK_BF16>(a, batch, s) : launch_verify<ATK_F16>(a, batch, s);
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // extern "C"
