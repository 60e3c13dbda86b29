// Joins the ranges of keys of the rows of an attention (see atk_attention_kernel.h).
#pragma once

#include "atk_attention_kernel.h"

namespace atk {

// One wavefront a row: LPR lanes have four elements each, 64 / LPR parts at a time.
template <int ELT, int LPR>
__global__ __launch_bounds__(256) void attn_join_kernel(const AttnDev a) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.batch * a.tokens * a.heads) return;
    const float2 *ml = a.parts_ml + row * a.parts;
    float m = kNoMax;
    for (int p = lane; p < a.parts; p += 64) m = fmaxf(m, ml[p].x);
    for (int w = 1; w < 64; w <<= 1) m = fmaxf(m, __shfl_xor(m, w, 64));
    float l = 0.0f;
    for (int p = lane; p < a.parts; p += 64) {
        const float2 x = ml[p];
        l += x.y * (x.x == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((x.x - m) * a.scale2));
    }
    for (int w = 1; w < 64; w <<= 1) l += __shfl_xor(l, w, 64);
    const int d = (lane % LPR) * 4;
    f32x4 o = {0, 0, 0, 0};
    if (d < a.dim) {
        // eight parts in flight: one after the other their loads were nearly all of the time (64 samples of 17 parts each: 9.9 us against 7.5; of the nine that the plan makes for them by now, 5.0)
        constexpr int kStep = 64 / LPR;
        const float *from = a.parts_o + row * a.parts * a.dim + d;
        for (int p0 = lane / LPR; p0 < a.parts; p0 += 8 * kStep) {
            float2 x[8];
            f32x4 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int p = min(p0 + j * kStep, a.parts - 1);
                x[j] = ml[p];
                v[j] = *(const f32x4 *)(from + (int64_t)p * a.dim);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (p0 + j * kStep >= a.parts) continue;
                const float f = x[j].x == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((x[j].x - m) * a.scale2);
                o += f * v[j];
            }
        }
    }
#pragma unroll
    for (int w = LPR; w < 64; w <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], w, 64);
    const int head = (int)(row % a.heads);
    const int64_t bt = row / a.heads;
    const int64_t b = bt / a.tokens, t = bt % a.tokens;
    if (l == 0.0f) o = f32x4{0, 0, 0, 0};  // no key, or scores of -inf alone, whose values do not count even if they are NaN
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    if (lane < LPR && d < a.dim) {
        store_out<ELT>((char *)a.out + (b * a.os[0] + t * a.os[1] + head * a.os[2] + d) * AttnElt<ELT>::kBytes, o * f);
    }
    if (a.lse && lane == 0) a.lse[row] = row_lse<ELT>(a, m, l);
}

template <int ELT>
static hipError_t launch_join(const AttnDev &a, int dp, hipStream_t stream) {
    const int64_t rows = (int64_t)a.batch * a.tokens * a.heads;
    const dim3 grid((uint32_t)((rows + 3) / 4)), threads(256);
    if (dp == 64)
        hipLaunchKernelGGL((attn_join_kernel<ELT, 16>), grid, threads, 0, stream, a);
    else if (dp == 128)
        hipLaunchKernelGGL((attn_join_kernel<ELT, 32>), grid, threads, 0, stream, a);
    else
        hipLaunchKernelGGL((attn_join_kernel<ELT, 64>), grid, threads, 0, stream, a);
    return hipGetLastError();
}

}  // namespace atk
