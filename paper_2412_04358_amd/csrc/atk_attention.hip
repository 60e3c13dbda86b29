// shared_prefix_attention: checks, launch plan, and the kernel that joins the ranges of keys (see atk_attention_kernel.h).
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
        for (int p = lane / LPR; p < a.parts; p += 64 / LPR) {
            const float2 x = ml[p];
            if (x.y == 0.0f) continue;  // no visible key in it
            const float f = x.x == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((x.x - m) * a.scale2);
            o += f * *(const f32x4 *)(a.parts_o + (row * a.parts + p) * a.dim + d);
        }
    }
#pragma unroll
    for (int w = LPR; w < 64; w <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], w, 64);
    const int head = (int)(row % a.heads);
    const int64_t bt = row / a.heads;
    const int64_t b = bt / a.tokens, t = bt % a.tokens;
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    if (lane < LPR && d < a.dim) {
        char *out = (char *)a.out + (b * a.os[0] + t * a.os[1] + head * a.os[2] + d) * AttnElt<ELT>::kBytes;
        if constexpr (ELT == ATK_F32)
            *(f32x4 *)out = o * f;
        else
            *(u32x2 *)out = u32x2{AttnElt<ELT>::pack(o[0] * f, o[1] * f), AttnElt<ELT>::pack(o[2] * f, o[3] * f)};
    }
    if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? kNoMax : (m == kNoMax ? l : fmaf(m, a.scale, (log2f(l) - AttnElt<ELT>::kBias) * 0.6931471805599453f));
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

struct AttnPlan {
    int dp, rt, waves, prefix_splits, prefix_blocks, prefix_keys, own_splits, own_blocks;
    int64_t rows, parts, o_bytes, bytes;
};

static int64_t attn_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }

static int check_attention(const atk_attention_args *p, bool pointers) {
    if (!p) return ATK_ERR_NULL_PTR;
    if (p->dtype != ATK_F32 && p->dtype != ATK_BF16 && p->dtype != ATK_F16) return ATK_ERR_DTYPE;
    const int es = p->dtype == ATK_F32 ? 4 : 2, piece = 16 / es;
    const int64_t most = INT64_C(1) << 30;
    if (p->batch < 1 || p->tokens < 1 || p->heads < 1 || p->kv_heads < 1 || p->dim < 1 || p->page_size < 1 || p->n_pages < 1 || p->rows < 1 || p->row_pages < 1)
        return ATK_ERR_ARGS;
    if (p->batch > most || p->tokens > most || p->heads > most || p->page_size > most || p->n_pages > most || p->rows > most || p->row_pages > most) return ATK_ERR_ARGS;
    if (p->heads % p->kv_heads || p->batch * p->tokens > most || p->batch * p->tokens * p->heads > most) return ATK_ERR_ARGS;
    if (p->row_pages * p->page_size > most || p->prefix_len < 0 || p->prefix_len > p->row_pages * p->page_size) return ATK_ERR_ARGS;
    if (!p->seqs && p->batch > p->rows) return ATK_ERR_ARGS;
    if (p->table_stride < p->row_pages) return ATK_ERR_ARGS;
    if (!(p->scale > 0) || p->scale > 1e30) return ATK_ERR_ARGS;
    if (p->dim > 256 || p->dim % piece) return ATK_ERR_UNSUPPORTED;
    for (int i = 0; i < 3; ++i) {
        if (p->q_stride[i] < 0 || p->out_stride[i] < 0 || p->k_stride[i] < 0 || p->v_stride[i] < 0) return ATK_ERR_ARGS;
        if (p->q_stride[i] % piece || p->out_stride[i] % piece || p->k_stride[i] % piece || p->v_stride[i] % piece) return ATK_ERR_ALIGN;
    }
    if (pointers) {
        if (!p->q || !p->k || !p->v || !p->out || !p->page_table || !p->lens) return ATK_ERR_NULL_PTR;
        if (((uintptr_t)p->q | (uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->out) & 15) return ATK_ERR_ALIGN;
        if (((uintptr_t)p->page_table | (uintptr_t)p->lens | (uintptr_t)p->seqs | (uintptr_t)p->lse | (uintptr_t)p->status) & 3) return ATK_ERR_ALIGN;
    }
    return ATK_OK;
}

static int plan_attention(const atk_attention_args *p, AttnPlan *pl) {
    const int group = (int)(p->heads / p->kv_heads);
    pl->dp = p->dim <= 64 ? 64 : p->dim <= 128 ? 128 : 256;
    const int64_t rows = p->batch * p->tokens * group, own_rows = p->tokens * group;
    // how the shared keys meet the rows: up to two 16-row tiles in every wavefront, or 32 rows a wavefront and keys by way of LDS
    pl->rt = rows <= 16 || p->prefix_len == 0 ? 1 : 2, pl->waves = kAttnWaves;
    int64_t block = 16 * pl->rt, step = kAttnWaves * kTileKeys;
    int64_t wanted = 2 * kNumCU;
    const int64_t small = INT64_C(1) << 28;  // (four tokens' offsets are 32 bits)
    if (rows > 32 && p->dtype != ATK_F32 && p->prefix_len > 0 && p->page_size % 4 == 0 && p->k_stride[1] < small && p->v_stride[1] < small) {
        pl->rt = 0, pl->waves = rows <= 128 ? 4 : attn_max_waves(pl->dp);
        block = 32 * pl->waves, step = kBlockKeys;
        wanted = pl->waves == 8 ? kNumCU : 2 * kNumCU;
    } else if (pl->rt > attn_max_rt(p->dtype, pl->dp)) {
        pl->rt = 1, block = 16;
    }
    pl->prefix_blocks = (int)attn_ceil(rows, block);
    const int64_t base = pl->prefix_blocks * p->kv_heads;
    pl->prefix_splits = 0, pl->prefix_keys = 0;
    if (p->prefix_len > 0) {
        const int64_t steps = attn_ceil(p->prefix_len, step);
        const int64_t splits = std::min(steps, std::max<int64_t>(1, wanted / base));
        pl->prefix_keys = (int)(attn_ceil(steps, splits) * step);
        pl->prefix_splits = (int)attn_ceil(p->prefix_len, pl->prefix_keys);
    }
    // a sequence's own keys: as many as its row could hold, the device knows how many there are
    const int64_t own = p->row_pages * p->page_size - p->prefix_len;
    pl->own_blocks = (int)attn_ceil(own_rows, 16);
    const int64_t own_base = p->batch * p->kv_heads * pl->own_blocks;
    pl->own_splits = own > 0 ? (int)std::min(attn_ceil(own, kAttnWaves * kTileKeys), std::max<int64_t>(1, 2 * kNumCU / own_base)) : 0;
    pl->rows = p->batch * p->tokens * p->heads;
    pl->parts = pl->prefix_splits + pl->own_splits;
    pl->o_bytes = pl->rows * pl->parts * p->dim * 4;
    pl->bytes = pl->o_bytes + pl->rows * pl->parts * 8;
    const int64_t most = INT64_C(1) << 30;  // workgroups
    return base * std::max(1, pl->prefix_splits) < most && own_base * std::max(1, pl->own_splits) < most ? ATK_OK : ATK_ERR_ARGS;
}

}  // namespace atk

using namespace atk;

extern "C" {

int64_t atk_attention_workspace_bytes(const atk_attention_args *p) {
    int rc = check_attention(p, false);
    AttnPlan pl;
    if (rc == ATK_OK) rc = plan_attention(p, &pl);
    return rc == ATK_OK ? pl.bytes : rc;
}

int atk_shared_prefix_attention(const atk_attention_args *p, void *work, int64_t work_bytes, void *stream) {
    int rc = check_attention(p, true);
    AttnPlan pl;
    if (rc == ATK_OK) rc = plan_attention(p, &pl);
    if (rc != ATK_OK) return rc;
    if (!work) return ATK_ERR_NULL_PTR;
    if ((uintptr_t)work & 15) return ATK_ERR_ALIGN;
    if (work_bytes < pl.bytes) return ATK_ERR_WORKSPACE;
    AttnDev a;
    a.q = p->q, a.k = p->k, a.v = p->v, a.out = p->out, a.lse = p->lse;
    a.table = p->page_table, a.lens = p->lens, a.seqs = p->seqs, a.status = p->status;
    a.parts_o = (float *)work, a.parts_ml = (float2 *)((char *)work + pl.o_bytes);
    a.table_stride = p->table_stride;
    for (int i = 0; i < 3; ++i) a.qs[i] = p->q_stride[i], a.os[i] = p->out_stride[i], a.ks[i] = p->k_stride[i], a.vs[i] = p->v_stride[i];
    a.batch = (int)p->batch, a.tokens = (int)p->tokens, a.heads = (int)p->heads, a.kv_heads = (int)p->kv_heads;
    a.group = a.heads / a.kv_heads, a.dim = (int)p->dim;
    a.rows = (int)p->rows, a.row_pages = (int)p->row_pages, a.n_pages = (int)p->n_pages;
    a.prefix_len = (int)p->prefix_len;
    a.prefix_splits = pl.prefix_splits, a.prefix_blocks = pl.prefix_blocks, a.prefix_keys = pl.prefix_keys;
    a.own_splits = pl.own_splits, a.own_blocks = pl.own_blocks;
    a.n_prefix = pl.prefix_splits * pl.prefix_blocks * a.kv_heads;
    a.prefix_grid = (a.n_prefix + 7) / 8 * 8;
    a.n_own = a.batch * a.kv_heads * pl.own_blocks * pl.own_splits;
    a.parts = (int)pl.parts;
    a.page.set((uint32_t)p->page_size);
    a.scale = (float)p->scale;
    a.scale2 = (float)(p->scale * 1.4426950408889634);
    hipStream_t s = (hipStream_t)stream;
    hipError_t e = p->dtype == ATK_F32    ? launch_attn_f32(a, pl.dp, pl.rt, pl.waves, s)
                   : p->dtype == ATK_BF16 ? launch_attn_bf16(a, pl.dp, pl.rt, pl.waves, s)
                                          : launch_attn_f16(a, pl.dp, pl.rt, pl.waves, s);
    if (e == hipSuccess)
        e = p->dtype == ATK_F32    ? launch_join<ATK_F32>(a, pl.dp, s)
            : p->dtype == ATK_BF16 ? launch_join<ATK_BF16>(a, pl.dp, s)
                                   : launch_join<ATK_F16>(a, pl.dp, s);
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // extern "C"
