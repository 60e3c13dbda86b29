// shared_prefix_attention: checks, launch plan, and the kernel that joins the ranges of keys (see atk_attention_kernel.h).
#include <cfloat>

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

static int64_t attn_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The plan goes by what the rows of the table could hold, as the host does not know the lengths: a table much wider than its sequences is cut for keys that are not there (two sequences of
// 230 keys: 8 us, under a table of 32768 18; 12 in f32 of 2240 33 and 40; 64 of 8576 and 24 of 5580 as long as before).
struct AttnPlan {
    int dp, rt, waves, own_from, prefix_splits, prefix_blocks, prefix_keys, own_splits, own_blocks;
    bool around;
    int64_t rows, parts, o_bytes, bytes;
};

// Keys of a sequence (by its row's pages) up to which a workgroup takes them all, shared ones and own, in one launch without parts.  Heads of 128: 8 sequences of 460 keys 14.3 us against
// 16.5 with shared keys apart, of 700 18.4 against 16.6; workgroups that fill the chip twice: 64 sequences of 700 22.5 against 26.9, of 1000 28.2 against 28.4; f32: 4 sequences of
// 120 10.4 against 14.3, of 240 15.3 against 14.4.
static int64_t attn_together(int dtype, int64_t groups) { return dtype == ATK_F32 ? 192 : groups >= 2 * kNumCU ? 896 : 512; }
// Own keys past the caches from more bytes on than the Infinity Cache holds (128 samples on 65536 + 1125 keys: 280 us -> 269; with less, 12 sequences in f32: 33 us -> 37).
constexpr int64_t kCacheBytes = INT64_C(256) << 20;

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
    if (!(p->scale >= FLT_MIN) || p->scale > 1e30) return ATK_ERR_ARGS;  // (the kernels have it in f32, where less is 0 or nearly so, and 0 * inf no number)
    if (p->dim > 256 || p->dim % piece) return ATK_ERR_UNSUPPORTED;
    const int64_t rows[3] = {p->batch, p->tokens, p->heads}, keys[3] = {p->n_pages, p->page_size, p->kv_heads};
    for (int i = 0; i < 3; ++i) {
        if (p->q_stride[i] < 0 || p->out_stride[i] < 0 || p->k_stride[i] < 0 || p->v_stride[i] < 0) return ATK_ERR_ARGS;
        if (rows[i] > 1 && (p->q_stride[i] % piece || p->out_stride[i] % piece)) return ATK_ERR_ALIGN;
        if (keys[i] > 1 && (p->k_stride[i] % piece || p->v_stride[i] % piece)) return ATK_ERR_ALIGN;
    }
    if (pointers) {
        if (!p->q || !p->k || !p->v || !p->out || !p->page_table || !p->lens) return ATK_ERR_NULL_PTR;
        if (((uintptr_t)p->q | (uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->out) & 15) return ATK_ERR_ALIGN;
        if (((uintptr_t)p->page_table | (uintptr_t)p->lens | (uintptr_t)p->seqs | (uintptr_t)p->lse | (uintptr_t)p->status) & 3) return ATK_ERR_ALIGN;
    }
    return ATK_OK;
}

// The shared keys in (at most) that many ranges of whole steps.
static void split_prefix(const atk_attention_args *p, AttnPlan *pl, int64_t step, int64_t splits) {
    const int64_t steps = attn_ceil(p->prefix_len, step);
    pl->prefix_keys = (int)(attn_ceil(steps, std::min(steps, splits)) * step);
    pl->prefix_splits = (int)attn_ceil(p->prefix_len, pl->prefix_keys);
}

// attn_block_kernel: four or eight wavefronts a workgroup, and how many ranges.  More ranges fill more CUs, and every range costs each row a partial result that is written and read
// again.  In microseconds, as measured with heads of 128: a workgroup takes 7 and for each tile of 64 keys 2.2 with eight wavefronts, 1.4 with four and 2.5 with two workgroups
// of four on a CU; partial results 0.65 a megabyte.
// attn_mixed_kernel: one workgroup of four on a CU, of which own keys then take the other half; `own`: microseconds of own keys by themselves (4.4 TB/s, and a launch), as many
// as the sequences' rows could hold.  64 samples on 8192 + 384 keys, 32 heads on 8 of 128: 58 us -> 49.  Only the device knows the lengths, so it may not cost much where own keys
// are few (kMixedLoss): 128 samples on 65536 + 1125 keys would take 248 us and not 270, but on 65536 alone 200 and not 165.
constexpr double kMixedLoss = 10;
static void plan_blocks(const atk_attention_args *p, int64_t rows, double own, AttnPlan *pl) {
    const double wide = pl->dp == 64 ? 0.6 : pl->dp == 128 ? 1.0 : 2.0;
    const int64_t steps = attn_ceil(p->prefix_len, kBlockKeys);
    double best = 0, mixed = 0;
    int64_t best_splits = 1, mixed_splits = 0;
    pl->waves = 4;
    auto each = [&](int waves, int64_t most, auto cost) {
        const int64_t blocks = attn_ceil(rows, 32 * waves), base = blocks * p->kv_heads;
        for (int64_t wanted = kNumCU / 8; wanted <= most; wanted += std::min<int64_t>(wanted, kNumCU)) {  // workgroups: an eighth of the CUs to four on each
            const int64_t splits = std::min(steps, std::max<int64_t>(1, wanted / base));
            const int64_t tiles = attn_ceil(steps, splits), ranges = attn_ceil(steps, tiles);
            cost(splits, tiles, base * ranges, 0.65e-6 * 4 * (double)(rows * p->kv_heads * p->dim) * (double)ranges);
        }
    };
    for (int waves = 4; waves <= attn_max_waves(pl->dp); waves *= 2)
        each(waves, 4 * kNumCU, [&](int64_t splits, int64_t tiles, int64_t groups, double partial) {
            const bool full = waves == 8 || (groups > kNumCU && pl->dp <= 128);
            const double rounds = (double)attn_ceil(groups, waves == 4 && full ? 2 * kNumCU : kNumCU);
            const double us = rounds * (7 + tiles * wide * (waves == 8 ? 2.2 : full ? 2.5 : 1.4)) + partial;
            if (best == 0 || us < best) best = us, best_splits = splits, pl->waves = waves;
        });
    if (own > 0 && attn_max_waves(pl->dp) >= 8)
        each(kAttnWaves, kNumCU, [&](int64_t splits, int64_t tiles, int64_t groups, double partial) {
            const double alone = 7 + tiles * wide * 1.4, us = std::max(alone, own) + partial;
            if (groups <= kNumCU && alone + partial <= best + kMixedLoss && us < best + own && (mixed == 0 || us < mixed)) mixed = us, mixed_splits = splits;
        });
    if (mixed_splits) pl->rt = kMixed, pl->waves = kAttnWaves, best_splits = mixed_splits;
    pl->prefix_blocks = (int)attn_ceil(rows, 32 * pl->waves);
    split_prefix(p, pl, kBlockKeys, best_splits);
}

static int plan_attention(const atk_attention_args *p, AttnPlan *pl) {
    const int group = (int)(p->heads / p->kv_heads);
    pl->dp = p->dim <= 64 ? 64 : p->dim <= 128 ? 128 : 256;
    const int64_t rows = p->batch * p->tokens * group, own_rows = p->tokens * group;
    // A sequence's own keys: as many as its row could hold, the device knows how many there are; workgroups for about three a CU.  Few keys are one workgroup's, shared ones and own,
    // and that is the whole call.
    const int64_t step = kAttnWaves * kTileKeys, all = p->row_pages * p->page_size;
    pl->own_blocks = (int)attn_ceil(own_rows, 16);
    const int64_t own_base = p->batch * p->kv_heads * pl->own_blocks;
    const bool together = all <= attn_together(p->dtype, own_base);
    const int64_t own = together ? all : all - p->prefix_len;
    pl->own_from = together ? 0 : (int)p->prefix_len;
    pl->own_splits = together ? 1 : own > 0 ? (int)std::min(attn_ceil(own, step), std::max<int64_t>(1, 3 * kNumCU / own_base)) : 0;
    const int64_t own_bytes = p->batch * own * p->kv_heads * p->dim * 2 * (p->dtype == ATK_F32 ? 4 : 2);
    pl->around = own_bytes > kCacheBytes;
    // how the shared keys meet the rows: up to two 16-row tiles in every wavefront, or 32 rows a wavefront and keys by way of LDS
    // (attn_block_kernel's addresses: four tokens' offsets and a page's place in 16 bytes are 32 bits)
    auto reaches = [&](const int64_t *stride) {
        const int64_t most = INT64_C(1) << 34;
        return stride[1] < (INT64_C(1) << 28) && stride[1] <= most / p->page_size && stride[0] <= most / p->n_pages;
    };
    const bool shared = p->prefix_len > 0 && !together;
    pl->rt = rows <= 16 || !shared ? 1 : 2, pl->waves = kAttnWaves;
    pl->prefix_splits = 0, pl->prefix_keys = 0;
    if (rows > 32 && p->dtype != ATK_F32 && shared && p->page_size % 4 == 0 && reaches(p->k_stride) && reaches(p->v_stride)) {
        pl->rt = 0;
        plan_blocks(p, rows, own > 0 ? 3 + own_bytes / 4.4e6 : 0, pl);
    } else {
        if (pl->rt > attn_max_rt(p->dtype, pl->dp)) pl->rt = 1;
        pl->prefix_blocks = (int)attn_ceil(rows, 16 * pl->rt);
        if (shared) split_prefix(p, pl, step, std::max<int64_t>(1, 2 * kNumCU / (pl->prefix_blocks * p->kv_heads)));
    }
    pl->rows = p->batch * p->tokens * p->heads;
    pl->parts = pl->prefix_splits + pl->own_splits;
    pl->o_bytes = pl->rows * pl->parts * p->dim * 4;
    pl->bytes = pl->o_bytes + pl->rows * pl->parts * 8;
    // launch_attn_dp's launches, and the join's
    const int64_t shared_groups = (pl->prefix_blocks * p->kv_heads * pl->prefix_splits + 7) / 8 * 8, own_groups = (own_base * pl->own_splits + 7) / 8 * 8;
    const bool fit = launches(shared_groups, 64 * pl->waves) && launches((pl->rt == kMixed ? 2 : 1) * shared_groups + own_groups, 64 * kAttnWaves) && launches(attn_ceil(pl->rows, 4), 256);
    return fit ? ATK_OK : ATK_ERR_ARGS;
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
    a.own_splits = pl.own_splits, a.own_blocks = pl.own_blocks, a.own_from = pl.own_from, a.around = pl.around;
    a.n_prefix = pl.prefix_splits * pl.prefix_blocks * a.kv_heads;
    a.prefix_grid = (a.n_prefix + 7) / 8 * 8;
    a.masked_grid = 0, a.block_rows = pl.rt <= 0 ? 32 * pl.waves : 0;
    a.n_own = a.batch * a.kv_heads * pl.own_blocks * pl.own_splits;
    a.parts = (int)pl.parts;
    a.direct = pl.parts == 1 && pl.rt > 0;  // attn_block writes parts only, and where its ranges are all there is, they can be one
    a.page.set((uint32_t)p->page_size);
    a.scale = (float)p->scale;
    a.scale2 = (float)(p->scale * 1.4426950408889634);
    hipStream_t s = (hipStream_t)stream;
    hipError_t e = p->dtype == ATK_F32    ? launch_attn_f32(a, pl.dp, pl.rt, pl.waves, s)
                   : p->dtype == ATK_BF16 ? launch_attn_bf16(a, pl.dp, pl.rt, pl.waves, s)
                                          : launch_attn_f16(a, pl.dp, pl.rt, pl.waves, s);
    if (e == hipSuccess && !a.direct)
        e = p->dtype == ATK_F32    ? launch_join<ATK_F32>(a, pl.dp, s)
            : p->dtype == ATK_BF16 ? launch_join<ATK_BF16>(a, pl.dp, s)
                                   : launch_join<ATK_F16>(a, pl.dp, s);
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // extern "C"
