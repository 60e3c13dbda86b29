// quantized_attention: checks and launch plan (see atk_quant_attention_kernel.h).
#include <cfloat>

#include "atk_quant_attention_kernel.h"

namespace atk {

static int64_t quant_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct QuantPlan {
    int dp, rt, row_blocks, ranges, chunk, pitch, mode, team, subtiles, row_chunks, code_chunks;
    int64_t units, rows, o_bytes, ml_bytes, bytes;
};

static int check_quant(const atk_quant_attention_args *p, bool pointers) {
    if (!p) return ATK_ERR_NULL_PTR;
    if (p->dtype != ATK_F32 && p->dtype != ATK_BF16 && p->dtype != ATK_F16) return ATK_ERR_DTYPE;
    const int64_t token_bytes = atk_quant_token_bytes(p->kv_heads, p->dim, p->bits);
    if (token_bytes < 0) return (int)token_bytes;
    const int es = p->dtype == ATK_F32 ? 4 : 2, piece = 16 / es;
    const int64_t most = INT64_C(1) << 30;
    if (p->batch < 1 || p->tokens < 1 || p->heads < 1 || p->page_size < 1 || p->n_pages < 1 || p->rows < 1 || p->row_pages < 1) return ATK_ERR_ARGS;
    if (p->batch > most || p->tokens > most || p->heads > most || p->page_size > most || p->n_pages > most || p->rows > most || p->row_pages > most) return ATK_ERR_ARGS;
    if (p->heads % p->kv_heads || p->batch * p->tokens > most || p->batch * p->tokens * p->heads > most) return ATK_ERR_ARGS;
    if (p->row_pages * p->page_size > most) return ATK_ERR_ARGS;
    if (p->n_pages * p->page_size > (INT64_C(1) << 36) / token_bytes - 1) return ATK_ERR_ARGS;  // (a row's place in 16 bytes is 32 bits)
    if (!p->seqs && p->batch > p->rows) return ATK_ERR_ARGS;
    if (p->table_stride < p->row_pages) return ATK_ERR_ARGS;
    if (!(p->scale >= FLT_MIN) || p->scale > 1e30) return ATK_ERR_ARGS;  // (the kernels have it in f32, where less is 0 or nearly so, and 0 * inf no number)
    const int64_t rows[3] = {p->batch, p->tokens, p->heads};
    for (int i = 0; i < 3; ++i) {
        if (p->q_stride[i] < 0 || p->out_stride[i] < 0) return ATK_ERR_ARGS;
        if (rows[i] > 1 && (p->q_stride[i] % piece || p->out_stride[i] % piece)) return ATK_ERR_ALIGN;
        if (rows[i] > 1 && p->out_stride[i] < p->dim) return ATK_ERR_ARGS;  // (rows over each other)
    }
    if (pointers) {
        if (!p->q || !p->k || !p->v || !p->out || !p->page_table || !p->lens) return ATK_ERR_NULL_PTR;
        if (((uintptr_t)p->q | (uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->out) & 15) return ATK_ERR_ALIGN;
        if (((uintptr_t)p->page_table | (uintptr_t)p->lens | (uintptr_t)p->seqs | (uintptr_t)p->lse | (uintptr_t)p->status) & 3) return ATK_ERR_ALIGN;
    }
    return ATK_OK;
}

// Queries of a sequence and a head of the cache from which on they share operands by way of LDS (kShared), 256 of them a workgroup (f32: 128): 8 sequences of 4000 to 8000 keys, 64 queries 79 us so and 56
// with 64 of them in one wavefront, 96 queries 84 and 77, 128 88 and more.  Heads past 128 do not: their two slots of 128 keys would take 256 KB (2 x 512 queries over 4096 to 8192 keys, 16 heads on 4 of
// 256: 319 us, 663 in f32).
constexpr int64_t kSharedRows = 97;
// A staged head is less than 128 bytes, so 64 at most, and a team's exponents are 16 bytes at most, which may lie over two pieces: what that takes of a lane's loads, and of LDS without asking for more.
constexpr bool staged_fits(int team) { return 32 * (4 * team + 2) <= kStagedPieces * 64 * team && quant_stage_bytes(4 * team + 2, kStagedWaves / team) <= 65536; }
static_assert(staged_fits(1) && staged_fits(2) && staged_fits(3) && staged_fits(4) && kStagedWaves == 4);
// Parts of a row from which on four wavefronts join them: 16 sequences of 8000 keys (24 parts) 36 us so and 38 by one, one of 100000 46 and 72, 32 of 8000 (12 parts) 61 and 60, 64 108 and 104.
constexpr int64_t kWideParts = 16;
// Sequences from which on wavefronts have theirs alone where workgroups would take several tiles at once.  One head of 64 in 4 bits: 8000 of 1100 keys 120 us so and 1450 by workgroups, 3500 of 8000 keys 385 and
// 588, a tenth of them long 248 and 338, 2500 of these 231 and 201 (in f32 317 and 242), 1600 211 and 108.
constexpr int64_t kManyParts = 3200;
// Sequences up to which short heads go by way of LDS: 8192 of 1100 keys, 8 heads of 128 in 4 bits, 1570 us so and 2020 by wavefronts; 9000 with 32 queries of 600 keys, 4 heads of 64, 580 and 425.
constexpr int64_t kStagedBatch = 8192;

static int plan_quant(const atk_quant_attention_args *p, QuantPlan *pl) {
    const int64_t group = p->heads / p->kv_heads, rows = p->tokens * group, all = p->row_pages * p->page_size;
    pl->dp = p->dim <= 64 ? 64 : p->dim <= 128 ? 128 : 256;
    pl->rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    pl->rt = std::min(pl->rt, quant_max_rt(p->dtype, pl->dp));
    const int64_t tiles = quant_ceil(all, 32);
    // few keys (by the rows of the table, as the host does not know the lengths): a workgroup's wavefronts share them, in one launch.  Two sequences, 2 heads of 64 in 4 bits: 256 keys 6.0 us so and 12.8
    // cut, 1024 10.2 and 13.4, 2048 13.7 and 13.8, 4096 23.5 and 14.0; 64 sequences, 8 heads of 128: 1024 18 and 25, 2048 40 and 39; 256 of these: 512 43 and 49, 1024 78 and 76.
    pl->mode = pl->rt == 1 && tiles <= 32 ? kJoin : kApart;
    if (rows >= kSharedRows && pl->dp <= 128) pl->mode = kShared, pl->rt = quant_shared_rt(p->dtype);
    const int block_rows = 16 * pl->rt * (pl->mode == kShared ? kSharedWaves : 1);
    pl->row_blocks = (int)quant_ceil(rows, block_rows);
    pl->team = pl->subtiles = 1, pl->row_chunks = pl->code_chunks = 0;
    const int64_t head_codes = p->dim * p->bits / 8, head_units = p->dim / kMxBlock;
    if (pl->mode == kApart && pl->dp * p->bits / 8 < 128 && pl->rt <= 2 && p->batch <= kStagedBatch) {
        // heads of less than a line of 128 bytes: rows by way of LDS, since loads of half a line cost as much as of a whole one (64 sequences of 4096 to 8192 keys, 8 heads of 64 bytes: the
        // loads alone 146 us head by head, 98 by rows)
        const int64_t teams = quant_ceil(p->kv_heads, kStagedWaves);
        pl->mode = kStaged;
        pl->team = (int)quant_ceil(p->kv_heads, teams);
        pl->subtiles = kStagedWaves / pl->team;
        pl->code_chunks = (int)(pl->team * head_codes / 16);
        int64_t units = 1;  // pieces that a team's exponents lie in, at most
        for (int64_t t = 0; t < teams; ++t) {
            const int64_t from = t * pl->team * head_units, to = from + pl->team * head_units;
            units = std::max(units, (std::min(to, p->kv_heads * head_units) + 15) / 16 - from / 16);
        }
        pl->row_chunks = pl->code_chunks + (int)units;
    }
    // ranges for wavefronts that fill the chip once, if that is more than one and a half for each sequence (8 heads of 128 in 4 bits, 6000 keys, 384 ranges: 128 sequences cut 174 us and not cut 294, 192 331
    // and 335, 256 370 and 342, 320 463 and 426; where a tenth of them are long cutting would go on helping: 256 87 and 291, 320 101 and 305, but the host does not know); of kShared twice, as their lengths differ (2 x 512 queries over 8192 to 16384 keys: once 430 us,
    // twice 296, three times 299)
    int64_t per_range = (pl->mode == kStaged ? quant_ceil(p->kv_heads, pl->team) : p->kv_heads) * pl->row_blocks;
    const int64_t slots = 4 * kNumCU * quant_waves(p->dtype, pl->dp, pl->rt, pl->mode) / (pl->mode == kStaged ? pl->team * pl->subtiles : pl->mode == kShared ? kSharedWaves : 1);
    const int64_t wanted = (pl->mode == kShared ? 2 : 1) * slots / per_range, range_tiles = quant_ceil(tiles, pl->mode == kShared ? kSharedSubs : pl->subtiles);
    // a workgroup that takes several tiles at once (subtiles) leaves as many parts for each sequence, cut or not, and a launch to join them: for some thousand sequences more than it saves
    const bool many = pl->subtiles > 1 && p->batch >= kManyParts;
    if (many) pl->mode = kApart, pl->team = pl->subtiles = 1, per_range = p->kv_heads * pl->row_blocks;
    // (too few tiles to cut, and several at once: one range for each sequence)
    const bool cut = !many && pl->mode != kJoin && range_tiles > 4 && (pl->subtiles > 1 || 2 * wanted >= 3 * p->batch);
    pl->ranges = cut ? (int)std::max<int64_t>(2 * p->batch, std::min(wanted, p->batch * (1 + quant_ceil(range_tiles, 4)))) : pl->subtiles > 1 ? (int)p->batch : 0;
    pl->units = pl->ranges ? pl->ranges * per_range : p->batch * per_range;
    const int64_t per = pl->mode == kApart ? kQuantWaves : 1;
    pl->chunk = (int)(pl->mode == kStaged ? std::min<int64_t>(quant_ceil(p->kv_heads, pl->team), 16) : p->kv_heads % per ? 1 : std::min<int64_t>(p->kv_heads / per, 16));
    pl->pitch = (int)std::min<int64_t>(rows, block_rows);
    pl->rows = p->batch * p->tokens * p->heads;
    const int64_t parts = (int64_t)pl->ranges * pl->subtiles * pl->row_blocks * p->kv_heads * pl->pitch;
    pl->o_bytes = parts * p->dim * 4, pl->ml_bytes = parts * 8;
    pl->bytes = pl->o_bytes + pl->ml_bytes + (pl->ranges ? p->batch * 8 : 16);
    const bool fit = pl->units < (INT64_C(1) << 31) && launches(quant_ceil(pl->units, per) + 8 * pl->chunk, 64 * kSharedWaves) && (pl->ranges == 0 || launches(quant_ceil(pl->rows, 4), 256));
    return fit ? ATK_OK : ATK_ERR_ARGS;
}

}  // namespace atk

using namespace atk;

extern "C" {

int64_t atk_quant_attention_workspace_bytes(const atk_quant_attention_args *p) {
    int rc = check_quant(p, false);
    QuantPlan pl;
    if (rc == ATK_OK) rc = plan_quant(p, &pl);
    return rc == ATK_OK ? pl.bytes : rc;
}

int atk_quant_attention(const atk_quant_attention_args *p, void *work, int64_t work_bytes, void *stream) {
    int rc = check_quant(p, true);
    QuantPlan pl;
    if (rc == ATK_OK) rc = plan_quant(p, &pl);
    if (rc != ATK_OK) return rc;
    if (!work) return ATK_ERR_NULL_PTR;
    if ((uintptr_t)work & 15) return ATK_ERR_ALIGN;
    if (work_bytes < pl.bytes) return ATK_ERR_WORKSPACE;
    QuantAttnDev d = {};
    AttnDev &a = d.a;
    a.q = p->q, a.k = p->k, a.v = p->v, a.out = p->out, a.lse = p->lse;
    a.table = p->page_table, a.lens = p->lens, a.seqs = p->seqs, a.status = p->status;
    a.parts_o = (float *)work, a.parts_ml = (float2 *)((char *)work + pl.o_bytes);
    d.shares = (int2 *)((char *)work + pl.o_bytes + pl.ml_bytes);
    a.table_stride = p->table_stride;
    for (int i = 0; i < 3; ++i) a.qs[i] = p->q_stride[i], a.os[i] = p->out_stride[i];
    a.batch = (int)p->batch, a.tokens = (int)p->tokens, a.heads = (int)p->heads, a.kv_heads = (int)p->kv_heads;
    a.group = a.heads / a.kv_heads, a.dim = (int)p->dim;
    a.rows = (int)p->rows, a.row_pages = (int)p->row_pages, a.n_pages = (int)p->n_pages;
    a.page.set((uint32_t)p->page_size);
    a.scale = (float)p->scale;
    a.scale2 = (float)(p->scale * 1.4426950408889634);
    d.row16 = (uint32_t)(mx_token_bytes(p->kv_heads, p->dim, p->bits) / 16);
    d.head_codes = (uint32_t)(p->dim * p->bits / 8), d.head_units = (uint32_t)(p->dim / kMxBlock), d.code_bytes = (uint32_t)p->kv_heads * d.head_codes;
    d.row_blocks = pl.row_blocks, d.ranges = pl.ranges, d.units = (int)pl.units, d.chunk = pl.chunk, d.pitch = pl.pitch, d.by_four = p->page_size % 4 == 0;
    d.wide_join = pl.ranges > 0 && (int64_t)pl.ranges * pl.subtiles >= kWideParts * p->batch && pl.rows < (INT64_C(1) << 24);
    d.team = pl.team, d.subtiles = pl.subtiles, d.row_chunks = pl.row_chunks, d.unit_from = pl.code_chunks;
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = p->dtype == ATK_F32    ? launch_quant_f32(d, p->bits, pl.dp, pl.rt, pl.mode, s)
                         : p->dtype == ATK_BF16 ? launch_quant_bf16(d, p->bits, pl.dp, pl.rt, pl.mode, s)
                                                : launch_quant_f16(d, p->bits, pl.dp, pl.rt, pl.mode, s);
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // extern "C"
