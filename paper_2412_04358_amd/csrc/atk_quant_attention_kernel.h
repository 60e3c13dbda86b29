// Attention over a cache of few bits: one range of a sequence's keys against a block of its queries.
//
// Ranges, their join, what a wavefront takes (32 keys at a time, everything in registers) and how the two products follow each other are those of attn_range (atk_attention_kernel.h).
// What differs is where the operands come from.  A power of two is exact in 16 bits, and so are the codes, so keys and values become bf16 (f16) numbers by one conversion for two of them,
// unit included, and nothing is rounded:
//   K  a lane has 16 bytes of one key (4 bits and heads of 64: 8), of one or two blocks: operands in their order, those of q alike.
//   V  a lane has DP / 16 elements of each of the eight keys that its weights belong to, of one block; after the conversion they are paired up as in attn_range.
// f32 goes the same way, by three products each: a f32 number is the sum of three bf16 ones (its mantissa cut in three), so q and the weights are given whole, and the products
// with keys and values, which are bf16 numbers, are summed up in f32.  (f32 products take eight times as long as bf16 ones.)
//
// How the wavefronts of a workgroup share its work goes by what bounds it (the modes below): few keys by their latency, few queries by the loads, many by vector instructions and products.
// 64 sequences of 4096 to 8192 keys, 32 heads on 8 of 128, 4 bits, 429 MB: 107 to 109 us (4.0 TB/s) with the join's 5, 95 without what is computed, 81 without the loads; 2 x 512 queries over 8192 to
// 16384 keys, 206 GFLOP: 295 to 322 us (0.64 to 0.7 PFLOP/s) with the join's 21, the matrix units busy for 29 % and the vector unit for 40 % of the kernel's time, a SIMD's two wavefronts waiting
// for the same things too often; two sequences of 200 keys: 6.
#pragma once

#include "atk_attention_kernel.h"
#include "atk_mx.h"

namespace atk {

constexpr int kQuantWaves = 4;

struct QuantAttnDev {
    AttnDev a;              // (not its plan)
    uint32_t row16;         // a token's row in 16 bytes
    uint32_t head_codes, head_units, code_bytes;
    int row_blocks, units, pitch;  // pitch: rows of a part
    int ranges;             // of all sequences together, at most; 0: one each, and no parts
    int2 *shares;           // [sequence]: its first range, and how many it has
    bool by_four;           // pages are whole fours of tokens
    bool wide_join;         // a row's parts are joined by four wavefronts
    int team, subtiles;     // MODE kStaged: heads of a workgroup, 32 keys that it takes at a time for each of them
    int row_chunks, unit_from;  // ... pieces of 16 bytes of a token that it brings in, how many of those are codes (behind them: the exponents)
    int chunk;              // workgroups next to each other that read the same keys: they go to one XCD
};

// Range `which` of all sequences': their tiles are cut into equally many for each range, so that wavefronts that all fit the chip end together whatever the lengths are (64 sequences of
// 4096 to 8192 keys: with equally many ranges for each of them 160 us).  Every wavefront finds its own by the lengths; B sequences have at most all tiles / R + B of them.
struct QuantRange {
    int b, split, tiles;    // b: -1 where there are fewer ranges; tiles of 32 * subtiles keys
};
__device__ __forceinline__ QuantRange quant_range(const AttnDev &a, int2 *shares, int ranges, int which, int subtiles, int parts, bool *bad_len, bool *bad_seq) {
    const int lane = threadIdx.x & 63;
    auto tiles_of = [&](int b) {
        if (b >= a.batch) return 0;
        return (seq_len(a, seq_row(a, b, bad_seq), bad_len) + 32 * subtiles - 1) / (32 * subtiles);
    };
    int64_t total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) total += tiles_of(b0 + lane);
    for (int w = 1; w < 64; w <<= 1) total += __shfl_xor(total, w, 64);
    const int spare = ranges - a.batch, each = (int)max((int64_t)4, spare > 0 ? (total + spare - 1) / spare : total);  // (none to spare: nothing is cut)
    QuantRange r{-1, 0, 0};
    int before = 0;
    for (int b0 = 0; b0 < a.batch && r.b < 0; b0 += 64) {
        const int tiles = tiles_of(b0 + lane), n = b0 + lane < a.batch ? max(1, (tiles + each - 1) / each) : 0;
        int up = n;
        for (int w = 1; w < 64; w <<= 1) {
            const int o = __shfl_up(up, w, 64);
            if (lane >= w) up += o;
        }
        const int front = before + up - n;
        const uint64_t mine = __ballot(which >= front && which < front + n);
        if (mine) {
            const int at = __builtin_ctzll(mine);
            r.b = b0 + at, r.split = which - __builtin_amdgcn_readlane(front, at);
            r.tiles = __builtin_amdgcn_readlane(n > 0 ? (tiles + n - 1) / n : 0, at);
            if (lane == at && r.split == 0) shares[r.b] = int2{front * parts, n * parts};  // (from one wavefront for each head and row block, all alike)
        }
        before = __builtin_amdgcn_readlane(front + n, 63);
    }
    r.b = __builtin_amdgcn_readfirstlane(r.b), r.split = __builtin_amdgcn_readfirstlane(r.split), r.tiles = __builtin_amdgcn_readfirstlane(r.tiles);
    return r;
}

// How a workgroup's wavefronts share its work.
enum { kApart = 0,   // each has a range of its own, for a head (workgroups' wavefronts: neighbouring heads)
       kJoin = 1,    // they take turns at the tiles of one range, for one head, and join through LDS
       kStaged = 2,  // a range for several heads: rows come into LDS whole, a tile ahead, and a wavefront has one head's part of them
       kShared = 3   // a range for one head and many queries: operands are made once, go through LDS, and each wavefront has queries of its own
};
constexpr int kSharedWaves = 8, kSharedSubs = 4;  // of kShared: each wavefront makes keys' or values' operands of 32 of a tile's 128 keys
constexpr int quant_shared_bytes(int dp) { return 2 * kSharedSubs * (2 * (dp / 32) + dp / 16) * 1024 + 64; }
constexpr int kStagedWaves = 4, kStagedPieces = 3;
constexpr int quant_stage_bytes(int row_chunks, int subtiles) { return 4 * subtiles * 32 * row_chunks * 16; }

constexpr int quant_products(int elt) { return elt == ATK_F32 ? ATK_BF16 : elt; }  // type of the products' operands
constexpr int quant_parts(int elt) { return elt == ATK_F32 ? 3 : 1; }              // operands that a number of q or a weight is the sum of

// A pair of f32 numbers as pairs of bf16 ones of which they are the sums: cut, not rounded, so that the largest numbers stay finite.
__device__ __forceinline__ void split_pair(float a, float b, uint32_t *w) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        w[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        a = a - __uint_as_float(x & 0xffff0000u), b = b - __uint_as_float(y & 0xffff0000u);
    }
}

template <int ELT>
struct QuantWeights {
    Weights<quant_products(ELT)> p[quant_parts(ELT)];
    __device__ __forceinline__ void set(const f32x4 *s) {
        if constexpr (ELT == ATK_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[3];
                split_pair(s[i / 2][2 * (i & 1)], s[i / 2][2 * (i & 1) + 1], w);
#pragma unroll
                for (int j = 0; j < 3; ++j) p[j].w[i] = w[j];
            }
        } else {
            p[0].set(s);
        }
    }
};

// Eight elements of a query.
template <int ELT>
struct QuantQuery {
    u32x4 w[quant_parts(ELT)];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < quant_parts(ELT); ++j) w[j] = u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void load(const char *p) {
        if constexpr (ELT == ATK_F32) {
            const f32x4 a = ((const f32x4 *)p)[0], b = ((const f32x4 *)p)[1];
            const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t y[3];
                split_pair(x[2 * i], x[2 * i + 1], y);
                // (what is left of an infinity is NaN, and the infinity alone is right)
                const bool all = fabsf(x[2 * i]) < __builtin_inff(), all2 = fabsf(x[2 * i + 1]) < __builtin_inff();
                const uint32_t keep = (all ? 0xffffu : 0u) | (all2 ? 0xffff0000u : 0u);
                // (a NaN whose mantissa's upper bits are clear would be cut to an infinity)
                w[0][i] = y[0] | (x[2 * i] != x[2 * i] ? 0x40u : 0u) | (x[2 * i + 1] != x[2 * i + 1] ? 0x400000u : 0u);
                w[1][i] = y[1] & keep, w[2][i] = y[2] & keep;
            }
        } else {
            w[0] = *(const u32x4 *)p;
        }
    }
};

// f(0), f(1), ... f(N - 1), each number a type's.
template <int N, int X = 0, typename F>
__device__ __forceinline__ void each_of(F f) {
    if constexpr (X < N) {
        f(std::integral_constant<int, X>{});
        each_of<N, X + 1>(f);
    }
}

// What a lane holds of 32 keys as it lies in memory.
template <int BITS, int DP>
struct QuantRaw {
    static constexpr int kStepWords = BITS / 4;                             // words of eight elements
    static constexpr int kPieceWords = BITS == 4 && DP == 64 ? 2 : 4;       // words of a piece of a key
    static constexpr int kPieceSteps = kPieceWords / kStepWords;            // products that it is for
    static constexpr int NC = DP / 32 / kPieceSteps;                        // pieces of a key
    static constexpr int kVBytes = DP / 16 * BITS / 8;                      // bytes of V's row
    static constexpr int kVWords = (kVBytes + 3) / 4;
    static constexpr int kPieceDims = 8 * kPieceSteps;
    uint32_t k[2][NC][kPieceWords], ku[2][NC], v[8][kVWords], vu[8];  // ku, vu: words that the exponents lie in (bytes that go round a loop are cleared above them where they arrive, which is a wait)
};

// Wavefronts of a SIMD, which share its registers.
constexpr int quant_waves(int elt, int dp, int rt, int mode) {
    if (mode == kShared) return 2;
    if (mode == kStaged) return rt == 1 ? (dp == 64 ? 4 : 3) - (elt == ATK_F32 ? 1 : 0) : 2;
    return rt == 1 ? (dp == 64 ? 4 : dp == 128 ? (elt == ATK_F32 ? 2 : 3) : 2) : rt == 2 && dp <= 128 ? 2 : 1;
}

// Loads stay on their sides of this.  A wait for one is a number of later ones, the least over all ways to it, so page numbers, keys and values have to be asked for in one order in front of the
// loop and in it, or each tile waits for the next one's values.
__device__ __forceinline__ void keep_loads() { __builtin_amdgcn_sched_barrier(0x78f); }

// FULL: heads of DP elements.  Shorter ones: what lies behind them is read at their first elements, and counts as 0 in keys; of values it goes into sums that are not written.
template <int ELT, int BITS, int DP, int RT, int MODE, bool FULL>
__global__ __launch_bounds__(64 * (MODE == kStaged ? kStagedWaves : MODE == kShared ? kSharedWaves : kQuantWaves), quant_waves(ELT, DP, RT, MODE)) void quant_attn_kernel(const QuantAttnDev d) {
    typedef AttnElt<ELT> E;
    constexpr int PE = quant_products(ELT), PARTS = quant_parts(ELT);
    typedef AttnElt<PE> P;
    typedef QuantRaw<BITS, DP> Raw;
    constexpr int NT = DP / 16, NS = DP / 32;       // products along d of the second product, of the first
    constexpr int TK = 32, NW = kQuantWaves;
    const AttnDev &a = d.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;

    // workgroups of a chunk are 8 apart, which is how they come to one XCD
    const uint32_t at8 = blockIdx.x / 8, block = (at8 / d.chunk * 8 + blockIdx.x % 8) * d.chunk + at8 % d.chunk;
    const uint32_t unit = MODE == kApart ? block * NW + wave : block;
    if (unit >= (uint32_t)d.units) return;
    // of a staged workgroup: the heads from h0 on, a wavefront has one of them and 32 keys of a tile
    const int teams = MODE == kStaged ? (a.kv_heads + d.team - 1) / d.team : a.kv_heads;
    const int h0 = (int)(unit % (uint32_t)teams) * (MODE == kStaged ? d.team : 1);
    const int sub = MODE == kStaged ? wave / d.team : 0, member = MODE == kStaged ? wave % d.team : 0;
    const int h = MODE == kStaged ? min(h0 + member, a.kv_heads - 1) : h0;
    const bool idle = MODE == kStaged && h0 + member >= a.kv_heads;  // (one head too many for the last team: it helps with the loads)
    const uint32_t rest = unit / (uint32_t)teams;
    const int block_of = (int)(rest % (uint32_t)d.row_blocks);
    bool bad_len = false, bad_seq = false, bad_page = false;
    int b = (int)(rest / (uint32_t)d.row_blocks), split = 0, each = 0;
    const int range_at = b;
    if (MODE != kJoin && d.ranges) {
        const QuantRange r = quant_range(a, d.shares, d.ranges, b, MODE == kStaged ? d.subtiles : MODE == kShared ? kSharedSubs : 1, MODE == kStaged ? d.subtiles : 1, &bad_len, &bad_seq);
        if (r.b < 0) return;
        b = r.b, split = r.split, each = r.tiles;
    }
    constexpr int kBlockRows = 16 * RT * (MODE == kShared ? kSharedWaves : 1);
    const int n_rows = a.tokens * a.group, block_r0 = block_of * kBlockRows, r0 = block_r0 + (MODE == kShared ? wave * 16 * RT : 0);
    const int s_row = seq_row(a, b, &bad_seq);
    const int len = seq_len(a, s_row, &bad_len);
    // the keys that the block's last query sees
    const int last_t = (min(block_r0 + kBlockRows, n_rows) - 1) / a.group;
    const int end = max(0, len - (a.tokens - 1 - last_t));
    const bool whole = MODE == kJoin || !d.ranges;
    const int tile = MODE == kStaged ? TK * d.subtiles : MODE == kShared ? TK * kSharedSubs : TK;
    const int ka = whole ? 0 : (int)min((int64_t)end, (int64_t)split * each * tile), kb = whole ? end : (int)min((int64_t)end, (int64_t)ka + (int64_t)each * tile);
    const int32_t *table_row = a.table + max(s_row, 0) * a.table_stride;

    // first what the keys' addresses wait for.  lane j (and the one 32 behind it) looks key k0 + j up; keys past the end are read as the last one and masked
    const int kStep = MODE == kApart ? TK : MODE == kJoin ? NW * TK : tile;
    const int first = ka + (MODE == kApart ? 0 : MODE == kJoin ? wave * TK : MODE == kStaged ? sub * TK : (wave % kSharedSubs) * TK);
    auto page_of = [&](int k0) { return table_row[a.page.div(min(k0 + (lane & 31), kb - 1))]; };
    const int last = first + (kb - 1 - first) / kStep * kStep;  // (of this wavefront's tiles)
    const int last_tile = (kb - 1) & ~(TK - 1);  // (ranges begin at whole tiles)
    int page_next = MODE == kShared ? (ka < kb ? page_of(min(first, last_tile)) : 0) : first < kb ? page_of(first) : 0;

    QuantQuery<ELT> q[RT][NS];
    int lim[RT];
    int min_lim = kb;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + rt * 16 + n;
        const bool real = r < n_rows;
        const AttnRow x = attn_row(a, h, real ? r : 0, b);
        // rows past the end are computed as if they saw all keys, and not written: they must not make tiles masked
        lim[rt] = real ? min(kb, len - (a.tokens - 1 - x.t)) : kb;
        min_lim = min(min_lim, lim[rt]);
        const char *p = (const char *)a.q + (x.b * a.qs[0] + x.t * a.qs[1] + x.head * a.qs[2]) * E::kBytes;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int dim = (s / Raw::kPieceSteps * 4 + g) * Raw::kPieceDims + s % Raw::kPieceSteps * 8;
            if (FULL || dim < a.dim)
                q[rt][s].load(p + dim * E::kBytes);
            else
                q[rt][s].clear();
        }
    }
    for (int w = 1; w < 16; w <<= 1) min_lim = min(min_lim, __shfl_xor(min_lim, w, 64));

    float m[RT], l[RT];  // maximum, in units of s: c * s need not be finite where s is
    bool far = false;    // ... and is not for some query of the wavefront
    f32x4 acc[RT][NT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = kNoMax, l[rt] = 0.0f;
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[rt][i] = f32x4{0, 0, 0, 0};
    }

    // a lane's places in a row: of its pieces of a key, of its elements of a value
    const int v_dim = FULL || n * (DP / 16) < a.dim ? n * (DP / 16) : 0;
    int ku_bit[Raw::NC], k_dim[Raw::NC];
    bool inside[Raw::NC];
    auto unit_at = [&](int dim) { return d.code_bytes + h * d.head_units + dim / kMxBlock; };
#pragma unroll
    for (int c = 0; c < Raw::NC; ++c) {
        k_dim[c] = (c * 4 + g) * Raw::kPieceDims;
        inside[c] = FULL || k_dim[c] < a.dim;
        if (!inside[c]) k_dim[c] = 0;
        ku_bit[c] = 8 * (unit_at(k_dim[c]) & 3);
    }
    const int vu_bit = 8 * (unit_at(v_dim) & 3), v_bit = Raw::kVBytes < 4 ? 8 * ((v_dim * BITS / 8) & 3) : 0;
    // ... in memory
    struct {
        const char *kc[Raw::NC], *ku[Raw::NC], *vc, *vu;
    } row_of;
    auto find_rows = [&]() {
#pragma unroll
        for (int c = 0; c < Raw::NC; ++c) {
            row_of.kc[c] = (const char *)a.k + h * d.head_codes + k_dim[c] * BITS / 8;
            row_of.ku[c] = (const char *)a.k + (unit_at(k_dim[c]) & ~3u);
        }
        row_of.vc = (const char *)a.v + h * d.head_codes + (v_dim * BITS / 8 & ~(Raw::kVBytes < 4 ? 3 : 0));
        row_of.vu = (const char *)a.v + (unit_at(v_dim) & ~3u);
    };

    uint32_t valid = 0;
    auto places = [&](int k0, int page) {  // a key's row in 16 bytes
        const bool good = (unsigned)page < (unsigned)a.n_pages;
        bad_page |= !good;
        valid = (uint32_t)__ballot(good);
        // (by four: a lane whose key is behind the last one may be asked for the first of four)
        const int key = d.by_four ? k0 + (lane & 31) : min(k0 + (lane & 31), kb - 1);
        uint32_t first_of = (uint32_t)((good ? page : 0) - a.page.div(key)) * (a.page.d * d.row16);
        asm volatile("" : "+v"(first_of));  // (a product and a sum in one instruction of 64 bits would wait for whatever its unused half is being loaded with)
        return first_of + (uint32_t)key * d.row16;
    };
    Raw raw;
    auto load_k = [&](uint32_t place) {
        const uint32_t rows[2] = {(uint32_t)__shfl((int)place, n, 64), (uint32_t)__shfl((int)place, 16 + n, 64)};
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const uint64_t row = (uint64_t)rows[y] << 4;
#pragma unroll
            for (int c = 0; c < Raw::NC; ++c) {
                if constexpr (Raw::kPieceWords == 4) {
                    const u32x4 t = *(const u32x4 *)(row_of.kc[c] + row);
#pragma unroll
                    for (int z = 0; z < 4; ++z) raw.k[y][c][z] = t[z];
                } else {
                    const u32x2 t = *(const u32x2 *)(row_of.kc[c] + row);
                    raw.k[y][c][0] = t[0], raw.k[y][c][1] = t[1];
                }
                raw.ku[y][c] = *(const uint32_t *)(row_of.ku[c] + row);
            }
        }
    };
    auto load_v = [&](uint32_t place) {
        uint32_t rows[8];
        if (d.by_four) {  // four keys are in one page, one behind the other (those behind the last one, too: of the page, and not visible)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t at = (uint32_t)__shfl((int)place, x * 16 + g * 4, 64);
#pragma unroll
                for (int j = 0; j < 4; ++j) rows[x * 4 + j] = at + j * d.row16;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) rows[j] = (uint32_t)__shfl((int)place, (j / 4) * 16 + g * 4 + j % 4, 64);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint64_t row = (uint64_t)rows[j] << 4;
            const char *p = row_of.vc + row;
            if constexpr (Raw::kVBytes <= 4) {
                raw.v[j][0] = *(const uint32_t *)p;
            } else if constexpr (Raw::kVBytes == 8) {
                const u32x2 t = *(const u32x2 *)p;
                raw.v[j][0] = t[0], raw.v[j][1] = t[1];
            } else {
                const u32x4 t = *(const u32x4 *)p;
#pragma unroll
                for (int z = 0; z < 4; ++z) raw.v[j][z] = t[z];
            }
            raw.vu[j] = *(const uint32_t *)(row_of.vu + row);
        }
    };

    // K's operand of product c for 16 of the keys
    auto key_operand = [&](int x, int c) {
        const int piece = c / Raw::kPieceSteps;
        u32x4 kf = __builtin_bit_cast(u32x4, mx_eight<PE, BITS>(&raw.k[x][piece][c % Raw::kPieceSteps * Raw::kStepWords], mx_unit(raw.ku[x][piece] >> ku_bit[piece] & 0xff)));
        if (!FULL && !inside[piece]) kf = u32x4{0, 0, 0, 0};
        return kf;
    };
    // S^T of a tile
    f32x4 s[RT][2];
    auto scores = [&]() {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][x] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NS; ++c) {
                const u32x4 kf = key_operand(x, c);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int y = PARTS - 1; y >= 0; --y) s[rt][x] = P::mma(kf, q[rt][c].w[y], s[rt][x]);
            }
        }
    };
    auto hide = [&](int k0, uint32_t now) {
        asm volatile("");  // (a branch, no selections)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = x * 16 + g * 4 + j;
                    if (k0 + at >= lim[rt] || !(now >> at & 1)) s[rt][x][j] = kNoMax;
                }
    };
    auto raise_max = [&]() {
        float top[RT];
        bool raise = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float t = s[rt][0][0];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) t = fmaxf(t, s[rt][x][j]);
            top[rt] = t;
            raise |= (t - m[rt]) * a.scale2 > kLazyMax;
        }
        if (__any(raise)) {  // (a query's lanes find out what they have in common when one of them has to know, and not for every tile)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float t = fmaxf(top[rt], __shfl_xor(top[rt], 16, 64));
                t = fmaxf(t, __shfl_xor(t, 32, 64));
                const float to = fmaxf(m[rt], t);
                const float f = m[rt] == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((m[rt] - to) * a.scale2);  // (nothing is kept yet where there was no maximum)
                l[rt] *= f;
#pragma unroll
                for (int i = 0; i < NT; ++i) acc[rt][i] *= f;
                m[rt] = to;
                far |= fabsf(to) < __builtin_inff() && !(fabsf(to * a.scale2) < __builtin_inff());
            }
            far = __any(far);
        }
    };
    // weights, and their sums
    auto weigh = [&](QuantWeights<ELT> *p, float *sums) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float zero = m[rt] == kNoMax ? 0.0f : m[rt];
            const float ref = zero * a.scale2 - E::kBias;
            if (far) {
                asm volatile("");  // (a branch, no selections)
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[rt][x][j] = fmaf(s[rt][x][j] - zero, a.scale2, E::kBias);
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[rt][x][j] = fmaf(s[rt][x][j], a.scale2, -ref);
            }
            float sum = 0.0f;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[rt][x][j] = __builtin_amdgcn_exp2f(s[rt][x][j]);
                    sum += s[rt][x][j];
                }
            sums[rt] = sum;
            p[rt].set(s[rt]);
        }
    };
    // V^T's operands of products 2 * X and 2 * X + 1: elements 2 * X and 2 * X + 1 of all eight keys, by two conversions' worth of registers at a time
    auto operands = [&](auto x, u32x4 *o) {
        constexpr int X = decltype(x)::value;
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float unit = mx_unit(raw.vu[j] >> vu_bit & 0xff);
            if constexpr (Raw::kVBytes < 4) {
                const uint32_t two = raw.v[j][0] >> v_bit;
                w[j] = mx_pair<PE, BITS, X % 4>(&two, unit);
            } else {
                w[j] = mx_pair<PE, BITS, X % 4>(&raw.v[j][X / 4 * Raw::kStepWords], unit);
            }
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            o[0][y] = __builtin_amdgcn_perm(w[2 * y + 1], w[2 * y], 0x05040100u);
            o[1][y] = __builtin_amdgcn_perm(w[2 * y + 1], w[2 * y], 0x07060302u);
        }
    };
    // Whether row j of a lane's values may hold a number that is not finite: by the unit, or e4m3's NaN.
    auto odd_row = [&](int j) {
        bool odd = (raw.vu[j] >> vu_bit & 0xff) >= (PE == ATK_F16 ? 141u : 253u) - (BITS == 8 ? 6u : 0u);
        if constexpr (BITS == 8) {
#pragma unroll
            for (int z = 0; z < Raw::kVWords; ++z) {
                const uint32_t x = ~raw.v[j][z] & 0x7f7f7f7fu;  // a byte of 0: NaN
                odd |= ((x - 0x01010101u) & ~x & 0x80808080u) != 0;
            }
        }
        return odd;
    };
    auto drop_row = [&](int j) {
        raw.vu[j] = kMxLeast << vu_bit;
#pragma unroll
        for (int z = 0; z < Raw::kVWords; ++z) raw.v[j][z] = 0;
    };

    bool apart = false;  // rows of values that are not finite were left out, as 0 * them would not be 0 for queries that do not see them
    auto drop = [&](int k0, uint32_t now) {  // in tiles with a mask
        asm volatile("");  // (a branch, no selections)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (odd_row(j)) {
                const int at = (j / 4) * 16 + g * 4 + j % 4;
                apart |= k0 + at < kb && (now >> at & 1);  // (what no query sees is nothing)
                drop_row(j);
            }
    };
    auto products = [&](const QuantWeights<ELT> *p) {
        each_of<NT / 2>([&](auto x) {
            u32x4 o[2];
            operands(x, o);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int y = PARTS - 1; y >= 0; --y) acc[rt][2 * decltype(x)::value + i] = P::mma(o[i], p[rt].p[y].w, acc[rt][2 * decltype(x)::value + i]);
        });
    };

    int apart_lim = min_lim;  // tiles up to it have no mask for whoever made their operands
    if constexpr (MODE == kShared) {
        // Two slots of a tile's operands as the products take them, 16 bytes a lane.  A wavefront makes those of the next tile (from rows that it asked for a tile before), asks for the rows of
        // the one behind it, and then has this one's products: 16 KB from LDS for 32 keys and its 32 queries (heads of 128), a third of what LDS has for the time that they take.
        extern __shared__ char stage[];
        constexpr int kKey = 2 * NS * 1024, kSub = kKey + NT * 1024, kSlot = kSharedSubs * kSub;
        uint32_t *const masks = (uint32_t *)(stage + 2 * kSlot), *const any_apart = masks + 2 * kSharedSubs;
        const int mine = wave % kSharedSubs;
        const bool makes_values = wave >= kSharedSubs;
        apart_lim = min(kb, len - (a.tokens - 1 - block_r0 / a.group));
        if (threadIdx.x == 0) *any_apart = 0;
        find_rows();
        auto ask = [&](int t0) {
            const uint32_t place = places(min(t0 + mine * TK, last_tile), page_next);
            page_next = page_of(min(t0 + tile + mine * TK, last_tile));
            if (makes_values)
                load_v(place);
            else
                load_k(place);
        };
        auto make = [&](int t0, int slot, uint32_t now) {
            char *const to = stage + slot * kSlot + mine * kSub + lane * 16;
            const int k0 = t0 + mine * TK;
            if (makes_values) {
                if (k0 + TK > apart_lim || now != 0xffffffffu) drop(k0, now);
                each_of<NT / 2>([&](auto x) {
                    u32x4 o[2];
                    operands(x, o);
                    *(u32x4 *)(to + kKey + (2 * decltype(x)::value) * 1024) = o[0];
                    *(u32x4 *)(to + kKey + (2 * decltype(x)::value + 1) * 1024) = o[1];
                });
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int c = 0; c < NS; ++c) *(u32x4 *)(to + (x * NS + c) * 1024) = key_operand(x, c);
                if (lane == 0) masks[slot * kSharedSubs + mine] = now;
            }
        };
        const int my_end = min(kb, len - (a.tokens - 1 - (min(r0 + 16 * RT, n_rows) - 1) / a.group));
        const bool idle_rows = r0 >= n_rows;
        if (ka < kb) {
            ask(ka);
            uint32_t now = valid;
            make(ka, 0, now);
            ask(ka + tile);
            now = valid;
            __syncthreads();
            int slot = 0;
            for (int t0 = ka; t0 < kb; t0 += tile, slot ^= 1) {
                if (t0 + tile < kb) {
                    make(t0 + tile, slot ^ 1, now);
                    ask(t0 + 2 * tile);
                    now = valid;
                }
                if (!idle_rows)
                    for (int st = 0; st < kSharedSubs; ++st) {
                        const int k0 = t0 + st * TK;
                        if (k0 >= my_end) break;
                        const char *const from = stage + slot * kSlot + st * kSub + lane * 16;
                        const uint32_t seen = masks[slot * kSharedSubs + st];
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) s[rt][x] = f32x4{0, 0, 0, 0};
#pragma unroll
                            for (int c = 0; c < NS; ++c) {
                                const u32x4 kf = *(const u32x4 *)(from + (x * NS + c) * 1024);
#pragma unroll
                                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                                    for (int y = PARTS - 1; y >= 0; --y) s[rt][x] = P::mma(kf, q[rt][c].w[y], s[rt][x]);
                            }
                        }
                        if (k0 + TK > min_lim || seen != 0xffffffffu) hide(k0, seen);
                        raise_max();
                        QuantWeights<ELT> p[RT];
                        float sums[RT];
                        weigh(p, sums);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) l[rt] += sums[rt];
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            const u32x4 vi = *(const u32x4 *)(from + kKey + i * 1024);
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                                for (int y = PARTS - 1; y >= 0; --y) acc[rt][i] = P::mma(vi, p[rt].p[y].w, acc[rt][i]);
                        }
                    }
                __syncthreads();
            }
        }
        if (__any(apart) && lane == 0) *any_apart = 1;
        __syncthreads();
        apart = *any_apart && !idle_rows;
    } else if constexpr (MODE == kStaged) {
        // Two slots of a tile's rows, keys' and values'.  The team's wavefronts bring their 32 keys in, 16 bytes a lane, the lane's pieces of all tiles being the same ones of a row; in
        // LDS they lie as they are counted, a row's pieces next to each other.
        extern __shared__ char stage[];
        const int row_bytes = d.row_chunks * 16, sub_bytes = TK * row_bytes, slot_bytes = 2 * d.subtiles * sub_bytes;
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)stage;
        int token[kStagedPieces];
        uint32_t from[kStagedPieces];
        bool there[kStagedPieces];
#pragma unroll
        for (int k = 0; k < kStagedPieces; ++k) {
            const int i = (k * d.team + member) * 64 + lane, c = i % d.row_chunks;
            token[k] = i / d.row_chunks & 31, there[k] = i < TK * d.row_chunks;
            from[k] = min(d.row16 * 16 - 16, c < d.unit_from ? (uint32_t)h0 * d.head_codes + c * 16 : ((d.code_bytes + h0 * d.head_units) & ~15u) + (c - d.unit_from) * 16);  // (a last team may have fewer heads)
        }
        auto bring = [&](int slot, uint32_t place) {
#pragma unroll
            for (int k = 0; k < kStagedPieces; ++k) {
                const uint64_t at = ((uint64_t)(uint32_t)__shfl((int)place, token[k], 64) << 4) + from[k];
                const uint32_t to = __builtin_amdgcn_readfirstlane(lds + slot * slot_bytes + sub * sub_bytes + (k * d.team + member) * 1024);
                if (there[k]) {
                    load_to_lds((const char *)a.k + at, to);
                    load_to_lds((const char *)a.v + at, to + d.subtiles * sub_bytes);
                }
            }
        };
        // a wavefront's own places in a slot
        const char *lk[Raw::NC], *lu[Raw::NC];
        const int unit_at0 = d.unit_from * 16 + ((d.code_bytes + h0 * d.head_units) & 15) + (h - h0) * d.head_units;
        const char *mine = stage + sub * sub_bytes + (h - h0) * (int)d.head_codes;
#pragma unroll
        for (int c = 0; c < Raw::NC; ++c) {
            lk[c] = mine + n * row_bytes + k_dim[c] * BITS / 8;
            lu[c] = stage + sub * sub_bytes + n * row_bytes + ((unit_at0 + k_dim[c] / kMxBlock) & ~3);
        }
        const char *lv = mine + d.subtiles * sub_bytes + g * 4 * row_bytes + (v_dim * BITS / 8 & ~(Raw::kVBytes < 4 ? 3 : 0)),
                   *lvu = stage + (sub + d.subtiles) * sub_bytes + g * 4 * row_bytes + ((unit_at0 + v_dim / kMxBlock) & ~3);
        auto read_k = [&](int slot) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int c = 0; c < Raw::NC; ++c) {
                    const int at = slot * slot_bytes + y * 16 * row_bytes;
                    if constexpr (Raw::kPieceWords == 4) {
                        const u32x4 t = *(const u32x4 *)(lk[c] + at);
#pragma unroll
                        for (int z = 0; z < 4; ++z) raw.k[y][c][z] = t[z];
                    } else {
                        const u32x2 t = *(const u32x2 *)(lk[c] + at);
                        raw.k[y][c][0] = t[0], raw.k[y][c][1] = t[1];
                    }
                    raw.ku[y][c] = *(const uint32_t *)(lu[c] + at);
                }
        };
        auto read_v = [&](int slot) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = slot * slot_bytes + (j / 4 * 16 + j % 4) * row_bytes;
#pragma unroll
                for (int z = 0; z < Raw::kVWords; ++z) raw.v[j][z] = ((const uint32_t *)(lv + at))[z];
                raw.vu[j] = *(const uint32_t *)(lvu + at);
            }
        };
        if (ka < kb) {
            bring(0, places(first, page_next));
            uint32_t now = valid;
            page_next = page_of(min(first + kStep, kb - 1));
            int slot = 0;
            for (int t0 = ka; t0 < kb; t0 += kStep, slot ^= 1) {
                const int k0 = t0 + sub * TK;
                wait_loads<0>();
                __syncthreads();  // the tile is there, and the other slot has been read
                uint32_t next = 0;
                if (t0 + kStep < kb) {
                    bring(slot ^ 1, places(min(k0 + kStep, kb - 1), page_next));
                    next = valid;
                    page_next = page_of(min(k0 + 2 * kStep, kb - 1));
                }
                if (k0 < kb && !idle) {
                    read_k(slot);
                    scores();
                    const bool masked = k0 + TK > min_lim || now != 0xffffffffu;
                    if (masked) hide(k0, now);
                    raise_max();
                    QuantWeights<ELT> p[RT];
                    float sums[RT];
                    weigh(p, sums);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) l[rt] += sums[rt];
                    read_v(slot);
                    if (masked) drop(k0, now);
                    products(p);
                }
                now = next;
            }
        }
    } else {
    find_rows();
    keep_loads();
    if (first < kb) {
        const uint32_t place = places(first, page_next);
        page_next = page_of(min(first + kStep, last));
        keep_loads();
        load_k(place);
        keep_loads();
        load_v(place);
        keep_loads();
        int k0 = first;
        do {  // (the one way to it is from here: see keep_loads)
            // a tile's loads go out when the registers that they come to are free, a tile ahead (behind the last one it once more: a branch around them would cost a wait for them)
            const uint32_t now = valid;
            const int next = min(k0 + kStep, last);
            const uint32_t place = places(next, page_next);
            page_next = page_of(min(next + kStep, last));
            keep_loads();
            scores();
            load_k(place);
            keep_loads();
            if (k0 + TK > min_lim || now != 0xffffffffu) hide(k0, now);
            raise_max();
            QuantWeights<ELT> p[RT];
            float sums[RT];
            weigh(p, sums);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) l[rt] += sums[rt];
            if (k0 + TK > min_lim || now != 0xffffffffu) drop(k0, now);
            products(p);
            load_v(place);
            keep_loads();
            k0 += kStep;
        } while (k0 < kb);
    }
    }
    if (__any(apart)) {
        // what was left out, query by query with what it does not see at 0 (a product's columns are queries of their own)
        if (MODE == kStaged) find_rows();
        for (int k0 = MODE == kShared ? ka : first; k0 < kb; k0 += MODE == kShared ? TK : kStep) {
            const uint32_t place = places(k0, page_of(k0)), now = valid;
            if (!(k0 + TK > apart_lim || now != 0xffffffffu)) continue;
            load_k(place);
            load_v(place);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!odd_row(j)) drop_row(j);
            scores();
            hide(k0, now);
            QuantWeights<ELT> p[RT];
            float sums[RT];
            weigh(p, sums);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                for (int c = 0; c < 16; ++c) {
                    const int limit = __shfl(lim[rt], c, 64);
                    u32x4 seen;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int at = (y / 2) * 16 + g * 4 + y % 2 * 2;
                        seen[y] = (k0 + at < limit && (now >> at & 1) ? 0xffffu : 0u) | (k0 + at + 1 < limit && (now >> (at + 1) & 1) ? 0xffff0000u : 0u);
                    }
                    each_of<NT / 2>([&](auto x) {
                        u32x4 o[2];
                        operands(x, o);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            constexpr int at = 2 * decltype(x)::value;
                            f32x4 t = acc[rt][at + i];
#pragma unroll
                            for (int y = PARTS - 1; y >= 0; --y) t = P::mma(o[i] & seen, p[rt].p[y].w, t);
                            if (n == c) acc[rt][at + i] = t;
                        }
                    });
                }
        }
    }
    if (MODE == kStaged && idle) return;
    const int bad = (bad_page ? ATK_STATUS_BAD_PAGE : 0) | (bad_seq ? ATK_STATUS_BAD_SEQ : 0) | (bad_len ? ATK_STATUS_BAD_LEN : 0);
    if (bad && a.status) atomicOr(a.status, bad);

#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16, 64);
        l[rt] += __shfl_xor(l[rt], 32, 64);
    }
    if constexpr (MODE == kJoin) {
        // the wavefronts' ranges join in LDS, in their order
        constexpr int kPitch = DP + 4;
        __shared__ float ls_m[NW * RT * 16], ls_l[NW * RT * 16], ls_o[RT * 16 * kPitch];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            if (g == 0) ls_m[(wave * RT + rt) * 16 + n] = m[rt], ls_l[(wave * RT + rt) * 16 + n] = l[rt];
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float to = kNoMax;
            for (int w = 0; w < NW; ++w) to = fmaxf(to, ls_m[(w * RT + rt) * 16 + n]);
            l[rt] = 0.0f;
            for (int w = 0; w < NW; ++w) {
                const float mw = ls_m[(w * RT + rt) * 16 + n];
                l[rt] += ls_l[(w * RT + rt) * 16 + n] * (mw == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((mw - to) * a.scale2));
            }
            if (m[rt] != kNoMax) {
                const float f = __builtin_amdgcn_exp2f((m[rt] - to) * a.scale2);
#pragma unroll
                for (int i = 0; i < NT; ++i) acc[rt][i] *= f;
            }
            m[rt] = to;
        }
        for (int w = 0; w < NW; ++w) {
            if (wave == w) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float *o = ls_o + (rt * 16 + n) * kPitch + (g * 4 + j) * NT + i;
                            if (w > 0) acc[rt][i][j] += *o;
                            if (w < NW - 1) *o = acc[rt][i][j];
                        }
            }
            __syncthreads();
        }
        if (wave != NW - 1) return;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + rt * 16 + n;
        if (r >= n_rows) continue;
        const AttnRow x = attn_row(a, h, r, b);
        const int64_t row = ((int64_t)x.b * a.tokens + x.t) * a.heads + x.head;
        if (whole) {  // nothing to join
            if (g == 0 && a.lse) a.lse[row] = row_lse<ELT>(a, m[rt], l[rt]);
            const float f = 1.0f / l[rt];
            const bool none = l[rt] == 0.0f;  // no key, or scores of -inf alone, whose values do not count even if they are NaN
            char *out = (char *)a.out + (x.b * a.os[0] + x.t * a.os[1] + x.head * a.os[2]) * E::kBytes;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < NT; i += 4) {
                    const int dim = (g * 4 + j) * NT + i;
                    f32x4 o = f32x4{acc[rt][i][j] * f, acc[rt][i + 1][j] * f, acc[rt][i + 2][j] * f, acc[rt][i + 3][j] * f};
                    if (none) o = f32x4{0, 0, 0, 0};
                    if (FULL || dim < a.dim) store_out<ELT>(out + dim * E::kBytes, o);
                }
            continue;
        }
        const int64_t part = (((int64_t)range_at * (MODE == kStaged ? d.subtiles : 1) + sub) * d.row_blocks + block_of) * a.kv_heads * d.pitch + (int64_t)h * d.pitch + (r - block_r0);
        if (g == 0) a.parts_ml[part] = float2{m[rt], l[rt]};
        float *o = a.parts_o + part * a.dim;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < NT; i += 4) {
                const int dim = (g * 4 + j) * NT + i;
                if (FULL || dim < a.dim) *(f32x4 *)(o + dim) = f32x4{acc[rt][i][j], acc[rt][i + 1][j], acc[rt][i + 2][j], acc[rt][i + 3][j]};
            }
    }
}

// Joins the parts of a row: LPR lanes have four elements each, 64 / LPR parts at a time and four of those on their way; one wavefront, or with many parts four that take turns (one
// sequence of 100000 keys, which is cut in 380: 70 us -> 46).
template <int ELT, int LPR, int WAVES>
__global__ __launch_bounds__(256) void quant_join_kernel(const QuantAttnDev d, int rows_of) {
    const AttnDev &a = d.a;
    const int lane = threadIdx.x & 63, wave = WAVES > 1 ? threadIdx.x >> 6 : 0;
    const int64_t row = WAVES > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.batch * a.tokens * a.heads) return;
    const int head = (int)(row % a.heads);
    const int64_t bt = row / a.heads;
    const int b = (int)(bt / a.tokens), t = (int)(bt % a.tokens);
    const int r = t * a.group + head % a.group, block = r / rows_of;
    const int2 share = d.shares[b];
    // a sequence's parts are so far apart
    const int64_t first = (((int64_t)share.x * d.row_blocks + block) * a.kv_heads + head / a.group) * d.pitch + r % rows_of, step = (int64_t)d.row_blocks * a.kv_heads * d.pitch;
    const float2 *ml = a.parts_ml + first;
    float m = kNoMax;
    for (int p = lane; p < share.y; p += 64) m = fmaxf(m, ml[p * step].x);
    for (int w = 1; w < 64; w <<= 1) m = fmaxf(m, __shfl_xor(m, w, 64));
    float l = 0.0f;
    for (int p = lane; p < share.y; p += 64) {
        const float2 x = ml[p * step];
        l += x.y * (x.x == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((x.x - m) * a.scale2));
    }
    for (int w = 1; w < 64; w <<= 1) l += __shfl_xor(l, w, 64);
    const int dim = lane % LPR * 4;
    f32x4 o = {0, 0, 0, 0};
    if (dim < a.dim) {
        constexpr int kStep = 64 / LPR * WAVES;
        const float *from = a.parts_o + first * a.dim + dim;
        for (int p0 = wave * (64 / LPR) + lane / LPR; p0 < share.y; p0 += 4 * kStep) {
            float2 x[4];
            f32x4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int p = min(p0 + j * kStep, share.y - 1);
                x[j] = ml[p * step];
                v[j] = *(const f32x4 *)(from + p * step * a.dim);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (p0 + j * kStep >= share.y) continue;
                const float f = x[j].x == kNoMax ? 1.0f : __builtin_amdgcn_exp2f((x[j].x - m) * a.scale2);
                o += f * v[j];
            }
        }
    }
#pragma unroll
    for (int w = LPR; w < 64; w <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], w, 64);
    if constexpr (WAVES > 1) {
        __shared__ f32x4 sums[WAVES][LPR];
        if (lane < LPR) sums[wave][lane] = o;
        __syncthreads();
        if (wave > 0) return;
        o = sums[0][lane % LPR];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) o += sums[w][lane % LPR];
    }
    if (l == 0.0f) o = f32x4{0, 0, 0, 0};  // no key, or scores of -inf alone, whose values do not count even if they are NaN
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    if (lane < LPR && dim < a.dim) store_out<ELT>((char *)a.out + (b * a.os[0] + t * a.os[1] + head * a.os[2] + dim) * AttnElt<ELT>::kBytes, o * f);
    if (a.lse && lane == 0) a.lse[row] = row_lse<ELT>(a, m, l);
}
template <int ELT, int LPR>
static hipError_t launch_quant_join_of(const QuantAttnDev &d, int rows_of, hipStream_t stream) {
    const int64_t rows = (int64_t)d.a.batch * d.a.tokens * d.a.heads;
    if (d.wide_join)
        hipLaunchKernelGGL((quant_join_kernel<ELT, LPR, 4>), dim3((uint32_t)rows), dim3(256), 0, stream, d, rows_of);
    else
        hipLaunchKernelGGL((quant_join_kernel<ELT, LPR, 1>), dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, stream, d, rows_of);
    return hipGetLastError();
}
template <int ELT>
static hipError_t launch_quant_join(const QuantAttnDev &d, int dp, int rows_of, hipStream_t stream) {
    return dp == 64 ? launch_quant_join_of<ELT, 16>(d, rows_of, stream) : dp == 128 ? launch_quant_join_of<ELT, 32>(d, rows_of, stream) : launch_quant_join_of<ELT, 64>(d, rows_of, stream);
}

constexpr int quant_shared_rt(int elt) { return elt == ATK_F32 ? 1 : 2; }
// Row tiles of a wavefront at most: f32's queries are three operands each.
constexpr int quant_max_rt(int elt, int dp) { return dp == 256 ? (elt == ATK_F32 ? 1 : 2) : elt == ATK_F32 ? 2 : 4; }

template <int ELT, int BITS, int DP, int RT, int MODE, bool FULL>
static hipError_t launch_quant_as(const QuantAttnDev &d, hipStream_t stream) {
    const int64_t groups = MODE == kApart ? ((int64_t)d.units + kQuantWaves - 1) / kQuantWaves : d.units, whole = 8 * (int64_t)d.chunk;
    const int threads = MODE == kStaged ? 64 * d.team * d.subtiles : MODE == kShared ? 64 * kSharedWaves : 64 * kQuantWaves;
    const size_t lds = MODE == kStaged ? (size_t)quant_stage_bytes(d.row_chunks, d.subtiles) : MODE == kShared ? (size_t)quant_shared_bytes(DP) : 0;
    if (MODE == kShared) {  // (more than 64 KB)
        const hipError_t e = hipFuncSetAttribute((const void *)&quant_attn_kernel<ELT, BITS, DP, RT, MODE, FULL>, hipFuncAttributeMaxDynamicSharedMemorySize, quant_shared_bytes(DP));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((quant_attn_kernel<ELT, BITS, DP, RT, MODE, FULL>), dim3((uint32_t)((groups + whole - 1) / whole * whole)), dim3(threads), lds, stream, d);
    return hipGetLastError();
}
template <int ELT, int BITS, int DP, int RT, int MODE>
static hipError_t launch_quant(const QuantAttnDev &d, hipStream_t stream) {
    return d.a.dim == DP ? launch_quant_as<ELT, BITS, DP, RT, MODE, true>(d, stream) : launch_quant_as<ELT, BITS, DP, RT, MODE, false>(d, stream);
}
template <int ELT, int BITS, int DP, int MODE>
static hipError_t launch_quant_rt(const QuantAttnDev &d, int rt, hipStream_t stream) {
    if (rt == 1) return launch_quant<ELT, BITS, DP, 1, MODE>(d, stream);
    if constexpr (MODE != kJoin) {
        if constexpr (quant_max_rt(ELT, DP) >= 4 && MODE != kStaged)
            if (rt == 4) return launch_quant<ELT, BITS, DP, 4, MODE>(d, stream);
        if constexpr (quant_max_rt(ELT, DP) >= 2) return launch_quant<ELT, BITS, DP, 2, MODE>(d, stream);
    }
    return hipErrorInvalidValue;
}
template <int ELT, int BITS, int DP>
static hipError_t launch_quant_mode(const QuantAttnDev &d, int rt, int mode, hipStream_t stream) {
    if (mode == kJoin) return launch_quant_rt<ELT, BITS, DP, kJoin>(d, rt, stream);
    if constexpr (DP <= 128)
        if (mode == kShared) return launch_quant<ELT, BITS, DP, quant_shared_rt(ELT), kShared>(d, stream);
    if constexpr (DP * BITS / 8 < 128)
        if (mode == kStaged) return launch_quant_rt<ELT, BITS, DP, kStaged>(d, rt, stream);
    return launch_quant_rt<ELT, BITS, DP, kApart>(d, rt, stream);
}
template <int ELT>
static hipError_t launch_quant_elt(const QuantAttnDev &d, int bits, int dp, int rt, int mode, hipStream_t stream) {
    hipError_t e = bits == 4 ? (dp == 64 ? launch_quant_mode<ELT, 4, 64>(d, rt, mode, stream) : dp == 128 ? launch_quant_mode<ELT, 4, 128>(d, rt, mode, stream) : launch_quant_mode<ELT, 4, 256>(d, rt, mode, stream))
                             : (dp == 64 ? launch_quant_mode<ELT, 8, 64>(d, rt, mode, stream) : dp == 128 ? launch_quant_mode<ELT, 8, 128>(d, rt, mode, stream) : launch_quant_mode<ELT, 8, 256>(d, rt, mode, stream));
    if (e == hipSuccess && d.ranges) e = launch_quant_join<ELT>(d, dp, 16 * rt * (mode == kShared ? kSharedWaves : 1), stream);
    return e;
}

hipError_t launch_quant_f32(const QuantAttnDev &d, int bits, int dp, int rt, int mode, hipStream_t stream);
hipError_t launch_quant_bf16(const QuantAttnDev &d, int bits, int dp, int rt, int mode, hipStream_t stream);
hipError_t launch_quant_f16(const QuantAttnDev &d, int bits, int dp, int rt, int mode, hipStream_t stream);

}  // namespace atk
