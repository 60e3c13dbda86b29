// token_logprobs and token_logprobs_grad (include/atk_scores.h).
//
// One pass over a row: each lane keeps a reference r near the largest logit so far, z = sum e^(x - r) and y = sum (x - r) e^(x - r), which change their reference by
//   z' = e^d z,   y' = e^d (y + d z),   d = r - r'
// and join alike; then lse = r + log z and entropy = log z - y / z.  The likeliest tokens come out of the same pass: it leaves the largest logit of each 128 (a "mini"), and with
// ties broken by number the k likeliest tokens lie in the k minis whose largest logits come first (a token outside of them would have k before it).  These are read
// again, and what is not below the k-th mini's largest is ranked: hardly more than k tokens as a rule.
//
// Bound by memory where there are rows for the chip, by the chain of row, minis, tokens where there is one.  64 x 5 rows of 128256 bf16, 82 MB: 25 us without likeliest tokens, 34 with five, 36 to 39 with
// twenty; one row of 32000 f32 9, 11 and 14 us; the gradient of 4096 rows of 32000 bf16, 524 MB: 93 to 102 us (5.1 to 5.6 TB/s).
#include <type_traits>

#include "atk_decode_common.h"
#include "../../include/atk_scores.h"

namespace atk {

constexpr int kMini = 128;            // elements of a mini: 16 lanes' eight
constexpr int kChunk = 512;           // of a wavefront's step
constexpr int kTop = 32;
constexpr int kPlaces = 64;           // (groups of) minis whose tokens are looked at
constexpr int kHeld = 16;             // (groups of) minis of a lane of the wavefront that chooses among them
constexpr int kList = kTop * kMini;   // tokens that may have to be ranked
// (a row by 256, 512, 1024 threads, bf16: 2048 of 32000 30, 31, 47 us, with twenty likeliest 66, 58, 70; 320 of 128256 28, 25, 28 and 44, 38, 39; one of 32000 with twenty 16, 13, 13)
constexpr int kSplitThreads = 256, kRowThreads = 512;
constexpr int64_t kRowMinis = 2048;   // minis that a workgroup keeps in LDS
constexpr float kReach = 4.0f;        // how far the largest logit may be above the reference: e^d is off by |d| 2^-24 and more
constexpr float kLog2e = 1.4426950408889634f;

struct ScoresDev {
    const void *x;
    const int32_t *chosen;
    float *logprobs, *entropy, *lse, *top_logprobs;
    int32_t *top_tokens;
    float4 *stats;   // [row][split]: reference, z, y
    float *minis;    // [row][mini]
    int64_t stride[2], rows;
    int tokens, vocab, top, splits, n_minis, span;  // span: elements of a split, in whole chunks
};

struct Stats {
    float r, z, y;
};
// Changes the reference.  (Nothing yet: z is 0, and d may be anything.)
__device__ __forceinline__ void refer(Stats &s, float to) {
    if (s.z != 0.0f) {
        const float d = s.r - to, f = __builtin_amdgcn_exp2f(d * kLog2e);
        s.y = f > 0.0f ? f * fmaf(d, s.z, s.y) : 0.0f;
        s.z *= f;
    }
    s.r = to;
}
__device__ __forceinline__ void join(Stats &s, Stats t) {
    const float to = fmaxf(s.r, t.r);
    refer(s, to), refer(t, to);
    s.z += t.z, s.y += t.y;
}
constexpr float kNothing = -3.402823466e38f;  // the reference before there is one: finite, so that -inf is below it

// Numbers whose order as unsigned integers is that of the floats; NaN is -inf's.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = x != x ? 0xff800000u : x == 0.0f ? 0u : __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

template <int ELT>
__device__ __forceinline__ float logit(const void *row, int i) {
    if (ELT == ATK_F32) return ((const float *)row)[i];
    if (ELT == ATK_F16) return (float)((const _Float16 *)row)[i];
    return __uint_as_float((uint32_t)((const uint16_t *)row)[i] << 16);
}

// Rows begin at any element, so these are pieces of 16 bytes that lie on an element's boundary.
typedef uint32_t u32x4_on4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_on2 __attribute__((ext_vector_type(4), aligned(2)));
template <int ELT>
struct Piece { typedef u32x4_on2 T; };
template <>
struct Piece<ATK_F32> { typedef u32x4_on4 T; };

// Eight logits of a lane.
template <int ELT>
struct Logits8 {
    static constexpr int kWords = ELT == ATK_F32 ? 8 : 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void *row, int i) {
        typedef typename Piece<ELT>::T u32x4e;
        const char *p = (const char *)row + (int64_t)i * (ELT == ATK_F32 ? 4 : 2);
#pragma unroll
        for (int v = 0; v < kWords / 4; ++v) {
            const u32x4e t = ((const u32x4e *)p)[v];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * v + j] = t[j];
        }
    }
    // the row's last ones: -inf behind its end
    __device__ __forceinline__ void load_end(const void *row, int i, int n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t b;
            if (ELT == ATK_F32)
                b = i + j < n ? ((const uint32_t *)row)[i + j] : 0xff800000u;
            else
                b = i + j < n ? ((const uint16_t *)row)[i + j] : ELT == ATK_F16 ? 0xfc00u : 0xff80u;
            if (ELT == ATK_F32)
                w[j] = b;
            else
                w[j / 2] = j & 1 ? w[j / 2] | b << 16 : b;
        }
    }
    __device__ __forceinline__ float get(int j) const {
        if (ELT == ATK_F32) return __uint_as_float(w[j % kWords]);
        if (ELT == ATK_F16) {
            typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
            const uint32_t b = w[j / 2];
            return (float)__builtin_bit_cast(f16x2, b)[j & 1];
        }
        return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    }
};

// Over the 16 lanes of a mini, by rotations of them that cost no LDS.
template <int N>
__device__ __forceinline__ float rotated(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float max_of_16(float v) {
    v = fmaxf(v, rotated<8>(v));
    v = fmaxf(v, rotated<4>(v));
    v = fmaxf(v, rotated<2>(v));
    return fmaxf(v, rotated<1>(v));
}
// Over the wavefront, in a scalar: shifts within 16 lanes, then the last lane of those to the next ones.
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max_with<0x142>(max_with<0x118>(max_with<0x114>(max_with<0x112>(max_with<0x111>(v)))));
    return (uint32_t)__builtin_amdgcn_readlane((int)max_with<0x143>(v), 63);
}

// Elements from .. to - 1 of a row by the workgroup's wavefronts (from: whole chunks); mini's largest logits to minis[] from `from` / kMini on.
template <int ELT, bool TOP, int THREADS>
__device__ __forceinline__ Stats scan_row(const void *row, int from, int to, float *minis) {
    constexpr int kWaves = THREADS / 64, kAtOnce = ELT == ATK_F32 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Stats s{kNothing, 0.0f, 0.0f};
    auto take = [&](const Logits8<ELT> &v, int at) {
        float x[8], most = kNothing;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = v.get(j);
        float top = fmaxf(x[0], x[1]);
#pragma unroll
        for (int j = 2; j < 8; ++j) top = fmaxf(top, x[j]);
        most = fmaxf(most, top);
        if (TOP) {
            const float m = max_of_16(top);
            if ((lane & 15) == 0 && at < to) minis[at / kMini] = m;
        }
        if (most > s.r + kReach) refer(s, most);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = x[j] - s.r, e = __builtin_amdgcn_exp2f(d * kLog2e);
            s.z += e;
            s.y = fmaf(fmaxf(d, kNothing), e, s.y);  // (-inf * 0 is no number)
        }
    };
    int c = from + wave * kChunk;
    for (; c + ((kAtOnce - 1) * kWaves + 1) * kChunk <= to; c += kAtOnce * kWaves * kChunk) {
        Logits8<ELT> v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) v[j].load(row, c + j * kWaves * kChunk + lane * 8);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) take(v[j], c + j * kWaves * kChunk + lane * 8);
    }
    for (; c < to; c += kWaves * kChunk) {
        const int at = c + lane * 8;
        Logits8<ELT> v;
        if (at + 8 <= to)
            v.load(row, at);
        else
            v.load_end(row, at, to);
        take(v, at);
    }
    return s;
}

// The workgroup's sum, in every thread.
template <int THREADS>
__device__ __forceinline__ Stats join_threads(Stats s) {
    __shared__ Stats waves[THREADS / 64];
    for (int w = 1; w < 64; w <<= 1) join(s, Stats{__shfl_xor(s.r, w, 64), __shfl_xor(s.z, w, 64), __shfl_xor(s.y, w, 64)});
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
    __syncthreads();
    s = waves[0];
    for (int w = 1; w < THREADS / 64; ++w) join(s, waves[w]);
    return s;
}

// What a row's sums give, and its likeliest tokens.  minis: in LDS or not.
template <int ELT, bool TOP, int THREADS>
__device__ __forceinline__ void finish_row(const ScoresDev &a, int64_t r, const void *row, Stats s, const float *minis) {
    // (a logit's distance from the reference is small where its probability is not, whatever its size; from lse it would be off by |lse| 2^-24, all of it in rows of the type's lowest value)
    const float log_z = logf(s.z);
    auto log_p = [&](float x) { return s.z == 0.0f ? -__builtin_inff() : x - s.r - log_z; };
    if (threadIdx.x == 0) {
        const int t = a.chosen[r];
        a.logprobs[r] = (unsigned)t < (unsigned)a.vocab ? log_p(logit<ELT>(row, t)) : -__builtin_inff();
        a.lse[r] = s.z == 0.0f ? -__builtin_inff() : s.r + log_z;
        a.entropy[r] = s.z == 0.0f ? 0.0f : log_z - s.y / s.z;
    }
    if constexpr (TOP) {
        __shared__ int places[kPlaces], wanted;
        __shared__ uint32_t least;
        __shared__ int count;
        __shared__ uint64_t list[kList];
        const int lane = threadIdx.x & 63;
        // groups of minis, as many as one wavefront holds; groups of a lane are next to each other, so of equal ones the lowest lane's comes first
        int per = 1;
        while ((a.n_minis + per - 1) / per > 64 * kHeld) per *= 2;
        const int groups = (a.n_minis + per - 1) / per;
        if (threadIdx.x == 0) count = 0;
        if (threadIdx.x < 64) {
            const int held = (groups + 63) / 64;
            uint32_t key[kHeld], best = 0;
            int where = 0;
            float most_of[kHeld];
#pragma unroll
            for (int i = 0; i < kHeld; ++i) most_of[i] = -__builtin_inff();
#pragma unroll 1
            for (int j = 0; j < per; ++j)
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (i < held) most_of[i] = fmaxf(most_of[i], minis[min((lane * held + i) * per + j, a.n_minis - 1)]);
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                key[i] = i < held && lane * held + i < groups ? key_of(most_of[i]) : 0;  // (0 is below all keys: that of -inf is 0x007fffff)
                if (key[i] > best) best = key[i], where = i;
            }
            // The `top`-th largest of the lanes' best keys is one that `top` tokens reach, so all that count are in groups that reach it: as a rule hardly more than `top` of them.  For a few tokens
            // the groups one after the other are as fast (one row of 32000, five: 11.8 us against 13.0; 8 rows of 128256, twenty: 21.0 against 18.7).
            int n = kPlaces + 1;
            uint32_t reach = 0;
            if (a.top > 8) {
                int rank = 0;
#pragma unroll 8
                for (int w = 0; w < 64; ++w) {
                    const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)best, w);
                    rank += o > best || (o == best && w < lane);
                }
                reach = (uint32_t)__builtin_amdgcn_readlane((int)best, __builtin_ctzll(__ballot(rank == a.top - 1)));  // (0, if fewer lanes than that have a group)
                n = 0;
#pragma unroll
                for (int i = 0; i < kHeld; ++i) {
                    const bool in = key[i] > 0 && key[i] >= reach;
                    const uint64_t all = __ballot(in);
                    const int at = n + __popcll(all & ((uint64_t)1 << lane) - 1);
                    if (in && at < kPlaces) places[at] = lane * held + i;
                    n += __popcll(all);
                }
            }
            if (n <= kPlaces) {
                if (lane == 0) wanted = n, least = reach;
            } else {
                // a few, or many that are alike: the first `top` groups, one after the other
                const int first_few = min(a.top, groups);
                for (int k = 0; k < first_few; ++k) {
                    const uint32_t most = wave_max(best);
                    const int first = __builtin_ctzll(__ballot(best == most));
                    if (lane == first) {
                        places[k] = lane * held + where;
                        best = 0;
                        int next = 0;
#pragma unroll
                        for (int i = 0; i < kHeld; ++i) {
                            if (i == where) key[i] = 0;
                            if (key[i] > best) best = key[i], next = i;
                        }
                        where = next;
                    }
                    if (lane == 0 && k == first_few - 1) wanted = first_few, least = a.top <= groups ? most : 0u;
                }
            }
        }
        __syncthreads();
        // tokens that come into question; where more might come than there is room for, the k first of those so far are kept
        const int size = per * kMini, bits = 31 - __builtin_clz(size);
        uint32_t floor_key = least;
        auto sort = [&]() {  // descending, by all threads
            const int n = count;
            int two = 1;
            while (two < n) two *= 2;
            for (int i = n + threadIdx.x; i < two; i += THREADS) list[i] = 0;
            __syncthreads();
            for (int k = 2; k <= two; k *= 2)
                for (int j = k / 2; j > 0; j /= 2) {
                    for (int i = threadIdx.x; i < two; i += THREADS) {
                        const int o = i ^ j;
                        if (o > i) {
                            const uint64_t x = list[i], y = list[o];
                            if ((x < y) == ((i & k) == 0)) list[i] = y, list[o] = x;
                        }
                    }
                    __syncthreads();
                }
        };
        const int step = kList / 2;
#pragma unroll 1
        for (int e0 = 0; e0 < wanted * size; e0 += step) {
            if (wanted * size > kList && e0 > 0) {
                __syncthreads();
                const bool full = count > kList - step;
                __syncthreads();  // (all have seen it before any of them adds to it)
                if (full) {
                    sort();
                    floor_key = max(floor_key, (uint32_t)(list[a.top - 1] >> 32));
                    __syncthreads();
                    if (threadIdx.x == 0) count = a.top;
                    __syncthreads();
                }
            }
            for (int e = e0 + threadIdx.x; e < min(e0 + step, wanted * size); e += THREADS) {
                const int i = (places[e >> bits] << bits) + (e & (size - 1));
                if (i >= a.vocab) continue;
                const uint32_t key = key_of(logit<ELT>(row, i));
                if (key >= floor_key) list[atomicAdd(&count, 1)] = (uint64_t)key << 32 | (uint32_t)~i;
            }
        }
        __syncthreads();
        const int n = count;
        auto put = [&](int k, uint64_t x) {
            a.top_tokens[r * a.top + k] = (int)~(uint32_t)x;
            a.top_logprobs[r * a.top + k] = log_p(of_key((uint32_t)(x >> 32)));
        };
        if (n <= 256) {
            for (int i = threadIdx.x; i < n; i += THREADS) {
                const uint64_t x = list[i];
                int rank = 0;
#pragma unroll 4
                for (int j = 0; j < n; ++j) rank += list[j] > x;
                if (rank < a.top) put(rank, x);
            }
        } else {
            sort();
            for (int k = threadIdx.x; k < a.top; k += THREADS) put(k, list[k]);
        }
    }
}

template <int ELT>
__device__ __forceinline__ const void *row_of(const ScoresDev &a, int64_t r) {
    return (const char *)a.x + (r / a.tokens * a.stride[0] + r % a.tokens * a.stride[1]) * (ELT == ATK_F32 ? 4 : 2);
}

template <int ELT, bool TOP>
__global__ __launch_bounds__(kRowThreads) void scores_row_kernel(const ScoresDev a) {
    __shared__ float minis[TOP ? kRowMinis : 1];
    const int64_t r = blockIdx.x;
    const void *row = row_of<ELT>(a, r);
    const Stats s = join_threads<kRowThreads>(scan_row<ELT, TOP, kRowThreads>(row, 0, a.vocab, minis));
    finish_row<ELT, TOP, kRowThreads>(a, r, row, s, minis);
}

template <int ELT, bool TOP>
__global__ __launch_bounds__(kSplitThreads) void scores_split_kernel(const ScoresDev a) {
    const int64_t r = blockIdx.x / a.splits;
    const int split = (int)(blockIdx.x % a.splits), from = split * a.span;
    const Stats s = join_threads<kSplitThreads>(scan_row<ELT, TOP, kSplitThreads>(row_of<ELT>(a, r), from, min(a.vocab, from + a.span), TOP ? a.minis + r * a.n_minis : nullptr));
    if (threadIdx.x == 0) a.stats[r * a.splits + split] = float4{s.r, s.z, s.y, 0.0f};
}

template <int ELT, bool TOP>
__global__ __launch_bounds__(kSplitThreads) void scores_finish_kernel(const ScoresDev a) {
    const int64_t r = blockIdx.x;
    Stats s{kNothing, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < a.splits; i += kSplitThreads) {
        const float4 t = a.stats[r * a.splits + i];
        join(s, Stats{t.x, t.y, t.z});
    }
    s = join_threads<kSplitThreads>(s);
    finish_row<ELT, TOP, kSplitThreads>(a, r, row_of<ELT>(a, r), s, TOP ? a.minis + r * a.n_minis : nullptr);
}

// ---------------------------------------------------------------------------------------------------------------- gradient
struct GradDev {
    const void *x;
    void *grad;
    const int32_t *chosen;
    const float *lse, *entropy, *a, *b;
    int64_t xs[2], gs[2];
    int tokens, vocab, pieces;
};
constexpr int kGradThreads = 256, kGradPiece = kGradThreads * 8 * 4;
// From here on p = e^(x - lse) is off by more than 2^-14 through lse's rounding to f32, half a step of |lse| 2^-23 (in a row of the type's lowest value it is 1 for every token).  A row with such an lse
// is summed up first: log sum e^(x - lse) is what the rounding took, if it is no more than a rounding takes (an lse that is not these logits' own is taken as it is).  |lse| below it: 2^-24 of
// it at most, as any function of an lse in f32.
constexpr float kFarLse = 1024.0f;

template <int ELT>
__device__ __forceinline__ void store_logits8(void *row, int i, const float *x) {
    typedef typename Piece<ELT>::T u32x4e;
    char *p = (char *)row + (int64_t)i * (ELT == ATK_F32 ? 4 : 2);
    if constexpr (ELT == ATK_F32) {
#pragma unroll
        for (int v = 0; v < 2; ++v)
            ((u32x4e *)p)[v] = u32x4e{__float_as_uint(x[4 * v]), __float_as_uint(x[4 * v + 1]), __float_as_uint(x[4 * v + 2]), __float_as_uint(x[4 * v + 3])};
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (ELT == ATK_F16) {
                typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
                w[j] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x[2 * j], (_Float16)x[2 * j + 1]});
            } else {
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                w[j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * j], (__bf16)x[2 * j + 1]});
            }
        }
        *(u32x4e *)p = u32x4e{w[0], w[1], w[2], w[3]};
    }
}
template <int ELT>
__device__ __forceinline__ void store_logit(void *row, int i, float x) {
    if constexpr (ELT == ATK_F32)
        ((float *)row)[i] = x;
    else if constexpr (ELT == ATK_F16)
        ((_Float16 *)row)[i] = (_Float16)x;
    else
        ((__bf16 *)row)[i] = (__bf16)x;
}

template <int ELT>
__global__ __launch_bounds__(kGradThreads) void scores_grad_kernel(const GradDev d) {
    constexpr int es = ELT == ATK_F32 ? 4 : 2, kAtOnce = 4;
    const int64_t r = blockIdx.x / d.pieces;
    const int from = (int)(blockIdx.x % d.pieces) * kGradPiece;
    const void *row = (const char *)d.x + (r / d.tokens * d.xs[0] + r % d.tokens * d.xs[1]) * es;
    void *out = (char *)d.grad + (r / d.tokens * d.gs[0] + r % d.tokens * d.gs[1]) * es;
    const int t = d.chosen[r];
    const float lse = d.lse[r], b = d.b ? d.b[r] : 0.0f, h = d.b ? d.entropy[r] : 0.0f;
    const float a = d.a && (unsigned)t < (unsigned)d.vocab ? d.a[r] : 0.0f;
    const bool none = lse == -__builtin_inff();
    const bool far = fabsf(lse) >= kFarLse && fabsf(lse) < __builtin_inff();
    float more = 0.0f;
    auto of = [&](float x, int i) {
        const float l = x - lse - more, p = __builtin_amdgcn_exp2f(l * kLog2e);
        float g = p == 0.0f ? 0.0f : -p * fmaf(b, l + h, a);  // (0 * -inf is no number)
        if (i == t) g += a;
        return none ? 0.0f : g;
    };
    // whole: all of the piece is in the row, so that all loads go out before the branch, which waits for lse (with lanes' conditions around each, f16 rows took 54 us for 47)
    auto ordinary = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        Logits8<ELT> v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int i = from + (j * kGradThreads + (int)threadIdx.x) * 8;
            if (WHOLE || i + 8 <= d.vocab) v[j].load(row, i);
        }
        if (far) return;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int i = from + (j * kGradThreads + (int)threadIdx.x) * 8;
            if (WHOLE || i + 8 <= d.vocab) {
                float g[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) g[k] = of(v[j].get(k), i + k);
                store_logits8<ELT>(out, i, g);
            } else {
                for (int k = i; k < d.vocab; ++k) store_logit<ELT>(out, k, of(logit<ELT>(row, k), k));
            }
        }
    };
    if (from + kGradPiece <= d.vocab)
        ordinary(std::true_type{});
    else
        ordinary(std::false_type{});
    // one workgroup for the whole row, which may be the gradient's own memory: all of it is read before any is written (not always the row's first one: these can all be of one XCD; 2048 rows of 32000
    // bf16 181 us where all are like this, 47 where none is)
    if (!far || blockIdx.x % d.pieces != r % d.pieces) return;
    __shared__ float waves[kGradThreads / 64];
    float z = 0.0f;
#pragma unroll 8
    for (int i = threadIdx.x; i < d.vocab; i += kGradThreads) z += __builtin_amdgcn_exp2f((logit<ELT>(row, i) - lse) * kLog2e);
    for (int w = 1; w < 64; w <<= 1) z += __shfl_xor(z, w, 64);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = z;
    __syncthreads();
    z = 0.0f;
#pragma unroll
    for (int w = 0; w < kGradThreads / 64; ++w) z += waves[w];
    more = logf(z);
    if (!(fabsf(more) <= fabsf(lse) * 0x1p-23f)) more = 0.0f;
#pragma unroll 8
    for (int i = threadIdx.x; i < d.vocab; i += kGradThreads) store_logit<ELT>(out, i, of(logit<ELT>(row, i), i));
}

// ---------------------------------------------------------------------------------------------------------------- host
static int64_t scores_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct ScoresPlan {
    bool by_row;
    int64_t splits, span, minis, stats_bytes, bytes;
};
static int plan_scores(int64_t batch, int64_t tokens, int64_t vocab, int64_t top, int dtype, ScoresPlan *pl) {
    if (dtype != ATK_F32 && dtype != ATK_BF16 && dtype != ATK_F16) return ATK_ERR_DTYPE;
    if (batch < 1 || tokens < 1 || vocab < 1 || batch > (1 << 30) || tokens > (1 << 30) || vocab > (1 << 24) || top < 0 || top > kTop || top > vocab) return ATK_ERR_ARGS;
    const int64_t rows = batch * tokens;
    if (!launches(rows, kRowThreads)) return ATK_ERR_ARGS;
    pl->minis = scores_ceil(vocab, kMini);
    const int64_t chunks = scores_ceil(vocab, kChunk);
    // One workgroup a row in one launch, or splits of 16 chunks at least and eight workgroups a CU at most in two.  bf16, twenty likeliest: one row of 32000 13 us by row and 15 split, of 64000 16.5 and 16, of
    // 128256 23 and 17; 16 of 128256 24 and 18, 64 25 and 25, 128 26 and 29, 256 28 and 36, 320 38 and 42, 2048 118 and 149.  Splits of 8 chunks, or four workgroups a CU: level within 6 %.
    pl->by_row = pl->minis <= kRowMinis && (rows >= kNumCU || chunks <= 64);
    pl->splits = pl->by_row ? 1 : std::max<int64_t>(1, std::min(scores_ceil(chunks, 16), scores_ceil(8 * kNumCU, rows)));
    pl->span = scores_ceil(chunks, pl->splits) * kChunk;
    pl->splits = scores_ceil(vocab, pl->span);
    if (!launches(rows * pl->splits, kSplitThreads)) return ATK_ERR_ARGS;
    pl->stats_bytes = pl->by_row ? 0 : rows * pl->splits * (int64_t)sizeof(float4);
    pl->bytes = pl->by_row ? 16 : pl->stats_bytes + (top ? scores_ceil(rows * pl->minis * 4, 16) * 16 : 0);
    return ATK_OK;
}

template <int ELT, bool TOP>
static hipError_t launch_scores(const ScoresDev &a, bool by_row, hipStream_t s) {
    if (by_row) {
        hipLaunchKernelGGL((scores_row_kernel<ELT, TOP>), dim3((uint32_t)a.rows), dim3(kRowThreads), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((scores_split_kernel<ELT, TOP>), dim3((uint32_t)(a.rows * a.splits)), dim3(kSplitThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((scores_finish_kernel<ELT, TOP>), dim3((uint32_t)a.rows), dim3(kSplitThreads), 0, s, a);
    return hipGetLastError();
}
template <int ELT>
static hipError_t launch_scores_elt(const ScoresDev &a, bool by_row, hipStream_t s) {
    return a.top ? launch_scores<ELT, true>(a, by_row, s) : launch_scores<ELT, false>(a, by_row, s);
}

}  // namespace atk

using namespace atk;

extern "C" {

int64_t atk_token_logprobs_workspace_bytes(int64_t batch, int64_t tokens, int64_t vocab, int64_t top, int dtype) {
    ScoresPlan pl;
    const int rc = plan_scores(batch, tokens, vocab, top, dtype, &pl);
    return rc == ATK_OK ? pl.bytes : rc;
}

int atk_token_logprobs(const void *logits, const int64_t stride[2], const int32_t *chosen, int64_t batch, int64_t tokens, int64_t vocab, int64_t top, int dtype, float *logprobs,
                       float *entropy, float *lse, float *top_logprobs, int32_t *top_tokens, void *work, int64_t work_bytes, void *stream) {
    ScoresPlan pl;
    const int rc = plan_scores(batch, tokens, vocab, top, dtype, &pl);
    if (rc != ATK_OK) return rc;
    if (!logits || !stride || !chosen || !logprobs || !entropy || !lse || !work || (top > 0 && (!top_logprobs || !top_tokens))) return ATK_ERR_NULL_PTR;
    if ((uintptr_t)logits & (dtype == ATK_F32 ? 3 : 1)) return ATK_ERR_ALIGN;
    if (((uintptr_t)chosen | (uintptr_t)logprobs | (uintptr_t)entropy | (uintptr_t)lse | (uintptr_t)top_logprobs | (uintptr_t)top_tokens) & 3) return ATK_ERR_ALIGN;
    if ((uintptr_t)work & 15) return ATK_ERR_ALIGN;
    if (work_bytes < pl.bytes) return ATK_ERR_WORKSPACE;
    if (stride[0] < 0 || stride[1] < 0) return ATK_ERR_ARGS;
    ScoresDev a;
    a.x = logits, a.chosen = chosen, a.logprobs = logprobs, a.entropy = entropy, a.lse = lse, a.top_logprobs = top_logprobs, a.top_tokens = top_tokens;
    a.stats = (float4 *)work, a.minis = (float *)((char *)work + pl.stats_bytes);
    a.stride[0] = stride[0], a.stride[1] = stride[1], a.rows = batch * tokens;
    a.tokens = (int)tokens, a.vocab = (int)vocab, a.top = (int)top, a.splits = (int)pl.splits, a.n_minis = (int)pl.minis, a.span = (int)pl.span;
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t e = dtype == ATK_F32 ? launch_scores_elt<ATK_F32>(a, pl.by_row, s) : dtype == ATK_BF16 ? launch_scores_elt<ATK_BF16>(a, pl.by_row, s) : launch_scores_elt<ATK_F16>(a, pl.by_row, s);
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

int atk_token_logprobs_grad(const void *logits, const int64_t stride[2], const int32_t *chosen, const float *lse, const float *entropy, const float *grad_logprobs, const float *grad_entropy,
                            int64_t batch, int64_t tokens, int64_t vocab, int dtype, void *grad, const int64_t grad_stride[2], void *stream) {
    ScoresPlan pl;
    const int rc = plan_scores(batch, tokens, vocab, 0, dtype, &pl);
    if (rc != ATK_OK) return rc;
    const int64_t pieces = scores_ceil(vocab, kGradPiece);
    if (!launches(batch * tokens * pieces, kGradThreads)) return ATK_ERR_ARGS;
    if (!logits || !stride || !chosen || !lse || !grad || !grad_stride || (grad_entropy && !entropy)) return ATK_ERR_NULL_PTR;
    if (((uintptr_t)logits | (uintptr_t)grad) & (dtype == ATK_F32 ? 3 : 1)) return ATK_ERR_ALIGN;
    if (((uintptr_t)chosen | (uintptr_t)lse | (uintptr_t)entropy | (uintptr_t)grad_logprobs | (uintptr_t)grad_entropy) & 3) return ATK_ERR_ALIGN;
    GradDev d;
    d.x = logits, d.grad = grad, d.chosen = chosen, d.lse = lse, d.entropy = entropy, d.a = grad_logprobs, d.b = grad_entropy;
    for (int i = 0; i < 2; ++i) {
        if (stride[i] < 0 || grad_stride[i] < 0) return ATK_ERR_ARGS;
        d.xs[i] = stride[i], d.gs[i] = grad_stride[i];
    }
    if ((batch > 1 && grad_stride[0] < vocab) || (tokens > 1 && grad_stride[1] < vocab)) return ATK_ERR_ARGS;  // (rows over each other)
    d.tokens = (int)tokens, d.vocab = (int)vocab, d.pieces = (int)pieces;
    const dim3 grid((uint32_t)(batch * tokens * pieces)), threads(kGradThreads);
    const hipStream_t s = (hipStream_t)stream;
    if (dtype == ATK_F32)
        hipLaunchKernelGGL(scores_grad_kernel<ATK_F32>, grid, threads, 0, s, d);
    else if (dtype == ATK_BF16)
        hipLaunchKernelGGL(scores_grad_kernel<ATK_BF16>, grid, threads, 0, s, d);
    else
        hipLaunchKernelGGL(scores_grad_kernel<ATK_F16>, grid, threads, 0, s, d);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ATK_OK : set_hip_error(e);
}

}  // extern "C"
