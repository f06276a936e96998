// Attention of one new token of every sequence over the paged key-value cache (see qii_paged_attention in include/qii.h).
#include <math.h>

#include "kv_cache.h"

namespace qii {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4, kThreads = kWaves * 64;
constexpr int kRows = 16;      // query heads of a block: the columns of its matrix instructions
constexpr int kTile = 32;      // positions of a wave's step
constexpr int kMinChunk = 256; // positions of a block at least

struct Launch {
    int units, tiles, group, splits;   // (sequence, key-value head, 16 query heads) triples; row tiles of a head; heads of a group
    uint32_t page16, magic;            // page_size / 16, floor((2^32 - 1) / page16)
    float *part, *stat;                // partial results [row][split][head_dim], their maxima and sums [row][split][2]
};

// ------------------------------------------------------------------------------------------------ lanes
// maximum or sum of the four lanes that hold the same row (lane % 16)
__device__ __forceinline__ float rows_max(float v)
{
    u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false));
    v = fmaxf(u2f(r[0]), u2f(r[1]));
    r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false));
    return fmaxf(u2f(r[0]), u2f(r[1]));
}

__device__ __forceinline__ float rows_sum(float v)
{
    u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false));
    v = u2f(r[0]) + u2f(r[1]);
    r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false));
    return u2f(r[0]) + u2f(r[1]);
}

// ------------------------------------------------------------------------------------------------ 16-bit operands
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return (uint32_t)to_bf16(a) | (uint32_t)to_bf16(b) << 16; }

// piece kPiece of a number as a sum of f16 (kNv) or bf16 numbers, each the nearest to what the ones before leave; v becomes the rest
template <bool kNv>
__device__ __forceinline__ uint32_t next_piece(float &a, float &b)
{
    if constexpr (kNv) {
        const half2_t h = {(_Float16)a, (_Float16)b};
        a -= (float)h[0];
        b -= (float)h[1];
        return __builtin_bit_cast(uint32_t, h);
    } else {
        const uint32_t p = pack_bf16(a, b);
        a -= bf16_lo(p);
        b -= bf16_hi(p);
        return p;
    }
}

template <bool kNv>
__device__ __forceinline__ f32x4 multiply(const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    if constexpr (kNv) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// e2m1 * e4m3 exactly, as f16: (code * 2^8) * (scale * 2^-8), a scale byte b being the f16 with the bits b << 7 times 2^8
template <int kByte>
__device__ __forceinline__ uint32_t dequant(uint32_t codes, uint32_t scale2)
{
    const half2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 256.0f, kByte);
    return __builtin_bit_cast(uint32_t, (half2_t)(c * __builtin_bit_cast(half2_t, scale2)));
}

// ------------------------------------------------------------------------------------------------ a tile in registers
// Lane l (r = l % 16, g = l / 16) holds of the two halves of 16 positions of a tile
//   of the keys    position r, elements key_at(kk) .. + 7 of each step kk of the head dimension: rows of the first operand
//   of the values  positions 4 g + i of both halves, elements r * (DP / 16) ..: columns of the first operand once transposed
template <int DP, bool kNv>
struct Keys {
    static constexpr int kSteps = DP / 32, kWords = kNv ? 1 : 4;
    uint32_t w[2][kSteps][kWords];
    uint32_t scale[2];                 // NVFP4: the scale bytes of its DP / 64 groups
};

template <int DP, bool kNv>
struct Values {
    static constexpr int kWords = kNv ? (DP >= 128 ? DP / 128 : 1) : DP / 32;
    uint32_t w[8][kWords];
    uint32_t scale[2];                 // NVFP4: the scale bytes of its four positions
};

// NVFP4: a lane's 32 bytes of a row lie together (one load); bf16: those of the four lanes of a row do (64 bytes a step)
template <int DP, bool kNv>
__device__ __forceinline__ int key_at(int g, int kk)
{
    return kNv ? g * (DP / 4) + 8 * kk : 32 * kk + 8 * g;
}

template <int kBytes>
__device__ __forceinline__ void load_words(uint32_t *dst, const uint8_t *src)
{
    if constexpr (kBytes == 1) dst[0] = *src;
    else if constexpr (kBytes == 2) dst[0] = *reinterpret_cast<const uint16_t *>(src);
    else if constexpr (kBytes == 4) dst[0] = *reinterpret_cast<const uint32_t *>(src);
    else if constexpr (kBytes == 8) {
        const u32x2 v = *reinterpret_cast<const u32x2 *>(src);
        dst[0] = v[0]; dst[1] = v[1];
    } else {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) {
            const u32x4 v = reinterpret_cast<const u32x4 *>(src)[i];
            dst[4 * i] = v[0]; dst[4 * i + 1] = v[1]; dst[4 * i + 2] = v[2]; dst[4 * i + 3] = v[3];
        }
    }
}

// where a half of 16 positions lies: its page (-1: none) and its first slot there
struct Half { int32_t page; uint32_t slot; };

// kExact: the head dimension is DP; else what is beyond it is zero
template <int DP, bool kNv, bool kExact>
__device__ __forceinline__ void load_keys(Keys<DP, kNv> &k, const KvView &c, int kv_head, const Half half[2], int r, int g)
{
    const int D = kExact ? DP : c.head_dim;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int64_t page_head = (int64_t)(half[s].page < 0 ? 0 : half[s].page) * c.kv_heads + kv_head;
        const int64_t row0 = page_head * c.page_size + half[s].slot;
        if constexpr (kNv) {
            const uint8_t *codes = c.k + row0 * (D / 2), *scales = c.k_scales + row0 * (D / 16);
            if constexpr (kExact) {
                load_words<DP / 8>(&k.w[s][0][0], codes + r * (DP / 2) + g * (DP / 8));
                load_words<DP / 64>(&k.scale[s], scales + r * (DP / 16) + g * (DP / 64));
            } else {
                k.scale[s] = 0;
#pragma unroll
                for (int kk = 0; kk < DP / 32; ++kk) {
                    const int d = key_at<DP, kNv>(g, kk);
                    k.w[s][kk][0] = 0;
                    if (d < D) load_words<4>(&k.w[s][kk][0], codes + r * (D / 2) + d / 2);
                    if (kk % 2 == 0 && d < D) k.scale[s] |= (uint32_t)scales[r * (D / 16) + d / 16] << (4 * kk);
                }
            }
        } else {
            const uint8_t *rows = c.k + row0 * (2 * D);
#pragma unroll
            for (int kk = 0; kk < DP / 32; ++kk) {
                const int d = key_at<DP, kNv>(g, kk);
                if (!kExact) k.w[s][kk][0] = k.w[s][kk][1] = k.w[s][kk][2] = k.w[s][kk][3] = 0;
                if (kExact || d < D) load_words<16>(&k.w[s][kk][0], rows + r * (2 * D) + 2 * d);
            }
        }
    }
}

template <int DP, bool kNv, bool kExact>
__device__ __forceinline__ void load_values(Values<DP, kNv> &v, const KvView &c, int kv_head, const Half half[2], int r, int g)
{
    constexpr int kN = DP / 16;   // elements of a lane
    const int D = kExact ? DP : c.head_dim;
    const bool in = kExact || r * kN < D;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int64_t page_head = (int64_t)(half[s].page < 0 ? 0 : half[s].page) * c.kv_heads + kv_head;
        const int64_t row0 = page_head * c.page_size + half[s].slot;
        const uint8_t *rows = c.v + row0 * (kNv ? D / 2 : 2 * D);
        if (!kExact) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < Values<DP, kNv>::kWords; ++w) v.w[4 * s + i][w] = 0;
            v.scale[s] = 0;
        }
        if (in) {
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words<(kNv ? kN / 2 : kN * 2)>(v.w[4 * s + i], rows + (4 * g + i) * (kNv ? D / 2 : 2 * D) + r * (kNv ? kN / 2 : kN * 2));
            if constexpr (kNv) load_words<4>(&v.scale[s], c.v_scales + (page_head * (D / 16) + r * kN / 16) * c.page_size + half[s].slot + 4 * g);
        }
    }
}

// row kk of the keys' operand of half s
template <int DP, bool kNv>
__device__ __forceinline__ u32x4 key_operand(const Keys<DP, kNv> &k, int s, int kk)
{
    if constexpr (kNv) {
        const uint32_t b = k.scale[s] >> (8 * (kk / 2)) & 0xFFu, s2 = b << 7 | b << 23, w = k.w[s][kk][0];
        return u32x4{dequant<0>(w, s2), dequant<1>(w, s2), dequant<2>(w, s2), dequant<3>(w, s2)};
    } else {
        return u32x4{k.w[s][kk][0], k.w[s][kk][1], k.w[s][kk][2], k.w[s][kk][3]};
    }
}

// The values' operands (bf16): op(j, operand) for each j < DP / 16, whose row r' is element r' * (DP / 16) + j of the head and whose
// columns are the lane's eight positions.  Pairs of positions are put side by side before they are decoded (NVFP4: nibbles, by byte;
// bf16: halves of words).  NVFP4: e2m1 * e4m3 has 6 significant bits, so the upper half of the binary32 product is all of it.
template <int kByte>
__device__ __forceinline__ uint32_t dequant_pair(uint32_t codes, float scale_a, float scale_b)
{
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, kByte);
    return __builtin_amdgcn_perm(f2u(c[1] * scale_b), f2u(c[0] * scale_a), 0x07060302u);
}

template <int DP, bool kNv, typename Op>
__device__ __forceinline__ void for_value_operands(const Values<DP, kNv> &v, Op op)
{
    if constexpr (kNv) {
        float scale[8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            scale[4 * s] = __builtin_amdgcn_cvt_f32_fp8((int)v.scale[s], 0);
            scale[4 * s + 1] = __builtin_amdgcn_cvt_f32_fp8((int)v.scale[s], 1);
            scale[4 * s + 2] = __builtin_amdgcn_cvt_f32_fp8((int)v.scale[s], 2);
            scale[4 * s + 3] = __builtin_amdgcn_cvt_f32_fp8((int)v.scale[s], 3);
        }
#pragma unroll
        for (int w = 0; w < Values<DP, kNv>::kWords; ++w) {
            uint32_t even[4], odd[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = v.w[2 * i][w], b = v.w[2 * i + 1][w];
                even[i] = (a & 0x0F0F0F0Fu) | ((b << 4) & 0xF0F0F0F0u);
                odd[i] = ((a >> 4) & 0x0F0F0F0Fu) | (b & 0xF0F0F0F0u);
            }
#define QII_VALUES(J, C, B)                                                                                                              \
    op(8 * w + J, u32x4{dequant_pair<B>(C[0], scale[0], scale[1]), dequant_pair<B>(C[1], scale[2], scale[3]),                             \
                        dequant_pair<B>(C[2], scale[4], scale[5]), dequant_pair<B>(C[3], scale[6], scale[7])})
            QII_VALUES(0, even, 0); QII_VALUES(1, odd, 0); QII_VALUES(2, even, 1); QII_VALUES(3, odd, 1);
            if constexpr (DP > 64) {   // (a lane's share of 64 elements is half a word)
                QII_VALUES(4, even, 2); QII_VALUES(5, odd, 2); QII_VALUES(6, even, 3); QII_VALUES(7, odd, 3);
            }
#undef QII_VALUES
        }
    } else {
#pragma unroll
        for (int w = 0; w < Values<DP, kNv>::kWords; ++w) {
            u32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = __builtin_amdgcn_perm(v.w[2 * i + 1][w], v.w[2 * i][w], 0x05040100u);
                hi[i] = __builtin_amdgcn_perm(v.w[2 * i + 1][w], v.w[2 * i][w], 0x07060302u);
            }
            op(2 * w, lo);
            op(2 * w + 1, hi);
        }
    }
}

// values of positions that do not count become zeros (what their memory holds may be NaN): valid bit 4 s + i for position i of half s
template <int DP, bool kNv>
__device__ __forceinline__ void clear_values(Values<DP, kNv> &v, uint32_t valid)
{
    if constexpr (kNv) {   // a zero scale and any code
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (!(valid >> (4 * s + i) & 1u)) v.scale[s] &= ~(0xFFu << (8 * i));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int w = 0; w < Values<DP, kNv>::kWords; ++w) v.w[i][w] = valid >> i & 1u ? v.w[i][w] : 0u;
    }
}

// ------------------------------------------------------------------------------------------------ a sequence's share
struct Range { int32_t length, first, chunk, splits; };   // positions [first, length) in chunks from first rounded down to a tile

__device__ __forceinline__ Range range_of(const AttentionArgs &a, int splits, int seq)
{
    Range r;
    r.length = min(max(a.lengths[seq], 0), a.max_length);
    r.first = a.starts ? max(a.starts[seq], 0) : 0;
    if (a.window) r.first = max(r.first, r.length - a.window);
    if (r.first >= r.length) r.first = r.length = 0;   // (a start may be any integer: no position is computed from one beyond the length)
    const int span = r.length - (r.first & ~(kTile - 1));
    constexpr int kStep = kWaves * kTile;
    r.chunk = max(kMinChunk, ((span - 1) / splits / kStep + 1) * kStep);
    r.splits = span > 0 ? (span - 1) / r.chunk + 1 : 1;
    return r;
}

// element d of the (rotated) query in binary32
template <typename T>
__device__ __forceinline__ float query(const AttentionArgs &a, const T *q, int d, int pos)
{
    const float x = load_elem(q + d);
    const int pairs = a.rot.pairs;
    if (!a.rot.cos_sin || d >= 2 * pairs) return a.rot.cos_sin && pos >= a.rot.positions ? NAN : x;
    const bool second = a.rot.interleaved ? d & 1 : d >= pairs;
    const int u = a.rot.interleaved ? d >> 1 : second ? d - pairs : d;
    const float y = load_elem(q + (a.rot.interleaved ? d ^ 1 : second ? d - pairs : d + pairs));
    float c = NAN, s = NAN;
    if (pos >= 0 && pos < a.rot.positions) {
        c = a.rot.cos_sin[(int64_t)pos * 2 * pairs + u];
        s = a.rot.cos_sin[(int64_t)pos * 2 * pairs + pairs + u];
    }
    return second ? x * c + y * s : x * c - y * s;
}

// ------------------------------------------------------------------------------------------------ the kernel
// A block takes 16 query heads of one key-value head of one sequence over one chunk of its positions; each of its waves every fourth tile
// of 32.  A wave computes S^T = K q^T with the keys as first operand, so a lane holds eight scores of ONE row (query head), those of
// the positions whose values it holds: the probabilities are the second operand of O^T += V^T P^T as they are, no lane exchanges
// anything in the loop, and the factor of a raised maximum is the lane's own.
// The maximum is raised only where a score exceeds it by 2^8 or more: probabilities stay below 256, and the sums lose nothing (f32).
template <int DP, bool kNv, typename T, bool kExact>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void attention_kernel(AttentionArgs a, Launch n)
{
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int kSteps = DP / 32, kOut = DP / 16;
    // Pieces of a query and of a probability: f16 keeps 11 bits each, bf16 8.  A rotated query has 24 bits of its own whatever its type.
    // Probabilities are bf16 beside NVFP4 values too: f16 loses those below 2^-14, which is where a result comes from whose other
    // values are zeros.
    constexpr int kQ = kNv ? 2 : kF32 ? 3 : 2, kP = kF32 ? 3 : 2;
    __shared__ float lds[2 * kRows * DP];
    __shared__ float stats[kWaves][2][kRows];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int unit = blockIdx.x % n.units, split = blockIdx.x / n.units;
    const int tile = unit % n.tiles, kv_head = unit / n.tiles % a.c.kv_heads, seq = unit / n.tiles / a.c.kv_heads;
    const Range range = range_of(a, n.splits, seq);
    if (split >= range.splits) return;
    const int rows = min(kRows, n.group - kRows * tile), head0 = kv_head * n.group + kRows * tile;
    const int begin = (range.first & ~(kTile - 1)) + split * range.chunk;
    const int end = min(range.length, begin + range.chunk);
    const int D = kExact ? DP : a.c.head_dim;

    const int32_t *entries = a.c.entries + seq * a.c.entry_stride;
    // (a half that begins at or after the end has no page: its entry may not exist)
    const auto locate = [&](int t, Half half[2]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t p16 = (uint32_t)(t >> 4) + s;
            uint32_t j = __umulhi(p16, n.magic), rest = p16 - j * n.page16;
            if (rest >= n.page16) { ++j; rest -= n.page16; }
            half[s].slot = 16 * rest;
            half[s].page = -1;
            if (t + 16 * s < end) {
                const int32_t p = entries[j];
                half[s].page = (uint32_t)p < (uint32_t)a.c.pages ? p : -1;
            }
            if (half[s].page < 0) half[s].slot = 0;
        }
    };

    Keys<DP, kNv> keys;
    Values<DP, kNv> values;
    Half now[2], next[2];
    int t = begin + wave * kTile;
    locate(t, now);
    locate(t + kWaves * kTile, next);
    if (t < end) {
        load_keys<DP, kNv, kExact>(keys, a.c, kv_head, now, r, g);
        load_values<DP, kNv, kExact>(values, a.c, kv_head, now, r, g);
    }

    // the queries, rotated, through LDS; then each lane's elements of row r, in pieces
    for (int e = threadIdx.x; e < kRows * DP; e += kThreads) {
        const int row = e / DP, d = e % DP;
        float x = 0.0f;
        if (row < rows && d < D) x = query(a, static_cast<const T *>(a.q) + seq * a.qs.token + (head0 + row) * a.qs.head, d, range.length - 1);
        lds[e] = x;
    }
    __syncthreads();
    u32x4 q[kSteps][kQ];
    float factor = a.scale * 1.44269504088896341f * (kNv ? *a.c.k_ts : 1.0f);   // of a score, in units of log2
    {
        float x[kSteps][8], top = 0.0f;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[kk][i] = lds[r * DP + key_at<DP, kNv>(g, kk) + i];
                top = fmaxf(top, fabsf(x[kk][i]));
            }
        if (kNv) {   // f16 has a short range: the row is scaled by a power of two to a maximum in [1, 2)
            top = rows_max(top);
            const int e = top > 0.0f && top < INFINITY ? min(max(ilogbf(top), -126), 126) : 0;
            const float down = ldexpf(1.0f, -e);
            factor *= ldexpf(1.0f, e);
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[kk][i] *= down;
        }
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
            for (int p = 0; p < kQ; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) q[kk][p][i] = next_piece<kNv>(x[kk][2 * i], x[kk][2 * i + 1]);
    }

    f32x4 acc[kOut];
#pragma unroll
    for (int j = 0; j < kOut; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float top = -INFINITY, shift = 0.0f, sum = 0.0f;   // shift: top where that is finite

    for (; t < end; t += kWaves * kTile) {
        f32x4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk) {
                const u32x4 k = key_operand<DP, kNv>(keys, h, kk);
#pragma unroll
                for (int p = 0; p < kQ; ++p) s[h] = multiply<kNv>(k, q[kk][p], s[h]);
            }
        }
        const bool whole = t >= range.first && t + kTile <= end && now[0].page >= 0 && now[1].page >= 0;
        uint32_t valid = 0xFFu;
        if (!whole) {
            valid = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = t + 16 * (i / 4) + 4 * g + (i & 3);
                if (at >= range.first && at < end && now[i / 4].page >= 0) valid |= 1u << i;
            }
        }
        now[0] = next[0];
        now[1] = next[1];
        const bool more = t + kWaves * kTile < end;
        if (more) load_keys<DP, kNv, kExact>(keys, a.c, kv_head, now, r, g);
        locate(t + 2 * kWaves * kTile, next);

        float p[8], most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = s[i / 4][i & 3] * factor;
            if (!whole) p[i] = valid >> i & 1u ? p[i] : -INFINITY;
            most = fmaxf(most, p[i]);
        }
        if (__builtin_amdgcn_ballot_w64(most > top + 8.0f) != 0ull) {
            const float raised = fmaxf(top, rows_max(most));
            const float to = raised == -INFINITY ? 0.0f : raised, by = __builtin_amdgcn_exp2f(top - to);
            top = raised;
            shift = to;
            sum *= by;
#pragma unroll
            for (int j = 0; j < kOut; ++j) acc[j] *= by;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = __builtin_amdgcn_exp2f(p[i] - shift);
            sum += p[i];
        }
        u32x4 w[kP];
#pragma unroll
        for (int k = 0; k < kP; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[k][i] = next_piece<false>(p[2 * i], p[2 * i + 1]);
        if (!whole) clear_values<DP, kNv>(values, valid);
        for_value_operands<DP, kNv>(values, [&](int j, const u32x4 &v) {
#pragma unroll
            for (int k = 0; k < kP; ++k) acc[j] = multiply<false>(v, w[k], acc[j]);
        });
        if (more) load_values<DP, kNv, kExact>(values, a.c, kv_head, now, r, g);
    }

    // the four waves' results under their common maximum: two and two, then one and one
    sum = rows_sum(sum);
    if (g == 0) { stats[wave][0][r] = top; stats[wave][1][r] = sum; }
    __syncthreads();
    float common = -INFINITY, total = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) common = fmaxf(common, stats[w][0][r]);
    const float to = common == -INFINITY ? 0.0f : common;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += stats[w][1][r] * __builtin_amdgcn_exp2f(stats[w][0][r] - to);
    const float by = __builtin_amdgcn_exp2f(top - to);
#pragma unroll
    for (int j = 0; j < kOut; ++j) acc[j] *= by;
    // (a wave's 64 lanes of a register lie side by side)
#pragma unroll
    for (int half = kWaves / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int j = 0; j < kOut; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) lds[((wave - half) * kOut * 4 + 4 * j + i) * 64 + lane] = acc[j][i];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int j = 0; j < kOut; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] += lds[(wave * kOut * 4 + 4 * j + i) * 64 + lane];
        }
        __syncthreads();
    }
    if (wave != 0 || r >= rows) return;
    const int64_t row = (int64_t)seq * a.heads + head0 + r;
    if (range.splits > 1) {   // joined by join_kernel
        float *part = n.part + (row * n.splits + split) * D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kOut; ++j) {
                const int d = (4 * g + i) * kOut + j;
                if (kExact || d < D) part[d] = acc[j][i];
            }
        if (g == 0) {
            n.stat[(row * n.splits + split) * 2] = common;
            n.stat[(row * n.splits + split) * 2 + 1] = total;
        }
        return;
    }
    const float over = total == 0.0f ? 0.0f : (kNv ? *a.c.v_ts : 1.0f) / total;
    T *out = static_cast<T *>(a.out) + seq * a.os.token + (head0 + r) * a.os.head;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kOut; ++j) {
            const int d = (4 * g + i) * kOut + j;
            if (kExact || d < D) store_elem(out + d, acc[j][i] * over);
        }
    if (a.lse && g == 0) a.lse[row] = (common + __builtin_amdgcn_logf(total)) * 0.693147180559945309f;
}

// A block a row (sequence, query head) whose positions several blocks shared: their partial results in the order of the chunks.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(AttentionArgs a, Launch n)
{
    const int row = blockIdx.x, seq = row / a.heads, head = row % a.heads, D = a.c.head_dim;
    const Range range = range_of(a, n.splits, seq);
    if (range.splits <= 1) return;
    const float *stat = n.stat + (int64_t)row * n.splits * 2, *part = n.part + (int64_t)row * n.splits * D;
    float common = -INFINITY, total = 0.0f, x = 0.0f;
    for (int i = 0; i < range.splits; ++i) common = fmaxf(common, stat[2 * i]);
    const float to = common == -INFINITY ? 0.0f : common;
    const int d = threadIdx.x;
    for (int i = 0; i < range.splits; ++i) {
        const float w = __builtin_amdgcn_exp2f(stat[2 * i] - to);
        total += w * stat[2 * i + 1];
        if (d < D) x += w * part[i * D + d];
    }
    const float over = total == 0.0f ? 0.0f : (a.c.nvfp4 ? *a.c.v_ts : 1.0f) / total;
    if (d < D) store_elem(static_cast<T *>(a.out) + seq * a.os.token + head * a.os.head + d, x * over);
    if (a.lse && d == 0) a.lse[row] = (common + __builtin_amdgcn_logf(total)) * 0.693147180559945309f;
}

// Blocks that share a sequence: enough for kBlocks blocks in all, none of them shorter than kMinChunk positions.
int splits_of(int64_t units, int64_t max_length)
{
    constexpr int64_t kBlocks = 2048;
    const int64_t wanted = (kBlocks + units - 1) / units, most = (max_length + kTile - 1) / kMinChunk + 1;
    const int64_t s = wanted < most ? wanted : most;
    return s < 1 ? 1 : (int)s;
}

int64_t units_of(int64_t seqs, int64_t heads, int64_t kv_heads)
{
    const int64_t group = heads / kv_heads;
    return seqs * kv_heads * ((group + kRows - 1) / kRows);
}

template <int DP, bool kNv, typename T>
void launch(const AttentionArgs &a, const Launch &n, hipStream_t s)
{
    const unsigned grid = (unsigned)n.units * (unsigned)n.splits;
    if (a.c.head_dim == DP) attention_kernel<DP, kNv, T, true><<<grid, kThreads, 0, s>>>(a, n);
    else attention_kernel<DP, kNv, T, false><<<grid, kThreads, 0, s>>>(a, n);
}

template <bool kNv, typename T>
void launch_dim(const AttentionArgs &a, const Launch &n, hipStream_t s)
{
    if (a.c.head_dim <= 64) launch<64, kNv, T>(a, n, s);
    else if (a.c.head_dim <= 128) launch<128, kNv, T>(a, n, s);
    else launch<256, kNv, T>(a, n, s);
}

}  // namespace

size_t paged_attention_workspace_bytes(int64_t seqs, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t max_length)
{
    const int splits = splits_of(units_of(seqs, heads, kv_heads), max_length);
    return splits <= 1 ? 0 : (size_t)(seqs * heads * splits * (head_dim + 2)) * sizeof(float);
}

hipError_t launch_paged_attention(const AttentionArgs &a, hipStream_t s)
{
    Launch n;
    n.group = a.heads / a.c.kv_heads;
    n.tiles = (n.group + kRows - 1) / kRows;
    n.units = (int)units_of(a.c.seqs, a.heads, a.c.kv_heads);
    n.page16 = (uint32_t)a.c.page_size / 16;
    n.magic = 0xFFFFFFFFu / n.page16;
    // no more splits than the workspace has room for
    const int64_t rows = (int64_t)a.c.seqs * a.heads, room = (int64_t)(a.ws_bytes / ((size_t)(rows * (a.c.head_dim + 2)) * sizeof(float)));
    const int wanted = splits_of(n.units, a.max_length);
    n.splits = room < wanted ? (room < 1 ? 1 : (int)room) : wanted;
    n.stat = a.ws;
    n.part = a.ws + rows * n.splits * 2;
    if (a.c.nvfp4) {
        if (a.bf16) launch_dim<true, uint16_t>(a, n, s);
        else launch_dim<true, float>(a, n, s);
    } else {
        if (a.bf16) launch_dim<false, uint16_t>(a, n, s);
        else launch_dim<false, float>(a, n, s);
    }
    if (n.splits > 1) {
        if (a.bf16) join_kernel<uint16_t><<<(unsigned)rows, 256, 0, s>>>(a, n);
        else join_kernel<float><<<(unsigned)rows, 256, 0, s>>>(a, n);
    }
    return hipGetLastError();
}

}  // namespace qii
