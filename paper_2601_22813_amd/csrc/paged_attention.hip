// Attention of one new token of every sequence over the paged key-value cache (see qii_paged_attention in include/qii.h).
#include <math.h>

#include "kv_cache.h"

namespace qii {
namespace {

constexpr int kWaves = 4;
constexpr int kPerLane = 4;   // elements of a head a lane holds: 64 * 4 >= 256

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// element d of a cached key or value (rows as in qii_kv_cache)
__device__ __forceinline__ float cached(const KvView &c, bool value, int64_t page_head, int slot, int d)
{
    const int64_t row = page_head * c.page_size + slot;
    const uint8_t *buf = value ? c.v : c.k;
    if (!c.nvfp4) return load_elem(reinterpret_cast<const uint16_t *>(buf) + row * c.head_dim + d);
    const int groups = c.head_dim / 16, g = d / 16;
    const uint32_t b = value ? c.v_scales[(page_head * groups + g) * c.page_size + slot] : c.k_scales[row * groups + g];
    const uint32_t code = buf[row * (c.head_dim / 2) + d / 2] >> (4 * (d & 1));
    const float m = e2m1_decode_mag(code & 7u) * e4m3_decode(b);
    return code & 8u ? -m : m;
}

// a block a (sequence, query head); each wave takes every fourth position with a running maximum and sum of its own, and the
// waves are joined in LDS
template <typename T>
__global__ __launch_bounds__(kWaves * 64) void attention_kernel(AttentionArgs a)
{
    __shared__ float part[kWaves][64 * kPerLane], stat[kWaves][2];
    const int seq = blockIdx.x / a.heads, head = blockIdx.x % a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int kv_head = head / (a.heads / a.c.kv_heads), D = a.c.head_dim;
    const int len = min(max(a.lengths[seq], 0), a.max_length);
    int first = a.starts ? max(a.starts[seq], 0) : 0;
    if (a.window && len - a.window > first) first = len - a.window;
    const T *qp = static_cast<const T *>(a.q) + seq * a.qs.token + head * a.qs.head;
    float q[kPerLane], o[kPerLane] = {};
    for (int i = 0; i < kPerLane; ++i) {
        const int d = lane + 64 * i;
        q[i] = d < D ? load_elem(qp + d) : 0.0f;
        if (a.rot.cos_sin && d < 2 * a.rot.pairs && d < D) {
            const bool second = a.rot.interleaved ? d & 1 : d >= a.rot.pairs;
            const int u = a.rot.interleaved ? d >> 1 : second ? d - a.rot.pairs : d;
            const int other = a.rot.interleaved ? d ^ 1 : second ? d - a.rot.pairs : d + a.rot.pairs;
            float c = NAN, s = NAN;
            if (len > 0 && len - 1 < a.rot.positions) {
                c = a.rot.cos_sin[(int64_t)(len - 1) * 2 * a.rot.pairs + u];
                s = a.rot.cos_sin[(int64_t)(len - 1) * 2 * a.rot.pairs + a.rot.pairs + u];
            }
            const float p = load_elem(qp + other);
            q[i] = second ? q[i] * c + p * s : q[i] * c - p * s;
        }
    }
    const float k_scale = a.scale * (a.c.nvfp4 ? *a.c.k_ts : 1.0f);
    float top = -INFINITY, sum = 0.0f;
    for (int j = first + wave; j < len; j += kWaves) {
        const int32_t page = page_of(a.c, seq, j);
        if (page < 0) continue;
        const int64_t page_head = (int64_t)page * a.c.kv_heads + kv_head;
        const int slot = j % a.c.page_size;
        float s = 0.0f;
        for (int i = 0; i < kPerLane; ++i)
            if (lane + 64 * i < D) s += q[i] * cached(a.c, false, page_head, slot, lane + 64 * i);
        s = wave_sum(s) * k_scale;
        const float m = fmaxf(top, s), shift = m == -INFINITY ? 0.0f : m;
        const float old = expf(top - shift), p = expf(s - shift);
        sum = sum * old + p;
        for (int i = 0; i < kPerLane; ++i)
            if (lane + 64 * i < D) o[i] = o[i] * old + p * cached(a.c, true, page_head, slot, lane + 64 * i);
        top = m;
    }
    for (int i = 0; i < kPerLane; ++i) part[wave][lane + 64 * i] = o[i];
    if (lane == 0) { stat[wave][0] = top; stat[wave][1] = sum; }
    __syncthreads();
    if (wave != 0) return;
    float m = -INFINITY;
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stat[w][0]);
    const float shift = m == -INFINITY ? 0.0f : m;
    float total = 0.0f, f[kWaves];
    for (int w = 0; w < kWaves; ++w) {
        f[w] = expf(stat[w][0] - shift);
        total += f[w] * stat[w][1];
    }
    const float v_scale = a.c.nvfp4 ? *a.c.v_ts : 1.0f;
    T *op = static_cast<T *>(a.out) + seq * a.os.token + head * a.os.head;
    for (int i = 0; i < kPerLane; ++i) {
        float r = 0.0f;
        for (int w = 0; w < kWaves; ++w) r += f[w] * part[w][lane + 64 * i];
        if (lane + 64 * i < D) store_elem(op + lane + 64 * i, total == 0.0f ? 0.0f : r / total * v_scale);
    }
    if (a.lse && lane == 0) a.lse[(int64_t)seq * a.heads + head] = m + logf(total);
}

}  // namespace

size_t paged_attention_workspace_bytes(int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_paged_attention(const AttentionArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)a.heads * (unsigned)a.c.seqs;
    if (a.bf16) attention_kernel<uint16_t><<<grid, kWaves * 64, 0, s>>>(a);
    else attention_kernel<float><<<grid, kWaves * 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace qii
