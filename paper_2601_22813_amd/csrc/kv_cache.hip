// Keys and values of new tokens into the paged cache, and cached positions back as dense rows (see qii_kv_append, qii_kv_read in
// include/qii.h).
#include "kv_cache.h"
#include "quantize_core.h"

namespace qii {
namespace {

constexpr int kThreads = 256;

// the tensor constants of quantize_core.h for a given tensor scale (the divisions are the full IEEE ones: nothing is known of the
// magnitudes before they are read)
__device__ __forceinline__ TensorConsts consts_of_scale(float x32)
{
    TensorConsts tc;
    tc.x32 = x32;
    tc.d = x32 * 6.0f;
    tc.d4 = x32 * 4.0f;
    tc.rd = tc.rd4 = 0.0f;
    tc.zero = false;
    tc.fast = false;
    return tc;
}

// one thread a group of 16 elements of a token's key or value
template <typename T, int kMode>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a)
{
    const int groups = a.c.head_dim / 16;
    const int64_t per = (int64_t)a.c.kv_heads * groups, total = a.tokens * 2 * per;
    for (int64_t n = blockIdx.x * (int64_t)kThreads + threadIdx.x; n < total; n += (int64_t)gridDim.x * kThreads) {
        const int g = (int)(n % groups), h = (int)(n / groups % a.c.kv_heads), value = (int)(n / per & 1);
        const int64_t t = n / (2 * per);
        const int32_t pos = a.positions[t];
        const int32_t page = page_of(a.c, a.seqs ? a.seqs[t] : (int32_t)t, pos);
        if (page < 0 || (a.rot.cos_sin && pos >= a.rot.positions)) continue;
        const T *x = value ? static_cast<const T *>(a.v) + t * a.vs.token + h * a.vs.head
                           : static_cast<const T *>(a.k) + t * a.ks.token + h * a.ks.head;
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = load_elem(x + 16 * g + i);
        if (!value && a.rot.cos_sin) {
            const float *cs = a.rot.cos_sin + (int64_t)pos * 2 * a.rot.pairs;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int d = 16 * g + i;
                if (d >= 2 * a.rot.pairs) continue;
                const bool second = a.rot.interleaved ? d & 1 : d >= a.rot.pairs;
                const int u = a.rot.interleaved ? d >> 1 : second ? d - a.rot.pairs : d;
                const int other = a.rot.interleaved ? d ^ 1 : second ? d - a.rot.pairs : d + a.rot.pairs;
                const float o = load_elem(x + other), c = cs[u], s = cs[a.rot.pairs + u];
                y[i] = second ? y[i] * c + o * s : y[i] * c - o * s;
            }
        }
        const int slot = pos % a.c.page_size;
        const int64_t row = ((int64_t)page * a.c.kv_heads + h) * a.c.page_size + slot;
        uint8_t *buf = value ? a.c.v : a.c.k;
        if (!a.c.nvfp4) {
            uint16_t *out = reinterpret_cast<uint16_t *>(buf) + row * a.c.head_dim + 16 * g;
            for (int i = 0; i < 16; ++i) store_elem(out + i, y[i]);
            continue;
        }
        uint32_t packed[2];
        const uint32_t b = quantize_group16<kMode, 0>(y, consts_of_scale(value ? *a.c.v_ts : *a.c.k_ts), 0, 0, 0, 0, packed);
        *reinterpret_cast<uint2 *>(buf + row * (a.c.head_dim / 2) + 8 * g) = uint2{packed[0], packed[1]};
        if (value) a.c.v_scales[(((int64_t)page * a.c.kv_heads + h) * groups + g) * a.c.page_size + slot] = (uint8_t)b;
        else a.c.k_scales[row * groups + g] = (uint8_t)b;
    }
}

// one thread a group of 16 elements of a key or value
template <typename T>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a)
{
    const int groups = a.c.head_dim / 16;
    const int64_t per = (int64_t)a.c.kv_heads * groups, total = a.tokens * 2 * per;
    for (int64_t n = blockIdx.x * (int64_t)kThreads + threadIdx.x; n < total; n += (int64_t)gridDim.x * kThreads) {
        const int g = (int)(n % groups), h = (int)(n / groups % a.c.kv_heads), value = (int)(n / per & 1);
        const int64_t t = n / (2 * per);
        T *y = static_cast<T *>(value ? a.v : a.k);
        if (!y) continue;
        y += value ? t * a.vs.token + h * a.vs.head : t * a.ks.token + h * a.ks.head;
        const int32_t pos = a.positions[t];
        const int32_t page = page_of(a.c, a.seqs ? a.seqs[t] : (int32_t)t, pos);
        float x[16];
        if (page < 0) {
            for (int i = 0; i < 16; ++i) x[i] = 0.0f;
        } else {
            const int slot = pos % a.c.page_size;
            const int64_t row = ((int64_t)page * a.c.kv_heads + h) * a.c.page_size + slot;
            const uint8_t *buf = value ? a.c.v : a.c.k;
            if (!a.c.nvfp4) {
                const uint16_t *in = reinterpret_cast<const uint16_t *>(buf) + row * a.c.head_dim + 16 * g;
                for (int i = 0; i < 16; ++i) x[i] = load_elem(in + i);
            } else {
                const uint32_t b = value ? a.c.v_scales[(((int64_t)page * a.c.kv_heads + h) * groups + g) * a.c.page_size + slot]
                                         : a.c.k_scales[row * groups + g];
                const float s = e4m3_decode(b), ts = value ? *a.c.v_ts : *a.c.k_ts;
                const uint2 w = *reinterpret_cast<const uint2 *>(buf + row * (a.c.head_dim / 2) + 8 * g);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t code = (i < 8 ? w.x : w.y) >> (4 * (i & 7));
                    const float m = e2m1_decode_mag(code & 7u) * s * ts;
                    x[i] = code & 8u ? -m : m;
                }
            }
        }
        for (int i = 0; i < 16; ++i) store_elem(y + 16 * g + i, x[i]);
    }
}

unsigned grid_of(int64_t total)
{
    const int64_t blocks = (total + kThreads - 1) / kThreads;
    return (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20);
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs &a, hipStream_t s)
{
    const unsigned grid = grid_of(a.tokens * 2 * a.c.kv_heads * (a.c.head_dim / 16));
    if (a.bf16) {
        if (a.rtn46) append_kernel<uint16_t, QII_RTN_46><<<grid, kThreads, 0, s>>>(a);
        else append_kernel<uint16_t, QII_RTN><<<grid, kThreads, 0, s>>>(a);
    } else {
        if (a.rtn46) append_kernel<float, QII_RTN_46><<<grid, kThreads, 0, s>>>(a);
        else append_kernel<float, QII_RTN><<<grid, kThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_kv_read(const ReadArgs &a, hipStream_t s)
{
    const unsigned grid = grid_of(a.tokens * 2 * a.c.kv_heads * (a.c.head_dim / 16));
    if (a.bf16) read_kernel<uint16_t><<<grid, kThreads, 0, s>>>(a);
    else read_kernel<float><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace qii
