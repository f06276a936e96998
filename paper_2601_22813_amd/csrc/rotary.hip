// Rotary positions: the table of a plan, and the rotation of [tokens][heads][head_dim] by it (see qii_rotary in include/qii.h).
#include <math.h>

#include "kv_cache.h"

namespace qii {
namespace {

constexpr int kThreads = 256;

// theta(p, i) = p f_i in binary64: at a million positions still good to 1e-10 of a turn, far below the binary32 rounding of its cosine
__global__ __launch_bounds__(kThreads) void rotary_table_kernel(RotaryTableArgs a)
{
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= a.pairs) return;
    const double rot = 2.0 * a.pairs;
    double base = a.base;
    if (a.scaling == QII_ROTARY_SCALING_BASE) base *= pow(a.factor, rot / (a.pairs > 1 ? rot - 2.0 : 1.0));
    double f = pow(base, -2.0 * i / rot);
    if (a.scaling == QII_ROTARY_SCALING_LINEAR) f /= a.factor;
    if (a.scaling == QII_ROTARY_SCALING_BY_PARTS) {
        const double turns = a.original * f / 6.283185307179586476925;
        const double keep = fmin(fmax((turns - a.slow) / (a.fast - a.slow), 0.0), 1.0);
        f = f * keep + f / a.factor * (1.0 - keep);
    }
    for (int64_t p = blockIdx.y; p < a.positions; p += gridDim.y) {
        double sn, cs;
        sincos((double)p * f, &sn, &cs);
        float *row = a.cos_sin + p * 2 * a.pairs;
        row[i] = (float)(a.magnitude * cs);
        row[a.pairs + i] = (float)(a.magnitude * sn);
    }
}

// one thread a pair, or an element after the rotated ones
template <typename T>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a)
{
    const int pairs = a.rot.pairs, units = a.head_dim - pairs;
    const int64_t total = a.tokens * a.heads * units;
    for (int64_t n = blockIdx.x * (int64_t)kThreads + threadIdx.x; n < total; n += (int64_t)gridDim.x * kThreads) {
        const int u = (int)(n % units);
        const int64_t th = n / units, t = th / a.heads;
        const int h = (int)(th % a.heads);
        const T *x = static_cast<const T *>(a.x) + t * a.xs.token + h * a.xs.head;
        T *y = static_cast<T *>(a.y) + t * a.ys.token + h * a.ys.head;
        const int pos = a.positions[t];
        if (u >= pairs) {
            const float v = load_elem(x + pairs + u);
            store_elem(y + pairs + u, pos < 0 ? 0.0f : pos < a.rot.positions ? v : NAN);
            continue;
        }
        const int e0 = a.rot.interleaved ? 2 * u : u, e1 = a.rot.interleaved ? e0 + 1 : u + pairs;
        float cs = NAN, sn = NAN;
        if (pos >= 0 && pos < a.rot.positions) {
            cs = a.rot.cos_sin[(int64_t)pos * 2 * pairs + u];
            sn = a.rot.cos_sin[(int64_t)pos * 2 * pairs + pairs + u];
        }
        if (a.inverse) sn = -sn;
        const float p = load_elem(x + e0), q = load_elem(x + e1);
        store_elem(y + e0, pos < 0 ? 0.0f : p * cs - q * sn);
        store_elem(y + e1, pos < 0 ? 0.0f : q * cs + p * sn);
    }
}

}  // namespace

hipError_t launch_rotary_table(const RotaryTableArgs &a, hipStream_t s)
{
    const int64_t rows = a.positions < 16384 ? a.positions : 16384;
    rotary_table_kernel<<<dim3((a.pairs + kThreads - 1) / kThreads, (unsigned)rows), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_rotary(const RotaryArgs &a, hipStream_t s)
{
    const int64_t total = a.tokens * a.heads * (a.head_dim - a.rot.pairs), blocks = (total + kThreads - 1) / kThreads;
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20);
    if (a.bf16) rotary_kernel<uint16_t><<<grid, kThreads, 0, s>>>(a);
    else rotary_kernel<float><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace qii
