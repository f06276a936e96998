// Rotary positions: the table of a plan, and the rotation of [tokens][heads][head_dim] by it (see qii_rotary in include/qii.h).
#include <math.h>

#include <type_traits>

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

// One thread a pair, or an element after the rotated ones: any strides, alignments and rot_dim.
template <typename T>
__global__ __launch_bounds__(kThreads) void rotary_any_kernel(RotaryArgs a)
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

// kBytes (16, 8 or 4) of a head, as loaded and in binary32
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int kBytes>
using Words = std::conditional_t<kBytes == 16, u32x4, std::conditional_t<kBytes == 8, u32x2, uint32_t>>;

template <int kBytes>
__device__ __forceinline__ uint32_t word(const Words<kBytes> &w, int i)
{
    if constexpr (kBytes == 4) return w;
    else return w[i];
}
template <bool kStream, int kBytes>
__device__ __forceinline__ Words<kBytes> load(const void *p)
{
    const auto *word = static_cast<const Words<kBytes> *>(p);
    if constexpr (kStream) return __builtin_nontemporal_load(word);
    else return *word;
}
template <int kBytes>
__device__ __forceinline__ void unpack(const Words<kBytes> &w, float *v, const float *)
{
#pragma unroll
    for (int i = 0; i < kBytes / 4; ++i) v[i] = u2f(word<kBytes>(w, i));
}
template <int kBytes>
__device__ __forceinline__ void unpack(const Words<kBytes> &w, float *v, const uint16_t *)
{
#pragma unroll
    for (int i = 0; i < kBytes / 4; ++i) {
        v[2 * i] = bf16_lo(word<kBytes>(w, i));
        v[2 * i + 1] = bf16_hi(word<kBytes>(w, i));
    }
}
template <bool kStream, int kBytes>
__device__ __forceinline__ void pack(const float *v, float *out)
{
    Words<kBytes> w;
    if constexpr (kBytes == 4) w = f2u(v[0]);
    else
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) w[i] = f2u(v[i]);
    if constexpr (kStream) __builtin_nontemporal_store(w, reinterpret_cast<Words<kBytes> *>(out));
    else *reinterpret_cast<Words<kBytes> *>(out) = w;
}
template <bool kStream, int kBytes>
__device__ __forceinline__ void pack(const float *v, uint16_t *out)
{
    const auto two = [&](int i) { return to_bf16(v[2 * i], v[2 * i + 1]); };
    Words<kBytes> w;
    if constexpr (kBytes == 4) w = two(0);
    else
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) w[i] = two(i);
    if constexpr (kStream) __builtin_nontemporal_store(w, reinterpret_cast<Words<kBytes> *>(out));
    else *reinterpret_cast<Words<kBytes> *>(out) = w;
}
template <int kN>
__device__ __forceinline__ void load_floats(const float *p, float *v)
{
#pragma unroll
    for (int i = 0; i < kN; i += 4) {
        const float4 w = *reinterpret_cast<const float4 *>(p + i);
        v[i] = w.x; v[i + 1] = w.y; v[i + 2] = w.z; v[i + 3] = w.w;
    }
}

// How the vector kernel divides its work: a thread has one unit of a head, kHeads heads apart by `groups`, of one token, so that it
// reads their rotation once; neighbouring threads have neighbouring units, then neighbouring heads.
struct RotaryGrid { uint32_t units, turned, columns, groups, items; };   // units of a head, those that turn; (token, head group) items a block; items

// (y0, y1) = (x0 c - x1 s, x0 s + x1 c) for the pairs of a head, the gradient with -s; products and sums in binary32, rounded once.
// Bound by memory: kBytes of x a load, all of a thread's loads under way together.  A unit is kBytes of interleaved pairs, or as much
// of each half; after the rotated elements, kBytes that are copied.  kStream: past the caches.  32768 tokens x 32 bf16 heads of 128 (537 MB):
// 86 us, 6.2 TB/s, where a copy makes 5.1; 5003 x 24 f32 heads of 96 (92 MB) 15 to 17 us.  4 tokens of 16 heads: 2.2 us, a launch.
template <typename T, bool kInterleaved, int kHeads, int kBytes, bool kStream>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, RotaryGrid n)
{
    constexpr int V = kBytes / sizeof(T), kCos = kInterleaved ? V / 2 : V;
    const uint32_t u = threadIdx.x % n.units, column = threadIdx.x / n.units;
    const uint32_t item = blockIdx.x * n.columns + column;
    if (column >= n.columns || item >= n.items) return;
    const uint32_t t = item / n.groups, h0 = item % n.groups;
    const int pairs = a.rot.pairs;
    const bool turns = u < n.turned;
    // elements of the unit, and of its other half
    const int e0 = turns || kInterleaved ? u * V : 2 * pairs + (u - n.turned) * V, e1 = e0 + pairs;
    const T *x = static_cast<const T *>(a.x) + t * a.xs.token;
    T *y = static_cast<T *>(a.y) + t * a.ys.token;
    const int pos = a.positions[t];
    Words<kBytes> w0[kHeads], w1[kHeads];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        const uint32_t h = min(h0 + k * n.groups, (uint32_t)a.heads - 1);   // (a head too many is read again and not stored)
        w0[k] = load<kStream, kBytes>(x + h * a.xs.head + e0);
        if (!kInterleaved && turns) w1[k] = load<kStream, kBytes>(x + h * a.xs.head + e1);
    }
    float c[kCos], s[kCos];
    const bool known = pos >= 0 && pos < a.rot.positions;
    if (turns && known) {
        const float *row = a.rot.cos_sin + (int64_t)pos * 2 * pairs + u * kCos;
        if constexpr (kCos % 4 == 0) {
            load_floats<kCos>(row, c);
            load_floats<kCos>(row + pairs, s);
        } else {
#pragma unroll
            for (int i = 0; i < kCos; ++i) { c[i] = row[i]; s[i] = row[pairs + i]; }
        }
        if (a.inverse)
#pragma unroll
            for (int i = 0; i < kCos; ++i) s[i] = -s[i];
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        const uint32_t h = h0 + k * n.groups;
        if (h >= (uint32_t)a.heads) break;
        T *out = y + h * a.ys.head;
        float p[V], q[V];
        unpack<kBytes>(w0[k], p, static_cast<const T *>(nullptr));
        if (turns) {
            if (kInterleaved) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float v = p[i];
                    p[i] = v * c[i / 2] - p[i + 1] * s[i / 2];
                    p[i + 1] = p[i + 1] * c[i / 2] + v * s[i / 2];
                }
            } else {
                unpack<kBytes>(w1[k], q, static_cast<const T *>(nullptr));
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float v = p[i];
                    p[i] = v * c[i % kCos] - q[i] * s[i % kCos];
                    q[i] = q[i] * c[i % kCos] + v * s[i % kCos];
                }
            }
        }
        if (!known) {
#pragma unroll
            for (int i = 0; i < V; ++i) p[i] = q[i] = pos < 0 ? 0.0f : NAN;
        }
        pack<kStream, kBytes>(p, out + e0);
        if (!kInterleaved && turns) pack<kStream, kBytes>(q, out + e1);
    }
}

// whether rows and units are aligned to kBytes throughout, and one grid holds them
template <typename T, int kBytes>
bool vector_grid(const RotaryArgs &a, int heads_each, RotaryGrid *n)
{
    constexpr int V = kBytes / sizeof(T);
    const int pairs = a.rot.pairs, rest = a.head_dim - 2 * pairs;
    const auto rows = [](const void *p, const Strides &s) { return reinterpret_cast<uintptr_t>(p) % kBytes == 0 && s.token % V == 0 && s.head % V == 0; };
    if (!rows(a.x, a.xs) || !rows(a.y, a.ys) || rest % V || (a.rot.interleaved ? 2 * pairs : pairs) % V) return false;
    n->turned = (uint32_t)((a.rot.interleaved ? 2 * pairs : pairs) / V);
    n->units = n->turned + (uint32_t)(rest / V);
    if (n->units > kThreads) return false;
    n->columns = kThreads / n->units;
    n->groups = (uint32_t)((a.heads + heads_each - 1) / heads_each);
    const int64_t items = a.tokens * n->groups;
    n->items = (uint32_t)items;
    return items / n->columns < (int64_t)1 << 23;   // (a launch has fewer than 2^32 threads)
}

// Whether a large tensor goes past the caches (loads and stores): where its stores fill whole lines of 64 bytes, half a head or a head at a
// time.  32768 x 32 bf16 heads of 128 98 us, past the caches 86; 2048 x 16 f32 8.7 and 6.8; halves of 48 bytes, 20000 x 24 bf16 heads, 38 and
// 49.  With a kernel behind it that reads the result (negation), bf16 heads of 128: 8 MB 12.9 and 12.3 us, 34 MB 28.4 and 27.6, 67 MB 48.8 and
// 49.5, 268 MB 180 and 175; with stores alone going past them 12.4, 29.8, 50.6 and 192.
template <typename T>
bool streams(const RotaryArgs &a)
{
    const int64_t size = sizeof(T), run = (a.rot.interleaved ? a.head_dim : a.rot.pairs) * size, rest = a.rot.interleaved ? 0 : (a.head_dim - 2 * a.rot.pairs) * size;
    return run % 64 == 0 && rest % 64 == 0 && a.ys.head * size % 64 == 0 && a.ys.token * size % 64 == 0 && reinterpret_cast<uintptr_t>(a.y) % 64 == 0;
}

template <typename T, int kBytes>
bool launch_vectors(const RotaryArgs &a, hipStream_t s)
{
    // One head a thread where threads are few.  Else what a token's heads share is read for two (halves) or four (pairs side by side), which
    // with 1 / 2 / 4 heads, 32 of 128 elements, through the caches: halves, 32768 tokens bf16 96 / 97 / 100 us, 16384 f32 98 / 97 / 103, 4096 bf16
    // 15.3 / 15.5 / 13.6; pairs, 32768 bf16 109 / 101 / 96, 16384 f32 100 / 92 / 91; 50 heads of 80, halves of 20, by 8 bytes
    // 135 / 112 / 107; 512 tokens of 16 heads 3.8 / 3.8 / 5.1.
    RotaryGrid n;
    const int several = a.rot.interleaved ? 4 : 2;
    const bool many = a.tokens * a.heads * (int64_t)a.head_dim >= (int64_t)1 << 22 && a.heads >= several;
    if (!vector_grid<T, kBytes>(a, many ? several : 1, &n)) return false;
    const unsigned blocks = (n.items + n.columns - 1) / n.columns;
    const bool stream = many && kBytes == 16 && streams<T>(a);
    const auto go = [&](auto interleaved, auto heads) {
        constexpr bool kInter = decltype(interleaved)::value;
        constexpr int kHeads = decltype(heads)::value;
        if constexpr (kHeads > 1 && kBytes == 16) {
            if (stream) {
                rotary_kernel<T, kInter, kHeads, kBytes, true><<<blocks, kThreads, 0, s>>>(a, n);
                return;
            }
        }
        rotary_kernel<T, kInter, kHeads, kBytes, false><<<blocks, kThreads, 0, s>>>(a, n);
    };
    const std::integral_constant<int, 1> one;
    if constexpr (kBytes >= 2 * (int)sizeof(T)) {
        if (a.rot.interleaved) {
            if (many) go(std::true_type(), std::integral_constant<int, 4>());
            else go(std::true_type(), one);
            return true;
        }
    }
    if (a.rot.interleaved) return false;   // (a pair does not fit)
    if (many) go(std::false_type(), std::integral_constant<int, 2>());
    else go(std::false_type(), one);
    return true;
}

// The widest words that rows and units are aligned to: 32768 x 50 heads of 80 elements, 40 of them turned in halves, bf16, take 457 us
// element by element and 114 by 8 bytes (with 80 turned 114 by 16).
template <typename T>
void launch(const RotaryArgs &a, hipStream_t s)
{
    if (launch_vectors<T, 16>(a, s) || launch_vectors<T, 8>(a, s) || launch_vectors<T, 4>(a, s)) return;
    const int64_t total = a.tokens * a.heads * (a.head_dim - a.rot.pairs), blocks = (total + kThreads - 1) / kThreads;
    rotary_any_kernel<T><<<(unsigned)(blocks < (1 << 20) ? blocks : 1 << 20), kThreads, 0, s>>>(a);
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
    if (a.bf16) launch<uint16_t>(a, s);
    else launch<float>(a, s);
    return hipGetLastError();
}

}  // namespace qii
