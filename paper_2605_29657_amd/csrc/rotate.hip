// Rotary positions with several axes: pair p of every head of a row turns by
// positions[row][axis[p]] * inv_freq[p].
//
// The angle.  A position's turns are kept as a 64-bit fraction, F_p = inv_freq_p / 2 pi in
// units of 2^-64, so position * F_p modulo 2^64 is the angle's fraction of a turn with no
// rounding but F's own: exact where a float32 product (error 2^-24 of the angle) would
// be wrong by a radian at position 10^7.  Sine and cosine are taken of its 24 leading bits,
// which float32 holds, and turned by what is left, r: s + c r and c - s r (|r| is below 2^-22,
// and r^2 / 2 below 2^-45).
//
// Bound by memory: every element is read and written once, and a row's sines and cosines
// are computed once for all heads of all tensors (queries and keys share a launch), staged
// in LDS.  A workgroup takes a run of rows; a thread's unit is VEC bytes of each side of
// the pairs (two 16-byte loads and stores where alignment allows), heads and chunks
// spread over the threads so that consecutive threads touch consecutive addresses.
// 362 MB of bfloat16 queries and keys: 152 us, 4.8 TB/s in and out (what a large copy
// reaches); 151 MB of float32, 32 heads of 72: 69 us, 4.4 TB/s; 8 rows: 4.3 us, a launch and
// three loads.
#include <string.h>

#include "cache_internal.hpp"

namespace occam {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotPairs = 2048;          // (row, pair) angles a workgroup holds

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(unsigned short x) { return __uint_as_float((unsigned)x << 16); }
template <> __device__ __forceinline__ float to_f(float x) { return x; }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f(float x) { return x; }
template <> __device__ __forceinline__ unsigned short from_f(float x) {
    return __builtin_bit_cast(unsigned short, (__bf16)x);
}

template <typename T, int N>
struct alignas(sizeof(T) * N) Pack { T x[N]; };

// STREAM: for tensors larger than the last-level cache, in units of 16 bytes: 2 x 362 MB take
// 152 us against 159; at 2 x 151 MB, 80 us against 71.
template <bool STREAM, typename T, int N>
__device__ __forceinline__ Pack<T, N> load(const T* p) {
    typedef Pack<T, N> V;
    if constexpr (sizeof(V) == 16) return __builtin_bit_cast(V, get<STREAM>(reinterpret_cast<const u32x4*>(p)));
    else return *reinterpret_cast<const V*>(p);
}
template <bool STREAM, typename T, int N>
__device__ __forceinline__ void store(const Pack<T, N>& x, T* p) {
    if constexpr (sizeof(x) == 16) put<STREAM>(__builtin_bit_cast(u32x4, x), reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<Pack<T, N>*>(p) = x;
}

// N elements per unit (a power of two; both sides of N pairs for HALVES, N / 2 pairs for
// ADJACENT when N > 1).
template <typename T, int N, bool ADJ, bool STREAM, typename Args>
__global__ __launch_bounds__(kRotThreads) void rotate(Args a, int rows_per) {
    __shared__ float2 cs[kRotPairs];
    const int row0 = blockIdx.x * rows_per;
    const int rows = a.rows - row0 < rows_per ? a.rows - row0 : rows_per;
    for (int i = threadIdx.x; i < rows * a.pairs; i += kRotThreads) {
        const int r = i / a.pairs, p = i - r * a.pairs;
        const int pos = a.pos[(size_t)(row0 + r) * a.axes + a.axis[p]];
        const unsigned long long turn = (unsigned long long)(long long)pos * a.turn[p];
        // To the nearest 2^-24 of a turn, signed, in half-turns; the rest in radians.
        const long long lead = (long long)(turn + (1ull << 39)) >> 40;
        const float left = (float)(int)((long long)(turn - ((unsigned long long)lead << 40)) >> 8) * 0x1.921fb6p-54f;
        float s, c;
        sincospif((float)(int)lead * 0x1p-23f, &s, &c);
        const float s1 = __builtin_fmaf(c, left, s), c1 = __builtin_fmaf(-s, left, c);
        cs[i] = make_float2(c1, a.inverse ? -s1 : s1);
    }
    __syncthreads();
    typedef Pack<T, N> V;
    // Units of a head: pairs first, then what is only copied (absent in place).
    const int np = ADJ && N > 1 ? 2 * a.pairs / N : a.pairs / N;
    const int rest = (a.d - 2 * a.pairs) / N, per = np + rest, total = rows * a.heads * per;
    for (int u = threadIdx.x; u < total; u += kRotThreads) {
        const int hr = u / per, w = u - hr * per;
        const int r = hr / a.heads, hh = hr - r * a.heads;
        int ti = 0;
        while (ti + 1 < a.n && hh >= a.t[ti + 1].first) ++ti;
        const RotTensor& t = a.t[ti];
        const size_t col = (size_t)(hh - t.first) * a.d;
        const T* x = reinterpret_cast<const T*>(t.src + (size_t)(row0 + r) * t.src_stride) + col;
        T* y = reinterpret_cast<T*>(t.dst + (size_t)(row0 + r) * t.dst_stride) + col;
        if (w >= np) {
            if (x == y) continue;
            const int e = 2 * a.pairs + (w - np) * N;
            store<STREAM>(load<STREAM, T, N>(x + e), y + e);
            continue;
        }
        const float2* f = cs + r * a.pairs;
        if constexpr (ADJ && N == 1) {
            const float2 q = f[w];
            const float p0 = to_f<T>(x[2 * w]), p1 = to_f<T>(x[2 * w + 1]);
            y[2 * w] = from_f<T>(p0 * q.x - p1 * q.y);
            y[2 * w + 1] = from_f<T>(p0 * q.y + p1 * q.x);
        } else if constexpr (ADJ) {
            V v = load<STREAM, T, N>(x + w * N);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float2 q = f[w * (N / 2) + i];
                const float p0 = to_f<T>(v.x[2 * i]), p1 = to_f<T>(v.x[2 * i + 1]);
                v.x[2 * i] = from_f<T>(p0 * q.x - p1 * q.y);
                v.x[2 * i + 1] = from_f<T>(p0 * q.y + p1 * q.x);
            }
            store<STREAM>(v, y + w * N);
        } else {
            V v0 = load<STREAM, T, N>(x + w * N);
            V v1 = load<STREAM, T, N>(x + a.pairs + w * N);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float2 q = f[w * N + i];
                const float p0 = to_f<T>(v0.x[i]), p1 = to_f<T>(v1.x[i]);
                v0.x[i] = from_f<T>(p0 * q.x - p1 * q.y);
                v1.x[i] = from_f<T>(p0 * q.y + p1 * q.x);
            }
            store<STREAM>(v0, y + w * N);
            store<STREAM>(v1, y + a.pairs + w * N);
        }
    }
}

// Arguments for two tensors and 64 pairs where they suffice: enqueueing the full 1.6 KB takes
// 4.6 us, these 0.7 KB 4.4 us.
typedef RotArgsOf<2, 64> RotArgsSmall;
RotArgsSmall small_args(const RotArgs& a) {
    RotArgsSmall b = {a.n, a.heads, a.rows, a.d, a.pairs, a.axes, a.adjacent, a.inverse, a.pos};
    for (int i = 0; i < a.n; ++i) b.t[i] = a.t[i];
    memcpy(b.turn, a.turn, sizeof b.turn);
    memcpy(b.axis, a.axis, sizeof b.axis);
    return b;
}

template <typename T, int N, bool ADJ, typename Args>
hipError_t go(const Args& a, hipStream_t s) {
    // Rows per workgroup: what the angle table holds, fewer while that leaves the chip empty.
    int per = kRotPairs / a.pairs;
    while (per > 1 && (a.rows - 1) / per + 1 < 2048) per >>= 1;
    const dim3 grid((a.rows - 1) / per + 1);
    if constexpr (sizeof(T) * N == 16)
        if ((long long)a.rows * a.heads * a.d * (long long)sizeof(T) > kLastLevelBytes)
            return launch(rotate<T, N, ADJ, true, Args>, grid, dim3(kRotThreads), 0, s, a, per);
    return launch(rotate<T, N, ADJ, false, Args>, grid, dim3(kRotThreads), 0, s, a, per);
}

template <typename T, int N>
hipError_t pick(const RotArgs& a, hipStream_t s) {
    if (a.n <= RotArgsSmall::kTensors && a.pairs <= RotArgsSmall::kPairs) {
        const RotArgsSmall b = small_args(a);
        return a.adjacent ? go<T, N, true>(b, s) : go<T, N, false>(b, s);
    }
    return a.adjacent ? go<T, N, true>(a, s) : go<T, N, false>(a, s);
}

}  // namespace

// vec: elements per unit that every pointer, stride and the head layout allow.
hipError_t launch_rotate(const RotArgs& a, int f32, int vec, hipStream_t s) {
    if (f32) {
        if (vec >= 4) return pick<float, 4>(a, s);
        if (vec >= 2) return pick<float, 2>(a, s);
        return pick<float, 1>(a, s);
    }
    if (vec >= 8) return pick<unsigned short, 8>(a, s);
    if (vec >= 4) return pick<unsigned short, 4>(a, s);
    if (vec >= 2) return pick<unsigned short, 2>(a, s);
    return pick<unsigned short, 1>(a, s);
}

}  // namespace occam
