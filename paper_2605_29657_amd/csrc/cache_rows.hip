// A layer's rows in the paged 8-bit cache: quantising new ones in, reading them back as
// values, and moving survivors into fresh pages.  All three are bound by memory traffic.
//
// Work is cut into units of four tokens x eight elements: the smallest piece that is
// contiguous in both orders of a page (keys [token][dp], values [token / 4][dp][4]: 8 bytes
// of four rows, or 32 bytes), so one unit is owned by one thread and no byte is shared.  A
// (page, key head) block of keys or of values has U = page_tokens * dp / 32 units (32 to
// 2048) and one scale; a workgroup of 256 threads takes 256 / U blocks at a time, or one
// block with U / 256 units per thread.
#include <type_traits>

#include "cache_internal.hpp"

namespace occam {
namespace {

constexpr int kRowThreads = 256;

// Largest of x over the block's units: the `span` threads (a power of two) of this group.
// Every thread of the workgroup must call it.
__device__ __forceinline__ float group_max(float x, int span, float* red) {
    const int within = span < 64 ? span : 64;
    for (int o = 1; o < within; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
    if (span <= 64) return x;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    const int w0 = (threadIdx.x & ~(span - 1)) >> 6;
    for (int w = 0; w < span >> 6; ++w) x = fmaxf(x, red[w0 + w]);
    return x;
}

// Four tokens' codes of one unit, as float32 without the scale: v[t * 8 + e].
__device__ __forceinline__ void load_codes(const unsigned char* blk, bool val, int dp, int quad, int e0,
                                           float* v) {
    if (val) {
        const u32x4* w = reinterpret_cast<const u32x4*>(blk + ((size_t)quad * dp + e0) * 4);
        const u32x4 a = w[0], b = w[1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const f32x4 x = dec4(e < 4 ? a[e & 3] : b[e & 3]);
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t * 8 + e] = x[t];
        }
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(blk + (size_t)(quad * 4 + t) * dp + e0);
            const f32x4 x = dec4(w[0]), y = dec4(w[1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[t * 8 + e] = x[e]; v[t * 8 + 4 + e] = y[e]; }
        }
    }
}

__device__ __forceinline__ void store_codes(unsigned char* blk, bool val, int dp, int quad, int e0,
                                            const float* v) {
    if (val) {
        u32x4 a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] = enc4(v[e], v[8 + e], v[16 + e], v[24 + e]);
            b[e] = enc4(v[4 + e], v[12 + e], v[20 + e], v[28 + e]);
        }
        u32x4* w = reinterpret_cast<u32x4*>(blk + ((size_t)quad * dp + e0) * 4);
        w[0] = a;
        w[1] = b;
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float* x = v + t * 8;
            *reinterpret_cast<u32x2*>(blk + (size_t)(quad * 4 + t) * dp + e0) =
                u32x2{enc4(x[0], x[1], x[2], x[3]), enc4(x[4], x[5], x[6], x[7])};
        }
    }
}

// Eight elements of a row as they lie in memory, and as float32.
template <bool F32>
struct Row8 {
    u32x4 w[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const char* p) {
        w[0] = reinterpret_cast<const u32x4*>(p)[0];
        if constexpr (F32) w[1] = reinterpret_cast<const u32x4*>(p)[1];
    }
    __device__ __forceinline__ void zero() {
        w[0] = u32x4{0, 0, 0, 0};
        if constexpr (F32) w[1] = u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ float at(int e) const {
        if constexpr (F32) return __uint_as_float(w[e >> 2][e & 3]);
        return __uint_as_float(e & 1 ? w[0][e >> 1] & 0xffff0000u : w[0][e >> 1] << 16);
    }
};

// One (page, head) block of keys (kv = 0) or values (kv = 1) of an item.
struct Block {
    int item, head, kv;
    bool live;
};
__device__ __forceinline__ Block block_at(int w, int items, int Hkv) {
    Block b;
    b.live = w < items * Hkv * 2;
    if (!b.live) w = 0;
    b.kv = w & 1;
    w >>= 1;
    b.item = w / Hkv;
    b.head = w - b.item * Hkv;
    return b;
}

// UPT units per thread.  Up to two are held in registers between the search for the
// largest magnitude and the conversion; larger blocks are read a second time (from L2).
template <bool F32, int UPT>
__global__ __launch_bounds__(kRowThreads) void cache_append(PageView p, CacheView c, BatchView b,
                                                            const int* plan, const char* k,
                                                            long long kst, const char* v,
                                                            long long vst) {
    constexpr bool KEEP = UPT <= 2;
    __shared__ float red[kRowThreads / 64];
    const int n = b.n, G = 1 << p.shift;
    if (plan[0] != kPlanReserve || plan[1] != n) return;
    const int items = plan[2];
    const int* pre = plan_array(plan, n, PL_ITEMS);
    const int* owner = plan_owner(plan, n, p.max_pages);
    const int units = (G >> 2) * (c.dp >> 3), span = units < kRowThreads ? units : kRowThreads;
    const int side = kRowThreads / span;                 // blocks of this workgroup at a time
    const int shift = c.dp == 64 ? 3 : c.dp == 128 ? 4 : 5;            // units per group of tokens
    const int total = items * c.Hkv * 2;
    constexpr int ESZ = F32 ? 4 : 2;
    for (int w0 = blockIdx.x * side; w0 < total; w0 += gridDim.x * side) {
        const Block bl = block_at(w0 + threadIdx.x / span, items, c.Hkv);
        const int i = owner[bl.item];
        const int len = plan_array(plan, n, PL_FIRST)[i], rows = plan_array(plan, n, PL_ROWS)[i];
        const int j = (len >> p.shift) + bl.item - pre[i];
        const int page = p.table[(size_t)plan_array(plan, n, PL_SLOT)[i] * p.max_pages + j];
        const int pos0 = j << p.shift;
        const int had = len > pos0 ? len - pos0 : 0;     // tokens the page held
        const int tail = had ? plan_array(plan, n, PL_TAIL)[i] : page;
        const size_t at = (size_t)page * c.Hkv + bl.head, from = (size_t)tail * c.Hkv + bl.head;
        unsigned char* blk = (bl.kv ? c.v : c.k) + at * c.block;
        const unsigned char* src = (bl.kv ? c.v : c.k) + from * c.block;
        float* scale = bl.kv ? c.vs : c.ks;
        const long long st = bl.kv ? vst : kst;
        // Row of the page's token 0 in the packed rows, at this head.
        const char* x = (bl.kv ? v : k) +
                        (((long long)row_begin(b, i) - len + pos0) * st + (long long)bl.head * c.d) * ESZ;
        const int end = len + rows - pos0 < G ? len + rows - pos0 : G;     // tokens it holds now
        Row8<F32> raw[KEEP ? UPT : 1][4];
        auto load = [&](int u, Row8<F32>* r) {
            const int quad = u >> shift, e0 = (u - (quad << shift)) * 8;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int tok = quad * 4 + t;
                if (bl.live && e0 < c.d && tok >= had && tok < end) r[t].load(x + (tok * st + e0) * ESZ);
                else r[t].zero();
            }
        };
        float top = 0.f;
#pragma unroll
        for (int y = 0; y < UPT; ++y) {
            Row8<F32>* r = raw[KEEP ? y : 0];
            load(y * span + threadIdx.x % span, r);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(r[t].at(e)));
        }
        top = group_max(top, span, red);
        const int oldexp = had ? exp_of(scale[from]) : kMinExp;
        const int newexp = scale_exp(top) > oldexp ? scale_exp(top) : oldexp;
        const float inv = exp_scale(-newexp);
        const float most = newexp == kMaxExp ? kMostAtMaxExp : 448.f;
        const float again = exp_scale(oldexp - newexp < -126 ? -126 : oldexp - newexp);
        const bool rewrite = had && (tail != page || newexp != oldexp);
        if (bl.live)
#pragma unroll
            for (int y = 0; y < UPT; ++y) {
                const int u = y * span + threadIdx.x % span;
                const int quad = u >> shift, e0 = (u - (quad << shift)) * 8;
                if (quad * 4 >= end || (quad * 4 + 3 < had && !rewrite)) continue;
                Row8<F32>* r = raw[KEEP ? y : 0];
                if (!KEEP) load(u, r);
                float z[32] = {};
                if (quad * 4 < had) load_codes(src, bl.kv, c.dp, quad, e0, z);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        z[t * 8 + e] = quad * 4 + t < had
                                           ? z[t * 8 + e] * again
                                           : __builtin_amdgcn_fmed3f(r[t].at(e) * inv, -most, most);
                store_codes(blk, bl.kv, c.dp, quad, e0, z);
            }
        // Every thread of the block has read scale[from], which is scale[at] where the page
        // stays the sequence's own.
        if (span > 64) __syncthreads();
        if (bl.live && threadIdx.x % span == 0) scale[at] = exp_scale(newexp);
    }
}

template <bool F32>
__global__ __launch_bounds__(kRowThreads) void cache_read(PageView p, CacheView c, BatchView b,
                                                          const int* start, char* k, long long kst,
                                                          char* v, long long vst) {
    const int i = blockIdx.y, rows = row_count(b, i), s = slot_of(b, i);
    if (s < 0 || s >= p.num_seqs) return;
    const int a = start ? start[i] : 0, len = p.length[s];
    const long long last = (long long)a + rows < len ? (long long)a + rows : len;   // past the end
    const int lo = a > 0 ? a : 0;
    const int chunks = c.d >> 3;
    const unsigned per = c.Hkv * chunks;
    const unsigned u = blockIdx.x * kRowThreads + threadIdx.x;
    const long long quad = (lo >> 2) + (long long)(u / per);
    const int r = (int)(u % per), head = r / chunks, e0 = (r - head * chunks) * 8;
    if (quad * 4 >= last) return;
    const int page = p.table[(size_t)s * p.max_pages + (int)(quad * 4 >> p.shift)];
    const int in_page = (int)(quad * 4 & ((1 << p.shift) - 1)) >> 2;
    const size_t at = (size_t)page * c.Hkv + head;
    for (int kv = 0; kv < 2; ++kv) {
        char* out = kv ? v : k;
        if (!out) continue;
        const long long st = kv ? vst : kst;
        float y[32];
        load_codes((kv ? c.v : c.k) + at * c.block, kv, c.dp, in_page, e0, y);
        const float sc = (kv ? c.vs : c.ks)[at];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const long long pos = quad * 4 + t;
            if (pos < lo || pos >= last) continue;
            const long long row = (long long)row_begin(b, i) + pos - a;
            char* to = out + (row * st + (long long)head * c.d + e0) * (F32 ? 4 : 2);
            const float* x = y + t * 8;
            if constexpr (F32) {
                reinterpret_cast<f32x4*>(to)[0] = f32x4{x[0] * sc, x[1] * sc, x[2] * sc, x[3] * sc};
                reinterpret_cast<f32x4*>(to)[1] = f32x4{x[4] * sc, x[5] * sc, x[6] * sc, x[7] * sc};
            } else {
                // Exact: the low 16 bits are zero (4 significant bits, normal numbers only).
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = (__float_as_uint(x[2 * e] * sc) >> 16) |
                           (__float_as_uint(x[2 * e + 1] * sc) & 0xffff0000u);
                *reinterpret_cast<u32x4*>(to) = w;
            }
        }
    }
}

// The source token of the compacted sequence's token x.
struct Kept {
    int start, span, count;
    const int* idx;
};
__device__ __forceinline__ int source_of(const Kept& s, int x) {
    const int r = x - s.start;
    if (r < 0) return x;
    if (r >= s.count) return x - s.count + s.span;
    int v = s.idx[r];
    v = v < 0 ? 0 : v >= s.span ? s.span - 1 : v;        // never outside the old pages
    return s.start + v;
}

// Codes and their scales stay in registers between the search and the conversion (12 per
// unit).
template <int UPT>
__global__ __launch_bounds__(kRowThreads) void cache_move(PageView p, CacheView c, int n,
                                                          const int* plan, const int* idx,
                                                          const int* off) {
    __shared__ float red[kRowThreads / 64];
    if (plan[0] != kPlanKeep || plan[1] != n) return;
    const int items = plan[2], G = 1 << p.shift;
    const int* pre = plan_array(plan, n, PL_ITEMS);
    const int* owner = plan_owner(plan, n, p.max_pages);
    const int units = (G >> 2) * (c.dp >> 3), span = units < kRowThreads ? units : kRowThreads;
    const int shift = c.dp == 64 ? 3 : c.dp == 128 ? 4 : 5;
    const int side = kRowThreads / span, total = items * c.Hkv * 2;
    for (int w0 = blockIdx.x * side; w0 < total; w0 += gridDim.x * side) {
        const Block bl = block_at(w0 + threadIdx.x / span, items, c.Hkv);
        const int i = owner[bl.item];
        const int first = plan_array(plan, n, PL_FIRST)[i], now = plan_array(plan, n, PL_NEW)[i];
        const int* olds = plan_pages(plan, n, p.max_pages, i);
        const int j = first + bl.item - pre[i];
        const Kept kept{plan_array(plan, n, PL_START)[i], plan_array(plan, n, PL_SPAN)[i],
                        off[i + 1] - off[i], idx + off[i]};
        const int pos0 = j << p.shift, end = now - pos0 < G ? now - pos0 : G;
        const int page = p.table[(size_t)plan_array(plan, n, PL_SLOT)[i] * p.max_pages + j];
        unsigned char* store = bl.kv ? c.v : c.k;
        float* scale = bl.kv ? c.vs : c.ks;
        u32x2 code[UPT][4];                     // eight codes of a token
        float sc[UPT][4], top = 0.f;
        // Where the tokens come from, then their codes and scales, all at once.
#pragma unroll
        for (int y = 0; y < UPT; ++y) {
            const int u = y * span + threadIdx.x % span;
            const int quad = u >> shift, e0 = (u - (quad << shift)) * 8;
            int from[4];
            size_t at[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int tok = quad * 4 + t;
                from[t] = bl.live && tok < end ? source_of(kept, pos0 + tok) : -1;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
                at[t] = from[t] < 0 ? 0 : (size_t)olds[from[t] >> p.shift] * c.Hkv + bl.head;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                code[y][t] = u32x2{0, 0};
                sc[y][t] = 1.f;
                if (from[t] < 0) continue;
                sc[y][t] = scale[at[t]];
                const int in = from[t] & (G - 1);
                const unsigned char* blk = store + at[t] * c.block;
                if (bl.kv) {
                    const unsigned char* w = blk + ((size_t)(in >> 2) * c.dp + e0) * 4;
                    const u32x4 a = reinterpret_cast<const u32x4*>(w)[0];
                    const u32x4 b = reinterpret_cast<const u32x4*>(w)[1];
                    const int sh = (in & 3) * 8;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        code[y][t][0] |= (a[e] >> sh & 255u) << (8 * e);
                        code[y][t][1] |= (b[e] >> sh & 255u) << (8 * e);
                    }
                } else {
                    code[y][t] = *reinterpret_cast<const u32x2*>(blk + (size_t)in * c.dp + e0);
                }
            }
        }
#pragma unroll
        for (int y = 0; y < UPT; ++y)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const f32x4 q = dec4(code[y][t][0]), r = dec4(code[y][t][1]);
                float m = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, fmaxf(fabsf(q[e]), fabsf(r[e])));
                top = fmaxf(top, m * sc[y][t]);
            }
        top = group_max(top, span, red);
        const int newexp = scale_exp(top);
        if (!bl.live) continue;
#pragma unroll
        for (int y = 0; y < UPT; ++y) {
            const int u = y * span + threadIdx.x % span;
            const int quad = u >> shift, e0 = (u - (quad << shift)) * 8;
            if (quad * 4 >= end) continue;
            float z[32];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                int d = exp_of(sc[y][t]) - newexp;
                d = d < -126 ? -126 : d > 127 ? 127 : d;       // 127: a block of zeros
                const float f = exp_scale(d);
                const f32x4 q = dec4(code[y][t][0]), r = dec4(code[y][t][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) { z[t * 8 + e] = q[e] * f; z[t * 8 + 4 + e] = r[e] * f; }
            }
            store_codes(store + ((size_t)page * c.Hkv + bl.head) * c.block, bl.kv, c.dp, quad, e0, z);
        }
        if (threadIdx.x % span == 0) scale[(size_t)page * c.Hkv + bl.head] = exp_scale(newexp);
    }
}

// Workgroups for `blocks` (page, head) blocks of keys and of values: what fills the chip
// eight times over at most; the kernels walk the rest.
int row_grid(const PageView& p, const CacheView& c, long long blocks) {
    const int units = (1 << p.shift) / 4 * (c.dp / 8);
    const int side = units < kRowThreads ? kRowThreads / units : 1;
    const long long wgs = (blocks + side - 1) / side;
    return (int)(wgs < 4096 ? wgs : 4096);
}

// Calls f(UPT) with the units per thread of a block as a compile-time number.
template <typename F>
hipError_t with_units(const PageView& p, const CacheView& c, F f) {
    switch ((1 << p.shift) / 4 * (c.dp / 8) / kRowThreads) {
        case 8: return f(std::integral_constant<int, 8>{});
        case 4: return f(std::integral_constant<int, 4>{});
        case 2: return f(std::integral_constant<int, 2>{});
        default: return f(std::integral_constant<int, 1>{});
    }
}

}  // namespace

hipError_t launch_cache_append(const PageView& p, const CacheView& c, const BatchView& b,
                               const int* plan, int f32, const void* k, long long ks,
                               const void* v, long long vs, hipStream_t s) {
    const long long most = b.off ? b.max_rows : b.rows;
    const long long pages = (long long)b.n * (((most - 1) >> p.shift) + 2);
    const dim3 grid(row_grid(p, c, pages * c.Hkv * 2));
    auto kk = static_cast<const char*>(k), vv = static_cast<const char*>(v);
    return with_units(p, c, [&](auto upt) {
        constexpr int U = decltype(upt)::value;
        return f32 ? launch(cache_append<true, U>, grid, dim3(kRowThreads), 0, s, p, c, b, plan, kk, ks, vv, vs)
                   : launch(cache_append<false, U>, grid, dim3(kRowThreads), 0, s, p, c, b, plan, kk, ks, vv, vs);
    });
}

hipError_t launch_cache_read(const PageView& p, const CacheView& c, const BatchView& b,
                             const int* start, int f32, void* k, long long ks, void* v,
                             long long vs, hipStream_t s) {
    const long long most = b.off ? b.max_rows : b.rows;
    const long long units = (most / 4 + 2) * c.Hkv * (c.d / 8);
    const dim3 grid((unsigned)((units + kRowThreads - 1) / kRowThreads), b.n);
    auto kk = static_cast<char*>(k), vv = static_cast<char*>(v);
    return f32 ? launch(cache_read<true>, grid, dim3(kRowThreads), 0, s, p, c, b, start, kk, ks, vv, vs)
               : launch(cache_read<false>, grid, dim3(kRowThreads), 0, s, p, c, b, start, kk, ks, vv, vs);
}

hipError_t launch_cache_move(const PageView& p, const CacheView& c, int n, const int* plan,
                             const int* idx, const int* off, hipStream_t s) {
    long long pages = (long long)n * p.max_pages;
    if (pages > p.num_pages) pages = p.num_pages;
    const dim3 grid(row_grid(p, c, pages * c.Hkv * 2));
    return with_units(p, c, [&](auto upt) {
        return launch(cache_move<decltype(upt)::value>, grid, dim3(kRowThreads), 0, s, p, c, n, plan, idx, off);
    });
}

}  // namespace occam
