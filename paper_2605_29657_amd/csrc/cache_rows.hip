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
    // ONCE: nothing reads them again here (the caches are left to the codes: 222 us against
    // 226 us for 80000 tokens of 8 heads of 128 and their reading back).
    template <bool ONCE>
    __device__ __forceinline__ void load(const char* p) {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) {
            const u32x4* x = reinterpret_cast<const u32x4*>(p) + i;
            w[i] = get<ONCE>(x);
        }
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
// 80000 tokens of 8 heads of 128 from bfloat16, 495 MB in and out: 103 us, 4.8 TB/s (what a
// large copy reaches); 131 tokens of 4 heads of 80: 5 us.
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
    const int units = (G >> 2) * (c.dp >> 3), span = units < kRowThreads ? units : kRowThreads;
    const int side = kRowThreads / span;                 // blocks of this workgroup at a time
    const int shift = c.dp == 64 ? 3 : c.dp == 128 ? 4 : 5;            // units per group of tokens
    const int total = items * c.Hkv * 2;
    constexpr int ESZ = F32 ? 4 : 2;
    for (int w0 = blockIdx.x * side; w0 < total; w0 += gridDim.x * side) {
        const Block bl = block_at(w0 + threadIdx.x / span, items, c.Hkv);
        const int* rec = plan_record(plan, n, p.max_pages, bl.item);
        const int page = rec[RR_PAGE], tail = rec[RR_TAIL], row0 = rec[RR_ROW];
        const int had = rec[RR_HAD], end = rec[RR_END];  // tokens the page held, and holds now
        const size_t at = (size_t)page * c.Hkv + bl.head, from = (size_t)tail * c.Hkv + bl.head;
        unsigned char* blk = (bl.kv ? c.v : c.k) + at * c.block;
        const unsigned char* src = (bl.kv ? c.v : c.k) + from * c.block;
        float* scale = bl.kv ? c.vs : c.ks;
        const long long st = bl.kv ? vst : kst;
        // Row of the page's token 0 in the packed rows, at this head.
        const char* x = (bl.kv ? v : k) + (row0 * st + (long long)bl.head * c.d) * ESZ;
        Row8<F32> raw[KEEP ? UPT : 1][4];
        auto load = [&](int u, Row8<F32>* r) {
            const int quad = u >> shift, e0 = (u - (quad << shift)) * 8;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int tok = quad * 4 + t;
                if (bl.live && e0 < c.d && tok >= had && tok < end) r[t].template load<KEEP>(x + (tok * st + e0) * ESZ);
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

// 80000 tokens of 8 heads of 128 to bfloat16, 495 MB: 77 us, 6.4 TB/s; 131 tokens of 4 heads of 80: 5 us.
// STREAM: for outputs larger than the last-level cache.  2 x 134 MB take 60 us against 71,
// 137 against 145 us with an addition of the two behind it; at 2 x 67 MB both ways take
// 31.5 us, but 63.5 against 61.3 us with the addition.
template <bool F32, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void cache_read(PageView p, CacheView c, BatchView b,
                                                          const int* start, char* k, long long kst,
                                                          char* v, long long vst) {
    const int i = blockIdx.y, rows = stated_rows(b, i), s = slot_of(b, i);
    if (s < 0 || s >= p.num_seqs || rows < 0) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.status, batch_faults(p, s, rows));
        return;
    }
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
                f32x4* o = reinterpret_cast<f32x4*>(to);
                put<STREAM>(f32x4{x[0] * sc, x[1] * sc, x[2] * sc, x[3] * sc}, o);
                put<STREAM>(f32x4{x[4] * sc, x[5] * sc, x[6] * sc, x[7] * sc}, o + 1);
            } else {
                // Exact: the low 16 bits are zero (4 significant bits, normal numbers only).
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = (__float_as_uint(x[2 * e] * sc) >> 16) |
                           (__float_as_uint(x[2 * e + 1] * sc) & 0xffff0000u);
                put<STREAM>(w, reinterpret_cast<u32x4*>(to));
            }
        }
    }
}

// A span's survivors: token r of them is token start + idx[r] of the sequence.
struct Kept {
    int start, span, count;
    const int* idx;
};

// What bounds the move is the chain of loads that finds a token (item, sequence, index,
// page) before its codes can be read.  It is the same for all heads, so a workgroup follows
// it once for HG heads of an item's keys or values and then has all their codes in flight;
// they stay in registers between the search for the scale and the conversion (12 per unit).
// A block takes `span` threads; workgroups with room for several take several head groups.
// 64 forks' survivors, a tenth of 2880 tokens each, 8 heads of 128: 36 us for 38 MB of codes
// in and out, and the three neighbours in every group of four that a value's byte lies with:
// 132 MB in all, 3.7 TB/s behind a chain of six loads.  (HG = 4 and 1: 3 us more, 8: 12.)
template <int UPT, int HG>
__global__ __launch_bounds__(kRowThreads) void cache_move(PageView p, CacheView c, int n,
                                                          const int* plan, const int* idx) {
    __shared__ float red[kRowThreads / 64];
    if (plan[0] != kPlanKeep || plan[1] != n) return;
    const int items = plan[2], G = 1 << p.shift;
    const int units = (G >> 2) * (c.dp >> 3), span = units < kRowThreads ? units : kRowThreads;
    const int shift = c.dp == 64 ? 3 : c.dp == 128 ? 4 : 5;
    const int groups = (c.Hkv + HG - 1) / HG;
    const int side = kRowThreads / span, total = items * groups * 2;
    for (int w0 = blockIdx.x * side; w0 < total; w0 += gridDim.x * side) {
        const Block bl = block_at(w0 + threadIdx.x / span, items, groups);
        const int head0 = bl.head * HG;
        const int* rec = plan_record(plan, n, p.max_pages, bl.item);
        const int* olds = plan_pages(plan, n, p.max_pages, rec[RK_SEQ]);
        const Kept kept{rec[RK_START], rec[RK_SPAN], rec[RK_COUNT], idx + rec[RK_OFF]};
        const int page = rec[RK_PAGE], pos0 = rec[RK_POS], end = rec[RK_END];
        unsigned char* store = bl.kv ? c.v : c.k;
        float* scale = bl.kv ? c.vs : c.ks;
        u32x2 code[HG][UPT][4];                 // eight codes of a token
        float sc[HG][UPT][4];
#pragma unroll
        for (int y = 0; y < UPT; ++y) {
            const int u = y * span + threadIdx.x % span;
            const int quad = u >> shift, e0 = (u - (quad << shift)) * 8;
            // No branches: a place without a token reads what the page's first one reads, and
            // drops it, so that all loads of a thread are in flight together.
            int in[4], old[4];
            bool is[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int tok = quad * 4 + t;
                is[t] = bl.live && tok < end;
                // The source of the compacted sequence's token: itself before the span, behind
                // it moved by what was dropped, listed within (any valid address elsewhere).
                const int to = pos0 + (is[t] ? tok : 0), r = to - kept.start;
                int v = *(r >= 0 && r < kept.count ? kept.idx + r : rec);
                // An ascending list has idx[r] >= r.  Holding any list to that and to the span
                // keeps the source within the pages that the plan lists.
                v = v < r ? r : v;
                v = v >= kept.span ? kept.span - 1 : v;
                in[t] = r < 0 ? to : r >= kept.count ? to - kept.count + kept.span : kept.start + v;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) old[t] = olds[in[t] >> p.shift];
#pragma unroll
            for (int t = 0; t < 4; ++t) in[t] &= G - 1;
#pragma unroll
            for (int x = 0; x < HG; ++x) {
                const int head = head0 + x < c.Hkv ? head0 + x : c.Hkv - 1;
#pragma unroll
                for (int t = 0; t < 4; ++t) sc[x][y][t] = scale[(size_t)old[t] * c.Hkv + head];
                if (bl.kv) {
                    u32x4 a[4], b[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const unsigned char* w = store + ((size_t)old[t] * c.Hkv + head) * c.block +
                                                 ((size_t)(in[t] >> 2) * c.dp + e0) * 4;
                        a[t] = reinterpret_cast<const u32x4*>(w)[0];
                        b[t] = reinterpret_cast<const u32x4*>(w)[1];
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        // Byte in & 3 of every dword.
                        const unsigned pick = 0x0c0c0000u | (4u + (in[t] & 3)) << 8 | (unsigned)(in[t] & 3);
                        const unsigned a01 = __builtin_amdgcn_perm(a[t][1], a[t][0], pick);
                        const unsigned a23 = __builtin_amdgcn_perm(a[t][3], a[t][2], pick);
                        const unsigned b01 = __builtin_amdgcn_perm(b[t][1], b[t][0], pick);
                        const unsigned b23 = __builtin_amdgcn_perm(b[t][3], b[t][2], pick);
                        code[x][y][t] = u32x2{a01 | a23 << 16, b01 | b23 << 16};
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        code[x][y][t] = *reinterpret_cast<const u32x2*>(
                            store + ((size_t)old[t] * c.Hkv + head) * c.block + (size_t)in[t] * c.dp + e0);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    code[x][y][t][0] = is[t] ? code[x][y][t][0] : 0;
                    code[x][y][t][1] = is[t] ? code[x][y][t][1] : 0;
                    sc[x][y][t] = is[t] ? sc[x][y][t] : 1.f;
                }
            }
        }
#pragma unroll
        for (int x = 0; x < HG; ++x) {
            float top = 0.f;
#pragma unroll
            for (int y = 0; y < UPT; ++y)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const f32x4 q = dec4(code[x][y][t][0]), r = dec4(code[x][y][t][1]);
                    float m = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = fmaxf(m, fmaxf(fabsf(q[e]), fabsf(r[e])));
                    top = fmaxf(top, m * sc[x][y][t]);
                }
            top = group_max(top, span, red);
            const int newexp = scale_exp(top);
            if (!bl.live || head0 + x >= c.Hkv) continue;
            const size_t at = (size_t)page * c.Hkv + head0 + x;
#pragma unroll
            for (int y = 0; y < UPT; ++y) {
                const int u = y * span + threadIdx.x % span;
                const int quad = u >> shift, e0 = (u - (quad << shift)) * 8;
                if (quad * 4 >= end) continue;
                float z[32];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    int d = exp_of(sc[x][y][t]) - newexp;
                    d = d < -126 ? -126 : d > 127 ? 127 : d;       // 127: a block of zeros
                    const float f = exp_scale(d);
                    const f32x4 q = dec4(code[x][y][t][0]), r = dec4(code[x][y][t][1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { z[t * 8 + e] = q[e] * f; z[t * 8 + 4 + e] = r[e] * f; }
                }
                store_codes(store + at * c.block, bl.kv, c.dp, quad, e0, z);
            }
            if (threadIdx.x % span == 0) scale[at] = exp_scale(newexp);
        }
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
    const long long bytes = b.n * most * c.Hkv * c.d * (f32 ? 4 : 2) * ((k != nullptr) + (v != nullptr));
    const bool stream = bytes > kLastLevelBytes;
    auto go = [&](auto kernel) {
        return launch(kernel, grid, dim3(kRowThreads), 0, s, p, c, b, start, kk, ks, vv, vs);
    };
    if (f32) return stream ? go(cache_read<true, true>) : go(cache_read<true, false>);
    return stream ? go(cache_read<false, true>) : go(cache_read<false, false>);
}

hipError_t launch_cache_move(const PageView& p, const CacheView& c, int n, const int* plan,
                             const int* idx, hipStream_t s) {
    long long pages = (long long)n * p.max_pages;
    if (pages > p.num_pages) pages = p.num_pages;
    return with_units(p, c, [&](auto upt) {
        constexpr int U = decltype(upt)::value, HG = U <= 2 ? 2 : 1;
        const dim3 grid(row_grid(p, c, pages * ((c.Hkv + HG - 1) / HG) * 2));
        return launch(cache_move<U, HG>, grid, dim3(kRowThreads), 0, s, p, c, n, plan, idx);
    });
}

}  // namespace occam
