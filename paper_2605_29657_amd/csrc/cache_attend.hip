// Attention of the sequences' last rows over the paged 8-bit cache: out = softmax(scale q
// K^T) V with the row's log-normaliser, one pass over the keys with a running maximum.
//
// Both products run transposed on the matrix cores, so that a lane keeps one query row from
// the scores to the output and the scores never leave registers:
//
//   S^T = K Q^T   A = keys (rows), B = queries (columns)
//   O^T = V^T P^T A = values (rows: elements), B = probabilities (columns: queries)
//
// A tile of S^T gives lane group g (of 16 lanes) tokens 4g .. 4g+3 of 16 for its column,
// which is, unmoved, the B operand of the second product if its reduction slots are numbered
// the same way; the values' order in a page, [token / 4][dp][4], is made for that: a 16-byte
// load gives four elements of a group of four tokens.
//
// 8 bits to matrix operands: one conversion instruction turns two codes and a power-of-two
// scale into two bf16 (keys) or f16 (values) numbers.  Keys are exact in bf16.  Values are
// converted relative to the largest value scale met so far (`ref`), which keeps them within
// f16's range; they are exact down to 2^-15 of it, and off by at most 2^-25 below.
// Probabilities are rounded to f16 (11 bits, half a step 2^-12: a bf16 probability, 2^-9,
// would cost as much accuracy as rounding the output) times 2^14, so that they lose nothing
// before 2^-28.  Maxima, sums and outputs are float32.
#include "cache_internal.hpp"

namespace occam {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kLift = 14.f;              // probabilities are held times 2^14
constexpr float kLn2 = 0.6931471805599453f;

// Eight codes (two dwords) as bf16 / f16, times a power of two.
__device__ __forceinline__ bf16x8 codes_bf16(unsigned a, unsigned b, float s) {
    union { bf16x2 p[4]; bf16x8 v; } r;
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true);
    return r.v;
}
__device__ __forceinline__ f16x8 codes_f16(unsigned a, float sa, unsigned b, float sb) {
    union { f16x2 p[4]; f16x8 v; } r;
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, sa, false);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, sa, true);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, sb, false);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, sb, true);
    return r.v;
}
__device__ __forceinline__ f16x2 round_f16(float a, float b) {     // to nearest
    return f16x2{(_Float16)a, (_Float16)b};
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---------------------------------------------------------------------------------------
// Few rows: 16 rows of one key head per workgroup, the keys of one split dealt to its four
// waves in steps of 32, joined in LDS.  Bound by reading the codes once: a wave has the
// loads of two steps in flight (8 KB each at d = 128) and several workgroups share a CU.
// ---------------------------------------------------------------------------------------
constexpr int kStep = 32, kFewWaves = 4, kFewRows = 16;

// Page numbers and scales of the 64 16-token groups around a wave's position, one per lane.
struct Window {
    int base, page;
    float ks, vs;
};

template <int DP>
__global__ __launch_bounds__(64 * kFewWaves) void attend_few(AttendArgs a) {
    constexpr int NC = DP / 64;            // 64-element chunks of a row
    __shared__ float jo[kFewWaves][kFewRows][64 + 4];
    __shared__ float jm[kFewWaves][kFewRows], jl[kFewWaves][kFewRows];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int n = lane & 15, g4 = lane >> 4;
    // blockIdx.x: (row block, split, key head, sequence), the last slowest.
    int w = blockIdx.x;
    const int blocks = (((a.b.off ? a.b.max_rows : a.b.rows) * a.g) + kFewRows - 1) / kFewRows;
    const int rb = w % blocks; w /= blocks;
    const int sp = w % a.splits; w /= a.splits;
    const int h = w % a.c.Hkv, i = w / a.c.Hkv;
    const int T = row_count(a.b, i), slot = slot_of(a.b, i);
    const int r0 = rb * kFewRows;
    if (r0 >= T * a.g) return;
    const bool known = slot >= 0 && slot < a.pg.num_seqs;
    const int len = known ? a.pg.length[slot] : 0;
    const int row = r0 + n, t = row / a.g, hh = h * a.g + row - t * a.g;
    const bool live = t < T;
    const int last = live ? (a.causal ? len - T + t : len - 1) : -1;       // last key seen
    const int tmax = (r0 + kFewRows - 1) / a.g < T - 1 ? (r0 + kFewRows - 1) / a.g : T - 1;
    const int end = a.causal ? len - T + tmax + 1 : len;                   // keys of the block
    // The split's keys; the last split of the launch takes all that is left.
    const int lo = sp * a.chunk;
    int hi = sp == a.splits - 1 ? end : lo + a.chunk;
    hi = hi < end ? hi : end;
    if (sp > 0 && lo >= end) return;
    const int* table = a.pg.table + (size_t)(known ? slot : 0) * a.pg.max_pages;

    // Queries: reduction slots as the keys' 16-byte loads number them.
    bf16x8 q[NC][2];
    {
        const long long qrow = (long long)row_begin(a.b, i) + t;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const int e = c * 64 + g4 * 16 + f * 8;
                u32x4 x = {0, 0, 0, 0};
                if (live && e < a.c.d)
                    x = *reinterpret_cast<const u32x4*>(a.q + qrow * a.q_stride + (long long)hh * a.c.d + e);
                q[c][f] = __builtin_bit_cast(bf16x8, x);
            }
    }
    f32x4 acc[NC][4] = {};
    float m = -INFINITY, l = 0.f;
    int ref = kMinExp;

    const int groups = hi > 0 ? (hi + 15) >> 4 : 0;                        // of 16 tokens
    Window win;
    win.base = -1;
    auto load_window = [&](int group) {
        win.base = group & ~63;
        const int mine = win.base + lane;
        win.page = 0; win.ks = 1.f; win.vs = 1.f;
        if (mine < groups) {
            win.page = table[mine >> (a.pg.shift - 4)];
            const size_t at = (size_t)win.page * a.c.Hkv + h;
            win.ks = a.c.ks[at];
            win.vs = a.c.vs[at];
        }
    };
    struct Codes { u32x4 k[2][NC], v[2][NC]; float ks[2], vs[2]; };
    auto load_step = [&](int pos, Codes& x) {
        const int gr = pos >> 4;
        if ((gr & ~63) != win.base) load_window(gr);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // A group past the end reads the one before it again; its keys are masked.
            const int at = gr + u < groups ? gr + u : groups - 1, src = at & 63;
            const int page = __builtin_amdgcn_readlane(win.page, src);
            x.ks[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(win.ks), src));
            x.vs[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(win.vs), src));
            const int tok = (at << 4) & ((1 << a.pg.shift) - 1);
            const size_t off = ((size_t)page * a.c.Hkv + h) * a.c.block + (size_t)tok * DP;
            const unsigned char* kp = a.c.k + off + n * DP + g4 * 16;
            const unsigned char* vp = a.c.v + off + g4 * DP * 4 + n * 16;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                x.k[u][c] = *reinterpret_cast<const u32x4*>(kp + c * 64);
                x.v[u][c] = *reinterpret_cast<const u32x4*>(vp + c * 256);
            }
        }
    };
    auto compute = [&](int pos, Codes& x) {
        f32x4 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    codes_bf16(x.k[u][c][0], x.k[u][c][1], x.ks[u]), q[c][0], s[u], 0, 0, 0);
                s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    codes_bf16(x.k[u][c][2], x.k[u][c][3], x.ks[u]), q[c][1], s[u], 0, 0, 0);
            }
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = pos + u * 16 + g4 * 4 + e;
                s[u][e] = key <= last && key < hi ? s[u][e] * a.scale2 : -INFINITY;
                top = fmaxf(top, s[u][e]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // The largest value scale so far; a step whose scales are larger shrinks the sums.
        const int e0 = exp_of(x.vs[0]), e1 = exp_of(x.vs[1]), em = e0 > e1 ? e0 : e1;
        const int now = em > ref ? em : ref;
        const float base = top == -INFINITY ? 0.f : top;
        const float fade = __builtin_amdgcn_exp2f(m - base);             // 0 while m is -inf
        const int dref = ref - now < -126 ? -126 : ref - now;
        const float fo = fade * exp_scale(dref);
        m = top;
        ref = now;
        float sum = 0.f;
        f16x8 p;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = __builtin_amdgcn_exp2f(s[u][e] - base + kLift);
                sum += y[e];
            }
            const f16x2 a0 = round_f16(y[0], y[1]), a1 = round_f16(y[2], y[3]);
            p[u * 4] = a0[0]; p[u * 4 + 1] = a0[1]; p[u * 4 + 2] = a1[0]; p[u * 4 + 3] = a1[1];
        }
        l = l * fade + sum;
        const float v0 = exp_scale(e0 - now < -126 ? -126 : e0 - now);
        const float v1 = exp_scale(e1 - now < -126 ? -126 : e1 - now);
        // Codes behind the sequence's end may be anything, NaN among it: 0 * NaN is not 0.
        if (pos + kStep > len) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int left = len - (pos + u * 16 + g4 * 4);
                const unsigned keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int d = 0; d < 4; ++d) x.v[u][c][d] &= keep;
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                acc[c][d] *= fo;
                acc[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    codes_f16(x.v[0][c][d], v0, x.v[1][c][d], v1), p, acc[c][d], 0, 0, 0);
            }
    };
    {
        Codes x[2];
        const int stride = kStep * kFewWaves;
        int pos = lo + wave * kStep;
        if (pos < hi) load_step(pos, x[0]);
        while (pos < hi) {
            if (pos + stride < hi) load_step(pos + stride, x[1]);
            compute(pos, x[0]);
            pos += stride;
            if (pos >= hi) break;
            if (pos + stride < hi) load_step(pos + stride, x[0]);
            compute(pos, x[1]);
            pos += stride;
        }
    }
    // The row's sum over the lane groups (each added its own tokens), then the waves join.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    constexpr float kDrop = 0x1p-14f;                       // undoes kLift
    if (g4 == 0) { jm[wave][n] = m; jl[wave][n] = l * kDrop; }
    __syncthreads();
    // 16 threads per row, four elements each of every 64-element chunk.
    const int r = threadIdx.x >> 4, part = threadIdx.x & 15;
    const int rr = r0 + r, rt = rr / a.g, rh = h * a.g + rr - rt * a.g;
    float top = jm[0][r];
#pragma unroll
    for (int x = 1; x < kFewWaves; ++x) top = fmaxf(top, jm[x][r]);
    float wgt[kFewWaves], sum = 0.f;
#pragma unroll
    for (int x = 0; x < kFewWaves; ++x) {
        wgt[x] = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(jm[x][r] - top);
        sum += wgt[x] * jl[x][r];
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const float lse2 = sum > 0.f ? top + __builtin_amdgcn_logf(sum) : -INFINITY;   // base 2
    const float unref = exp_scale(ref - (int)kLift);
    const long long orow = (long long)row_begin(a.b, i) + rt;
    const size_t at = ((size_t)orow * a.H + rh) * a.splits + sp;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c) __syncthreads();
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) jo[wave][n][g4 * 16 + e * 4 + d] = acc[c][d][e] * unref;
        __syncthreads();
        const int e0 = c * 64 + part * 4;
        if (rt >= T || e0 >= a.c.d) continue;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < kFewWaves; ++x)
            y += wgt[x] * *reinterpret_cast<const f32x4*>(&jo[x][r][part * 4]);
        y *= inv;
        if (a.splits == 1) {
            ushort4 o;
            o.x = __builtin_bit_cast(unsigned short, (__bf16)y[0]);
            o.y = __builtin_bit_cast(unsigned short, (__bf16)y[1]);
            o.z = __builtin_bit_cast(unsigned short, (__bf16)y[2]);
            o.w = __builtin_bit_cast(unsigned short, (__bf16)y[3]);
            *reinterpret_cast<ushort4*>(a.out + orow * a.out_stride + (long long)rh * a.c.d + e0) = o;
        } else {
            *reinterpret_cast<f32x4*>(a.part_o + at * a.c.d + e0) = y;
        }
    }
    if (part == 0 && rt < T) {
        if (a.splits == 1) { if (a.lse) a.lse[orow * a.H + rh] = lse2 * kLn2; }
        else a.part_l[at] = lse2;
    }
}

// Joins the splits of a row and head: weights 2^(lse - max), each split's output already
// divided by its own sum.  A wave per (row, head).
__global__ __launch_bounds__(256) void attend_join(AttendArgs a) {
    const int lane = threadIdx.x & 63;
    const int maxr = a.b.off ? a.b.max_rows : a.b.rows;
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int per = maxr * a.H;
    const int i = (int)(w / per), x = (int)(w - (long long)i * per), t = x / a.H, hh = x - t * a.H;
    if (i >= a.b.n) return;
    const int T = row_count(a.b, i), slot = slot_of(a.b, i);
    if (t >= T) return;
    const int len = slot >= 0 && slot < a.pg.num_seqs ? a.pg.length[slot] : 0;
    // The keys of the row block that the row was computed in decide which splits exist.
    const int r = t * a.g + hh % a.g, r1 = (r / kFewRows + 1) * kFewRows - 1;
    const int tm = r1 / a.g < T - 1 ? r1 / a.g : T - 1;
    const int end = a.causal ? len - T + tm + 1 : len;
    int parts = end > 0 ? (end + a.chunk - 1) / a.chunk : 1;
    parts = parts < a.splits ? parts : a.splits;
    const long long orow = (long long)row_begin(a.b, i) + t;
    const size_t at = ((size_t)orow * a.H + hh) * a.splits;
    float top = -INFINITY;
    for (int p = lane; p < parts; p += 64) top = fmaxf(top, a.part_l[at + p]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    float sum = 0.f, y[4] = {};
    const float base = top == -INFINITY ? 0.f : top;
    for (int p = 0; p < parts; ++p) {
        const float wgt = __builtin_amdgcn_exp2f(a.part_l[at + p] - base);
        sum += wgt;
        for (int e = lane, k = 0; e < a.c.d; e += 64, ++k) y[k] += wgt * a.part_o[(at + p) * a.c.d + e];
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    unsigned short* o = a.out + orow * a.out_stride + (long long)hh * a.c.d;
    for (int e = lane, k = 0; e < a.c.d; e += 64, ++k)
        o[e] = __builtin_bit_cast(unsigned short, (__bf16)(y[k] * inv));
    if (lane == 0 && a.lse)
        a.lse[orow * a.H + hh] = sum > 0.f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

}  // namespace

// Keys per split and splits: enough workgroups to fill the chip several times over, at
// least 128 keys (a step of every wave) each.
void attend_splits(const CacheView& c, const BatchView& b, int H, long long max_tokens, int* chunk,
                   int* splits) {
    const long long rows = (long long)(b.off ? b.max_rows : b.rows) * (H / c.Hkv);
    const long long tasks = (long long)b.n * c.Hkv * ((rows + kFewRows - 1) / kFewRows);
    const long long least = kStep * kFewWaves;
    long long want = 2048 / tasks;
    const long long most = (max_tokens + least - 1) / least;
    want = want < 1 ? 1 : want > most ? most : want;
    want = want < 1 ? 1 : want;
    long long per = (max_tokens + want - 1) / want;
    per = (per + kStep - 1) / kStep * kStep;
    per = per < least ? least : per;
    *chunk = (int)per;
    *splits = (int)((max_tokens + per - 1) / per);
    if (*splits < 1) *splits = 1;
}

hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t s) {
    const long long rows = (long long)(a.b.off ? a.b.max_rows : a.b.rows) * a.g;
    const long long blocks = (rows + kFewRows - 1) / kFewRows;
    const dim3 grid((unsigned)(blocks * a.splits * a.c.Hkv * a.b.n)), block(64 * kFewWaves);
    hipError_t e = a.c.dp == 64    ? launch(attend_few<64>, grid, block, 0, s, a)
                   : a.c.dp == 128 ? launch(attend_few<128>, grid, block, 0, s, a)
                                   : launch(attend_few<256>, grid, block, 0, s, a);
    if (e != hipSuccess || a.splits == 1) return e;
    const long long waves = (long long)a.b.n * (a.b.off ? a.b.max_rows : a.b.rows) * a.H;
    return launch(attend_join, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a);
}

}  // namespace occam
