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
// scale into two bf16 (keys) or f16 (values) numbers.  Keys are exact in bf16, and so are
// values in f16, converted relative to the largest value scale met so far (`ref`) as long as
// all scales met lie within 2^kSpread (see Scales below).  Probabilities are rounded to f16
// (half a step, 2^-11 of them; a bf16 one, 2^-8, would cost as much as rounding the output
// does), held times 2^14 (few rows) or 2^9 (many): they keep all bits down to 2^-28 and
// 2^-23, and are off by at most 2^-39 and 2^-34 below.  Maxima, sums and outputs are float32.
#include <type_traits>

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
// Scales.  Pages have scales of their own, 2^-100 to 2^120.  A row's output is a sum of codes
// times weights, w_j = p_j s_j, and a weight is held relative to ref.  While the scales met lie
// within 2^kFewSpread or 2^kManySpread, the row's largest weight is at least 2^-spread of that,
// so weights are within 2^-27 of the largest, and the powers of two between scale and ref are
// in the converted values.  From the first keys on that pass the spread (which may be keys that
// some rows do not see, or give no probability) a row's sums are in units of an exponent of its
// own, ceil(W - m), W = the largest of (score + scale's exponent, base 2) of the keys it has
// seen, m its maximum; the exponent that gives a weight has the scale in it, and values are bare
// codes.  So what a row does not see, or gives little, moves nothing in its output by more than
// 2^-26 of its largest weight, and ordinary caches, whose scales differ by a few binades, never
// get there.  (Keeping rows' own units in the common loop costs 25 %: its registers spill.
// Watching the spread costs 0.3 us of 11 in a small call and 1.5 % of the prompt below.)
// ---------------------------------------------------------------------------------------
constexpr int kFewSpread = 12, kManySpread = 7;
// The unit of a row's sums: the exponent of its largest weight (`w`) over its maximum.
__device__ __forceinline__ int unit_of(float w, float m) { return w == -INFINITY ? 0 : (int)ceilf(w - m); }

// ---------------------------------------------------------------------------------------
// Division of work.  Per key head there is a row block of so many rows of every sequence,
// and of each as many units of keys as its rows see.  Lengths are known on the device only.
// A row block's keys may be cut into parts; each leaves its output and normaliser in a slot
// of the workspace, and attend_join puts a block's parts together.
// ---------------------------------------------------------------------------------------
typedef AttendBlock Block;
// Later row blocks of every sequence come first: under a causal mask they are the long ones.
__device__ __forceinline__ Block block_of(const AttendArgs& a, int entry, int rows) {
    Block t;
    const int rb = entry / a.b.n;
    t.i = entry - rb * a.b.n;
    t.r0 = (a.shape.blocks - 1 - rb) * rows;
    t.T = row_count(a.b, t.i);
    t.slot = slot_of(a.b, t.i);
    const bool known = t.slot >= 0 && t.slot < a.pg.num_seqs;
    t.len = known ? a.pg.length[t.slot] : 0;
    t.slot = known ? t.slot : 0;
    const int last = (t.r0 + rows - 1) / a.g;
    t.end = a.causal ? t.len - t.T + (last < t.T - 1 ? last : t.T - 1) + 1 : t.len;
    return t;
}
// One workgroup, the last, which has little or nothing else to do, looks for slots that there
// are not and for rows that the offsets give wrongly.
template <int NT>
__device__ __forceinline__ void report_faults(const AttendArgs& a) {
    if (!a.b.seq && !a.b.off) return;
    for (int i = threadIdx.x; i < a.b.n; i += NT)
        if (const int bad = batch_faults(a.pg, slot_of(a.b, i), stated_rows(a.b, i))) atomicOr(a.pg.status, bad);
}
// Units of keys of a row block: one where there is nothing to see (zeros are written), none
// where there are no rows.
__device__ __forceinline__ int units_of(const AttendArgs& a, const Block& t, int unit) {
    return t.r0 >= t.T * a.g ? 0 : t.end > 0 ? (t.end + unit - 1) / unit : 1;
}

// The few-row form lays the row blocks end to end and cuts the whole into equal ranges, one
// per workgroup, as many as the chip holds at once.  Every workgroup sums the lengths up for
// itself.  A range has at most two parts: of the block it goes on with (slot 0) and of the
// one it leaves unfinished (slot 1).
struct Range {
    int start, stop;               // in units
    int entry, first;              // the row block that holds `start`, and its first unit
    int each;                      // units per range
    Block block;                   // that row block
};
// Range `w` of a.shape.ranges over the row blocks of the batch; all NT threads call it.  `red`:
// NT / 64 + 8 ints of LDS.
template <int NT>
__device__ __forceinline__ Range range_of(const AttendArgs& a, int w, int rows, int unit,
                                          int least, int* red) {
    const int entries = a.b.n * a.shape.blocks, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int total = 0, base = 0, mine = 0, before = 0;
    Block block = {};
    Range r;
    auto divide = [&]() {
        r.each = (total + a.shape.ranges - 1) / a.shape.ranges;
        r.each = r.each < least ? least : r.each;
        // (Products past 2^31 would be past the end: ranges * each < total + ranges * least.)
        r.start = w * r.each;
        r.stop = r.start + r.each < total ? r.start + r.each : total;
        r.entry = r.first = 0;
    };
    if (entries <= 64) {                   // every wave by itself
        if (lane < entries) {
            block = block_of(a, lane, rows);
            mine = units_of(a, block, unit);
        }
        int s = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(s, o);
            if (lane >= o) s += y;
        }
        total = __builtin_amdgcn_readlane(s, 63);
        divide();
        if (r.start >= total) return r;
        const int from = __ffsll((unsigned long long)__ballot(r.start < s)) - 1;   // sums ascend
        r.entry = from;
        r.first = __builtin_amdgcn_readlane(s - mine, from);
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, from); };
        r.block = Block{of(block.i), of(block.T), of(block.len), of(block.slot), of(block.r0), of(block.end)};
        return r;
    }
    // Exclusive prefix of the units of entries c .. c + NT - 1, and their sum.
    auto scan = [&](int c) {
        const int e = c + (int)threadIdx.x;
        mine = 0;
        if (e < entries) {
            block = block_of(a, e, rows);
            mine = units_of(a, block, unit);
        }
        int s = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(s, o);
            if (lane >= o) s += y;
        }
        __syncthreads();
        if (lane == 63) red[wave] = s;
        __syncthreads();
        int sum = 0;
        before = s - mine;
#pragma unroll
        for (int x = 0; x < NT / 64; ++x) {
            const int y = red[x];
            before += x < wave ? y : 0;
            sum += y;
        }
        return sum;
    };
    for (int c = 0; c < entries; c += NT) total += scan(c);
    divide();
    if (r.start >= total) return r;
    for (int c = 0; c < entries; c += NT) {
        const int sum = entries <= NT ? total : scan(c);
        if (r.start < base + sum) {
            const int at = base + before;
            if (at <= r.start && r.start < at + mine) {
                int* out = red + NT / 64;
                out[0] = c + (int)threadIdx.x; out[1] = at;
                out[2] = block.i; out[3] = block.T; out[4] = block.len;
                out[5] = block.slot; out[6] = block.r0; out[7] = block.end;
            }
            __syncthreads();
            const int* out = red + NT / 64;
            r.entry = uniform(out[0]);
            r.first = uniform(out[1]);
            r.block = Block{uniform(out[2]), uniform(out[3]), uniform(out[4]),
                            uniform(out[5]), uniform(out[6]), uniform(out[7])};
            break;
        }
        base += sum;
    }
    return r;
}
// Tells attend_join of the row block that the range's start cuts, where this is the block's
// first cut: {entry, parts, first slot, slots from a part to the next}; {-1} otherwise.
// Written for every range, the empty ones behind the end of the work among them:
// attend_join reads them all.
__device__ __forceinline__ void note_cut(const AttendArgs& a, const Range& r, int w, int unit) {
    int4 cut = {-1, 0, 0, 0};
    if (r.start < r.stop && r.first < r.start && r.first >= r.start - r.each) {
        const int end = r.first + units_of(a, r.block, unit);
        cut = int4{r.entry, (end - 1) / r.each - w + 2, 2 * (w - 1) + 1, 2};
    }
    a.cuts[w] = cut;
}

// ---------------------------------------------------------------------------------------
// Few rows: 16 rows of one key head at a time (or 32: NR = 2), their keys dealt to the
// workgroup's four waves in steps of 32, joined in LDS.  Bound by reading the codes once: a wave
// has the loads of two steps in flight (8 KB each at d = 128) and several workgroups share a CU.
// One row of each of 8 sequences of 16640 tokens, 32 key heads of 128: 174 us, 6.3 TB/s; of 64
// sequences of 272 to 4608 tokens, 8 key heads: 54 us, 5.2 TB/s, about 8 us of it before the
// first codes arrive (rows, lengths, pages, codes: four loads one after the other); of one
// sequence of 3011 tokens: 7 us, nothing but latency.  Scales past the spread change none of them.
// ---------------------------------------------------------------------------------------
constexpr int kStep = 32, kFewWaves = 4, kFewRows = 16;
constexpr int kFewUnit = kStep * kFewWaves;
constexpr long long kFewBytes = 64ll << 20;   // of codes: from here on 17 to 32 rows are one block
// Workgroups of a CU: what the registers of 16 * NR rows leave room for.
constexpr int few_resident(int dp, int nr) {
    return dp == 64 ? (nr == 1 ? 4 : 3) : dp == 128 ? (nr == 1 ? 3 : 2) : 1;
}

// Page numbers and scales of the 64 16-token groups around a wave's position, one per lane.
struct Window {
    int base, page;
    float ks, vs;
};

template <int DP, int NR, bool STREAM>
__global__ __launch_bounds__(64 * kFewWaves, few_resident(DP, NR)) void attend_few(AttendArgs a) {
    constexpr int NC = DP / 64;            // 64-element chunks of a row
    constexpr int ROWS = kFewRows * NR;
    __shared__ float jo[kFewWaves][kFewRows][64 + 4];
    __shared__ float jm[kFewWaves][ROWS], jl[kFewWaves][ROWS];
    __shared__ int ju[kFewWaves][ROWS];
    __shared__ int red[kFewWaves + 8];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int n = lane & 15, g4 = lane >> 4;
    const int w = blockIdx.x / a.c.Hkv, h = blockIdx.x - w * a.c.Hkv;
    const Range range = range_of<64 * kFewWaves>(a, w, ROWS, kFewUnit, 1, red);
    if (a.shape.slots > 0 && h == 0 && threadIdx.x == 0) note_cut(a, range, w, kFewUnit);
    if (w + 1 == a.shape.ranges && h + 1 == a.c.Hkv) report_faults<64 * kFewWaves>(a);
    int entry = range.entry, at_unit = range.start - range.first;
    for (int now = range.start; now < range.stop && entry < a.b.n * a.shape.blocks; ++entry, at_unit = 0) {
    const Block block = entry == range.entry ? range.block : block_of(a, entry, ROWS);
    const int units = units_of(a, block, kFewUnit);
    if (units == 0) continue;
    const int take = units - at_unit < range.stop - now ? units - at_unit : range.stop - now;
    const bool whole = take == units;
    now += take;
    const int i = block.i, T = block.T, len = block.len, r0 = block.r0;
    const int lo = at_unit * kFewUnit;
    const int hi = lo + take * kFewUnit < block.end ? lo + take * kFewUnit : block.end;
    const int* table = a.pg.table + (size_t)block.slot * a.pg.max_pages;

    // Queries: reduction slots as the keys' 16-byte loads number them.
    bf16x8 q[NR][NC][2];
    int last[NR];                          // last key that the lane's rows see
    float m[NR], l[NR];
#pragma unroll
    for (int b = 0; b < NR; ++b) {
        const int row = r0 + b * kFewRows + n, t = row / a.g, hh = h * a.g + row - t * a.g;
        const bool live = t < T;
        last[b] = live ? (a.causal ? len - T + t : len - 1) : -1;
        m[b] = -INFINITY;
        l[b] = 0.f;
        const long long qrow = (long long)row_begin(a.b, i) + t;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const int e = c * 64 + g4 * 16 + f * 8;
                u32x4 x = {0, 0, 0, 0};
                if (live && e < a.c.d)
                    x = *reinterpret_cast<const u32x4*>(a.q + qrow * a.q_stride + (long long)hh * a.c.d + e);
                q[b][c][f] = __builtin_bit_cast(bf16x8, x);
            }
    }
    f32x4 acc[NR][NC][4] = {};
    int ref = kMinExp, least = kMaxExp;    // the largest and the least value scale so far

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
            const int tok = (at << 4) & ((1 << a.pg.shift) - 1);
            const size_t off = ((size_t)page * a.c.Hkv + h) * a.c.block + (size_t)tok * DP;
            const unsigned char* kp = a.c.k + off + n * DP + g4 * 16;
            const unsigned char* vp = a.c.v + off + g4 * DP * 4 + n * 16;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                x.k[u][c] = get<STREAM>(reinterpret_cast<const u32x4*>(kp + c * 64));
                x.v[u][c] = get<STREAM>(reinterpret_cast<const u32x4*>(vp + c * 256));
            }
        }
        // The scales after the codes, which need only the page numbers of a new window.
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int src = (gr + u < groups ? gr + u : groups - 1) & 63;
            x.ks[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(win.ks), src));
            x.vs[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(win.vs), src));
        }
    };
    // Whether the scales met, this step's among them, lie within the spread.
    auto regular = [&](const Codes& x) {
        const int e0 = exp_of(x.vs[0]), e1 = exp_of(x.vs[1]), hi2 = e0 > e1 ? e0 : e1, lo2 = e0 < e1 ? e0 : e1;
        return (hi2 > ref ? hi2 : ref) - (lo2 < least ? lo2 : least) <= kFewSpread;
    };
    // OWN: rows have units of their own (`unit`, and `most`, their largest weight's exponent).
    int unit[NR];
    float most[NR];
    auto compute = [&](auto own, int pos, Codes& x) {
        constexpr bool OWN = decltype(own)::value;
        f32x4 s[NR][2] = {};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const bf16x8 k = codes_bf16(x.k[u][c][2 * f], x.k[u][c][2 * f + 1], x.ks[u]);
#pragma unroll
                    for (int b = 0; b < NR; ++b)
                        s[b][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[b][c][f], s[b][u], 0, 0, 0);
                }
        // The largest value scale so far; a step whose scales are larger shrinks the sums.
        const int e0 = exp_of(x.vs[0]), e1 = exp_of(x.vs[1]);
        float shrink = 1.f;
        if constexpr (!OWN) {
            const int em = e0 > e1 ? e0 : e1, el = e0 < e1 ? e0 : e1, now = em > ref ? em : ref;
            shrink = exp_scale(ref - now < -126 ? -126 : ref - now);       // (-126: of sums of zero)
            ref = now;
            least = el < least ? el : least;
        }
        f16x8 p[NR];
        float fo[NR];
#pragma unroll
        for (int b = 0; b < NR; ++b) {
            float top = m[b], weight = -INFINITY;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = pos + u * 16 + g4 * 4 + e;
                    s[b][u][e] = key <= last[b] && key < hi ? s[b][u][e] * a.scale2 : -INFINITY;
                    top = fmaxf(top, s[b][u][e]);
                    if constexpr (OWN) weight = fmaxf(weight, s[b][u][e] + (float)(u ? e1 : e0));
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -INFINITY ? 0.f : top;
            const float fade = __builtin_amdgcn_exp2f(m[b] - base);      // 0 while m is -inf
            fo[b] = fade * shrink;
            float by[2] = {0.f, 0.f};
            if constexpr (OWN) {
                weight = fmaxf(weight, __shfl_xor(weight, 16));
                weight = fmaxf(weight, __shfl_xor(weight, 32));
                most[b] = fmaxf(most[b], weight);
                const int now = unit_of(most[b], base);
                fo[b] = __builtin_amdgcn_exp2f(m[b] - base + (float)(unit[b] - now));
                unit[b] = now;
                by[0] = (float)(now - e0);
                by[1] = (float)(now - e1);
            }
            m[b] = top;
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = __builtin_amdgcn_exp2f(s[b][u][e] - base + kLift);
                    sum += y[e];
                    if constexpr (OWN) y[e] = __builtin_amdgcn_exp2f(s[b][u][e] - base + kLift - by[u]);
                }
                const f16x2 a0 = round_f16(y[0], y[1]), a1 = round_f16(y[2], y[3]);
                p[b][u * 4] = a0[0]; p[b][u * 4 + 1] = a0[1]; p[b][u * 4 + 2] = a1[0]; p[b][u * 4 + 3] = a1[1];
            }
            l[b] = l[b] * fade + sum;
        }
        const float v0 = OWN ? 1.f : exp_scale(e0 - ref), v1 = OWN ? 1.f : exp_scale(e1 - ref);
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
                const f16x8 v = codes_f16(x.v[0][c][d], v0, x.v[1][c][d], v1);
#pragma unroll
                for (int b = 0; b < NR; ++b) {
                    acc[b][c][d] *= fo[b];
                    acc[b][c][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[b], acc[b][c][d], 0, 0, 0);
                }
            }
    };
    {
        Codes x[2];
        const int stride = kStep * kFewWaves;
        int pos = lo + wave * kStep;
        const std::false_type shared;
        const std::true_type own;
        if (pos < hi) load_step(pos, x[0]);
        while (pos < hi) {
            if (pos + stride < hi) load_step(pos + stride, x[1]);
            if (!regular(x[0])) break;
            compute(shared, pos, x[0]);
            pos += stride;
            if (pos >= hi) break;
            if (pos + stride < hi) load_step(pos + stride, x[0]);
            if (!regular(x[1])) break;
            compute(shared, pos, x[1]);
            pos += stride;
        }
#pragma unroll
        for (int b = 0; b < NR; ++b) {
            unit[b] = ref;
            most[b] = m[b] + (float)ref;
        }
        for (; pos < hi; pos += stride) {          // (one step at a time: these are rare)
            load_step(pos, x[0]);
            compute(own, pos, x[0]);
        }
    }
    // The row's sum over the lane groups (each added its own tokens), then the waves join.
    constexpr float kDrop = 0x1p-14f;                       // undoes kLift
    __syncthreads();                                        // read for the row block before
#pragma unroll
    for (int b = 0; b < NR; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
        if (g4 == 0) {
            jm[wave][b * kFewRows + n] = m[b];
            jl[wave][b * kFewRows + n] = l[b] * kDrop;
            ju[wave][b * kFewRows + n] = unit[b];
        }
    }
    __syncthreads();
    // 16 threads per row, four elements each of every 64-element chunk.
    const int r = threadIdx.x >> 4, part = threadIdx.x & 15;
#pragma unroll
    for (int b = 0; b < NR; ++b) {
        const int rb = b * kFewRows + r, rr = r0 + rb, rt = rr / a.g, rh = h * a.g + rr - rt * a.g;
        float top = jm[0][rb];
#pragma unroll
        for (int x = 1; x < kFewWaves; ++x) top = fmaxf(top, jm[x][rb]);
        // A wave's outputs are in units of 2^(m + unit), and come together in the largest such;
        // their mean is taken before the unit, as a sum of values could pass float32's range.
        float wgt[kFewWaves], units = -INFINITY, sum = 0.f;
#pragma unroll
        for (int x = 0; x < kFewWaves; ++x) {
            wgt[x] = jm[x][rb] + (float)ju[x][rb];
            units = fmaxf(units, wgt[x]);
            sum += top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(jm[x][rb] - top) * jl[x][rb];
        }
#pragma unroll
        for (int x = 0; x < kFewWaves; ++x)
            wgt[x] = sum > 0.f ? __builtin_amdgcn_exp2f(wgt[x] - units) : 0.f;
        const float inv = sum > 0.f ? kDrop / sum : 0.f, up = sum > 0.f ? __builtin_amdgcn_exp2f(units - top) : 0.f;
        const float lse2 = sum > 0.f ? top + __builtin_amdgcn_logf(sum) : -INFINITY;   // base 2
        const long long orow = (long long)row_begin(a.b, i) + rt;
        const size_t at = ((size_t)h * a.shape.slots + 2 * w + (lo > 0 ? 0 : 1)) * ROWS + rb;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (b || c) __syncthreads();
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) jo[wave][n][g4 * 16 + e * 4 + d] = acc[b][c][d][e];
            __syncthreads();
            const int e0 = c * 64 + part * 4;
            if (rt >= T || e0 >= a.c.d) continue;
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < kFewWaves; ++x)
                y += wgt[x] * *reinterpret_cast<const f32x4*>(&jo[x][r][part * 4]);
            y = y * inv * up;
            if (whole) {
                ushort4 o;
                o.x = __builtin_bit_cast(unsigned short, (__bf16)y[0]);
                o.y = __builtin_bit_cast(unsigned short, (__bf16)y[1]);
                o.z = __builtin_bit_cast(unsigned short, (__bf16)y[2]);
                o.w = __builtin_bit_cast(unsigned short, (__bf16)y[3]);
                *reinterpret_cast<ushort4*>(a.out + orow * a.out_stride + (long long)rh * a.c.d + e0) = o;
            } else {
                *reinterpret_cast<f32x4*>(a.part_o + at * DP + e0) = y;
            }
        }
        if (part == 0 && rt < T) {
            if (whole) { if (a.lse) a.lse[orow * a.H + rh] = lse2 * kLn2; }
            else a.part_l[at] = lse2;
        }
    }
    }
}

// ---------------------------------------------------------------------------------------
// Many rows: 32 rows of one key head per wave, WAVES waves per workgroup, which share every
// tile of 64 keys and values through LDS.  The tile is converted to 16 bits once, on its way
// into LDS (a wave that converted its own operands would spend as long on that as on the
// products).  The running maximum only moves the sums when some row's maximum passed the
// one in use by more than 2^6: probabilities are held times 2^9, so they stay within 2^15.
//
// A wave alternates between a vector phase (the softmax of tile t) and a matrix phase (the
// output of tile t, the scores of t + 1).  With eight waves, the two of a SIMD belong to two
// groups, B a phase behind A, so that one feeds the matrix core while the other does vector
// work.  There is one barrier per tile: behind the matrix phase for A, before it for B.
// Between two barriers (step t) A reads values t and keys t + 1, B values t - 1 and keys t,
// and both store their share of tile t + 2 (beside their products, whose issue slots leave
// room), so four buffers are enough: tile t + 2 takes the place of t - 2, whose values B read
// last in step t - 1.  The codes of two further tiles are on their way from memory.
// (A barrier behind every phase: 337 us for the prompt below, against 328.)
// With four waves (up to 128 rows, and dp = 64 and 256) the other waves of a CU are another
// workgroup's, if it has room for one, and a tile is stored in the vector phase before its
// matrix phase, with a barrier behind each and two buffers.
//
// What bounds it is the issue of vector instructions beside the matrix core (the products of a
// tile would take 2100 clocks of a SIMD, the 290 other instructions of its two waves about as
// many) and the card's power: the prompt below takes 281 us on constant data, at a higher clock,
// as a large library product gains 28 % there.  In a long run (the first dispatches after idle
// take a tenth longer) a causal prompt of 4 x 3012 tokens, 32 heads of 128: 328 us, 906 TFLOP/s
// (large library products 1371 to 1398), all keys for every row 563 us, 1056; 16 to 512 text rows
// of 32 images each, behind 256 to 4096 tokens, 32 heads on 8: 243 us, 913 TFLOP/s.  4 x 3000
// tokens with 32 heads of 64: 738 TFLOP/s, with 16 of 256: 727.  The loop for scales past the
// spread fetches a tile at a time: 523 us for the prompt.
// ---------------------------------------------------------------------------------------
constexpr int kTile = 64;
constexpr int kManyLeast = 4;              // tiles per part at least
constexpr int kManyRounds = 4;             // of parts (their outputs: 128 KB each at dp = 128)
constexpr float kManyLift = 9.f, kManySlack = 6.f;
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float max_over_halves(float x) {            // lanes l and l ^ 32
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// A barrier that orders LDS only: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A matrix phase reads its operands from LDS this many products ahead (the compiler by
// itself reads two and waits for them; with 8 and 12 the prompt takes 1 and 2 % longer).  It
// runs at a higher wave priority than the vector phase beside it: 12 % at the prompt.
constexpr int kReads = 6;

// The row blocks of a ragged batch, longest first: a workgroup that starts late on a long
// one would end long after the others.  (In which order blocks of one length come is left
// open; it decides where they run, not what they give.)  5 us; the text rows above take
// 244 us with it and 303 without.
__global__ __launch_bounds__(kMaxOrder) void attend_order(AttendArgs a, int entries) {
    __shared__ int bin[kMaxOrder], sums[kMaxOrder / 64];
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    bin[e] = 0;
    __syncthreads();
    Block b = {};
    int to = 0, at = 0;
    if (e < entries) {
        b = block_of(a, e, a.shape.block_rows);
        const int units = units_of(a, b, kTile);
        to = kMaxOrder - 1 - (units < kMaxOrder ? units : kMaxOrder - 1);
        at = atomicAdd(&bin[to], 1);
    }
    __syncthreads();
    const int own = bin[e];
    int s = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(s, o);
        if (lane >= o) s += y;
    }
    if (lane == 63) sums[wave] = s;
    __syncthreads();
    int before = s - own;
    for (int w = 0; w < wave; ++w) before += sums[w];
    bin[e] = before;
    __syncthreads();
    if (e < entries) a.order[bin[to] + at] = b;
}

// A buffer: keys [64] of 2 DP + 16 bytes, so that 16 rows' reads of 16 bytes fall on all
// banks; values [tile of 32][16 tokens][half][DP][8 tokens], the 8 reduction slots of a lane.
template <int DP> constexpr int many_keys() { return kTile * (DP * 2 + 16); }
template <int DP> constexpr int many_buf() { return many_keys<DP>() + kTile * DP * 2; }
template <int DP, int WAVES> constexpr int many_lds() { return WAVES / 2 * many_buf<DP>(); }

// (Waves of a SIMD: 168 registers leave room for three at dp = 64, 199 us against 223 with two for
// 4 x 3000 tokens of 32 heads.)
template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP == 256 ? 1 : DP == 64 ? 3 : 2) void attend_many(AttendArgs a) {
    constexpr int THREADS = 64 * WAVES, ROWS = 32 * WAVES;
    constexpr int AHEAD = WAVES / 4, BUFS = WAVES / 2;
    constexpr int SETS = WAVES / 4;          // tiles in flight from memory
    constexpr int NK = DP / 16;              // 16-element steps of the score product
    constexpr int ND = DP / 32;              // 32-element tiles of the output
    constexpr int CH = DP / 8;               // 16-byte chunks of a key row in LDS
    constexpr int UK = kTile * DP / 16 / THREADS;    // key units (16 codes) per thread
    constexpr int UV = kTile * DP / 16 / THREADS;    // value units (2 elements x 8 tokens)
    static_assert(UK * THREADS * 16 == kTile * DP, "tile units");
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int KP = DP * 2 + 16, HALF = many_keys<DP>(), BUF = many_buf<DP>();
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int n = lane & 31, half = lane >> 5;
    // A workgroup per part of a row block; every sequence's last row block first.
    const int task = blockIdx.x / a.c.Hkv, h = blockIdx.x - task * a.c.Hkv;
    const int entry = task / a.shape.ranges, part = task - entry * a.shape.ranges;
    const Block block = a.order ? a.order[entry] : block_of(a, entry, ROWS);
    const int units = units_of(a, block, kTile);
    int each = (units + a.shape.ranges - 1) / a.shape.ranges;              // tiles of a part
    each = each < kManyLeast ? kManyLeast : each;
    const int parts = (units + each - 1) / each;
    if (a.shape.slots > 0 && h == 0 && part == 0 && threadIdx.x == 0)
        a.cuts[entry] = int4{parts > 1 ? entry : -1, parts, entry * a.shape.ranges, 1};
    if (h + 1 == a.c.Hkv && entry + 1 == a.b.n * a.shape.blocks && part + 1 == a.shape.ranges) report_faults<THREADS>(a);
    if (part >= parts) return;
    const bool whole = parts == 1;
    const int i = block.i, T = block.T, len = block.len, r0 = block.r0;
    const int lo = part * each * kTile;
    const int hi = block.end - lo < each * kTile ? block.end : lo + each * kTile;
    auto block_end = [&](int first, int rows) {              // keys that these rows see
        if (first >= T * a.g) return 0;
        if (!a.causal) return len;
        const int t = (first + rows - 1) / a.g;
        return len - T + (t < T - 1 ? t : T - 1) + 1;
    };
    const int mine = uniform(block_end(r0 + wave * 32, 32));
    const int wave_hi = mine < hi ? mine : hi;
    const int* table = a.pg.table + (size_t)block.slot * a.pg.max_pages;
    const int row = r0 + wave * 32 + n, t = row / a.g, hh = h * a.g + row - t * a.g;
    const bool live = t < T;
    const int last = live ? (a.causal ? len - T + t : len - 1) : -1;

    const long long orow = (long long)row_begin(a.b, i) + t;       // of the packed rows
    bf16x8 q[NK];
    f32x16 acc[ND] = {};
    float m = -INFINITY, l = 0.f;            // m: the maximum in use, in base 2
    int ref = kMinExp, unit = kMinExp;       // of the values summed (the same in every wave), and
                                             // at last the exponent that the sums are in units of

    const int groups = hi > 0 ? (hi + 15) >> 4 : 0;
    // 64 groups of 16 tokens, one per lane, and the next 64: where a group's codes lie, its
    // scales, and the largest and the least value exponent of the groups of its tile, packed.
    struct Win { int page; unsigned lo, hi; float ks; int ve, top; } win, nxt;
    auto win_page = [&](int base) {
        const int x = base + lane;
        return x < groups ? table[x >> (a.pg.shift - 4)] : 0;
    };
    auto win_scales = [&](int base, Win& v) {
        v.ks = 1.f;
        v.ve = kMinExp;                      // no group: no claim on the reference
        int least = kMaxExp;
        const size_t at = (size_t)v.page * a.c.Hkv + h;
        size_t off = at * a.c.block;         // past the part's end: page 0, whose codes are masked
        if (base + lane < groups) {
            v.ks = a.c.ks[at];
            v.ve = least = exp_of(a.c.vs[at]);
            off += (size_t)(((base + lane) << 4) & ((1 << a.pg.shift) - 1)) * DP;
        }
        v.lo = (unsigned)off;
        v.hi = (unsigned)(off >> 32);
        int o = __builtin_amdgcn_mov_dpp(v.ve, 0xB1, 15, 15, true);      // lane ^ 1
        int top = v.ve > o ? v.ve : o;
        o = __builtin_amdgcn_mov_dpp(top, 0x4E, 15, 15, true);           // lane ^ 2
        top = top > o ? top : o;
        o = __builtin_amdgcn_mov_dpp(least, 0xB1, 15, 15, true);
        least = least < o ? least : o;
        o = __builtin_amdgcn_mov_dpp(least, 0x4E, 15, 15, true);
        least = least < o ? least : o;
        v.top = top * 512 + (least - kMinExp);
    };
    // A tile on its way from memory to LDS: codes, and what converts them.  Unit x of a
    // group of 16 tokens: 16 codes of a key row; two elements of 8 tokens' values.
    struct Raw {
        u32x4 k[UK];
        u32x2 v[UV][2];
        float sk[UK];
        int sv[UV], top;
    } raw[SETS];
    const int x0 = threadIdx.x % DP, hf = x0 / (DP / 2);
    const unsigned koff = x0 * 16, voff = (hf * DP + (x0 - hf * (DP / 2)) * 2) * 4;
    auto group_of = [&](int u) { return (u * THREADS + wave * 64) / DP; };
    auto load_tile = [&](int tile, const Win& v, Raw& r) {
        const int g0 = (tile * (kTile / 16)) & 63;
        r.top = __builtin_amdgcn_readlane(v.top, g0);
#pragma unroll
        for (int u = 0; u < UK; ++u) {
            const int g = g0 + group_of(u);
            r.sk[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v.ks), g));
            r.sv[u] = __builtin_amdgcn_readlane(v.ve, g);
            const size_t off = (unsigned)__builtin_amdgcn_readlane((int)v.lo, g) |
                               (size_t)(unsigned)__builtin_amdgcn_readlane((int)v.hi, g) << 32;
            const unsigned char* kp = a.c.k + off;
            const unsigned char* vp = a.c.v + off;
            r.k[u] = *reinterpret_cast<const u32x4*>(kp + koff);
            r.v[u][0] = *reinterpret_cast<const u32x2*>(vp + voff);
            r.v[u][1] = *reinterpret_cast<const u32x2*>(vp + voff + 2 * DP * 4);
        }
    };
    // Where this thread's units go, relative to the buffer.
    unsigned kto[UK], vto[UV];
#pragma unroll
    for (int u = 0; u < UK; ++u) {
        const int unit = u * THREADS + threadIdx.x;
        const int mrow = unit / (DP / 16), c = (unit - mrow * (DP / 16)) * 2;
        kto[u] = mrow * KP + c * 16;
        vto[u] = HALF + unit * 32;
    }
    auto mask_tile = [&](int pos, Raw& r) {
        // Codes behind the part's last key may be anything, NaN among it (behind the sequence's
        // end, and page 0's in place of groups that no row sees): 0 * NaN is not 0.
        if (pos + kTile > hi) {
#pragma unroll
            for (int u = 0; u < UV; ++u)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int left = hi - (pos + group_of(u) * 16 + (hf + 2 * k) * 4);
                    const unsigned keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
                    r.v[u][k][0] &= keep;
                    r.v[u][k][1] &= keep;
                }
        }
    };
    // Part x of four, of unit u.
    auto store_part = [&](const Raw& r, int buf, int to, int u, int x) {
        unsigned char* d = lds + buf * BUF;
        if (x < 2) {
            *reinterpret_cast<bf16x8*>(d + kto[u] + x * 16) = codes_bf16(r.k[u][x * 2], r.k[u][x * 2 + 1], r.sk[u]);
        } else {
            const float sc = exp_scale(r.sv[u] - to < -126 ? -126 : r.sv[u] - to);     // (-126: no group)
            *reinterpret_cast<f16x8*>(d + vto[u] + (x - 2) * 16) =
                codes_f16(r.v[u][0][x - 2], sc, r.v[u][1][x - 2], sc);
        }
    };
    auto store_tile = [&](const Raw& r, int buf, int to) {
#pragma unroll
        for (int u = 0; u < UK; ++u)
#pragma unroll
            for (int x = 0; x < 4; ++x) store_part(r, buf, to, u, x);
    };
    f32x16 s[2];
    f16x8 p[4];
    // The output of the tile in buffer `out` (values times p) and the scores of the one in
    // `in`, one product after the other; more(i) is other work for after product i.
    constexpr int OUT = 4 * ND, PRODUCTS = OUT + 2 * NK;
    auto matrix = [&](auto first, int out, int in, auto&& more) {
        constexpr int FIRST = decltype(first)::value;
        const unsigned char* kd = lds + in * BUF + n * KP + half * 16;
        const unsigned char* vd = lds + out * BUF + HALF + (half * DP + n) * 16;
        u32x4 f[kReads];
        auto operand = [&](int i) {
            if (i < OUT) return *reinterpret_cast<const u32x4*>(vd + (i / ND) * 2 * DP * 16 + (i % ND) * 512);
            const int c = (i - OUT) / 2, u = (i - OUT) % 2;
            return *reinterpret_cast<const u32x4*>(kd + u * 32 * KP + c * 32);
        };
#pragma unroll
        for (int i = FIRST; i < FIRST + kReads; ++i) f[i % kReads] = operand(i);
#pragma unroll
        for (int i = FIRST; i < PRODUCTS; ++i) {
            if (i < OUT) {
                acc[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, f[i % kReads]),
                                                                     p[i / ND], acc[i % ND], 0, 0, 0);
            } else {
                const int c = (i - OUT) / 2, u = (i - OUT) % 2;
                f32x16 z = {};
                if (c) z = s[u];
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[i % kReads]), q[c], z,
                                                               0, 0, 0);
            }
            if (i + kReads < PRODUCTS) f[i % kReads] = operand(i + kReads);
            more(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto softmax = [&](int pos, int refs) {
        // The first of the wave's rows sees up to 31 keys fewer than the last.
        if (pos + kTile > wave_hi || (a.causal && pos + kTile > mine - 32)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = pos + u * 32 + (e >> 2) * 8 + half * 4 + (e & 3);
                    s[u][e] = key <= last && key < hi ? s[u][e] : -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, s[0][e]);
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[1][e]);
        top = max_over_halves(top) * a.scale2;
        if (__any(top > m + kManySlack) || refs != ref) {
            const float now = fmaxf(m, top);
            const float fade = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
            const float fo = fade * exp_scale(ref - refs < -126 ? -126 : ref - refs);
            l *= fade;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[d][e] *= fo;
            m = now;
            ref = refs;
        }
        const float base = m == -INFINITY ? 0.f : m - kManyLift;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};     // of the unrounded ones: the normaliser is float32
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float y0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], a.scale2, -base));
                const float y1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e + 1], a.scale2, -base));
                sum[u * 2] += y0;
                sum[u * 2 + 1] += y1;
                const f16x2 y = round_f16(y0, y1);
                p[u * 2 + (e >> 3)][e & 7] = y[0];
                p[u * 2 + (e >> 3)][(e & 7) + 1] = y[1];
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    // The softmax behind scales past the spread, e the four groups' exponents.
    auto own_softmax = [&](int pos, const int* e, float& most) {
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float x = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int u = g >> 1, at = (g & 1) * 8 + i;
                const int key = pos + g * 16 + (i >> 2) * 8 + half * 4 + (i & 3);
                s[u][at] = key <= last && key < hi ? s[u][at] : -INFINITY;
                x = fmaxf(x, s[u][at]);
            }
            x = max_over_halves(x) * a.scale2;
            top = fmaxf(top, x);
            most = fmaxf(most, x + (float)e[g]);
        }
        const float now = fmaxf(m, top), from = now == -INFINITY ? 0.f : now;
        const int to = unit_of(most, from);
        const float fo = __builtin_amdgcn_exp2f(m - from + (float)(unit - to));      // 0 while m is -inf
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] *= fo;
        l *= __builtin_amdgcn_exp2f(m - from);
        m = now;
        unit = to;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = s[g >> 1][(g & 1) * 8 + i];
                sum[(g >> 1) * 2 + (i & 1)] += __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.scale2, kManyLift - from));
                p[g][i] = (_Float16)__builtin_amdgcn_exp2f(
                    __builtin_fmaf(x, a.scale2, kManyLift - from - (float)(to - e[g])));
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    if (hi > lo) {
        const int tiles = (hi - lo + kTile - 1) / kTile;
        int base = lo >> 4;                      // windows count from the part's first group
        win.page = win_page(base);
        nxt.page = win_page(base + 64);
        win_scales(base, win);
        // Tiles past the last one are fetched (page 0's codes) and stored like the others, so
        // that a matrix phase has no branches; nothing reads them.
        auto window = [&](int tile) {
            const int in = (tile * (kTile / 16)) & 63;
            if (in == 0) {
                win = nxt;
                base += 64;
                nxt.page = win_page(base + 64);
            }
            if (in == 32) win_scales(base + 64, nxt);
        };
        auto fetch = [&](int tile, Raw& r) { load_tile(tile, win, r); };
        // The references of the tiles from the present one on: the largest value scale up to there
        // (`to`: of the tile being stored).  `stop`: the first tile whose scales pass the spread.
        int refs[3], to = kMinExp, least = kMaxExp, stop = tiles;
        auto refer = [&](int x, int packed) {
            const int top = packed >> 9, low = (packed & 511) + kMinExp;
            to = top > to ? top : to;
            least = low < least ? low : least;
            stop = to - least > kManySpread && x < stop ? x : stop;
        };
        Raw start[AHEAD];
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) fetch(x, start[x]);
#pragma unroll
        for (int x = 0; x < SETS; ++x) fetch(AHEAD + x, raw[x]);
        // Queries: whole rows from memory, after the tiles (loads return in order), turned
        // into operands through the buffers that no tile is stored to yet.
        constexpr int RPI = 64 / CH;                               // rows per instruction
        static_assert(WAVES * 32 * DP * 2 <= (BUFS - AHEAD) * BUF, "queries in the free buffers");
        // Rows behind the last one read the sequence's first row; nothing of theirs is written.
        const long long from = live ? orow * a.q_stride + (long long)hh * a.c.d
                                    : (long long)row_begin(a.b, i) * a.q_stride + (long long)h * a.g * a.c.d;
        const int chunk = lane & (CH - 1);
        const bool inside = chunk * 8 < a.c.d;
        u32x4 qx[32 / RPI];
#pragma unroll
        for (int x = 0; x < 32 / RPI; ++x) {
            const long long src = __shfl(from, x * RPI + lane / CH);
            qx[x] = *reinterpret_cast<const u32x4*>(a.q + src + (inside ? chunk * 8 : 0));
        }
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
            mask_tile(lo + x * kTile, start[x]);
            refer(x, start[x].top);
            store_tile(start[x], x % BUFS, to);
            refs[x] = to;
        }
        // (16-byte chunk c of row r in slot c ^ (r % 16).)
        constexpr int SW = CH < 16 ? CH - 1 : 15;
        unsigned char* qd = lds + AHEAD * BUF + wave * 32 * DP * 2;
#pragma unroll
        for (int x = 0; x < 32 / RPI; ++x) {
            const int r = x * RPI + lane / CH;
            if (!inside) qx[x] = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4*>(qd + r * DP * 2 + (chunk ^ (r & SW)) * 16) = qx[x];
        }
#pragma unroll
        for (int c = 0; c < NK; ++c)
            q[c] = *reinterpret_cast<const bf16x8*>(qd + n * DP * 2 + ((c * 2 + half) ^ (n & SW)) * 16);
        lds_barrier();
        const auto nothing = [](int) {};
        const std::integral_constant<int, 0> all;
        const std::integral_constant<int, OUT> scores;
        if constexpr (AHEAD == 1) {
            matrix(scores, 0, 0, nothing);
            lds_barrier();
            for (int tile = 0; tile < stop; ++tile) {
                const int pos = lo + tile * kTile;
                if (pos < wave_hi) softmax(pos, refs[0]);
                mask_tile(pos + kTile, raw[0]);
                refer(tile + 1, raw[0].top);
                store_tile(raw[0], (tile + 1) % BUFS, to);
                window(tile + 1 + SETS);
                fetch(tile + 1 + SETS, raw[0]);
                lds_barrier();
                // (After the last tile the scores are of a stale one and unused.)
                if (pos < wave_hi) matrix(all, tile % BUFS, (tile + 1) % BUFS, nothing);
                refs[0] = to;
                lds_barrier();
            }
        } else {
            const int behind = wave >= 4;
            // What a matrix phase does beside its products: tile x from `r` to LDS, and what
            // comes after it into `r`.
            auto coming = [&](int x, Raw& r) {
                mask_tile(lo + x * kTile, r);
                window(x + SETS);
                refer(x, r.top);
            };
            auto beside = [&](int i, int x, Raw& r) {
                if (i % 2 == 0 && i < 8) store_part(r, x % BUFS, to, 0, i / 2);
                if (i == 9) fetch(x + SETS, r);
            };
            if (behind) {
                coming(2, raw[0]);
                matrix(scores, 0, 0, [&](int i) { beside(i - OUT, 2, raw[0]); });
                refs[2] = to;
                const Raw r = raw[0];
                raw[0] = raw[1];
                raw[1] = r;
            } else {
                matrix(scores, 0, 0, nothing);
            }
            // One tile: `r` holds the one that is stored beside its output.
            auto step = [&](int tile, Raw& r) {
                const int pos = lo + tile * kTile, x = tile + 2 + behind;
                if (pos < wave_hi) softmax(pos, refs[0]);
                if (behind) lds_barrier();
                __builtin_amdgcn_s_setprio(1);
                coming(x, r);
                if (pos < wave_hi) {
                    matrix(all, tile % BUFS, (tile + 1) % BUFS, [&](int i) { beside(i, x, r); });
                } else {
                    store_tile(r, x % BUFS, to);
                    fetch(x + SETS, r);
                }
                __builtin_amdgcn_s_setprio(0);
                refs[0] = refs[1];
                refs[1] = behind ? refs[2] : to;
                refs[2] = to;
                if (!behind) lds_barrier();
            };
            // (`stop` is known a tile ahead at least, and the same in every wave.)
            for (int tile = 0; tile < stop; tile += SETS) {
                step(tile, raw[0]);
                if (tile + 1 < stop) step(tile + 1, raw[SETS - 1]);
            }
            lds_barrier();                       // the last tile has been read by everyone
        }
        unit = ref;
        if (stop < tiles) {
            // Scales past the spread: a tile at a time, bare codes and rows' own units.
            float most = m + (float)ref;             // the rows' largest weights' exponents
            for (int tile = stop; tile < tiles; ++tile) {
                const int pos = lo + tile * kTile, base = pos >> 4;
                Win v;
                v.page = win_page(base);
                win_scales(base, v);
                Raw& r = raw[0];
                load_tile(0, v, r);
                mask_tile(pos, r);
#pragma unroll
                for (int u = 0; u < UK; ++u) r.sv[u] = 0;
                store_tile(r, 0, 0);
                lds_barrier();
                if (pos < wave_hi) {
                    int e[4];
#pragma unroll
                    for (int g = 0; g < 4; ++g) e[g] = __builtin_amdgcn_readlane(v.ve, g);
                    matrix(scores, 0, 0, nothing);
                    own_softmax(pos, e, most);
                    const unsigned char* vd = lds + HALF + (half * DP + n) * 16;
#pragma unroll
                    for (int i = 0; i < OUT; ++i)
                        acc[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                            *reinterpret_cast<const f16x8*>(vd + (i / ND) * 2 * DP * 16 + (i % ND) * 512), p[i / ND],
                            acc[i % ND], 0, 0, 0);
                }
                lds_barrier();
            }
        }
    }
    l += __shfl_xor(l, 32);
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const float lse2 = l > 0.f ? m + __builtin_amdgcn_logf(l) - kManyLift : -INFINITY;
    const float f = exp_scale(unit);
    const size_t at = ((size_t)h * a.shape.slots + task) * ROWS + wave * 32 + n;
    if (whole) {
        // Through LDS, a part of the buffers for each wave (no wave reads a tile any more): a
        // lane's four elements of a row would leave as pieces of 16 bytes.
        constexpr int PITCH = DP * 2 + 16, RPI = 64 / CH;          // rows per instruction
        static_assert(WAVES * 32 * PITCH <= many_lds<DP, WAVES>(), "output tile");
        unsigned char* o = lds + wave * 32 * PITCH;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                union { bf16x2 p[2]; u32x2 v; } y;
                y.p[0] = bf16x2{(__bf16)(acc[d][e4 * 4] * inv * f), (__bf16)(acc[d][e4 * 4 + 1] * inv * f)};
                y.p[1] = bf16x2{(__bf16)(acc[d][e4 * 4 + 2] * inv * f), (__bf16)(acc[d][e4 * 4 + 3] * inv * f)};
                *reinterpret_cast<u32x2*>(o + n * PITCH + (d * 32 + 8 * e4 + 4 * half) * 2) = y.v;
            }
        const long long to = live ? orow * a.out_stride + (long long)hh * a.c.d : -1;
        const int chunk = lane & (CH - 1);
#pragma unroll
        for (int x = 0; x < 32 / RPI; ++x) {
            const int r = x * RPI + lane / CH;
            const long long dst = __shfl(to, r);
            const u32x4 y = *reinterpret_cast<const u32x4*>(o + r * PITCH + chunk * 16);
            if (dst >= 0 && chunk * 8 < a.c.d) *reinterpret_cast<u32x4*>(a.out + dst + chunk * 8) = y;
        }
    } else {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const int e0 = d * 32 + 8 * e4 + 4 * half;
                if (!live || e0 >= a.c.d) continue;
                f32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = acc[d][e4 * 4 + e] * inv * f;
                *reinterpret_cast<f32x4*>(a.part_o + at * DP + e0) = y;
            }
    }
    if (live && half == 0) {
        if (whole) { if (a.lse) a.lse[orow * a.H + hh] = lse2 * kLn2; }
        else a.part_l[at] = lse2;
    }
}

// Joins the parts of the row blocks that were cut: weights 2^(lse - max), each part's output
// already divided by its own sum.  (They are multiplied in halves, and held times 2^-12: a part of
// little weight can hold values 2^220 times the others', and a sum of values could pass
// float32's range.)  blockIdx.y: a place in the list of cut blocks; z: key
// head; x: groups of 1024 / DP rows of the block, four elements a thread.  5 us, the latency
// of a launch and three loads.
constexpr float kJoinDrop = 12.f;
template <int DP>
__global__ __launch_bounds__(256) void attend_join(AttendArgs a) {
    constexpr int TE = DP / 4, NR = 256 / TE;
    const int h = blockIdx.z;
    const int4 cut = a.cuts[blockIdx.y];
    if (cut.x < 0) return;
    const int block_rows = a.shape.block_rows;
    const Block b = block_of(a, cut.x, block_rows);
    const int te = threadIdx.x % TE, rr = blockIdx.x * NR + threadIdx.x / TE;
    const int i = b.i, row = b.r0 + rr, t = row / a.g, hh = h * a.g + row - t * a.g;
    if (t >= b.T || te * 4 >= a.c.d) return;
    const int parts = cut.y;
    auto at = [&](int p) {
        const int slot = cut.z + (p ? p * cut.w - (cut.w - 1) : 0);
        return ((size_t)h * a.shape.slots + slot) * block_rows + rr;
    };
    float top = -INFINITY, sum = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8;                       // parts read side by side
#pragma unroll 1
    for (int p0 = 0; p0 < parts; p0 += U) {
        float l[U], most = top;
        f32x4 o[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            l[u] = -INFINITY;
            o[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (p0 + u >= parts) continue;
            l[u] = a.part_l[at(p0 + u)];
            o[u] = *reinterpret_cast<const f32x4*>(a.part_o + at(p0 + u) * DP + te * 4);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) most = fmaxf(most, l[u]);
        if (most == -INFINITY) continue;
        const float fade = __builtin_amdgcn_exp2f(0.5f * (top - most));
        sum *= fade * fade;
        y = y * fade * fade;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float root = __builtin_amdgcn_exp2f(0.5f * (l[u] - most) - kJoinDrop / 2);
            sum += root * root;
            y += o[u] * root * root;
        }
        top = most;
    }
    const long long orow = (long long)row_begin(a.b, i) + t;
    y *= sum > 0.f ? 1.f / sum : 0.f;
    ushort4 o;
    o.x = __builtin_bit_cast(unsigned short, (__bf16)y[0]);
    o.y = __builtin_bit_cast(unsigned short, (__bf16)y[1]);
    o.z = __builtin_bit_cast(unsigned short, (__bf16)y[2]);
    o.w = __builtin_bit_cast(unsigned short, (__bf16)y[3]);
    *reinterpret_cast<ushort4*>(a.out + orow * a.out_stride + (long long)hh * a.c.d + te * 4) = o;
    if (te == 0 && a.lse)
        a.lse[orow * a.H + hh] = sum > 0.f ? (top + __builtin_amdgcn_logf(sum) + kJoinDrop) * kLn2 : -INFINITY;
}

}  // namespace

// Rows of a row block.  More than 32 go to the many-row form (16 x 48 rows over 2048 tokens: 36
// us few, 31 us many; 64 x 48 rows 112 and 68 us; 4 x 33 rows on 32 key heads 68 and 45 us; 16 x
// 32 rows 29 us few, 36 us many), up to 128 with four waves, of which a CU holds two workgroups
// at dp = 128 (64 x 48 rows: 96 us with eight waves, a third of them with rows; a prompt of 4 x
// 3012 tokens: 370 us with four, 341 with eight beside it).
// 17 to 32 are one block of the few-row form where that saves reading codes that no cache holds
// close (64 x 32 rows over 4096 tokens of 8 heads, 537 MB: 97 us against 180 in two blocks; 16 x
// 32 over 2048, 67 MB: 27 and 29; 4 x 32 over 4096, 34 MB: 25 and 23.5), not at dp = 256, whose
// registers hold 16.  `bytes` goes by the caller's bound of the lengths, which the device alone
// knows: without one, in tables of 128k tokens, 4 x 32 rows over 4096 take 30.6 us in place of
// 24.7, 16 x 32 over 2048 33.9 and 26.6.
static int attend_block_rows(const CacheView& c, long long rows, double bytes) {
    if (rows > 2 * kFewRows) return c.dp == 128 && rows > 128 ? 256 : 128;
    return rows > kFewRows && c.dp <= 128 && bytes >= kFewBytes ? 2 * kFewRows : kFewRows;
}

// Ranges per key head of the few-row form: the workgroups that are resident at once, no more
// than there is work at the longest.
static long long few_ranges(const CacheView& c, int block_rows, long long entries, long long max_tokens) {
    const long long want = 256 * few_resident(c.dp, block_rows / kFewRows) / c.Hkv;
    const long long most = entries * ((max_tokens + kFewUnit - 1) / kFewUnit);
    const long long ranges = want > most ? most : want;
    return ranges < 1 ? 1 : ranges;
}

// Workgroups of a CU: what registers and LDS leave room for.
static int many_resident(int dp, int block_rows) { return dp <= 128 && block_rows == 128 ? 2 : 1; }

// The most parts of a row block of the many-row form, of at least kManyLeast tiles each.  A
// launch takes as many rounds as it has workgroups beyond those resident, each as long as a part
// (at the longest), the time of about 4 tiles before and behind it and, where blocks are cut, of
// 8 for the part's output to be written, and of one for every part to be joined.  (32 heads on 8
// of 128: two prompts of 600 tokens, 160 row blocks of 10 tiles, 24 us whole, 38 us in three
// parts; 4 x 128 rows over 4096 tokens 29 us in 8 parts, 32 in 16; 32 x 64 rows over 4096 80 us
// in two, 98 whole; 64 heads, 18 x 30 rows over 12812 tokens 278 us in 5, 299 whole; 32 heads of
// 64, 18 x 30 rows over 8000 tokens 71 us in 3, 131 whole.)
static long long many_parts(long long tasks, long long max_tokens, int resident) {
    const long long tiles = (max_tokens + kTile - 1) / kTile, wgs = 256 * resident;
    long long parts = 1, best = (tasks + wgs - 1) / wgs * (tiles + 4);
    for (int half = 1; half <= 2 * kManyRounds; ++half) {
        long long p = half * wgs / (2 * tasks);                // as many as so many half rounds hold
        p = p < tiles / kManyLeast ? p : tiles / kManyLeast;
        if (p < 2) continue;
        const long long each = (tiles + p - 1) / p;
        p = (tiles + each - 1) / each;
        const long long cost = (tasks * p + wgs - 1) / wgs * (each + 12) + p;
        if (cost < best) {
            best = cost;
            parts = p;
        }
    }
    return parts;
}

AttendShape attend_shape(const CacheView& c, const BatchView& b, int H, long long max_tokens) {
    AttendShape x = {};
    const long long rows = (long long)b.max_rows * (H / c.Hkv);
    const double bytes = 2.0 * b.n * max_tokens * c.Hkv * c.dp;            // of codes, at the longest
    x.block_rows = attend_block_rows(c, rows, bytes);
    x.blocks = (int)((rows + x.block_rows - 1) / x.block_rows);
    const long long entries = (long long)b.n * x.blocks;
    x.few = x.block_rows <= 2 * kFewRows;
    x.ranges = (int)(x.few ? few_ranges(c, x.block_rows, entries, max_tokens)
                           : many_parts(entries * c.Hkv, max_tokens, many_resident(c.dp, x.block_rows)));
    // The few-row form reads the codes past the caches where nothing reads them twice (one row
    // block per sequence and key head) and they may be more than the last-level cache holds.  64
    // x 4096 tokens of 8 heads take 96 us against 106, with two row blocks each 208 against 177
    // us; 4 x 2048 tokens 14.7 against 14.3 us.  (At the caller's bound, again: a step over 144 MB
    // that states 302 takes 63.7 us, and 68.7 where it states less than 256.)
    x.stream = x.few && x.blocks == 1 && bytes > kLastLevelBytes;
    // A call sorts its row blocks, with one more launch, only where rows differ from sequence to
    // sequence and there are blocks for more than a round of the chip, up to a number whose
    // unevenness still shows at the end.
    if (!x.few && b.off && x.ranges == 1 && entries > 1 && entries <= kMaxOrder) x.ordered = (int)entries;
    // Slots for parts per key head, and places in the list of cut blocks: none where nothing can
    // be cut.
    if (x.ranges > 1) {
        x.slots = x.few ? 2 * x.ranges : entries * x.ranges;
        x.cuts = x.few ? x.ranges : entries;
    }
    return x;
}

template <int DP, int WAVES>
static hipError_t many_launch(const AttendArgs& a, dim3 grid, hipStream_t s) {
    constexpr int bytes = many_lds<DP, WAVES>();
    static std::atomic<uint64_t> done{0};
    const hipError_t e = bytes <= 65536
        ? hipSuccess : allow_lds(reinterpret_cast<const void*>(attend_many<DP, WAVES>), bytes, done);
    return e != hipSuccess ? e : launch(attend_many<DP, WAVES>, grid, dim3(64 * WAVES), bytes, s, a);
}

template <int DP>
static hipError_t attend_dp(const AttendArgs& a, hipStream_t s) {
    const AttendShape& x = a.shape;
    const long long tasks = x.few ? x.ranges : (long long)a.b.n * x.blocks * x.ranges;
    const dim3 grid((unsigned)(tasks * a.c.Hkv));
    hipError_t e;
    if (x.few) {
        auto kernel = x.stream ? attend_few<DP, 1, true> : attend_few<DP, 1, false>;
        if constexpr (DP <= 128)
            if (x.block_rows > kFewRows) kernel = x.stream ? attend_few<DP, 2, true> : attend_few<DP, 2, false>;
        e = launch(kernel, grid, dim3(64 * kFewWaves), 0, s, a);
    } else {
        if (a.order) {
            e = launch(attend_order, dim3(1), dim3(kMaxOrder), 0, s, a, x.ordered);
            if (e != hipSuccess) return e;
        }
        e = x.block_rows == 128 ? many_launch<DP, 4>(a, grid, s) : many_launch<128, 8>(a, grid, s);
    }
    if (e != hipSuccess || x.slots == 0) return e;
    return launch(attend_join<DP>, dim3(x.block_rows / (1024 / DP), (unsigned)x.cuts, a.c.Hkv), dim3(256), 0, s, a);
}

hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t s) {
    return a.c.dp == 64 ? attend_dp<64>(a, s) : a.c.dp == 128 ? attend_dp<128>(a, s) : attend_dp<256>(a, s);
}

}  // namespace occam
