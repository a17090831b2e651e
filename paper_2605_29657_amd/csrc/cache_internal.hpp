// Internal definitions of the paged 8-bit cache (include/occam_cache.h): views passed by
// value to the kernels, the plan's layout, and the 8-bit conversions.
#pragma once

#include "occam_cache.h"
#include "occam_internal.hpp"

namespace occam {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct PageView {
    int num_pages, shift, num_seqs, max_pages;   // page_tokens = 1 << shift
    int *table, *length, *refs;
    unsigned* taken;
    int* status;
};

// A layer's storage.  One (page, key head) block is `block` = page_tokens * dp bytes.
struct CacheView {
    int Hkv, d, dp;
    unsigned block;
    unsigned char *k, *v;
    float *ks, *vs;
};

struct BatchView {
    int n, rows, max_rows;
    const int *seq, *off;
};

__device__ __forceinline__ int slot_of(const BatchView& b, int i) { return b.seq ? b.seq[i] : i; }
__device__ __forceinline__ int row_begin(const BatchView& b, int i) {
    return b.off ? b.off[i] : i * b.rows;
}
// Rows that the offsets give sequence i, or -1 where they descend or pass the host's bound;
// such a sequence's rows are left alone.
__device__ __forceinline__ int stated_rows(const BatchView& b, int i) {
    if (!b.off) return b.rows;
    const int r = b.off[i + 1] - b.off[i];
    return r <= b.max_rows ? r < 0 ? -1 : r : -1;
}
__device__ __forceinline__ int row_count(const BatchView& b, int i) {
    const int r = stated_rows(b, i);
    return r < 0 ? 0 : r;
}
// The status bits of a sequence: a slot that there is not, rows that the offsets give wrongly.
__device__ __forceinline__ int batch_faults(const PageView& p, int slot, int stated) {
    return (slot < 0 || slot >= p.num_seqs ? (int)OCCAM_PAGES_BAD_SEQ : 0) |
           (stated < 0 ? (int)OCCAM_PAGES_BAD_ROWS : 0);
}

// The plan: a header of four ints (kind, n, page items, 0), arrays of n + 1 ints, for keep
// a page list of max_pages ints per sequence, and a record of eight ints for every page item
// (a page that receives rows, or that is rewritten): what the kernels that work on items
// need to know, found with one load.
//   keep:    FIRST page rewritten, OLD tokens before, NEW tokens after
//   fork:    LENS tokens of the source, or -1 where the call failed
//   reserve and keep use the other arrays while they plan.
constexpr int kPlanReserve = 1, kPlanKeep = 2, kPlanFork = 3;
constexpr int kPlanHeader = 4, kPlanArrays = 4, kRecord = 8;
enum { PL_FIRST = 0, PL_OLD = 1, PL_NEW = 2, PL_TAIL = 1, PL_ROWS = 2, PL_SLOT = 3, PL_LENS = 0 };
// reserve: the page, the page its tokens so far lie in, how many those are, how many it
// holds now, and the batch's row that would be its token 0 (may be negative).
enum { RR_PAGE = 0, RR_TAIL = 1, RR_HAD = 2, RR_END = 3, RR_ROW = 4 };
// keep: the fresh page, the sequence's first token in it, the tokens it holds, the index in
// the call, the span's start and length, and where its survivors are listed.
enum { RK_PAGE = 0, RK_POS = 1, RK_END = 2, RK_SEQ = 3, RK_START = 4, RK_SPAN = 5, RK_OFF = 6, RK_COUNT = 7 };

// Items there can be: pages of the call's tables, and no more than fresh pages and partly
// filled ones.
__host__ __device__ inline size_t plan_items(int n, int max_pages, int num_pages) {
    const size_t a = (size_t)n * max_pages, b = (size_t)num_pages + n;
    return a < b ? a : b;
}
__host__ __device__ inline size_t plan_ints(int n, int max_pages, int num_pages) {
    return kPlanHeader + (size_t)kPlanArrays * (n + 1) + (size_t)n * max_pages +
           kRecord * plan_items(n, max_pages, num_pages);
}
__device__ __forceinline__ int* plan_array(int* plan, int n, int a) {
    return plan + kPlanHeader + (size_t)a * (n + 1);
}
__device__ __forceinline__ const int* plan_array(const int* plan, int n, int a) {
    return plan + kPlanHeader + (size_t)a * (n + 1);
}
__device__ __forceinline__ int* plan_pages(int* plan, int n, int max_pages, int i) {
    return plan + kPlanHeader + (size_t)kPlanArrays * (n + 1) + (size_t)i * max_pages;
}
__device__ __forceinline__ const int* plan_pages(const int* plan, int n, int max_pages, int i) {
    return plan + kPlanHeader + (size_t)kPlanArrays * (n + 1) + (size_t)i * max_pages;
}
__device__ __forceinline__ int* plan_record(int* plan, int n, int max_pages, int item) {
    return plan_pages(plan, n, max_pages, n) + (size_t)item * kRecord;
}
__device__ __forceinline__ const int* plan_record(const int* plan, int n, int max_pages, int item) {
    return plan_pages(plan, n, max_pages, n) + (size_t)item * kRecord;
}
// The last i in [0, n) with prefix[i] <= x: the sequence that item x belongs to.
__device__ __forceinline__ int owner_of(const int* prefix, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Four e4m3 codes of a dword (byte 0 first) as float32, unscaled.
__device__ __forceinline__ f32x4 dec4(unsigned w) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return f32x4{a[0], a[1], b[0], b[1]};
}
// Four values, already divided by their scale, as codes: nearest, ties to even (measured
// over every code and midpoint).  The clamp keeps a magnitude past the largest number,
// which a scale held at its largest exponent can leave, from becoming NaN.
__device__ __forceinline__ float sat8(float x) { return __builtin_amdgcn_fmed3f(x, -448.f, 448.f); }
__device__ __forceinline__ unsigned enc4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(sat8(a), sat8(b), 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(sat8(c), sat8(d), w, true);
}

// The block scale's exponent for the largest magnitude `amax`: amax = m 2^x with m in
// [1, 2) needs 2^(x - 8) while m <= 1.75 (448 = 1.75 * 2^8), twice that above.
constexpr int kMinExp = -100, kMaxExp = 120;
constexpr float kMostAtMaxExp = 240.f;     // 256 * 2^120 is no float32 any more
__device__ __forceinline__ int scale_exp(float amax) {
    const unsigned u = __float_as_uint(amax) & 0x7fffffffu;
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    e = e < kMinExp ? kMinExp : e;
    return e > kMaxExp ? kMaxExp : e;
}
__device__ __forceinline__ float exp_scale(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
__device__ __forceinline__ int exp_of(float scale) {       // of a power of two
    return (int)((__float_as_uint(scale) >> 23) & 255) - 127;
}

// What a call touches once and is larger than the last-level cache goes past the caches: it
// would push out everything else, itself included.
constexpr long long kLastLevelBytes = 256ll << 20;
template <bool STREAM, typename V>
__device__ __forceinline__ V get(const V* from) {
    if constexpr (STREAM) return __builtin_nontemporal_load(from);
    else return *from;
}
template <bool STREAM, typename V>
__device__ __forceinline__ void put(V x, V* to) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, to);
    else *to = x;
}

struct RotTensor {
    const char* src;
    char* dst;
    int heads, first;            // heads before this tensor's
    long long src_stride, dst_stride;   // bytes
};
template <int TENSORS, int PAIRS>
struct RotArgsOf {
    static constexpr int kTensors = TENSORS, kPairs = PAIRS;
    int n, heads;                // tensors, heads over all of them
    int rows, d, pairs, axes, adjacent, inverse;
    const int* pos;
    RotTensor t[TENSORS];
    unsigned long long turn[PAIRS];
    unsigned char axis[PAIRS];
};
typedef RotArgsOf<OCCAM_MAX_ROW_TENSORS, OCCAM_MAX_PAIRS> RotArgs;

// One row block of one sequence: its place in the batch, rows, length, slot, first row, and
// the keys that its rows see (0 or less: none).
struct AttendBlock {
    int i, T, len, slot, r0, end;
};
constexpr int kMaxOrder = 1024;          // row blocks that a call sorts by length at most

// The form that an attention takes.
struct AttendShape {
    int few, stream;             // the few-row form; whether it reads the codes past the caches
    int block_rows, blocks;      // rows of a row block; row blocks per sequence and key head
    int ranges;                  // few rows: ranges of work per key head; many: parts of a block
    int ordered;                 // row blocks that are sorted first (0: they run as they come)
    long long slots, cuts;       // slots for parts per key head; places in the list of cut blocks
};

struct AttendArgs {
    PageView pg;
    CacheView c;
    BatchView b;
    AttendShape shape;
    int H, g;                    // query heads, query heads per key head
    int causal;
    float scale2;                // softmax scale * log2(e)
    const unsigned short* q;
    unsigned short* out;
    long long q_stride, out_stride;     // elements
    float* lse;
    float *part_o, *part_l;      // [Hkv][slots][block rows][dp], [Hkv][slots][block rows]
    int4* cuts;                  // [cuts]
    AttendBlock* order;          // row blocks, longest first, or NULL: as block_of numbers them
};

hipError_t launch_rotate(const RotArgs& a, int f32, int vec, hipStream_t s);
hipError_t launch_pages_reset(const PageView& p, hipStream_t s);
hipError_t launch_pages_reserve(const PageView& p, const BatchView& b, int* plan, hipStream_t s);
hipError_t launch_pages_fork(const PageView& p, int n, const int* src, const int* dst, int* plan,
                             hipStream_t s);
hipError_t launch_pages_free(const PageView& p, int n, const int* seq, hipStream_t s);
hipError_t launch_pages_keep(const PageView& p, int n, const int* seq, const int* start,
                             const int* span, const int* idx, const int* off, int* plan,
                             hipStream_t s);
hipError_t launch_cache_append(const PageView& p, const CacheView& c, const BatchView& b,
                               const int* plan, int f32, const void* k, long long ks,
                               const void* v, long long vs, hipStream_t s);
hipError_t launch_cache_read(const PageView& p, const CacheView& c, const BatchView& b,
                             const int* start, int f32, void* k, long long ks, void* v,
                             long long vs, hipStream_t s);
hipError_t launch_cache_move(const PageView& p, const CacheView& c, int n, const int* plan,
                             const int* idx, hipStream_t s);
hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t s);
AttendShape attend_shape(const CacheView& c, const BatchView& b, int H, long long max_tokens);

}  // namespace occam
