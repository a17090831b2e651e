// Page operations of the cache: room for new tokens, forks, giving sequences up, and the
// page side of compaction.  Everything runs on the device, so that a batch whose survivor
// counts only the device knows needs no host synchronisation.
//
// Free pages are the clear bits of a map, taken lowest number first by ranking: a prefix
// sum over the words' clear bits gives every free page its rank, and page rank r goes to
// the sequence whose range of the prefix sum of the needs contains r.  Nothing depends on
// the order in which threads run.  Freeing subtracts a reference; whoever takes the last
// one clears the bit.  One workgroup plans a whole call (all or nothing needs one place that
// knows the total); the per-sequence page lists are walked by a workgroup each.  What
// bounds these kernels is latency: a handful of dependent loads and barriers.
#include "cache_internal.hpp"

namespace occam {
namespace {

constexpr int kPlanThreads = 1024;

// Exclusive prefix of x over the workgroup (NT threads), and the total.
template <int NT>
__device__ __forceinline__ int block_scan(int x, int* total, int* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(s, o);
        if (lane >= o) s += y;
    }
    __syncthreads();                       // red may still be read from the scan before
    if (lane == 63) red[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const int y = red[w];
        before += w < wave ? y : 0;
        all += y;
    }
    *total = all;
    return before + s - x;
}

struct PlanShared {
    int need[OCCAM_MAX_BATCH + 1];         // prefix of the pages wanted
    unsigned seen[OCCAM_MAX_SLOTS / 32];   // slots of the call
    int red[kPlanThreads / 64];
    int bad;
};
static_assert(sizeof(PlanShared) <= 65536, "plan state exceeds the default LDS limit");

// Prefix of the values that get(i) gives for i in [0, n) into out[0 .. n] (LDS or global).
template <typename F>
__device__ __forceinline__ int prefix_of(int n, int* out, int* red, F get) {
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        int total;
        const int at = block_scan<kPlanThreads>(i < n ? get(i) : 0, &total, red);
        if (i < n) out[i] = base + at;
        base += total;
    }
    if (threadIdx.x == 0) out[n] = base;
    return base;
}

// Whether `need` pages are free (every thread gets the answer).
__device__ __forceinline__ bool enough_free(const PageView& p, int need, int* red) {
    const int words = (p.num_pages + 31) / 32;
    int have = 0;
    for (int w0 = 0; w0 < words && have < need; w0 += kPlanThreads) {
        const int w = w0 + threadIdx.x;
        unsigned f = w < words ? ~p.taken[w] : 0;
        if (w == words - 1 && (p.num_pages & 31)) f &= (1u << (p.num_pages & 31)) - 1;
        int total;
        block_scan<kPlanThreads>(__popc(f), &total, red);
        have += total;
    }
    return have >= need;
}

// Takes the lowest `need` free pages; give(r, page) places the one of rank r.
template <typename F>
__device__ __forceinline__ void take_free(const PageView& p, int need, int* red, F give) {
    const int words = (p.num_pages + 31) / 32;
    int base = 0;
    for (int w0 = 0; w0 < words && base < need; w0 += kPlanThreads) {
        const int w = w0 + threadIdx.x;
        const unsigned was = w < words ? p.taken[w] : ~0u;
        unsigned f = ~was;
        if (w == words - 1 && (p.num_pages & 31)) f &= (1u << (p.num_pages & 31)) - 1;
        int total, r = base + block_scan<kPlanThreads>(__popc(f), &total, red);
        unsigned now = was;
        while (f && r < need) {
            const int bit = __ffs(f) - 1;
            f &= f - 1;
            now |= 1u << bit;
            const int page = w * 32 + bit;
            p.refs[page] = 1;
            give(r++, page);
        }
        if (now != was) p.taken[w] = now;
        base += total;
    }
}

__device__ __forceinline__ void drop_ref(const PageView& p, int page) {
    if (atomicSub(&p.refs[page], 1) == 1) atomicAnd(&p.taken[page >> 5], ~(1u << (page & 31)));
}

// Marks slot s of the call; true if it is out of range or was marked before.
__device__ __forceinline__ bool bad_slot(const PageView& p, unsigned* seen, int s) {
    if (s < 0 || s >= p.num_seqs) return true;
    return (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31)) & 1;
}
__device__ __forceinline__ void begin_call(const PageView& p, PlanShared* sh) {
    for (int w = threadIdx.x; w < (p.num_seqs + 31) / 32; w += kPlanThreads) sh->seen[w] = 0;
    if (threadIdx.x == 0) sh->bad = 0;
    __syncthreads();
}
__device__ __forceinline__ void write_header(int* plan, int kind, int n, int items) {
    plan[0] = kind; plan[1] = n; plan[2] = items; plan[3] = 0;
}

__global__ __launch_bounds__(256) void pages_reset(PageView p) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < p.num_pages) p.refs[i] = 0;
    if (i < (p.num_pages + 31) / 32) p.taken[i] = 0;
    if (i < p.num_seqs) p.length[i] = 0;
    if (i == 0) *p.status = 0;
}

__global__ __launch_bounds__(kPlanThreads) void pages_reserve(PageView p, BatchView b, int* plan) {
    __shared__ PlanShared sh;
    const int n = b.n, G = 1 << p.shift;
    int* items = plan_array(plan, n, PL_ITEMS);
    int* first = plan_array(plan, n, PL_FIRST);
    int* tail = plan_array(plan, n, PL_TAIL);
    int* rows = plan_array(plan, n, PL_ROWS);
    begin_call(p, &sh);
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int s = slot_of(b, i), r = row_count(b, i);
        int bad = 0, len = 0, src = -1;
        if (bad_slot(p, sh.seen, s)) {
            bad = OCCAM_PAGES_BAD_SEQ;
        } else {
            len = p.length[s];
            if ((long long)len + r > ((long long)p.max_pages << p.shift)) bad = OCCAM_PAGES_TOO_LONG;
            else if (r > 0 && (len & (G - 1))) src = p.table[(size_t)s * p.max_pages + (len >> p.shift)];
        }
        first[i] = len;
        tail[i] = src;
        rows[i] = bad ? 0 : r;
        if (bad) atomicOr(&sh.bad, bad);
    }
    __syncthreads();
    // The pages wanted: those behind the present last one, and one in the place of a shared
    // partly filled one.
    const int need = prefix_of(n, sh.need, sh.red, [&](int i) {
        const int len = first[i], r = rows[i];
        const int more = ((len + r + G - 1) >> p.shift) - ((len + G - 1) >> p.shift);
        return more + (tail[i] >= 0 && p.refs[tail[i]] > 1);
    });
    __syncthreads();
    if (!sh.bad && !enough_free(p, need, sh.red)) {
        if (threadIdx.x == 0) sh.bad = OCCAM_PAGES_FULL;
        __syncthreads();
    }
    if (sh.bad) {
        for (int i = threadIdx.x; i <= n; i += kPlanThreads) {
            items[i] = 0;
            if (i < n) rows[i] = 0;
        }
        if (threadIdx.x == 0) {
            atomicOr(p.status, sh.bad);
            write_header(plan, kPlanReserve, n, 0);
        }
        return;
    }
    // A shared last page is replaced by the first page its sequence gets: table entry
    // len / G; otherwise the first one goes behind, at ceil(len / G).
    take_free(p, need, sh.red, [&](int r, int page) {
        const int i = owner_of(sh.need, n, r), len = first[i];
        const int wanted = sh.need[i + 1] - sh.need[i];
        const int pages = (len + rows[i] + G - 1) >> p.shift;
        const int j = pages - wanted + (r - sh.need[i]);
        p.table[(size_t)slot_of(b, i) * p.max_pages + j] = page;
    });
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        if (rows[i] == 0) continue;
        const int s = slot_of(b, i), len = first[i];
        // Freed only now: a page given up here is not one of those just taken.
        if (tail[i] >= 0 && p.table[(size_t)s * p.max_pages + (len >> p.shift)] != tail[i])
            drop_ref(p, tail[i]);
        p.length[s] = len + rows[i];
    }
    const int total = prefix_of(n, items, sh.red, [&](int i) {
        const int len = first[i], r = rows[i];
        return r > 0 ? ((len + r + G - 1) >> p.shift) - (len >> p.shift) : 0;
    });
    if (threadIdx.x == 0) write_header(plan, kPlanReserve, n, total);
}

__global__ __launch_bounds__(kPlanThreads) void fork_plan(PageView p, int n, const int* src,
                                                          const int* dst, int* plan) {
    __shared__ PlanShared sh;
    int* lens = plan_array(plan, n, PL_ITEMS);
    begin_call(p, &sh);
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int s = src[i], t = dst[i];
        int len = 0;
        if (bad_slot(p, sh.seen, t) || s < 0 || s >= p.num_seqs || p.length[t] != 0) sh.bad = 1;
        else len = p.length[s];
        lens[i] = len;
    }
    __syncthreads();
    if (sh.bad) {
        for (int i = threadIdx.x; i < n; i += kPlanThreads) lens[i] = -1;
        if (threadIdx.x == 0) atomicOr(p.status, OCCAM_PAGES_BAD_SEQ);
    }
    if (threadIdx.x == 0) write_header(plan, kPlanFork, n, 0);
}

__global__ __launch_bounds__(256) void fork_copy(PageView p, int n, const int* src, const int* dst,
                                                 const int* plan) {
    const int i = blockIdx.x;
    const int len = plan_array(plan, n, PL_ITEMS)[i];
    if (len <= 0) return;
    const int* from = p.table + (size_t)src[i] * p.max_pages;
    int* to = p.table + (size_t)dst[i] * p.max_pages;
    const int pages = (len + (1 << p.shift) - 1) >> p.shift;
    for (int j = threadIdx.x; j < pages; j += 256) {
        const int page = from[j];
        to[j] = page;
        atomicAdd(&p.refs[page], 1);
    }
    if (threadIdx.x == 0) p.length[dst[i]] = len;
}

__global__ __launch_bounds__(256) void pages_free(PageView p, const int* seq) {
    __shared__ int len;
    const int s = seq[blockIdx.x];
    if (s < 0 || s >= p.num_seqs) {
        if (threadIdx.x == 0) atomicOr(p.status, OCCAM_PAGES_BAD_SEQ);
        return;
    }
    if (threadIdx.x == 0) len = atomicExch(&p.length[s], 0);   // a slot listed again gets 0
    __syncthreads();
    const int pages = (len + (1 << p.shift) - 1) >> p.shift;
    const int* row = p.table + (size_t)s * p.max_pages;
    for (int j = threadIdx.x; j < pages; j += 256) drop_ref(p, row[j]);
}

// Compaction, first part: what every sequence drops and which fresh pages it gets, written
// into the plan's page lists from the first changed page on.
__global__ __launch_bounds__(kPlanThreads) void keep_plan(PageView p, int n, const int* seq,
                                                          const int* start, const int* span,
                                                          const int* idx, const int* off, int* plan) {
    __shared__ PlanShared sh;
    const int G = 1 << p.shift;
    int* items = plan_array(plan, n, PL_ITEMS);
    int* first = plan_array(plan, n, PL_FIRST);
    int* olds = plan_array(plan, n, PL_OLD);
    int* news = plan_array(plan, n, PL_NEW);
    int* starts = plan_array(plan, n, PL_START);
    int* spans = plan_array(plan, n, PL_SPAN);
    int* slots = plan_array(plan, n, PL_SLOT);
    begin_call(p, &sh);
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int s = seq[i], a = start[i], m = span[i], o = off[i], c = off[i + 1] - o;
        int bad = 0, len = 0, now = 0, f = 0;
        if (bad_slot(p, sh.seen, s)) {
            bad = OCCAM_PAGES_BAD_SEQ;
        } else {
            len = now = p.length[s];
            if (a < 0 || m < 0 || (long long)a + m > len || c < 0 || c > m) {
                bad = OCCAM_PAGES_BAD_SPAN;
            } else if (c < m) {
                // The first index that is not its own position: the first token dropped.
                int lo = 0, hi = c;
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (idx[o + mid] == mid) lo = mid + 1; else hi = mid;
                }
                now = len - m + c;
                f = (a + lo) >> p.shift;
            } else {
                f = (len + G - 1) >> p.shift;            // nothing dropped
            }
        }
        olds[i] = len; news[i] = now; first[i] = f; starts[i] = a; spans[i] = m; slots[i] = s;
        if (bad) atomicOr(&sh.bad, bad);
    }
    __syncthreads();
    const int need = prefix_of(n, sh.need, sh.red, [&](int i) {
        const int pages = ((news[i] + G - 1) >> p.shift) - first[i];
        return sh.bad || pages < 0 ? 0 : pages;
    });
    __syncthreads();
    if (!sh.bad && !enough_free(p, need, sh.red)) {
        if (threadIdx.x == 0) sh.bad = OCCAM_PAGES_FULL;
        __syncthreads();
    }
    if (sh.bad) {
        for (int i = threadIdx.x; i <= n; i += kPlanThreads) {
            items[i] = 0;
            if (i < n) { news[i] = olds[i]; first[i] = (olds[i] + G - 1) >> p.shift; }
        }
        if (threadIdx.x == 0) {
            atomicOr(p.status, sh.bad);
            write_header(plan, kPlanKeep, n, 0);
        }
        return;
    }
    take_free(p, need, sh.red, [&](int r, int page) {
        const int i = owner_of(sh.need, n, r);
        plan_pages(plan, n, p.max_pages, i)[first[i] + r - sh.need[i]] = page;
    });
    for (int i = threadIdx.x; i <= n; i += kPlanThreads) items[i] = sh.need[i];
    if (threadIdx.x == 0) write_header(plan, kPlanKeep, n, need);
}

// Second part, a workgroup per sequence: the fresh pages go into the table, the old ones
// into the plan's list (the move reads from them), and the old ones' references end.
__global__ __launch_bounds__(256) void keep_swap(PageView p, int n, const int* seq, int* plan) {
    const int i = blockIdx.x, G = 1 << p.shift;
    const int f = plan_array(plan, n, PL_FIRST)[i];
    const int len = plan_array(plan, n, PL_OLD)[i], now = plan_array(plan, n, PL_NEW)[i];
    const int had = (len + G - 1) >> p.shift, has = (now + G - 1) >> p.shift;
    if (f >= had) return;                     // nothing changes (or the call failed)
    int* list = plan_pages(plan, n, p.max_pages, i);
    int* row = p.table + (size_t)seq[i] * p.max_pages;
    for (int j = f + (int)threadIdx.x; j < had; j += 256) {
        const int old = row[j];
        if (j < has) row[j] = list[j];
        list[j] = old;
        drop_ref(p, old);
    }
    if (threadIdx.x == 0) p.length[seq[i]] = now;
}

}  // namespace

hipError_t launch_pages_reset(const PageView& p, hipStream_t s) {
    int most = p.num_pages > p.num_seqs ? p.num_pages : p.num_seqs;
    return launch(pages_reset, dim3((most + 255) / 256), dim3(256), 0, s, p);
}

hipError_t launch_pages_reserve(const PageView& p, const BatchView& b, int* plan, hipStream_t s) {
    return launch(pages_reserve, dim3(1), dim3(kPlanThreads), 0, s, p, b, plan);
}

hipError_t launch_pages_fork(const PageView& p, int n, const int* src, const int* dst, int* plan,
                             hipStream_t s) {
    hipError_t e = launch(fork_plan, dim3(1), dim3(kPlanThreads), 0, s, p, n, src, dst, plan);
    if (e != hipSuccess) return e;
    return launch(fork_copy, dim3(n), dim3(256), 0, s, p, n, src, dst, plan);
}

hipError_t launch_pages_free(const PageView& p, int n, const int* seq, hipStream_t s) {
    return launch(pages_free, dim3(n), dim3(256), 0, s, p, seq);
}

hipError_t launch_pages_keep(const PageView& p, int n, const int* seq, const int* start,
                             const int* span, const int* idx, const int* off, int* plan,
                             hipStream_t s) {
    hipError_t e = launch(keep_plan, dim3(1), dim3(kPlanThreads), 0, s, p, n, seq, start, span, idx,
                          off, plan);
    if (e != hipSuccess) return e;
    return launch(keep_swap, dim3(n), dim3(256), 0, s, p, n, seq, plan);
}

}  // namespace occam
