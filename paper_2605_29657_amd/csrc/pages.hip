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
// bounds these kernels is latency: a handful of dependent loads and barriers.  The kernels
// themselves: room for one sequence's 131 tokens 5.3 us, for a token of 32 sequences 6.7 us, for
// 32 prompts (1300 pages of 64) 11.7 us; forking 32 sequences 4.6 us, freeing them 4.1 us; what 64
// pruned forks drop 13.5 us, swapping their pages 4.0 us.
#include "cache_internal.hpp"

namespace occam {
namespace {

// Workgroups of the planning kernels: 256 threads for calls of up to 256 sequences and, where
// the host knows a bound, kSmallPages pages (fewer waves at every barrier), 1024 beyond.
// Reserving, one call's time between events, with 256 and 1024 threads: 32 sequences of one page
// 8.8 and 10.7 us, of 8 pages 9.1 and 11.0, 16: 11.1 and 11.2, 31: 15.2 and 11.7, 60: 22.8 and
// 14.0; 128 of 4: 11.6 and 11.4; one of 512: 10.0 and 10.5, of 1000: 12.8 and 10.9.
// What a call reads again of its sequences is kept in LDS for up to kNear of them, in the plan
// beyond; the pages it takes for up to kList of them.
constexpr int kSmallPages = 512, kNear = 1024, kList = 4096;
// Table entries of a fork call that one workgroup of 1024 threads copies by itself: between
// events, in one and in two launches, 32 tables of 64 entries 7.2 and 9.2 us, of 127 9.0 and 9.6,
// of 250 11.7 and 9.3; 8 of 512 8.7 and 9.6, of 1000 11.3 and 10.3; 1000 of 4 9.4 and 9.2.
constexpr int kSmallTables = 4096;

// Exclusive prefix of x over the workgroup (NT threads), and the total.
template <int NT, typename T>
__device__ __forceinline__ T block_scan(T x, T* total, T* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T y = __shfl_up(s, o);
        if (lane >= o) s += y;
    }
    __syncthreads();                       // red may still be read from the scan before
    if (lane == 63) red[wave] = s;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const T y = red[w];
        before += w < wave ? y : 0;
        all += y;
    }
    *total = all;
    return before + s - x;
}

template <int NT>
struct PlanShared {
    static constexpr int kSeqs = NT == 256 ? 256 : OCCAM_MAX_BATCH;
    long long red2[NT / 64];
    int need[kSeqs + 1], items[kSeqs + 1]; // prefixes over the call's sequences
    unsigned seen[OCCAM_MAX_SLOTS / 32];   // slots of the call
    int bad;
    int near[4][kSeqs < kNear ? kSeqs : kNear];
    int list[kList];                       // pages taken, by rank
    int rank[NT];                          // of a stretch of the map: ranks of the words' free
    unsigned free[NT];                     // pages, and their bits
    int red[NT / 64];
};

// Prefixes of the two numbers that get(i) gives for i in [0, n) into out[0 .. n] each;
// returns their sums.  (For what follows from a call's rows, which stay below 2^31.)
struct Two { int a, b; };
template <int NT, typename F>
__device__ __forceinline__ Two prefix_of(int n, int* out_a, int* out_b, long long* red, F get) {
    long long base = 0;
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + threadIdx.x;
        long long total;
        const Two x = i < n ? get(i) : Two{0, 0};
        const long long at = base + block_scan<NT>((long long)x.a << 32 | (unsigned)x.b, &total, red);
        if (i < n) {
            out_a[i] = (int)(at >> 32);
            out_b[i] = (int)at;
        }
        base += total;
    }
    if (threadIdx.x == 0) {
        out_a[n] = (int)(base >> 32);
        out_b[n] = (int)base;
    }
    return Two{(int)(base >> 32), (int)base};
}

// Prefixes of the number that get(i) gives for i in [0, n) into out[0 .. n]; returns their sum,
// which may pass 2^31 (forks share pages: what a call replaces can be many times the pool).
// The prefixes are right where it does not.
template <int NT, typename F>
__device__ __forceinline__ long long wide_prefix_of(int n, int* out, long long* red, F get) {
    long long base = 0;
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + threadIdx.x;
        long long total;
        const long long at = base + block_scan<NT>(i < n ? (long long)get(i) : 0ll, &total, red);
        if (i < n) out[i] = (int)at;
        base += total;
    }
    if (threadIdx.x == 0) out[n] = (int)base;
    return base;
}

// The clear bits of word w of the map that are pages.
__device__ __forceinline__ unsigned free_bits(const PageView& p, int w, unsigned was) {
    unsigned f = ~was;
    if (w == p.num_pages >> 5) f &= (1u << (p.num_pages & 31)) - 1;
    return w < (p.num_pages + 31) / 32 ? f : 0;
}
// This thread's word of the map's first NT words: read ahead of everything else, because
// the pages of an ordinary call come from there.
template <int NT>
__device__ __forceinline__ unsigned first_word(const PageView& p) {
    return (int)threadIdx.x < (p.num_pages + 31) / 32 ? p.taken[threadIdx.x] : ~0u;
}

// The position of the set bit of f with k set bits below it.
__device__ __forceinline__ int nth_bit(unsigned f, int k) {
    int at = 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const int c = __popc(f & ((1u << o) - 1));
        const bool up = k >= c;
        k -= up ? c : 0;
        at += up ? o : 0;
        f = up ? f >> o : f;
    }
    return at;
}

// Takes the lowest `need` free pages, or none if there are not as many (false, in every
// thread), and lists them by rank in list[0 .. need), which the caller may read after a barrier.
template <int NT>
__device__ __forceinline__ bool take_free(const PageView& p, unsigned word0, int need, PlanShared<NT>& sh,
                                          int* list) {
    if (need == 0) return true;
    const int words = (p.num_pages + 31) / 32;
    int total, rank = block_scan<NT, int>(__popc(free_bits(p, threadIdx.x, word0)), &total, sh.red);
    const int total0 = total;
    int have = total0;
    for (int w0 = NT; w0 < words && have < need; w0 += NT) {
        const int w = w0 + threadIdx.x;
        block_scan<NT, int>(__popc(free_bits(p, w, w < words ? p.taken[w] : ~0u)), &total, sh.red);
        have += total;
    }
    if (have < need) return false;
    // A stretch of NT words, whose first free page has rank `base` and whose free pages are
    // `count`: the words' owners mark what is taken, then any thread lists any page (those of
    // a small call all come from one or two words).
    auto take = [&](int w0, unsigned was, int base, int r, int count) {
        const int w = w0 + threadIdx.x;
        const unsigned f = free_bits(p, w, was);
        if (f && base + r < need) {
            const int n = need - base - r;       // free pages of this word that are taken
            const unsigned below = n < __popc(f) ? (1u << nth_bit(f, n)) - 1 : ~0u;
            p.taken[w] = was | (f & below);
        }
        sh.rank[threadIdx.x] = r;
        sh.free[threadIdx.x] = f;
        __syncthreads();
        const int end = need - base < count ? need - base : count;
        for (int x = threadIdx.x; x < end; x += NT) {
            const int o = owner_of(sh.rank, NT, x);
            list[base + x] = (w0 + o) * 32 + nth_bit(sh.free[o], x - sh.rank[o]);
        }
    };
    take(0, word0, 0, rank, total0);
    int base = total0;
    for (int w0 = NT; w0 < words && base < need; w0 += NT) {
        const int w = w0 + threadIdx.x;
        const unsigned was = w < words ? p.taken[w] : ~0u;
        rank = block_scan<NT, int>(__popc(free_bits(p, w, was)), &total, sh.red);   // (its barriers end
        take(w0, was, base, rank, total);                                           // the use of sh.rank)
        base += total;
    }
    return true;
}

// Pages of one word of the map that a wave frees are cleared together (a sequence's pages
// mostly lie side by side: freeing 32 prompts takes 5.2 us against 8.4), those of further
// words one by one.
__device__ __forceinline__ void drop_ref(const PageView& p, int page) {
    const bool last = atomicSub(&p.refs[page], 1) == 1;
    const int lane = threadIdx.x & 63;
    unsigned long long left = __ballot(last);
    for (int k = 0; k < 4 && left; ++k) {
        const int lead = __ffsll(left) - 1, word = __builtin_amdgcn_readlane(page, lead) >> 5;
        const unsigned long long same = __ballot(last && page >> 5 == word);
        unsigned bits = 0;
        for (unsigned long long x = same; x; x &= x - 1)
            bits |= 1u << (__builtin_amdgcn_readlane(page, __ffsll(x) - 1) & 31);
        if (lane == lead) atomicAnd(&p.taken[word], ~bits);
        left &= ~same;
    }
    if (left >> lane & 1) atomicAnd(&p.taken[page >> 5], ~(1u << (page & 31)));
}

// Marks slot s of the call; true if it is out of range or was marked before.
__device__ __forceinline__ bool bad_slot(const PageView& p, unsigned* seen, int s) {
    if (s < 0 || s >= p.num_seqs) return true;
    return (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31)) & 1;
}
template <int NT>
__device__ __forceinline__ void begin_call(const PageView& p, unsigned* seen, int* bad) {
    for (int w = threadIdx.x; w < (p.num_seqs + 31) / 32; w += NT) seen[w] = 0;
    if (threadIdx.x == 0) *bad = 0;
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

template <int NT>
__global__ __launch_bounds__(NT) void pages_reserve(PageView p, BatchView b, int* plan) {
    extern __shared__ __align__(16) unsigned char lds[];
    PlanShared<NT>& sh = *reinterpret_cast<PlanShared<NT>*>(lds);
    const int n = b.n, G = 1 << p.shift;
    const unsigned word0 = first_word<NT>(p);
    int* g_first = plan_array(plan, n, PL_FIRST);
    int* g_tail = plan_array(plan, n, PL_TAIL);
    int* g_rows = plan_array(plan, n, PL_ROWS);
    int* g_slot = plan_array(plan, n, PL_SLOT);
    const bool near = n <= kNear;
    int* first = near ? sh.near[0] : g_first;
    int* tail = near ? sh.near[1] : g_tail;
    int* rows = near ? sh.near[2] : g_rows;
    int* slot = near ? sh.near[3] : g_slot;
    begin_call<NT>(p, sh.seen, &sh.bad);
    for (int i = threadIdx.x; i < n; i += NT) {
        const int s = slot_of(b, i), stated = stated_rows(b, i), r = stated < 0 ? 0 : stated;
        int bad = stated < 0 ? (int)OCCAM_PAGES_BAD_ROWS : 0, len = 0, src = -1;
        if (bad_slot(p, sh.seen, s)) {
            bad |= OCCAM_PAGES_BAD_SEQ;
        } else {
            len = p.length[s];
            if ((long long)len + r > ((long long)p.max_pages << p.shift)) bad |= OCCAM_PAGES_TOO_LONG;
            else if (r > 0 && (len & (G - 1))) src = p.table[(size_t)s * p.max_pages + (len >> p.shift)];
        }
        first[i] = len;
        tail[i] = src;
        rows[i] = bad ? 0 : r;
        slot[i] = s;
        if (bad) atomicOr(&sh.bad, bad);
    }
    __syncthreads();
    // The pages wanted: those behind the present last one, and one in the place of a shared
    // partly filled one; and the pages that receive rows.
    const Two sums = prefix_of<NT>(n, sh.need, sh.items, sh.red2, [&](int i) {
        const int len = first[i], r = rows[i];
        const int end = (len + r + G - 1) >> p.shift;
        return Two{end - ((len + G - 1) >> p.shift) + (tail[i] >= 0 && p.refs[tail[i]] > 1),
                   r > 0 ? end - (len >> p.shift) : 0};
    });
    const int need = sums.a, total = sums.b;
    __syncthreads();
    const bool listed = need <= kList;
    int* list = listed ? sh.list : plan_record(plan, n, p.max_pages, 0);
    if (sh.bad || !take_free<NT>(p, word0, need, sh, list)) {
        if (threadIdx.x == 0) {
            atomicOr(p.status, sh.bad ? sh.bad : (int)OCCAM_PAGES_FULL);
            write_header(plan, kPlanReserve, n, 0);
        }
        return;
    }
    __syncthreads();
    // The first table entry that sequence i gets: a shared last page is replaced by the first
    // page taken (entry len / G); otherwise that one goes behind, at ceil(len / G).
    auto fresh_from = [&](int i) {
        return ((first[i] + rows[i] + G - 1) >> p.shift) - (sh.need[i + 1] - sh.need[i]);
    };
    for (int r = threadIdx.x; r < need; r += NT) {
        const int i = owner_of(sh.need, n, r), page = list[r];
        p.refs[page] = 1;
        p.table[(size_t)slot[i] * p.max_pages + fresh_from(i) + r - sh.need[i]] = page;
    }
    if (!listed) __syncthreads();          // the list lies where the records go
    for (int x = threadIdx.x; x < total; x += NT) {
        const int i = owner_of(sh.items, n, x), len = first[i];
        const int j = (len >> p.shift) + x - sh.items[i], pos0 = j << p.shift, from = fresh_from(i);
        const int page = j < from ? tail[i]
                         : listed ? list[sh.need[i] + j - from]
                                  : p.table[(size_t)slot[i] * p.max_pages + j];
        const int had = len > pos0 ? len - pos0 : 0, now = len + rows[i] - pos0;
        int* r = plan_record(plan, n, p.max_pages, x);
        r[RR_PAGE] = page;
        r[RR_TAIL] = had ? tail[i] : page;
        r[RR_HAD] = had;
        r[RR_END] = now < G ? now : G;
        r[RR_ROW] = row_begin(b, i) - len + pos0;
    }
    // References end after the taking: a page given up here is not one of those just taken.
    for (int i = threadIdx.x; i < n; i += NT) {
        if (rows[i] == 0) continue;
        p.length[slot[i]] = first[i] + rows[i];
        // One page more than lies behind: the shared tail was replaced.
        const int more = ((first[i] + rows[i] + G - 1) >> p.shift) - ((first[i] + G - 1) >> p.shift);
        if (sh.need[i + 1] - sh.need[i] > more) drop_ref(p, tail[i]);
    }
    if (threadIdx.x == 0) write_header(plan, kPlanReserve, n, total);
}

// COPY: the forks' table rows too (where they are short enough for one workgroup: a launch
// less).
template <int NT, bool COPY>
__global__ __launch_bounds__(NT) void fork_plan(PageView p, int n, const int* src, const int* dst,
                                                int* plan) {
    __shared__ unsigned seen[OCCAM_MAX_SLOTS / 32];
    __shared__ int bad, near[COPY ? kSmallTables : 1];
    int* lens = plan_array(plan, n, PL_LENS);
    begin_call<NT>(p, seen, &bad);
    for (int i = threadIdx.x; i < n; i += NT) {
        const int s = src[i], t = dst[i];
        int len = 0;
        if (bad_slot(p, seen, t) || s < 0 || s >= p.num_seqs || p.length[t] != 0) bad = 1;
        else len = p.length[s];
        lens[i] = len;
        if (COPY) near[i] = len;
    }
    __syncthreads();
    if (bad) {
        for (int i = threadIdx.x; i < n; i += NT) lens[i] = -1;
        if (threadIdx.x == 0) atomicOr(p.status, (int)OCCAM_PAGES_BAD_SEQ);
    }
    if (threadIdx.x == 0) write_header(plan, kPlanFork, n, 0);
    if (!COPY || bad) return;
    for (int x = threadIdx.x; x < n * p.max_pages; x += NT) {
        const int i = x / p.max_pages, j = x - i * p.max_pages, len = near[i];
        if (j >= (len + (1 << p.shift) - 1) >> p.shift) continue;
        const int page = p.table[(size_t)src[i] * p.max_pages + j];
        p.table[(size_t)dst[i] * p.max_pages + j] = page;
        atomicAdd(&p.refs[page], 1);
    }
    for (int i = threadIdx.x; i < n; i += NT)
        if (near[i] > 0) p.length[dst[i]] = near[i];
}

__global__ __launch_bounds__(256) void fork_copy(PageView p, int n, const int* src, const int* dst,
                                                 const int* plan) {
    const int i = blockIdx.x;
    const int len = plan_array(plan, n, PL_LENS)[i];
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
    const int* row = p.table + (size_t)s * p.max_pages;
    int page = (int)threadIdx.x < p.max_pages ? row[threadIdx.x] : 0;      // beside the length
    __syncthreads();
    const int pages = (len + (1 << p.shift) - 1) >> p.shift;
    for (int j = threadIdx.x; j < pages; j += 256) {
        if (j >= 256) page = row[j];
        drop_ref(p, page);
    }
}

// The first of m ascending distinct indices that is not its own position (m if none): the
// first token dropped.  Probes side by side: at first 0, 1, 3, 7, ... (a pruned span has its
// first gap early), then seven a round.
struct Gap {
    static constexpr int K = 14;
    int at[K];
    __device__ __forceinline__ void probe(const int* idx, int m) {
#pragma unroll
        for (int k = 0; k < K; ++k) at[k] = (1 << k) - 1 < m ? idx[(1 << k) - 1] - ((1 << k) - 1) : 1;
    }
    __device__ __forceinline__ int find(const int* idx, int m) const {
        int good = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) good += at[k] == 0 && good == k;
        int lo = good ? 1 << (good - 1) : 0, hi = m;     // idx[lo - 1] == lo - 1; idx[hi] != hi or hi == m
        if (good < K && (1 << good) - 1 < hi) hi = (1 << good) - 1;
        while (hi - lo > 0) {
            const int step = (hi - lo + 7) >> 3;
            int d[7];
            good = 0;
#pragma unroll
            for (int k = 0; k < 7; ++k) {
                const int x = lo + (k + 1) * step - 1;
                d[k] = x < hi ? idx[x] - x : 1;
            }
#pragma unroll
            for (int k = 0; k < 7; ++k) good += d[k] == 0 && good == k;
            const int from = lo + good * step;
            const int to = good < 7 ? lo + (good + 1) * step - 1 : hi;
            lo = from;
            hi = to < hi ? to : hi;
        }
        return lo;
    }
};

// Compaction, first part: what every sequence drops and which fresh pages it gets, written
// into the plan's page lists from the first changed page on.
template <int NT>
__global__ __launch_bounds__(NT) void keep_plan(PageView p, int n, const int* seq, const int* start,
                                                const int* span, const int* idx, const int* off,
                                                int* plan) {
    extern __shared__ __align__(16) unsigned char lds[];
    PlanShared<NT>& sh = *reinterpret_cast<PlanShared<NT>*>(lds);
    const int G = 1 << p.shift;
    const unsigned word0 = first_word<NT>(p);
    int* g_first = plan_array(plan, n, PL_FIRST);
    int* g_olds = plan_array(plan, n, PL_OLD);
    int* g_news = plan_array(plan, n, PL_NEW);
    const bool near = n <= kNear;
    int* first = near ? sh.near[0] : g_first;
    int* olds = near ? sh.near[1] : g_olds;
    int* news = near ? sh.near[2] : g_news;
    begin_call<NT>(p, sh.seen, &sh.bad);
    for (int i = threadIdx.x; i < n; i += NT) {
        const int s = seq[i], a = start[i], m = span[i], o = off[i], c = off[i + 1] - o;
        int bad = 0, len = 0, now = 0, f = 0;
        Gap gap;
        gap.probe(idx + o, c < m ? c : 0);             // beside the length
        if (bad_slot(p, sh.seen, s)) {
            bad = OCCAM_PAGES_BAD_SEQ;
        } else {
            len = now = p.length[s];
            if (a < 0 || m < 0 || (long long)a + m > len || c < 0 || c > m) {
                bad = OCCAM_PAGES_BAD_SPAN;
            } else if (c < m) {
                now = len - m + c;
                f = (a + gap.find(idx + o, c)) >> p.shift;
            } else {
                f = (len + G - 1) >> p.shift;            // nothing dropped
            }
        }
        first[i] = g_first[i] = f;
        olds[i] = g_olds[i] = len;
        news[i] = g_news[i] = now;
        if (bad) atomicOr(&sh.bad, bad);
    }
    __syncthreads();
    const long long want = wide_prefix_of<NT>(n, sh.need, sh.red2, [&](int i) {
        const int pages = ((news[i] + G - 1) >> p.shift) - first[i];
        return sh.bad || pages < 0 ? 0 : pages;
    });
    const int need = want > p.num_pages ? p.num_pages + 1 : (int)want;     // (more than there can be)
    __syncthreads();
    const bool listed = need <= kList;
    int* list = listed ? sh.list : plan_record(plan, n, p.max_pages, 0);
    if (sh.bad || !take_free<NT>(p, word0, need, sh, list)) {
        for (int i = threadIdx.x; i < n; i += NT) {
            g_news[i] = olds[i];
            g_first[i] = (olds[i] + G - 1) >> p.shift;
        }
        if (threadIdx.x == 0) {
            atomicOr(p.status, sh.bad ? sh.bad : (int)OCCAM_PAGES_FULL);
            write_header(plan, kPlanKeep, n, 0);
        }
        return;
    }
    __syncthreads();
    auto place = [&](int x, int i) {
        const int page = list[x];
        p.refs[page] = 1;
        plan_pages(plan, n, p.max_pages, i)[first[i] + x - sh.need[i]] = page;
        return page;
    };
    auto record = [&](int x, int i, int page) {
        const int j = first[i] + x - sh.need[i], now = news[i] - (j << p.shift);
        int* r = plan_record(plan, n, p.max_pages, x);
        r[RK_PAGE] = page;
        r[RK_POS] = j << p.shift;
        r[RK_END] = now < G ? now : G;
        r[RK_SEQ] = i;
        r[RK_START] = start[i];
        r[RK_SPAN] = span[i];
        r[RK_OFF] = off[i];
        r[RK_COUNT] = off[i + 1] - off[i];
    };
    for (int x = threadIdx.x; x < need; x += NT) {
        const int i = owner_of(sh.need, n, x), page = place(x, i);
        if (listed) record(x, i, page);
    }
    if (!listed) {                         // the list lies where the records go
        __syncthreads();
        for (int x = threadIdx.x; x < need; x += NT) {
            const int i = owner_of(sh.need, n, x);
            record(x, i, plan_pages(plan, n, p.max_pages, i)[first[i] + x - sh.need[i]]);
        }
    }
    if (threadIdx.x == 0) write_header(plan, kPlanKeep, n, need);
}

// Compaction, second part, a workgroup per sequence: the fresh pages go into the table, the
// old ones into the plan's list (the move reads from them), and the old ones' references
// end.
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

// A planning kernel with its state in LDS.
template <int NT, auto kernel, typename... A>
static hipError_t plan_launch(hipStream_t s, A... args) {
    constexpr int bytes = sizeof(PlanShared<NT>);
    static std::atomic<uint64_t> done{0};
    const hipError_t e = bytes <= 65536 ? hipSuccess
                                        : allow_lds(reinterpret_cast<const void*>(kernel), bytes, done);
    return e != hipSuccess ? e : launch(kernel, dim3(1), dim3(NT), bytes, s, args...);
}

hipError_t launch_pages_reserve(const PageView& p, const BatchView& b, int* plan, hipStream_t s) {
    const bool small = b.n <= 256 && b.n * (((long long)b.max_rows >> p.shift) + 1) <= kSmallPages;
    return small ? plan_launch<256, pages_reserve<256>>(s, p, b, plan)
                      : plan_launch<1024, pages_reserve<1024>>(s, p, b, plan);
}

hipError_t launch_pages_fork(const PageView& p, int n, const int* src, const int* dst, int* plan,
                             hipStream_t s) {
    if ((long long)n * p.max_pages <= kSmallTables)
        return launch(fork_plan<1024, true>, dim3(1), dim3(1024), 0, s, p, n, src, dst, plan);
    hipError_t e = n <= 256
        ? launch(fork_plan<256, false>, dim3(1), dim3(256), 0, s, p, n, src, dst, plan)
        : launch(fork_plan<1024, false>, dim3(1), dim3(1024), 0, s, p, n, src, dst, plan);
    if (e != hipSuccess) return e;
    return launch(fork_copy, dim3(n), dim3(256), 0, s, p, n, src, dst, plan);
}

hipError_t launch_pages_free(const PageView& p, int n, const int* seq, hipStream_t s) {
    return launch(pages_free, dim3(n), dim3(256), 0, s, p, seq);
}

hipError_t launch_pages_keep(const PageView& p, int n, const int* seq, const int* start,
                             const int* span, const int* idx, const int* off, int* plan,
                             hipStream_t s) {
    hipError_t e = n <= 256
        ? plan_launch<256, keep_plan<256>>(s, p, n, seq, start, span, idx, off, plan)
        : plan_launch<1024, keep_plan<1024>>(s, p, n, seq, start, span, idx, off, plan);
    if (e != hipSuccess) return e;
    return launch(keep_swap, dim3(n), dim3(256), 0, s, p, n, seq, plan);
}

}  // namespace occam
