// From the lengths of requests to what a step's operators read: row starts, positions, slots, owners, and the table of pages, for which pages are taken
// from a stack of free ones or given back to it.
//
//   q_start = sums of fresh;  want = ceil((cached + fresh) / page_size) pages of a request;  more than it holds are taken, fewer are given back
//
// Everything is a sum over the requests before, so one workgroup does it, 1024 requests at a time: first the row starts and what is given back (the
// taking may need it), then what is taken.  The pages themselves are moved by all threads, each finding the request of its page in the sums.
// Bound by latency: a launch (3 us), and some ten steps in a row of 0.3 to 1 us each (loads, sums over the threads, lookups).  8 requests: the kernel 4.3 us.  1000 requests, 50 of which
// give back 6000 pages, 7000 rows: 8.5, and 4 for a second launch that fills rows with many workgroups (up to 4096 rows the first fills them in at most as long).
#include "bcq_internal.h"
#include "bcq_lanes.h"

namespace bcq {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kOneLaunch = 4096;  // rows of the batch that the one workgroup fills too
constexpr int kFillThreads = 256;
constexpr int kAtOnce = 4;

typedef long long i64;

// Sum over the threads up to and with this one; `all`: over all of them.  `shared`: kWaves, free again after the next barrier.
template <class T>
__device__ __forceinline__ T sum_of_threads(T v, T *shared, T &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = sum_upto(v, lane);
    if (lane == 63) shared[wave] = v;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) v += shared[w];
        all += shared[w];
    }
    __syncthreads();
    return v;
}

// What the step asks of a request, whatever the arrays hold.
struct Wish {
    int cached, fresh;
    int held, want;  // pages
    bool fits;       // its row of the table
};
__device__ __forceinline__ Wish load_wish(const PlanArgs &p, int r)
{
    Wish w;
    w.cached = max(p.cached[r], 0);
    w.fresh = max(p.fresh[r], 0);
    w.held = min(max(p.held[r], 0), p.max_pages);
    const int fixed = p.fixed ? min(max(p.fixed[r], 0), w.held) : 0;
    const i64 pages = ((i64)w.cached + w.fresh + p.page_size - 1) >> p.page_shift;
    w.fits = pages <= p.max_pages;
    w.want = w.fits ? max((int)pages, fixed) : w.held;
    return w;
}

// The first i with upto[i] > k, of n; upto rises.
__device__ __forceinline__ int first_beyond(const int *upto, int n, int k)
{
    int low = 0;
    for (int high = n - 1; low < high;) {
        const int middle = (low + high) / 2;
        if (upto[middle] > k) high = middle;
        else low = middle + 1;
    }
    return low;
}

// The same of kThreads in LDS (the last if there is none), for N numbers that are k[0] and kThreads apart, side by side.
template <int N>
__device__ __forceinline__ void first_beyond(const int *upto, const int (&k)[N], int (&i)[N])
{
#pragma unroll
    for (int n = 0; n < N; ++n) i[n] = 0;
#pragma unroll
    for (int step = kThreads / 2; step > 0; step >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (upto[i[n] + step - 1] <= k[n]) i[n] += step;
}

// move(k, request, which of its pages) in two halves, for k = 0 .. all - 1 pages of requests whose sums are `upto`: all threads, kAtOnce each at a time, since each waits for what it
// finds and then for what it loads (1000 requests of which 50 give back 6000 pages: 13.9 us a call, 15.7 with one at a time; 24 that take 7000: 11.4 and 15.0).
// (k counts in unsigned numbers: 1024 requests may have up to 2^31 - 1 pages, and a signed k would wrap to negative places before it has passed them.)
template <class LOAD, class STORE>
__device__ __forceinline__ void move_pages(const int *upto, int all, LOAD load, STORE store)
{
    const unsigned pages = all;
    for (unsigned k0 = threadIdx.x; k0 < pages; k0 += kAtOnce * kThreads) {
        int k[kAtOnce], i[kAtOnce], page[kAtOnce];
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) k[n] = (int)min(k0 + n * kThreads, pages - 1);
        first_beyond(upto, k, i);
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) page[n] = load(k[n], i[n], k[n] - (i[n] ? upto[i[n] - 1] : 0));
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n)
            if (k0 + n * kThreads < pages) store(k[n], i[n], k[n] - (i[n] ? upto[i[n] - 1] : 0), page[n]);
    }
}

// Row t of the batch: which request's, where it is, where its key and value go.
__device__ __forceinline__ void fill_row(const PlanArgs &p, int t, int r, int start, bool any)
{
    int position = 0, slot = -1;
    if (any) {
        position = (int)min((i64)max(p.cached[r], 0) + t - start, 0x7fffffffll);
        if (p.lack[r] == 0) {
            const int page = p.pages[(i64)r * p.max_pages + min(position >> p.page_shift, p.max_pages - 1)];
            if ((unsigned)page < (unsigned)p.num_pages) slot = (page << p.page_shift) + (position & (p.page_size - 1));
        }
    }
    p.positions[t] = position;
    p.slots[t] = slot;
    p.owner[t] = any ? r : -1;
}

}  // namespace

// FEW: at most 1024 requests, a thread keeps its own; then so few rows of the batch as kOneLaunch are filled here too.
template <bool FEW>
__global__ __launch_bounds__(kThreads) void bcq_plan_kernel(PlanArgs p)
{
    __shared__ i64 sums64[kWaves];
    __shared__ int sums[kWaves], upto[kThreads], first[kThreads], starts[FEW ? kThreads : 1];
    const int thread = threadIdx.x;
    const int count = min(max(*p.free_count, 0), p.num_pages);
    const int requests = p.requests, end_of_requests = FEW ? 1 : requests;
    Wish w = {0, 0, 0, 0, false};

    // ---- row starts; pages that are given back, in the order of requests, onto the stack ----
    i64 rows = 0;
    int back = 0;
    for (int c = 0; c < end_of_requests; c += kThreads) {
        const int r = c + thread;
        w = Wish{0, 0, 0, 0, true};
        if (r < requests) w = load_wish(p, r);
        i64 all_rows;
        const i64 end = rows + sum_of_threads<i64>(w.fresh, sums64, all_rows);
        rows += all_rows;
        w.fits = w.fits && end <= p.tokens;
        const int start = (int)min(end, (i64)p.tokens);
        if (FEW) starts[thread] = start;
        if (r < requests) {
            p.q_start[r + 1] = start;
            if (!FEW) p.lack[r] = w.fits ? 0 : -1;
        }
        const int mine = w.fits ? max(w.held - w.want, 0) : 0;
        int all;
        upto[thread] = sum_of_threads<int>(mine, sums, all);
        first[thread] = w.want;
        __syncthreads();
        move_pages(
            upto, all, [&](int, int i, int j) { return p.pages[(i64)(c + i) * p.max_pages + first[i] + j]; },
            [&](int k, int, int, int page) {
                const i64 at = (i64)count + back + k;
                if (at < p.num_pages) p.free_pages[at] = page;
            });
        back += all;
        __syncthreads();
    }
    if (thread == 0) p.q_start[0] = 0;
    const int there = (int)min((i64)count + back, (i64)p.num_pages);

    // ---- pages that are taken, from its top ----
    int asked = 0, taken = 0;  // by all requests before; by those that got them
    for (int c = 0; c < end_of_requests; c += kThreads) {
        const int r = c + thread;
        if (!FEW) {
            w = Wish{0, 0, 0, 0, false};
            if (r < requests) {
                w = load_wish(p, r);
                w.fits = p.lack[r] == 0;
            }
        }
        const int need = w.fits ? max(w.want - w.held, 0) : 0;
        int all;
        const int end = asked + sum_of_threads<int>(need, sums, all);
        const bool served = w.fits && (need == 0 || end <= there);
        // (who is served gets what stands before, so the pages of all that are served are the first ones)
        int got;
        upto[thread] = sum_of_threads<int>(served ? need : 0, sums, got);
        first[thread] = w.held;
        __syncthreads();
        move_pages(
            upto, got, [&](int k, int, int) { return p.free_pages[there - 1 - (taken + k)]; },
            [&](int, int i, int j, int page) { p.pages[(i64)(c + i) * p.max_pages + first[i] + j] = page; });
        if (r < requests) {
            p.kv_len[r] = served ? w.cached + w.fresh : 0;
            p.held_out[r] = served ? w.want : w.held;
            if (FEW || (w.fits && !served)) p.lack[r] = !w.fits ? -1 : served ? 0 : need;
        }
        asked += all;
        taken += got;
        __syncthreads();
    }
    if (thread == 0) *p.free_count_out = there - taken;

    // ---- rows of the batch ----
    if (FEW && p.tokens <= kOneLaunch) {
        const int all = requests ? starts[requests - 1] : 0;
        for (int t = thread; t < p.tokens; t += kThreads) {
            int r[1] = {0};
            if (t < all) first_beyond<1>(starts, {t}, r);
            fill_row(p, t, r[0], r[0] ? starts[r[0] - 1] : 0, t < all);
        }
    }
}

// The rows of a large batch, after the kernel above.
template <bool FEW>
__global__ __launch_bounds__(kFillThreads) void bcq_plan_fill_kernel(PlanArgs p)
{
    __shared__ int ends[FEW ? kThreads : 1];
    const int t = blockIdx.x * kFillThreads + threadIdx.x;
    int r = 0;
    if (FEW) {
#pragma unroll
        for (int i = threadIdx.x; i < kThreads; i += kFillThreads) ends[i] = p.requests ? p.q_start[min(i + 1, p.requests)] : 0;
        __syncthreads();
        first_beyond<1>(ends, {t}, reinterpret_cast<int(&)[1]>(r));
        r = max(min(r, p.requests - 1), 0);
    } else if (t < p.tokens) {
        r = first_beyond(p.q_start + 1, p.requests, t);
    }
    if (t >= p.tokens) return;
    const int start = p.requests && r ? FEW ? ends[r - 1] : p.q_start[r] : 0;
    fill_row(p, t, r, start, p.requests && (FEW ? ends[r] : p.q_start[r + 1]) > t);
}

hipError_t launch_plan(const PlanArgs &p, hipStream_t stream)
{
    const bool few = p.requests <= kThreads;
    if (few) bcq_plan_kernel<true><<<1, kThreads, 0, stream>>>(p);
    else bcq_plan_kernel<false><<<1, kThreads, 0, stream>>>(p);
    if (!few || p.tokens > kOneLaunch) {
        const int groups = (p.tokens + kFillThreads - 1) / kFillThreads;
        if (few) bcq_plan_fill_kernel<true><<<groups, kFillThreads, 0, stream>>>(p);
        else if (groups) bcq_plan_fill_kernel<false><<<groups, kFillThreads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace bcq
