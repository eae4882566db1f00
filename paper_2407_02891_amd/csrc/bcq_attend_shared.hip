// Attention over a paged cache where groups of requests share their first keys: those are read once for the group.
//
//   out = sum_j softmax_j(scale q . k_j) v_j = join of (sums over the shared keys) and (sums over the request's own)
//
// A row is a (new token, query head) pair.  The rows of all requests of a group are the tiles of the shared keys (bcq_attend_tile.h), the rows of a request
// those of its own keys.  Bound by the matrix instructions where many rows share much, by the bytes of K and V where few do, or own much.
//  * The blocks of keys of all tiles, shared ones first, form one line, which is cut into as many equal pieces as there are workgroups for a kv head.  A workgroup walks
//    its piece, over the ends of tiles, and leaves sums, maximum and weight of each row of a tile (place: the row, and 128 further for each worker, which no two
//    share).  The lengths are on the device, so a first launch lays out the line.
//  * A last launch joins what was left of a row: of its shared keys and of its own.
#include "bcq_attend_tile.h"

namespace bcq {

namespace {

constexpr int kLineThreads = 1024;
constexpr int kJoinWaves = 4;

// A tile's place in the line.
struct Slot {
    int upto;   // blocks of the tiles up to and with it
    int part;   // whose tile: of a group's shared keys (below `groups`), of a request's own
    int row0;   // its first row
    int block;  // its first block of keys
};

struct SharedParams {
    AttendParams a;  // (workers, part, stat too)
    const int *group_start, *shared_len;
    int groups, max_shared;
    Slot *slots;
    int num_slots;
    long long space;  // rows that a kv head's sums have room for
};

// The rows of a group or request, and its keys.
struct Part {
    int start, rows;      // first token; rows
    int request;          // whose row of the table of pages
    int requests;         // of a group
    int from, to;         // its keys
};

__device__ __forceinline__ int start_of(const SharedParams &p, int r) { return min(max(p.a.q_start[r], 0), p.a.tokens); }
__device__ __forceinline__ int first_of_group(const SharedParams &p, int c) { return min(max(p.group_start[c], 0), p.a.requests); }

__device__ __forceinline__ int shared_keys(const SharedParams &p, int c)
{
    return (int)min((long long)min(max(p.shared_len[c], 0), p.max_shared), (long long)p.a.max_pages << p.a.page_shift);
}

// The group of a request, or -1.
__device__ __forceinline__ int group_of(const SharedParams &p, int r)
{
    int low = 0;
    for (int high = p.groups; high - low > 1;) {
        const int middle = (low + high) / 2;
        if (first_of_group(p, middle) <= r) low = middle;
        else high = middle;
    }
    return p.groups > 0 && first_of_group(p, low) <= r && r < first_of_group(p, low + 1) ? low : -1;
}

__device__ __forceinline__ Part load_part(const SharedParams &p, int v)
{
    Part q;
    if (v < p.groups) {
        const int first = first_of_group(p, v), end = max(first_of_group(p, v + 1), first);
        q.start = start_of(p, first);
        q.rows = max(start_of(p, end) - q.start, 0) * p.a.group;
        q.request = min(first, p.a.requests - 1);
        q.requests = end - first;
        q.from = 0;
        q.to = shared_keys(p, v);
    } else {
        const int r = v - p.groups, c = group_of(p, r);
        const Request own = load_request(p.a, r);
        q.start = own.start;
        q.rows = own.todo * p.a.group;
        q.request = r;
        q.requests = 1;
        q.from = c < 0 ? 0 : shared_keys(p, c);
        q.to = own.len;
    }
    return q;
}

// The tiles of a part begin at this slot.
__device__ __forceinline__ int slots_before(const SharedParams &p, int v, int start)
{
    const long long at = v < p.groups ? start : (long long)p.a.tokens + start;
    return (int)(at * p.a.group / kChunkRows) + v;
}

// Blocks of a tile: [first, end).
template <int DT>
__device__ __forceinline__ void blocks_of(const SharedParams &p, int v, const Part &q, int row0, int &first, int &end)
{
    constexpr int KB = tile_keys(DT);
    int from = q.from, to = q.to;
    const int token0 = row0 / p.a.group, token1 = (min(row0 + kChunkRows, q.rows) - 1) / p.a.group;
    if (v >= p.groups) {
        const Request own = load_request(p.a, q.request);
        int low, high, unused;
        visible_keys(p.a, own.n, own.len, token0, low, unused);
        visible_keys(p.a, own.n, own.len, token1, unused, high);
        from = max(from, low), to = min(to, max(high, 0));
    }
    first = min(from, to) / KB;
    end = from < to ? (to + KB - 1) / KB : first;
}

}  // namespace

// Lays out the line: blocks of each slot, then their sums.
template <int DT>
__global__ __launch_bounds__(kLineThreads) void bcq_attend_shared_line_kernel(SharedParams p)
{
    __shared__ int sums[kLineThreads / 64];
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    for (int s = thread; s < p.num_slots; s += kLineThreads) p.slots[s] = Slot{0, 0, 0, 0};
    __syncthreads();
    for (int v = thread; v < p.groups + p.a.requests; v += kLineThreads) {
        const Part q = load_part(p, v);
        const int slot = slots_before(p, v, q.start);
        for (int row0 = 0, s = slot; row0 < q.rows && s < p.num_slots; row0 += kChunkRows, ++s) {
            int first, end;
            blocks_of<DT>(p, v, q, row0, first, end);
            p.slots[s] = Slot{end - first, v, row0, first};
        }
    }
    __syncthreads();
    int before = 0;
    for (int c = 0; c < p.num_slots; c += kLineThreads) {
        const int s = c + thread;
        const int upto = prefix_sum(s < p.num_slots ? p.slots[s].upto : 0, lane);
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int mine = before + upto;
        for (int w = 0; w < kLineThreads / 64; ++w) {
            if (w < wave) mine += sums[w];
            before += sums[w];
        }
        if (s < p.num_slots) p.slots[s].upto = mine;
        __syncthreads();
    }
}

template <int DT, bool BF, bool ANY>
__global__ __launch_bounds__(64 * kTileWaves, tile_occupancy(DT)) void bcq_attend_shared_kernel(SharedParams p)
{
    constexpr int DV = DT / 32;
    __shared__ int bounds[kTileWaves][2];
    const AttendParams &a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, h = lane >> 5;
    const int head = blockIdx.x % a.kv_heads, worker = blockIdx.x / a.kv_heads;
    const int total = p.slots[p.num_slots - 1].upto, workers = min(a.workers, max(total, 1));
    if (worker >= workers) return;
    int at = first_block(worker, workers, total);
    const int stop = first_block(worker + 1, workers, total);
    if (at >= stop) return;
    // the slot that holds block `at`: the first with upto > at
    int slot = 0;
    for (int high = p.num_slots - 1; slot < high;) {
        const int stride = (high - slot + 63) / 64, probe = slot + lane * stride;
        const int beyond = __popcll(__ballot(probe < high && p.slots[probe].upto <= at));  // (rises, so these are the first lanes)
        if (!beyond) break;
        const int last = slot + (beyond - 1) * stride;  // not yet
        high = min(high, last + stride);
        slot = last + 1;
    }
    slot = __builtin_amdgcn_readfirstlane(slot);
    while (at < stop) {
        const Slot s = p.slots[slot];
        const int before = slot ? p.slots[slot - 1].upto : 0, end = min(s.upto, stop);
        if (end <= at) {  // (a slot without blocks)
            ++slot;
            continue;
        }
        const Part q = load_part(p, s.part);
        const bool of_group = s.part < p.groups;
        // ---- the lane's row, and what it sees ----
        const int row = s.row0 + 32 * wave + r32;
        const int token = row / a.group, member = row - token * a.group, global_token = min(q.start + token, a.tokens - 1);
        int r = q.request;
        if (of_group) {  // the request of the token: where each has one, as many behind the first
            const int end_request = min(q.request + q.requests, a.requests) - 1;
            const int guess = min(q.request + token, end_request);
            if (a.q_start[guess] <= global_token && a.q_start[guess + 1] > global_token) {
                r = guess;
            } else {
                int low = q.request;
                for (int high = end_request + 1; high - low > 1;) {
                    const int middle = (low + high) / 2;
                    if (a.q_start[middle] <= global_token) low = middle;
                    else high = middle;
                }
                r = low;
            }
        }
        const Request own = load_request(a, r);
        const int i = q.start + token - own.start;
        const bool real = row < q.rows && i >= 0 && i < own.todo;
        int from = 0, to = 0;
        if (real) {
            visible_keys(a, own.n, own.len, i, from, to);
            from = max(from, q.from), to = min(to, q.to);
        }
        Tile t;
        t.head = head, t.request = q.request, t.last = max(q.to - 1, 0);
        t.b0 = s.block + at - before, t.b1 = s.block + end - before;
        int all_from = real ? from : 0, all_to = real ? to : 0x7fffffff, any_from = real ? from : 0x7fffffff, any_to = real ? to : 0;
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) {
            all_from = max(all_from, __shfl_xor(all_from, x));
            all_to = min(all_to, __shfl_xor(all_to, x));
            any_from = min(any_from, __shfl_xor(any_from, x));
            any_to = max(any_to, __shfl_xor(any_to, x));
        }
        t.all_from = __builtin_amdgcn_readfirstlane(all_from), t.all_to = __builtin_amdgcn_readfirstlane(all_to);
        t.any_from = __builtin_amdgcn_readfirstlane(any_from), t.any_to = __builtin_amdgcn_readfirstlane(any_to);
        if (lane == 0) bounds[wave][0] = all_from, bounds[wave][1] = all_to;
        __syncthreads();  // (the buffers of the tile before are free too)
        int tile_from = 0, tile_to = 0x7fffffff;
#pragma unroll
        for (int w = 0; w < kTileWaves; ++w) tile_from = max(tile_from, bounds[w][0]), tile_to = min(tile_to, bounds[w][1]);
        t.tile_from = __builtin_amdgcn_readfirstlane(tile_from), t.tile_to = __builtin_amdgcn_readfirstlane(tile_to);
        t.has_rows = __ballot(real) != 0;
        t.real = real, t.from = from, t.to = to;
        t.q = a.q + (long long)(real ? q.start + token : q.start < a.tokens ? q.start : 0) * a.ld_q + (head * a.group + (real ? member : 0)) * a.head_dim;
        f32x16 o[DV];
        float most, sum;
        attend_tile<DT, BF, ANY, false>(a, t, o, most, sum);

        const auto twin = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, sum), __builtin_bit_cast(unsigned, sum), false, false);
        sum = __builtin_bit_cast(float, (unsigned)twin[0]) + __builtin_bit_cast(float, (unsigned)twin[1]);
        if (real) {
            const long long place = head * p.space + (of_group ? 0 : (long long)a.tokens * a.group) + (long long)q.start * a.group + row + (long long)kChunkRows * worker;
#pragma unroll
            for (int d = 0; d < DV; ++d)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    *reinterpret_cast<f32x4 *>(a.part + place * DT + 32 * d + 8 * u + 4 * h) =
                        f32x4{o[d][4 * u], o[d][4 * u + 1], o[d][4 * u + 2], o[d][4 * u + 3]};
            if (h == 0) a.stat[place] = f32x2{most, sum};
        }
        at = end;
        ++slot;
        __syncthreads();  // (every wave is through with the bounds and the buffers)
    }
}

// Joins what was left of a row: a wave has a row.
template <int DT, bool BF>
__global__ __launch_bounds__(64 * kJoinWaves) void bcq_attend_shared_join_kernel(SharedParams p)
{
    constexpr int E = DT / 64;
    const AttendParams &a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % a.kv_heads, row = blockIdx.x / a.kv_heads * kJoinWaves + wave;
    const int token = row / a.group, member = row - token * a.group;
    if (token >= a.tokens) return;
    const int r = last_request(a, lane, [&](int i) { return a.q_start[i] <= token; });
    const Request own = load_request(a, r);
    const int i = token - own.start;
    if (i < 0 || i >= own.todo) return;
    const int c = group_of(p, r);
    const int total = p.slots[p.num_slots - 1].upto, workers = min(a.workers, max(total, 1));
    // pieces of the shared keys, then of its own
    long long place[2];
    int pieces[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int v = k ? p.groups + r : c;
        if (v < 0) continue;
        const int start = k ? own.start : start_of(p, first_of_group(p, c)), in_part = (token - start) * a.group + member;
        const int s = slots_before(p, v, start) + in_part / kChunkRows;
        if (in_part < 0 || s >= p.num_slots) continue;
        const int from = s ? p.slots[s - 1].upto : 0, upto = p.slots[s].upto;
        if (upto <= from) continue;
        const int w0 = worker_of(from, workers, total);
        pieces[k] = worker_of(upto - 1, workers, total) - w0 + 1;
        place[k] = head * p.space + (k ? (long long)a.tokens * a.group : 0) + (long long)token * a.group + member + (long long)kChunkRows * w0;
    }
    const auto at = [&](int n) { return n < pieces[0] ? place[0] + (long long)n * kChunkRows : place[1] + (long long)(n - pieces[0]) * kChunkRows; };
    float y[E], weight;
    join_pieces<DT, 1>(a, at, 0, pieces[0] + pieces[1], 0, lane, y, weight);
    int from, to;
    visible_keys(a, own.n, own.len, i, from, to);
    uint16_t *const dst = a.out + (long long)token * a.ld_out + (head * a.group + member) * a.head_dim;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (lane * E + e < a.head_dim) dst[lane * E + e] = from_float<BF>(to > from ? y[e] / weight : 0.0f);
}

namespace {

struct SharedPlan {
    int dim, workers, num_slots;
    long long space;
    size_t slot_bytes, part_bytes, stat_bytes;
};
SharedPlan shared_plan(const bcq_cache &c, int tokens, int requests, int groups, int q_heads)
{
    SharedPlan s;
    s.dim = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
    const int group = q_heads / c.kv_heads;
    const int per_head = compute_units() * tile_occupancy(s.dim) / c.kv_heads;  // as many workgroups as the chip holds
    s.workers = per_head > 1 ? per_head : 1;
    s.num_slots = (int)(2ll * tokens * group / kChunkRows) + groups + requests + 1;
    s.space = 2ll * tokens * group + (long long)kChunkRows * s.workers;
    s.slot_bytes = (size_t)s.num_slots * sizeof(Slot);
    s.part_bytes = (size_t)s.space * c.kv_heads * s.dim * sizeof(float);
    s.stat_bytes = (size_t)s.space * c.kv_heads * sizeof(f32x2);
    return s;
}

template <int DT, bool BF>
void shared_launches(const SharedParams &p, bool any, hipStream_t s)
{
    const AttendParams &a = p.a;
    bcq_attend_shared_line_kernel<DT><<<1, kLineThreads, 0, s>>>(p);
    const unsigned groups = (unsigned)a.workers * a.kv_heads;
    if (any) bcq_attend_shared_kernel<DT, BF, true><<<groups, 64 * kTileWaves, 0, s>>>(p);
    else bcq_attend_shared_kernel<DT, BF, false><<<groups, 64 * kTileWaves, 0, s>>>(p);
    const long long rows = (long long)a.tokens * a.group;
    bcq_attend_shared_join_kernel<DT, BF><<<(unsigned)((rows + kJoinWaves - 1) / kJoinWaves * a.kv_heads), 64 * kJoinWaves, 0, s>>>(p);
}

template <bool BF>
void shared_by_dim(const SharedParams &p, int dim, bool any, hipStream_t s)
{
    if (dim == 64) shared_launches<64, BF>(p, any, s);
    else if (dim == 128) shared_launches<128, BF>(p, any, s);
    else shared_launches<256, BF>(p, any, s);
}

}  // namespace

size_t attend_shared_workspace_bytes(const bcq_cache &c, int tokens, int requests, int groups, int q_heads)
{
    const SharedPlan s = shared_plan(c, tokens, requests, groups, q_heads);
    return s.part_bytes + s.stat_bytes + s.slot_bytes;
}

hipError_t launch_attend_shared(const AttendSharedArgs &args, hipStream_t stream)
{
    const AttendArgs &a = args.of;
    const bcq_cache &c = a.cache;
    const SharedPlan plan = shared_plan(c, a.tokens, a.requests, args.groups, a.q_heads);
    char *const ws = static_cast<char *>(a.workspace);
    SharedParams s = {};
    AttendParams &p = s.a;
    p.k = a.k, p.v = a.v, p.q = a.q, p.q_start = a.q_start, p.kv_len = a.kv_len, p.pages = a.pages, p.out = a.out;
    p.part = reinterpret_cast<float *>(ws);
    s.slots = reinterpret_cast<Slot *>(ws + plan.part_bytes);
    p.stat = reinterpret_cast<f32x2 *>(ws + plan.part_bytes + plan.slot_bytes);
    p.ld_q = a.ld_q, p.ld_out = a.ld_out, p.page_stride = c.page_stride, p.head_stride = c.head_stride, p.slot_stride = (int)c.slot_stride;
    p.tokens = a.tokens, p.requests = a.requests, p.kv_heads = c.kv_heads, p.group = a.q_heads / c.kv_heads;
    p.head_dim = c.head_dim, p.page_shift = __builtin_ctz(c.page_size), p.num_pages = c.num_pages, p.max_pages = a.max_pages;
    p.max_new = a.max_new, p.causal = a.causal;
    p.window = a.window > 1 << 30 ? 0 : a.window;  // (no request has so many keys, and positions less a window stay in range)
    p.scale = (float)(a.scale * 1.4426950408889634);
    p.workers = plan.workers;
    s.group_start = args.group_start, s.shared_len = args.shared_len, s.groups = args.groups, s.max_shared = args.max_shared;
    s.num_slots = plan.num_slots, s.space = plan.space;
    const bool any = c.head_dim != plan.dim || c.page_size < 16;
    if (c.dtype == BCQ_BF16) shared_by_dim<true>(s, plan.dim, any, stream);
    else shared_by_dim<false>(s, plan.dim, any, stream);
    return hipGetLastError();
}

}  // namespace bcq
