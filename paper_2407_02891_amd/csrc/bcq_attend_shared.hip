// Attention over a paged cache where groups of requests share their first keys: those are read once for the group.
//
//   out = sum_j softmax_j(scale q . k_j) v_j = join of (sums over the shared keys) and (sums over the request's own)
//
// A row is a (new token, query head) pair.  The rows of all requests of a group are the tiles of the shared keys (bcq_attend_tile.h), the rows of a request
// those of its own keys.  Bound by the matrix instructions where many rows share much, by the bytes of K and V where few do, or own much.
//  * The blocks of keys of the shared tiles form one line, those of the others a second.  Each is cut into as many equal pieces as there are workgroups for a kv head, and a
//    workgroup has one of each: half of them begin with the first, half with the second, so that what is bound by the matrix instructions runs beside what is bound by memory.  A
//    workgroup walks its pieces, over the ends of tiles, and leaves sums, maximum and weight of each row of a tile (place: the row, and 128 further for each worker, which no
//    two share).  The lengths are on the device, so a first launch lays out the lines.
//  * A last launch joins what was left of a row: of its shared keys and of its own.
#include "bcq_attend_tile.h"

namespace bcq {

namespace {

constexpr int kLineThreads = 1024;
constexpr int kJoinThreads = 256;

// A tile and its place in its line (64 bytes, one scalar load).
struct Slot {
    int upto;         // blocks of the line up to and with it
    int part;         // whose tile: of a group's shared keys (below `groups`), of a request's own; -1: nobody's
    int row0;         // its first row in the part
    int block;        // its first block of keys
    int start, rows;  // of the part: first token; rows
    int request;      // whose row of the table of pages
    int requests;     // of a group; a request's group, or -1
    int from, to;     // keys of the part
    int n, len;       // of a request: new tokens, keys; of a group: whether each row sees all of the keys
    int worker;       // the first that has a block of it
    int pieces;       // how many have
    int unused[2];
};
static_assert(sizeof(Slot) == 64, "");

struct SharedParams {
    AttendParams a;  // (workers, part, stat too)
    const int *group_start, *shared_len;
    int groups, max_shared;
    Slot *slots;
    int num_slots, own_slots;  // the slots of requests' own keys begin at own_slots
    long long space;           // rows that a kv head's sums have room for, of each line
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

// The tiles of a part begin at this slot.
__device__ __forceinline__ int slots_before(const SharedParams &p, int v, int start)
{
    const int at = (int)((long long)start * p.a.group / kChunkRows);
    return v < p.groups ? at + v : p.own_slots + at + v - p.groups;
}

// A slot by scalar loads (all lanes the same one, laid out by an earlier launch).
__device__ __forceinline__ Slot load_slot(const SharedParams &p, int slot)
{
    typedef const __attribute__((address_space(4))) int *scalar_int;
    const scalar_int from = (scalar_int) reinterpret_cast<const int *>(p.slots + __builtin_amdgcn_readfirstlane(slot));
    Slot s;
    s.upto = from[0], s.part = from[1], s.row0 = from[2], s.block = from[3], s.start = from[4], s.rows = from[5], s.request = from[6];
    s.requests = from[7], s.from = from[8], s.to = from[9], s.n = from[10], s.len = from[11], s.worker = from[12], s.pieces = from[13];
    return s;
}

}  // namespace

// Lays out the lines: the tiles of each part, then the sums of their blocks, then who has them.
template <int DT>
__global__ __launch_bounds__(kLineThreads) void bcq_attend_shared_line_kernel(SharedParams p)
{
    constexpr int KB = tile_keys(DT);
    __shared__ int sums[kLineThreads / 64];
    const AttendParams &a = p.a;
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    for (int s = thread; s < p.num_slots; s += kLineThreads) p.slots[s].upto = 0, p.slots[s].part = -1;
    __syncthreads();
    for (int v = thread; v < p.groups; v += kLineThreads) {
        const int first = first_of_group(p, v), end = max(first_of_group(p, v + 1), first);
        Slot q = {};
        q.part = v;
        q.start = start_of(p, first);
        q.rows = max(start_of(p, end) - q.start, 0) * a.group;
        q.request = min(first, a.requests - 1);
        q.requests = end - first;
        q.to = shared_keys(p, v);
        q.n = a.window == 0;
        q.upto = (q.to + KB - 1) / KB;
        for (int s = slots_before(p, v, q.start); q.row0 < q.rows && s < p.own_slots; q.row0 += kChunkRows, ++s) p.slots[s] = q;
    }
    __syncthreads();
    for (int r = thread; r < a.requests; r += kLineThreads) {
        const Request own = load_request(a, r);
        const int c = group_of(p, r);
        Slot q = {};
        q.part = p.groups + r;
        q.start = own.start;
        q.rows = own.todo * a.group;
        q.request = r;
        q.requests = c;
        q.from = c < 0 ? 0 : shared_keys(p, c);
        q.to = own.len;
        q.n = own.n, q.len = own.len;
        for (int s = slots_before(p, q.part, q.start); q.row0 < q.rows && s < p.num_slots; q.row0 += kChunkRows, ++s) {
            // the keys that a row of the tile sees
            int low, high, unused;
            visible_keys(a, own.n, own.len, q.row0 / a.group, low, unused);
            visible_keys(a, own.n, own.len, (min(q.row0 + kChunkRows, q.rows) - 1) / a.group, unused, high);
            low = max(low, q.from);
            q.block = low / KB;
            q.upto = low < high ? (high + KB - 1) / KB - q.block : 0;
            p.slots[s] = q;
        }
        // does each of its rows see all that is shared?
        int unused, high;
        visible_keys(a, own.n, own.len, 0, unused, high);
        if (c >= 0 && own.n > 0 && (high < q.from || own.todo < own.n)) {
            const int first = start_of(p, first_of_group(p, c)), rows = max(start_of(p, first_of_group(p, c + 1)) - first, 0) * a.group;
            const int s = slots_before(p, c, first);
            for (int i = 0; i * kChunkRows < rows && s + i < p.own_slots; ++i) p.slots[s + i].n = 0;
        }
    }
    __syncthreads();
    const auto lay = [&](int first, int end) {
        int before = 0;
        for (int c = first; c < end; c += kLineThreads) {
            const int s = c + thread;
            const int upto = prefix_sum(s < end ? p.slots[s].upto : 0, lane);
            if (lane == 63) sums[wave] = upto;
            __syncthreads();
            int mine = before + upto;
            for (int w = 0; w < kLineThreads / 64; ++w) {
                if (w < wave) mine += sums[w];
                before += sums[w];
            }
            if (s < end) p.slots[s].upto = mine;
            __syncthreads();
        }
        const int workers = min(a.workers, max(before, 1));
        for (int s = first + thread; s < end; s += kLineThreads) {
            const int from = s > first ? p.slots[s - 1].upto : 0, upto = p.slots[s].upto;
            const int w0 = upto > from ? worker_of(from, workers, before) : 0;
            p.slots[s].worker = w0;
            p.slots[s].pieces = upto > from ? worker_of(upto - 1, workers, before) - w0 + 1 : 0;
        }
    };
    lay(0, p.own_slots);
    lay(p.own_slots, p.num_slots);
}

// The pieces of both lines.
template <int DT, bool BF, bool ANY>
__global__ __launch_bounds__(64 * kTileWaves, tile_occupancy(DT)) void bcq_attend_shared_kernel(SharedParams p)
{
    constexpr int DV = DT / 32;
    __shared__ int bounds[kTileWaves][2];
    const AttendParams &a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, h = lane >> 5;
    const int head = blockIdx.x % a.kv_heads, me = blockIdx.x / a.kv_heads;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
        // the second line is shared out from the last worker on: few blocks of each are then not one worker's
        const bool of_group = (turn == 0) == (2 * me < a.workers);
        const int first_slot = of_group ? 0 : p.own_slots, end_slot = of_group ? p.own_slots : p.num_slots;
        const int total = load_slot(p, end_slot - 1).upto, workers = min(a.workers, max(total, 1)), worker = of_group ? me : a.workers - 1 - me;
        if (worker >= workers) continue;
        int at = first_block(worker, workers, total);
        const int stop = first_block(worker + 1, workers, total);
        if (at >= stop) continue;
        // the slot that holds block `at`: the first with upto > at
        int slot = first_slot;
        for (int high = end_slot - 1; slot < high;) {
            const int stride = (high - slot + 63) / 64, probe = slot + lane * stride;
            const int beyond = __popcll(__ballot(probe < high && p.slots[probe].upto <= at));  // (rises, so these are the first lanes)
            if (!beyond) break;
            const int last = slot + (beyond - 1) * stride;  // not yet
            high = min(high, last + stride);
            slot = last + 1;
        }
        slot = __builtin_amdgcn_readfirstlane(slot);
        int before = slot > first_slot ? load_slot(p, slot - 1).upto : 0;
#pragma unroll 1
        for (; at < stop; ++slot) {
            const Slot s = load_slot(p, slot);
            const int end = min(s.upto, stop);
            if (end <= at) {  // (a slot without blocks)
                before = s.upto;
                continue;
            }
            // ---- the lane's row, and what it sees ----
            const int row = s.row0 + 32 * wave + r32;
            const int token = row / a.group, member = row - token * a.group;
            bool real = row < s.rows;
            Tile t;
            t.head = head, t.request = s.request, t.last = max(s.to - 1, 0);
            t.b0 = __builtin_amdgcn_readfirstlane(s.block + at - before), t.b1 = __builtin_amdgcn_readfirstlane(s.block + end - before);
            t.has_rows = s.row0 + 32 * wave < s.rows;
            if (of_group && s.n) {  // all rows all keys
                t.from = t.tile_from = t.all_from = t.any_from = 0;
                t.to = t.tile_to = t.all_to = t.any_to = s.to;
            } else if (!of_group) {
                int from, to, all_from, all_to, tile_from, tile_to, any_from, any_to, unused;
                visible_keys(a, s.n, s.len, token, from, to);
                visible_keys(a, s.n, s.len, s.row0 / a.group, unused, tile_to);
                visible_keys(a, s.n, s.len, (min(s.row0 + kChunkRows, s.rows) - 1) / a.group, tile_from, unused);
                visible_keys(a, s.n, s.len, (s.row0 + 32 * wave) / a.group, any_from, all_to);
                visible_keys(a, s.n, s.len, (min(s.row0 + 32 * wave + 32, s.rows) - 1) / a.group, all_from, any_to);
                t.from = max(from, s.from), t.to = to;
                t.tile_from = max(tile_from, s.from), t.tile_to = tile_to;
                t.all_from = max(all_from, s.from), t.all_to = all_to, t.any_from = max(any_from, s.from), t.any_to = any_to;
            } else {
                // the request of the token: where each has one, as many behind the first
                const int global_token = min(s.start + token, a.tokens - 1), end_request = min(s.request + s.requests, a.requests) - 1;
                int r = min(s.request + token, end_request);
                if (a.q_start[r] > global_token || a.q_start[r + 1] <= global_token) {
                    r = s.request;
                    for (int high = end_request + 1; high - r > 1;) {
                        const int middle = (r + high) / 2;
                        if (a.q_start[middle] <= global_token) r = middle;
                        else high = middle;
                    }
                }
                const Request own = load_request(a, r);
                const int i = s.start + token - own.start;
                real = real && i >= 0 && i < own.todo;
                int from = 0, to = 0;
                if (real) visible_keys(a, own.n, own.len, i, from, to);
                to = min(to, s.to);
                int all_from = real ? from : 0, all_to = real ? to : 0x7fffffff, any_from = real ? from : 0x7fffffff, any_to = real ? to : 0;
#pragma unroll
                for (int x = 16; x > 0; x >>= 1) {
                    all_from = max(all_from, __shfl_xor(all_from, x));
                    all_to = min(all_to, __shfl_xor(all_to, x));
                    any_from = min(any_from, __shfl_xor(any_from, x));
                    any_to = max(any_to, __shfl_xor(any_to, x));
                }
                if (lane == 0) bounds[wave][0] = all_from, bounds[wave][1] = all_to;
                __syncthreads();
                int tile_from = 0, tile_to = 0x7fffffff;
#pragma unroll
                for (int w = 0; w < kTileWaves; ++w) tile_from = max(tile_from, bounds[w][0]), tile_to = min(tile_to, bounds[w][1]);
                __syncthreads();  // (before they are written again)
                t.from = from, t.to = to;
                t.tile_from = __builtin_amdgcn_readfirstlane(tile_from), t.tile_to = __builtin_amdgcn_readfirstlane(tile_to);
                t.all_from = __builtin_amdgcn_readfirstlane(all_from), t.all_to = __builtin_amdgcn_readfirstlane(all_to);
                t.any_from = __builtin_amdgcn_readfirstlane(any_from), t.any_to = __builtin_amdgcn_readfirstlane(any_to);
                t.has_rows = __ballot(real) != 0;
            }
            t.real = real;
            t.q = a.q + (long long)(real ? s.start + token : min(s.start, a.tokens - 1)) * a.ld_q + (head * a.group + (real ? member : 0)) * a.head_dim;
            f32x16 o[DV];
            float most, sum;
            const bool reading = attend_tile<DT, BF, ANY, false>(a, t, o, most, sum);

            const auto twin = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, sum), __builtin_bit_cast(unsigned, sum), false, false);
            sum = __builtin_bit_cast(float, (unsigned)twin[0]) + __builtin_bit_cast(float, (unsigned)twin[1]);
            if (real) {
                const long long place = (2ll * head + (of_group ? 0 : 1)) * p.space + (long long)s.start * a.group + row + (long long)kChunkRows * worker;
#pragma unroll
                for (int d = 0; d < DV; ++d)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        *reinterpret_cast<f32x4 *>(a.part + place * DT + 32 * d + 8 * u + 4 * h) =
                            f32x4{o[d][4 * u], o[d][4 * u + 1], o[d][4 * u + 2], o[d][4 * u + 3]};
                if (h == 0) a.stat[place] = f32x2{most, sum};
            }
            at = end;
            before = s.upto;
            if (reading) __syncthreads();
        }
    }
}

// Joins what was left of a row, its shared keys' pieces and its own: four elements to a thread.
template <int DT, bool BF>
__global__ __launch_bounds__(kJoinThreads) void bcq_attend_shared_join_kernel(SharedParams p)
{
    constexpr int kLanes = DT / 4, kAhead = 4;
    const AttendParams &a = p.a;
    const int head = blockIdx.x % a.kv_heads, row = blockIdx.x / a.kv_heads * (kJoinThreads / kLanes) + (int)threadIdx.x / kLanes, d = 4 * (threadIdx.x % kLanes);
    const int token = row / a.group, member = row - token * a.group;
    if (token >= a.tokens || d >= a.head_dim) return;
    // the request of the token: where each has one, as many behind the first
    int r = min(token, a.requests - 1);
    if (a.q_start[r] > token || a.q_start[r + 1] <= token) {
        r = 0;
        for (int high = a.requests; high - r > 1;) {
            const int middle = (r + high) / 2;
            if (a.q_start[middle] <= token) r = middle;
            else high = middle;
        }
    }
    const Request own = load_request(a, r);
    const int i = token - own.start;
    if (i < 0 || i >= own.todo) return;
    const int s1 = slots_before(p, p.groups + r, own.start) + (i * a.group + member) / kChunkRows;
    const Slot &mine = p.slots[min(s1, p.num_slots - 1)];
    const int c = mine.requests;
    int pieces0 = 0, pieces = mine.pieces;
    const long long place1 = (2ll * head + 1) * p.space + (long long)token * a.group + member + (long long)kChunkRows * mine.worker;
    long long place0 = 0;
    if (c >= 0) {
        const int start = start_of(p, first_of_group(p, c));
        const Slot &shared = p.slots[min(slots_before(p, c, start) + max((token - start) * a.group + member, 0) / kChunkRows, p.own_slots - 1)];
        pieces0 = shared.pieces;
        place0 = 2ll * head * p.space + (long long)token * a.group + member + (long long)kChunkRows * shared.worker;
    }
    pieces += pieces0;
    const auto at = [&](int n) { return n < pieces0 ? place0 + (long long)n * kChunkRows : place1 + (long long)(n - pieces0) * kChunkRows; };
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
    float most = -INFINITY, weight = 0.0f;
    for (int n = 0; n < pieces; n += kAhead) {
        f32x4 part[kAhead];
        f32x2 stat[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const long long place = at(min(n + k, pieces - 1));
            stat[k] = a.stat[place];
            part[k] = *reinterpret_cast<const f32x4 *>(a.part + place * DT + d);
        }
        float high = most;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) high = fmaxf(high, stat[k].x);
        const float base = high == -INFINITY ? 0.0f : high, shrink = shrink_by(most - base);
        weight *= shrink;
        y *= shrink;
        most = high;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (n + k < pieces) {
                const float scale = shrink_by(stat[k].x - base);
                weight = fmaf(stat[k].y, scale, weight);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = fmaf(part[k][e], scale, y[e]);
            }
    }
    int from, to;
    visible_keys(a, own.n, own.len, i, from, to);
    const float unit = 1.0f / weight;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = to > from ? y[e] * unit : 0.0f;
    *reinterpret_cast<u32x2 *>(a.out + (long long)token * a.ld_out + (head * a.group + member) * a.head_dim + d) =
        u32x2{from_float2<BF>(y[0], y[1]), from_float2<BF>(y[2], y[3])};
}

namespace {

struct SharedPlan {
    int dim, workers, num_slots, own_slots;
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
    s.own_slots = (int)((long long)tokens * group / kChunkRows) + groups + 1;
    s.num_slots = s.own_slots + (int)((long long)tokens * group / kChunkRows) + requests + 1;
    s.space = (long long)tokens * group + (long long)kChunkRows * s.workers;
    s.slot_bytes = (size_t)s.num_slots * sizeof(Slot);
    s.part_bytes = (size_t)s.space * 2 * c.kv_heads * s.dim * sizeof(float);
    s.stat_bytes = (size_t)s.space * 2 * c.kv_heads * sizeof(f32x2);
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
    constexpr int kRows = kJoinThreads / (DT / 4);
    bcq_attend_shared_join_kernel<DT, BF><<<(unsigned)((rows + kRows - 1) / kRows * a.kv_heads), kJoinThreads, 0, s>>>(p);
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
    s.num_slots = plan.num_slots, s.own_slots = plan.own_slots, s.space = plan.space;
    const bool any = c.head_dim != plan.dim || c.page_size < 16;
    if (c.dtype == BCQ_BF16) shared_by_dim<true>(s, plan.dim, any, stream);
    else shared_by_dim<false>(s, plan.dim, any, stream);
    return hipGetLastError();
}

}  // namespace bcq
