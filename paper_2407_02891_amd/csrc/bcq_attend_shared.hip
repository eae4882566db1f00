// Attention over a paged cache where groups of requests share their first keys: those are read once for the group.
//
//   out = sum_j softmax_j(scale q . k_j) v_j = join of (sums over the shared keys) and (sums over the request's own)
//
// A row is a (new token, query head) pair.  The rows of all requests of a group are the tiles of the shared keys: bound by the matrix instructions where there are many.  The
// rows of a request are a tile of its own keys: bound by the bytes of K and V where they are few.  One launch does both, so that each runs beside the other.
//  * Tiles of up to 128 rows (bcq_attend_tile.h): their blocks of keys form a line, shared keys first.  The own keys of requests with up to 16 rows form a second line,
//    of blocks of 32, which single waves stream as the kernel for few rows (bcq_attend.hip) does, four of them independent of each other in a workgroup.
//  * A compute unit has two workgroups of a kv head.  The first has a piece of the line of tiles, the second a piece of the other; who would be through first has a piece of
//    the other's line too (cuts below).  They walk their pieces over the ends of tiles and requests and leave sums, maximum and weight of each row (place: the row, and 128 or 16
//    further for each piece, which no two share).
//  * The lengths are on the device, so a first launch lays out the lines (up to kFusedSlots tiles each workgroup does it for itself).  A last one joins what was left of a row: of its shared
//    keys and of its own.
//
// Measured, heads 64 / 8 of 128: 64 requests behind 8192 keys, 100 to 900 of their own (binary16): 48.5 us and 7.5 for the join; 256 behind 32768, 60 to 1500 of their own (bfloat16): 376, 7 for
// the line, 14 for the join, 700 TFLOP/s over all, the matrix pipes busy 42 % of the time.  Of that the shared keys by themselves take 300 (916 TFLOP/s), the own ones 141: beside each other
// they wait for the same LDS and vector pipes.  All workgroups first with tiles, then with the other line: 412 for 404, and 69 for 57 of the 64 then.  56 heads with a kv head each, 32 requests behind
// 4112: 79 and 5, 5.2 TB/s.
#include "bcq_attend_tile.h"
#include "bcq_lanes.h"

namespace bcq {

namespace {

constexpr int kLineThreads = 1024;
constexpr int kJoinThreads = 256;
constexpr int kLocalSlots = 1024;  // whose sums the first launch has in LDS
constexpr int kFusedSlots = 128;   // that each workgroup lays out for itself, without a launch before it
constexpr int kFewRows = 16, kFewKeys = 32;  // of a request whose own keys are streamed; of a block of them
constexpr bool streams(int dim) { return dim <= 128; }  // (heads of 256: the waves' blocks would be more LDS than two tiles')

// A tile and its place in its line.
struct Slot {
    int upto;         // blocks of the line of tiles up to and with it
    int few_upto;     // the same of the other line
    int row0;         // its first row in the part
    int block;        // its first block of keys
    int start, rows;  // of the part: first token; rows
    int request;      // whose row of the table of pages
    int requests;     // of a group; a request's group, or -1
    int from, to;     // keys of the part
    int n, len;       // of a request: new tokens, keys; of a group: whether each row sees all of the keys
    int piece;        // the first that has a block of it
    int pieces;       // how many have
    int part;         // whose tile: of a group's shared keys (below `groups`), of a request's own; -1: nobody's
    int few;          // whether it is of the other line
    int group_start, group_slot;  // of a request: first token and slot of its group
};

struct SharedParams {
    AttendParams a;  // (workers, part, stat too)
    const int *group_start, *shared_len;
    int groups, max_shared;
    Slot *slots;
    int *sums;                 // four numbers for each slot
    int num_slots, own_slots;  // the slots of requests' own keys begin at own_slots
    int few;                   // whether there may be requests of few rows, whose own keys are streamed
    long long space, own_place, few_place;  // rows that a kv head's sums have room for; where those of own keys' tiles begin, and of the other line
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

// A line's blocks [0, middle) are cut into w0 pieces, the others into w1 more.
struct Cut {
    int total, middle, w0, w1;
    __device__ __forceinline__ Cut(int total, int others, int most0, int most1) : total(total), middle(total - others), w0(min(most0, max(middle, 1))), w1(min(most1, max(others, 1))) {}
    // (first_block and worker_of in binary64: the products are below 2^53, and quotients of integers that small do not round to the next one.  A division of 64-bit integers takes ten
    // times as long, and a few of them one behind the other were 1 of the 5 us before a workgroup begins)
    __device__ __forceinline__ int begin(int piece) const
    {
        const bool front = piece < w0;
        return (front ? 0 : middle) + (int)((double)(front ? piece : piece - w0) * (front ? middle : total - middle) / (front ? w0 : w1));
    }
    __device__ __forceinline__ int end(int piece) const
    {
        const bool front = piece < w0;
        return (front ? 0 : middle) + (int)((double)(front ? piece + 1 : piece - w0 + 1) * (front ? middle : total - middle) / (front ? w0 : w1));
    }
    __device__ __forceinline__ int piece_of(int block) const
    {
        const bool front = block < middle;
        return (front ? 0 : w0) + (int)((((double)(front ? block : block - middle) + 1.0) * (front ? w0 : w1) - 1.0) / (front ? middle : total - middle));
    }
};

// The first half of the workgroups has the line of tiles, the second the other; what of a line the other half helps with.  A workgroup takes 2.2 us for a tile's block, beside one that
// streams or another of its kind (1.5 alone), and 0.9 for four waves' blocks of the other line; to begin with tiles costs as much as two of their blocks.
// Where nothing is streamed the second half has that much less all the same: the end of the line is requests' own keys, whose tiles begin anew every block or two.  Even pieces took 40.0 us
// for 33.5 (16 requests behind 4096 keys, heads of 256), 29.4 for 25.7 (40 query heads to a kv head); 26.0 for 27.5 with fewer blocks than that (8 behind 1500, heads of 256), and for
// chunks 402 for 408 and 785 for 780.
struct Cuts {
    Cut tiles, few;
    __device__ __forceinline__ Cuts(int half, int rest, int tiles, int few)
        : tiles(tiles, half == 0 ? tiles : tiles <= half ? 0 : max(0, (tiles - (int)(0.4f * few)) / 2 - 2 * rest), half, rest),
          few(few, few <= kTileWaves * rest ? 0 : min(max(0, (few - (int)(1.85f * tiles)) / 2), half ? few : 0), kTileWaves * rest, kTileWaves * half)
    {
    }
};

// The tiles of a part begin at this slot.
__device__ __forceinline__ int slots_before(const SharedParams &p, int v, int start)
{
    const int at = (int)((long long)start * p.a.group / kChunkRows);
    return v < p.groups ? at + v : p.own_slots + at + v - p.groups;
}

// The slots as a workgroup has them: its own in LDS (FUSED), or those that an earlier launch laid out.
template <bool FUSED>
struct SlotList {
    const Slot *at;
    int n;
    // One slot, the same for all lanes.
    __device__ __forceinline__ Slot load(int slot) const
    {
        slot = __builtin_amdgcn_readfirstlane(slot);
        Slot s;
        if constexpr (FUSED) {
            s = at[slot];
            int *const x = reinterpret_cast<int *>(&s);
#pragma unroll
            for (int i = 0; i < (int)(sizeof(Slot) / sizeof(int)); ++i) x[i] = __builtin_amdgcn_readfirstlane(x[i]);
        } else {  // by scalar loads
            typedef const __attribute__((address_space(4))) int *scalar_int;
            asm volatile("" : "+s"(slot));
            const scalar_int from = (scalar_int) reinterpret_cast<const int *>(at + slot);
            s.upto = from[0], s.few_upto = from[1], s.row0 = from[2], s.block = from[3], s.start = from[4], s.rows = from[5], s.request = from[6];
            s.requests = from[7], s.from = from[8], s.to = from[9], s.n = from[10], s.len = from[11], s.piece = from[12], s.pieces = from[13];
            s.part = from[14], s.few = from[15];
        }
        return s;
    }
    // That holds block `block` of a line: the first with upto(slot) > block (all lanes).
    template <class F>
    __device__ __forceinline__ int that_holds(int block, int lane, F upto) const
    {
        int slot = 0;
        for (int high = n - 1; slot < high;) {
            const int stride = (high - slot + 63) / 64, probe = slot + lane * stride;
            const int beyond = __popcll(__ballot(probe < high && upto(at[probe]) <= block));  // (rises, so these are the first lanes)
            if (!beyond) break;
            const int last = slot + (beyond - 1) * stride;  // not yet
            high = min(high, last + stride);
            slot = last + 1;
        }
        return __builtin_amdgcn_readfirstlane(slot);
    }
};

// What a slot of a part holds, but for what follows from the sums.
template <int DT>
__device__ __forceinline__ Slot make_slot(const SharedParams &p, int v, int slot, int &first_slot)
{
    constexpr int KB = tile_keys(DT);
    const AttendParams &a = p.a;
    Slot q = {};
    q.part = v;
    if (v < p.groups) {
        const int first = first_of_group(p, v), end = max(first_of_group(p, v + 1), first);
        q.start = start_of(p, first);
        q.rows = max(start_of(p, end) - q.start, 0) * a.group;
        q.request = min(first, a.requests - 1);
        q.requests = end - first;
        q.to = shared_keys(p, v);
        first_slot = slots_before(p, v, q.start);
        q.row0 = (slot - first_slot) * kChunkRows;
        q.n = a.window == 0;
        q.upto = (q.to + KB - 1) / KB;
        return q;
    }
    const int r = v - p.groups, c = group_of(p, r);
    const Request own = load_request(a, r);
    q.start = own.start;
    q.rows = own.todo * a.group;
    q.request = r;
    q.requests = c;
    q.to = own.len;
    q.n = own.n, q.len = own.len;
    q.few = p.few && q.rows <= kFewRows;
    if (c >= 0) {
        q.from = shared_keys(p, c);
        q.group_start = start_of(p, first_of_group(p, c));
        q.group_slot = slots_before(p, c, q.group_start);
    }
    first_slot = slots_before(p, v, q.start);
    q.row0 = (slot - first_slot) * kChunkRows;
    return q;
}

// Blocks of keys that a row of a request's tile sees.
template <int DT>
__device__ __forceinline__ void own_blocks(const SharedParams &p, Slot &q)
{
    const AttendParams &a = p.a;
    int low, high, unused;
    visible_keys(a, q.n, q.len, q.row0 / a.group, low, unused);
    visible_keys(a, q.n, q.len, (min(q.row0 + kChunkRows, q.rows) - 1) / a.group, unused, high);
    low = max(low, q.from);
    const int keys = q.few ? kFewKeys : tile_keys(DT);
    q.block = low / keys;
    (q.few ? q.few_upto : q.upto) = low < high ? (high + keys - 1) / keys - q.block : 0;
}

// Lays out the lines, all of THREADS threads: the blocks of each part's tiles, their sums, then what the slots hold.  numbers: four for each slot, its two sums, whose it is (bit 30 of a
// group's: a row of it does not see all keys), and of a group's the first key that a row of it sees.
template <int DT, int THREADS>
__device__ __forceinline__ void lay_out(const SharedParams &p, int *numbers, Slot *slots)
{
    constexpr int KB = tile_keys(DT);
    __shared__ int sums[THREADS / 64][2];
    const AttendParams &a = p.a;
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6, n = p.num_slots;
    int *const upto = numbers, *const few_upto = numbers + n, *const owner = numbers + 2 * n, *const first = numbers + 3 * n;
    for (int s = thread; s < n; s += THREADS) upto[s] = few_upto[s] = 0, owner[s] = -1, first[s] = a.window == 0 ? 0 : 0x7fffffff;
    __syncthreads();
    // The parts, a thread each; what a thread has looked up of its first one it keeps.
    const int parts = p.groups + a.requests;
    int kept_slot = 0;
    Slot kept = {};
    if (thread < parts) kept = make_slot<DT>(p, thread, 0, kept_slot);
    const auto each_part = [&](auto use) {  // use(part's slot as it would be at its first tile, that slot, where the slots of its kind end)
        for (int v = thread; v < parts; v += THREADS) {
            int slot = kept_slot;
            Slot q = kept;
            if (v != thread) q = make_slot<DT>(p, v, 0, slot);
            q.row0 = 0;
            use(q, slot, v < p.groups ? p.own_slots : n);
        }
    };
    each_part([&](Slot q, int s, int end) {
        for (; q.row0 < q.rows && s < end; q.row0 += kChunkRows, ++s) {
            if (q.part >= p.groups) own_blocks<DT>(p, q);
            upto[s] = q.upto, few_upto[s] = q.few_upto, owner[s] = q.part;
        }
    });
    __syncthreads();
    each_part([&](const Slot &q, int, int) {  // does each row of a request see all that is shared?  From where on, with a window?
        if (q.part < p.groups || q.requests < 0 || q.n == 0) return;
        int low, high;
        visible_keys(a, q.n, q.len, 0, low, high);
        const bool all = high >= q.from && q.rows == q.n * a.group;
        if (all && a.window == 0) return;
        const int begin = start_of(p, first_of_group(p, q.requests)), rows = max(start_of(p, first_of_group(p, q.requests + 1)) - begin, 0) * a.group;
        const int s = slots_before(p, q.requests, begin), row = (q.start - begin) * a.group;
        for (int i = 0; i * kChunkRows < rows && s + i < p.own_slots; ++i) {
            if (!all) atomicOr(owner + s + i, 1 << 30);
            if (row < (i + 1) * kChunkRows && row + q.rows > i * kChunkRows) atomicMin(first + s + i, low);
        }
    });
    __syncthreads();
    for (int s = thread; s < p.own_slots; s += THREADS)  // blocks in front of the first key that is seen
        if (upto[s] > 0) upto[s] = first[s] < KB * upto[s] ? upto[s] - first[s] / KB : 0;
    __syncthreads();
    int before = 0, few_before = 0;
    for (int c = 0; c < n; c += THREADS) {
        const int s = c + thread;
        const int tiles = sum_upto(s < n ? upto[s] : 0, lane), few = sum_upto(s < n ? few_upto[s] : 0, lane);
        if (lane == 63) sums[wave][0] = tiles, sums[wave][1] = few;
        __syncthreads();
        int mine = before + tiles, few_mine = few_before + few;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) mine += sums[w][0], few_mine += sums[w][1];
            before += sums[w][0], few_before += sums[w][1];
        }
        if (s < n) upto[s] = mine, few_upto[s] = few_mine;
        __syncthreads();
    }
    const Cuts cuts(a.workers / 2, a.workers - a.workers / 2, before, few_before);
    for (int s = thread; s < n; s += THREADS) {
        Slot q = {};
        q.part = -1;
        if (owner[s] >= 0) {
            int unused;
            q = make_slot<DT>(p, owner[s] & ~(1 << 30), s, unused);
            if (q.part >= p.groups) own_blocks<DT>(p, q);
            else q.block = min(first[s], q.to) / KB;
            if (owner[s] >> 30) q.n = 0;
        }
        q.upto = upto[s], q.few_upto = few_upto[s];
        const int to = q.few ? q.few_upto : q.upto, from = s == 0 ? 0 : q.few ? few_upto[s - 1] : upto[s - 1];
        if (to > from) {
            const Cut cut = q.few ? cuts.few : cuts.tiles;
            q.piece = cut.piece_of(from);
            q.pieces = cut.piece_of(to - 1) - q.piece + 1;
        }
        slots[s] = q;
    }
    __syncthreads();
}

}  // namespace

template <int DT>
__global__ __launch_bounds__(kLineThreads) void bcq_attend_shared_line_kernel(SharedParams p)
{
    __shared__ int local[4 * kLocalSlots];
    lay_out<DT, kLineThreads>(p, p.num_slots <= kLocalSlots ? local : p.sums, p.slots);
}

namespace {

template <bool BF>
using FewWeights = Weights<BF, 1>;

// One wave: blocks [at, stop) of the line of requests with few rows, a piece of it; ks: LDS, 2 * kFewKeys * DT elements of the wave's own.  Column r16 of the products is token r16 / group, query
// head r16 mod group.  K and V come in whole rows and pass through LDS, the next block's are on their way; weights meet the values as the sum of two 16-bit numbers.
template <int DT, bool BF, bool ANY, bool PASSING, bool FUSED>
__device__ __forceinline__ void stream_piece(const SharedParams &p, const SlotList<FUSED> &slots, int head, int piece, int at, int stop, uint16_t *const ks)
{
    constexpr int C = DT / 32, DV = DT / 16;                    // matrix steps over head_dim; tiles of O
    constexpr int kRowLanes = DT / 8, kRows = 64 / kRowLanes;   // a load covers kRows keys
    const AttendParams &a = p.a;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // (what follows from it is not worth registers beside the tiles)
    const int r16 = lane & 15, g = lane >> 4;
    uint16_t *const vs = ks + kFewKeys * DT;
    // element d of key j in LDS: units of a row (8 elements of K, 16 of V) exchanged by the key, so that the units of one number fill all banks
    const auto k_at = [&](int key, int d) { return ks + key * DT + ((d >> 3 ^ (DT == 64 ? key >> 1 & 7 : key & 15)) << 3); };
    const auto v_at = [&](int key, int d) {
        const int turn = DT == 64 ? key >> 1 & 3 : key & 7;
        return vs + key * DT + ((d >> 4 ^ turn) << 4) + (d & 15);
    };
    const int token = r16 / a.group, member = r16 - token * a.group;
    // where the block is that is computed, the one that is on its way, the one whose pages are looked up
    struct Place {
        Slot s;
        int key;
    };
    int slot = slots.that_holds(at, lane, [](const Slot &s) { return s.few_upto; });
    int before = slot ? slots.load(slot - 1).few_upto : 0;
    Place now, next, ahead;
    ahead.s = slots.load(slot);
    const auto look_at = [&](int block) {
        while (block >= ahead.s.few_upto) before = ahead.s.few_upto, ahead.s = slots.load(++slot);
        ahead.key = (ahead.s.block + block - before) * kFewKeys;
    };
    look_at(at);
    const int in_rows = lane / kRowLanes, d_own = 8 * (lane % kRowLanes);
    const long long head_offset = head * a.head_stride;
    int dim = a.head_dim;
    u32x4 kr[2][C], vr[2][C];
    int id[2];  // page numbers of the block that is requested next
    const auto find_pages = [&](const Place &b) {
        if (ANY) return;
#pragma unroll
        for (int t = 0; t < 2; ++t) id[t] = page_of_all(a, b.s.request, min(b.key + 16 * t, max(b.s.len - 1, 0) & ~15));
    };
    const auto request = [&](const Place &b) {
        const Slot &s = b.s;
        const int last = max(s.len - 1, 0);
        if (ANY) asm volatile("" : "+v"(dim));  // (compared here, not held as masks through the loop)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = min(b.key + 16 * t, last & ~15);  // keys behind the last are the last's copies, and masked
            if (!ANY) {
                const long long base = __builtin_amdgcn_readfirstlane(id[t]) * a.page_stride + head_offset + (long long)((key & ((1 << a.page_shift) - 1)) * a.slot_stride);
                const char *const kp = reinterpret_cast<const char *>(a.k + base), *const vp = reinterpret_cast<const char *>(a.v + base);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const unsigned off = 2 * (unsigned)(min(c * kRows + in_rows, last - key) * a.slot_stride + d_own);
                    const u32x4 *const ka = reinterpret_cast<const u32x4 *>(kp + off), *const va = reinterpret_cast<const u32x4 *>(vp + off);
                    if (PASSING) kr[t][c] = __builtin_nontemporal_load(ka), vr[t][c] = __builtin_nontemporal_load(va);
                    else kr[t][c] = *ka, vr[t][c] = *va;
                }
            } else {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int j = min(key + c * kRows + in_rows, last);
                    const long long place = page_of(a, s.request, j) * a.page_stride + head_offset + (long long)((j & ((1 << a.page_shift) - 1)) * a.slot_stride);
                    kr[t][c] = *reinterpret_cast<const u32x4 *>(d_own < dim ? a.k + place + d_own : g_zeros);
                    vr[t][c] = *reinterpret_cast<const u32x4 *>(d_own < dim ? a.v + place + d_own : g_zeros);
                }
            }
        }
    };
    find_pages(ahead);
    request(ahead);
    now = next = ahead;
    if (at + 1 < stop) {
        look_at(at + 1);
        find_pages(ahead);
    }
    u32x4 q[C];
    f32x4 o[DV];
    float most, base, sum;
    int from, to;          // keys that the row sees
    int all_from, all_to;  // keys that every row sees
    const auto begin_request = [&](const Slot &s) {
        int unused;
        visible_keys(a, s.n, s.len, 0, unused, all_to);
        visible_keys(a, s.n, s.len, s.rows / a.group - 1, all_from, unused);
        visible_keys(a, s.n, s.len, token, from, to);
        all_from = max(all_from, s.from), from = max(from, s.from);
        most = -INFINITY;
        base = sum = 0.0f;
#pragma unroll
        for (int d = 0; d < DV; ++d) o[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const bool real = r16 < s.rows;
        const uint16_t *const src = a.q + (long long)(s.start + (real ? token : 0)) * a.ld_q + (head * a.group + member) * a.head_dim;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            q[c] = u32x4{0, 0, 0, 0};
            if (real && (!ANY || 32 * c + 8 * g < dim)) q[c] = *reinterpret_cast<const u32x4 *>(src + 32 * c + 8 * g);
        }
    };
    begin_request(now.s);
#pragma unroll 1
    for (;;) {
        const int key0 = now.key;
        const bool masked = key0 + kFewKeys > all_to || key0 < all_from;
        // Infinities or NaN among the values: zero times them must not reach the rows that do not see them, nor must the second number of a weight, which may be zero or
        // negative, or a weight too small for its type, make a NaN of an infinity.  They are replaced by zeros, and what they make of the rows that do see them is found by products of ones.
        float zero = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) zero = times_zero<BF>(vr[t][c][i], zero);
        const bool odd = __ballot(zero != 0.0f) != 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                *reinterpret_cast<u32x4 *>(k_at(16 * t + c * kRows + in_rows, d_own)) = kr[t][c];
                *reinterpret_cast<u32x4 *>(v_at(16 * t + c * kRows + in_rows, d_own)) = vr[t][c];
            }
        ++at;
        const bool through = at == now.s.few_upto || at == stop;  // with this request, or this piece of it
        if (at < stop) {
            request(ahead);
            next = ahead;
            if (at + 1 < stop) {
                look_at(at + 1);
                find_pages(ahead);
            }
        }
        f32x4 s[2];
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c) s[t] = mfma16<BF>(*reinterpret_cast<const u32x4 *>(k_at(16 * t + r16, 32 * c + 8 * g)), q[c], s[t]);
        }
        // weights: number 4 t + i of a lane is key 16 t + 4 g + i
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * a.scale;
        if (masked) {
            const unsigned span = max(to - from, 0);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (unsigned)(key0 + 16 * (e >> 2) + 4 * g + (e & 3) - from) < span ? x[e] : -INFINITY;
        }
        float high = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) high = fmaxf(high, x[e]);
        if (__ballot(high > most + FewWeights<BF>::grow)) {
            const float m = fmaxf(most, max_over_groups(high));
            const float shrink = most == -INFINITY ? 1.0f : shrink_by(most - m);
            most = m;
            base = m == -INFINITY ? 0.0f : m - FewWeights<BF>::lift;
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < DV; ++d) o[d] *= shrink;
        }
        u32x4 high_part, low_part;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float w0 = exp2_fast(x[e] - base), w1 = exp2_fast(x[e + 1] - base);
            sum += w0 + w1;
            const uint32_t pair = from_float2<BF>(w0, w1);
            const f32x2 kept = to_float2<BF>(pair);
            high_part[e / 2] = pair;
            low_part[e / 2] = from_float2<BF>(w0 - kept.x, w1 - kept.y);
        }
        asm volatile("" ::: "memory");
        const auto column = [&](int d) {  // the operand V^T: elements 16 d + r16 of keys 4 g .. and 16 + 4 g ..
            const u32x2 v0 = lds_column(v_at(lane >> 2, 16 * d + 4 * (lane & 3))), v1 = lds_column(v_at(16 + (lane >> 2), 16 * d + 4 * (lane & 3)));
            return u32x4{v0.x, v0.y, v1.x, v1.y};
        };
        if (odd) {
            u32x4 sees;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = key0 + 16 * (e >> 1) + 4 * g + 2 * (e & 1);
                sees[e] = (key >= from && key < to ? kOne<BF> : 0u) | (key + 1 >= from && key + 1 < to ? kOne<BF> << 16 : 0u);
            }
#pragma unroll
            for (int d = 0; d < DV; ++d) {
                const u32x4 v = column(d);
                u32x4 up, down;
#pragma unroll
                for (int e = 0; e < 4; ++e) up[e] = ones_where_infinite<BF>(v[e], 0), down[e] = ones_where_infinite<BF>(v[e], 0x8000u);
                const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
                const f32x4 ups = mfma16<BF>(up, sees, none), downs = mfma16<BF>(down, sees, none);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[d][i] += (ups[i] > 0.0f ? INFINITY : 0.0f) - (downs[i] > 0.0f ? INFINITY : 0.0f);
                __builtin_amdgcn_sched_barrier(0);  // (rare: registers count, not time)
            }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    u32x4 *const mine = reinterpret_cast<u32x4 *>(v_at(16 * t + c * kRows + in_rows, d_own));
                    u32x4 v = *mine;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = finite_only<BF>(v[i]);
                    *mine = v;
                }
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int d = 0; d < DV; ++d) {
            const u32x4 v = column(d);
            o[d] = mfma16<BF>(v, low_part, mfma16<BF>(v, high_part, o[d]));
        }
        asm volatile("" ::: "memory");
        if (!through) {
            now.key = next.key;
            continue;
        }
        const float weight = sum_over_groups(sum);
        if (r16 < now.s.rows) {
            const long long place = head * p.space + p.few_place + (long long)now.s.start * a.group + r16 + (long long)kFewRows * piece;
#pragma unroll
            for (int d = 0; d < DV; ++d) *reinterpret_cast<f32x4 *>(a.part + place * DT + 16 * d + 4 * g) = o[d];
            // (the tiles' weights are less: what both leave is relative to the maximum less the tiles' lift)
            if (g == 0) a.stat[place] = f32x2{most - (FewWeights<BF>::lift - TileWeights<BF>::lift), weight};
        }
        if (at == stop) return;
        now = next;
        begin_request(now.s);
    }
}

}  // namespace

// The pieces of both lines.  PASSING: what is streamed leaves nothing in the caches.  FUSED: there was no launch before this one.
template <int DT, bool BF, bool ANY, bool PASSING, bool FUSED>
__global__ __launch_bounds__(64 * kTileWaves, tile_occupancy(DT)) void bcq_attend_shared_kernel(SharedParams p)
{
    constexpr int KB = tile_keys(DT), DV = DT / 32;
    __shared__ __attribute__((aligned(1024))) uint16_t k0[KB * DT], k1[KB * DT], v0[KB * DT], v1[KB * DT];
    static_assert(!streams(DT) || KB * DT >= 2 * kFewKeys * DT, "");
    __shared__ int bounds[kTileWaves][2];
    const AttendParams &a = p.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % a.kv_heads, me = blockIdx.x / a.kv_heads, half = a.workers / 2;
    const bool first_half = me < half;
    SlotList<FUSED> slots{p.slots, p.num_slots};
    if constexpr (FUSED) {
        __shared__ Slot own[kFusedSlots];
        lay_out<DT, 64 * kTileWaves>(p, reinterpret_cast<int *>(k0), own);  // (which is not in use yet)
        slots.at = own;
        if (blockIdx.x == 0)  // for the join
            for (int i = threadIdx.x; i < p.num_slots; i += 64 * kTileWaves) p.slots[i] = own[i];
    }
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
        const Slot end_slot = slots.load(p.num_slots - 1);  // (again in each turn: not worth registers)
        const Cuts cuts(half, a.workers - half, end_slot.upto, end_slot.few_upto);
        if ((turn == 0) != first_half) {
            if constexpr (streams(DT)) {
                const int mine = kTileWaves * (first_half ? me : me - half) + wave;
                if (mine < (first_half ? cuts.few.w1 : cuts.few.w0)) {
                    const int piece = first_half ? cuts.few.w0 + mine : mine, at = cuts.few.begin(piece), stop = cuts.few.end(piece);
                    if (at < stop) stream_piece<DT, BF, ANY, PASSING, FUSED>(p, slots, head, piece, at, stop, wave == 0 ? k0 : wave == 1 ? k1 : wave == 2 ? v0 : v1);
                }
                __syncthreads();  // (the tiles' buffers)
            }
            continue;
        }
        const int mine = first_half ? me : me - half, piece = first_half ? mine : cuts.tiles.w0 + mine;
        if (mine >= (first_half ? cuts.tiles.w0 : cuts.tiles.w1)) continue;
        int at = __builtin_amdgcn_readfirstlane(cuts.tiles.begin(piece));
        const int stop = __builtin_amdgcn_readfirstlane(cuts.tiles.end(piece));
        if (at >= stop) continue;
        int slot = slots.that_holds(at, threadIdx.x & 63, [](const Slot &s) { return s.upto; });
        int before = slot ? slots.load(slot - 1).upto : 0;
#pragma unroll 1
        for (; at < stop; ++slot) {
            const Slot s = slots.load(slot);
            const int end = min(s.upto, stop);
            if (end <= at) {  // (a slot without blocks)
                before = s.upto;
                continue;
            }
            const bool of_group = s.part < p.groups;
            // ---- the lane's row, and what it sees ----
            int lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));  // (the same beside what is streamed)
            const int r32 = lane & 31, h = lane >> 5;
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
            __builtin_amdgcn_s_setprio(2);  // (beside a workgroup that streams: 256 requests behind 32768 keys 380 us, 404 without)
            const bool reading = attend_tile<DT, BF, ANY, false>(a, t, k0, k1, v0, v1, o, most, sum);

            const auto twin = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, sum), __builtin_bit_cast(unsigned, sum), false, false);
            sum = __builtin_bit_cast(float, (unsigned)twin[0]) + __builtin_bit_cast(float, (unsigned)twin[1]);
            if (real) {
                const long long place = head * p.space + (of_group ? 0 : p.own_place) + (long long)s.start * a.group + row + (long long)kChunkRows * piece;
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
        __builtin_amdgcn_s_setprio(0);
        __syncthreads();  // (before the waves' own blocks take the tiles' buffers)
    }
}

// Joins what was left of a row, its shared keys' pieces and its own: four elements to a thread, SHARE threads to share the pieces of them.
template <int DT, bool BF, int SHARE>
__global__ __launch_bounds__(kJoinThreads) void bcq_attend_shared_join_kernel(SharedParams p)
{
    constexpr int kLanes = DT / 4, kAhead = SHARE > 1 ? 4 : 8, kOwn = kJoinThreads / SHARE;
    __shared__ f32x4 shared_y[SHARE > 1 ? kJoinThreads : 1];
    __shared__ f32x2 shared_stat[SHARE > 1 ? kJoinThreads : 1];
    const AttendParams &a = p.a;
    const int share = threadIdx.x / kOwn, thread = threadIdx.x % kOwn;
    const int head = blockIdx.x % a.kv_heads, row = min(blockIdx.x / a.kv_heads * (kOwn / kLanes) + thread / kLanes, a.tokens * a.group - 1), d = 4 * (thread % kLanes);
    const bool twice = blockIdx.x / a.kv_heads * (kOwn / kLanes) + thread / kLanes >= a.tokens * a.group;  // (the last row again)
    const int token = row / a.group, member = row - token * a.group;
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
    const bool real = !twice && i >= 0 && i < own.todo && d < a.head_dim;
    const int s1 = slots_before(p, p.groups + r, own.start) + max(i * a.group + member, 0) / kChunkRows;
    const Slot &mine = p.slots[min(s1, p.num_slots - 1)];
    const int c = mine.requests;
    int pieces0 = 0, pieces = mine.pieces;
    const int step1 = mine.few ? kFewRows : kChunkRows;
    const long long place1 = head * p.space + (mine.few ? p.few_place : p.own_place) + (long long)token * a.group + member + (long long)step1 * mine.piece;
    long long place0 = 0;
    if (c >= 0) {
        const Slot &shared = p.slots[min(mine.group_slot + max((token - mine.group_start) * a.group + member, 0) / kChunkRows, p.own_slots - 1)];
        pieces0 = shared.pieces;
        place0 = head * p.space + (long long)token * a.group + member + (long long)kChunkRows * shared.piece;
    }
    pieces = real ? pieces + pieces0 : 0;
    const auto at = [&](int n) { return n < pieces0 ? place0 + (long long)n * kChunkRows : place1 + (long long)(n - pieces0) * step1; };
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
    float most = -INFINITY, weight = 0.0f;
    for (int n = share; n < pieces; n += kAhead * SHARE) {
        f32x4 part[kAhead];
        f32x2 stat[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const long long place = at(min(n + k * SHARE, pieces - 1));
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
            if (n + k * SHARE < pieces) {
                const float scale = shrink_by(stat[k].x - base);
                weight = fmaf(stat[k].y, scale, weight);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = fmaf(part[k][e], scale, y[e]);
            }
    }
    if constexpr (SHARE > 1) {
        shared_y[threadIdx.x] = y;
        shared_stat[threadIdx.x] = f32x2{most, weight};
        __syncthreads();
        if (share) return;
#pragma unroll
        for (int k = 1; k < SHARE; ++k) most = fmaxf(most, shared_stat[k * kOwn + thread].x);
        const float base = most == -INFINITY ? 0.0f : most;
        y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        weight = 0.0f;
#pragma unroll
        for (int k = 0; k < SHARE; ++k) {
            const f32x2 stat = shared_stat[k * kOwn + thread];
            const float scale = shrink_by(stat.x - base);
            weight = fmaf(stat.y, scale, weight);
            y += shared_y[k * kOwn + thread] * scale;
        }
    }
    if (!real) return;
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
    int dim, workers, num_slots, own_slots, few;
    long long space, own_place, few_place;
    size_t slot_bytes, part_bytes, stat_bytes;
};
SharedPlan shared_plan(const bcq_cache &c, int tokens, int requests, int groups, int q_heads, int max_new)
{
    SharedPlan s;
    s.dim = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
    const int group = q_heads / c.kv_heads;
    const int per_head = compute_units() * tile_occupancy(s.dim) / c.kv_heads;  // as many workgroups as the chip holds
    s.workers = per_head > 1 ? per_head : 1;
    s.own_slots = (int)((long long)tokens * group / kChunkRows) + groups + 1;
    s.num_slots = s.own_slots + (int)((long long)tokens * group / kChunkRows) + requests + 1;
    // rows of the shared tiles, of own keys' tiles where a request may have them, of the other line where it may
    const long long rows = (long long)tokens * group, tiles = rows + (long long)kChunkRows * s.workers;
    s.few = streams(s.dim) && group <= kFewRows;
    s.own_place = tiles;
    s.few_place = s.own_place + (s.few && (long long)max_new * group <= kFewRows ? 0 : tiles);
    s.space = s.few_place + (s.few ? rows + (long long)kFewRows * kTileWaves * s.workers : 0);
    s.slot_bytes = (size_t)s.num_slots * (sizeof(Slot) + 4 * sizeof(int));
    s.slot_bytes = (s.slot_bytes + 15) / 16 * 16;
    s.part_bytes = (size_t)s.space * c.kv_heads * s.dim * sizeof(float);
    s.stat_bytes = (size_t)s.space * c.kv_heads * sizeof(f32x2);
    return s;
}

template <int DT, bool BF, bool FUSED>
void shared_main(const SharedParams &p, bool any, bool passing, hipStream_t s)
{
    const unsigned groups = (unsigned)p.a.workers * p.a.kv_heads;
    if (any) bcq_attend_shared_kernel<DT, BF, true, false, FUSED><<<groups, 64 * kTileWaves, 0, s>>>(p);
    else if (passing && streams(DT)) bcq_attend_shared_kernel<DT, BF, false, streams(DT), FUSED><<<groups, 64 * kTileWaves, 0, s>>>(p);
    else bcq_attend_shared_kernel<DT, BF, false, false, FUSED><<<groups, 64 * kTileWaves, 0, s>>>(p);
}

template <int DT, bool BF>
void shared_launches(const SharedParams &p, bool any, bool passing, hipStream_t s)
{
    const AttendParams &a = p.a;
    if (p.num_slots <= kFusedSlots) {
        shared_main<DT, BF, true>(p, any, passing, s);
    } else {
        bcq_attend_shared_line_kernel<DT><<<1, kLineThreads, 0, s>>>(p);
        shared_main<DT, BF, false>(p, any, passing, s);
    }
    const long long rows = (long long)a.tokens * a.group;
    constexpr int kRows = kJoinThreads / (DT / 4);
    // (with fewer rows than the chip has room for threads, latency counts: calls of 4 requests 17.0 us with one
    // thread to a row's four elements, 15.0 with four; of 5 with drafts 41.8 and 38.1)
    if (rows * a.kv_heads < (long long)kRows * 8 * compute_units())
        bcq_attend_shared_join_kernel<DT, BF, 4><<<(unsigned)((4 * rows + kRows - 1) / kRows * a.kv_heads), kJoinThreads, 0, s>>>(p);
    else
        bcq_attend_shared_join_kernel<DT, BF, 1><<<(unsigned)((rows + kRows - 1) / kRows * a.kv_heads), kJoinThreads, 0, s>>>(p);
}

template <bool BF>
void shared_by_dim(const SharedParams &p, int dim, bool any, bool passing, hipStream_t s)
{
    if (dim == 64) shared_launches<64, BF>(p, any, passing, s);
    else if (dim == 128) shared_launches<128, BF>(p, any, passing, s);
    else shared_launches<256, BF>(p, any, passing, s);
}

}  // namespace

size_t attend_shared_workspace_bytes(const bcq_cache &c, int tokens, int requests, int groups, int q_heads, int max_new)
{
    const SharedPlan s = shared_plan(c, tokens, requests, groups, q_heads, max_new);
    return s.part_bytes + s.stat_bytes + s.slot_bytes;
}

hipError_t launch_attend_shared(const AttendSharedArgs &args, hipStream_t stream)
{
    const AttendArgs &a = args.of;
    const bcq_cache &c = a.cache;
    const SharedPlan plan = shared_plan(c, a.tokens, a.requests, args.groups, a.q_heads, a.max_new);
    char *const ws = static_cast<char *>(a.workspace);
    SharedParams s = {};
    AttendParams &p = s.a;
    p.k = a.k, p.v = a.v, p.q = a.q, p.q_start = a.q_start, p.kv_len = a.kv_len, p.pages = a.pages, p.out = a.out;
    p.part = reinterpret_cast<float *>(ws);
    s.slots = reinterpret_cast<Slot *>(ws + plan.part_bytes);
    s.sums = reinterpret_cast<int *>(s.slots + plan.num_slots);
    p.stat = reinterpret_cast<f32x2 *>(ws + plan.part_bytes + plan.slot_bytes);
    p.ld_q = a.ld_q, p.ld_out = a.ld_out, p.page_stride = c.page_stride, p.head_stride = c.head_stride, p.slot_stride = (int)c.slot_stride;
    p.tokens = a.tokens, p.requests = a.requests, p.kv_heads = c.kv_heads, p.group = a.q_heads / c.kv_heads;
    p.head_dim = c.head_dim, p.page_shift = __builtin_ctz(c.page_size), p.num_pages = c.num_pages, p.max_pages = a.max_pages;
    p.max_new = a.max_new, p.causal = a.causal;
    p.window = a.window > 1 << 30 ? 0 : a.window;  // (no request has so many keys, and positions less a window stay in range)
    p.scale = (float)(a.scale * 1.4426950408889634);
    p.workers = plan.workers;
    s.group_start = args.group_start, s.shared_len = args.shared_len, s.groups = args.groups, s.max_shared = args.max_shared;
    s.num_slots = plan.num_slots, s.own_slots = plan.own_slots, s.few = plan.few;
    s.space = plan.space, s.own_place = plan.own_place, s.few_place = plan.few_place;
    const bool any = c.head_dim != plan.dim || c.page_size < 16;
    const bool passing = 4 * (long long)c.num_pages * c.page_stride >= kPassingBytes;
    if (c.dtype == BCQ_BF16) shared_by_dim<true>(s, plan.dim, any, passing, stream);
    else shared_by_dim<false>(s, plan.dim, any, passing, stream);
    return hipGetLastError();
}

}  // namespace bcq
