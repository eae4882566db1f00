// Attention of a few new tokens per request over a paged cache: what serving does at every step.
//
//   out = sum_j softmax_j(scale q . k_j) v_j
//
// Bound by the bytes of K and V.  A row is a (new token, query head) pair; the rows that share a kv head are the columns of a matrix
// instruction, so a key is read once for all of them.
//  * The blocks of 32 keys of all requests form one line, which is cut into as many equal pieces as there are waves for a kv head
//    (from the lengths on the device: the host does not see them).  A wave walks its piece, over the ends of requests, and leaves for each
//    request sums, maximum and weight (slot wave + request, which no two share); a request that one wave has to itself is finished there, and
//    what a workgroup's waves have of one request is one piece (one request of 32768 keys: 30.5 us, 39.7 if every wave leaves its own).
//    A second launch joins the others.  Short requests take one launch instead, in which a workgroup has a request and kv head (one_launch below).
//  * K and V come from memory in whole rows (a load in the operand's layout touches sixteen rows for 64 bytes of each) and pass through LDS (the wave's own, no
//    barrier): K's pieces are read as the operand's, V through the transposing read, which gives four keys of one element.
//  * S^T = K Q^T: a lane gets four keys' scores of one row, and the same lane group's weights are the operand of O^T = V^T P^T as they
//    are, because the keys of a product may be numbered in any order.
//  * The next block's K and V are requested when this one's have gone to LDS, and its page numbers a block earlier: 16 KB a wave are on their way.
//  * Weights are taken relative to a running maximum (Weights in bcq_attend.h).  They enter the second product as the sum of two 16-bit numbers: it costs a matrix
//    instruction more, and those wait for memory.  bfloat16: 16 bits.  binary16: 22 bits of a weight down to 2^-17 of the largest, fewer below, 11 at 2^-28.
//
// Measured: 64 requests of 200 to 8000 keys, 64 / 8 heads of 128 (1.05 GB): 165 us and 8 for the join, 6.3 TB/s; with the loads alone, the arithmetic taken out, it
// took no less, so what is left to the 7.2 TB/s of a plain read is the start (lengths, pages, the first keys: three reads in a row) and the end.
// A first kernel without matrix instructions took 2278 us, K in the operand's layout and kept in the caches 201, one workgroup more than fits 24 us more.
#include "bcq_attend.h"

namespace bcq {

namespace {

constexpr int kBlock = 32;  // keys of a step
constexpr int kWaves = 4;
constexpr int kStreamRows = 16;
template <bool BF>
using StreamWeights = Weights<BF, 1>;  // (renewing costs nothing where memory is waited for)
constexpr int kMostRows = 128;  // of a tile of either kernel

// Waves per SIMD: what the registers allow.
constexpr int stream_occupancy(int dim, bool any) { return dim == 64 ? 3 : dim == 128 ? 2 : 1; }

// Waves of a workgroup that has a request and kv head to itself, where there are fewer of them than compute units: what LDS holds a block for.
constexpr int most_waves(int dim) { return 1024 / dim; }

// Blocks of a request in the line; a request whose rows see nothing has one, which writes its zeros.
__device__ __forceinline__ int blocks_of(const AttendParams &p, const Request &q)
{
    if (q.todo == 0 || q.todo * p.group > p.rows) return 0;
    return max(1, (q.end + kBlock - 1) / kBlock - q.begin / kBlock);
}

// Sixty-four requests, one a lane, with the blocks up to and with each of them.
struct Window {
    Request q;
    int blocks, upto;
    __device__ __forceinline__ void load(const AttendParams &p, int first, int before, int lane)
    {
        const int r = first + lane;
        q = load_request(p, min(r, p.requests - 1));
        blocks = r < p.requests ? blocks_of(p, q) : 0;
        upto = before + prefix_sum(blocks, lane);
    }
};

__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// Waves that share the line: no more than it has blocks.
__device__ __forceinline__ int workers_of(const AttendParams &p, int total) { return min(p.workers, max(total, 1)); }

// A wave's share of one request.
struct Segment {
    int r, start, n, todo, len;
    int key, blocks;   // first key (of a block), blocks
    bool whole;        // all of the request
    int from, upto;    // the request's blocks in the line
};

}  // namespace

// DT: head_dim, or what it is padded to.  ANY: head_dim < DT, or pages of fewer than 16 slots.  PASSING: K and V leave nothing in the caches.
// OWN: 0, or the waves of a workgroup that has a request and kv head to itself; they share its blocks and join their sums.
template <int DT, bool BF, bool ANY, bool PASSING, int OWN>
__global__ __launch_bounds__(64 * (OWN ? OWN : kWaves), OWN ? most_waves(DT) / 4 : stream_occupancy(DT, ANY)) void bcq_attend_stream_kernel(
    AttendParams p)
{
    constexpr bool DIRECT = OWN > 0;
    constexpr int W = DIRECT ? OWN : kWaves;
    constexpr int C = DT / 32, DV = DT / 16;     // matrix steps over head_dim; tiles of O
    constexpr int kRowLanes = DT / 8, kRows = 64 / kRowLanes;  // a load covers kRows keys
    __shared__ __attribute__((aligned(16))) uint16_t lds[W][2 * kBlock * DT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int head = blockIdx.x % p.kv_heads, first_worker = blockIdx.x / p.kv_heads * W, worker = first_worker + wave;
    int first_head = head * p.group;  // (of q)
    if (ANY) asm("" : "+v"(first_head));
    uint16_t *const ks = lds[wave], *const vs = ks + kBlock * DT;
    // element d of key j in LDS: units of a row (8 elements of K, 16 of V) exchanged by the key, so that the units of one number fill all banks
    const auto k_at = [&](int key, int d) { return ks + key * DT + ((d >> 3 ^ (DT == 64 ? key >> 1 & 7 : key & 15)) << 3); };
    const auto v_at = [&](int key, int d) {
        const int turn = DT == 64 ? key >> 1 & 3 : key & 7;
        return vs + key * DT + ((d >> 4 ^ turn) << 4) + (d & 15);
    };

    // ---- this wave's piece of the line, or of the request ----
    Window w;
    Segment now;
    int total = 0, first = 0, workers = 0, at, stop;
    if (DIRECT) {
        const int r = blockIdx.x / p.kv_heads;
        const Request own = load_request(p, r);
        total = blocks_of(p, own);
        if (total == 0) return;
        at = total * wave / W, stop = total * (wave + 1) / W;
        now = Segment{r, own.start, own.n, own.todo, own.len, (own.begin / kBlock + at) * kBlock, stop - at, false, 0, 0};
    } else {
        for (int c = 0; c < p.requests; c += 64) {
            w.load(p, c, total, lane);
            total = lane_of(w.upto, 63);
        }
        workers = workers_of(p, total);
        if (worker >= workers || total == 0) return;
        at = first_block(worker, workers, total);
        stop = first_block(worker + 1, workers, total);
        if (p.requests > 64) w.load(p, 0, 0, lane);
    }
    const auto segment_at = [&](int place) {
        while (lane_of(w.upto, 63) <= place) w.load(p, first += 64, lane_of(w.upto, 63), lane);
        const int l = __builtin_ctzll(__ballot(w.upto > place));
        const int upto = lane_of(w.upto, l), from = upto - lane_of(w.blocks, l);
        Segment e;
        e.r = first + l;
        e.start = lane_of(w.q.start, l);
        e.n = lane_of(w.q.n, l);
        e.todo = lane_of(w.q.todo, l);
        e.len = lane_of(w.q.len, l);
        e.key = (lane_of(w.q.begin, l) / kBlock + place - from) * kBlock;
        e.blocks = min(upto, stop) - place;
        e.whole = from == place && upto <= stop;
        e.from = from;
        e.upto = upto;
        return e;
    };

    // ---- requests to memory: whole rows, kRows of them at a time ----
    const int in_rows = lane / kRowLanes, d_own = 8 * (lane % kRowLanes);
    u32x4 kr[2][C], vr[2][C];
    long long page_stride = p.page_stride, head_offset = head * p.head_stride;
    int slot_stride = p.slot_stride, last_page = p.num_pages - 1;
    if (ANY) asm("" : "+v"(page_stride), "+v"(head_offset), "+v"(slot_stride), "+v"(last_page));  // (scalar registers are scarce there)
    int dim = p.head_dim;
    if (ANY) asm("" : "+v"(dim));
    int id[2];  // page numbers of the block that is requested next
    const auto find_pages = [&](int r, int len, int first_key) {
        if (ANY) return;
#pragma unroll
        for (int t = 0; t < 2; ++t) id[t] = page_of_all(p, r, min(first_key + 16 * t, max(len - 1, 0) & ~15));
    };
    const auto request = [&](int r, int len, int first_key) {
        const int last = max(len - 1, 0);
        if (ANY) asm volatile("" : "+v"(dim));  // (compared here, not held as masks through the loop)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = min(first_key + 16 * t, last & ~15);  // keys behind the last are the last's copies, and masked
            if (!ANY) {
                const long long base = __builtin_amdgcn_readfirstlane(id[t]) * page_stride + head_offset +
                                       (long long)((key & ((1 << p.page_shift) - 1)) * p.slot_stride);
                const char *const kp = reinterpret_cast<const char *>(p.k + base), *const vp = reinterpret_cast<const char *>(p.v + base);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const unsigned off = 2 * (unsigned)(min(c * kRows + in_rows, last - key) * p.slot_stride + d_own);
                    const u32x4 *const ka = reinterpret_cast<const u32x4 *>(kp + off), *const va = reinterpret_cast<const u32x4 *>(vp + off);
                    if (PASSING) kr[t][c] = __builtin_nontemporal_load(ka), vr[t][c] = __builtin_nontemporal_load(va);
                    else kr[t][c] = *ka, vr[t][c] = *va;
                }
            } else {
                const auto place = [&](int row) {
                    const int j = min(key + row, last);
                    const int page = min(max(p.pages[(long long)r * p.max_pages + (j >> p.page_shift)], 0), last_page);
                    return page * page_stride + head_offset + (long long)((j & ((1 << p.page_shift) - 1)) * slot_stride);
                };
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const long long at = place(c * kRows + in_rows);
                    kr[t][c] = *reinterpret_cast<const u32x4 *>(d_own < dim ? p.k + at + d_own : g_zeros);
                    vr[t][c] = *reinterpret_cast<const u32x4 *>(d_own < dim ? p.v + at + d_own : g_zeros);
                }
            }
        }
    };

    if (!DIRECT) now = segment_at(at);
    const bool any_block = !DIRECT || now.blocks > 0;
    // All of the workgroup's pieces are of one request (each of its waves finds the same): their sums are joined here, and left as its first wave's.
    const bool joint = DIRECT || (first_worker + W <= workers && first_block(first_worker, workers, total) >= now.from &&
                                  first_block(first_worker + W, workers, total) <= now.upto);
    if (any_block) {
        find_pages(now.r, now.len, now.key);
        request(now.r, now.len, now.key);
    }
    if (now.blocks > 1) find_pages(now.r, now.len, now.key + kBlock);

    // ---- rows: column r16 is token r16 / group, query head r16 mod group ----
    const int token = r16 / p.group, member = r16 % p.group;
    u32x4 q[C];
    f32x4 o[DV];
    float most, base, sum;
    int from, to;          // keys that the row sees
    int all_from, all_to;  // keys that every row sees
    const auto begin_request = [&](const Segment &b) {
        int unused;
        visible_keys(p, b.n, b.len, 0, unused, all_to);
        visible_keys(p, b.n, b.len, b.todo - 1, all_from, unused);
        visible_keys(p, b.n, b.len, token, from, to);
        most = -INFINITY;
        base = sum = 0.0f;
#pragma unroll
        for (int d = 0; d < DV; ++d) o[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const bool real = token < b.todo;
        const uint16_t *const src = p.q + (long long)(b.start + (real ? token : 0)) * p.ld_q + (first_head + member) * p.head_dim;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            q[c] = u32x4{0, 0, 0, 0};
            if (real && (!ANY || 32 * c + 8 * g < dim)) q[c] = *reinterpret_cast<const u32x4 *>(src + 32 * c + 8 * g);
        }
    };
    begin_request(now);

    while (any_block) {
        // K and V to LDS, scores
        const int key0 = now.key;
        const bool masked = key0 + kBlock > all_to || key0 < all_from;
        // Infinities or NaN among the values: zero times them must not reach the rows that do not see them, nor must the second number of a weight, which may be zero or
        // negative, or a weight too small for its type, make a NaN of an infinity.  They are replaced by zeros, and what they make of the rows that do see them, an infinity or a
        // NaN, is found by products of ones.
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
        now.key += kBlock;
        --now.blocks;
        ++at;
        Segment next = now;
        if (at < stop) {
            if (!DIRECT && !now.blocks) {
                next = segment_at(at);
                find_pages(next.r, next.len, next.key);
            }
            request(next.r, next.len, next.key);
            if (next.blocks > 1) find_pages(next.r, next.len, next.key + kBlock);
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
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * p.scale;
        if (masked) {
            const unsigned span = max(to - from, 0);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (unsigned)(key0 + 16 * (e >> 2) + 4 * g + (e & 3) - from) < span ? x[e] : -INFINITY;
        }
        float high = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) high = fmaxf(high, x[e]);
        if (__ballot(high > most + StreamWeights<BF>::grow)) {
            const float m = fmaxf(most, max_over_groups(high));
            const float shrink = most == -INFINITY ? 1.0f : shrink_by(most - m);
            most = m;
            base = m == -INFINITY ? 0.0f : m - StreamWeights<BF>::lift;
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < DV; ++d) o[d] *= shrink;
        }
        u32x4 high_part, low_part;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float a = exp2_fast(x[e] - base), b = exp2_fast(x[e + 1] - base);
            sum += a + b;
            const uint32_t pair = from_float2<BF>(a, b);
            const f32x2 kept = to_float2<BF>(pair);
            high_part[e / 2] = pair;
            low_part[e / 2] = from_float2<BF>(a - kept.x, b - kept.y);
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
                const u32x4 a = column(d);
                u32x4 up, down;
#pragma unroll
                for (int e = 0; e < 4; ++e) up[e] = ones_where_infinite<BF>(a[e], 0), down[e] = ones_where_infinite<BF>(a[e], 0x8000u);
                const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                const f32x4 ups = mfma16<BF>(up, sees, zero), downs = mfma16<BF>(down, sees, zero);
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
                    u32x4 x = *mine;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = finite_only<BF>(x[i]);
                    *mine = x;
                }
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int d = 0; d < DV; ++d) {
            const u32x4 a = column(d);
            o[d] = mfma16<BF>(a, low_part, mfma16<BF>(a, high_part, o[d]));
        }
        asm volatile("" ::: "memory");
        if (now.blocks) continue;
        if (joint) break;
        const float weight = sum_over_groups(sum), unit = 1.0f / weight;
        if (token < now.todo) {
            if (now.whole) {
                uint16_t *const dst = p.out + (long long)(now.start + token) * p.ld_out + (first_head + member) * p.head_dim;
                if (ANY) asm volatile("" : "+v"(dim));  // (compared here, not held as masks through the loop)
#pragma unroll
                for (int d = 0; d < DV; ++d)
                    if (!ANY || 16 * d + 4 * g < dim) {
                        f32x4 y = o[d] * unit;
                        if (to <= from) y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                        *reinterpret_cast<u32x2 *>(dst + 16 * d + 4 * g) = u32x2{from_float2<BF>(y[0], y[1]), from_float2<BF>(y[2], y[3])};
                    }
            } else {
                const long long slot = ((long long)(now.r + worker) * p.kv_heads + head) * kStreamRows + r16;
#pragma unroll
                for (int d = 0; d < DV; ++d) *reinterpret_cast<f32x4 *>(p.part + slot * DT + 16 * d + 4 * g) = o[d];
                if (g == 0) p.stat[slot] = f32x2{most, weight};
            }
        }
        if (at == stop) break;
        now = next;
        begin_request(now);
    }
    if (!joint) return;

    // ---- the waves' sums through LDS, each in its wave's own part; a row's are four banks from the next one's ----
    constexpr int kStep = DT + 4;
    static_assert(kStreamRows * kStep * sizeof(float) <= 2 * kBlock * DT * sizeof(uint16_t), "");
    __shared__ f32x2 stat[W][kStreamRows];
    const auto sums = [&](int w) { return reinterpret_cast<float *>(lds[w]); };
    const float part_weight = sum_over_groups(sum);
#pragma unroll
    for (int d = 0; d < DV; ++d) *reinterpret_cast<f32x4 *>(sums(wave) + r16 * kStep + 16 * d + 4 * g) = o[d];
    if (g == 0) stat[wave][r16] = f32x2{most, part_weight};
    __syncthreads();
    const int rows = now.todo * p.group;
    for (int i = threadIdx.x; i < rows * (DT / 4); i += 64 * W) {
        const int row = i / (DT / 4), d = 4 * (i % (DT / 4)), t = row / p.group;
        if (ANY && DIRECT && d >= p.head_dim) continue;
        float top = -INFINITY, all = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, stat[w][row].x);
        const float high = top == -INFINITY ? 0.0f : top;
        f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float scale = shrink_by(stat[w][row].x - high);
            all = fmaf(stat[w][row].y, scale, all);
            y += *reinterpret_cast<const f32x4 *>(sums(w) + row * kStep + d) * scale;
        }
        if (!DIRECT) {
            const long long slot = ((long long)(now.r + first_worker) * p.kv_heads + head) * kStreamRows + row;
            *reinterpret_cast<f32x4 *>(p.part + slot * DT + d) = y;
            if (d == 0) p.stat[slot] = f32x2{top, all};
            continue;
        }
        y *= 1.0f / all;
        visible_keys(p, now.n, now.len, t, from, to);
        if (to <= from) y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        uint16_t *const dst = p.out + (long long)(now.start + t) * p.ld_out + (head * p.group + row % p.group) * p.head_dim;
        *reinterpret_cast<u32x2 *>(dst + d) = u32x2{from_float2<BF>(y[0], y[1]), from_float2<BF>(y[2], y[3])};
    }
}

// Joins what the waves left of a request.  A workgroup has p.join_rows rows of a (request, kv head): a wave has a row to itself where the
// pieces are few, else all waves share the pieces of each row in turn.
template <int DT, bool BF>
__global__ __launch_bounds__(64 * kWaves) void bcq_attend_join_kernel(AttendParams p)
{
    constexpr int E = DT / 64;  // elements of a lane
    __shared__ float shared[kWaves][DT + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = blockIdx.x, head = blockIdx.y, first_row = blockIdx.z * p.join_rows;
    const Request q = load_request(p, r);
    const int own = blocks_of(p, q), rows = min(q.todo * p.group - first_row, p.join_rows);
    if (own == 0 || rows <= 0) return;
    int total = 0, upto = 0;
    for (int c = 0; c < p.requests; c += 64) {
        Window w;
        w.load(p, c, total, lane);
        total = lane_of(w.upto, 63);
        if (r >= c && r < c + 64) upto = lane_of(w.upto, r - c);
    }
    const int workers = workers_of(p, total);
    const int w0 = worker_of(upto - own, workers, total), w1 = worker_of(upto - 1, workers, total);
    if (w0 == w1) return;  // finished by its one wave
    // pieces: of single waves, of whole workgroups, of single waves
    const int g0 = (w0 + kWaves - 1) / kWaves + (w0 % kWaves == 0 && first_block(w0, workers, total) < upto - own ? 1 : 0);
    const int g1 = (w1 + 1) % kWaves == 0 && first_block(w1 + 1, workers, total) == upto ? (w1 + 1) / kWaves : w1 / kWaves;
    const int groups = max(g1 - g0, 0), lead = groups ? kWaves * g0 - w0 : w1 - w0 + 1, pieces = lead + groups + (groups ? w1 + 1 - kWaves * g1 : 0);
    const auto slots = [&](int row) {
        return [=](int i) {
            const int w = i < lead ? w0 + i : i < lead + groups ? kWaves * (g0 + i - lead) : kWaves * g1 + i - lead - groups;
            return ((long long)(w + r) * p.kv_heads + head) * kStreamRows + row;
        };
    };
    const auto finish = [&](int row, const float (&y)[E], float weight) {
        int from, to;
        visible_keys(p, q.n, q.len, row / p.group, from, to);
        uint16_t *const dst = p.out + (long long)(q.start + row / p.group) * p.ld_out + (head * p.group + row % p.group) * p.head_dim;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (lane * E + e < p.head_dim) dst[lane * E + e] = from_float<BF>(to > from ? y[e] / weight : 0.0f);
    };
    float y[E], weight;
    if (p.join_rows == kWaves && pieces <= 2 * kJoinAhead) {
        if (wave >= rows) return;
        const int row = first_row + wave;
        join_pieces<DT, 1>(p, slots(row), 0, pieces, 0, lane, y, weight);
        finish(row, y, weight);
        return;
    }
    for (int row = first_row; row < first_row + rows; ++row) {
        join_pieces<DT, kWaves>(p, slots(row), 0, pieces, wave, lane, y, weight);
#pragma unroll
        for (int e = 0; e < E; ++e) shared[wave][lane * E + e] = y[e];
        if (lane == 0) shared[wave][DT] = weight;
        __syncthreads();
        if (wave == 0) {
            weight = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                weight += shared[w][DT];
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] += shared[w][lane * E + e];
            }
            finish(row, y, weight);
        }
        __syncthreads();
    }
}

namespace {

int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// One launch, in which a workgroup has a (request, kv head) to itself, or the line and its join?  The line balances and fills the chip with few
// requests, but costs a launch more and its waves look at all requests first.  With fewer pairs than compute units a wave may have five blocks in a row, four (heads of 64:
// three) where there are so few pairs that the line's many waves have hardly one.  Measured, own against line (replayed graphs, all requests of a length, 8 kv heads of 8 query
// heads): heads of 128, 1 request of 500 keys 8.2 and 10.9 us, 1000 11.6 and 11.1 (eager calls 10.5 and 10.6), 1200 13.0 and 10.9; 4 of 1200 14.2 and 15.5, 16 of 1000
// 15.5 and 23.3; heads of 64, 1 of 1500 9.6 and 9.7, 2000 11.1 and 9.7, 4 of 2500 13.8 and 14.2; heads of 256, 1 of 300 13.8 and 16.3, 600 19.4 and 17.7, 4 of 600 20.5 and
// 26.0.  With four waves, heads of 128, 64 requests of 200 keys 13.3 and 21.6, of 1000 50.8 and 52.4; heads of 64, 64 of 1500 39.0 and 41.7.
bool one_launch(long long pairs, int dim, long long most_keys)
{
    if (pairs > 1 << 23) return false;  // (threads of a grid)
    const int cus = compute_units(), in_a_row = pairs >= cus / 16 ? 5 : dim == 64 ? 3 : 4;
    return most_keys <= (pairs < cus ? in_a_row * kBlock * most_waves(dim) : 1536);
}

struct StreamPlan {
    int dim, workers;
    bool any;
    size_t slots, part_bytes;
};
StreamPlan stream_plan(const bcq_cache &c, int requests)
{
    StreamPlan s;
    s.dim = padded_dim(c.head_dim);
    s.any = c.head_dim != s.dim || c.page_size < 16;
    // As many waves as the chip holds: one workgroup more would start when the others end.
    const int groups = compute_units() * stream_occupancy(s.dim, s.any) / c.kv_heads;
    s.workers = kWaves * (groups > 1 ? groups : 1);
    s.slots = (size_t)(s.workers + requests) * c.kv_heads * kStreamRows;
    s.part_bytes = s.slots * s.dim * sizeof(float);
    return s;
}

template <int DT, bool BF, int OWN>
void stream_own(const AttendParams &p, bool any, unsigned pairs, hipStream_t s)
{
    if (any) bcq_attend_stream_kernel<DT, BF, true, false, OWN><<<pairs, 64 * OWN, 0, s>>>(p);
    else bcq_attend_stream_kernel<DT, BF, false, false, OWN><<<pairs, 64 * OWN, 0, s>>>(p);
}

template <int DT, bool BF>
void stream_and_join(const AttendParams &p, bool any, bool passing, hipStream_t s)
{
    if (p.workers == 0) {  // no line: a workgroup per request and kv head
        const unsigned pairs = (unsigned)p.requests * p.kv_heads;
        if (pairs < (unsigned)compute_units()) stream_own<DT, BF, most_waves(DT)>(p, any, pairs, s);
        else stream_own<DT, BF, kWaves>(p, any, pairs, s);
        return;
    }
    const int groups = (p.workers + kWaves - 1) / kWaves * p.kv_heads;
    if (any) bcq_attend_stream_kernel<DT, BF, true, false, 0><<<groups, 64 * kWaves, 0, s>>>(p);
    else if (passing) bcq_attend_stream_kernel<DT, BF, false, true, 0><<<groups, 64 * kWaves, 0, s>>>(p);
    else bcq_attend_stream_kernel<DT, BF, false, false, 0><<<groups, 64 * kWaves, 0, s>>>(p);
    const long long most = (long long)p.max_new * p.group;
    const int rows = (int)(most < kStreamRows ? most : kStreamRows);
    AttendParams j = p;
    j.join_rows = (long long)p.requests * p.kv_heads * rows >= 2 * kWaves * compute_units() ? kWaves : 1;
    bcq_attend_join_kernel<DT, BF><<<dim3(p.requests, p.kv_heads, (rows + j.join_rows - 1) / j.join_rows), 64 * kWaves, 0, s>>>(j);
}

template <bool BF>
void by_dim(const AttendParams &p, int dim, bool any, bool passing, hipStream_t s)
{
    if (dim == 64) stream_and_join<64, BF>(p, any, passing, s);
    else if (dim == 128) stream_and_join<128, BF>(p, any, passing, s);
    else stream_and_join<256, BF>(p, any, passing, s);
}

// Which kernels a call needs: the stream kernel has the requests of up to kStreamRows rows, the chunk kernel the others.  The host knows tokens,
// requests and the longest chunk: where no request can be of one of the kinds, its kernel is not launched and the other takes what there is.
struct Split {
    bool stream, chunk;
};
Split split(int tokens, int requests, int group, int max_new)
{
    if ((long long)max_new * group <= kStreamRows) return {true, false};
    return {group <= kStreamRows && tokens != (long long)requests * max_new, true};
}

size_t chunk_part_bytes(int parts, int tokens, int q_heads, int dim) { return parts > 1 ? (size_t)parts * tokens * q_heads * dim * sizeof(float) : 0; }
size_t chunk_bytes(int parts, int tokens, int q_heads, int dim)
{
    return parts > 1 ? chunk_part_bytes(parts, tokens, q_heads, dim) + (size_t)parts * tokens * q_heads * sizeof(f32x2) : 0;
}

}  // namespace

size_t attend_workspace_bytes(const bcq_cache &c, int tokens, int requests, int q_heads, int max_new, int max_pages)
{
    const Split which = split(tokens, requests, q_heads / c.kv_heads, max_new);
    const StreamPlan s = stream_plan(c, requests);
    const long long most_keys = (long long)max_pages * c.page_size;  // (a window makes them fewer, and one launch no less likely)
    const size_t one = which.stream && !one_launch((long long)requests * c.kv_heads, s.dim, most_keys) ? s.part_bytes + s.slots * sizeof(f32x2) : 0;
    if (!which.chunk) return one;
    const int parts = chunk_parts(tokens, requests, max_new, q_heads / c.kv_heads, c.kv_heads, s.dim, most_keys);
    const size_t other = chunk_bytes(parts, tokens, q_heads, s.dim);
    return one > other ? one : other;  // one after the other
}

hipError_t launch_attend(const AttendArgs &a, hipStream_t stream)
{
    const bcq_cache &c = a.cache;
    const StreamPlan plan = stream_plan(c, a.requests);
    AttendParams p = {};
    p.k = a.k, p.v = a.v, p.q = a.q, p.q_start = a.q_start, p.kv_len = a.kv_len, p.pages = a.pages, p.out = a.out;
    p.part = static_cast<float *>(a.workspace);
    p.ld_q = a.ld_q, p.ld_out = a.ld_out, p.page_stride = c.page_stride, p.head_stride = c.head_stride, p.slot_stride = (int)c.slot_stride;
    p.tokens = a.tokens, p.requests = a.requests, p.kv_heads = c.kv_heads, p.group = a.q_heads / c.kv_heads;
    p.head_dim = c.head_dim, p.page_shift = __builtin_ctz(c.page_size), p.num_pages = c.num_pages, p.max_pages = a.max_pages;
    p.max_new = a.max_new, p.causal = a.causal;
    p.window = a.window > 1 << 30 ? 0 : a.window;  // (no request has so many keys, and positions less a window stay in range)
    // What the rows of a tile can see at most, as far as the host knows.
    long long most_keys = (long long)a.max_pages * c.page_size;
    const int tile_tokens = kMostRows / p.group + 2 < a.max_new ? kMostRows / p.group + 2 : a.max_new;
    if (a.window && (long long)a.window + tile_tokens < most_keys) most_keys = (long long)a.window + tile_tokens;
    p.scale = (float)(a.scale * 1.4426950408889634);
    const Split which = split(a.tokens, a.requests, p.group, a.max_new);
    // Where every byte of K and V is read once, loads that leave nothing behind for others are faster (8 heads of 128, 1 GiB: 177 us against
    // 199), unless the cache is so small that it may still be in the last level from the call before (32 x 2000 keys of 4 heads of 64,
    // 66 MB: 24.5 us against 22).
    const bool passing = 4 * (long long)c.num_pages * c.page_stride >= kPassingBytes;
    if (which.stream) {
        p.rows = kStreamRows, p.workers = one_launch((long long)a.requests * c.kv_heads, plan.dim, most_keys) ? 0 : plan.workers;
        p.stat = reinterpret_cast<f32x2 *>(static_cast<char *>(a.workspace) + plan.part_bytes);
        if (c.dtype == BCQ_BF16) by_dim<true>(p, plan.dim, plan.any, passing, stream);
        else by_dim<false>(p, plan.dim, plan.any, passing, stream);
    }
    if (which.chunk) {
        p.rows = which.stream ? kStreamRows : 0;
        p.parts = chunk_parts(a.tokens, a.requests, a.max_new, p.group, c.kv_heads, plan.dim, most_keys);  // (no more than the workspace is for)
        p.stat = reinterpret_cast<f32x2 *>(static_cast<char *>(a.workspace) + chunk_part_bytes(p.parts, a.tokens, a.q_heads, plan.dim));
        launch_chunks(p, plan.dim, plan.any, passing, c.dtype == BCQ_BF16, stream);
    }
    return hipGetLastError();
}

}  // namespace bcq
