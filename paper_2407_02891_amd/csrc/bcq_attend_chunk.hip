// Attention of chunks of new tokens over a paged cache: the requests with more rows than the stream kernel takes.
//
//   out = sum_j softmax_j(scale q . k_j) v_j
//
// Bound by the matrix instructions (4 head_dim operations for a pair of row and key), and by the vector instructions of the softmax beside
// them.  A workgroup has a tile of 128 rows ((new token, query head) pairs that share a kv head), 32 a wave, and walks the keys that any of
// them sees.
//  * What a tile does with its keys is in bcq_attend_tile.h.
//  * Few tiles and many keys: the keys of a tile are cut into `parts`, whose sums a second launch joins.
//
// Measured: 2048 tokens over 8192 keys, 56 heads of 128, bfloat16: 434 us, 970 TFLOP/s, three quarters of what a large library product reaches; the matrix
// pipe is busy 53 % of the time and the vector pipe 39 %, no bank conflicts, two waves per SIMD as the registers allow (226 of 256).  Sorting the
// exponentials of 32 keys among the matrix instructions of the others by hand took 487 us against 455, a higher priority for a wave in its matrix instructions 456.
// A first kernel without matrix instructions took 62 ms.  Five tokens over 131077 keys (537 MB): 86 us and 6 for the join, 6.2 TB/s.
#include "bcq_attend_tile.h"

namespace bcq {

namespace {

constexpr int kWaves = kTileWaves;
constexpr int kFewParts = 8;

__device__ __forceinline__ int tile_slots_before(const AttendParams &p, int r)
{
    return (int)((long long)min(max(p.q_start[r], 0), p.tokens) * p.group / kChunkRows) + r;
}

}  // namespace

// DT: head_dim, or what it is padded to.  ANY: head_dim < DT, or pages of fewer than 16 slots.
template <int DT, bool BF, bool ANY, bool PASSING>
__global__ __launch_bounds__(64 * kWaves, tile_occupancy(DT)) void bcq_attend_chunk_kernel(AttendParams p)
{
    constexpr int KB = tile_keys(DT), DV = DT / 32;
    __shared__ __attribute__((aligned(1024))) uint16_t k0[KB * DT], k1[KB * DT], v0[KB * DT], v1[KB * DT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, h = lane >> 5;

    // ---- which rows: the slots of a request's tiles begin at q_start * group / 128 + r, the last tiles (with the most keys) first ----
    const int head = blockIdx.x % p.kv_heads, part = blockIdx.y;
    const int slot = gridDim.x / p.kv_heads - 1 - blockIdx.x / p.kv_heads;
    const int r = last_request(p, lane, [&](int i) { return tile_slots_before(p, i) <= slot; });
    const Request q = load_request(p, r);
    const int rows = q.todo * p.group, row0 = (slot - tile_slots_before(p, r)) * kChunkRows;
    if (rows <= p.rows || row0 < 0 || row0 >= rows) return;

    // ---- which keys ----
    const int row = row0 + 32 * wave + r32;
    const bool real = row < rows;
    const int token = row / p.group, member = row - token * p.group;
    int from, to, low, end, tile_from, tile_to, all_from, all_to;
    visible_keys(p, q.n, q.len, token, from, to);
    visible_keys(p, q.n, q.len, row0 / p.group, low, tile_to);                                          // of the tile: any sees [low, end), all see
    visible_keys(p, q.n, q.len, (min(row0 + kChunkRows, rows) - 1) / p.group, tile_from, end);          // [tile_from, tile_to)
    const int first_token = (row0 + 32 * wave) / p.group, last_token = (min(row0 + 32 * wave + 32, rows) - 1) / p.group;
    int any_from, any_to;  // of the wave, the same
    visible_keys(p, q.n, q.len, first_token, any_from, all_to);
    visible_keys(p, q.n, q.len, last_token, all_from, any_to);
    const bool has_rows = row0 + 32 * wave < rows;
    end = max(end, 0);
    const int block0 = min(low, end) / KB, blocks = (end + KB - 1) / KB - block0;
    const int b0 = block0 + (int)((long long)blocks * part / p.parts), b1 = block0 + (int)((long long)blocks * (part + 1) / p.parts);

    Tile t;
    t.head = head, t.request = r, t.last = max(q.len - 1, 0), t.b0 = b0, t.b1 = b1;
    t.tile_from = tile_from, t.tile_to = tile_to, t.all_from = all_from, t.all_to = all_to, t.any_from = any_from, t.any_to = any_to;
    t.has_rows = has_rows, t.real = real, t.from = from, t.to = to;
    t.q = p.q + (long long)(q.start + (real ? token : 0)) * p.ld_q + (head * p.group + (real ? member : 0)) * p.head_dim;
    f32x16 o[DV];
    float most, sum;
    attend_tile<DT, BF, ANY, PASSING>(p, t, k0, k1, v0, v1, o, most, sum);

    // ---- results: lane (h, r32) has of row r32 the elements 32 d + 8 u + 4 h + i in number 4 u + i of o[d] ----
    const auto twin = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, sum), __builtin_bit_cast(unsigned, sum), false, false);
    sum = __builtin_bit_cast(float, (unsigned)twin[0]) + __builtin_bit_cast(float, (unsigned)twin[1]);
    if (!real) return;
    if (gridDim.y == 1) {  // (p.parts, which would have to be kept in a lane for this)
        const float unit = 1.0f / sum;
        const bool empty = to <= from;
        uint16_t *const dst = p.out + (long long)(q.start + token) * p.ld_out + (head * p.group + member) * p.head_dim;
#pragma unroll
        for (int d = 0; d < DV; ++d)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int e = 32 * d + 8 * u + 4 * h;
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = empty ? 0.0f : o[d][4 * u + i] * unit;
                if (!ANY || e < p.head_dim) *reinterpret_cast<u32x2 *>(dst + e) = u32x2{from_float2<BF>(y[0], y[1]), from_float2<BF>(y[2], y[3])};
            }
    } else {
        const long long at = ((long long)part * p.kv_heads + head) * p.tokens * p.group + (long long)q.start * p.group + row;
#pragma unroll
        for (int d = 0; d < DV; ++d)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *reinterpret_cast<f32x4 *>(p.part + at * DT + 32 * d + 8 * u + 4 * h) =
                    f32x4{o[d][4 * u], o[d][4 * u + 1], o[d][4 * u + 2], o[d][4 * u + 3]};
        if (h == 0) p.stat[at] = f32x2{most, sum};
    }
}

// Joins many parts: a workgroup per row, whose waves share them.
template <int DT, bool BF>
__global__ __launch_bounds__(64 * kWaves) void bcq_attend_chunk_join_kernel(AttendParams p)
{
    constexpr int E = DT / 64;
    __shared__ float shared[kWaves][DT + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = blockIdx.x / p.group, member = blockIdx.x % p.group, head = blockIdx.y;
    const Request q = load_request(p, last_request(p, lane, [&](int i) { return p.q_start[i] <= token; }));
    const int i = token - q.start;
    if (i < 0 || i >= q.todo || q.todo * p.group <= p.rows) return;
    const long long rows = (long long)p.tokens * p.group;
    float y[E], weight;
    join_pieces<DT, kWaves>(p, Slots{head * rows + blockIdx.x, p.kv_heads * rows}, 0, p.parts, wave, lane, y, weight);
#pragma unroll
    for (int e = 0; e < E; ++e) shared[wave][lane * E + e] = y[e];
    if (lane == 0) shared[wave][DT] = weight;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        weight += shared[w][DT];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] += shared[w][lane * E + e];
    }
    int from, to;
    visible_keys(p, q.n, q.len, i, from, to);
    uint16_t *const dst = p.out + (long long)token * p.ld_out + (head * p.group + member) * p.head_dim;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (lane * E + e < p.head_dim) dst[lane * E + e] = from_float<BF>(to > from ? y[e] / weight : 0.0f);
}

// Joins few parts: four elements of a row to a thread, which reads all parts of them at once.
template <int DT, bool BF>
__global__ __launch_bounds__(64 * kWaves) void bcq_attend_chunk_join_few_kernel(AttendParams p)
{
    constexpr int kLanes = DT / 4;  // of a row
    const int lane = threadIdx.x & 63, first = (blockIdx.x * 64 * kWaves + (threadIdx.x & ~63)) / kLanes, rows = p.tokens * p.group;
    const int row = min(first + lane / kLanes, rows - 1), d = 4 * (lane % kLanes), head = blockIdx.y;
    const int token = row / p.group, member = row % p.group, first_token = min(first, rows - 1) / p.group;
    int r = last_request(p, lane, [&](int i) { return p.q_start[i] <= first_token; });
    while (r + 1 < p.requests && p.q_start[r + 1] <= token) ++r;
    const Request q = load_request(p, r);
    const int i = token - q.start;
    if (first + lane / kLanes >= rows || i < 0 || i >= q.todo || q.todo * p.group <= p.rows || d >= p.head_dim) return;
    const long long at = (long long)head * rows + row, step = (long long)p.kv_heads * rows;
    f32x4 part[kFewParts], y = {0.0f, 0.0f, 0.0f, 0.0f};
    f32x2 stat[kFewParts];
    float most = -INFINITY, weight = 0.0f;
#pragma unroll
    for (int k = 0; k < kFewParts; ++k)
        if (k < p.parts) {
            stat[k] = p.stat[k * step + at];
            part[k] = *reinterpret_cast<const f32x4 *>(p.part + (k * step + at) * DT + d);
        }
#pragma unroll
    for (int k = 0; k < kFewParts; ++k)
        if (k < p.parts) most = fmaxf(most, stat[k].x);
    const float base = most == -INFINITY ? 0.0f : most;
#pragma unroll
    for (int k = 0; k < kFewParts; ++k)
        if (k < p.parts) {
            const float scale = shrink_by(stat[k].x - base);
            weight = fmaf(stat[k].y, scale, weight);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = fmaf(part[k][e], scale, y[e]);
        }
    int from, to;
    visible_keys(p, q.n, q.len, i, from, to);
    const float unit = 1.0f / weight;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = to > from ? y[e] * unit : 0.0f;
    *reinterpret_cast<u32x2 *>(p.out + (long long)token * p.ld_out + (head * p.group + member) * p.head_dim + d) =
        u32x2{from_float2<BF>(y[0], y[1]), from_float2<BF>(y[2], y[3])};
}

// Pieces that the keys of a tile are cut into, none with fewer than four blocks of the longest row of pages.  The least of what the rounds of workgroups take (2 us a
// block, whatever the head) and of writing and joining the pieces' sums (6 TB/s), if that saves a tenth.  More keys never make it fewer pieces.
// (2 requests of 512 tokens over 4096 keys, 16 / 8 heads of 256, 128 tiles: one piece 198 us, two 119; 4 of 300 to 600, window 1000, 32 / 8 heads of 128, 480 tiles: one
// 58, two 78; 700 over 3000, 176 tiles: two 68, three 72, five 64.)
int chunk_parts(int tokens, int requests, int max_new, int group, int kv_heads, int dim, long long most_keys)
{
    const long long rows = (long long)tokens * group;
    // tiles: all of them where the requests are alike, else half a tile more for each request
    const long long tiles = kv_heads * (tokens == (long long)requests * max_new ? requests * (((long long)max_new * group + kChunkRows - 1) / kChunkRows)
                                                                               : rows / kChunkRows + (requests + 1) / 2);
    const long long at_once = (long long)compute_units() * tile_occupancy(dim), blocks = most_keys / tile_keys(dim), most = blocks / 4 < 64 ? blocks / 4 : 64;
    const double all = 2.0 * blocks, join = rows * kv_heads * dim * 8 / 6e6;
    const auto rounds = [&](long long parts) { return (double)((tiles * parts + at_once - 1) / at_once) / parts; };
    int parts = 1;
    double least = 0.9 * all * rounds(1);
    for (int n = 2; n <= most && 4.0 + n * join < least; ++n) {
        const double time = all * rounds(n) + 4.0 + n * join;
        if (time < least) least = time, parts = n;
    }
    return parts;
}

template <int DT, bool BF>
static void chunks(const AttendParams &p, bool any, bool passing, hipStream_t s)
{
    const long long slots = (long long)p.tokens * p.group / kChunkRows + p.requests;
    const dim3 grid((unsigned)(slots * p.kv_heads), p.parts);
    // (where a request has one tile, each byte of K and V is read once)
    if (any) bcq_attend_chunk_kernel<DT, BF, true, false><<<grid, 64 * kWaves, 0, s>>>(p);
    else if (passing && (long long)p.max_new * p.group <= kChunkRows) bcq_attend_chunk_kernel<DT, BF, false, true><<<grid, 64 * kWaves, 0, s>>>(p);
    else bcq_attend_chunk_kernel<DT, BF, false, false><<<grid, 64 * kWaves, 0, s>>>(p);
    const int rows = p.tokens * p.group;
    if (p.parts > kFewParts) bcq_attend_chunk_join_kernel<DT, BF><<<dim3(rows, p.kv_heads), 64 * kWaves, 0, s>>>(p);
    else if (p.parts > 1) bcq_attend_chunk_join_few_kernel<DT, BF><<<dim3((rows + 1024 / DT - 1) / (1024 / DT), p.kv_heads), 64 * kWaves, 0, s>>>(p);
}

template <bool BF>
static void by_dim(const AttendParams &p, int dim, bool any, bool passing, hipStream_t s)
{
    if (dim == 64) chunks<64, BF>(p, any, passing, s);
    else if (dim == 128) chunks<128, BF>(p, any, passing, s);
    else chunks<256, BF>(p, any, passing, s);
}

void launch_chunks(const AttendParams &p, int dim, bool any, bool passing, bool bf16, hipStream_t s)
{
    if (bf16) by_dim<true>(p, dim, any, passing, s);
    else by_dim<false>(p, dim, any, passing, s);
}

}  // namespace bcq
