// Attention of chunks of new tokens over a paged cache: the requests with more rows than the stream kernel takes.
//
//   out = sum_j softmax_j(scale q . k_j) v_j
//
// Bound by the matrix instructions (4 head_dim operations for a pair of row and key), and by the vector instructions of the softmax beside
// them.  A workgroup has a tile of 128 rows ((new token, query head) pairs that share a kv head), 32 a wave, and walks the keys that any of
// them sees.
//  * K and V blocks go straight to LDS, two buffers each: the next block is on its way while this one is used.  The 16-byte pieces of a row are exchanged by the row's number, on the global side of the transfer, so that
//    both kinds of reads find all banks.
//  * S^T = K Q^T with Q in registers: a lane has one row's scores, 32 for a block of 64 keys, so a row's maximum and sum need one exchange between
//    two lanes; its weights, rounded to 16 bits, are the operand of O^T = V^T P^T as they are, for the keys of a product may be numbered in any order.
//    V's side of it comes from the transposing read.  The rounding of the weights adds to a result what its own rounding does (1.3 times in the mean square); held as
//    two numbers they cost 8 to 30 % from two waves' rows on (5 tokens over 131077 keys, 8 query heads a kv head: 116 us against 97).  Weights are taken
//    relative to a running maximum (Weights in bcq_attend.h).
//  * Blocks that all of a wave's rows see have no masks, those that none sees are left out.
//  * Few tiles and many keys: the keys of a tile are cut into `parts`, whose sums a second launch joins.
//
// Measured: 2048 tokens over 8192 keys, 56 heads of 128, bfloat16: 434 us, 970 TFLOP/s, three quarters of what a large library product reaches; the matrix
// pipe is busy 53 % of the time and the vector pipe 39 %, no bank conflicts, two waves per SIMD as the registers allow (226 of 256).  Sorting the
// exponentials of 32 keys among the matrix instructions of the others by hand took 487 us against 455, a higher priority for a wave in its matrix instructions 456.
// A first kernel without matrix instructions took 62 ms.  Five tokens over 131077 keys (537 MB): 86 us and 6 for the join, 6.2 TB/s.
#include "bcq_attend.h"

namespace bcq {

namespace {

constexpr int kWaves = 4, kChunkRows = 32 * kWaves;
constexpr int kFewParts = 8;
// (Renewed at half of that, heads of 128 take 1 % more and heads of 256 10; at a quarter 2 and 20.)
template <bool BF>
using ChunkWeights = Weights<BF, 8>;
constexpr int chunk_keys(int dim) { return dim == 256 ? 32 : 64; }  // a block
constexpr int chunk_occupancy(int dim) { return dim == 256 ? 1 : 2; }

typedef __attribute__((address_space(3))) void *lds_void;
typedef const __attribute__((address_space(1))) void *global_void;

// Sixteen bytes a lane from memory to LDS: lane l's to `to` (the wave's) + 16 l.  PASSING: nothing is left behind in the caches.
template <bool PASSING>
__device__ __forceinline__ void load_to_lds(const uint16_t *from, uint16_t *to)
{
    __builtin_amdgcn_global_load_lds((global_void)from, (lds_void)to, 16, 0, PASSING ? 2 : 0);
}

// This wave's transfers to LDS have arrived, and its reads of LDS have returned: what the barrier after it promises the other waves.
__device__ __forceinline__ void all_arrived() { __builtin_amdgcn_s_waitcnt(0x0070); }  // vmcnt(0) lgkmcnt(0)

__device__ __forceinline__ int tile_slots_before(const AttendParams &p, int r)
{
    return (int)((long long)min(max(p.q_start[r], 0), p.tokens) * p.group / kChunkRows) + r;
}

}  // namespace

// DT: head_dim, or what it is padded to.  ANY: head_dim < DT, or pages of fewer than 16 slots.
template <int DT, bool BF, bool ANY, bool PASSING>
__global__ __launch_bounds__(64 * kWaves, chunk_occupancy(DT)) void bcq_attend_chunk_kernel(AttendParams p)
{
    constexpr int KB = chunk_keys(DT), KT = KB / 32, C = DT / 16, DV = DT / 32;
    constexpr int kPieces = DT / 8, kRows = 64 / kPieces;       // 16-byte pieces of a key; keys of one transfer of a wave
    constexpr int kTransfers = KB / (kRows * kWaves);           // of a wave for a block of K, and for one of V
    // Two buffers each, as objects of their own: the compiler holds reads of one back for the transfers to it alone.
    __shared__ __attribute__((aligned(1024))) uint16_t k0[KB * DT], k1[KB * DT], v0[KB * DT], v1[KB * DT];
    __shared__ int votes[kWaves];
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

    // ---- K and V of a block to LDS ----
    // A wave brings KB / 4 neighbouring keys, which lie in one page of 16 slots or more.
    const int piece = lane % kPieces, in_rows = lane / kPieces;
    const uint16_t *const k_head = p.k + head * p.head_stride, *const v_head = p.v + head * p.head_stride;
    const int last = max(q.len - 1, 0);
    constexpr int kOwn = KB / kWaves;
    int id[ANY ? kTransfers : 1];
    const auto find_pages = [&](int key0) {
        if (ANY) {
#pragma unroll
            for (int i = 0; i < kTransfers; ++i) id[i] = page_of(p, r, min(key0 + kOwn * wave + i * kRows + in_rows, last));
        } else {
            id[0] = page_of_all(p, r, min(key0 + kOwn * wave, last));
        }
    };
    // the 16-element unit of a row of V that unit 0 is exchanged with: four keys' pairs of units, which are read together, fill all banks
    const auto v_turn = [](int key) { return DT == 64 ? (key & 2) | (key >> 2 & 1) : (key & 3) << 1 | (key >> 2 & 1); };
    const auto k_turn = [](int key) { return key & (DT == 64 ? 7 : 15); };
    const int row_off = in_rows * p.slot_stride;
    const auto request = [&](int key0, uint16_t *to_k, uint16_t *to_v) {
        int dim = p.head_dim;
        if (ANY) asm volatile("" : "+v"(dim));  // (compared here, not held as masks through the loop)
        const int first = min(key0 + kOwn * wave, last & -kOwn);         // keys behind the last are the last's copies, and masked
        const long long base = ANY ? 0 : __builtin_amdgcn_readfirstlane(id[0]) * p.page_stride + (long long)((first & ((1 << p.page_shift) - 1)) * p.slot_stride);
        const int most = min(last - first, kOwn - 1) * p.slot_stride;   // (inside the page: the keys that are left would pass 32 bits)
#pragma unroll
        for (int i = 0; i < kTransfers; ++i) {
            const int in_lds = kOwn * wave + i * kRows + in_rows;
            const int k_d = 8 * (piece ^ k_turn(in_lds)), v_d = 8 * (piece ^ v_turn(in_lds) << 1);
            const uint16_t *k, *v;
            if (ANY) {
                const int key = min(key0 + in_lds, last);
                const long long at = id[i] * p.page_stride + (long long)((key & ((1 << p.page_shift) - 1)) * p.slot_stride);
                k = k_d < dim ? k_head + at + k_d : g_zeros;
                v = v_d < dim ? v_head + at + v_d : g_zeros;
            } else {
                const unsigned row = (unsigned)min(row_off + i * kRows * p.slot_stride, most);
                k = reinterpret_cast<const uint16_t *>(reinterpret_cast<const char *>(k_head + base) + 2u * (row + k_d));
                v = reinterpret_cast<const uint16_t *>(reinterpret_cast<const char *>(v_head + base) + 2u * (row + v_d));
            }
            load_to_lds<PASSING>(k, to_k + (kOwn * wave + i * kRows) * DT);
            load_to_lds<PASSING>(v, to_v + (kOwn * wave + i * kRows) * DT);
        }
    };
    // element d of key j
    const auto k_at = [&](const uint16_t *buffer, int key, int d) { return buffer + key * DT + ((d >> 3 ^ k_turn(key)) << 3); };
    const auto v_at = [&](const uint16_t *buffer, int key, int d) { return buffer + key * DT + ((d >> 4 ^ v_turn(key)) << 4) + (d & 15); };

    // ---- Q: lane (h, r32) has of row r32 the elements 16 c + 8 h .. ----
    u32x4 qr[C];
    {
        const uint16_t *const src = p.q + (long long)(q.start + (real ? token : 0)) * p.ld_q + (head * p.group + (real ? member : 0)) * p.head_dim;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int d = 16 * c + 8 * h;
            qr[c] = u32x4{0, 0, 0, 0};
            if (real && (!ANY || d < p.head_dim)) qr[c] = *reinterpret_cast<const u32x4 *>(src + d);
        }
    }
    f32x16 o[DV];
    float most, base, sum;
    bool careful = false;  // all blocks of V are looked at for infinities and NaN, not only those with masks

    const auto step = [&](int b, const uint16_t *kb, uint16_t *vb, uint16_t *next_k, uint16_t *next_v) {
        const int key0 = b * KB;
        const bool more = b + 1 < b1;
        if (more) find_pages(key0 + KB);
        asm volatile("" ::: "memory");
        all_arrived();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (more) request(key0 + KB, next_k, next_v);  // (every wave is through with the other buffers)
        const bool work = has_rows && key0 < any_to && key0 + KB > any_from;
        if (DT == 256) {  // Q stays where the matrix instructions can read it and nothing else needs the place
#pragma unroll
            for (int c = 0; c < C; ++c) asm volatile("" : "+a"(qr[c]));
        }
        // the operand V^T: elements 32 d + r32 of keys 16 u + 4 h .. and 16 u + 8 + 4 h ..
        const auto column = [&](int u, int d, int lane) {
            const int key = 16 * u + 4 * (lane >> 5) + ((lane & 15) >> 2), e = 32 * d + (lane & 16) + 4 * (lane & 3);
            const u32x2 v0 = lds_column(v_at(vb, key, e)), v1 = lds_column(v_at(vb, key + 8, e));
            return u32x4{v0.x, v0.y, v1.x, v1.y};
        };
        if (careful || key0 + KB > tile_to || key0 < tile_from) {
            // Not all rows of the tile see all of these keys.  Infinities or NaN among the values: zero times them must not reach the rows that do not
            // see them.  They are replaced by zeros, and what they make of the rows that do, an infinity or a NaN, is found by products of ones.  (Every wave looks at the whole block, so all of them meet at the barriers or none.)
            int it = lane;
            asm volatile("" : "+v"(it));  // what follows from it is not worth registers over the loop
            float zero = 0.0f;
#pragma unroll 1
            for (int i = it; i < KB * DT / 8; i += 64) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(vb + 8 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) zero = times_zero<BF>(x[e], zero);
            }
            if (__ballot(zero != 0.0f)) {
                if (work) {
                    const unsigned span = max(to - from, 0);
#pragma unroll
                    for (int d = 0; d < DV; ++d) {
#pragma unroll 1
                        for (uint32_t sign = 0; sign <= 0x8000u; sign += 0x8000u) {
                            f32x16 found;
#pragma unroll
                            for (int i = 0; i < 16; ++i) found[i] = 0.0f;
#pragma unroll 1
                            for (int u = 0; u < KB / 16; ++u) {
                                u32x4 a = column(u, d, it), sees;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int key = key0 + 16 * u + 8 * (e >> 1) + 4 * (it >> 5) + 2 * (e & 1);
                                    sees[e] = ((unsigned)(key - from) < span ? kOne<BF> : 0u) | ((unsigned)(key + 1 - from) < span ? kOne<BF> << 16 : 0u);
                                    a[e] = ones_where_infinite<BF>(a[e], sign);
                                }
                                found = mfma32<BF>(a, sees, found);
                            }
                            const float infinity = sign ? -INFINITY : INFINITY;
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[d][i] += found[i] > 0.0f ? infinity : 0.0f;
                        }
                        asm volatile("" : "+v"(o[d]));  // (before the next ones)
                    }
                }
                asm volatile("" ::: "memory");
                all_arrived();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
#pragma unroll 1
                for (int i = wave * 64 + it; i < KB * DT / 8; i += 64 * kWaves) {
                    u32x4 x = *reinterpret_cast<const u32x4 *>(vb + 8 * i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = finite_only<BF>(x[e]);
                    *reinterpret_cast<u32x4 *>(vb + 8 * i) = x;
                }
                asm volatile("" ::: "memory");
                all_arrived();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
        }
        u32x4 weight[KB / 16];
        if (work) {
            f32x16 s[KT];
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
            // (a few pieces of K ahead of their use: the compiler would wait for each)
            constexpr int kAhead = 6, kSteps = KT * C;
            u32x4 a[kAhead];
#pragma unroll
            for (int n = 0; n < kAhead; ++n) a[n] = *reinterpret_cast<const u32x4 *>(k_at(kb, 32 * (n / C) + r32, 16 * (n % C) + 8 * h));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < kSteps; ++n) {
                s[n / C] = mfma32<BF>(a[n % kAhead], qr[n % C], s[n / C]);
                if (n + kAhead < kSteps) a[n % kAhead] = *reinterpret_cast<const u32x4 *>(k_at(kb, 32 * ((n + kAhead) / C) + r32, 16 * ((n + kAhead) % C) + 8 * h));
                __builtin_amdgcn_sched_barrier(0);
            }
            // number 16 t + 4 u + i of a lane is key 32 t + 8 u + 4 h + i
            float x[16 * KT];
#pragma unroll
            for (int e = 0; e < 16 * KT; ++e) x[e] = s[e >> 4][e & 15];
            if (key0 + KB > all_to || key0 < all_from) {
                const unsigned span = max(to - from, 0);
                int key = key0 + 4 * h - from;
                asm volatile("" : "+v"(key));  // (or 32 sums of it would take registers over the loop)
#pragma unroll
                for (int e = 0; e < 16 * KT; ++e) x[e] = (unsigned)(key + 32 * (e >> 4) + 8 * (e >> 2 & 3) + (e & 3)) < span ? x[e] : -INFINITY;
            }
            float high = x[0];
#pragma unroll
            for (int e = 1; e < 16 * KT; ++e) high = fmaxf(high, x[e]);
            high *= p.scale;
            if (__ballot(high > most + ChunkWeights<BF>::grow)) {
                const auto other = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, high), __builtin_bit_cast(unsigned, high), false, false);
                const float m = fmaxf(most, fmaxf(__builtin_bit_cast(float, (unsigned)other[0]), __builtin_bit_cast(float, (unsigned)other[1])));
                if (DT == 256) {  // (or it copies O from the accumulation registers for every block, not here)
#pragma unroll
                    for (int d = 0; d < DV; ++d) asm volatile("" : "+a"(o[d]));
                }
                const float shrink = most == -INFINITY ? 1.0f : shrink_by(most - m);
                most = m;
                base = m == -INFINITY ? 0.0f : m - ChunkWeights<BF>::lift;
                sum *= shrink;
#pragma unroll
                for (int d = 0; d < DV; ++d) o[d] *= shrink;
            }
#pragma unroll
            for (int e = 0; e < 16 * KT; e += 2) {
                const float w0 = exp2_fast(fmaf(x[e], p.scale, -base)), w1 = exp2_fast(fmaf(x[e + 1], p.scale, -base));
                sum += w0 + w1;
                weight[e >> 3][e >> 1 & 3] = from_float2<BF>(w0, w1);
            }
        }
        if (work) {
            constexpr int kAhead = 4, kSteps = KB / 16 * DV;
            u32x4 a[kAhead];
#pragma unroll
            for (int n = 0; n < kAhead; ++n) a[n] = column(n / DV, n % DV, lane);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < kSteps; ++n) {
                o[n % DV] = mfma32<BF>(a[n % kAhead], weight[n / DV], o[n % DV]);
                if (n + kAhead < kSteps) a[n % kAhead] = column((n + kAhead) / DV, (n + kAhead) % DV, lane);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // Once, and again with care if a result is not finite: an infinity that all rows see would be a NaN of the rows whose weight for it is too small for its type.
    for (;;) {
#pragma unroll
        for (int d = 0; d < DV; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
        most = -INFINITY;
        base = sum = 0.0f;
        int first = b0;
        asm volatile("" : "+s"(first));  // (or what the first request computes would be kept for the second time)
        if (first < b1) {
            find_pages(first * KB);
            request(first * KB, k0, v0);
        }
        for (int b = first; b < b1; b += 2) {
            step(b, k0, v0, k1, v1);
            if (b + 1 < b1) step(b + 1, k1, v1, k0, v0);
        }
        if (careful) break;
        float zero = 0.0f;
#pragma unroll
        for (int d = 0; d < DV; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) zero = fmaf(o[d][i], 0.0f, zero);
        const unsigned long long odd = __ballot(real && zero != 0.0f);  // (a NaN)
        if (lane == 0) votes[wave] = odd != 0;
        asm volatile("" ::: "memory");
        all_arrived();
        __builtin_amdgcn_s_barrier();  // (and every wave is through with the buffers)
        asm volatile("" ::: "memory");
        int any = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) any |= votes[w];
        careful = __builtin_amdgcn_readfirstlane(any) != 0;
        if (!careful) break;
    }

    // ---- results: lane (h, r32) has of row r32 the elements 32 d + 8 u + 4 h + i in number 4 u + i of o[d] ----
    const auto twin = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, sum), __builtin_bit_cast(unsigned, sum), false, false);
    sum = __builtin_bit_cast(float, (unsigned)twin[0]) + __builtin_bit_cast(float, (unsigned)twin[1]);
    if (!real) return;
    if (p.parts == 1) {
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
    const long long at_once = (long long)compute_units() * chunk_occupancy(dim), blocks = most_keys / chunk_keys(dim), most = blocks / 4 < 64 ? blocks / 4 : 64;
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
