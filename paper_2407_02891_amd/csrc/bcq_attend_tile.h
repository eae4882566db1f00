// A tile of 128 rows over blocks of a paged cache's keys: what the two kernels of large tiles (chunks of new tokens, requests behind a shared prefix) have in common (not public).
//
//  * K and V blocks go straight to LDS, two buffers each: the next block is on its way while this one is used.  The 16-byte pieces of a row are exchanged by the row's number, on the global side of the transfer, so that
//    both kinds of reads find all banks.
//  * S^T = K Q^T with Q in registers: a lane has one row's scores, 32 for a block of 64 keys, so a row's maximum and sum need one exchange between
//    two lanes; its weights, rounded to 16 bits, are the operand of O^T = V^T P^T as they are, for the keys of a product may be numbered in any order.
//    V's side of it comes from the transposing read.  The rounding of the weights adds to a result what its own rounding does (1.3 times in the mean square); held as
//    two numbers they cost 8 to 30 % from two waves' rows on (5 tokens over 131077 keys, 8 query heads a kv head: 116 us against 97).  Weights are taken
//    relative to a running maximum (Weights in bcq_attend.h).
//  * Blocks that all of a wave's rows see have no masks, those that none sees are left out.
#pragma once
#include "bcq_attend.h"

namespace bcq {

namespace {

constexpr int kTileWaves = 4, kChunkRows = 32 * kTileWaves;
// (Renewed at half of that, heads of 128 take 1 % more and heads of 256 10; at a quarter 2 and 20.)
template <bool BF>
using TileWeights = Weights<BF, 8>;
constexpr int tile_keys(int dim) { return dim == 256 ? 32 : 64; }  // a block
constexpr int tile_occupancy(int dim) { return dim == 256 ? 1 : 2; }

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

// A workgroup's tile.  Its waves agree on all up to tile_to; wave w has the rows 32 w .. 32 w + 31, lane l the row l mod 32 of them.
struct Tile {
    int head, request;                       // kv head; whose row of the table of pages
    int last;                                // the last key
    int b0, b1;                              // blocks
    int tile_from, tile_to;                  // keys that all rows see: [tile_from, tile_to)
    int all_from, all_to, any_from, any_to;  // that all of the wave's rows see; outside of which none of them sees any
    bool has_rows;                           // of the wave
    bool real;                               // the lane has a row
    const uint16_t *q;                       // its row of q, this head's elements
    int from, to;                            // keys that it sees
};

// Sums over the keys of the tile's blocks, relative to `most` (times log2 e), and their weight, this lane's half of it.  Number 4 u + i of o[d] is element 32 d + 8 u + 4 (lane / 32) + i
// of the lane's row.  All waves of the workgroup together.
// Returns (all waves the same) whether some may still be reading LDS.
// k0, k1, v0, v1: LDS, tile_keys(DT) * DT elements each, as objects of their own: the compiler holds reads of one back for the transfers to it alone.
template <int DT, bool BF, bool ANY, bool PASSING>
__device__ __forceinline__ bool attend_tile(const AttendParams &p, const Tile &t, uint16_t *k0, uint16_t *k1, uint16_t *v0, uint16_t *v1, f32x16 (&o)[DT / 32], float &most,
                                            float &sum)
{
    constexpr int KB = tile_keys(DT), KT = KB / 32, C = DT / 16, DV = DT / 32;
    constexpr int kPieces = DT / 8, kRows = 64 / kPieces;       // 16-byte pieces of a key; keys of one transfer of a wave
    constexpr int kTransfers = KB / (kRows * kTileWaves);       // of a wave for a block of K, and for one of V
    __shared__ int votes[kTileWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, h = lane >> 5, from = t.from, to = t.to, b0 = t.b0, b1 = t.b1, any_to = t.has_rows ? t.any_to : 0;

    // ---- K and V of a block to LDS ----
    // A wave brings KB / 4 neighbouring keys, which lie in one page of 16 slots or more.
    const int piece = lane % kPieces, in_rows = lane / kPieces;
    const uint16_t *const k_head = p.k + t.head * p.head_stride, *const v_head = p.v + t.head * p.head_stride;
    const int last = t.last;
    constexpr int kOwn = KB / kTileWaves;
    int id[ANY ? kTransfers : 1];
    const auto find_pages = [&](int key0) {
        if (ANY) {
#pragma unroll
            for (int i = 0; i < kTransfers; ++i) id[i] = page_of(p, t.request, min(key0 + kOwn * wave + i * kRows + in_rows, last));
        } else {
            id[0] = page_of_all(p, t.request, min(key0 + kOwn * wave, last));
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
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int d = 16 * c + 8 * h;
        qr[c] = u32x4{0, 0, 0, 0};
        if (t.real && (!ANY || d < p.head_dim)) qr[c] = *reinterpret_cast<const u32x4 *>(t.q + d);
    }
    float base;
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
        const bool work = key0 < any_to && key0 + KB > t.any_from;
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
        if (careful || key0 + KB > t.tile_to || key0 < t.tile_from) {
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
                for (int i = wave * 64 + it; i < KB * DT / 8; i += 64 * kTileWaves) {
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
            if (key0 + KB > t.all_to || key0 < t.all_from) {
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
            if (__ballot(high > most + TileWeights<BF>::grow)) {
                const auto other = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, high), __builtin_bit_cast(unsigned, high), false, false);
                const float m = fmaxf(most, fmaxf(__builtin_bit_cast(float, (unsigned)other[0]), __builtin_bit_cast(float, (unsigned)other[1])));
                if (DT == 256) {  // (or it copies O from the accumulation registers for every block, not here)
#pragma unroll
                    for (int d = 0; d < DV; ++d) asm volatile("" : "+a"(o[d]));
                }
                const float shrink = most == -INFINITY ? 1.0f : shrink_by(most - m);
                most = m;
                base = m == -INFINITY ? 0.0f : m - TileWeights<BF>::lift;
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
        const unsigned long long odd = __ballot(t.real && zero != 0.0f);  // (a NaN)
        if (lane == 0) votes[wave] = odd != 0;
        asm volatile("" ::: "memory");
        all_arrived();
        __builtin_amdgcn_s_barrier();  // (and every wave is through with the buffers)
        asm volatile("" ::: "memory");
        int any = 0;
#pragma unroll
        for (int w = 0; w < kTileWaves; ++w) any |= votes[w];
        careful = __builtin_amdgcn_readfirstlane(any) != 0;
        if (!careful) break;
    }
    return careful;
}

}  // namespace

}  // namespace bcq
