// Low-rank adapters of many requests beside a shared projection:  Y[t] = base[t] + scale[a] * B[a] (A[a] X[t]),  a = adapter[t].
//
// Bound by the bytes: A and B of the adapters that occur, and with many tokens X, base and Y.  Tokens of the same adapter are taken together, 16 or 64
// at a time (a tile), so that a piece of A or B is read once for them and the sums run on the matrix cores.  Up to 64 tokens every wave finds
// its tile's tokens by comparing all adapter numbers at once; beyond, a small launch sorts the tokens by adapter first.  Two launches:
//
//  * v = A x: a workgroup has a tile, 16 to 64 rows of A and a slice of N; its waves share the slice and add up in LDS.  The slices, as many as fill
//    the chip, leave their sums in binary32 side by side, and whoever reads them adds them in order.
//  * Y = base + B v: a workgroup has a tile and a range of rows of B.  v (times the scale) is held as a sum of 16-bit numbers beside the 16-bit rows of B:
//    two for binary16 (after a power of two for each token: 22 bits and more of its largest value), three for bfloat16 (24 bits).  The operand's 32
//    places are 16 of v's first numbers and the same 16 of its second ones.  The rows of B are numbered so that a lane ends up with eight
//    neighbouring outputs of a token and four lanes with 32.
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

namespace {

constexpr int kWaves = 4;
constexpr int kFewTokens = 64;     // that every wave sorts out by itself
constexpr int kPlanGroups = 4096;  // adapters (and none) whose tokens are counted in LDS

struct LoraParams {
    LoraArgs a;
    float *part;       // [slice][token][max_rank]
    int *order;        // many tokens: by adapter
    int *tiles;        // many tokens: {adapter or -1, first of order, count} each, their number in front
    int *cursor;       // many adapters: scratch, one per adapter and one for none
    int slices;
    int row_groups;    // expand: groups of 64 rows of B of a wave
    bool copy;         // Y is not base
    bool wide;         // base and Y in 16-byte pieces
};

__device__ __forceinline__ int adapter_of(const LoraArgs &a, int t)
{
    const int id = a.adapter[t];
    return id >= 0 && id < a.desc.count ? id : -1;
}

__device__ __forceinline__ int rank_of(const LoraArgs &a, int id)
{
    return id < 0 ? 0 : a.rank ? min(max(a.rank[id], 0), a.desc.max_rank) : a.desc.max_rank;
}

struct Tile {
    int adapter, count;  // count 0: no tile here
};

// The tile of number `slot`, its tokens in `members` (places behind the last hold the first token).  Few tokens: slot is the place of the tile's first
// token, and a token that is not a tile's first has none.
template <int TOKENS, bool FEW>
__device__ __forceinline__ Tile find_tile(const LoraParams &p, int slot, int *members)
{
    const int lane = threadIdx.x & 63;
    Tile tile;
    if (FEW) {
        const int id = lane < p.a.tokens ? adapter_of(p.a, lane) : -2;
        tile.adapter = __builtin_amdgcn_readlane(id, slot);
        const unsigned long long same = __ballot(id == tile.adapter);
        const int before = __popcll(same & ((1ull << slot) - 1));
        if (before % TOKENS) return {-1, 0};
        tile.count = min(__popcll(same) - before, TOKENS);
        const int place = __popcll(same & ((1ull << lane) - 1)) - before;
        if (threadIdx.x < 64) {
            if (lane < TOKENS && lane >= tile.count) members[lane] = slot;
            if (id == tile.adapter && place >= 0 && place < TOKENS) members[place] = lane;
        }
    } else {
        if (slot >= p.tiles[0]) return {-1, 0};
        const int *const t = p.tiles + 1 + 3 * slot;
        tile.adapter = t[0];
        tile.count = t[2];
        if (threadIdx.x < TOKENS) members[threadIdx.x] = p.order[t[1] + (threadIdx.x < tile.count ? threadIdx.x : 0)];
    }
    __syncthreads();
    return tile;
}

}  // namespace

// Many tokens: sorts them by adapter and lists the tiles.  One workgroup; which of an adapter's tokens share a tile has no part in the result.
__global__ __launch_bounds__(1024) void bcq_lora_plan_kernel(LoraParams p, int tile_tokens)
{
    __shared__ int scan_tokens[1024], scan_tiles[1024], few_cursors[kPlanGroups];
    const int tid = threadIdx.x, groups = p.a.desc.count + 1;
    int *const cursor = groups <= kPlanGroups ? few_cursors : p.cursor;
    const auto all_see = [&] {  // (cursors in memory: their atomics pass by the caches of loads and stores)
        if (groups > kPlanGroups) __threadfence();
        __syncthreads();
    };
    for (int g = tid; g < groups; g += 1024) __hip_atomic_store(&cursor[g], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all_see();
    for (int t = tid; t < p.a.tokens; t += 1024) {
        const int id = adapter_of(p.a, t);
        atomicAdd(&cursor[id < 0 ? groups - 1 : id], 1);
    }
    all_see();
    int token_base = 0, tile_base = 0;
    for (int g0 = 0; g0 < groups; g0 += 1024) {
        const int g = g0 + tid, count = g < groups ? __hip_atomic_load(&cursor[g], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
        const int tiles = (count + tile_tokens - 1) / tile_tokens;
        scan_tokens[tid] = count, scan_tiles[tid] = tiles;
        __syncthreads();
        for (int step = 1; step < 1024 && step < groups; step <<= 1) {
            const int a = tid >= step ? scan_tokens[tid - step] : 0, b = tid >= step ? scan_tiles[tid - step] : 0;
            __syncthreads();
            scan_tokens[tid] += a, scan_tiles[tid] += b;
            __syncthreads();
        }
        const int first = token_base + scan_tokens[tid] - count, first_tile = tile_base + scan_tiles[tid] - tiles;
        for (int k = 0; k < tiles; ++k) {
            int *const t = p.tiles + 1 + 3 * (first_tile + k);
            t[0] = g == groups - 1 ? -1 : g;
            t[1] = first + k * tile_tokens;
            t[2] = min(tile_tokens, count - k * tile_tokens);
        }
        if (g < groups) __hip_atomic_store(&cursor[g], first, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int last = min(groups - g0, 1024) - 1;
        token_base += scan_tokens[last], tile_base += scan_tiles[last];
        __syncthreads();
    }
    if (tid == 0) p.tiles[0] = tile_base;
    all_see();
    for (int t = tid; t < p.a.tokens; t += 1024) {
        const int id = adapter_of(p.a, t);
        p.order[atomicAdd(&cursor[id < 0 ? groups - 1 : id], 1)] = t;
    }
}

// NT: tokens of a tile in sixteens.  RT: rows of A of a workgroup in sixteens.
template <bool BF, int NT, int RT, bool FEW>
__global__ __launch_bounds__(64 * kWaves) void bcq_lora_shrink_kernel(LoraParams p)
{
    __shared__ int members[16 * NT];
    __shared__ f32x4 sums[kWaves][NT * RT][64];
    const Tile tile = find_tile<16 * NT, FEW>(p, blockIdx.x, members);
    const int rank = rank_of(p.a, tile.adapter), row0 = blockIdx.z * 16 * RT;
    if (tile.count == 0 || row0 >= rank) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int N = p.a.desc.N, width = p.a.desc.max_rank;
    // steps of 32 columns, cut into slices and those among the waves
    const int steps = (N + 31) / 32, pieces = p.slices * kWaves, piece = blockIdx.y * kWaves + wave;
    const int s0 = (int)((long long)steps * piece / pieces), s1 = (int)((long long)steps * (piece + 1) / pieces);
    const uint16_t *x[NT], *a[RT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) x[nt] = p.a.X + (long long)members[16 * nt + r16] * p.a.ldx + 8 * g;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) a[rt] = p.a.A + ((long long)tile.adapter * width + min(row0 + 16 * rt + r16, rank - 1)) * N + 8 * g;
    f32x4 acc[NT][RT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[nt][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const auto products = [&](const u32x4 (&xr)[NT], const u32x4 (&ar)[RT]) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[nt][rt] = mfma16<BF>(ar[rt], xr[nt], acc[nt][rt]);
    };
    constexpr int kUnroll = NT * RT >= 8 ? 2 : 4;  // steps whose loads are under way together
    int s = s0;
    for (; s + kUnroll <= min(s1, N / 32); s += kUnroll) {
        u32x4 xr[kUnroll][NT], ar[kUnroll][RT];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) ar[k][rt] = *reinterpret_cast<const u32x4 *>(a[rt] + 32 * (s + k));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) xr[k][nt] = *reinterpret_cast<const u32x4 *>(x[nt] + 32 * (s + k));
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) products(xr[k], ar[k]);
    }
    for (; s < s1; ++s) {  // what is left, the last columns among it
        const bool inside = 32 * s + 8 * g < N;
        u32x4 xr[NT], ar[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            ar[rt] = u32x4{0, 0, 0, 0};
            if (inside) ar[rt] = *reinterpret_cast<const u32x4 *>(a[rt] + 32 * s);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            xr[nt] = u32x4{0, 0, 0, 0};
            if (inside) xr[nt] = *reinterpret_cast<const u32x4 *>(x[nt] + 32 * s);
        }
        products(xr, ar);
    }
    // lane (g, r16) has of token r16 the rows 4 g .. 4 g + 3
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) sums[wave][nt * RT + rt][lane] = acc[nt][rt];
    __syncthreads();
    for (int i = wave; i < NT * RT; i += kWaves) {
        const int token = 16 * (i / RT) + r16, row = row0 + 16 * (i % RT) + 4 * g;
        f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += sums[w][i][lane];
        if (token < tile.count && row < width)
            *reinterpret_cast<f32x4 *>(p.part + ((long long)blockIdx.y * p.a.tokens + members[token]) * width + row) = v;
    }
}

// v of a tile as matrix operands in LDS: [part][step of 16][tokens in sixteens][lane] 16 bytes; part 1 (bfloat16 only) the third numbers.
constexpr size_t expand_lds_bytes(bool bf, int tiles, int steps) { return (size_t)(bf ? 2 : 1) * steps * tiles * 1024; }

template <bool BF, int NT, bool FEW>
__global__ __launch_bounds__(64 * kWaves) void bcq_lora_expand_kernel(LoraParams p)
{
    constexpr int kTokens = 16 * NT, kItems = NT == 1 ? 2 : 4;  // eights of v that a thread prepares
    extern __shared__ __attribute__((aligned(16))) u32x4 operand[];
    __shared__ int members[kTokens];
    __shared__ uint32_t largest[kTokens];
    if (threadIdx.x < kTokens) largest[threadIdx.x] = 0;
    const Tile tile = find_tile<kTokens, FEW>(p, blockIdx.x, members);
    if (tile.count == 0) return;
    const int rank = rank_of(p.a, tile.adapter), steps = (rank + 15) / 16;
    if (steps == 0 && !p.copy) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int M = p.a.desc.M, width = p.a.desc.max_rank, third = steps * NT * 64;
    const float scale = tile.adapter >= 0 && p.a.scale ? p.a.scale[tile.adapter] : 1.0f;

    // ---- rows: lane (g, r16) ends up with outputs 8 g .. + 7 of each 32 of token r16: row r of tile q is output 32 (q / 2) + 8 (r / 4) + 4 (q mod 2) + r mod 4.
    // What a group of 64 rows needs first, base and the first columns of B, is requested before v is made, and for the next group before this one's stores ----
    const auto first_row = [&](int group) { return (int)((group * gridDim.y + blockIdx.y) * kWaves + wave) * 64; };  // (the workgroups' rows of one moment are neighbours)
    const int widest = width > 8 ? 8 * (g & 1) : 0;  // (a row of B may have eight columns only; what is loaded twice is masked)
    u32x4 out[NT][2], head[4];
    const uint16_t *b[4];
    const auto request = [&](int row0) {
        if (row0 >= M) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            b[q] = p.a.B + ((long long)max(tile.adapter, 0) * M + min(row0 + 32 * (q >> 1) + 8 * (r16 >> 2) + 4 * (q & 1) + (r16 & 3), M - 1)) * width;
            if (steps) head[q] = *reinterpret_cast<const u32x4 *>(b[q] + widest);
        }
        if (p.wide && row0 + 64 <= M) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    out[nt][h] = *reinterpret_cast<const u32x4 *>(p.a.base + (long long)members[16 * nt + r16] * p.a.ld_base + row0 + 32 * h + 8 * g);
        }
    };
    // ---- v ----
    float v[kItems][8];
    request(first_row(0));
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int item = threadIdx.x + k * 64 * kWaves, token = item % kTokens, j = item / kTokens * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = 0.0f;
        if (j >= rank) continue;
        const float *src = p.part + (long long)members[token] * width + j;
#pragma unroll 4
        for (int s = 0; s < p.slices; ++s, src += (long long)p.a.tokens * width) {
            const f32x4 low = *reinterpret_cast<const f32x4 *>(src), high = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k][i] += low[i], v[k][4 + i] += high[i];
        }
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[k][i] = j + i < rank ? v[k][i] * scale : 0.0f;
            most = fmaxf(most, fabsf(v[k][i]));
        }
        if (!BF) atomicMax(&largest[token], __builtin_bit_cast(uint32_t, most));
    }
    // binary16: the token's largest value is brought to 2^13 .. 2^14
    const auto exponent = [&](int token) { return min(max((int)(largest[token] >> 23) - 127, -100), 100) - 13; };
    if (!BF) __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int item = threadIdx.x + k * 64 * kWaves, token = item % kTokens, eight = item / kTokens;
        if (eight >= 2 * steps) continue;
        u32x4 first, second, rest;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float a = v[k][i], b = v[k][i + 1];
            if (!BF) a = ldexpf(a, -exponent(token)), b = ldexpf(b, -exponent(token));
            uint32_t pair = from_float2<BF>(a, b);
            first[i / 2] = pair;
            f32x2 kept = to_float2<BF>(pair);
            a = fabsf(kept.x) < INFINITY ? a - kept.x : 0.0f, b = fabsf(kept.y) < INFINITY ? b - kept.y : 0.0f;
            second[i / 2] = pair = from_float2<BF>(a, b);
            if (BF) {
                kept = to_float2<BF>(pair);
                rest[i / 2] = from_float2<BF>(a - kept.x, b - kept.y);
            }
        }
        u32x4 *const at = operand + ((eight >> 1) * NT + (token >> 4)) * 64 + (token & 15) + 16 * (eight & 1);
        at[0] = first, at[32] = second;
        if (BF) at[third] = rest, at[third + 32] = u32x4{0, 0, 0, 0};
    }
    __syncthreads();

    u32x4 kept_last;  // of the last step: the columns that belong to the adapter
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 16 * (steps - 1) + 8 * (g & 1) + 2 * i;
        kept_last[i] = (j < rank ? 0xffffu : 0u) | (j + 1 < rank ? 0xffff0000u : 0u);
    }
    for (int group = 0; group < p.row_groups; ++group) {
        const int row0 = first_row(group);
        if (row0 >= M) break;
        const bool vector = p.wide && row0 + 64 <= M;
        f32x4 acc[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[nt][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        u32x4 ahead[4];
        for (int s = 0; s < steps; ++s) {
            u32x4 rows[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) rows[q] = s ? ahead[q] : head[q];
            if (s + 1 < steps) {
                const int at = 16 * (s + 1) + 8 * (g & 1) < width ? 16 * (s + 1) + 8 * (g & 1) : 16 * (s + 1);
#pragma unroll
                for (int q = 0; q < 4; ++q) ahead[q] = *reinterpret_cast<const u32x4 *>(b[q] + at);
            }
            if (s == steps - 1) {
#pragma unroll
                for (int q = 0; q < 4; ++q) rows[q] &= kept_last;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const u32x4 o = operand[(s * NT + nt) * 64 + lane];
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[nt][q] = mfma16<BF>(rows[q], o, acc[nt][q]);
                if (BF) {
                    const u32x4 o3 = operand[third + (s * NT + nt) * 64 + lane];
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[nt][q] = mfma16<BF>(rows[q], o3, acc[nt][q]);
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int token = 16 * nt + r16;
            if (token >= tile.count) continue;
            const float unit = BF || steps == 0 ? 1.0f : ldexpf(1.0f, exponent(token));
            const uint16_t *const base = p.a.base + (long long)members[token] * p.a.ld_base;
            uint16_t *const y = p.a.Y + (long long)members[token] * p.a.ldy;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int m = row0 + 32 * h + 8 * g;
                if (vector) {
                    u32x4 pairs = out[nt][h];
                    if (steps) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const f32x2 x = to_float2<BF>(pairs[i]);
                            const f32x4 a = acc[nt][2 * h + (i >> 1)];
                            pairs[i] = from_float2<BF>(fmaf(a[2 * (i & 1)], unit, x.x), fmaf(a[2 * (i & 1) + 1], unit, x.y));
                        }
                    }
                    *reinterpret_cast<u32x4 *>(y + m) = pairs;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (m + i < M) y[m + i] = steps ? from_float<BF>(fmaf(acc[nt][2 * h + (i >> 2)][i & 3], unit, to_float<BF>(base[m + i]))) : base[m + i];
                }
            }
        }
        if (group + 1 < p.row_groups) request(first_row(group + 1));
    }
}

namespace {

struct LoraPlan {
    int tiles;          // tokens of a tile in sixteens
    int slots;          // most tiles there can be
    int row_tiles, row_blocks;  // shrink: rows of A of a workgroup in sixteens, and how many such blocks
    int slices, row_groups;
    bool few;
    size_t part_bytes, order_bytes, tile_bytes, cursor_bytes;
};

size_t whole(size_t bytes) { return (bytes + 15) & ~(size_t)15; }

LoraPlan lora_plan(const bcq_adapters &d, int tokens)
{
    LoraPlan s;
    s.few = tokens <= kFewTokens;
    // 64 tokens a tile where adapters have 32 or more on average (and their operands leave LDS for three workgroups)
    const int steps = (d.max_rank + 15) / 16;
    s.tiles = !s.few && d.max_rank <= 128 && expand_lds_bytes(d.dtype == BCQ_BF16, 4, steps) <= 48 * 1024 && tokens >= 32LL * d.count ? 4 : 1;
    const int most = tokens < d.count + 1 ? tokens : d.count + 1;
    s.slots = s.few ? tokens : tokens / (16 * s.tiles) + most;
    s.row_tiles = d.max_rank <= 16 ? 1 : d.max_rank <= 32 ? 2 : 4;
    s.row_blocks = (d.max_rank + 16 * s.row_tiles - 1) / (16 * s.row_tiles);
    const int likely = s.few ? (tokens < d.count ? tokens : d.count) : s.slots;  // tiles, if adapters are spread
    const int wanted = 2 * compute_units() / (likely * s.row_blocks), longest = (d.N + 511) / 512;
    s.slices = wanted < longest ? wanted : longest;
    // (with 64 tokens a tile there is work enough, and every workgroup of the second launch reads all slices: 4 slices 124 us, 13 134, 2 140 for 2048 tokens,
    // rank 64, 7168 to 28672; one token, rank 64, 28672 to 7168: 16 slices 17 us, 8 23, 4 38)
    const int cap = s.tiles == 4 ? 4 : 16;
    s.slices = s.slices < 1 ? 1 : s.slices > cap ? cap : s.slices;
    const int blocks = (d.M + 64 * kWaves - 1) / (64 * kWaves);
    // as many workgroups as the chip holds at once (registers: two to a compute unit with 64 tokens, four with 16), so that each makes v once
    const long long resident = (s.tiles == 4 ? 2 : 4) * compute_units(), groups = ((long long)blocks * (s.few ? likely : tokens / (16 * s.tiles) + 1) + resident - 1) / resident;
    s.row_groups = (int)(groups < 1 ? 1 : groups > 16 ? 16 : groups);
    s.part_bytes = whole((size_t)s.slices * tokens * d.max_rank * sizeof(float));
    s.order_bytes = s.few ? 0 : whole((size_t)tokens * sizeof(int));
    s.tile_bytes = s.few ? 0 : whole((size_t)(1 + 3 * s.slots) * sizeof(int));
    s.cursor_bytes = s.few || d.count + 1 <= kPlanGroups ? 0 : whole((size_t)(d.count + 1) * sizeof(int));
    return s;
}

template <bool BF, int NT, bool FEW>
hipError_t launch(const LoraParams &p, const LoraPlan &s, hipStream_t stream)
{
    const dim3 shrink(s.slots, s.slices, s.row_blocks);
    if (s.row_tiles == 1) bcq_lora_shrink_kernel<BF, NT, 1, FEW><<<shrink, 64 * kWaves, 0, stream>>>(p);
    else if (s.row_tiles == 2) bcq_lora_shrink_kernel<BF, NT, 2, FEW><<<shrink, 64 * kWaves, 0, stream>>>(p);
    else bcq_lora_shrink_kernel<BF, NT, 4, FEW><<<shrink, 64 * kWaves, 0, stream>>>(p);
    const int rows = 64 * kWaves * s.row_groups;
    const dim3 expand(s.slots, (p.a.desc.M + rows - 1) / rows);
    const size_t lds = expand_lds_bytes(BF, NT, (p.a.desc.max_rank + 15) / 16);
    bcq_lora_expand_kernel<BF, NT, FEW><<<expand, 64 * kWaves, lds, stream>>>(p);
    return hipGetLastError();
}

template <bool BF>
hipError_t by_plan(const LoraParams &p, const LoraPlan &s, hipStream_t stream)
{
    if (s.few) return launch<BF, 1, true>(p, s, stream);
    bcq_lora_plan_kernel<<<1, 1024, 0, stream>>>(p, 16 * s.tiles);
    return s.tiles == 4 ? launch<BF, 4, false>(p, s, stream) : launch<BF, 1, false>(p, s, stream);
}

}  // namespace

size_t lora_workspace_bytes(const bcq_adapters &d, int tokens)
{
    const LoraPlan s = lora_plan(d, tokens);
    return s.part_bytes + s.order_bytes + s.tile_bytes + s.cursor_bytes;
}

hipError_t launch_lora(const LoraArgs &a, hipStream_t stream)
{
    const LoraPlan s = lora_plan(a.desc, a.tokens);
    LoraParams p;
    p.a = a;
    char *at = static_cast<char *>(a.workspace);
    p.part = reinterpret_cast<float *>(at);
    p.order = reinterpret_cast<int *>(at += s.part_bytes);
    p.tiles = reinterpret_cast<int *>(at += s.order_bytes);
    p.cursor = reinterpret_cast<int *>(at + s.tile_bytes);
    p.slices = s.slices;
    p.row_groups = s.row_groups;
    p.copy = a.Y != a.base;
    p.wide = a.ld_base % 8 == 0 && a.ldy % 8 == 0 && ((reinterpret_cast<uintptr_t>(a.base) | reinterpret_cast<uintptr_t>(a.Y)) & 15) == 0;
    return a.desc.dtype == BCQ_BF16 ? by_plan<true>(p, s, stream) : by_plan<false>(p, s, stream);
}

}  // namespace bcq
