// Low-rank adapters of many requests beside a shared projection:  Y[t] = base[t] + scale[a] * B[a] (A[a] X[t]),  a = adapter[t].
//
// Bound by the bytes: A and B of the adapters that occur, and with many tokens X, base and Y.  Tokens of the same adapter are taken together, 16 or 64
// at a time (a tile), so that a piece of A or B is read once for them and the sums run on the matrix cores.  Up to 64 tokens every wave finds
// its tile's tokens by comparing all adapter numbers at once; beyond, a small launch sorts the tokens by adapter first (plan).  Then:
//
//  * v = A x (shrink): a workgroup has a tile, 16 to 64 rows of A and a slice of N; its waves share the slice and add up in LDS.  The slices, as many as fill
//    the chip, leave their sums in binary32 side by side, and whoever reads them adds them in order.
//  * Y = base + B v (expand): a workgroup has a tile and a range of rows of B.  v (times the scale) is held as a sum of 16-bit numbers beside the 16-bit rows of B:
//    two for binary16 (after a power of two for each token: 21 bits and more of its largest value), three for bfloat16 (23 bits).  The operand's 32
//    places are 16 of v's first numbers and the same 16 of its second ones.  The rows of B are numbered so that a lane ends up with eight
//    neighbouring outputs of a token and four lanes with 32.
//  * Many tokens of few adapters: v is turned into operands once (pack), and rows of B go through LDS for 64 tokens (many).
//  * One token of a small adapter: one launch, each workgroup makes v for itself (one).
//
// Measured: rank 16, 8192 to 10240: one token 6.1 us (8.6 with shrink and expand), 64 tokens of 32 adapters 14 (shrink 6.4, expand 8: a launch and four reads
// in a row each); 2048 tokens of 4 adapters of rank 64, 7168 to 28672, bfloat16: 98 us (plan 5, shrink 17, pack 5, many 70: 235 MB of base and Y at 3.4 TB/s;
// its loads and stores of 16 rows each cost 64 clocks of the address unit, a third of the time, matrix and vector pipes and LDS a fifth each, and a barrier for
// every 64 rows keeps them apart).  First kernels without matrix
// instructions took 19, 67 us and 11.8 ms.
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

namespace {

constexpr int kWaves = 4;
constexpr int kFewTokens = 64;     // that every wave sorts out by itself
constexpr int kManyTokens = 64;    // a tile where adapters have many
constexpr long long kOneElements = 240 * 1024;  // of an adapter's A that every workgroup may read for itself
constexpr int kPlanGroups = 4096;  // adapters (and none) whose tokens are counted in LDS

// Sixteen bytes of base and Y, whose rows begin anywhere.  (785 tokens, 25 adapters of rank 17, 15248 to 25668, where rows are not whole pieces: 63 us, element by
// element 147.)
typedef u32x4 u32x4_even __attribute__((aligned(2)));

struct LoraParams {
    LoraArgs a;
    float *part;       // [slice][token][max_rank]
    int *order;        // more than kFewTokens: tokens by tile; behind a tile's last one nothing
    int *tiles;        // more than kFewTokens: {adapter or -1, tokens} each, their number in front
    int *cursor;       // many adapters: scratch, one per adapter and one for none
    u32x4 *operands;   // many tokens of few adapters: v as matrix operands, by tile
    float *units;      // and what they are to be multiplied by, [tile][64]
    int operand_pieces;  // 16-byte pieces of sixteen tokens' operands
    int slices;
    int row_groups;    // expand: groups of 64 rows of B of a wave
    bool copy;         // Y is not base
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
        tile.adapter = p.tiles[2 + 2 * slot];
        tile.count = p.tiles[3 + 2 * slot];
        if (threadIdx.x < TOKENS) members[threadIdx.x] = p.order[slot * TOKENS + (threadIdx.x < tile.count ? threadIdx.x : 0)];
    }
    __syncthreads();
    return tile;
}

}  // namespace

// Many tokens: sorts them by adapter and lists the tiles.  One workgroup; which of an adapter's tokens share a tile has no part in the result.
__global__ __launch_bounds__(1024) void bcq_lora_plan_kernel(LoraParams p, int tile_tokens)
{
    __shared__ int scan[1024], few_cursors[kPlanGroups];
    const int tid = threadIdx.x, groups = p.a.desc.count + 1;
    int *const cursor = groups <= kPlanGroups ? few_cursors : p.cursor;
    const auto all_see = [&] {  // (cursors in memory: their atomics pass by the caches of loads and stores)
        if (groups > kPlanGroups) __threadfence();
        __syncthreads();
    };
    for (int g = tid; g < groups; g += 1024) __hip_atomic_store(&cursor[g], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all_see();
    // this lane's place among all that add one to the same cursor: one atomic for each of a wave's adapters (a request's tokens are neighbours)
    const auto next_of = [&](int g) {
        int place = 0;
        for (unsigned long long left = __ballot(g >= 0); left;) {
            const int one = __builtin_amdgcn_readlane(g, __builtin_ctzll(left));
            const unsigned long long same = __ballot(g == one);
            int from = 0;
            if ((threadIdx.x & 63) == (unsigned)__builtin_ctzll(left)) from = atomicAdd(&cursor[one], __popcll(same));
            from = __builtin_amdgcn_readlane(from, __builtin_ctzll(left));
            if (g == one) place = from + __popcll(same & ((1ull << (threadIdx.x & 63)) - 1));
            left &= ~same;
        }
        return place;
    };
    const auto group_of = [&](int t) {
        if (t >= p.a.tokens) return -1;
        const int id = adapter_of(p.a, t);
        return id < 0 ? groups - 1 : id;
    };
    for (int t = 0; t < p.a.tokens; t += 1024) next_of(group_of(t + tid));
    all_see();
    int tile_base = 0;
    for (int g0 = 0; g0 < groups; g0 += 1024) {
        const int g = g0 + tid, count = g < groups ? __hip_atomic_load(&cursor[g], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
        const int tiles = (count + tile_tokens - 1) / tile_tokens;
        scan[tid] = tiles;
        __syncthreads();
        for (int step = 1; step < 1024 && step < groups; step <<= 1) {
            const int before = tid >= step ? scan[tid - step] : 0;
            __syncthreads();
            scan[tid] += before;
            __syncthreads();
        }
        const int first = tile_base + scan[tid] - tiles;
        for (int k = 0; k < tiles; ++k) {
            p.tiles[2 + 2 * (first + k)] = g == groups - 1 ? -1 : g;
            p.tiles[3 + 2 * (first + k)] = min(tile_tokens, count - k * tile_tokens);
        }
        if (g < groups) __hip_atomic_store(&cursor[g], first * tile_tokens, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        tile_base += scan[min(groups - g0, 1024) - 1];
        __syncthreads();
    }
    if (tid == 0) p.tiles[0] = tile_base;
    all_see();
    for (int t = 0; t < p.a.tokens; t += 1024) {
        const int place = next_of(group_of(t + tid));
        if (t + tid < p.a.tokens) p.order[place] = t + tid;
    }
}

// Sums of the steps s0 .. s1 - 1 of 32 columns: RT sixteens of rows of A[adapter] from row0 on, times NT sixteens of tokens, those of this lane's columns in
// `tokens`.  Rows behind the rank are copies of its last.
template <bool BF, int NT, int RT>
__device__ __forceinline__ void shrink_products(const LoraArgs &p, int adapter, const int (&tokens)[NT], int row0, int rank, int s0, int s1, int lane,
                                                f32x4 (&acc)[NT][RT])
{
    const int r16 = lane & 15, g = lane >> 4, N = p.desc.N;
    const uint16_t *x[NT], *a[RT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) x[nt] = p.X + (long long)tokens[nt] * p.ldx + 8 * g;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) a[rt] = p.A + ((long long)adapter * p.desc.max_rank + min(row0 + 16 * rt + r16, rank - 1)) * N + 8 * g;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[nt][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // Steps whose loads are under way together, and as many that are used meanwhile (the compiler would rather save the registers and load one at a time).
    constexpr int kUnroll = NT + RT > 5 ? 2 : 4;
    u32x4 xr[2][kUnroll][NT], ar[2][kUnroll][RT];
    const auto load = [&](int s, int to) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) ar[to][k][rt] = *reinterpret_cast<const u32x4 *>(a[rt] + 32 * (s + k));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) xr[to][k][nt] = *reinterpret_cast<const u32x4 *>(x[nt] + 32 * (s + k));
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto products = [&](int of) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) acc[nt][rt] = mfma16<BF>(ar[of][k][rt], xr[of][k][nt], acc[nt][rt]);
        __builtin_amdgcn_sched_barrier(0);
    };
    const int batches = max(min(s1, N / 32) - s0, 0) / kUnroll;
    int s = s0;
    if (batches > 0) load(s, 0);
    for (int i = 0; i < batches; i += 2) {
        if (i + 1 < batches) load(s + kUnroll, 1);
        products(0);
        if (i + 1 < batches) {
            if (i + 2 < batches) load(s + 2 * kUnroll, 0);
            products(1);
        }
        s += 2 * kUnroll;
    }
    for (s = s0 + batches * kUnroll; s < s1; ++s) {  // what is left, the last columns among it
        const bool inside = 32 * s + 8 * g < N;
        u32x4 x1[NT], a1[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            a1[rt] = u32x4{0, 0, 0, 0};
            if (inside) a1[rt] = *reinterpret_cast<const u32x4 *>(a[rt] + 32 * s);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            x1[nt] = u32x4{0, 0, 0, 0};
            if (inside) x1[nt] = *reinterpret_cast<const u32x4 *>(x[nt] + 32 * s);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[nt][rt] = mfma16<BF>(a1[rt], x1[nt], acc[nt][rt]);
        }
    }
}

// A product's row r of tile q is output 32 (q / 2) + 8 (r / 4) + 4 (q mod 2) + r mod 4 of a group of 64, so that lane (g, r16) ends up with the outputs
// 8 g .. + 7 of each 32 of token r16.
__device__ __forceinline__ int row_of(int r16, int q) { return 32 * (q >> 1) + 8 * (r16 >> 2) + 4 * (q & 1) + (r16 & 3); }

template <bool BF>
__device__ __forceinline__ u32x4 add_pairs(u32x4 base, f32x4 low, f32x4 high, float unit)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 x = to_float2<BF>(base[i]);
        const f32x4 a = i < 2 ? low : high;
        base[i] = from_float2<BF>(fmaf(a[2 * (i & 1)], unit, x.x), fmaf(a[2 * (i & 1) + 1], unit, x.y));
    }
    return base;
}

// Y = base + unit * (low, high) for eight outputs of a token from m on, as far as there are so many; without an adapter they are the base bit for bit.
template <bool BF>
__device__ __forceinline__ void store_ends(const LoraArgs &p, int token, int m, bool adapted, float unit, f32x4 low, f32x4 high)
{
    const uint16_t *const base = p.base + (long long)token * p.ld_base;
    uint16_t *const y = p.Y + (long long)token * p.ldy;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (m + i < p.desc.M) y[m + i] = adapted ? from_float<BF>(fmaf(i < 4 ? low[i & 3] : high[i & 3], unit, to_float<BF>(base[m + i]))) : base[m + i];
}

// All of a lane's outputs of a token, in the order that the products leave: 8 g .. + 7 of each 32.  `loaded` holds the base where all 64 exist (whole).
template <bool BF>
__device__ __forceinline__ void store_rows(const LoraArgs &p, int token, int row0, int lane, bool whole, bool adapted, float unit, const u32x4 (&loaded)[2],
                                           const f32x4 (&acc)[4])
{
    uint16_t *const y = p.Y + (long long)token * p.ldy;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int m = row0 + 32 * h + 8 * (lane >> 4);
        if (whole) *reinterpret_cast<u32x4_even *>(y + m) = adapted ? add_pairs<BF>(loaded[h], acc[2 * h], acc[2 * h + 1], unit) : loaded[h];
        else store_ends<BF>(p, token, m, adapted, unit, acc[2 * h], acc[2 * h + 1]);
    }
}

// binary16: v's largest value is brought to 2^13 .. 2^14; its bits -> the power of two to divide by.
__device__ __forceinline__ int power_of(uint32_t largest) { return min(max((int)(largest >> 23) - 127, -100), 100) - 13; }

// Two values of v as sums of 16-bit numbers, all of a value's sign and none of them zero unless it is: an infinity among B's weights is then one of the result, as it
// is without the split, where a zero or a second number of the other sign would make a NaN of it.  (What that adds, 2^-24 beside 2^13 or 2^-126, is behind the last
// bit.)  Nothing is left of an infinity or a NaN.  binary16: first and second; bfloat16: third too, half of what is left, which is used twice.
template <bool BF>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t &first, uint32_t &second, uint32_t &third)
{
    const uint32_t tiny = (a != 0.0f ? (BF ? 0x0080u : 1u) : 0u) | (b != 0.0f ? (BF ? 0x00800000u : 0x10000u) : 0u);
    const uint32_t sign = (__builtin_bit_cast(uint32_t, a) >> 16 & 0x8000u) | (__builtin_bit_cast(uint32_t, b) & 0x80000000u);
    const auto no_zero = [&](uint32_t pair) {
        if (!(pair & 0x7fffu)) pair |= (tiny | sign) & 0xffffu;
        if (!(pair & 0x7fff0000u)) pair |= (tiny | sign) & 0xffff0000u;
        return pair;
    };
    first = toward_zero2<BF>(a, b);
    f32x2 kept = to_float2<BF>(first);
    a = fabsf(kept.x) < INFINITY ? a - kept.x : 0.0f, b = fabsf(kept.y) < INFINITY ? b - kept.y : 0.0f;
    second = BF ? toward_zero2<BF>(a, b) : from_float2<BF>(a, b);
    kept = to_float2<BF>(second);
    third = BF ? no_zero(from_float2<BF>(0.5f * (a - kept.x), 0.5f * (b - kept.y))) : 0u;
    first = no_zero(first), second = no_zero(second);
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
    const int width = p.a.desc.max_rank;
    // steps of 32 columns, cut into slices and those among the waves
    const int steps = (p.a.desc.N + 31) / 32, pieces = p.slices * kWaves, piece = blockIdx.y * kWaves + wave;
    const int s0 = (int)((long long)steps * piece / pieces), s1 = (int)((long long)steps * (piece + 1) / pieces);
    int tokens[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) tokens[nt] = members[16 * nt + r16];
    f32x4 acc[NT][RT];
    shrink_products<BF, NT, RT>(p.a, tile.adapter, tokens, row0, rank, s0, s1, lane, acc);
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

// v of sixteen tokens as matrix operands: [part][step of 16][lane] 16 bytes; part 1 (bfloat16 only) the third numbers, twice their halves.
constexpr size_t operand_bytes(bool bf, int steps) { return (size_t)(bf ? 2 : 1) * steps * 1024; }

// Adds up the slices of v of sixteen tokens and turns it into operands.  binary16: largest[] (zeros before) becomes each token's largest value's bits, of
// which power_of() is what it was divided by.  For all of a workgroup's threads.
template <bool BF>
__device__ __forceinline__ void make_operands(const LoraParams &p, int adapter, int rank, const int *members, uint32_t *largest, u32x4 *operands)
{
    constexpr int kItems = 16 * BCQ_MAX_RANK / 8 / (64 * kWaves);  // eights of v of a thread
    const int steps = (rank + 15) / 16, width = p.a.desc.max_rank;
    const float scale = p.a.scale && adapter >= 0 ? p.a.scale[adapter] : 1.0f;
    float v[kItems][8];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int item = threadIdx.x + k * 64 * kWaves, token = item % 16, j = item / 16 * 8;
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
    if (!BF) __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int item = threadIdx.x + k * 64 * kWaves, token = item % 16, eight = item / 16;
        if (eight >= 2 * steps) continue;
        const int power = BF ? 0 : power_of(largest[token]);
        u32x4 first, second, rest;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint32_t x, y, z;
            split_pair<BF>(BF ? v[k][i] : ldexpf(v[k][i], -power), BF ? v[k][i + 1] : ldexpf(v[k][i + 1], -power), x, y, z);
            first[i / 2] = x, second[i / 2] = y, rest[i / 2] = z;
        }
        u32x4 *const at = operands + (eight >> 1) * 64 + token + 16 * (eight & 1);
        at[0] = first, at[32] = second;
        if (BF) at[64 * steps] = rest, at[64 * steps + 32] = rest;
    }
}

template <bool BF, bool FEW>
__global__ __launch_bounds__(64 * kWaves) void bcq_lora_expand_kernel(LoraParams p)
{
    constexpr int kTokens = 16;
    extern __shared__ __attribute__((aligned(16))) u32x4 operand[];
    __shared__ int members[kTokens];
    __shared__ uint32_t largest[kTokens];
    if (threadIdx.x < kTokens) largest[threadIdx.x] = 0;
    const Tile tile = find_tile<kTokens, FEW>(p, blockIdx.x, members);
    if (tile.count == 0) return;
    const int rank = rank_of(p.a, tile.adapter), steps = (rank + 15) / 16;
    if (steps == 0 && !p.copy) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int M = p.a.desc.M, width = p.a.desc.max_rank, third = steps * 64;
    // What a group of 64 rows needs first, base and the first columns of B, is requested before v is made, and for the next group before this one's stores.
    const auto first_row = [&](int group) { return (int)((group * gridDim.y + blockIdx.y) * kWaves + wave) * 64; };  // (the workgroups' rows of one moment are neighbours)
    const int widest = width > 8 ? 8 * (g & 1) : 0;  // (a row of B may have eight columns only; what is loaded twice is masked)
    u32x4 out[2], head[4];
    const uint16_t *b[4];
    const auto request = [&](int row0) {
        if (row0 >= M) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            b[q] = p.a.B + ((long long)max(tile.adapter, 0) * M + min(row0 + row_of(r16, q), M - 1)) * width;
            if (steps) head[q] = *reinterpret_cast<const u32x4 *>(b[q] + widest);
        }
        if (row0 + 64 <= M) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                out[h] = *reinterpret_cast<const u32x4_even *>(p.a.base + (long long)members[r16] * p.a.ld_base + row0 + 32 * h + 8 * g);
        }
    };
    request(first_row(0));
    make_operands<BF>(p, tile.adapter, rank, members, largest, operand);
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
        const bool vector = row0 + 64 <= M;
        f32x4 acc[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
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
            const u32x4 o = operand[s * 64 + lane];
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[q] = mfma16<BF>(rows[q], o, acc[q]);
            if (BF) {
                const u32x4 o3 = operand[third + s * 64 + lane];
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[q] = mfma16<BF>(rows[q], o3, acc[q]);
            }
        }
        if (r16 < tile.count) {
            const float unit = BF || steps == 0 ? 1.0f : ldexpf(1.0f, power_of(largest[r16]));
            store_rows<BF>(p.a, members[r16], row0, lane, vector, steps != 0, unit, out, acc);
        }
        if (group + 1 < p.row_groups) request(first_row(group + 1));
    }
}

// ---- one token of a small adapter: one launch, in which every workgroup makes v for itself ----

constexpr int kOneWaves = 8;

// acc + the dot product of eight pairs, in binary32.
template <bool BF>
__device__ __forceinline__ float dot8(u32x4 a, u32x4 x, float acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 p = to_float2<BF>(a[i]), q = to_float2<BF>(x[i]);
        acc = fmaf(p.y, q.y, fmaf(p.x, q.x, acc));
    }
    return acc;
}

// The sums over a wave's lanes of COUNT values each (a power of two up to 64): lane l gets that of value l / (64 / COUNT).
template <int COUNT, int STEP = 32>
__device__ __forceinline__ float sum_over_lanes(const float (&v)[COUNT], int lane)
{
    constexpr int kHalf = COUNT > 1 ? COUNT / 2 : 1;
    float half[kHalf];
    if (COUNT > 1) {
        const bool upper = (lane & STEP) != 0;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            const float low = v[i], high = v[COUNT > 1 ? i + kHalf : 0];
            half[i] = (upper ? high : low) + __shfl_xor(upper ? low : high, STEP);
        }
    } else {
        half[0] = v[0] + __shfl_xor(v[0], STEP);
    }
    if constexpr (STEP == 1) return half[0];
    else return sum_over_lanes<kHalf, STEP / 2>(half, lane);
}

// A workgroup has p.row_groups * 512 rows of B, a row to a thread.  Each reads all of A, contiguously, 512 columns of sixteen rows a wave at a time.
template <bool BF>
__global__ __launch_bounds__(64 * kOneWaves) void bcq_lora_one_kernel(LoraParams p)
{
    __shared__ float sums[kOneWaves][16];
    __shared__ __attribute__((aligned(16))) float v[BCQ_MAX_RANK];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int M = p.a.desc.M, N = p.a.desc.N, width = p.a.desc.max_rank;
    const int adapter = adapter_of(p.a, 0), rank = rank_of(p.a, adapter);
    if (rank == 0 && !p.copy) return;
    const int first = blockIdx.x * p.row_groups * 64 * kOneWaves + threadIdx.x;
    const uint16_t *const b = p.a.B + (long long)max(adapter, 0) * M * width;
    // the first row of B, its first sixteen columns, and its base are on their way while v is made
    u32x4 head[2] = {};
    uint16_t base = p.a.base[min(first, M - 1)];
    if (rank) {
        const uint16_t *const row = b + (long long)min(first, M - 1) * width;
        head[0] = *reinterpret_cast<const u32x4 *>(row), head[1] = *reinterpret_cast<const u32x4 *>(row + (width > 8 ? 8 : 0));
        const char *const a = reinterpret_cast<const char *>(p.a.A + (long long)adapter * width * N);
        const float scale = p.a.scale ? p.a.scale[adapter] : 1.0f;
        for (int row0 = 0; row0 < rank; row0 += 16) {
            float acc[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[j] = 0.0f;
            for (int col = 512 * wave; col < N; col += 512 * kOneWaves) {
                const int mine = col + 8 * lane;
                u32x4 x = {0, 0, 0, 0}, rows[16];
                if (mine < N) x = *reinterpret_cast<const u32x4 *>(p.a.X + mine);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    rows[j] = u32x4{0, 0, 0, 0};
                    if (mine < N) rows[j] = *reinterpret_cast<const u32x4 *>(a + 2u * (unsigned)(min(row0 + j, rank - 1) * N + mine));
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[j] = dot8<BF>(rows[j], x, acc[j]);
            }
            const float mine = sum_over_lanes<16>(acc, lane);
            if ((lane & 3) == 0) sums[wave][lane >> 2] = mine;
            __syncthreads();
            if (threadIdx.x < 16) {
                float all = 0.0f;
#pragma unroll
                for (int w = 0; w < kOneWaves; ++w) all += sums[w][threadIdx.x];
                v[row0 + threadIdx.x] = all * scale;
            }
            __syncthreads();
        }
    }
    for (int group = 0; group < p.row_groups; ++group) {
        const int m = first + group * 64 * kOneWaves;
        if (m >= M) break;
        if (group) base = p.a.base[m];
        const uint16_t *const row = b + (long long)m * width;
        float acc = 0.0f;
        for (int j = 0; j < rank; j += 8) {
            const u32x4 eight = group == 0 && j < 16 ? (j ? head[1] : head[0]) : *reinterpret_cast<const u32x4 *>(row + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2 pair = to_float2<BF>(eight[i]);
                // (columns behind the rank hold anything)
                acc = fmaf(j + 2 * i < rank ? pair.x : 0.0f, j + 2 * i < rank ? v[j + 2 * i] : 0.0f, acc);
                acc = fmaf(j + 2 * i + 1 < rank ? pair.y : 0.0f, j + 2 * i + 1 < rank ? v[j + 2 * i + 1] : 0.0f, acc);
            }
        }
        p.a.Y[m] = rank ? from_float<BF>(to_float<BF>(base) + acc) : base;
    }
}

// ---- many tokens: v is turned into operands once, and waves that share nothing but the caches go by the rows of B ----

template <bool BF>
__global__ __launch_bounds__(64 * kWaves) void bcq_lora_pack_kernel(LoraParams p)
{
    __shared__ int members[kManyTokens];
    __shared__ uint32_t largest[16];
    if (threadIdx.x < 16) largest[threadIdx.x] = 0;
    const Tile tile = find_tile<kManyTokens, false>(p, blockIdx.x, members);
    const int rank = rank_of(p.a, tile.adapter), sixteen = blockIdx.y;
    if (rank == 0 || 16 * sixteen >= tile.count) return;
    make_operands<BF>(p, tile.adapter, rank, members + 16 * sixteen, largest, p.operands + (size_t)(blockIdx.x * (kManyTokens / 16) + sixteen) * p.operand_pieces);
    if (!BF) {
        __syncthreads();
        if (threadIdx.x < 16) p.units[blockIdx.x * kManyTokens + 16 * sixteen + threadIdx.x] = ldexpf(1.0f, power_of(largest[threadIdx.x]));
    }
}

// A workgroup has a tile, 16 tokens a wave, whose operands stay in registers, and walks row_groups groups of 64 rows of B.  These come through LDS (two buffers, a
// row 16 bytes longer than it is, without which 16 rows' pieces of one column would meet few banks; numbered as row_of() has it, two rows meet in eight places, which is
// 44 % of the kernel's LDS cycles and a tenth of its time): read in the operand's layout from memory, sixteen rows' 32 bytes each, a
// load costs four times a contiguous one, and there would be four times as many.  Rows of the next group and base of the next two are on
// their way during this one.
// ST: steps that the operands have at most.
constexpr int many_occupancy(int steps) { return steps == 8 ? 2 : steps == 1 ? 6 : 4; }  // workgroups of a compute unit: what the registers allow
template <bool BF, int ST>
__global__ __launch_bounds__(64 * kWaves, many_occupancy(ST)) void bcq_lora_many_kernel(LoraParams p)
{
    constexpr int kParts = BF ? 2 : 1, kOwn = (64 * 2 * ST + 64 * kWaves - 1) / (64 * kWaves);  // 16-byte pieces of a group's rows that a thread brings
    __shared__ u32x4 rows_lds[2][64 * (2 * ST + 1)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int slot = blockIdx.y, M = p.a.desc.M, width = p.a.desc.max_rank;
    if (slot >= p.tiles[0]) return;
    const int adapter = p.tiles[2 + 2 * slot], count = p.tiles[3 + 2 * slot] - 16 * wave;
    const int rank = rank_of(p.a, adapter), steps = (rank + 15) / 16;
    if (steps == 0 && !p.copy) return;
    // Low ranks: base and Y in whole lines.  A load or store takes all 64 outputs of eight tokens, the first and then the second eight; lanes r16 and r16 ^ 8 exchange what
    // is the other's.  (In the order that the products leave, 32 outputs of sixteen tokens, an instruction costs twice the time of the address unit: 4096 tokens of rank 16,
    // 4096 to 4096, 47 us against 41.  High ranks gain nothing, 57.3 and 57.5 us with 2048 tokens of rank 64, 8192 to 10240, and lack the registers.)
    // 32 outputs after the other, because sixteen registers less are two workgroups more.
    constexpr bool kLines = ST <= 2;
    const bool upper = r16 & 8;
    const auto place_of = [&](int i) { return kLines ? (r16 & 7) + 8 * i : r16; };         // of the lane's i-th piece: token of the wave
    const auto column_of = [&](int i) { return 8 * g + 32 * (kLines ? upper : i); };        // and output of a group
    int tokens[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) tokens[i] = p.order[slot * kManyTokens + (place_of(i) < count ? 16 * wave + place_of(i) : 0)];
    const auto exchange = [&](u32x4 (&x)[2]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t give = upper ? x[0][e] : x[1][e];
            const uint32_t got = __builtin_amdgcn_mov_dpp(give, 0x128, 0xf, 0xf, true);  // row_ror:8
            x[0][e] = upper ? got : x[0][e];
            x[1][e] = upper ? x[1][e] : got;
        }
    };
    const float unit = BF ? 1.0f : p.units[slot * kManyTokens + 16 * wave + r16];
    u32x4 v[kParts][ST];
    const u32x4 *const operands = p.operands + (size_t)(slot * (kManyTokens / 16) + wave) * p.operand_pieces;
#pragma unroll
    for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int s = 0; s < ST; ++s)
            if (s < steps) v[part][s] = operands[(part * steps + s) * 64 + lane];
    // pieces of a row, and where the piece number threadIdx.x + 256 i of a group goes
    const int pieces = width >> 3;
    int place[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) place[i] = threadIdx.x + i * 64 * kWaves + (threadIdx.x + i * 64 * kWaves) / pieces;
    const uint16_t *const b = p.a.B + (long long)max(adapter, 0) * M * width;
    u32x4 own[kOwn], base[2], next_base[2], later_base[2];  // base two groups ahead: a load takes longer than a group
    const auto first_row = [&](int group) { return (int)(group * gridDim.x + blockIdx.x) * 64; };
    const auto fetch = [&](int row0) {
        if (steps == 0) return;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            if (place[i] < 64 * (pieces + 1)) own[i] = *reinterpret_cast<const u32x4 *>(b + min((long long)row0 * width + 8 * (threadIdx.x + i * 64 * kWaves), (long long)M * width - 8));
    };
    const auto put = [&](u32x4 *to) {
        if (steps == 0) return;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            if (rank < width) {  // columns behind the rank hold anything
                const int first = 8 * (place[i] % (pieces + 1));
#pragma unroll
                for (int e = 0; e < 4; ++e) own[i][e] &= (first + 2 * e < rank ? 0xffffu : 0u) | (first + 2 * e + 1 < rank ? 0xffff0000u : 0u);
            }
            if (place[i] < 64 * (pieces + 1)) to[place[i]] = own[i];
        }
    };
    const auto request = [&](int row0, u32x4 (&to)[2]) {
        if (row0 + 64 > M) return;
#pragma unroll
        for (int i = 0; i < 2; ++i) to[i] = *reinterpret_cast<const u32x4_even *>(p.a.base + (long long)tokens[kLines ? i : 0] * p.a.ld_base + row0 + column_of(i));
    };
    int groups = p.row_groups;  // those that exist
    while (groups > 0 && first_row(groups - 1) >= M) --groups;
    if (groups == 0) return;
    if (threadIdx.x < 128) rows_lds[threadIdx.x >> 6][(threadIdx.x & 63) * (pieces + 1) + pieces] = u32x4{0, 0, 0, 0};  // (a row may end in the first eight of a sixteen)
    fetch(first_row(0));
    request(first_row(0), base);
    if (groups > 1) request(first_row(1), next_base);
    put(rows_lds[0]);
    if (groups > 1) fetch(first_row(1));
    __syncthreads();
    for (int group = 0; group < groups; ++group) {
        const int row0 = first_row(group);
        if (group + 2 < groups) request(first_row(group + 2), later_base);
        const bool whole = row0 + 64 <= M;
        const u32x4 *const at = rows_lds[group & 1];
        const auto next_rows = [&] {
            if (group + 1 < groups) put(rows_lds[(group + 1) & 1]);
            if (group + 2 < groups) fetch(first_row(group + 2));
        };
        if constexpr (kLines) {
            if (whole && steps) exchange(base);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 acc[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
                if (count > 0) {
#pragma unroll
                    for (int s = 0; s < ST; ++s) {
                        if (s >= steps) break;
                        u32x4 rows[2];
#pragma unroll
                        for (int q = 0; q < 2; ++q) rows[q] = at[row_of(r16, 2 * h + q) * (pieces + 1) + 2 * s + (g & 1)];
#pragma unroll
                        for (int part = 0; part < kParts; ++part)
#pragma unroll
                            for (int q = 0; q < 2; ++q) acc[q] = mfma16<BF>(rows[q], v[part][s], acc[q]);
                    }
                }
                if (whole && steps) base[h] = add_pairs<BF>(base[h], acc[0], acc[1], unit);
                else if (!whole && r16 < count) store_ends<BF>(p.a, (upper ? tokens[1] : tokens[0]), row0 + 32 * h + 8 * g, steps != 0, unit, acc[0], acc[1]);
                __builtin_amdgcn_sched_barrier(0);
            }
            next_rows();
            if (whole) {
                if (steps) exchange(base);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (place_of(i) < count)
                        __builtin_nontemporal_store(base[i], reinterpret_cast<u32x4_even *>(p.a.Y + (long long)tokens[i] * p.a.ldy + row0 + column_of(i)));
            }
        } else {
            f32x4 acc[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (count > 0) {
#pragma unroll
                for (int s = 0; s < ST; ++s) {
                    if (s >= steps) break;
                    u32x4 rows[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) rows[q] = at[row_of(r16, q) * (pieces + 1) + 2 * s + (g & 1)];
#pragma unroll
                    for (int part = 0; part < kParts; ++part)
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[q] = mfma16<BF>(rows[q], v[part][s], acc[q]);
                }
            }
            next_rows();
            if (r16 < count) store_rows<BF>(p.a, tokens[0], row0, lane, whole, steps != 0, unit, base, acc);
        }
        base[0] = next_base[0], base[1] = next_base[1];
        next_base[0] = later_base[0], next_base[1] = later_base[1];
        // (LDS alone: the stores need not have arrived)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
}

namespace {

struct LoraPlan {
    bool few, many;     // at most kFewTokens; many tokens of few adapters
    bool one;           // one token of a small adapter
    int slots;          // most tiles there can be
    int row_tiles, row_blocks;  // shrink: rows of A of a workgroup in sixteens, and how many such blocks
    int slices, row_groups;
    size_t part_bytes, order_bytes, tile_bytes, cursor_bytes, operand_bytes, unit_bytes;
};

size_t whole(size_t bytes) { return (bytes + 15) & ~(size_t)15; }

int steps_up_to(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8; }

LoraPlan lora_plan(const bcq_adapters &d, int tokens)
{
    LoraPlan s;
    s.few = tokens <= kFewTokens;
    const int most = tokens < d.count + 1 ? tokens : d.count + 1;
    // Operands made in a launch of their own pay from about 1024 tokens of rank 64 on, if adapters have 16 tokens and more (4 adapters, 8192 to 10240, bfloat16; each
    // workgroup for itself / once: 512 tokens of rank 64 39.0 / 36.3 us, 1024 52.6 / 42.8, 2048 98.8 / 59.8; 8 adapters of rank 16: 1024 29.2 / 31.3, 2048 47.9 / 50.0).
    s.many = (long long)tokens * d.max_rank >= 64 * 1024 && d.max_rank <= 128 && tokens >= 16LL * d.count &&
             tokens / kManyTokens + most <= 65535;  // (a grid's second number)
    s.slots = s.few ? tokens : tokens / (s.many ? kManyTokens : 16) + most;
    s.row_tiles = d.max_rank <= 16 ? 1 : d.max_rank <= 32 ? 2 : 4;
    s.row_blocks = (d.max_rank + 16 * s.row_tiles - 1) / (16 * s.row_tiles);
    const int likely = s.few ? (tokens < d.count ? tokens : d.count) : s.slots;  // tiles, if adapters are spread
    // (one token, rank 64, 28672 to 7168: 16 slices 17 us, 8 23, 4 38)
    const int wanted = 2 * compute_units() / (likely * s.row_blocks), longest = (d.N + 511) / 512;
    s.slices = wanted < longest ? wanted : longest;
    s.slices = s.slices < 1 ? 1 : s.slices > 16 ? 16 : s.slices;
    // as many workgroups as the chip holds at once, four to a compute unit, so that each makes v once
    const int blocks = (d.M + 64 * kWaves - 1) / (64 * kWaves);
    const long long resident = 4 * compute_units(), groups = ((long long)blocks * likely + resident - 1) / resident;
    s.row_groups = (int)(groups < 1 ? 1 : groups > 16 ? 16 : groups);
    // (A launch less, but A from the caches for every 512 rows of B.  One launch against two: rank 16, 4096 to 4096 5.0 and 7.8 us, 8192 to 10240 6.1 and 8.6,
    // 14336 to 7168 7.6 and 9.3; rank 32, 8192 to 10240 9.8 and 9.4; rank 16, 28672 to 7168 12.9 and 10.0.)
    s.one = tokens == 1 && (long long)d.max_rank * d.N <= kOneElements;
    if (s.one) {
        const int rows = 64 * kOneWaves, all = (d.M + rows - 1) / rows, parts = compute_units() < all ? compute_units() : all;
        s.row_groups = (all + parts - 1) / parts;
        s.part_bytes = s.order_bytes = s.tile_bytes = s.cursor_bytes = s.operand_bytes = s.unit_bytes = 0;
        return s;
    }
    const bool bf = d.dtype == BCQ_BF16;
    s.part_bytes = whole((size_t)s.slices * tokens * d.max_rank * sizeof(float));
    s.order_bytes = s.few ? 0 : whole((size_t)s.slots * (s.many ? kManyTokens : 16) * sizeof(int));
    s.tile_bytes = s.few ? 0 : whole((size_t)(2 + 2 * s.slots) * sizeof(int));
    s.cursor_bytes = s.few || d.count + 1 <= kPlanGroups ? 0 : whole((size_t)(d.count + 1) * sizeof(int));
    s.operand_bytes = s.many ? (size_t)s.slots * (kManyTokens / 16) * operand_bytes(bf, (d.max_rank + 15) / 16) : 0;
    s.unit_bytes = s.many ? whole((size_t)s.slots * kManyTokens * sizeof(float)) : 0;
    return s;
}

template <bool BF, int NT, bool FEW>
void launch_shrink(const LoraParams &p, const LoraPlan &s, hipStream_t stream)
{
    const dim3 shrink(s.slots, s.slices, s.row_blocks);
    if (s.row_tiles == 1) bcq_lora_shrink_kernel<BF, NT, 1, FEW><<<shrink, 64 * kWaves, 0, stream>>>(p);
    else if (s.row_tiles == 2) bcq_lora_shrink_kernel<BF, NT, 2, FEW><<<shrink, 64 * kWaves, 0, stream>>>(p);
    else bcq_lora_shrink_kernel<BF, NT, 4, FEW><<<shrink, 64 * kWaves, 0, stream>>>(p);
}

template <bool BF, bool FEW>
void launch(const LoraParams &p, const LoraPlan &s, hipStream_t stream)
{
    launch_shrink<BF, 1, FEW>(p, s, stream);
    const int rows = 64 * kWaves * s.row_groups;
    const dim3 expand(s.slots, (p.a.desc.M + rows - 1) / rows);
    bcq_lora_expand_kernel<BF, FEW><<<expand, 64 * kWaves, operand_bytes(BF, (p.a.desc.max_rank + 15) / 16), stream>>>(p);
}

template <bool BF>
void launch_many(LoraParams p, const LoraPlan &s, hipStream_t stream)
{
    launch_shrink<BF, kManyTokens / 16, false>(p, s, stream);
    p.operand_pieces = (int)(operand_bytes(BF, (p.a.desc.max_rank + 15) / 16) / 16);
    bcq_lora_pack_kernel<BF><<<dim3(s.slots, kManyTokens / 16), 64 * kWaves, 0, stream>>>(p);
    const int blocks = (p.a.desc.M + 63) / 64, steps = steps_up_to(p.a.desc.max_rank);
    // All workgroups at once, as the registers allow.  (4 adapters, 2048 tokens of rank 64, 7168 to 28672: 101 us, 107 with eight groups of rows to each.)
    const int columns = compute_units() * many_occupancy(steps) / s.slots;
    p.row_groups = columns > 0 ? (blocks + columns - 1) / columns : blocks;
    if (p.row_groups > 32) p.row_groups = 32;
    const dim3 grid((blocks + p.row_groups - 1) / p.row_groups, s.slots);
    switch (steps) {
        case 1: bcq_lora_many_kernel<BF, 1><<<grid, 64 * kWaves, 0, stream>>>(p); break;
        case 2: bcq_lora_many_kernel<BF, 2><<<grid, 64 * kWaves, 0, stream>>>(p); break;
        case 4: bcq_lora_many_kernel<BF, 4><<<grid, 64 * kWaves, 0, stream>>>(p); break;
        default: bcq_lora_many_kernel<BF, 8><<<grid, 64 * kWaves, 0, stream>>>(p);
    }
}

template <bool BF>
void by_plan(const LoraParams &p, const LoraPlan &s, hipStream_t stream)
{
    if (s.one) {
        const int rows = 64 * kOneWaves * s.row_groups;
        bcq_lora_one_kernel<BF><<<(p.a.desc.M + rows - 1) / rows, 64 * kOneWaves, 0, stream>>>(p);
        return;
    }
    if (s.few) return launch<BF, true>(p, s, stream);
    bcq_lora_plan_kernel<<<1, 1024, 0, stream>>>(p, s.many ? kManyTokens : 16);
    s.many ? launch_many<BF>(p, s, stream) : launch<BF, false>(p, s, stream);
}

}  // namespace

size_t lora_workspace_bytes(const bcq_adapters &d, int tokens)
{
    const LoraPlan s = lora_plan(d, tokens);
    return s.part_bytes + s.order_bytes + s.tile_bytes + s.cursor_bytes + s.operand_bytes + s.unit_bytes;
}

hipError_t launch_lora(const LoraArgs &a, hipStream_t stream)
{
    const LoraPlan s = lora_plan(a.desc, a.tokens);
    LoraParams p;
    p.a = a;
    char *at = static_cast<char *>(a.workspace);
    const auto take = [&](size_t bytes) {
        char *const here = at;
        at += bytes;
        return here;
    };
    p.part = reinterpret_cast<float *>(take(s.part_bytes));
    p.order = reinterpret_cast<int *>(take(s.order_bytes));
    p.tiles = reinterpret_cast<int *>(take(s.tile_bytes));
    p.cursor = reinterpret_cast<int *>(take(s.cursor_bytes));
    p.operands = reinterpret_cast<u32x4 *>(take(s.operand_bytes));
    p.units = reinterpret_cast<float *>(take(s.unit_bytes));
    p.slices = s.slices;
    p.row_groups = s.row_groups;
    p.copy = a.Y != a.base;
    if (a.desc.dtype == BCQ_BF16) by_plan<true>(p, s, stream);
    else by_plan<false>(p, s, stream);
    return hipGetLastError();
}

}  // namespace bcq
