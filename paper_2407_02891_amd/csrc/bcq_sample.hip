// The next tokens from logits, by temperature, top-k, top-p and min-p, with given random numbers.
//
//   w_i = exp((x_i - max x) / temperature); tokens in the order of descending x, then ascending index; the first top_k of them, S their weight;
//   of those the ones before which less than top_p S stands, and whose w is min_p or more; M their weight; the first at which more than u M stands.
//
// Logits of 16 bits have 65536 values, so a row is what its values' counts are: no token is sorted, and a weight is computed once for a value, in binary64,
// as the borders (u M in a sum of 131072 weights) ask for.  Counts are exact in any order.
//  * A workgroup has a row.  It counts the row's values in LDS: a word for each magnitude, the positive value's entries in its low half, the negative one's in its high half.  Where
//    counters pass 16 bits, they are moved to a list between chunks of 32768 entries.
//  * The weight and number of each unit of 512 values, in descending order, by all waves; then, in one wave, the borders one after the other: which unit, which eight values, which value,
//    how many of its entries.
//  * The entry: the row is read again (from L2) and the drawn value's entries counted, in the order of the index.
//
// Bound by one compute unit's steps in a row.  64 rows of 131072: 26.5 us, of which 10 count (64 additions to LDS take 4 clocks, at random addresses 7.5), 1.5 sum the counts, 0.8 find the
// largest, 1.9 weigh, 4.4 search the borders, 3.8 find the entry.  One row of 32000: 12.5.  Rows of four chunks kept in registers, and 512 threads, were slower; for the entry, a stretch of the
// row for each wave without a barrier a chunk gained 1 us with 64 rows and lost 1 with 256.
#include "bcq_half.h"
#include "bcq_internal.h"
#include "bcq_lanes.h"

namespace bcq {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kUnit = 512, kUnits = 65536 / kUnit;  // units of values: eight a lane
constexpr int kPieces = 4;                          // of eight entries, of a thread in a chunk
constexpr int kChunk = 8 * kPieces * kThreads;      // entries
constexpr int kBig = 32768;                         // entries of a value that are moved from its counter: what is left and the next chunk's fit 16 bits
static_assert(kBig - 1 + kChunk <= 0xffff, "");
constexpr int kMostBig = BCQ_MAX_VOCAB / kBig;

typedef unsigned long long u64;
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

struct SampleParams {
    const uint16_t *logits;
    const float *temperature, *top_p, *min_p, *uniform;
    const int *top_k;
    int *token;
    float *probability;
    long long ld;
    int vocab;
};

// A value's place in descending order: +infinity's is kFirst, -infinity's kEnd; NaN are in front of the one and behind the other, and -0 behind +0.
constexpr uint32_t kPlus0 = 0x7fff, kMinus0 = 0x8000;
template <bool BF>
constexpr uint32_t kInfinity = BF ? 0x7f80u : 0x7c00u;
template <bool BF>
constexpr uint32_t kFirst = 0x7fffu - kInfinity<BF>;
template <bool BF>
constexpr uint32_t kEnd = 0x8000u | kInfinity<BF>;

__device__ __forceinline__ uint32_t bits_at(uint32_t place) { return place & 0x8000u ? place : place ^ 0x7fffu; }

template <bool BF>
__device__ __forceinline__ double value_at(uint32_t place)
{
    return to_float<BF>(bits_at(place));
}

// 2^y, y <= 0: 2^n times the series of e^(r ln 2), |r| <= 1/2, whose next term is below 2^-47.  2^-1020 for less, and for NaN: beside the largest value's weight, 1, that is none.
__device__ __forceinline__ double exp2_series(double y)
{
    y = fmax(y, -1020.0);
    const double n = __builtin_rint(y), z = (y - n) * 0.6931471805599453094;
    double s = 1.0 / 39916800.0;
    constexpr double c[] = {1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
    for (int i = 0; i < 11; ++i) s = __builtin_fma(s, z, c[i]);
    return __builtin_ldexp(s, (int)n);
}

// What a row's weights are computed from.
struct Weigh {
    double most, per;  // the largest value; log2 e / temperature
    uint32_t top;      // its place
    template <bool BF>
    __device__ __forceinline__ double of(uint32_t place) const
    {
        return place <= top ? 1.0 : exp2_series((value_at<BF>(place) - most) * per);  // (no larger one occurs; none may become an infinity that a count of zero meets)
    }
    // What the n[e] entries of the eight values from `place`, a multiple of eight, on weigh.  They have one exponent, so they are as far from each other and their weights are a
    // geometric sequence: a polynomial of its ratio.
    template <bool BF>
    __device__ __forceinline__ double eight(uint32_t place, const int (&n)[8]) const
    {
        const double ratio = exp2_series((value_at<BF>(place + 1) - value_at<BF>(place)) * per);
        double sum = 0.0;
        if (place / kUnit == top / kUnit) {  // (all lanes) the largest may be in the midst of the eight
            double w = of<BF>(place);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e) w = place + e <= top ? 1.0 : w * ratio;
                sum = __builtin_fma(n[e], w, sum);
            }
            return sum;
        }
#pragma unroll
        for (int e = 7; e >= 0; --e) sum = __builtin_fma(sum, ratio, n[e]);
        return sum * of<BF>(place);
    }
};

__device__ __forceinline__ u64 least_of_all(u64 v)
{
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        const u64 other = __shfl_xor(v, s);
        v = other < v ? other : v;
    }
    return v;
}

// Entries from the 16 bytes that a row's first one lies in to that.
__device__ __forceinline__ int in_front(const uint16_t *row) { return (int)(reinterpret_cast<uintptr_t>(row) >> 1 & 7); }

// The entries of a chunk of a row in pieces of eight that begin at 16 bytes, thread t's the pieces t, t + kThreads, ..; what is outside of the row is a
// negative NaN.
struct Chunk {
    u32x4 x[kPieces];
    int first;  // index of the first piece's first entry
    __device__ __forceinline__ int index(int j) const { return first + 8 * (j * kThreads + (int)threadIdx.x); }
    __device__ __forceinline__ bool any(int j, int vocab) const { return first + 8 * j * kThreads < vocab; }  // of all threads
    // Chunk c of the row; its first one begins in front of the row if that does not begin at 16 bytes.
    __device__ __forceinline__ void load(const uint16_t *row, int c, int vocab)
    {
        first = c * kChunk - in_front(row);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            x[j] = u32x4{0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
            const int at = index(j);
            if (at >= 0 && at + 8 <= vocab) {
                x[j] = *reinterpret_cast<const u32x4 *>(row + at);
            } else if (at < vocab) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at + e >= 0 && at + e < vocab) x[j][e >> 1] = e & 1 ? (x[j][e >> 1] & 0xffffu) | (uint32_t)row[at + e] << 16 : (x[j][e >> 1] & 0xffff0000u) | row[at + e];
            }
        }
    }
};
__device__ __forceinline__ int chunks_of(const uint16_t *row, int vocab) { return (vocab + in_front(row) + kChunk - 1) / kChunk; }

// A row's chunks.  KEPT: there is one, which stays in registers.
template <bool KEPT>
struct Row {
    const uint16_t *row;
    int vocab, chunks;
    Chunk kept;
    __device__ __forceinline__ Row(const uint16_t *row, int vocab) : row(row), vocab(vocab), chunks(chunks_of(row, vocab))
    {
        if (KEPT) kept.load(row, 0, vocab);
    }
    // use(chunk, whether there are more) for one after the other, until it returns true.
    template <class F>
    __device__ __forceinline__ void each(F use) const
    {
        if constexpr (KEPT) {
            use(kept, false);
        } else {
            Chunk next;
            int c = 0;
            asm volatile("" : "+s"(c));  // (the masks of its edges are not held where a row is counted again)
            next.load(row, c, vocab);
#pragma unroll 1
            for (; c < chunks; ++c) {
                const Chunk now = next;
                if (c + 1 < chunks) next.load(row, c + 1, vocab);
                if (use(now, c + 1 < chunks)) return;
            }
        }
    }
};

// Rows whose token is the first of the largest values, whatever the random number.
__device__ __forceinline__ bool greedy(const SampleParams &p, int row)
{
    return !(p.temperature[row] > 0.0f) || (p.top_k && p.top_k[row] == 1);
}

__device__ __forceinline__ void write_token(const SampleParams &p, int row, int token, float probability)
{
    p.token[row] = token;
    if (p.probability) p.probability[row] = probability;
}

// What is compared of a pair of entries to find those of the value at `place`, and with what: zeros of both signs are one value.
struct Wanted {
    uint32_t mask, pair;
    __device__ __forceinline__ explicit Wanted(uint32_t place) : mask(place == kPlus0 || place == kMinus0 ? 0x7fff7fffu : 0xffffffffu), pair((bits_at(place) << 16 | bits_at(place)) & mask) {}
    // The entries of a piece that are of it, a bit each.
    __device__ __forceinline__ uint32_t which(const u32x4 &x) const
    {
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t other = (x[i] ^ pair) & mask;
            found |= (uint32_t)((other & 0xffffu) == 0) << 2 * i | (uint32_t)(other >> 16 == 0) << (2 * i + 1);
        }
        return found;
    }
    // Whether any lane has one.
    __device__ __forceinline__ bool any(const u32x4 &x) const
    {
        u32x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = x[i] ^ pair;
        if (mask != 0xffffffffu) y &= mask;
        u16x2 least = {0xffff, 0xffff};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t two = y[i];
            least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, two));
        }
        return __ballot(least.x == 0 || least.y == 0) != 0;
    }
    __device__ __forceinline__ int count(const u32x4 &x) const
    {
        u16x2 others = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) others += __builtin_elementwise_min(__builtin_bit_cast(u16x2, (x[i] ^ pair) & mask), (u16x2){1, 1});
        return 8 - others.x - others.y;
    }
};

struct Shared {
    double mass[kUnits];
    int entries[kUnits];
    u64 best[kWaves];
    int found[kPieces * kWaves];
    uint32_t big[kMostBig];  // places of kBig entries each that are not in the table
    int num_big;
    int passed;              // entries that were met and are not in the table
    uint32_t place;          // of the drawn value
    int nth;                 // which of its entries
};

// The first entry of the largest value: place << 32 | index, all ones if there is none.  All threads get it.
template <bool BF, bool KEPT>
__device__ __forceinline__ u64 first_of_largest(const Row<KEPT> &row, Shared &sh)
{
    u64 best = ~0ull;
    row.each([&](const Chunk &now, bool) {
        // (places less kFirst, so that NaN of either sign and -infinity are behind all others)
        constexpr u16x2 first = {(unsigned short)kFirst<BF>, (unsigned short)kFirst<BF>};
        u16x2 least = {0xffff, 0xffff};
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t x = now.x[j][i], places = x ^ 0x7fff7fffu ^ (x >> 15 & 0x00010001u) * 0x7fffu;
                least = __builtin_elementwise_min(least, (u16x2)(__builtin_bit_cast(u16x2, places) - first));
            }
        uint32_t place = min((uint32_t)least.x, (uint32_t)least.y) + kFirst<BF>;
        if (place == kMinus0) place = kPlus0;
        if (place < kEnd<BF> && place < (uint32_t)(best >> 32)) {
            const Wanted wanted(place);
#pragma unroll
            for (int j = kPieces - 1; j >= 0; --j) {
                const uint32_t found = wanted.which(now.x[j]);
                if (found) best = (u64)place << 32 | (uint32_t)(now.index(j) + __builtin_ctz(found));
            }
        }
        return false;
    });
    best = least_of_all(best);
    if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = best;
    __syncthreads();
    best = sh.best[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) best = sh.best[w] < best ? sh.best[w] : best;
    return best;
}

// How often each value occurs: the counters of magnitude m are in word m.  careful (of rows of more than a chunk): none passes 16 bits.
template <bool BF, bool KEPT>
__device__ __forceinline__ void count_values(const Row<KEPT> &row, uint32_t *table, Shared &sh, bool careful)
{
    const int lane = threadIdx.x & 63;
    int passed = 0;
    const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 32768 / 4 / kThreads; ++i) reinterpret_cast<u32x4 *>(table)[i * kThreads + threadIdx.x] = zero;
    if (threadIdx.x == 0) sh.num_big = sh.passed = 0;
    __syncthreads();
    row.each([&](const Chunk &now, bool more) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            if (!now.any(j, row.vocab)) break;
            const u32x4 x = now.x[j];
            u16x2 high = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t two = x[i];  // (of a vector's element itself __builtin_bit_cast makes element 0)
                high = __builtin_elementwise_max(high, __builtin_bit_cast(u16x2, two));
            }
            const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)x[0]);
            if (__ballot(x[0] == w) == ~0ull && w >> 16 == (w & 0xffffu) && __ballot(x[1] == w && x[2] == w && x[3] == w) == ~0ull) {
                // entries that are all alike, a mask's: one by one they would take 64 turns each
                if (lane == 0) {
                    if ((w & 0xffffu) < kEnd<BF>) atomicAdd(table + (w & 0x7fffu), 512u << (w >> 31 << 4));
                    else passed += 512;
                }
            } else if (__ballot(max((uint32_t)high.x, (uint32_t)high.y) >= kEnd<BF>)) {
                // -infinities, another mask, would all meet at one counter
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t bits = e ? x[i] >> 16 : x[i] & 0xffffu;
                        if (bits < kEnd<BF>) atomicAdd(table + (bits & 0x7fffu), bits >> 15 ? 0x10000u : 1u);
                        else ++passed;
                    }
            } else {
                // (three vector instructions an entry: the low and the high half's address and what is added)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t two = x[i], magnitudes = two & 0x7fff7fffu;
                    const s16x2 sign = __builtin_bit_cast(s16x2, two) >> (s16x2){15, 15};  // 0 or 0xffff
                    uint32_t low, high;
                    asm("v_lshlrev_b32_sdwa %0, %2, %3 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:WORD_0\n\t"
                        "v_lshlrev_b32_sdwa %1, %2, %3 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:WORD_1"
                        : "=&v"(low), "=v"(high)
                        : "v"(2), "v"(magnitudes));
                    atomicAdd(reinterpret_cast<uint32_t *>(reinterpret_cast<char *>(table) + low), (uint32_t)(uint16_t)sign.x + 1u);
                    atomicAdd(reinterpret_cast<uint32_t *>(reinterpret_cast<char *>(table) + high), (uint32_t)(uint16_t)sign.y + 1u);
                }
            }
        }
        if (!KEPT && careful && more) {  // what the next chunk could bring beyond 16 bits
            __syncthreads();
            for (int i = threadIdx.x; i < 32768 / 4; i += kThreads) {
                u32x4 x = reinterpret_cast<u32x4 *>(table)[i];
                if (!((x[0] | x[1] | x[2] | x[3]) & 0x80008000u)) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t m = 4 * i + e;
                    if (x[e] & 0x8000u) sh.big[atomicAdd(&sh.num_big, 1)] = kPlus0 - m;
                    if (x[e] & 0x80000000u) sh.big[atomicAdd(&sh.num_big, 1)] = m ? kMinus0 + m : kPlus0;
                    x[e] &= 0x7fff7fffu;
                }
                reinterpret_cast<u32x4 *>(table)[i] = x;
            }
            __syncthreads();
        }
        return false;
    });
    __syncthreads();
    // NaN go, -0 are zeros
    static_assert(0x7fff - kInfinity<BF> <= kThreads, "");
    if (threadIdx.x < 0x7fff - kInfinity<BF>) {
        const uint32_t nan = table[kInfinity<BF> + 1 + threadIdx.x];
        table[kInfinity<BF> + 1 + threadIdx.x] = 0;
        passed += (nan & 0xffffu) + (nan >> 16);
    }
    if (!KEPT) {
        passed = sum_all(passed);
        if (lane == 0) atomicAdd(&sh.passed, passed);
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < sh.num_big; ++i)
            if (sh.big[i] < kFirst<BF>) sh.big[i] = 0xffffffffu;
        const uint32_t zeros = (table[0] >> 16) + (table[0] & 0xffffu);
        table[0] = zeros & 0x7fffu;
        for (uint32_t n = zeros / kBig; n > 0; --n) sh.big[sh.num_big++] = kPlus0;
    }
    __syncthreads();
}

// What is counted.
struct Counts {
    const uint32_t *table;
    const Shared &sh;
    int num_big;
    // Of a block of words (the positive unit kUnits / 2 - 1 - b and the negative one kUnits / 2 + b) what the lane has; the table alone.
    __device__ __forceinline__ void block(int b, int lane, int &low, int &high) const
    {
        const u32x4 *const at = reinterpret_cast<const u32x4 *>(table + b * kUnit + 4 * lane);
        const u32x4 c[2] = {at[0], at[64]};
        uint32_t l = 0, h = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t two = c[e >> 2][e & 3];
            l = __builtin_amdgcn_udot2(__builtin_bit_cast(u16x2, two), (u16x2){1, 0}, l, false);
            h = __builtin_amdgcn_udot2(__builtin_bit_cast(u16x2, two), (u16x2){0, 1}, h, false);
        }
        low = (int)l, high = (int)h;
    }
    // A unit's, eight a lane.
    __device__ __forceinline__ void unit(int u, int lane, int (&n)[8]) const
    {
        const bool negative = u >= kUnits / 2;
        const u32x4 *const at = reinterpret_cast<const u32x4 *>(table + (negative ? (u - kUnits / 2) * kUnit + 8 * lane : 32768 - 8 - u * kUnit - 8 * lane));
        const u32x4 c[2] = {at[0], at[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = (int)(negative ? c[e >> 2][e & 3] >> 16 : c[(7 - e) >> 2][3 - (e & 3)] & 0xffffu);
        const uint32_t first = u * kUnit + 8 * lane;
        for (int i = 0; i < num_big; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) n[e] += sh.big[i] == first + e ? kBig : 0;
    }
    __device__ __forceinline__ int of(uint32_t place) const
    {
        int n = (int)(place & 0x8000u ? table[place & 0x7fffu] >> 16 : table[kPlus0 - place] & 0xffffu);
        for (int i = 0; i < num_big; ++i) n += sh.big[i] == place ? kBig : 0;
        return n;
    }
};

// The number of each unit's entries.
__device__ __forceinline__ void count_units(const Counts &c, Shared &sh)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int b = wave; b < kUnits / 2; b += kWaves) {
        int low, high;
        c.block(b, lane, low, high);
        low = sum_all(low), high = sum_all(high);
        if (lane == 0) sh.entries[kUnits / 2 - 1 - b] = low, sh.entries[kUnits / 2 + b] = high;
    }
    __syncthreads();
    if ((int)threadIdx.x < c.num_big && sh.big[threadIdx.x] < 0x10000u) atomicAdd(sh.entries + sh.big[threadIdx.x] / kUnit, kBig);
    if (c.num_big) __syncthreads();
}

// The draw of a row: the value, and which of its entries, in sh.  False if there is nothing to draw from.
template <bool BF>
__device__ __forceinline__ bool draw(const SampleParams &p, int row, const Counts &c, Shared &sh)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // ---- the largest value, then the units' weight as far as a border needs it ----
    const int e0 = sh.entries[2 * lane], e1 = sh.entries[2 * lane + 1];
    const int entries_upto = sum_upto(e0 + e1, lane), n0 = entries_upto - (e0 + e1);
    const int all = from_lane(entries_upto, 63), top_k = p.top_k ? p.top_k[row] : 0;
    const double top_p = p.top_p ? p.top_p[row] : 1.0, min_p = p.min_p ? p.min_p[row] : 0.0;
    if (all == 0) {
        if (threadIdx.x == 0) write_token(p, row, -1, 0.0f);
        return false;
    }
    int top_unit = 2 * __builtin_ctzll(__ballot(e0 || e1));
    if (!from_lane(e0, top_unit / 2)) ++top_unit;
    Weigh weigh;
    {
        int n[8], e = 8;
        c.unit(top_unit, lane, n);
#pragma unroll
        for (int i = 7; i >= 0; --i) e = n[i] ? i : e;
        const int l = __builtin_ctzll(__ballot(e < 8));
        weigh.top = top_unit * kUnit + 8 * l + from_lane(e, l);
    }
    weigh.most = value_at<BF>(weigh.top);
    weigh.per = 1.4426950408889634074 / (double)p.temperature[row];
    int last_unit = kUnits - 1;  // that counts: of the first top_k entries; without top_p, of those with weights of min_p
    if (top_k > 0 && top_k < all) {
        const int l = __builtin_ctzll(__ballot(entries_upto >= top_k));
        last_unit = 2 * l + (from_lane(n0 + e0, l) >= top_k ? 0 : 1);
    }
    if (min_p > 0.0 && !(top_p < 1.0)) {
        const double least = fmin(min_p, 1.0);
        const u64 behind0 = __ballot(weigh.of<BF>(2 * lane * kUnit) < least), behind1 = __ballot(weigh.of<BF>(2 * lane * kUnit + kUnit) < least);
        last_unit = min(last_unit, max(kUnits - 1 - __popcll(behind0) - __popcll(behind1), top_unit));
    }
    for (int u = wave; u < kUnits; u += kWaves) {
        double mass = 0.0;
        if (u <= last_unit && sh.entries[u]) {
            int n[8];
            c.unit(u, lane, n);
            mass = sum_all(weigh.eight<BF>(u * kUnit + 8 * lane, n));
        }
        if (lane == 0) sh.mass[u] = mass;
    }
    __syncthreads();
    // ---- the borders, in one wave ----
    if (wave == 0) {
        const double m0 = sh.mass[2 * lane], m1 = sh.mass[2 * lane + 1];
        const double mass_upto = sum_upto(m0 + m1, lane), before0 = mass_upto - (m0 + m1);  // before the lane's first unit
        const float number = p.uniform[row];
        // the end of what is kept: `kept` entries of the value at `end`, all of those before it
        uint32_t end = 0xffffffffu;
        int kept = 0;
        double sum = from_lane(mass_upto, 63);
        // A search for each of the borders (in one body, so that its instructions are fetched once): the unit, the lane's eight values in it, the value.  0, 1, 3: the first
        // value where what stands up to and with it reaches the goal; 2: the last value, whether it occurs or not, whose weight does.
#pragma unroll 1
        for (int border = 0; border < 4; ++border) {
            if (border == 0 ? top_k <= 0 || top_k >= all : border == 1 ? !(top_p < 1.0) : border == 2 ? !(min_p > 0.0) : false) continue;
            // (the number is below 1 by more than the sums round, so that an entry that is kept is found)
            const double goal = border == 0 ? top_k : border == 1 ? top_p * sum : border == 2 ? fmin(min_p, 1.0) : (double)(number > 0.0f ? fminf(number, 1.0f - 0x1p-24f) : 0.0f) * sum;
            const auto reached = [&](double mass, int entries) { return border == 0 ? entries >= goal : border == 3 ? mass > goal : mass >= goal; };
            bool in0, in1;
            if (border == 2) {  // the value behind the unit has not
                in0 = weigh.of<BF>(2 * lane * kUnit + kUnit) < goal, in1 = weigh.of<BF>(2 * lane * kUnit + 2 * kUnit) < goal;
            } else {
                in0 = e0 && reached(before0 + m0, n0 + e0), in1 = e1 && reached(mass_upto, entries_upto);
            }
            u64 votes = __ballot(in0 || in1);
            const bool never = votes == 0;  // (sums that round otherwise: the last that occurs)
            if (never) votes = 1ull << (63 - __builtin_clzll(__ballot(e0 || e1)));
            int l = __builtin_ctzll(votes);
            const bool second = never ? from_lane(e1, l) != 0 : from_lane((int)in0, l) == 0;
            const int u = 2 * l + second;
            const double before_unit = from_lane(second ? before0 + m0 : before0, l);
            const int entries_before_unit = from_lane(second ? n0 + e0 : n0, l);
            int k[8], many = 0;
            c.unit(u, lane, k);
#pragma unroll
            for (int e = 0; e < 8; ++e) many += k[e];
            const double own = weigh.eight<BF>(u * kUnit + 8 * lane, k), upto = before_unit + sum_upto(own, lane);
            const int entries = entries_before_unit + sum_upto(many, lane);
            votes = border == 2 ? __ballot(weigh.of<BF>(u * kUnit + 8 * lane) >= goal) : __ballot(many && reached(upto, entries));
            if (border != 2 && !votes) votes = 1ull << (63 - __builtin_clzll(__ballot(many) | 1));
            l = border == 2 ? 63 - __builtin_clzll(votes | 1) : __builtin_ctzll(votes);
            const double before_eight = from_lane(upto - own, l);
            const int entries_before_eight = from_lane(entries - many, l);
            const uint32_t first = u * kUnit + 8 * l, place = first + (lane & 7);
            const int n = c.of(place);
            const double w = weigh.of<BF>(place);
            double mass = n * w;
            int number_of = n;
            mass += in_row<0x111>(mass), number_of += in_row<0x111>(number_of);
            mass += in_row<0x112>(mass), number_of += in_row<0x112>(number_of);
            mass += in_row<0x114>(mass), number_of += in_row<0x114>(number_of);
            const u64 eight = 0xff;
            votes = eight & (border == 2 ? __ballot(w >= goal) : __ballot(n && reached(before_eight + mass, entries_before_eight + number_of)));
            if (border != 2 && !votes) votes = 1ull << (63 - __builtin_clzll((eight & __ballot(n)) | 1));
            l = border == 2 ? 63 - __builtin_clzll(votes | 1) : __builtin_ctzll(votes);
            const uint32_t found = first + l;
            const double weight = from_lane(w, l), before = before_eight + from_lane(mass - n * w, l);
            const int its = from_lane(n, l);
            if (border == 3) {
                kept = found == end ? kept : its;
                const double more = (goal - before) / weight;
                const int nth = more < kept ? max((int)more, 0) : max(kept - 1, 0);
                if (lane == 0) {
                    sh.place = found, sh.nth = nth;
                    if (p.probability) p.probability[row] = (float)(weight / sum);
                }
                break;
            }
            int count = its;
            if (border == 0) {
                count = min(max(top_k - (entries_before_eight + from_lane(number_of, l) - its), 1), its);
            } else if (border == 1) {
                const double more = __builtin_ceil((goal - before) / weight);
                count = more < its ? max((int)more, 1) : its;
            }
            if (found < end || (found == end && count < kept)) {
                end = found, kept = count;
                sum = __builtin_fma(kept, weight, before);
            }
        }
    }
    __syncthreads();
    return true;
}

// The drawn entry: its piece, in the order of pieces, chunk after chunk.
template <bool KEPT>
__device__ __forceinline__ void find_entry(const SampleParams &p, int row, const Row<KEPT> &logits, Shared &sh)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Wanted wanted(sh.place);
    int nth = sh.nth;
    logits.each([&](const Chunk &now, bool) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            int all = 0;
            if (now.any(j, p.vocab) && wanted.any(now.x[j])) {
                const int found = wanted.count(now.x[j]);
#pragma unroll
                for (int bit = 0; bit < 4; ++bit) all += __popcll(__ballot(found >> bit & 1)) << bit;
            }
            if (lane == 0) sh.found[j * kWaves + wave] = all;
        }
        __syncthreads();
        const int here = sh.found[lane], upto = sum_upto(here, lane);
        const u64 votes = __ballot(upto > nth);
        if (votes) {
            const int l = __builtin_ctzll(votes);
            if (l % kWaves != wave) return true;
            const int before = from_lane(upto - here, l);
            uint32_t bits = 0;
            int index = 0;
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
                if (j == l / kWaves) bits = wanted.which(now.x[j]), index = now.index(j);
            const int own = __popc(bits), in_front = before + sum_upto(own, lane) - own;
            if (nth < in_front || nth >= in_front + own) return true;
            for (int i = in_front; i < nth; ++i) bits &= bits - 1;
            p.token[row] = index + __builtin_ctz(bits);
            return true;
        }
        nth -= from_lane(upto, 63);
        __syncthreads();
        return false;
    });
}
static_assert(kPieces * kWaves == 64, "");

}  // namespace

template <bool BF, bool KEPT>
__global__ __launch_bounds__(kThreads) void bcq_sample_kernel(SampleParams p)
{
    __shared__ __attribute__((aligned(16))) uint32_t table[32768];
    __shared__ Shared sh;
    const int row = blockIdx.x;
    const Row<KEPT> logits(p.logits + row * p.ld, p.vocab);
    if (greedy(p, row)) {
        const u64 best = first_of_largest<BF>(logits, sh);
        if (threadIdx.x == 0) write_token(p, row, best == ~0ull ? -1 : (int)(uint32_t)best, best == ~0ull ? 0.0f : 1.0f);
        return;
    }
    // A counter that passes 16 bits loses 65535 or 65536 entries each time, so the sum of all tells whether any did.  Then (half of the first 131072 entries alike, say) they are counted again,
    // with a look at every counter between chunks.  (64 rows of 131072: 26.9 us, with that look in the first place 29.6.)
    const int lane = threadIdx.x & 63, met = (p.vocab + in_front(logits.row) + 8 * kThreads - 1) / (8 * kThreads) * (8 * kThreads);
    bool careful = KEPT;
#pragma unroll 1
    for (;; careful = true) {
        count_values<BF>(logits, table, sh, careful);
        count_units(Counts{table, sh, __builtin_amdgcn_readfirstlane(sh.num_big)}, sh);
        if (careful || sum_all(sh.entries[2 * lane] + sh.entries[2 * lane + 1]) + sh.passed == met) break;
        __syncthreads();
    }
    if (draw<BF>(p, row, Counts{table, sh, __builtin_amdgcn_readfirstlane(sh.num_big)}, sh)) find_entry(p, row, logits, sh);
}

namespace {

template <bool BF>
void sample(const SampleParams &p, int rows, hipStream_t s)
{
    if (p.vocab + 7 <= kChunk) bcq_sample_kernel<BF, true><<<rows, kThreads, 0, s>>>(p);
    else bcq_sample_kernel<BF, false><<<rows, kThreads, 0, s>>>(p);
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t stream)
{
    const SampleParams p = {a.logits, a.temperature, a.top_p, a.min_p, a.uniform, a.top_k, a.token, a.probability, a.ld, a.vocab};
    if (a.bf16) sample<true>(p, a.rows, stream);
    else sample<false>(p, a.rows, stream);
    return hipGetLastError();
}

}  // namespace bcq
