// The next tokens from logits, by temperature, top-k, top-p and min-p, with given random numbers.
//
//   w_i = exp((x_i - max x) / temperature); tokens in the order of descending x, then ascending index; the first top_k of them, S their weight;
//   of those the ones before which less than top_p S stands, and whose w is min_p or more; M their weight; the first at which more than u M stands.
//
// Logits of 16 bits have 65536 values, so a row is what its values' counts are: no token is sorted, and a weight is computed once for a value, in binary64,
// as the borders (u M in a sum of 131072 weights) ask for.  Counts are exact in any order.
//  * A workgroup has a row.  It counts the row's values in LDS: a word for each magnitude, the positive value's entries in its low half, the negative one's in its high half.  Counts that
//    could pass 16 bits are moved to a list between chunks of 32768 entries.
//  * The weight and number of each unit of 512 values, in descending order, by all waves; then, in one wave, the borders one after the other: which unit, which eight values, which value,
//    how many of its entries.
//  * The entry: the row is read again (from L2) and the drawn value's entries counted, in the order of the index.
#include "bcq_half.h"
#include "bcq_internal.h"

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

// 2^y, y <= 0, to a few units of the last place: 2^n times the series of e^(r ln 2), |r| <= 1/2, whose next term is below 2^-53.  2^-1020 for less, and for NaN: beside
// the largest value's weight, 1, that is none.
__device__ __forceinline__ double exp2_series(double y)
{
    y = fmax(y, -1020.0);
    const double n = __builtin_rint(y), z = (y - n) * 0.6931471805599453094;
    double s = 1.0 / 6227020800.0;
    constexpr double c[] = {1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0,
                            1.0 / 120.0,       1.0 / 24.0,       1.0 / 6.0,       0.5,            1.0,           1.0};
#pragma unroll
    for (int i = 0; i < 13; ++i) s = __builtin_fma(s, z, c[i]);
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

__device__ __forceinline__ double from_lane(double v, int lane)
{
    const u64 b = __builtin_bit_cast(u64, v);
    return __builtin_bit_cast(double, (u64)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}
__device__ __forceinline__ int from_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

template <int CTRL>
__device__ __forceinline__ int in_row(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ double in_row(double v)
{
    const u64 b = __builtin_bit_cast(u64, v);
    return __builtin_bit_cast(double, (u64)(uint32_t)in_row<CTRL>((int)(b >> 32)) << 32 | (uint32_t)in_row<CTRL>((int)b));
}

// Sum over the lanes up to and with this one: in rows of sixteen by shifts, then the rows before.
template <class T>
__device__ __forceinline__ T sum_upto(T v, int lane)
{
    v += in_row<0x111>(v);
    v += in_row<0x112>(v);
    v += in_row<0x114>(v);
    v += in_row<0x118>(v);
    const T r0 = from_lane(v, 15), r1 = r0 + from_lane(v, 31), r2 = r1 + from_lane(v, 47);
    return v + (lane < 32 ? lane < 16 ? T(0) : r0 : lane < 48 ? r1 : r2);
}
template <class T>
__device__ __forceinline__ T sum_all(T v)
{
    v += in_row<0x111>(v);
    v += in_row<0x112>(v);
    v += in_row<0x114>(v);
    v += in_row<0x118>(v);
    return from_lane(v, 15) + from_lane(v, 31) + (from_lane(v, 47) + from_lane(v, 63));
}
__device__ __forceinline__ u64 least_of_all(u64 v)
{
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        const u64 other = __shfl_xor(v, s);
        v = other < v ? other : v;
    }
    return v;
}

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
        first = c * kChunk - (int)(reinterpret_cast<uintptr_t>(row) >> 1 & 7);
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
__device__ __forceinline__ int chunks_of(const uint16_t *row, int vocab) { return (int)((vocab + (reinterpret_cast<uintptr_t>(row) >> 1 & 7) + kChunk - 1) / kChunk); }

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
    uint32_t tops[kWaves];
    uint32_t big[kMostBig];  // places of kBig entries each that are not in the table
    int num_big;
    uint32_t place;          // of the drawn value
    int nth;                 // which of its entries
};

// The place of the largest of the entries, as compared to signed numbers: right where it is zero or more and no NaN (false otherwise).
template <bool BF>
__device__ __forceinline__ bool top_of(uint32_t most, uint32_t &place)
{
    place = kPlus0 - most;
    return most <= kInfinity<BF>;
}

// The first entry of the largest value: place << 32 | index, all ones if there is none.  All threads get it.
template <bool BF>
__device__ __forceinline__ u64 first_of_largest(const uint16_t *row, int vocab, Shared &sh)
{
    u64 best = ~0ull;
    Chunk next;
    next.load(row, 0, vocab);
    const int chunks = chunks_of(row, vocab);
    for (int c = 0; c < chunks; ++c) {
        const Chunk now = next;
        if (c + 1 < chunks) next.load(row, c + 1, vocab);
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
    }
    best = least_of_all(best);
    if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = best;
    __syncthreads();
    best = sh.best[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) best = sh.best[w] < best ? sh.best[w] : best;
    return best;
}

// How often each value occurs: the counters of magnitude m are in word m.  Returns the place of the largest, kEnd or more if there is none.
template <bool BF>
__device__ __forceinline__ uint32_t count_values(const uint16_t *row, int vocab, uint32_t *table, Shared &sh)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Chunk next;
    next.load(row, 0, vocab);
    const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) reinterpret_cast<u32x4 *>(table)[i * kThreads + threadIdx.x] = zero;
    if (threadIdx.x == 0) sh.num_big = 0;
    __syncthreads();
    s16x2 most = {-32768, -32768};
    const int chunks = chunks_of(row, vocab);
    for (int c = 0; c < chunks; ++c) {
        const Chunk now = next;
        if (c + 1 < chunks) next.load(row, c + 1, vocab);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            if (!now.any(j, vocab)) break;
            const u32x4 x = now.x[j];
            // entries that are all alike, a mask's: one by one they would take 64 turns each
            const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)x[0]);
            u16x2 magnitude = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t two = x[i];  // (of a vector's element itself __builtin_bit_cast makes element 0)
                magnitude = __builtin_elementwise_max(magnitude, __builtin_bit_cast(u16x2, two & 0x7fff7fffu));
                most = __builtin_elementwise_max(most, __builtin_bit_cast(s16x2, two));
            }
            if (__ballot(x[0] == w && x[1] == w && x[2] == w && x[3] == w) == ~0ull && w >> 16 == (w & 0xffffu)) {
                if ((w & 0x7fffu) < kInfinity<BF> + (w >> 31 ? 0u : 1u) && lane == 0) atomicAdd(table + (w & 0x7fffu), 512u << (w >> 31 << 4));
                continue;
            }
            // infinities and NaN: not counted, but for +infinity (a mask of them would all meet at one counter)
            const bool odd = __ballot(max((uint32_t)magnitude.x, (uint32_t)magnitude.y) >= kInfinity<BF>) != 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t address = (e ? x[i] >> 14 : x[i] << 2) & 0x1fffcu, negative = x[i] >> (e ? 31 : 15) & 1u;
                    if (odd && address >= 4 * kInfinity<BF> + (negative ? 0 : 4)) continue;
                    atomicAdd(reinterpret_cast<uint32_t *>(reinterpret_cast<char *>(table) + address), negative * 0xffffu + 1u);
                }
        }
        __syncthreads();
        if (c + 1 < chunks) {  // what the next chunk could bring beyond 16 bits
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
    }
    int top_signed = max((int)most.x, (int)most.y);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top_signed = max(top_signed, __shfl_xor(top_signed, s));
    if (lane == 0) sh.tops[wave] = (uint32_t)top_signed;
    if (threadIdx.x == 0 && table[0] >> 16) {  // -0 are zeros
        const uint32_t zeros = (table[0] >> 16) + (table[0] & 0xffffu);
        table[0] = zeros & 0x7fffu;
        for (uint32_t n = zeros / kBig; n > 0; --n) sh.big[atomicAdd(&sh.num_big, 1)] = kPlus0;
    }
    __syncthreads();
    int largest = (int)sh.tops[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) largest = max(largest, (int)sh.tops[w]);
    uint32_t top;
    if (largest >= 0 && top_of<BF>((uint32_t)largest, top)) return (uint32_t)__builtin_amdgcn_readfirstlane((int)top);
    // all of them negative, or a NaN among them: from the table
    top = 0xffffffffu;
    for (int m = threadIdx.x; m <= (int)kInfinity<BF>; m += kThreads) {
        if (table[m] & 0xffffu) top = min(top, kPlus0 - m);
        if (table[m] >> 16) top = min(top, kMinus0 + m);
    }
    for (int i = threadIdx.x; i < sh.num_big; i += kThreads) top = min(top, sh.big[i]);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = min(top, (uint32_t)__shfl_xor((int)top, s));
    __syncthreads();
    if (lane == 0) sh.tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = min(top, sh.tops[w]);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)top);
}

// What is counted.
struct Counts {
    const uint32_t *table;
    const Shared &sh;
    // A unit's, eight a lane.
    __device__ __forceinline__ void unit(int u, int lane, int (&n)[8]) const
    {
        const bool negative = u >= kUnits / 2;
        const u32x4 *const at = reinterpret_cast<const u32x4 *>(table + (negative ? (u - kUnits / 2) * kUnit + 8 * lane : 32768 - 8 - u * kUnit - 8 * lane));
        const u32x4 c[2] = {at[0], at[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = (int)(negative ? c[e >> 2][e & 3] >> 16 : c[(7 - e) >> 2][3 - (e & 3)] & 0xffffu);
        const uint32_t first = u * kUnit + 8 * lane;
        for (int i = 0; i < sh.num_big; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) n[e] += sh.big[i] == first + e ? kBig : 0;
    }
    __device__ __forceinline__ int of(uint32_t place) const
    {
        int n = (int)(place & 0x8000u ? table[place & 0x7fffu] >> 16 : table[kPlus0 - place] & 0xffffu);
        for (int i = 0; i < sh.num_big; ++i) n += sh.big[i] == place ? kBig : 0;
        return n;
    }
};

// The draw of a row whose largest value is at `top`: the value, and which of its entries, in sh.  False if there is nothing to draw from.
template <bool BF>
__device__ __forceinline__ bool draw(const SampleParams &p, int row, uint32_t top, const Counts &c, Shared &sh)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (top >= kEnd<BF>) {
        if (threadIdx.x == 0) write_token(p, row, -1, 0.0f);
        return false;
    }
    Weigh weigh;
    weigh.top = top;
    weigh.most = value_at<BF>(top);
    weigh.per = 1.4426950408889634074 / (double)p.temperature[row];
    // ---- weight and number of each unit's entries ----
    for (int u = wave; u < kUnits; u += kWaves) {
        double mass = 0.0;
        int entries = 0;
        if (u >= (int)(top / kUnit)) {
            int n[8];
            c.unit(u, lane, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) entries += n[e];
            if (__ballot(entries)) {
                mass = sum_all(weigh.eight<BF>(u * kUnit + 8 * lane, n));
                entries = sum_all(entries);
            }
        }
        if (lane == 0) sh.mass[u] = mass, sh.entries[u] = entries;
    }
    __syncthreads();
    // ---- the borders, in one wave ----
    if (wave == 0) {
        const double m0 = sh.mass[2 * lane], m1 = sh.mass[2 * lane + 1];
        const int e0 = sh.entries[2 * lane], e1 = sh.entries[2 * lane + 1];
        const double mass_upto = sum_upto(m0 + m1, lane), before0 = mass_upto - (m0 + m1);  // before the lane's first unit
        const int entries_upto = sum_upto(e0 + e1, lane), n0 = entries_upto - (e0 + e1);
        const int all = from_lane(entries_upto, 63), top_k = p.top_k ? p.top_k[row] : 0;
        const double top_p = p.top_p ? p.top_p[row] : 1.0, min_p = p.min_p ? p.min_p[row] : 0.0;
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
__device__ __forceinline__ void find_entry(const SampleParams &p, int row, const uint16_t *logits, Shared &sh)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Wanted wanted(sh.place);
    int nth = sh.nth;
    Chunk next;
    next.load(logits, 0, p.vocab);
    const int chunks = chunks_of(logits, p.vocab);
    for (int c = 0; c < chunks; ++c) {
        const Chunk now = next;
        if (c + 1 < chunks) next.load(logits, c + 1, p.vocab);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int found = now.any(j, p.vocab) ? wanted.count(now.x[j]) : 0;
            int all = 0;
            if (__ballot(found))
#pragma unroll
                for (int bit = 0; bit < 4; ++bit) all += __popcll(__ballot(found >> bit & 1)) << bit;
            if (lane == 0) sh.found[j * kWaves + wave] = all;
        }
        __syncthreads();
        const int here = sh.found[lane], upto = sum_upto(here, lane);
        const u64 votes = __ballot(upto > nth);
        if (votes) {
            const int l = __builtin_ctzll(votes);
            if (l % kWaves != wave) return;
            const int before = from_lane(upto - here, l);
            uint32_t bits = 0;
            int index = 0;
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
                if (j == l / kWaves) bits = wanted.which(now.x[j]), index = now.index(j);
            const int own = __popc(bits), in_front = before + sum_upto(own, lane) - own;
            if (nth < in_front || nth >= in_front + own) return;
            for (int i = in_front; i < nth; ++i) bits &= bits - 1;
            p.token[row] = index + __builtin_ctz(bits);
            return;
        }
        nth -= from_lane(upto, 63);
        __syncthreads();
    }
}
static_assert(kPieces * kWaves == 64, "");

}  // namespace

template <bool BF>
__global__ __launch_bounds__(kThreads) void bcq_sample_kernel(SampleParams p)
{
    __shared__ __attribute__((aligned(16))) uint32_t table[32768];
    __shared__ Shared sh;
    const int row = blockIdx.x;
    const uint16_t *const logits = p.logits + row * p.ld;
    if (greedy(p, row)) {
        const u64 best = first_of_largest<BF>(logits, p.vocab, sh);
        if (threadIdx.x == 0) write_token(p, row, best == ~0ull ? -1 : (int)(uint32_t)best, best == ~0ull ? 0.0f : 1.0f);
        return;
    }
    const uint32_t top = count_values<BF>(logits, p.vocab, table, sh);
    if (draw<BF>(p, row, top, Counts{table, sh}, sh)) find_entry(p, row, logits, sh);
}

size_t sample_workspace_bytes(int, int) { return 0; }

hipError_t launch_sample(const SampleArgs &a, hipStream_t stream)
{
    const SampleParams p = {a.logits, a.temperature, a.top_p, a.min_p, a.uniform, a.top_k, a.token, a.probability, a.ld, a.vocab};
    if (a.bf16) bcq_sample_kernel<true><<<a.rows, kThreads, 0, stream>>>(p);
    else bcq_sample_kernel<false><<<a.rows, kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace bcq
