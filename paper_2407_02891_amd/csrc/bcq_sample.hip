// The next tokens from logits, by temperature, top-k, top-p and min-p, with given random numbers.
//
//   w_i = exp((x_i - max x) / temperature); tokens in the order of descending x, then ascending index; the first top_k of them, S their weight;
//   of those the ones before which less than top_p S stands, and whose w is min_p or more; M their weight; the first at which more than u M stands.
//
// Logits of 16 bits have 65536 values, so a row is what its values' counts are: no token is sorted, and a weight is computed once for a value, in binary64,
// as the borders (u M in a sum of 131072 weights) ask for.  Counts are exact in any order.
//  * A row is cut into slices of less than 65536 entries, a workgroup each, which counts the values of its slice in LDS: 65536 counters of 16 bits, in descending
//    order of the value.  Units of 512 values that occur go to the workspace, with a map of them.
//  * A second launch has a workgroup a row: the weight and number of entries of each unit (all waves), then in one wave the borders one after the other: which
//    unit, which value in it, how many of its entries.  The entry itself is found by counting the value in the one slice that holds it.
//  * Rows of one slice need no workspace and no second launch.
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kValues = 65536, kUnit = 512, kUnits = kValues / kUnit;  // a unit: eight values a lane
constexpr int kMostSlice = 65528;                                      // entries that counters of 16 bits hold
constexpr int kMap = kUnits / 32;

typedef unsigned long long u64;

struct SampleParams {
    const uint16_t *logits;
    const float *temperature, *top_p, *min_p, *uniform;
    const int *top_k;
    int *token;
    float *probability;
    uint16_t *counts;  // [row of the launch][slice][kValues]
    uint32_t *maps;    // [row of the launch][slice][kMap]
    u64 *largest;      // [row of the launch][slice]: place of the largest value, then of the entry
    long long ld;
    int vocab, slices, slice, first_row;
};

// A value's place in descending order; +-0 are one value, NaN and -infinity have none.
template <bool BF>
__device__ __forceinline__ uint32_t place_of(uint32_t bits)
{
    if (bits == 0x8000u) return 0x7fffu;
    return bits & 0x8000u ? bits : bits ^ 0x7fffu;
}
template <bool BF>
constexpr uint32_t kFirst = BF ? 0x7fffu - 0x7f80u : 0x7fffu - 0x7c00u;  // +infinity's
template <bool BF>
constexpr uint32_t kEnd = BF ? 0xff80u : 0xfc00u;  // -infinity's

template <bool BF>
__device__ __forceinline__ bool counts(uint32_t place) { return place - kFirst<BF> < kEnd<BF> - kFirst<BF>; }

template <bool BF>
__device__ __forceinline__ double value_at(uint32_t place)
{
    return to_float<BF>(place & 0x8000u ? place : place ^ 0x7fffu);
}

// 2^y, y <= 0, to a few units of the last place: 2^n times the series of e^(r ln 2), |r| <= 1/2, whose next term is below 2^-53.
__device__ __forceinline__ double exp2_series(double y)
{
    if (!(y > -1020.0)) return 0.0;
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
};

__device__ __forceinline__ double from_lane(double v, int lane)
{
    const u64 b = __builtin_bit_cast(u64, v);
    return __builtin_bit_cast(double, (u64)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}
__device__ __forceinline__ int from_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

template <class T>
__device__ __forceinline__ T sum_upto(T v, int lane)
{
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) {
        const T below = __shfl_up(v, step);
        if (lane >= step) v += below;
    }
    return v;
}
template <class T>
__device__ __forceinline__ T sum_all(T v)
{
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
    return v;
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

// A row's entries from `from` to `end`, f(index, bits) of each, shared by `threads` threads.  Pieces of 16 bytes where they begin at such an address.
template <class F>
__device__ __forceinline__ void each_entry(const uint16_t *row, int from, int end, int thread, int threads, F f)
{
    const int head = (int)((16 - (reinterpret_cast<uintptr_t>(row + from) & 15)) & 15) / 2, first = min(from + head, end), pieces = (end - first) / 8;
    for (int i = from + thread; i < first; i += threads) f(i, (uint32_t)row[i]);
    const u32x4 *const body = reinterpret_cast<const u32x4 *>(row + first);
    for (int i = thread; i < pieces; i += threads) {
        const u32x4 x = body[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) f(first + 8 * i + e, x[e >> 1] >> 16 * (e & 1) & 0xffffu);
    }
    for (int i = first + 8 * pieces + thread; i < end; i += threads) f(i, (uint32_t)row[i]);
}

// Rows whose token is the first of the largest values, whatever the random number.
__device__ __forceinline__ bool greedy(const SampleParams &p, int row)
{
    return !(p.temperature[row] > 0.0f) || (p.top_k && p.top_k[row] == 1);
}

// The first entry of the largest value in [from, end): place << 32 | index, all ones if there is none.  All threads get it.
template <bool BF>
__device__ __forceinline__ u64 first_of_largest(const uint16_t *row, int from, int end, u64 *shared)
{
    u64 best = ~0ull;
    each_entry(row, from, end, threadIdx.x, kThreads, [&](int i, uint32_t bits) {
        const uint32_t place = place_of<BF>(bits);
        const u64 mine = (u64)place << 32 | (uint32_t)i;
        if (counts<BF>(place) && mine < best) best = mine;
    });
    best = least_of_all(best);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = best;
    __syncthreads();
    best = shared[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) best = shared[w] < best ? shared[w] : best;
    return best;
}

// How often each value occurs in [from, end).
template <bool BF>
__device__ __forceinline__ void count_values(const uint16_t *row, int from, int end, uint32_t *table)
{
    const u32x4 zero = {0, 0, 0, 0};
    for (int i = threadIdx.x; i < kValues / 8; i += kThreads) reinterpret_cast<u32x4 *>(table)[i] = zero;
    __syncthreads();
    each_entry(row, from, end, threadIdx.x, kThreads, [&](int, uint32_t bits) {
        const uint32_t place = place_of<BF>(bits);
        if (!counts<BF>(place)) return;
        // (entries that are all alike, a mask's, one by one would take 64 turns)
        const u64 here = __ballot(1), same = __ballot(place == (uint32_t)__builtin_amdgcn_readfirstlane((int)place));
        if (here == same) {
            if (__builtin_amdgcn_mbcnt_hi((uint32_t)(here >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)here, 0)) == 0)
                atomicAdd(table + (place >> 1), (uint32_t)__popcll(here) << 16 * (place & 1));
        } else {
            atomicAdd(table + (place >> 1), 1u << 16 * (place & 1));
        }
    });
    __syncthreads();
}

__device__ __forceinline__ u32x4 unit_of(const uint16_t *table, int unit, int lane)
{
    return *reinterpret_cast<const u32x4 *>(table + unit * kUnit + 8 * lane);
}

struct DrawShared {
    double mass[kUnits];
    int entries[kUnits];
    uint32_t map[kMap];
    u64 least[kWaves];
    int found[kWaves];
    uint32_t place;  // of the drawn value
    int nth;         // which of its entries
};

// The draw of a row from the counts of its slices' values.  table(slice), map: null for one slice whose table is in LDS.
struct Counted {
    const uint16_t *table;  // of slice 0; the next ones follow at kValues
    const uint32_t *maps;   // of slice 0, kMap words each (null: all units)
    int slices;
    // The counts of a unit: eight values a lane.
    __device__ __forceinline__ void unit(int u, int lane, int (&n)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = 0;
        for (int s = 0; s < slices; ++s) {
            if (maps && !(maps[s * kMap + (u >> 5)] >> (u & 31) & 1)) continue;
            const u32x4 c = unit_of(table + (long long)s * kValues, u, lane);
#pragma unroll
            for (int e = 0; e < 8; ++e) n[e] += (int)(c[e >> 1] >> 16 * (e & 1) & 0xffffu);
        }
    }
};

// Where a border lies: the value, what stands before it, and the number of its entries.
struct Border {
    uint32_t place;
    double before, weight;
    int entries_before, entries;
};

template <bool BF>
__device__ void draw(const SampleParams &p, int row, const Counted &c, const uint16_t *logits, DrawShared &sh)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // ---- which units occur ----
    if (c.maps) {
        if (wave == 0) {
            uint32_t all = 0;
            for (int s = 0; s < c.slices; ++s) all |= c.maps[s * kMap + (lane & (kMap - 1))];
            if (lane < kMap) sh.map[lane] = all;
        }
        __syncthreads();
    }
    // ---- the largest value: the first of the first unit ----
    int first_unit = kUnits;
#pragma unroll
    for (int m = kMap - 1; m >= 0; --m)
        if (sh.map[m]) first_unit = 32 * m + __builtin_ctz(sh.map[m]);
    if (first_unit == kUnits) {
        if (threadIdx.x == 0) {
            p.token[row] = -1;
            if (p.probability) p.probability[row] = 0.0f;
        }
        return;
    }
    int n[8];
    c.unit(first_unit, lane, n);
    int mine = 8;
#pragma unroll
    for (int e = 7; e >= 0; --e)
        if (n[e]) mine = e;
    const int leader = __builtin_ctzll(__ballot(mine < 8));
    Weigh weigh;
    weigh.top = first_unit * kUnit + 8 * leader + from_lane(mine, leader);
    weigh.most = value_at<BF>(weigh.top);
    weigh.per = 1.4426950408889634074 / (double)p.temperature[row];
    // ---- weight and number of each unit's entries ----
    for (int u = wave; u < kUnits; u += kWaves) {
        double mass = 0.0;
        int entries = 0;
        if (sh.map[u >> 5] >> (u & 31) & 1) {
            c.unit(u, lane, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                entries += n[e];
                if (__ballot(n[e])) mass = __builtin_fma(n[e], weigh.of<BF>(u * kUnit + 8 * lane + e), mass);
            }
            mass = sum_all(mass);
            entries = sum_all(entries);
        }
        if (lane == 0) sh.mass[u] = mass, sh.entries[u] = entries;
    }
    __syncthreads();
    // ---- the borders, in one wave ----
    if (wave == 0) {
        const double m0 = sh.mass[2 * lane], m1 = sh.mass[2 * lane + 1];
        const int e0 = sh.entries[2 * lane], e1 = sh.entries[2 * lane + 1];
        const double mass_upto = sum_upto(m0 + m1, lane);
        const int entries_upto = sum_upto(e0 + e1, lane);
        const double total = from_lane(mass_upto, 63);
        const int all = from_lane(entries_upto, 63);
        // The first value at which reached(weight up to and with it, entries up to and with it) holds; the last that occurs, if it never does.
        const auto find = [&](auto reached) {
            const double before0 = mass_upto - (m0 + m1);
            const int n0 = entries_upto - (e0 + e1);
            const bool in0 = e0 && reached(before0 + m0, n0 + e0), in1 = e1 && reached(mass_upto, entries_upto);
            u64 votes = __ballot(in0 || in1);
            const bool never = votes == 0;
            if (never) votes = 1ull << (63 - __builtin_clzll(__ballot(e0 || e1)));
            const int l = __builtin_ctzll(votes);
            const bool second = never ? from_lane(e1, l) != 0 : from_lane((int)in0, l) == 0;
            const int u = 2 * l + second;
            const double before = from_lane(second ? before0 + m0 : before0, l);
            const int entries_before = from_lane(second ? n0 + e0 : n0, l);
            int k[8];
            c.unit(u, lane, k);
            double w[8], own = 0.0;
            int many = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = weigh.of<BF>(u * kUnit + 8 * lane + e);
                own = __builtin_fma(k[e], w[e], own);
                many += k[e];
            }
            double upto = before + (sum_upto(own, lane) - own);
            int upto_entries = entries_before + sum_upto(many, lane) - many;
            Border b = {0, 0.0, 0.0, 0, 0};
            bool hit = false, any = false;
            Border last = b;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!k[e]) continue;
                const Border here = {(uint32_t)(u * kUnit + 8 * lane + e), upto, w[e], upto_entries, k[e]};
                upto = __builtin_fma(k[e], w[e], upto);
                upto_entries += k[e];
                any = true;
                last = here;
                if (!hit && reached(upto, upto_entries)) hit = true, b = here;
            }
            if (!hit) b = last;
            u64 hits = __ballot(hit);
            const int from = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(__ballot(any));
            Border r;
            r.place = (uint32_t)from_lane((int)b.place, from);
            r.before = from_lane(b.before, from);
            r.weight = from_lane(b.weight, from);
            r.entries_before = from_lane(b.entries_before, from);
            r.entries = from_lane(b.entries, from);
            return r;
        };
        // the end of what is kept: `kept` entries of the value at `end`, all of those before it
        uint32_t end = 0xffffffffu;
        int kept = 0;
        double sum = total;
        const int top_k = p.top_k ? p.top_k[row] : 0;
        if (top_k > 0 && top_k < all) {
            const Border b = find([&](double, int entries) { return entries >= top_k; });
            end = b.place, kept = min(top_k - b.entries_before, b.entries);
            sum = __builtin_fma(kept, b.weight, b.before);
        }
        const double top_p = p.top_p ? p.top_p[row] : 1.0;
        if (top_p < 1.0) {
            const double goal = top_p * sum;
            const Border b = find([&](double mass, int) { return mass >= goal; });
            int count = 1;
            if (goal > b.before && b.weight > 0.0) {
                const double more = __builtin_ceil((goal - b.before) / b.weight);
                count = more < b.entries ? max((int)more, 1) : b.entries;
            }
            if (b.place < end || (b.place == end && count < kept)) {
                end = b.place, kept = count;
                sum = __builtin_fma(kept, b.weight, b.before);
            }
        }
        const double min_p = p.min_p ? p.min_p[row] : 0.0;
        if (min_p > 0.0) {
            // the last value whose weight is that much: a step of the search asks for 64 of them
            const double least = min_p < 1.0 ? min_p : 1.0;
            uint32_t low = weigh.top, high = kEnd<BF>;  // low's weight is enough, high's is not
            while (high - low > 1) {
                const uint32_t step = (high - low + 63) / 64, at = low + lane * step;
                const int enough = __popcll(__ballot(at < high && weigh.of<BF>(at) >= least));
                low += (max(enough, 1) - 1) * step;
                high = min(high, low + step);
            }
            if (low < end) {
                // the first value behind it, what stands before that
                const double before0 = mass_upto - (m0 + m1);
                const uint32_t u = low / kUnit;
                const int l = u / 2;
                const double before = from_lane(u & 1 ? before0 + m0 : before0, l);
                int k[8];
                c.unit(u, lane, k);
                double own = 0.0;
                int many = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t place = u * kUnit + 8 * lane + e;
                    if (place <= low) own = __builtin_fma(k[e], weigh.of<BF>(place), own);
                    if (place == low) many = k[e];
                }
                sum = before + sum_all(own);
                end = low, kept = sum_all(many);
            }
        }
        // (below 1 by more than the sums round, so that an entry that is kept is found)
        const float u = p.uniform[row], share = u > 0.0f ? fminf(u, 1.0f - 0x1p-24f) : 0.0f;
        const double goal = (double)share * sum;
        const Border b = find([&](double mass, int) { return mass > goal; });
        const int most = b.place == end ? kept : b.entries;
        int nth = 0;
        if (b.weight > 0.0) {
            const double more = (goal - b.before) / b.weight;
            nth = more < most ? max((int)more, 0) : max(most - 1, 0);
        }
        if (lane == 0) {
            sh.place = b.place, sh.nth = nth;
            if (p.probability) p.probability[row] = (float)(b.weight / sum);
        }
    }
    __syncthreads();
    // ---- which entry of the row it is: the slice, then the wave's share of it ----
    const uint32_t place = sh.place;
    int nth = sh.nth, slice = 0;
    if (c.maps) {
        int before = 0;
        for (int first = 0; first < c.slices; first += 64) {
            const int s = first + lane;
            const bool there = s < c.slices && (c.maps[s * kMap + (place / kUnit >> 5)] >> (place / kUnit & 31) & 1);
            const int mine_here = there ? c.table[(long long)s * kValues + place] : 0;
            const int upto = before + sum_upto(mine_here, lane);
            const u64 votes = __ballot(upto > nth);
            if (votes) {
                const int l = __builtin_ctzll(votes);
                slice = first + l;
                nth -= from_lane(upto - mine_here, l);
                break;
            }
            before = from_lane(upto, 63);
        }
    }
    const int from = slice * p.slice, end = min(from + p.slice, p.vocab);
    const int share = (end - from + kWaves - 1) / kWaves, low = min(from + wave * share, end), high = min(low + share, end);
    const auto matches = [&](int i) { return i < high && place_of<BF>(logits[i]) == place; };
    int found = 0;
    for (int i = low; i < high; i += 64) found += __popcll(__ballot(matches(i + lane)));
    if (lane == 0) sh.found[wave] = found;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += sh.found[w];
    if (nth < before || nth >= before + found) return;
    for (int i = low; i < high; i += 64) {
        const u64 votes = __ballot(matches(i + lane));
        const int here = __popcll(votes);
        if (nth < before + here) {
            const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(votes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)votes, 0));
            if ((votes >> lane & 1) && rank == nth - before) p.token[row] = i + lane;
            return;
        }
        before += here;
    }
}

}  // namespace

// Rows of one slice: all of it.
template <bool BF>
__global__ __launch_bounds__(kThreads) void bcq_sample_row_kernel(SampleParams p)
{
    __shared__ __attribute__((aligned(16))) uint32_t table[kValues / 2];
    __shared__ DrawShared sh;
    const int row = p.first_row + blockIdx.x;
    const uint16_t *const logits = p.logits + row * p.ld;
    if (greedy(p, row)) {
        const u64 best = first_of_largest<BF>(logits, 0, p.vocab, sh.least);
        if (threadIdx.x == 0) {
            p.token[row] = best == ~0ull ? -1 : (int)(uint32_t)best;
            if (p.probability) p.probability[row] = best == ~0ull ? 0.0f : 1.0f;
        }
        return;
    }
    if (threadIdx.x < kMap) sh.map[threadIdx.x] = 0;
    count_values<BF>(logits, 0, p.vocab, table);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int u = wave; u < kUnits; u += kWaves) {
        const u32x4 c = unit_of(reinterpret_cast<const uint16_t *>(table), u, lane);
        if (__ballot(c[0] | c[1] | c[2] | c[3]) && lane == 0) atomicOr(sh.map + (u >> 5), 1u << (u & 31));
    }
    __syncthreads();
    draw<BF>(p, row, Counted{reinterpret_cast<const uint16_t *>(table), nullptr, 1}, logits, sh);
}

// A slice of a row: how often its values occur, or its largest.
template <bool BF>
__global__ __launch_bounds__(kThreads) void bcq_sample_slice_kernel(SampleParams p)
{
    __shared__ __attribute__((aligned(16))) uint32_t table[kValues / 2];
    __shared__ u64 least[kWaves];
    __shared__ uint32_t map[kMap];
    const int row = p.first_row + blockIdx.x / p.slices, slice = blockIdx.x % p.slices;
    const uint16_t *const logits = p.logits + row * p.ld;
    const int from = slice * p.slice, end = min(from + p.slice, p.vocab);
    if (greedy(p, row)) {
        const u64 best = first_of_largest<BF>(logits, from, end, least);
        if (threadIdx.x == 0) p.largest[blockIdx.x] = best;
        return;
    }
    if (threadIdx.x < kMap) map[threadIdx.x] = 0;
    count_values<BF>(logits, from, end, table);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int u = wave; u < kUnits; u += kWaves) {
        const u32x4 c = unit_of(reinterpret_cast<const uint16_t *>(table), u, lane);
        if (!__ballot(c[0] | c[1] | c[2] | c[3])) continue;
        *reinterpret_cast<u32x4 *>(p.counts + (long long)blockIdx.x * kValues + u * kUnit + 8 * lane) = c;
        if (lane == 0) atomicOr(map + (u >> 5), 1u << (u & 31));
    }
    __syncthreads();
    if (threadIdx.x < kMap) p.maps[blockIdx.x * kMap + threadIdx.x] = map[threadIdx.x];
}

// The draw of a row from its slices.
template <bool BF>
__global__ __launch_bounds__(kThreads) void bcq_sample_draw_kernel(SampleParams p)
{
    __shared__ DrawShared sh;
    const int row = p.first_row + blockIdx.x;
    const long long first = (long long)blockIdx.x * p.slices;
    if (greedy(p, row)) {
        if (threadIdx.x >= 64) return;
        u64 best = ~0ull;
        for (int s = threadIdx.x; s < p.slices; s += 64) best = p.largest[first + s] < best ? p.largest[first + s] : best;
        best = least_of_all(best);
        if (threadIdx.x == 0) {
            p.token[row] = best == ~0ull ? -1 : (int)(uint32_t)best;
            if (p.probability) p.probability[row] = best == ~0ull ? 0.0f : 1.0f;
        }
        return;
    }
    draw<BF>(p, row, Counted{p.counts + first * kValues, p.maps + first * kMap, p.slices}, p.logits + row * p.ld, sh);
}

namespace {

// Slices of a row, and rows of a launch.
struct SamplePlan {
    int slices, slice, rows;
};
SamplePlan sample_plan(int rows, int vocab)
{
    SamplePlan s;
    s.slices = (vocab + kMostSlice - 1) / kMostSlice;
    const int share = compute_units() / rows, most = (vocab + 4095) / 4096;  // a workgroup a compute unit, none with fewer than 4096 entries
    if (s.slices < share) s.slices = share < most ? share : most > s.slices ? most : s.slices;
    s.slice = ((vocab + s.slices - 1) / s.slices + 7) / 8 * 8;
    s.slices = (vocab + s.slice - 1) / s.slice;
    s.rows = s.slices == 1 ? rows : 1024 / s.slices;
    if (s.rows < 1) s.rows = 1;
    if (s.rows > rows) s.rows = rows;
    return s;
}

size_t rounded(size_t bytes) { return (bytes + 15) & ~(size_t)15; }

}  // namespace

size_t sample_workspace_bytes(int rows, int vocab)
{
    const SamplePlan s = sample_plan(rows, vocab);
    const size_t n = (size_t)s.rows * s.slices;
    return s.slices == 1 ? 0 : n * kValues * 2 + n * kMap * 4 + rounded(n * 8);
}

hipError_t launch_sample(const SampleArgs &a, hipStream_t stream)
{
    const SamplePlan s = sample_plan(a.rows, a.vocab);
    const size_t n = (size_t)s.rows * s.slices;
    SampleParams p = {};
    p.logits = a.logits, p.temperature = a.temperature, p.top_p = a.top_p, p.min_p = a.min_p, p.uniform = a.uniform, p.top_k = a.top_k;
    p.token = a.token, p.probability = a.probability, p.ld = a.ld, p.vocab = a.vocab, p.slices = s.slices, p.slice = s.slice;
    char *const ws = static_cast<char *>(a.workspace);
    if (s.slices > 1) {
        p.counts = reinterpret_cast<uint16_t *>(ws);
        p.maps = reinterpret_cast<uint32_t *>(ws + n * kValues * 2);
        p.largest = reinterpret_cast<u64 *>(ws + n * kValues * 2 + n * kMap * 4);
    }
    for (int first = 0; first < a.rows; first += s.rows) {
        const int rows = a.rows - first < s.rows ? a.rows - first : s.rows;
        p.first_row = first;
        if (s.slices == 1) {
            if (a.bf16) bcq_sample_row_kernel<true><<<rows, kThreads, 0, stream>>>(p);
            else bcq_sample_row_kernel<false><<<rows, kThreads, 0, stream>>>(p);
            continue;
        }
        if (a.bf16) {
            bcq_sample_slice_kernel<true><<<rows * s.slices, kThreads, 0, stream>>>(p);
            bcq_sample_draw_kernel<true><<<rows, kThreads, 0, stream>>>(p);
        } else {
            bcq_sample_slice_kernel<false><<<rows * s.slices, kThreads, 0, stream>>>(p);
            bcq_sample_draw_kernel<false><<<rows, kThreads, 0, stream>>>(p);
        }
    }
    return hipGetLastError();
}

}  // namespace bcq
