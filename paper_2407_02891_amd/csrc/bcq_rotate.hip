// Norm of the q and k heads, rotation by position, append of k and v to the paged cache: one pass over what the stacked projection left.
//
//   n = x weight / sqrt(mean(x^2) + eps);   (n_a, n_b) -> (n_a cos - n_b sin, n_b cos + n_a sin)
//
// Bound by the bytes: each value is read once and written once.  A lane has eight neighbouring elements (16 bytes) of a head, 8, 16 or 32 lanes have
// a head, and a wave has U rows of heads of one token: their loads are under way at once, and they share the cosines and sines, which depend on the place
// in the head alone.  A head's sum of squares goes over its lanes by lane exchanges; the other half of a pair in the first half of the rotated
// elements comes through the wave's own LDS, as it was loaded.
//
// Measured: 4096 tokens of 168 heads of 128, half of each rotated (353 MB): 76 us, 4.6 TB/s read and written (a copy of 2 GB: 4.7); one token of 80 heads 3.2 us, which
// is a launch and two reads in a row.  A first kernel with a head to a workgroup took 282 and 13 us.
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

namespace {

constexpr int kWaves = 4;

template <int CTRL>
__device__ __forceinline__ float other_lane(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// Sum over the L lanes of a head, in all of them.
template <int L>
__device__ __forceinline__ float head_sum(float v)
{
    v += other_lane<0xb1>(v);    // quad_perm: the neighbour
    v += other_lane<0x4e>(v);    // quad_perm: the other pair
    v += other_lane<0x141>(v);   // row_half_mirror: the other four of eight
    if (L >= 16) v += other_lane<0x140>(v);  // row_mirror: the other eight of sixteen
    if (L == 32) {
        const auto rows = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        v = __builtin_bit_cast(float, (unsigned)rows[0]) + __builtin_bit_cast(float, (unsigned)rows[1]);
    }
    return v;
}

}  // namespace

// L: lanes of a head.  WIDE: the rotated halves begin at multiples of eight elements (neighbouring pairs: end at one) and the table is aligned, so that
// cosines, sines and the other half come in 16-byte pieces.  U: rows of heads of a wave.
template <bool BF, int L, bool WIDE, int U>
__global__ __launch_bounds__(64 * kWaves) void bcq_rotate_kernel(RotateArgs p, int groups)
{
    constexpr int kHeads = 64 / L;
    __shared__ __attribute__((aligned(16))) uint16_t exchange[kWaves][U][64 * 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int index = blockIdx.x * kWaves + wave, t = index / groups, first = index % groups * (kHeads * U);
    if (t >= p.tokens) return;
    const int D = p.cache.head_dim, d = 8 * (lane % L), own = lane / L;
    const int qh = p.q_heads, kvh = p.cache.kv_heads, heads = qh + 2 * kvh;
    const bool in_head = d < D;
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int head = first + u * kHeads + own;
        raw[u] = u32x4{0, 0, 0, 0};
        if (in_head && head < heads) raw[u] = *reinterpret_cast<const u32x4 *>(p.qkv + (long long)t * p.ld_qkv + (long long)head * D + d);
    }
    const int slot = p.slots[t], position = min(max(p.positions[t], 0), p.max_position - 1);
    const int rot = p.rot_dim, half = rot >> 1;
    const bool turned = in_head && d < rot;
    u32x4 wq = {0, 0, 0, 0}, wk = wq;
    if (in_head && p.q_weight) wq = *reinterpret_cast<const u32x4 *>(p.q_weight + d);
    if (in_head && p.k_weight) wk = *reinterpret_cast<const u32x4 *>(p.k_weight + d);
    // element e of this lane: its angle, the distance to the other one of the pair (in the head), and the sign of the sine
    float cosine[8], sine[8];
    const float *const table = p.cos_sin + (long long)position * rot;
    const int pairs = WIDE ? (p.interleaved ? d >> 1 : d < half ? d : d - half) : 0;  // the first of the lane's pairs
#pragma unroll
    for (int e = 0; e < 8; ++e) cosine[e] = 1.0f, sine[e] = 0.0f;
    if (turned) {
        if (WIDE) {
            if (p.interleaved) {
                const f32x4 c = *reinterpret_cast<const f32x4 *>(table + pairs), z = *reinterpret_cast<const f32x4 *>(table + half + pairs);
#pragma unroll
                for (int e = 0; e < 8; ++e) cosine[e] = c[e >> 1], sine[e] = e & 1 ? z[e >> 1] : -z[e >> 1];
            } else {
                const float sign = d < half ? -1.0f : 1.0f;
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const f32x4 c = *reinterpret_cast<const f32x4 *>(table + pairs + i), z = *reinterpret_cast<const f32x4 *>(table + half + pairs + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) cosine[i + e] = c[e], sine[i + e] = sign * z[e];
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int at = d + e, pair = p.interleaved ? at >> 1 : at < half ? at : at - half;
                const bool second = p.interleaved ? at & 1 : at >= half;
                if (at < rot) cosine[e] = table[pair], sine[e] = second ? table[half + pair] : -table[half + pair];
            }
        }
    }
    if (!p.interleaved && rot > 0) {
#pragma unroll
        for (int u = 0; u < U; ++u) *reinterpret_cast<u32x4 *>(exchange[wave][u] + lane * 8) = raw[u];
    }
    asm volatile("" ::: "memory");  // (a wave's LDS instructions run in order)
    // the other half's place and weights
    u32x4 wq2 = wq, wk2 = wk;
    const int other = d < half ? d + half : d - half;
    if (!p.interleaved && turned) {
        if (WIDE) {
            if (p.q_weight) wq2 = *reinterpret_cast<const u32x4 *>(p.q_weight + other);
            if (p.k_weight) wk2 = *reinterpret_cast<const u32x4 *>(p.k_weight + other);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                uint32_t pair_q = 0, pair_k = 0;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int at = d + e + i, o = at < half ? at + half : at - half;
                    if (at < rot) {
                        if (p.q_weight) pair_q |= (uint32_t)p.q_weight[o] << (16 * i);
                        if (p.k_weight) pair_k |= (uint32_t)p.k_weight[o] << (16 * i);
                    }
                }
                wq2[e / 2] = pair_q, wk2[e / 2] = pair_k;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int head = first + u * kHeads + own;
        const bool is_q = head < qh, is_v = head >= qh + kvh;
        const bool normed = !is_v && (is_q ? p.q_weight : p.k_weight) != nullptr;
        float x[8], square = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const f32x2 v = to_float2<BF>(raw[u][e / 2]);
            x[e] = v.x, x[e + 1] = v.y;
            square = fmaf(v.x, v.x, fmaf(v.y, v.y, square));
        }
        const float unit = 1.0f / sqrtf(head_sum<L>(square) / (float)D + p.eps);
        const u32x4 w = is_q ? wq : wk, w2 = is_q ? wq2 : wk2;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const f32x2 weight = to_float2<BF>(w[e / 2]);
            y[e] = normed ? x[e] * unit * weight.x : x[e];
            y[e + 1] = normed ? x[e + 1] * unit * weight.y : x[e + 1];
        }
        u32x4 out = raw[u];
        if (rot > 0) {
            float z[8];
            if (p.interleaved) {
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = y[e ^ 1];
            } else {
                u32x4 far = {0, 0, 0, 0};
                const uint16_t *const mine = exchange[wave][u] + own * (L * 8);
                if (WIDE) {
                    far = *reinterpret_cast<const u32x4 *>(mine + (turned ? other : d));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const int a = d + e, b = a + 1;
                        const uint32_t low = mine[a < rot ? (a < half ? a + half : a - half) : a], high = mine[b < rot ? (b < half ? b + half : b - half) : b];
                        far[e / 2] = low | high << 16;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const f32x2 v = to_float2<BF>(far[e / 2]), weight = to_float2<BF>(w2[e / 2]);
                    z[e] = normed ? v.x * unit * weight.x : v.x;
                    z[e + 1] = normed ? v.y * unit * weight.y : v.y;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const bool first_turned = WIDE ? turned : d + e < rot, second_turned = WIDE ? turned : d + e + 1 < rot;
                const float a = first_turned ? fmaf(z[e], sine[e], y[e] * cosine[e]) : y[e];
                const float b = second_turned ? fmaf(z[e + 1], sine[e + 1], y[e + 1] * cosine[e + 1]) : y[e + 1];
                if (!is_v) out[e / 2] = from_float2<BF>(a, b);
            }
        } else if (normed) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) out[e / 2] = from_float2<BF>(y[e], y[e + 1]);
        }
        if (!in_head || head >= heads) continue;
        // (whole lines, which no one reads before this kernel has ended: kept out of the caches' way, 4096 tokens of 80 heads take 38.7 us instead of 47.1, of 168 heads 76
        // instead of 84, 512 of 80 9.2 instead of 10.1, few the same)
        if (is_q) {
            __builtin_nontemporal_store(out, reinterpret_cast<u32x4 *>(p.q_out + (long long)t * p.ld_q + (long long)head * D + d));
        } else if (slot >= 0 && slot < p.cache.num_pages * p.cache.page_size) {
            const int shift = __builtin_ctz(p.cache.page_size);
            const long long at = (long long)(slot >> shift) * p.cache.page_stride + (long long)(slot & (p.cache.page_size - 1)) * p.cache.slot_stride;
            if (is_v) __builtin_nontemporal_store(out, reinterpret_cast<u32x4 *>(p.v + at + (long long)(head - qh - kvh) * p.cache.head_stride + d));
            else __builtin_nontemporal_store(out, reinterpret_cast<u32x4 *>(p.k + at + (long long)(head - qh) * p.cache.head_stride + d));
        }
    }
}

namespace {

template <bool BF, int L, bool WIDE, int U>
void launch(const RotateArgs &a, hipStream_t stream)
{
    const int heads = a.q_heads + 2 * a.cache.kv_heads, groups = (heads + 64 / L * U - 1) / (64 / L * U);
    const long long waves = (long long)a.tokens * groups;
    bcq_rotate_kernel<BF, L, WIDE, U><<<(unsigned)((waves + kWaves - 1) / kWaves), 64 * kWaves, 0, stream>>>(a, groups);
}

template <bool BF, int L, bool WIDE>
void by_size(const RotateArgs &a, hipStream_t stream)
{
    // Four rows of heads a wave where there are many (4096 tokens of 64 + 16 heads of 128: one 57.9, four 46.9 us; of 168 heads 94.5 / 85.0), else one:
    // the longer program costs a short call 2 us (one token 3.1 / 5.3, 512 of 80 heads 10.1 / 10.6, 4096 of 36 heads of 64 15.5 / 17.0).
    const long long rows = (long long)a.tokens * (a.q_heads + 2 * a.cache.kv_heads) * L / 64;
    if (rows >= 32768) launch<BF, L, WIDE, 4>(a, stream);
    else launch<BF, L, WIDE, 1>(a, stream);
}

template <bool BF>
void by_dim(const RotateArgs &a, bool wide, hipStream_t stream)
{
    const int D = a.cache.head_dim;
    if (D <= 64) wide ? by_size<BF, 8, true>(a, stream) : by_size<BF, 8, false>(a, stream);
    else if (D <= 128) wide ? by_size<BF, 16, true>(a, stream) : by_size<BF, 16, false>(a, stream);
    else wide ? by_size<BF, 32, true>(a, stream) : by_size<BF, 32, false>(a, stream);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &a, hipStream_t stream)
{
    const bool wide = a.rot_dim % (a.interleaved ? 8 : 16) == 0 && (reinterpret_cast<uintptr_t>(a.cos_sin) & 15) == 0;
    if (a.cache.dtype == BCQ_BF16) by_dim<true>(a, wide, stream);
    else by_dim<false>(a, wide, stream);
    return hipGetLastError();
}

}  // namespace bcq
