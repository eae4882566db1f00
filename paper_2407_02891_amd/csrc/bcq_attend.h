// Shared by the two attention kernels (not public): their parameters, what a request needs, and the softmax's running statistics.
#pragma once
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

struct AttendParams {
    const uint16_t *k, *v, *q;
    const int *q_start, *kv_len, *pages;
    uint16_t *out;
    float *part;       // unnormalised sums of a split request: [slot][kv head][row][head_dim of the kernel]
    f32x2 *stat;       // their (maximum, sum of weights): [slot][kv head][row]
    long long ld_q, ld_out, page_stride, head_stride;
    int slot_stride;
    int tokens, requests, kv_heads, group;  // group: query heads of a kv head
    int head_dim, page_shift, num_pages, max_pages;
    int max_new, window, causal;
    float scale;       // times log2 e
    int rows;          // requests of at most this many rows (new tokens times group) are the stream kernel's
    int workers;       // stream kernel: waves per kv head
    int join_rows;     // its join: rows of a workgroup
    int parts;         // chunk kernel: pieces that a tile's keys are cut into
};

// One request as the kernels see it, whatever the arrays hold: rows of q inside 0 .. tokens, keys inside its row of pages.
struct Request {
    int start, n;      // new tokens
    int todo;          // those of them that are computed
    int len;           // keys
    int begin, end;    // keys that any of them sees
};

__device__ __forceinline__ Request load_request(const AttendParams &p, int r)
{
    Request q;
    q.start = min(max(p.q_start[r], 0), p.tokens);
    q.n = min(max(p.q_start[r + 1], q.start), p.tokens) - q.start;
    q.todo = min(q.n, p.max_new);
    q.len = (int)min((long long)max(p.kv_len[r], 0), (long long)p.max_pages << p.page_shift);
    const int first = q.len - q.n;  // position of the first new token
    q.end = p.causal ? min(max(first + q.todo, 0), q.len) : q.len;
    q.begin = p.window ? min(max(first + 1 - p.window, 0), q.end) : 0;
    return q;
}

// Keys that token i of a request sees: [begin, end), none if end <= begin.
__device__ __forceinline__ void visible_keys(const AttendParams &p, const int n, const int len, int i, int &begin, int &end)
{
    const int position = len - n + i;
    end = p.causal ? min(position + 1, len) : len;
    begin = p.window ? max(position + 1 - p.window, 0) : 0;
}

// The last request of which begins(r) holds, all lanes together (begins(0) is taken to hold, and begins is never true again once it is false).
template <class F>
__device__ __forceinline__ int last_request(const AttendParams &p, int lane, F begins)
{
    int r = 0;
    for (int high = p.requests; high - r > 1;) {
        const int stride = (high - r + 63) / 64, probe = r + lane * stride;
        const int count = __popcll(__ballot(probe < high && begins(probe)));
        r += max(count - 1, 0) * stride;
        high = min(high, r + stride);
    }
    return r;
}

__device__ __forceinline__ int page_of(const AttendParams &p, int r, int key)
{
    return min(max(p.pages[(long long)r * p.max_pages + (key >> p.page_shift)], 0), p.num_pages - 1);
}

// The same where all lanes of a wave ask for one key: a scalar load, which does not wait behind the wave's other loads (chunk kernel, 5 tokens over 131077 keys: 98 us
// against 104 with a vector load, 4 x 1024 tokens, heads of 64, 145 against 160).
__device__ __forceinline__ int page_of_all(const AttendParams &p, int r, int key)
{
    typedef const __attribute__((address_space(4))) int *scalar_int;
    const int *const at = p.pages + (long long)r * p.max_pages + (__builtin_amdgcn_readfirstlane(key) >> p.page_shift);
    return min(max(*(scalar_int)at, 0), p.num_pages - 1);
}

// What elements behind head_dim are loaded from.
static __device__ __attribute__((aligned(16))) const uint16_t g_zeros[8] = {};

// The softmax's weights are 2^(score - base), base = the running maximum - lift.  The maximum is renewed only when a score passes it by `grow`, so that sums are
// hardly ever rescaled.  The weights become 16-bit numbers for the second product: bfloat16 has the range of binary32, but binary16 ends at 2^16 and loses bits below
// 2^-14, so there weights reach up to 2^15.  Small ones count where the key that has the most weight has a value near zero: without the lift, 1000 keys 13
// nats below such a key came out 3 % off, and 131072 keys 18 nats below it were lost.  The lift that GROW leaves: 7 bits (full precision down to 14.5 nats below the
// maximum) or 14 (19.4).
template <bool BF, int GROW>
struct Weights {
    static constexpr float grow = BF ? 8.0f : GROW, lift = BF ? 0.0f : 15.0f - GROW;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 2^x, x <= 0, that sums are multiplied by: never zero, which would make a NaN of a sum that is infinite.
__device__ __forceinline__ float shrink_by(float x) { return fmaxf(exp2_fast(x), 0x1p-149f); }

// Joining the pieces of a row: piece i has its sums in part and its (maximum, weight) in stat at at(i).
struct Slots {
    long long first, step;
    __device__ __forceinline__ long long operator()(int i) const { return first + i * step; }
};
constexpr int kJoinAhead = 8;  // pieces requested together

// y, weight: sums over the pieces from + share, from + share + STRIDE, .. < end, relative to the maximum over all pieces from .. end - 1.
template <int DT, int STRIDE, class At>
__device__ __forceinline__ void join_pieces(const AttendParams &p, const At &at, int from, int end, int share, int lane, float (&y)[DT / 64], float &weight)
{
    constexpr int E = DT / 64;  // elements of a lane
    float most = -INFINITY;
    for (int i = from + lane; i < end; i += 64) most = fmaxf(most, p.stat[at(i)].x);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    const float base = most == -INFINITY ? 0.0f : most;
    weight = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = 0.0f;
    for (int c = from + share; c < end; c += 64 * STRIDE) {  // sixty-four pieces, a lane has the statistics of one
        const int mine = c + lane * STRIDE, n = min((end - 1 - c) / STRIDE + 1, 64);
        const f32x2 stat = p.stat[at(min(mine, end - 1))];
        const float scale = shrink_by(stat.x - base);
        if (mine < end) weight = fmaf(stat.y, scale, weight);
        for (int i = 0; i < n; i += kJoinAhead) {
            float part[kJoinAhead][E];
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) part[j][e] = p.part[at(c + min(i + j, n - 1) * STRIDE) * DT + lane * E + e];
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j) {
                const float times = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scale), min(i + j, n - 1)));
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] = i + j < n ? fmaf(part[j][e], times, y[e]) : y[e];
            }
        }
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) weight += __shfl_xor(weight, s);
}

// The chunk kernel (bcq_attend_chunk.hip): requests of more than p.rows rows.  dim: the padded head_dim.
int chunk_parts(int tokens, int requests, int max_new, int group, int kv_heads, int dim, long long most_keys);
void launch_chunks(const AttendParams &p, int dim, bool any, bool passing, bool bf16, hipStream_t s);

}  // namespace bcq
