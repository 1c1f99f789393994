// Attention over packed sequences: what the forward and the gradient kernels share.
//
// Rows.  The query heads of one key head see the same keys, so their queries are the rows of one problem: row r of (sequence,
// key head) is the query at place r / G of the sequence under head r % G of the G that share the key head.  One tile of rows then
// reads a tile of keys once for all heads of the group, the gradient of a shared key head is a sum over rows like any other, and
// a single new token fills G rows of a tile instead of one.
#pragma once
#include "block_ops.h"

namespace fuse {

constexpr int kMaxDim = 128;

struct Mat {
    void *p;
    long long token, head;                 // strides in elements
};

struct AttnArgs {
    Mat q, k, v, out, dout, dq, dk, dv;
    float *lse;                            // q_tokens x heads
    float *delta, *lse2;                   // gradients: sum of dout o out, and lse in base 2; see stat_at
    int *lifts;                            // gradients in fp16: of every 32 rows, see lift_at
    float *parts;                          // gradients of keys and values by split: (key token, key head, split, K or V) x dim
    int splits;
    const void *q_off, *k_off, *k_len;     // k_len NULL: the distances of k_off
    long long q_tokens, k_tokens;
    int seqs, heads, kv_heads, group, dim, causal, off64;
    float scale;
    unsigned div_mul, div_shift;           // rows / group, see place_of
};

struct Seq {
    long long q0, k0;                      // first query and first key
    int nq, nk;
};

__device__ __forceinline__ long long offset_at(const void *p, int i, int is64)
{
    return is64 ? static_cast<const long long *>(p)[i] : (long long)static_cast<const int *>(p)[i];
}

// Sequence s, cut down to the arrays whatever the offsets say (their lengths are below 2^31, which the host checks).
__device__ __forceinline__ Seq seq_at(const AttnArgs &a, int s)
{
    Seq x;
    const long long q0 = offset_at(a.q_off, s, a.off64), q1 = offset_at(a.q_off, s + 1, a.off64);
    const long long k0 = offset_at(a.k_off, s, a.off64), k1 = offset_at(a.k_off, s + 1, a.off64);
    x.q0 = min(max(q0, 0LL), a.q_tokens);
    x.k0 = min(max(k0, 0LL), a.k_tokens);
    x.nq = (int)(min(max(q1, x.q0), a.q_tokens) - x.q0);
    long long n = min(max(k1, x.k0), a.k_tokens) - x.k0;
    if (a.k_len)
        n = min(max(offset_at(a.k_len, s, a.off64), 0LL), n);
    x.nk = (int)n;
    return x;
}

// Lane `from`'s sequence, in scalar registers: a lookup by many lanes is one round of loads, not another one for the one that is found.
__device__ __forceinline__ long long of_lane(long long v, int from)
{
    return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)v, from) |
                       (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), from) << 32);
}
__device__ __forceinline__ Seq of_lane(const Seq &v, int from)
{
    Seq x;
    x.q0 = of_lane(v.q0, from);
    x.k0 = of_lane(v.k0, from);
    x.nq = __builtin_amdgcn_readlane(v.nq, from);
    x.nk = __builtin_amdgcn_readlane(v.nk, from);
    return x;
}

// Tiles of `tile` rows over all sequences without their lengths on the host: sequence s starts at tile
// floor(offset / tile) + s, which leaves it at least as many tiles as it needs (some stay empty).
__host__ __device__ inline long long first_tile(long long rows_before, int s, int tile) { return rows_before / tile + s; }

// A tile of a sequence: of its keys, or of its rows.
struct Work {
    Seq x;
    int seq;
    int first;                             // first row, or key
    bool any;
};

// Tile t, sequence by sequence: the sequence is the last one that starts at or before it.  A wave looks at 64 sequences at a time, first
// far apart, then between the two that are left: two rounds of loads for 4096 sequences, three for 262144.
template <bool KEYS>
__device__ __forceinline__ Work tile_at(const AttnArgs &a, int tile, long long t)
{
    const int lane = threadIdx.x & 63;
    Work w = {};
    long long start = 0;
    int low = 0;
    for (int step = (a.seqs + 63) / 64;; step = (step + 63) / 64) {
        const long long s = low + (long long)lane * step;
        Seq x = {};
        long long at = 0;
        bool starts = false;
        if (s < a.seqs) {
            x = seq_at(a, (int)s);
            at = first_tile(KEYS ? x.k0 : x.q0 * a.group, (int)s, tile);
            starts = at <= t;
        }
        const unsigned long long m = __ballot(starts);
        if (!m)
            return w;
        const int found = 63 - __builtin_clzll(m);
        low += found * step;
        if (step == 1) {
            w.x = of_lane(x, found);
            w.seq = low;
            start = of_lane(at, found);
            break;
        }
    }
    const long long first = (t - start) * tile;
    w.any = first < (KEYS ? (long long)w.x.nk : (long long)w.x.nq * a.group);
    w.first = (int)first;
    return w;
}

// Tiles in the order of their work, as block `b` finds its own: with a causal mask the last rows see most keys, and the first keys are
// seen by most rows, so tiles are taken by how far they are from the end of a sequence where that is little, most work first, over all
// sequences: the tiles with M ones behind them before those with M - 1.  Long blocks that begin last are what other compute units
// wait for: 8192 tokens in sequences of 2285, 2647 and 3260 take 333 us by sequence and 314 us in this order (queries' gradient),
// 572 and 521 us (keys').
//
// The search looks at every sequence, so beyond kSorted of them tiles go one after the other.  Whole calls, 32 heads over 8, dim 128, 8192 tokens
// in so many sequences of mixed length, one after the other and sorted (us, forward / gradients): 8 sequences 147 and 137 / 507 and 425; 16:
// 90 and 91 / 305 and 248; 24: 75 and 86 / 230 and 213; 32: 66 and 83 / 211 and 212; 64: 55 and 80 / 172 and 187.
constexpr int kSorted = 16;

// KEYS: tiles of keys, the first ones first; else of rows, the last ones first.
template <bool KEYS>
__device__ __forceinline__ Work work_of(const AttnArgs &a, int tile, unsigned b)
{
    if (a.seqs > kSorted)
        return tile_at<KEYS>(a, tile, b);
    Work w = {};
    const int lane = threadIdx.x & 63;
    int n = 0;                             // this lane's sequence's tiles
    Seq x = {};
    if (lane < a.seqs) {
        x = seq_at(a, lane);
        n = ((KEYS ? x.nk : x.nq * a.group) + tile - 1) / tile;
    }
    int most = 0, total = 0;
    for (int s = 0; s < a.seqs; ++s) {
        const int m = __builtin_amdgcn_readlane(n, s);
        most = max(most, m);
        total += m;
    }
    w.any = (int)b < total;
    if (!w.any)
        return w;
    // the largest M with more than b tiles that have at least M - 1 behind them: 64 values of M at a time
    int low = 1, before = 0;
    for (int step = (most + 63) / 64;; step = (step + 63) / 64) {
        const int m = low + lane * step;
        int count = 0, next = 0;
        for (int s = 0; s < a.seqs; ++s) {
            const int have = __builtin_amdgcn_readlane(n, s);
            count += max(0, have - m + 1);
            next += max(0, have - m);
        }
        const int last = 63 - __builtin_clzll(__ballot(count > (int)b));
        low = __builtin_amdgcn_readlane(m, last);
        before = __builtin_amdgcn_readlane(next, last);
        if (step == 1)
            break;
    }
    unsigned long long have = __ballot(n >= low);
    for (int i = (int)b - before; i > 0; --i)
        have &= have - 1;
    const int s = __builtin_ctzll(have);
    w.x = of_lane(x, s);
    w.seq = s;
    w.first = (KEYS ? __builtin_amdgcn_readlane(n, s) - low : low - 1) * tile;
    return w;
}

// Keys that the query at `place` sees: 0 .. the result.
__device__ __forceinline__ int seen_by(const AttnArgs &a, const Seq &x, int place)
{
    return a.causal ? min(max(place + x.nk - x.nq + 1, 0), x.nk) : x.nk;
}

// r / group for r < 2^31, with mul = floor(2^(31 + n) / group) + 1 and 2^n the next power of two: mul * group lies between 2^(31 + n)
// and 2^(31 + n) + 2^n, so the quotient of any 31 bits is exact.
__device__ __forceinline__ int place_of(const AttnArgs &a, int r)
{
    return a.group == 1 ? r : (int)(__umulhi((unsigned)r, a.div_mul) >> a.div_shift);
}

// First place whose query sees key j (nq: none).
__device__ __forceinline__ int first_that_sees(const AttnArgs &a, const Seq &x, int j)
{
    return a.causal ? min(max(j - (x.nk - x.nq), 0), x.nq) : 0;
}

template <typename T>
__device__ __forceinline__ T *row_of(const Mat &m, long long token, int head)
{
    return static_cast<T *>(m.p) + token * m.token + head * m.head;
}

// Place of a row's delta and lse2: key heads x rows, so that the rows of one problem follow each other.
__device__ __forceinline__ long long stat_at(const AttnArgs &a, long long token, int head)
{
    return (head / a.group * a.q_tokens + token) * a.group + head % a.group;
}

// Place of the lift of a sequence's rows r .. r + 31 (r a multiple of 32): key heads x tiles of 32 rows.
__host__ __device__ inline long long lift_tiles(const AttnArgs &a) { return first_tile(a.q_tokens * a.group, a.seqs, 32); }
__device__ __forceinline__ long long lift_at(const AttnArgs &a, const Work &w, int kvh, int r)
{
    return kvh * lift_tiles(a) + first_tile(w.x.q0 * a.group, w.seq, 32) + r / 32;
}

// Checks of both directions, and the arguments that both have (host).
int check_attn(const fuse_attn *f);
AttnArgs attn_args(const fuse_attn *f);
int check_rows(const fuse_attn *f, const void *p, int64_t token_ld, int64_t head_ld, int64_t heads, int64_t tokens, const char *what);

}  // namespace fuse
