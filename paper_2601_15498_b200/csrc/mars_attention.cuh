// Pieces shared by the tree-attention kernels: call parameters, the split of a ragged batch's work
// over the thread blocks, the draft tree's ancestor masks, partial results and their merge.
//
// Work is cut along the keys, evenly over the grid.  An item is (sequence, KV head, tile of query
// rows); its keys come in units of a kernel-specific number of keys, chosen so that every unit costs
// about the same; the units of all items, laid end to end, are dealt to the blocks in equal contiguous
// ranges.  Lengths live on the device, so every block works the split out
// by itself (one pass over seq_len).  A block's range begins and ends anywhere, so the first and the
// last item of it may be shared with neighbours: such a block leaves a partial result (unnormalised
// output, maximum, sum) in the workspace, and the last one to arrive merges them in block order.
// Results therefore depend on the sizes alone.
#pragma once

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "mars_kv.cuh"
#include "mars_stream.cuh"

namespace mars {

// Tile shapes: query rows per tile, keys per unit of the split, the least number of units per block (a
// block more costs a partial result and its merge), and what an item costs besides its keys
// (decoding, Q, masks, the pipeline's fill and drain, the result) in units.  Counting that in evens out
// the blocks where items are short.  Measured, us without / as here / with twice that: 64 tokens 122 / 106 /
// 110, 64 chains 236 / 197 / 206; four prompts 188 / 131 / 143, 64 trees 485 / 419 / 413 (TileShape).
template <int kRows>
struct RowsShape {
    static __device__ constexpr int rows(int) { return kRows; }
    static constexpr int kFixed = kRows >= 24 ? 8 : 6, kLeast = 2;
    static __host__ __device__ constexpr int unit_keys(int) { return 64; }
};
struct TileShape {
    static constexpr int kMost = 256;
    static __device__ int rows(int tile_rows) { return tile_rows; }    // 128 or 256, chosen per call
    static constexpr int kFixed = 4, kLeast = 4;
    // up to 128 rows fill one of the kernel's two accumulators; the two then share the keys
    static __host__ __device__ constexpr int unit_keys(int rows) { return rows > 128 ? 128 : 256; }
};

struct AttnParams {
    KvView kv;
    unsigned char *layer;            // this layer's pages
    const float *scales;             // this layer's [2][kv_heads]
    const unsigned char *q;
    unsigned char *out;
    int64_t q_row, q_head, out_row, out_head;   // elements
    const int32_t *parent;           // or null: chains
    const int32_t *count;            // or null
    int32_t *status;                 // or null
    int shared_parent;
    int B, N, group;
    int tile_rows;                   // query rows per tile of TileShape
    uint64_t group_inv;              // floor(2^64 / group) + 1 (unused for 1)
    float scale_log2;                // softmax scale * log2(e)
    unsigned give_up;                // blocks from this one on give up (test hook)
    unsigned *counters;              // [grid]
    float *partial;                  // [2 * grid] slots of rows * (d + 2) floats
};

// The reference maximum of a row is kept in units of S = q K^T (q scaled, see row_scale), where it is finite and
// exact; `rs` (below) brings differences of scores to log2 units.  Kept in log2 units, its rounding would pass
// the 2^15 that P has room for once scores pass 2^28, and overflow with them.

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// Nodes of sequence b that take part, and whether its pages hold them; len < 0 counts as no room.
__device__ __forceinline__ int attn_nodes(const AttnParams &p, int b, int *len, int *status)
{
    const int count = p.count ? p.count[b] : p.N, l = p.kv.seq_len[b], cap = kv_capacity(p.kv, b);
    const int n = min(max(count, 0), p.N);
    const bool room = n == 0 || (l >= 0 && (int64_t)l + n <= cap);
    *len = l;
    *status = room ? MARS_SEQ_OK : MARS_SEQ_NO_ROOM;
    return room ? n : 0;
}

// Node of a query row (rows of a KV head are node-major): row / group.
__device__ __forceinline__ int attn_node(const AttnParams &p, int row)
{
    return p.group == 1 ? row : (int)__umul64hi((uint64_t)(uint32_t)row, p.group_inv);
}

template <class S>
__device__ __forceinline__ int attn_tiles(const AttnParams &p, int n) { return (n * p.group + S::rows(p.tile_rows) - 1) / S::rows(p.tile_rows); }

template <class S>
__device__ __forceinline__ int attn_tile_rows(const AttnParams &p, int n, int mt) { return min(S::rows(p.tile_rows), n * p.group - mt * S::rows(p.tile_rows)); }

// Keys that the rows of tile mt (rows mt*M .. of n*group) may see: all nodes of a tree, the nodes up
// to the tile's last one of a chain.
template <class S>
__device__ __forceinline__ int attn_keys(const AttnParams &p, int len, int n, int mt)
{
    if (p.parent) return len + n;
    return len + min(n, attn_node(p, (mt + 1) * S::rows(p.tile_rows) - 1) + 1);
}

// Units of an item: its fixed cost, then its keys.
template <class S>
__device__ __forceinline__ int attn_units(const AttnParams &p, int len, int n, int mt)
{
    const int uk = S::unit_keys(attn_tile_rows<S>(p, n, mt));
    return S::kFixed + (attn_keys<S>(p, len, n, mt) + uk - 1) / uk;
}

// a / b for a >= 0, b > 0; nearly always in 32 bits, where it takes a third of the time.
__device__ __forceinline__ int64_t attn_div(int64_t a, int64_t b)
{
    if (((uint64_t)a | (uint64_t)b) >> 32 == 0) return (uint32_t)a / (uint32_t)b;
    return a / b;
}

// Units of one KV head of a sequence; whole warps call (lanes share the tiles of a long chain).
template <class S>
__device__ __forceinline__ int64_t attn_head_units(const AttnParams &p, int len, int n)
{
    if (n == 0) return 0;
    const int tiles = attn_tiles<S>(p, n);
    if (p.parent || tiles == 1)
        return (int64_t)(tiles - 1) * attn_units<S>(p, len, n, 0) + attn_units<S>(p, len, n, tiles - 1);
    int64_t u = 0;
    for (int mt = threadIdx.x & 31; mt < tiles; mt += 32) u += attn_units<S>(p, len, n, mt);
#pragma unroll
    for (int o = 16; o; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    return u;
}

// What the block's first sequences come to, in shared memory: segments are decoded from here.
constexpr int kSeqCache = 32;
struct AttnSeqs {
    int64_t units[kSeqCache];     // per KV head
    int len[kSeqCache], n[kSeqCache];
};

struct AttnRange {
    int64_t begin, end;     // this block's units
    int64_t per;            // units per block
    int64_t at;             // first unit of sequence b
    int b, b0;              // sequence of the unit reached, of unit `begin`
};

// The block's share of the batch (all threads call; kThreads = blockDim.x).  Block 0 also reports the
// status of sequences that have no work.
template <class S, int kThreads>
__device__ AttnRange attn_split(const AttnParams &p, AttnSeqs *seqs)
{
    __shared__ int64_t s_sum[kThreads / 32 + 1];
    __shared__ int64_t s_at;
    __shared__ int s_b;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // sequences go to threads in contiguous chunks; where a sequence has many tiles, to warps
    const bool by_warp = !p.parent && (int64_t)p.N * p.group > S::rows(p.tile_rows);
    const int who = by_warp ? warp : tid, of = by_warp ? kThreads / 32 : kThreads;
    const int chunk = (p.B + of - 1) / of;
    const int lo = min(who * chunk, p.B), hi = min(lo + chunk, p.B);
    int64_t sum = 0;
    int len = 0, n = 0;           // of the last sequence of the chunk; with one per chunk nothing is read twice
    for (int b = lo; b < hi; ++b) {
        int st;
        n = attn_nodes(p, b, &len, &st);
        sum += attn_head_units<S>(p, len, n) * p.kv.kv_heads;
        if (n == 0 && p.status && blockIdx.x == 0) p.status[b] = st;
    }
    const int64_t chunk_sum = sum;
    if (by_warp && lane) sum = 0;
    int64_t inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) s_sum[warp] = inc;
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    AttnRange r;
    r.per = max(attn_div(total + gridDim.x - 1, gridDim.x), (int64_t)S::kLeast);
    r.begin = min(r.per * blockIdx.x, total);
    r.end = min(r.begin + r.per, total);
    int64_t at = before + inc - sum;
    if (by_warp) at = __shfl_sync(0xffffffffu, at, 0);
    if (r.begin < r.end && at <= r.begin && r.begin < at + chunk_sum) {
        if (chunk == 1) {
            s_b = lo;
            s_at = at;
        } else {
            for (int b = lo; b < hi; ++b) {
                int st;
                n = attn_nodes(p, b, &len, &st);
                const int64_t u = attn_head_units<S>(p, len, n) * p.kv.kv_heads;
                if (r.begin < at + u) { s_b = b; s_at = at; break; }
                at += u;
            }
        }
    }
    __syncthreads();
    r.b = r.b0 = s_b;
    r.at = s_at;
    if (r.begin < r.end) {
        if (chunk == 1) {
            const int i = lo - r.b0;
            if (lo < hi && i >= 0 && i < kSeqCache) {
                seqs->units[i] = attn_div(chunk_sum, p.kv.kv_heads); seqs->len[i] = len; seqs->n[i] = n;
            }
        } else {
            // whole warps where lanes share a sequence's tiles, else a lane per sequence
            for (int i = by_warp ? warp : tid; i < kSeqCache && r.b0 + i < p.B; i += of) {
                int st;
                n = attn_nodes(p, r.b0 + i, &len, &st);
                const int64_t u = attn_head_units<S>(p, len, n);
                seqs->units[i] = u; seqs->len[i] = len; seqs->n[i] = n;
            }
        }
    }
    __syncthreads();
    return r;
}

// One stretch of an item that a block works on.
struct AttnSegment {
    int b, head, tile;
    int len, n, keys;        // committed tokens, nodes, keys of the tile
    int unit0, unit1;        // this block's units of keys, of `units`; none if unit0 >= unit1
    int units;
    int64_t span;            // units on from here to the next segment
    int c0, c1;              // first and last block with keys of the item
    int64_t item;            // first unit of the item in the whole batch
};

// Decodes the segment that begins at unit u (whole warps, uniform); moves r.b / r.at on as sequences end.
template <class S>
__device__ __forceinline__ AttnSegment attn_segment(const AttnParams &p, const AttnSeqs *seqs, AttnRange &r, int64_t u)
{
    AttnSegment s;
    int st;
    int64_t hu;
    for (;;) {
        const int i = r.b - r.b0;
        if (i < kSeqCache) {
            s.n = seqs->n[i]; s.len = seqs->len[i]; hu = seqs->units[i];
        } else {
            s.n = attn_nodes(p, r.b, &s.len, &st);
            hu = attn_head_units<S>(p, s.len, s.n);
        }
        if (u < r.at + hu * p.kv.kv_heads) break;
        r.at += hu * p.kv.kv_heads;
        ++r.b;
    }
    s.b = r.b;
    const int64_t in_seq = u - r.at;
    s.head = (int)attn_div(in_seq, hu);
    int64_t rest = in_seq - s.head * hu;
    int64_t item = r.at + s.head * hu;       // first unit of the item in the whole batch
    s.tile = 0;
    s.units = attn_units<S>(p, s.len, s.n, 0);
    if (p.parent) {
        const int last = attn_tiles<S>(p, s.n) - 1;
        s.tile = (int)min(attn_div(rest, s.units), (int64_t)last);
        rest -= (int64_t)s.tile * s.units;
        item += (int64_t)s.tile * s.units;
        if (s.tile == last) s.units = attn_units<S>(p, s.len, s.n, last);
    } else {
        // lanes look at 32 tiles at a time for the one that holds unit `rest`
        const int tiles = attn_tiles<S>(p, s.n), lane = threadIdx.x & 31;
        if (tiles > 1) {
            for (int mt0 = 0;; mt0 += 32) {
                const int64_t mine = mt0 + lane < tiles ? attn_units<S>(p, s.len, s.n, mt0 + lane) : 0;
                int64_t inc = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int64_t t = __shfl_up_sync(0xffffffffu, inc, o);
                    if (lane >= o) inc += t;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, rest < inc);
                if (hit || mt0 + 32 >= tiles) {
                    const int l = hit ? __ffs((int)hit) - 1 : 0;
                    s.tile = mt0 + l;
                    s.units = (int)__shfl_sync(0xffffffffu, mine, l);
                    const int64_t skip = __shfl_sync(0xffffffffu, inc - mine, l);
                    rest -= skip;
                    item += skip;
                    break;
                }
                const int64_t all = __shfl_sync(0xffffffffu, inc, 31);
                rest -= all;
                item += all;
            }
        }
    }
    s.keys = attn_keys<S>(p, s.len, s.n, s.tile);
    s.span = min((int64_t)s.units - rest, r.end - u);
    s.unit0 = max((int)rest - S::kFixed, 0);
    s.unit1 = max((int)(rest + s.span) - S::kFixed, 0);
    s.units -= S::kFixed;
    s.c0 = (int)attn_div(item + S::kFixed, r.per);
    s.c1 = (int)attn_div(item + S::kFixed + s.units - 1, r.per);
    s.item = item;
    return s;
}

// Score scale of a query row in log2 units: never 0 or infinite, so that differences of 0 and of infinity stay that.
__device__ __forceinline__ float row_log2(const AttnParams &p, int head, float up)
{
    return fminf(fmaxf(p.scale_log2 * p.scales[head] * up, 1.17549435e-38f), 3.40282347e38f);
}

template <int DT>
__device__ __forceinline__ float2 widen2(uint32_t w)
{
    if constexpr (DT == MARS_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return f16x2_to_float2(w);
}

// Power of two that brings a row whose largest magnitude is m into [1, 2), and its inverse.
__device__ __forceinline__ void row_scale(float m, float *down, float *up)
{
    const uint32_t e = (__float_as_uint(m) >> 23) & 0xffu;
    if (e == 0u || e >= 254u) { *down = e == 0u ? 1.0f : 0x1p-127f; *up = e == 0u ? 1.0f : 0x1p127f; }
    else { *down = __uint_as_float((254u - e) << 23); *up = __uint_as_float(e << 23); }
    // e == 0: zero or subnormal rows count as they are (their products vanish next to any other term);
    // e >= 254: 2^-127 is subnormal; infinities stay infinities
}

// 8 consecutive output values at element `at` (16-byte aligned).
template <int DT>
__device__ __forceinline__ void store_out8(unsigned char *out, int64_t at, const float *x)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = DT == MARS_BF16 ? bf16x2_from(x[2 * i], x[2 * i + 1]) : f16x2_from(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<uint4 *>(out + at * 2) = make_uint4(w[0], w[1], w[2], w[3]);
}

constexpr int kAttnSms = 148;                   // SM count that the grids are sized for
constexpr size_t kAttnCounterBytes = 4096;      // one counter per block, at the head of the workspace

// Kernel for many query rows per KV head (mars_attention_tile.cu).
constexpr int kTileMaxTree = 128;               // its mask store holds trees of up to this many nodes
size_t attn_tile_partial_bytes(int d);
mars_status_t attn_tile_launch(const AttnParams &p, int d, int dt, cudaStream_t st);

// Ancestor-or-self masks of nodes first .. first + nodes - 1, and which of them are computed.
//   mask   [nodes][words]  bit m of node i: m is i or an ancestor of i
//   live   [nodes]         1: node takes part; absent nodes (no way to the root) do not
// Trees only; the nthr threads that share `sync` call.  par is scratch for n ints, *s_bad one int.
// Returns MARS_SEQ_BAD_TREE if the parents are no tree (then only the root is live).
template <class Sync>
__device__ __forceinline__ int attn_tree_masks(const AttnParams &p, int b, int n, int first, int nodes, int *par,
                                               uint32_t *mask, int words, unsigned char *live, int *s_bad, int tid,
                                               int nthr, Sync sync)
{
    const int32_t *g = p.shared_parent ? p.parent : p.parent + (int64_t)b * p.N;
    if (tid == 0) *s_bad = 0;
    sync();
    for (int i = tid; i < n; i += nthr) {
        const int x = g[i];
        if (i == 0 ? x != -1 : (x >= i || x < -1)) *s_bad = 1;
        par[i] = x;
    }
    sync();
    const bool bad = *s_bad != 0;
    for (int i = tid; i < nodes; i += nthr) {
        const int node = first + i;
        bool ok = node < n;
        uint32_t *m = mask + i * words;
        for (int w = 0; w < words; ++w) m[w] = 0u;
        if (bad) {
            ok = node == 0;
            if (ok) m[0] = 1u;
        } else if (ok) {
            int x = node;
            for (;;) {                      // parents fall strictly: at most n steps
                m[x >> 5] |= 1u << (x & 31);
                if (x <= 0) break;
                const int up = par[x];
                if (up < 0) { ok = false; break; }
                x = up;
            }
        }
        live[i] = ok;
    }
    sync();
    return bad ? MARS_SEQ_BAD_TREE : MARS_SEQ_OK;
}

}  // namespace mars
