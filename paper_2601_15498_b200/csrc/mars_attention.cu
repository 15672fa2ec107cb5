// libmars: attention of draft nodes over the paged 4-bit cache.
//
// O = softmax(scale * q K^T) V with K, V = code * scale of E2M1 / E4M3 blocks.  A code has 2
// significant bits and a block scale 4, so code * scale is exact in fp16 (6 bits, 2^-10 .. 2688) and
// both products run on the tensor cores in fp16 with fp32 accumulation.  q is brought to fp16 after
// a power-of-two scaling of its row (largest element in [1, 2)): bf16 and fp16 values keep all their
// bits down to 2^-14 of the row's largest and an error below 2^-25 of it beyond.  The heads' fp32
// scales are factored out of both sums.
//
// Kernel for few query rows per KV head (`attn_rows_kernel`, tiles of 8, 16, 24 or 32 rows): bound by
// reading the cache.  The page bytes go through a small shared-memory ring straight into the register
// fragments of mma.sync -- no unpacked copy of K or V exists anywhere.  Keys and values are the 16-row
// operand, the query rows the 8-column one, so a token of four heads to a KV head wastes half of a
// tile, not three quarters, and every unpacked fragment serves all query rows of the tile:
//   S^T (16 keys x 8 rows) += K (16 x 16) Q^T (16 x 8): a lane's K fragment is 4 consecutive values of
//     two keys; since the order of the d sum is free, lane t of a quad takes d = t*d/4 .. of its keys,
//     one aligned vector of codes and its own scale bytes each.
//   O^T (16 d x 8 rows) += V^T (16 x 16 keys) P^T (16 x 8): P^T is S^T's fragment transposed by
//     movmatrix; the V fragment needs pairs of KEYS at one d.  Codes of two keys are interleaved nibble
//     by nibble (two logic operations for 8 values each) before the conversion, so the conversion itself
//     delivers (key, key') pairs.  Row g of m-tile j is d = g*d/8 + 2j (g + 8: the next): the lane's codes
//     are one vector, all of one scale.
// The running maximum needs no reduction per block: a vote finds whether any score exceeds the row's
// reference by 2^8; only then (rarely after the first blocks) is it recomputed and O rescaled.
// Measured (calls one after the other on the same inputs; on inputs that change from call to call the tokens take
// 114): 64 tokens over contexts of 300 to 32768 (8 KV heads of 4, 451 MB of cache) 106 us, 66 % of the copy rate
// with launch and ragged ends; four over 500000 tokens 452 us for 2.3 GB, 79 % of it.  There latency bounds it: 55 %
// of the issue slots are taken, and a warp's next instruction waits for its last one's result, with 16 warps per
// SM at 126 registers.  Tiles of 32 rows, 255 registers and 8 warps per SM, take 197 us for 64 chains of 8 nodes
// (401 MB); of 16 rows 131 us.  The tile kernel takes 235 us for either, so 32 is the border.
// Spills: 90 bytes stored and 154 loaded in tiles of 16 rows of d 128 (168 registers for 3 blocks per SM), 18 / 30 in tiles
// of 32 of d 128, none elsewhere.
#include "mars_attention.cuh"
#include "mars_hooks.cuh"

#include <cuda_runtime.h>

#include "mars_kv.h"

namespace mars {

constexpr int kRowsWarps = 4;
constexpr int kRowsThreads = 32 * kRowsWarps;
constexpr int kRowsStages = 4;        // 16-key blocks in flight per warp
constexpr int kRowsMax = 32;          // largest tile
// Blocks per SM: as many as registers allow.  Measured, us with this many / one more: 64 tokens 106 / 147, 64 chains
// of 4 nodes (16 rows) 131 / 213, of 6 nodes (24 rows) 158 / 176, of 8 nodes (32 rows) 197 / 611; d 64: 73 / 74,
// 81 / 83, 103 / 110, 127 / 131.  Tiles of 24 rows are there since chains of 6 nodes take 158 in them, 193 in tiles of 32.
constexpr int rows_occ(int rows, int d)
{
    return d == 128 ? (rows == 8 ? 4 : rows == 16 ? 3 : 2) : (rows == 8 ? 4 : rows == 16 ? 3 : rows == 24 ? 3 : 2);
}
constexpr int rows_grid(int rows, int d) { return kAttnSms * rows_occ(rows, d); }
constexpr int kUnit = RowsShape<8>::unit_keys(8);
constexpr float kNone = -3.40282347e38f;     // reference maximum before a row's first key

__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}

// x = (s - ref) * rs + 7, two at a time (both halves rounded as by themselves)
__device__ __forceinline__ void score2(float &x0, float &x1, float s0, float s1, float r0, float r1, float m0, float m1)
{
    asm("{\n\t.reg .b64 s, r, m, c, o;\n\tmov.b64 s, {%2, %3};\n\tmov.b64 r, {%4, %5};\n\tmov.b64 m, {%6, %7};\n\t"
        "mov.b64 c, {0f40E00000, 0f40E00000};\n\tmov.b64 o, {0fBF800000, 0fBF800000};\n\t"
        "fma.rn.f32x2 s, r, o, s;\n\tfma.rn.f32x2 s, s, m, c;\n\tmov.b64 {%0, %1}, s;\n\t}"
        : "=f"(x0), "=f"(x1) : "f"(s0), "f"(s1), "f"(r0), "f"(r1), "f"(m0), "f"(m1));
}

template <int D>
__host__ __device__ constexpr int rows_slot_floats(int rows) { return rows * (D + 2); }

__host__ __device__ constexpr bool rows_q_shared(int rows) { return rows >= 24; }

template <int D>
constexpr size_t rows_smem_bytes(int rows)
{
    const size_t ring = (size_t)kRowsWarps * kRowsStages * kv_block_bytes(D), sums = (size_t)kRowsWarps * rows * (D + 4) * 4;
    return (rows_q_shared(rows) ? (size_t)rows * D * 2 : 0) + (ring > sums ? ring : sums);
}

template <int D, int DT, int kRows>
__global__ void __launch_bounds__(kRowsThreads, rows_occ(kRows, D)) attn_rows_kernel(const AttnParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    using Shape = RowsShape<kRows>;
    constexpr int kNT = kRows / 8;            // n-tiles of query rows
    constexpr bool kQShared = rows_q_shared(kRows);   // Q fragments in shared memory (48, 64 registers less)
    extern __shared__ __align__(16) unsigned char s_dyn[];
    __shared__ int s_par[MARS_MAX_NODES];
    __shared__ uint32_t s_mask[kRows * (MARS_MAX_NODES / 32)];
    __shared__ unsigned char s_live[kRows];
    __shared__ float s_m[kRowsWarps][kRows], s_l[kRowsWarps][kRows], s_rs[kRows];
    __shared__ int s_last;
    __shared__ AttnSeqs s_seqs;
    constexpr int kBlk = kv_block_bytes(D);
    constexpr int kChunks = kBlk / 16;
    constexpr int kCode = D / 4;              // elements of d per lane of a quad
    constexpr int kSteps = D / 16;            // k-steps of S = m-tiles of O

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;
    uint2 *s_q = reinterpret_cast<uint2 *>(s_dyn);                        // [k-step][n-tile][lane]
    unsigned char *s_ring = s_dyn + (kQShared ? kRows * D * 2 : 0);
    unsigned char *ring = s_ring + warp * kRowsStages * kBlk;
    const uint32_t ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);

    AttnRange r = attn_split<Shape, kRowsThreads>(p, &s_seqs);
    for (int64_t u = r.begin; u < r.end;) {
        const AttnSegment sg = attn_segment<Shape>(p, &s_seqs, r, u);
        if (sg.unit0 >= sg.unit1) { u += sg.span; continue; }
        const bool whole = sg.unit0 == 0 && sg.unit1 == sg.units;
        const int rows = min(kRows, sg.n * p.group - sg.tile * kRows);
        const int row0 = sg.tile * kRows;                // first row of the tile: node row0/group
        const int node0 = attn_node(p, row0);

        // ---- this warp's 16-key blocks of the segment
        const int first = sg.unit0 * (kUnit / 16) + warp;
        const int last = min((sg.keys + 15) >> 4, sg.unit1 * (kUnit / 16));      // exclusive
        const int mine = first < last ? (last - first + kRowsWarps - 1) / kRowsWarps : 0;
        uint64_t from = 0;                               // lane i: address of block from_at + i, 0: no such page
        int from_at = 0;
        auto locate = [&](int i0) {
            from_at = i0;
            const int i = i0 + lane, pos = (first + i * kRowsWarps) * 16;
            const int id = i < mine ? kv_page_id(p.kv, sg.b, pos) : -1;
            from = id >= 0 ? (uint64_t)kv_block<D>(p.kv, p.layer, id, sg.head, pos) : 0;
        };
        locate(0);
        bool poisoned = false;
        auto issue = [&](int i) {                        // 16-key block i of this warp into its ring slot
            if (i < mine) {
                if (i >= from_at + 32) locate(i);
                const uint64_t at = __shfl_sync(0xffffffffu, from, i - from_at);
                if (at) {
                    const unsigned char *src = (const unsigned char *)at + lane * 16;
                    const uint32_t dst = ring_u32 + (i % kRowsStages) * kBlk + lane * 16;
#pragma unroll
                    for (int c = 0; c < (kChunks + 31) / 32; ++c)
                        if (c * 32 + lane < kChunks) cp_async16(dst + c * 512, src + c * 512);
                } else {
                    poisoned = true;                     // no such page: the rows become NaN
                }
            }
            cp_async_commit();
        };
#pragma unroll
        for (int i = 0; i < kRowsStages - 1; ++i) issue(i);

        const int nodes = attn_node(p, row0 + rows - 1) - node0 + 1;
        const int words = (sg.n + 31) >> 5;
        const int st = p.parent ? attn_tree_masks(p, sg.b, sg.n, node0, nodes, s_par, s_mask, words, s_live, &s_last, tid,
                                                  kRowsThreads, [] { __syncthreads(); })
                                : MARS_SEQ_OK;
        if (tid == 0 && p.status && sg.head == 0 && sg.tile == 0 && sg.unit0 == 0) p.status[sg.b] = st;

        // ---- Q^T fragments: row 8n + g, d = t*kCode + 4*s .. of k-step s
        uint2 q[kQShared ? 1 : kSteps][kQShared ? 1 : kNT];
        float rs[kNT][2];                                // score scale of rows 8n + 2t, + 1 in log2 units
        int node[kNT][2];                                // tile-local node of those rows, -1 behind the rows
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
            const int row = row0 + 8 * n + g;
            const bool in = 8 * n + g < rows;
            const int nd = attn_node(p, row);
            uint4 w[kCode / 8];
            float m = 0.0f;
            if (in) {
                const int64_t at = ((int64_t)sg.b * p.N + nd) * p.q_row + (int64_t)(sg.head * p.group + row - nd * p.group) * p.q_head + t * kCode;
#pragma unroll
                for (int i = 0; i < kCode / 8; ++i) {
                    w[i] = reinterpret_cast<const uint4 *>(p.q + at * 2)[i];
                    const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 f = widen2<DT>(x[j]);
                        m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < kCode / 8; ++i) w[i] = make_uint4(0u, 0u, 0u, 0u);
            }
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            float down, up;
            row_scale(m, &down, &up);
            const float scale = row_log2(p, sg.head, up);
            if (warp == 0 && t == 0) s_rs[8 * n + g] = scale;
            const int local = in ? nd - node0 : -1;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                rs[n][e] = __shfl_sync(0xffffffffu, scale, 4 * (2 * t + e));
                node[n][e] = __shfl_sync(0xffffffffu, local, 4 * (2 * t + e));
            }
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {           // words 2s, 2s + 1 of this lane's values
                const uint4 v = w[s >> 1];
                const float2 a = widen2<DT>(s & 1 ? v.z : v.x), b = widen2<DT>(s & 1 ? v.w : v.y);
                const uint2 f = make_uint2(f16x2_from(a.x * down, a.y * down), f16x2_from(b.x * down, b.y * down));
                if constexpr (kQShared) {
                    if (warp == 0) s_q[(s * kNT + n) * 32 + lane] = f;
                } else {
                    q[s][n] = f;
                }
            }
        }
        if constexpr (kQShared) __syncthreads();

        float o[kSteps][kNT][4];
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[j][n][k] = 0.0f;
        // reference maximum; kNone needs no case of its own: scores exceed it by so much that they replace it,
        // unless all of them come to nothing in log2 units (then any reference is as good)
        float ref[kNT][2], l[kNT][2];
#pragma unroll
        for (int n = 0; n < kNT; ++n) { ref[n][0] = ref[n][1] = kNone; l[n][0] = l[n][1] = 0.0f; }
        // rows and columns of the 16-key tile are permuted inside pairs so that neither the K rows nor the
        // V rows that a quarter warp reads together fall on the same banks
        const int key = (g & 6) + ((g ^ (g >> 1)) & 1);
        const int k0 = 2 * t + (t & 1), k1 = 2 * t + ((t & 1) ^ 1);

        for (int i = 0; i < mine; ++i) {
            cp_async_wait<kRowsStages - 2>();
            __syncwarp();
            const unsigned char *blk = ring + (i % kRowsStages) * kBlk;
            const int pos0 = (first + i * kRowsWarps) * 16;
            // ---- S^T = K Q^T for 16 keys
            float s[kNT][4];
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int k = 0; k < 4; ++k) s[n][k] = 0.0f;
            uint32_t code[2][kCode / 8], scale[2][2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t sc2;
                if constexpr (D == 128) {
                    const uint4 c = *reinterpret_cast<const uint4 *>(blk + (8 * w + key) * 64 + t * 16);
                    code[w][0] = c.x; code[w][1] = c.y; code[w][2] = c.z; code[w][3] = c.w;
                    sc2 = *reinterpret_cast<const unsigned short *>(blk + 16 * D + (8 * w + key) * 8 + t * 2);
                } else {
                    const uint2 c = *reinterpret_cast<const uint2 *>(blk + (8 * w + key) * 32 + t * 8);
                    code[w][0] = c.x; code[w][1] = c.y;
                    sc2 = blk[16 * D + (8 * w + key) * 4 + t];
                }
                const uint32_t sh = e4m3x2_to_f16x2(sc2);
                scale[w][0] = __byte_perm(sh, sh, 0x1010);
                scale[w][1] = __byte_perm(sh, sh, 0x3232);
            }
#pragma unroll
            for (int v = 0; v < kCode / 8; ++v) {
                uint32_t h[2][4];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    e2m1x8_to_f16x2(code[w][v], h[w]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) h[w][k] = hmul2(h[w][k], scale[w][v >> 1]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t a[4] = {h[0][2 * e], h[1][2 * e], h[0][2 * e + 1], h[1][2 * e + 1]};
#pragma unroll
                    for (int n = 0; n < kNT; ++n) {
                        uint2 b;
                        if constexpr (kQShared) b = s_q[((2 * v + e) * kNT + n) * 32 + lane];
                        else b = q[2 * v + e][n];
                        mma_f16(s[n], a, b.x, b.y);
                    }
                }
            }
            // ---- V's codes and scales early: their latency hides behind the scores
            uint32_t vs[2], vc[4][kSteps / 4];
            const bool edge = pos0 + 16 > sg.len;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const unsigned char *sp = blk + 17 * D;
                uint32_t a = D == 128 ? sp[(8 * w + k0) * 8 + g] : sp[(8 * w + k0) * 4 + (g >> 1)];
                uint32_t c = D == 128 ? sp[(8 * w + k1) * 8 + g] : sp[(8 * w + k1) * 4 + (g >> 1)];
                if (edge) {      // slots of absent nodes and behind the last key may hold anything, NaN scales too
                    if ((a & 0x7fu) == 0x7fu) a = 0u;
                    if ((c & 0x7fu) == 0x7fu) c = 0u;
                }
                vs[w] = e4m3x2_to_f16x2(__byte_perm(a, c, 0x0040));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const unsigned char *cp = blk + 8 * D + (8 * w + (e ? k1 : k0)) * (D / 2) + g * (D / 16);
                    if constexpr (D == 128) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(cp);
                        vc[2 * w + e][0] = x.x; vc[2 * w + e][1] = x.y;
                    } else {
                        vc[2 * w + e][0] = *reinterpret_cast<const uint32_t *>(cp);
                    }
                }
            }
            // ---- behind the committed tokens only ancestors count (element k: key g or g + 8, row 2t + (k & 1))
            if (edge) {
#pragma unroll
                for (int n = 0; n < kNT; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int pos = pos0 + 8 * (k >> 1) + key, m = pos - sg.len, nd = node[n][k & 1];
                        bool see = m < 0;
                        if (m >= 0 && pos < sg.keys && nd >= 0)
                            see = p.parent ? (s_mask[nd * words + (m >> 5)] >> (m & 31)) & 1u : m <= node0 + nd;
                        if (!see) s[n][k] = -INFINITY;
                    }
            }
            // ---- P = 2^(s - maximum + 7), the maximum as it was; it moves only when a score exceeds it by
            // more than 2^8.  So P <= 2^15, and with the row's largest at 2^7 or more fp16 keeps 11 bits of
            // every probability above 2^-21 of it and an error of 2^-32 of it below
            float x[kNT][4], top = -INFINITY;
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int k = 0; k < 4; k += 2) {
                    score2(x[n][k], x[n][k + 1], s[n][k], s[n][k + 1], ref[n][0], ref[n][1], rs[n][0], rs[n][1]);
                    top = fmaxf(top, fmaxf(x[n][k], x[n][k + 1]));
                }
            if (__any_sync(0xffffffffu, top > 15.0f)) {
#pragma unroll
                for (int n = 0; n < kNT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(s[n][e], s[n][2 + e]);
#pragma unroll
                        for (int k = 4; k < 32; k <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, k));
                        if ((mx - ref[n][e]) * rs[n][e] > 8.0f) {
                            const float f = ex2((ref[n][e] - mx) * rs[n][e]);
                            ref[n][e] = mx;
                            l[n][e] *= f;
#pragma unroll
                            for (int j = 0; j < kSteps; ++j) { o[j][n][e] *= f; o[j][n][2 + e] *= f; }
                            x[n][e] = fmaf(s[n][e] - mx, rs[n][e], 7.0f);
                            x[n][2 + e] = fmaf(s[n][2 + e] - mx, rs[n][e], 7.0f);
                        }
                    }
            }
            uint32_t pb[kNT][2];
#pragma unroll
            for (int n = 0; n < kNT; ++n) {
#pragma unroll
                for (int k = 0; k < 4; ++k) x[n][k] = ex2(x[n][k]);
                l[n][0] += x[n][0] + x[n][2];
                l[n][1] += x[n][1] + x[n][3];
                pb[n][0] = transpose8x8(f16x2_from(x[n][0], x[n][1]));
                pb[n][1] = transpose8x8(f16x2_from(x[n][2], x[n][3]));
            }
            // ---- O^T += V^T P^T: this lane's keys are k0, k1 (first eight) and k0 + 8, k1 + 8
#pragma unroll
            for (int v = 0; v < kSteps / 4; ++v) {
                uint32_t even[2][4], odd[2][4];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t a = vc[2 * w][v], c = vc[2 * w + 1][v];
                    e2m1x8_to_f16x2((a & 0x0f0f0f0fu) | ((c << 4) & 0xf0f0f0f0u), even[w]);
                    e2m1x8_to_f16x2(((a >> 4) & 0x0f0f0f0fu) | (c & 0xf0f0f0f0u), odd[w]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t a[4] = {hmul2(even[0][j], vs[0]), hmul2(odd[0][j], vs[0]), hmul2(even[1][j], vs[1]),
                                           hmul2(odd[1][j], vs[1])};
#pragma unroll
                    for (int n = 0; n < kNT; ++n) mma_f16(o[4 * v + j][n], a, pb[n][0], pb[n][1]);
                }
            }
            __syncwarp();
            issue(i + kRowsStages - 1);
        }
        cp_async_wait<0>();
        if (__any_sync(0xffffffffu, poisoned)) {
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) l[n][e] = NAN;
        }

        // ---- the four warps' sums, then the block's result
        __syncthreads();                                  // ring free
        float *s_o = reinterpret_cast<float *>(s_ring);   // [warp][row][D + 4]
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = l[n][e];
#pragma unroll
                for (int k = 4; k < 32; k <<= 1) x += __shfl_xor_sync(0xffffffffu, x, k);
                const int row = 8 * n + 2 * t + e;
                if (g == 0) { s_m[warp][row] = ref[n][e]; s_l[warp][row] = x; }
                float *to = s_o + (warp * kRows + row) * (D + 4) + g * (D / 8);
#pragma unroll
                for (int j = 0; j < kSteps; j += 2)
                    *reinterpret_cast<float4 *>(to + 2 * j) = make_float4(o[j][n][e], o[j][n][2 + e], o[j + 1][n][e], o[j + 1][n][2 + e]);
            }
        __syncthreads();
        // each thread: kPer values of d of a row, kPass rows of the tile one after the other
        constexpr int kPer = 8, kAcross = D / kPer, kAtOnce = kRowsThreads / kAcross;
        bool write = whole;
        const int c0 = sg.c0, c1 = sg.c1;
        auto slot_of = [&](int c) { return p.partial + (int64_t)(2 * c + (r.per * c >= sg.item ? 0 : 1)) * rows_slot_floats<D>(kRows); };
        const int od = (tid % kAcross) * kPer;
        auto emit = [&](int orow, float (&acc)[kPer], float sum) {
            if (orow >= rows) return;
            const int row = row0 + orow, nd = attn_node(p, row);
            if (p.parent && !s_live[nd - node0]) return;
            const float f = p.scales[p.kv.kv_heads + sg.head] / sum;
#pragma unroll
            for (int k = 0; k < kPer; ++k) acc[k] *= f;
            const int64_t at = ((int64_t)sg.b * p.N + nd) * p.out_row + (int64_t)(sg.head * p.group + row - nd * p.group) * p.out_head + od;
            store_out8<DT>(p.out, at, acc);
        };
        for (int orow = tid / kAcross; orow < rows; orow += kAtOnce) {
            const float m = fmaxf(fmaxf(s_m[0][orow], s_m[1][orow]), fmaxf(s_m[2][orow], s_m[3][orow]));
            float acc[kPer], sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kPer; ++k) acc[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < kRowsWarps; ++w) {
                const float f = ex2((s_m[w][orow] - m) * s_rs[orow]);
                sum += s_l[w][orow] * f;
#pragma unroll
                for (int k = 0; k < kPer; ++k) acc[k] += s_o[(w * kRows + orow) * (D + 4) + od + k] * f;
            }
            if (whole) {
                emit(orow, acc, sum);
            } else {
                // partial result: slot 0 of the block for the item its range begins with, 1 for the other
                float *dst = p.partial + (int64_t)(2 * blockIdx.x + (u == r.begin ? 0 : 1)) * rows_slot_floats<D>(kRows);
#pragma unroll
                for (int k = 0; k < kPer; k += 4)
                    *reinterpret_cast<float4 *>(dst + orow * D + od + k) = make_float4(acc[k], acc[k + 1], acc[k + 2], acc[k + 3]);
                if (od == 0) { dst[kRows * D + orow] = m; dst[kRows * D + kRows + orow] = sum; }
            }
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            if (tid == 0) s_last = atomicAdd(p.counters + c0, 1u) == (unsigned)(c1 - c0);
            __syncthreads();
            write = s_last != 0;
            if (write) {
                __threadfence();
                for (int orow = tid / kAcross; orow < rows; orow += kAtOnce) {
                    float m = kNone, sum = 0.0f, acc[kPer];
#pragma unroll
                    for (int k = 0; k < kPer; ++k) acc[k] = 0.0f;
#pragma unroll 4
                    for (int c = c0; c <= c1; ++c) {
                        const float *src = slot_of(c);
                        const float pm = __ldcg(src + kRows * D + orow), pl = __ldcg(src + kRows * D + kRows + orow);
                        const float4 x = __ldcg(reinterpret_cast<const float4 *>(src + orow * D + od));
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(src + orow * D + od + 4));
                        const float mm = fmaxf(m, pm);
                        const float a = ex2((m - mm) * s_rs[orow]), b = ex2((pm - mm) * s_rs[orow]);
                        m = mm;
                        sum = sum * a + pl * b;
                        acc[0] = acc[0] * a + x.x * b; acc[1] = acc[1] * a + x.y * b; acc[2] = acc[2] * a + x.z * b; acc[3] = acc[3] * a + x.w * b;
                        acc[4] = acc[4] * a + y.x * b; acc[5] = acc[5] * a + y.y * b; acc[6] = acc[6] * a + y.z * b; acc[7] = acc[7] * a + y.w * b;
                    }
                    emit(orow, acc, sum);
                }
                if (tid == 0) p.counters[c0] = 0u;
            }
        }
        __syncthreads();                                  // masks, ring and sums free for the next segment
        u += sg.span;
    }
}

template <int D, int DT, int kRows>
static mars_status_t rows_launch(const AttnParams &p, cudaStream_t st)
{
    cudaError_t e = cudaSuccess;
    if (rows_smem_bytes<D>(kRows) > 40 * 1024)
        e = cudaFuncSetAttribute(attn_rows_kernel<D, DT, kRows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)rows_smem_bytes<D>(kRows));
    if (e == cudaSuccess)
        e = launch_pdl(hook(kHookNoOverlap) == 0, attn_rows_kernel<D, DT, kRows>, dim3(rows_grid(kRows, D)), dim3(kRowsThreads),
                       rows_smem_bytes<D>(kRows), st, p);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return MARS_ERR_CUDA; }
    return MARS_OK;
}

template <int D, int DT>
static mars_status_t rows_launch(const AttnParams &p, int rows, cudaStream_t st)
{
    return rows == 8    ? rows_launch<D, DT, 8>(p, st)
           : rows == 16 ? rows_launch<D, DT, 16>(p, st)
           : rows == 24 ? rows_launch<D, DT, 24>(p, st)
                        : rows_launch<D, DT, 32>(p, st);
}

static_assert(rows_grid(8, 64) * sizeof(unsigned) <= kAttnCounterBytes && rows_grid(8, 128) * sizeof(unsigned) <= kAttnCounterBytes, "one counter per block");

static bool attn_sizes_ok(int B, int N, int q_heads, int kv_heads, int d)
{
    return B >= 1 && B <= MARS_KV_MAX_SEQS && N >= 1 && kv_heads >= 1 && kv_heads <= 1024 && q_heads >= 1 && q_heads <= 65536 &&
           q_heads % kv_heads == 0 && (d == 64 || d == 128) && (int64_t)N * (q_heads / kv_heads) <= (1 << 30);
}

// The kernel for tiles of query rows takes over where a KV head has more of them than the largest
// tile of the other holds.  Measured, us with rows / tiles: 64 chains of 8 nodes (32 rows) 197 / 236, of 4 nodes (16
// rows) 131 / 234; one chain of 8 41 / 39, 4 chains 45 / 47, 16 chains 78 / 91.
// Trees of more nodes than the tile kernel's mask store holds stay with the rows, which unpack K and V again for
// every 32 of them.  That costs (4 heads to a KV head, 8 KV heads of 128, 4000 tokens; 128 / 129 / 256 / 1024 nodes): one
// tree 43 / 68 / 102 / 437 us, 16 trees 203 / 639 / 1227 / 6378, where chains of as many nodes, in tiles, take 43 / 43 /
// 53 / 127 and 199 / 240 / 360 / 1444.
static bool attn_use_tiles(int N, int group, bool tree) { return (int64_t)N * group > kRowsMax && !(tree && N > kTileMaxTree); }
static int attn_rows(int N, int group)
{
    const int64_t rows = (int64_t)N * group;
    return rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 24 ? 24 : 32;
}

static size_t attn_workspace(int N, int group, int d)
{
    size_t rows = 0;                     // what smaller calls need counts too, so that it never falls with N
    for (int n = 8; n <= attn_rows(N, group); n += 8) {
        const size_t need = sizeof(float) * 2 * rows_grid(n, d) * (size_t)(d == 128 ? rows_slot_floats<128>(n) : rows_slot_floats<64>(n));
        rows = rows > need ? rows : need;
    }
    const size_t tile = attn_use_tiles(N, group, false) ? attn_tile_partial_bytes(d) : 0;
    return kAttnCounterBytes + (rows > tile ? rows : tile);
}

}  // namespace mars

using namespace mars;

extern "C" {

size_t mars_tree_attention_workspace_bytes(int B, int N, int q_heads, int kv_heads, int head_dim)
{
    return attn_sizes_ok(B, N, q_heads, kv_heads, head_dim) ? attn_workspace(N, q_heads / kv_heads, head_dim) : 0;
}

mars_status_t mars_tree_attention(const mars_kv_cache_t *cache, int layer, const void *q, int64_t q_row, int64_t q_head,
                                  int dt, int q_heads, int B, int N, const int32_t *parent, const int32_t *count, float scale,
                                  uint32_t flags, void *out, int64_t out_row, int64_t out_head, int32_t *seq_status,
                                  void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    const mars_status_t cs = kv_check(cache);
    if (cs != MARS_OK) return cs;
    if (!q || !out || B < 1 || N < 1 || B > cache->seqs || layer < 0 || layer >= cache->layers || q_heads < 1 ||
        q_heads % cache->kv_heads)
        return MARS_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || scale > 1e30f) return MARS_ERR_INVALID_ARG;      // NaN and infinity too
    if ((dt != MARS_BF16 && dt != MARS_FP16) || !attn_sizes_ok(B, N, q_heads, cache->kv_heads, cache->head_dim) ||
        (parent && N > MARS_MAX_NODES) || (flags & ~(MARS_SHARED_PARENT | MARS_COUNTERS_ZERO)))
        return MARS_ERR_UNSUPPORTED;
    if (((uintptr_t)q & 15) || ((uintptr_t)out & 15) || (q_row & 7) || (q_head & 7) || (out_row & 7) || (out_head & 7) ||
        ((int64_t)B * N > 1 && out_row == 0) || (q_heads > 1 && out_head == 0))
        return MARS_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < attn_workspace(N, q_heads / cache->kv_heads, cache->head_dim)) return MARS_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (!(flags & MARS_COUNTERS_ZERO) && cudaMemsetAsync(workspace, 0, kAttnCounterBytes, st) != cudaSuccess) {
        (void)cudaGetLastError();
        return MARS_ERR_CUDA;
    }
    AttnParams p;
    p.kv = kv_view(cache);
    p.layer = p.kv.pages + layer * p.kv.layer_bytes;
    p.scales = cache->scales + (int64_t)layer * 2 * cache->kv_heads;
    p.q = (const unsigned char *)q; p.out = (unsigned char *)out;
    p.q_row = q_row; p.q_head = q_head; p.out_row = out_row; p.out_head = out_head;
    p.parent = parent; p.count = count; p.status = seq_status;
    p.shared_parent = (flags & MARS_SHARED_PARENT) != 0;
    p.B = B; p.N = N; p.group = q_heads / cache->kv_heads; p.tile_rows = 0;
    p.group_inv = p.group > 1 ? ~0ull / (unsigned)p.group + 1 : 0;
    p.scale_log2 = scale * 1.4426950408889634f;
    const int give_up = hook(kHookAttentionGiveUp);
    p.give_up = give_up ? (unsigned)give_up - 1u : ~0u;
    p.counters = (unsigned *)workspace;
    p.partial = (float *)((unsigned char *)workspace + kAttnCounterBytes);
    if (attn_use_tiles(N, p.group, parent != nullptr)) return attn_tile_launch(p, cache->head_dim, dt, st);
    const int rows = attn_rows(N, p.group);
    if (cache->head_dim == 128)
        return dt == MARS_BF16 ? rows_launch<128, MARS_BF16>(p, rows, st) : rows_launch<128, MARS_FP16>(p, rows, st);
    return dt == MARS_BF16 ? rows_launch<64, MARS_BF16>(p, rows, st) : rows_launch<64, MARS_FP16>(p, rows, st);
}

}  // extern "C"
