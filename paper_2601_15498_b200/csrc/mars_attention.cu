// libmars: attention of draft nodes over the paged 4-bit cache.
//
// O = softmax(scale * q K^T) V with K, V = code * scale of E2M1 / E4M3 blocks.  A code has 2
// significant bits and a block scale 4, so code * scale is exact in fp16 (6 bits, 2^-10 .. 2688) and
// both products run on the tensor cores in fp16 with fp32 accumulation.  q is brought to fp16 after
// a power-of-two scaling of its row (largest element in [1, 2)): bf16 and fp16 values keep all their
// bits down to 2^-14 of the row's largest and an error below 2^-25 of it beyond.  The heads' fp32
// scales are factored out of both sums.
//
// Kernel for few query rows per KV head (`attn_rows_kernel`, tiles of 16 rows): bound by reading the
// cache.  The page bytes go through a small shared-memory ring straight into the register fragments of
// mma.sync -- no unpacked copy of K or V exists anywhere:
//   S (16 rows x 8 keys) += Q (16 x 16) K^T (16 x 8): a lane's B fragment is 4 consecutive values of
//     one key; since the order of the d sum is free, lane t of a quad takes d = t*d/4 .. of its key,
//     one aligned vector of codes and its own scale bytes.
//   O (16 x 8) += P (16 x 16) V (16 x 8): the fragment needs pairs of KEYS at one d.  Codes of two
//     keys are interleaved nibble by nibble (two logic operations for 8 values each) before the
//     conversion, so the conversion itself delivers (key, key') pairs.  Output column g of n-tile j is
//     d = g*d/8 + j: the lane's codes are one vector, all of one scale.
#include "mars_attention.cuh"
#include "mars_hooks.cuh"

#include <cuda_runtime.h>

#include "mars_kv.h"

namespace mars {

constexpr int kRowsM = RowsShape::M;  // query rows per tile
constexpr int kUnit = RowsShape::unit_keys(kRowsM);
constexpr int kRowsWarps = 4;
constexpr int kRowsThreads = 32 * kRowsWarps;
constexpr int kRowsStages = 4;        // 16-key blocks in flight per warp
constexpr int kRowsOcc = 3;           // blocks per SM
constexpr int kRowsGrid = kAttnSms * kRowsOcc;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D>
__host__ __device__ constexpr int rows_slot_floats() { return kRowsM * (D + 2); }

template <int D>
constexpr size_t rows_smem_bytes()
{
    return (size_t)kRowsWarps * kRowsStages * kv_block_bytes(D) > (size_t)kRowsWarps * kRowsM * (D + 4) * 4
               ? (size_t)kRowsWarps * kRowsStages * kv_block_bytes(D)
               : (size_t)kRowsWarps * kRowsM * (D + 4) * 4;
}

template <int D, int DT>
__global__ void __launch_bounds__(kRowsThreads, kRowsOcc) attn_rows_kernel(const AttnParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(16) unsigned char s_ring[];
    __shared__ int s_par[MARS_MAX_NODES];
    __shared__ uint32_t s_mask[kRowsM * (MARS_MAX_NODES / 32)];
    __shared__ unsigned char s_live[kRowsM];
    __shared__ float s_m[kRowsWarps][kRowsM], s_l[kRowsWarps][kRowsM];
    __shared__ int s_last;
    __shared__ AttnSeqs s_seqs;
    constexpr int kBlk = kv_block_bytes(D);
    constexpr int kChunks = kBlk / 16;
    constexpr int kCode = D / 4;              // elements of d per lane of a quad
    constexpr int kTiles = D / 8;             // n-tiles of the output

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;
    unsigned char *ring = s_ring + warp * kRowsStages * kBlk;
    const uint32_t ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);

    AttnRange r = attn_split<RowsShape, kRowsThreads>(p, &s_seqs);
    for (int64_t u = r.begin; u < r.end;) {
        const AttnSegment sg = attn_segment<RowsShape>(p, &s_seqs, r, u);
        const bool whole = sg.unit0 == 0 && sg.unit1 == sg.units;
        const int rows = min(kRowsM, sg.n * p.group - sg.tile * kRowsM);
        const int row0 = sg.tile * kRowsM;               // first row of the tile: node row0/group
        const int node0 = attn_node(p, row0);
        const int nodes = attn_node(p, row0 + rows - 1) - node0 + 1;
        const int words = (sg.n + 31) >> 5;
        const int st = p.parent ? attn_tree_masks(p, sg.b, sg.n, node0, nodes, s_par, s_mask, words, s_live, &s_last, tid,
                                                  kRowsThreads, [] { __syncthreads(); })
                                : MARS_SEQ_OK;
        if (tid == 0 && p.status && sg.head == 0 && sg.tile == 0 && sg.unit0 == 0) p.status[sg.b] = st;

        // ---- Q fragments: rows g and g + 8, d = t*kCode + 4*s .. of k-step s
        uint32_t qa[D / 16][4];
        float rs[2];                                     // score scale of the two rows, in log2 units
        int node[2];                                     // tile-local node of the row, -1 behind the rows
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = row0 + g + 8 * half;
            const bool in = g + 8 * half < rows;
            const int nd = attn_node(p, row);
            node[half] = in ? nd - node0 : -1;
            uint4 w[kCode / 8];
            float m = 0.0f;
            if (in) {
                const int64_t at = ((int64_t)sg.b * p.N + nd) * p.q_row +
                                   (int64_t)(sg.head * p.group + row - nd * p.group) * p.q_head + t * kCode;
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
            rs[half] = p.scale_log2 * p.scales[sg.head] * up;
#pragma unroll
            for (int i = 0; i < kCode / 8; ++i) {
                const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = widen2<DT>(x[j]);
                    // word 4*i + j holds d = t*kCode + 8*i + 2*j, +1: k-step 2*i + j/2, register j&1
                    qa[2 * i + (j >> 1)][half + 2 * (j & 1)] = f16x2_from(f.x * down, f.y * down);
                }
            }
        }

        // ---- this warp's 16-key blocks of the segment
        const int first = sg.unit0 * (kUnit / 16) + warp;
        const int last = min((sg.keys + 15) >> 4, sg.unit1 * (kUnit / 16));      // exclusive
        const int mine = first < last ? (last - first + kRowsWarps - 1) / kRowsWarps : 0;
        int ids = -1, ids_at = 0;                        // lane i: page of block ids_at + i
        auto fetch_ids = [&](int i0) {
            ids_at = i0;
            const int i = i0 + lane;
            ids = i < mine ? kv_page_id(p.kv, sg.b, (first + i * kRowsWarps) * 16) : -1;
        };
        fetch_ids(0);
        bool poisoned = false;
        auto issue = [&](int i) {                        // 16-key block i of this warp into its ring slot
            if (i < mine) {
                if (i >= ids_at + 32) fetch_ids(i);
                const int id = __shfl_sync(0xffffffffu, ids, i - ids_at);
                if (id >= 0) {
                    const unsigned char *src = kv_block<D>(p.kv, p.layer, id, sg.head, (first + i * kRowsWarps) * 16);
                    const uint32_t dst = ring_u32 + (i % kRowsStages) * kBlk;
#pragma unroll
                    for (int c = 0; c < (kChunks + 31) / 32; ++c)
                        if (c * 32 + lane < kChunks) cp_async16(dst + (c * 32 + lane) * 16, src + (c * 32 + lane) * 16);
                } else {
                    poisoned = true;                     // no such page: the rows become NaN
                }
            }
            cp_async_commit();
        };
#pragma unroll
        for (int i = 0; i < kRowsStages - 1; ++i) issue(i);

        float o[kTiles][4];
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[j][k] = 0.0f;
        float mref[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

        for (int i = 0; i < mine; ++i) {
            cp_async_wait<kRowsStages - 2>();
            __syncwarp();
            const unsigned char *blk = ring + (i % kRowsStages) * kBlk;
            const int pos0 = (first + i * kRowsWarps) * 16;
            // ---- S = Q K^T for 16 keys: n-tile w, column c is key 8w + 2*(c/2) + ((c&1) ^ (c/2 & 1))
            float s[2][4];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
#pragma unroll
                for (int k = 0; k < 4; ++k) s[w][k] = 0.0f;
                const int key = 8 * w + (g & 6) + ((g ^ (g >> 1)) & 1);
                uint32_t code[kCode / 8], sc2;
                if constexpr (D == 128) {
                    const uint4 c = *reinterpret_cast<const uint4 *>(blk + key * 64 + t * 16);
                    code[0] = c.x; code[1] = c.y; code[2] = c.z; code[3] = c.w;
                    sc2 = *reinterpret_cast<const unsigned short *>(blk + 16 * D + key * 8 + t * 2);
                } else {
                    const uint2 c = *reinterpret_cast<const uint2 *>(blk + key * 32 + t * 8);
                    code[0] = c.x; code[1] = c.y;
                    sc2 = blk[16 * D + key * 4 + t];
                }
                const uint32_t sh = e4m3x2_to_f16x2(sc2);
                const uint32_t scale[2] = {__byte_perm(sh, sh, 0x1010), __byte_perm(sh, sh, 0x3232)};
#pragma unroll
                for (int v = 0; v < kCode / 8; ++v) {
                    uint32_t h[4];
                    e2m1x8_to_f16x2(code[v], h);
                    const uint32_t f = scale[v >> 1];
                    mma_f16(s[w], qa[2 * v], hmul2(h[0], f), hmul2(h[1], f));
                    mma_f16(s[w], qa[2 * v + 1], hmul2(h[2], f), hmul2(h[3], f));
                }
            }
            // ---- scores in log2 units; behind the committed tokens only ancestors count
            const bool edge = pos0 + 16 > sg.len;
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x = s[w][k] * rs[k >> 1];
                    if (edge) {
                        const int m = pos0 + 8 * w + 2 * t + ((k ^ t) & 1) - sg.len;    // draft node of the key
                        bool see = m < 0;
                        if (m >= 0 && pos0 + 8 * w + 2 * t + ((k ^ t) & 1) < sg.keys && node[k >> 1] >= 0)
                            see = p.parent ? (s_mask[node[k >> 1] * words + (m >> 5)] >> (m & 31)) & 1u
                                           : m <= node0 + node[k >> 1];
                        if (!see) x = -INFINITY;
                    }
                    s[w][k] = x;
                }
            // ---- running maximum, moved only when it grows by more than 2^8
            float mx[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                mx[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
                mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
                mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
            }
            if (__any_sync(0xffffffffu, mx[0] > mref[0] + 8.0f || mx[1] > mref[1] + 8.0f)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float to = fmaxf(mref[h], mx[h]);
                    const float f = to == -INFINITY ? 1.0f : ex2(mref[h] - to);
                    mref[h] = to;
                    l[h] *= f;
#pragma unroll
                    for (int j = 0; j < kTiles; ++j) { o[j][2 * h] *= f; o[j][2 * h + 1] *= f; }
                }
            }
            // P = 2^(s - mref + 7) <= 2^15: with the row's largest at 2^7 or more, fp16 keeps 11 bits of
            // every probability above 2^-21 of it and an error of 2^-32 of it below
            const float base[2] = {mref[0] == -INFINITY ? 0.0f : mref[0] - 7.0f,
                                   mref[1] == -INFINITY ? 0.0f : mref[1] - 7.0f};
            uint32_t pa[4];
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float p0 = ex2(s[w][2 * h] - base[h]), p1 = ex2(s[w][2 * h + 1] - base[h]);
                    l[h] += p0 + p1;
                    pa[2 * w + h] = f16x2_from(p0, p1);
                }
            // ---- O += P V: this lane's keys are k0, k1 (n-tile 0) and k0 + 8, k1 + 8 (n-tile 1)
            const int k0 = 2 * t + (t & 1), k1 = 2 * t + ((t & 1) ^ 1);
            uint32_t vs[2], vc[4][kTiles / 8];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const unsigned char *sp = blk + 17 * D;
                uint32_t a = D == 128 ? sp[(8 * w + k0) * 8 + g] : sp[(8 * w + k0) * 4 + (g >> 1)];
                uint32_t c = D == 128 ? sp[(8 * w + k1) * 8 + g] : sp[(8 * w + k1) * 4 + (g >> 1)];
                if (edge) {      // slots behind the last key may hold anything, a NaN scale too
                    if (pos0 + 8 * w + k0 >= sg.len + sg.n) a = 0u;
                    if (pos0 + 8 * w + k1 >= sg.len + sg.n) c = 0u;
                }
                vs[w] = e4m3x2_to_f16x2(a | (c << 8));
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
#pragma unroll
            for (int v = 0; v < kTiles / 8; ++v) {
                uint32_t even[2][4], odd[2][4];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t a = vc[2 * w][v], c = vc[2 * w + 1][v];
                    e2m1x8_to_f16x2((a & 0x0f0f0f0fu) | ((c << 4) & 0xf0f0f0f0u), even[w]);
                    e2m1x8_to_f16x2(((a >> 4) & 0x0f0f0f0fu) | (c & 0xf0f0f0f0u), odd[w]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    mma_f16(o[8 * v + 2 * j], pa, hmul2(even[0][j], vs[0]), hmul2(even[1][j], vs[1]));
                    mma_f16(o[8 * v + 2 * j + 1], pa, hmul2(odd[0][j], vs[0]), hmul2(odd[1][j], vs[1]));
                }
            }
            __syncwarp();
            issue(i + kRowsStages - 1);
        }
        cp_async_wait<0>();
        if (__any_sync(0xffffffffu, poisoned)) { l[0] = l[1] = NAN; if (mref[0] == -INFINITY) mref[0] = 0.0f; if (mref[1] == -INFINITY) mref[1] = 0.0f; }

        // ---- the four warps' sums, then the block's result
        __syncthreads();                                  // ring free
        float *s_o = reinterpret_cast<float *>(s_ring);   // [warp][16][D + 4]
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            if (t == 0) { s_m[warp][g + 8 * h] = mref[h]; s_l[warp][g + 8 * h] = l[h]; }
            float *to = s_o + (warp * kRowsM + g + 8 * h) * (D + 4) + 2 * t * kTiles;
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
                to[j] = o[j][2 * h];
                to[kTiles + j] = o[j][2 * h + 1];
            }
        }
        __syncthreads();
        constexpr int kPer = D / 8;                       // output values per thread: row tid/8
        const int orow = tid >> 3, od = (tid & 7) * kPer;
        float m = fmaxf(fmaxf(s_m[0][orow], s_m[1][orow]), fmaxf(s_m[2][orow], s_m[3][orow]));
        float acc[kPer], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kPer; ++k) acc[k] = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) {
            const float f = s_m[w][orow] == -INFINITY ? 0.0f : ex2(s_m[w][orow] - m);
            sum += s_l[w][orow] * f;
#pragma unroll
            for (int k = 0; k < kPer; ++k) acc[k] += s_o[(w * kRowsM + orow) * (D + 4) + od + k] * f;
        }
        bool write = whole;
        if (!whole) {
            // partial result: slot 0 of the block for the item its range begins with, 1 for the other
            const int slot = 2 * blockIdx.x + (u == r.begin ? 0 : 1);
            float *dst = p.partial + (int64_t)slot * rows_slot_floats<D>();
#pragma unroll
            for (int k = 0; k < kPer; k += 4)
                *reinterpret_cast<float4 *>(dst + orow * D + od + k) = make_float4(acc[k], acc[k + 1], acc[k + 2], acc[k + 3]);
            if ((tid & 7) == 0) { dst[kRowsM * D + orow] = m; dst[kRowsM * D + kRowsM + orow] = sum; }
            const int c0 = (int)(sg.item / r.per), c1 = (int)((sg.item + sg.units - 1) / r.per);
            __threadfence();
            __syncthreads();
            if (tid == 0) s_last = atomicAdd(p.counters + c0, 1u) == (unsigned)(c1 - c0);
            __syncthreads();
            if (s_last) {
                __threadfence();
                m = -INFINITY;
                for (int c = c0; c <= c1; ++c) {
                    const int sl = 2 * c + (r.per * c >= sg.item ? 0 : 1);
                    m = fmaxf(m, __ldcg(p.partial + (int64_t)sl * rows_slot_floats<D>() + kRowsM * D + orow));
                }
                sum = 0.0f;
#pragma unroll
                for (int k = 0; k < kPer; ++k) acc[k] = 0.0f;
                for (int c = c0; c <= c1; ++c) {
                    const int sl = 2 * c + (r.per * c >= sg.item ? 0 : 1);
                    const float *src = p.partial + (int64_t)sl * rows_slot_floats<D>();
                    const float pm = __ldcg(src + kRowsM * D + orow);
                    const float f = pm == -INFINITY ? 0.0f : ex2(pm - m);
                    sum += __ldcg(src + kRowsM * D + kRowsM + orow) * f;
#pragma unroll
                    for (int k = 0; k < kPer; k += 4) {
                        const float4 x = __ldcg(reinterpret_cast<const float4 *>(src + orow * D + od + k));
                        acc[k] += x.x * f; acc[k + 1] += x.y * f; acc[k + 2] += x.z * f; acc[k + 3] += x.w * f;
                    }
                }
                if (tid == 0) p.counters[c0] = 0u;
                write = true;
            }
        }
        if (write && orow < rows) {
            const int row = row0 + orow, nd = attn_node(p, row);
            if (!p.parent || s_live[nd - node0]) {
                const float f = p.scales[p.kv.kv_heads + sg.head] / sum;
#pragma unroll
                for (int k = 0; k < kPer; ++k) acc[k] *= f;
                const int64_t at = ((int64_t)sg.b * p.N + nd) * p.out_row + (int64_t)(sg.head * p.group + row - nd * p.group) * p.out_head + od;
#pragma unroll
                for (int k = 0; k < kPer; k += 8) store_out8<DT>(p.out, at + k, acc + k);
            }
        }
        __syncthreads();                                  // masks, ring and sums free for the next segment
        u += sg.unit1 - sg.unit0;
    }
}

template <int D, int DT>
static mars_status_t rows_launch(const AttnParams &p, cudaStream_t st)
{
    const cudaError_t e = launch_pdl(hook(kHookNoOverlap) == 0, attn_rows_kernel<D, DT>, dim3(kRowsGrid), dim3(kRowsThreads),
                                     rows_smem_bytes<D>(), st, p);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return MARS_ERR_CUDA; }
    return MARS_OK;
}

static_assert(kRowsGrid * sizeof(unsigned) <= kAttnCounterBytes, "one counter per block");

static bool attn_sizes_ok(int B, int N, int q_heads, int kv_heads, int d)
{
    return B >= 1 && B <= MARS_KV_MAX_SEQS && N >= 1 && kv_heads >= 1 && kv_heads <= 1024 && q_heads >= 1 && q_heads <= 65536 &&
           q_heads % kv_heads == 0 && (d == 64 || d == 128) && (int64_t)N * (q_heads / kv_heads) <= (1 << 30);
}

// The kernel for tiles of query rows takes over where a KV head has more of them than two tiles of the
// other hold.
static bool attn_use_tiles(int N, int group, bool tree) { return (int64_t)N * group > 2 * kRowsM && !(tree && N > kTileMaxTree); }

static size_t attn_workspace(int N, int group, int d)
{
    const size_t rows = sizeof(float) * 2 * kRowsGrid * (size_t)(d == 128 ? rows_slot_floats<128>() : rows_slot_floats<64>());
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
    p.B = B; p.N = N; p.group = q_heads / cache->kv_heads;
    p.group_inv = p.group > 1 ? ~0ull / (unsigned)p.group + 1 : 0;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.counters = (unsigned *)workspace;
    p.partial = (float *)((unsigned char *)workspace + kAttnCounterBytes);
    if (attn_use_tiles(N, p.group, parent != nullptr)) return attn_tile_launch(p, cache->head_dim, dt, st);
    if (cache->head_dim == 128)
        return dt == MARS_BF16 ? rows_launch<128, MARS_BF16>(p, st) : rows_launch<128, MARS_FP16>(p, st);
    return dt == MARS_BF16 ? rows_launch<64, MARS_BF16>(p, st) : rows_launch<64, MARS_FP16>(p, st);
}

}  // extern "C"
