// libmars: attention of draft nodes over the paged 4-bit cache, many query rows per KV head.
//
// The products run on tcgen05.mma (kind::f16, 128 x 128 x 16 steps, fp32 accumulators in tensor
// memory); see mars_attention.cu for the arithmetic.  Up to 256 query rows of one KV head -- a whole
// tree of 60 nodes with four heads to a KV head -- share every key that is unpacked.  One block per SM:
//
//   warps 0-3   softmax of accumulator 0 (thread = query row): score scale, mask, running maximum and
//   warps 4-7   sum, P back into tensor memory; the same for accumulator 1
//   warps 8-11  unpack: 16-byte loads of codes two key tiles ahead into registers, code * scale in fp16
//               into two stages of K and of V tiles [128 keys][d] (128-byte swizzle)
//   warp 12     tensor memory, and the MMAs: S = Q K^T (both operands in shared memory), O += P V (P in
//               tensor memory over the columns of S; V's tile read with d as its leading dimension,
//               so that neither K nor V is ever transposed)
//
// Two accumulators keep the tensor cores busy while a softmax runs: with more than 128 rows they hold
// the two halves of the rows and both see every key tile; with fewer they hold the same rows and take
// the key tiles in turn, and their results are merged at the end like those of two blocks.
// The step order of the issuing warp is S(0) S(1) | P V(0) S(2) | P V(1) S(3) | ...: tensor operations
// execute in issue order, so S(u + 2) may overwrite the P that P V(u) has read.
//
// Every wait is bounded.  One that gives up raises the block's abort flag; all roles fall through to
// the common end, the sequence's status becomes MARS_SEQ_TIMEOUT, tensor memory is freed.
#include "mars_attention.cuh"
#include "mars_hooks.cuh"
#include "mars_tcgen05.cuh"

#include <cuda_runtime.h>

#include "mars_kv.h"

namespace mars {

constexpr int kTileThreads = 416;
constexpr int kTileKeys = 128;
constexpr uint32_t kTmemAll = 512;
constexpr uint32_t kColS = 0, kColO = 256;             // accumulator i: S at 128 i, O at 256 + 128 i

template <int D> constexpr uint32_t tile_bytes() { return 128u * D * 2; }    // 128 rows of d fp16
template <int D> constexpr int tile_slot_floats() { return TileShape::M * (D + 2); }

constexpr int kMaskWords = kTileMaxTree / 32;
constexpr uint32_t kTileBarBytes = 256;

// shared memory: Q (2 tiles) | K (2 stages) | V (2 stages) | masks | parents | barriers
template <int D> constexpr size_t tile_smem_bytes()
{
    const size_t need = 1024 + 6 * (size_t)tile_bytes<D>() + 256 * kMaskWords * 4 + kTileMaxTree * 4 + 256 + kTileBarBytes;
    return need > 120 * 1024 ? need : 120 * 1024;      // one block per SM: each takes all of tensor memory
}

// Operand with its MN dimension contiguous (V as [keys][d]): rows of 64 values per 128-byte swizzle row, 8
// keys per 1024 bytes, the next 64 values of d `lead` bytes further on.
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t smem_addr, uint32_t lead)
{
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3ffffu) >> 4);
    d |= (uint64_t)(lead >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

__device__ __forceinline__ void tc_mma_f16_ss(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Instruction descriptors: D fp32, A and B fp16, M = 128; S: N = 128 keys, both operands K-major;
// O: N = d, B with d as its leading dimension.
constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kTileKeys >> 3) << 17) | ((128u >> 4) << 24);
template <int D> constexpr uint32_t idesc_o() { return (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((128u >> 4) << 24); }

// The 32 keys from position p0 on that node `node` may see, as bits.
__device__ __forceinline__ uint32_t visible32(int p0, int len, int node, bool tree, const uint32_t *mask, int words)
{
    const int m0 = p0 - len;
    if (m0 <= -32) return 0xffffffffu;
    if (!tree) {
        const int cnt = node + 1 - m0;                  // first cnt keys
        return cnt >= 32 ? 0xffffffffu : cnt <= 0 ? 0u : (1u << cnt) - 1u;
    }
    if (m0 < 0) {
        const int k = -m0;                              // 1..31 committed tokens, then nodes 0, 1, ...
        return ((1u << k) - 1u) | (words > 0 ? mask[0] << k : 0u);
    }
    const int w = m0 >> 5;
    const uint32_t lo = w < words ? mask[w] : 0u, hi = w + 1 < words ? mask[w + 1] : 0u;
    return __funnelshift_r(lo, hi, m0 & 31);
}

struct TileRegs {
    uint4 c[4];               // codes of (key, part) chunk it
    uint32_t s[4];            // their scales: two E4M3 bytes
};

template <int D, int DT>
__global__ void __launch_bounds__(kTileThreads, 1) attn_tile_kernel(const AttnParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    unsigned char *sm = smem_raw + (base - raw);
    constexpr uint32_t kT = tile_bytes<D>();
    const uint32_t q_at = base, k_at = base + 2 * kT, v_at = base + 4 * kT;
    uint32_t *s_mask = reinterpret_cast<uint32_t *>(sm + 6 * kT);
    int *s_par = reinterpret_cast<int *>(s_mask + 256 * kMaskWords);
    unsigned char *s_live = reinterpret_cast<unsigned char *>(s_par + kTileMaxTree);
    const uint32_t bars = smem_u32(s_live + 256);
    const uint32_t kfull = bars, kempty = bars + 16, vfull = bars + 32, vempty = bars + 48;
    const uint32_t sfull = bars + 64, pfull = bars + 80, odone = bars + 96, drain = bars + 112;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_last;
    __shared__ unsigned s_word;
    __shared__ float s_m[256], s_l[256];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    AttnRange r = attn_split<TileShape, kTileThreads>(p);

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(kfull + 8 * i, 4);
            mbar_init(vfull + 8 * i, 4);
            mbar_init(kempty + 8 * i, 1);
            mbar_init(vempty + 8 * i, 1);
            mbar_init(sfull + 8 * i, 1);
            mbar_init(pfull + 8 * i, 4);
            mbar_init(odone + 8 * i, 1);
        }
        mbar_init(drain, 1);
        s_abort = 0;
        s_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&s_tmem)), "r"(kTmemAll) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    volatile int *abort_flag = &s_abort;

    // pipeline positions; every role keeps those it uses, over all segments
    uint32_t n_kv = 0;                   // key tiles so far (unpack and issue warps)
    uint32_t n_s[2] = {0, 0};            // S tiles of an accumulator so far (softmax uses its own, issue both)
    bool ok = true;

    for (int64_t u = r.begin; u < r.end;) {
        const AttnSegment sg = attn_segment<TileShape>(p, r, u);
        const int rows = attn_tile_rows<TileShape>(p, sg.n, sg.tile);
        const int row0 = sg.tile * TileShape::M;
        const int node0 = row0 / p.group;
        const int nodes = (row0 + rows - 1) / p.group - node0 + 1;
        const int words = p.parent ? (sg.n + 31) >> 5 : 0;
        const bool two = rows > 128;     // accumulators hold different rows (else they take turns on the keys)
        const int uk = TileShape::unit_keys(rows);
        const int key0 = sg.unit0 * uk, key1 = min(sg.keys, sg.unit1 * uk);
        const int tiles = (key1 - key0 + kTileKeys - 1) / kTileKeys;
        const int steps = two ? 2 * tiles : tiles;
        const bool whole = sg.unit0 == 0 && sg.unit1 == sg.units;
        const int st = attn_tree_masks(p, sg.b, sg.n, node0, nodes, s_par, s_mask, words, s_live);
        if (tid == 0 && p.status && sg.head == 0 && sg.tile == 0 && sg.unit0 == 0) p.status[sg.b] = st;

        float rs = 0.0f;                 // softmax threads: score scale of the row in log2 units
        int node = -1;                   // its node, -1 behind the rows
        const int acc = warp >> 2;       // softmax: accumulator 0 / 1
        const int row = (two ? acc * 128 : 0) + (tid & 127);
        if (warp < 8) {
            // ---- Q: this thread's row, scaled to fp16, into its swizzled tile
            const bool in = row < rows;
            if (in) node = (row0 + row) / p.group;
            if (two || acc == 0) {
                const unsigned char *src = p.q + 2 * (((int64_t)sg.b * p.N + (in ? node : 0)) * p.q_row +
                                                      (int64_t)(sg.head * p.group + (in ? (row0 + row) % p.group : 0)) * p.q_head);
                float m = 0.0f;
                if (in) {
#pragma unroll 4
                    for (int c = 0; c < D / 8; ++c) {
                        const uint4 w = reinterpret_cast<const uint4 *>(src)[c];
                        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = widen2<DT>(x[j]);
                            m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
                        }
                    }
                }
                float down, up;
                row_scale(m, &down, &up);
                rs = fmaxf(p.scale_log2 * p.scales[sg.head] * up, 1.17549435e-38f);
                const int rr = tid & 127;
                unsigned char *dst = sm + acc * kT + rr * 128;
#pragma unroll 4
                for (int c = 0; c < D / 8; ++c) {
                    uint32_t h[4] = {0u, 0u, 0u, 0u};
                    if (in) {
                        const uint4 w = reinterpret_cast<const uint4 *>(src)[c];
                        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = widen2<DT>(x[j]);
                            h[j] = f16x2_from(f.x * down, f.y * down);
                        }
                    }
                    *reinterpret_cast<uint4 *>(dst + (c >> 3) * (128 * 128) + (((c & 7) ^ (rr & 7)) * 16)) = make_uint4(h[0], h[1], h[2], h[3]);
                }
                if (!two) s_m[rr] = rs;
            }
            fence_proxy_async();
        }
        __syncthreads();
        if (warp < 8 && !two && acc == 1) rs = s_m[tid & 127];
        __syncthreads();                 // s_m is used again below

        if (warp >= 8 && warp < 12) {
            // ------------------------------------------------------------------ unpack
            const int ut = tid - 256;
            constexpr int kParts = D / 32;                // 16-byte chunks per key
            // chunk `it` of this thread: K (or V) codes of key (it / (kParts/2)) * 64 + ut/2, 32 values from part
            auto key_of = [&](int it) { return (it / (kParts / 2)) * 64 + (ut >> 1); };
            auto part_of = [&](int it) { return (it % (kParts / 2)) * 2 + (ut & 1); };
            constexpr int kIt = 2 * (kParts / 2);         // 4 (d = 128) or 2 (d = 64) chunks for K, the same for V
            const int valid = sg.len + sg.n;              // keys from here on were never written
            auto page_of = [&](int t, int half) {         // page id of this thread's key in half `half` of tile t; -2: no key
                const int pos = key0 + t * kTileKeys + half * 64 + (ut >> 1);
                return t < tiles && pos < valid ? kv_page_id(p.kv, sg.b, pos) : -2;
            };
            auto load = [&](int t, const int (&ids)[2], bool v, TileRegs &g) {
#pragma unroll
                for (int it = 0; it < kIt; ++it) {
                    const int key = key_of(it), part = part_of(it), id = ids[key >> 6];
                    g.c[it] = make_uint4(0u, 0u, 0u, 0u);
                    g.s[it] = id == -1 && v ? 0x7f7fu : 0u;       // no such page: NaN
                    if (id >= 0) {
                        const int pos = key0 + t * kTileKeys + key;
                        const unsigned char *blk = kv_block<D>(p.kv, p.layer, id, sg.head, pos);
                        const int slot = pos & 15;
                        g.c[it] = ld_stream(reinterpret_cast<const uint4 *>(blk + (v ? 8 * D : 0) + slot * (D / 2) + part * 16));
                        g.s[it] = *reinterpret_cast<const unsigned short *>(blk + 16 * D + (v ? D : 0) + slot * (D / 16) + part * 2);
                    }
                }
            };
            auto store = [&](unsigned char *tile, const TileRegs &g) {
#pragma unroll
                for (int it = 0; it < kIt; ++it) {
                    const int key = key_of(it), part = part_of(it);
                    unsigned char *dst = tile + (part >> 1) * (128 * 128) + key * 128;
                    const uint32_t sh = e4m3x2_to_f16x2(g.s[it]);
                    const uint32_t sc[2] = {__byte_perm(sh, sh, 0x1010), __byte_perm(sh, sh, 0x3232)};
                    const uint32_t w[4] = {g.c[it].x, g.c[it].y, g.c[it].z, g.c[it].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t h[4];
                        e2m1x8_to_f16x2(w[k], h);
                        const uint32_t f = sc[k >> 1];
                        *reinterpret_cast<uint4 *>(dst + ((((part & 1) * 4 + k) ^ (key & 7)) * 16)) =
                            make_uint4(hmul2(h[0], f), hmul2(h[1], f), hmul2(h[2], f), hmul2(h[3], f));
                    }
                }
            };
            TileRegs gk[2], gv[2];
            int ids[2][2];
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                ids[a][0] = page_of(a, 0);
                ids[a][1] = page_of(a, 1);
                load(a, ids[a], false, gk[a]);
                load(a, ids[a], true, gv[a]);
            }
            int nid[2] = {page_of(2, 0), page_of(2, 1)};
            for (int t0 = 0; t0 < tiles && ok; t0 += 2) {
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const int t = t0 + a;
                    if (t >= tiles || !ok) break;
                    const uint32_t stage = n_kv & 1u, phase = (n_kv >> 1) & 1u;
                    ok = __all_sync(0xffffffffu, mbar_wait(kempty + 8 * stage, phase ^ 1u, abort_flag, &s_word));
                    if (!ok) break;
                    store(sm + 2 * kT + stage * kT, gk[a]);
                    load(t + 2, nid, false, gk[a]);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(kfull + 8 * stage);
                    ok = __all_sync(0xffffffffu, mbar_wait(vempty + 8 * stage, phase ^ 1u, abort_flag, &s_word));
                    if (!ok) break;
                    store(sm + 4 * kT + stage * kT, gv[a]);
                    load(t + 2, nid, true, gv[a]);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(vfull + 8 * stage);
                    nid[0] = page_of(t + 3, 0);
                    nid[1] = page_of(t + 3, 1);
                    ++n_kv;
                }
            }
        } else if (warp == 12) {
            // ------------------------------------------------------------------ MMA issue
            if (lane == 0) {
                auto issue_s = [&](int s) {
                    const int i = s & 1, t = two ? s >> 1 : s;
                    const uint32_t stage = (n_kv + t) & 1u, phase = ((n_kv + t) >> 1) & 1u;
                    if ((!two || i == 0) && !mbar_wait(kfull + 8 * stage, phase, abort_flag, &s_word)) return false;
                    tc_fence_after();
                    const uint32_t a = q_at + (two ? i * kT : 0), b = k_at + stage * kT;
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = (k >> 2) * (128 * 128);
                        tc_mma_f16_ss(tmem + kColS + 128 * i, umma_desc_k_sw128(a + off) + 2 * (k & 3),
                                      umma_desc_k_sw128(b + off) + 2 * (k & 3), kIdescS, k != 0);
                    }
                    tc_commit(sfull + 8 * i);
                    if (!two || i == 1) tc_commit(kempty + 8 * stage);
                    return true;
                };
                for (int s = 0; s < min(2, steps) && ok; ++s) ok = issue_s(s);
                for (int s = 0; s < steps && ok; ++s) {
                    const int i = s & 1, t = two ? s >> 1 : s;
                    const uint32_t stage = (n_kv + t) & 1u, phase = ((n_kv + t) >> 1) & 1u;
                    ok = mbar_wait(pfull + 8 * i, n_s[i] & 1u, abort_flag, &s_word);
                    ++n_s[i];
                    if (ok && (!two || i == 0)) ok = mbar_wait(vfull + 8 * stage, phase, abort_flag, &s_word);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < kTileKeys / 16; ++k)
                        tc_mma_f16_ts(tmem + kColO + 128 * i, tmem + kColS + 128 * i + 8 * k,
                                      umma_desc_mn_sw128(v_at + stage * kT + k * 2048, 128 * 128), idesc_o<D>(), s >= 2 || k != 0);
                    tc_commit(odone + 8 * i);
                    if (!two || i == 1) tc_commit(vempty + 8 * stage);
                    if (s + 2 < steps) ok = issue_s(s + 2);
                }
                n_kv += tiles;
            }
        } else {
            // ------------------------------------------------------------------ softmax
            const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
            const uint32_t sc = lanes + kColS + 128 * acc, oc = lanes + kColO + 128 * acc;
            const uint32_t *mask = s_mask + (node >= 0 ? node - node0 : 0) * words;
            float mref = -INFINITY, l = 0.0f;
            const int my = two ? tiles : (tiles + 1 - acc) >> 1;      // this accumulator's key tiles
            for (int j = 0; j < my; ++j) {
                const int pos0 = key0 + (two ? j : 2 * j + acc) * kTileKeys;
                ok = __all_sync(0xffffffffu, mbar_wait(sfull + 8 * acc, n_s[0] & 1u, abort_flag, &s_word));
                if (!ok) break;
                tc_fence_after();
                const bool edge = pos0 + kTileKeys > sg.len;
                float mx = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < kTileKeys / 32; ++c) {
                    float v[32];
                    tc_ld32(sc + c * 32, v);
                    if (edge) {
                        uint32_t see = visible32(pos0 + 32 * c, sg.len, node, p.parent != nullptr, mask, words);
                        if (pos0 + 32 * c >= sg.len && node < 0) see = 0u;
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = (see >> k) & 1u ? v[k] : -INFINITY;
                    }
                    float a = v[0], b = v[1];
#pragma unroll
                    for (int k = 2; k < 32; k += 2) { a = fmaxf(a, v[k]); b = fmaxf(b, v[k + 1]); }
                    mx = fmaxf(mx, fmaxf(a, b));
                }
                mx *= rs;
                // the maximum moves only when it grows by more than 2^8; the first tile just sets it
                const bool grow = mx > mref + 8.0f;
                if (__any_sync(0xffffffffu, grow)) {
                    const float to = grow ? mx : mref;
                    const float f = to == -INFINITY || mref == to ? 1.0f : ex2(mref - to);
                    mref = to;
                    l *= f;
                    if (j > 0) {
                        ok = __all_sync(0xffffffffu, mbar_wait(odone + 8 * acc, (n_s[0] - 1u) & 1u, abort_flag, &s_word));
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            float v[32];
                            tc_ld32(oc + c * 32, v);
#pragma unroll
                            for (int k = 0; k < 32; ++k) v[k] *= f;
                            tc_st32(oc + c * 32, v);
                        }
                    }
                }
                // P = 2^(s - mref + 7), see mars_attention.cu
                const float ref = mref == -INFINITY ? 0.0f : mref - 7.0f;
                float l2[2] = {0.0f, 0.0f};
#pragma unroll 1
                for (int c = 0; c < kTileKeys / 32; ++c) {
                    float v[32];
                    tc_ld32(sc + c * 32, v);
                    if (edge) {
                        uint32_t see = visible32(pos0 + 32 * c, sg.len, node, p.parent != nullptr, mask, words);
                        if (pos0 + 32 * c >= sg.len && node < 0) see = 0u;
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = (see >> k) & 1u ? v[k] : -INFINITY;
                    }
                    uint32_t h[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float p0 = ex2(fmaf(v[2 * k], rs, -ref)), p1 = ex2(fmaf(v[2 * k + 1], rs, -ref));
                        l2[0] += p0;
                        l2[1] += p1;
                        h[k] = f16x2_from(p0, p1);
                    }
                    tc_st16(sc + c * 16, h);        // over columns of S that were read already
                }
                l += l2[0] + l2[1];
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull + 8 * acc);
                ++n_s[0];
            }
            if (ok && my > 0) {
                ok = __all_sync(0xffffffffu, mbar_wait(odone + 8 * acc, (n_s[0] - 1u) & 1u, abort_flag, &s_word));
                tc_fence_after();
            }
            s_m[acc * 128 + (tid & 127)] = mref;
            s_l[acc * 128 + (tid & 127)] = l;
            if (ok && !two && acc == 1 && my > 0) {
                // second accumulator of the same rows: over to the first through the free K stages
                float *x = reinterpret_cast<float *>(sm + 2 * kT);
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    float v[32];
                    tc_ld32(oc + c * 32, v);
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[(c * 32 + k) * 128 + (tid & 127)] = v[k];
                }
            }
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        ok = *abort_flag == 0;
        __syncthreads();
        if (!ok) {
            if (tid == 0 && p.status) p.status[sg.b] = MARS_SEQ_TIMEOUT;
            break;
        }

        // ---- result of the segment: thread = row, columns of d in order
        const bool has_row = warp < 8 && (two || acc == 0);
        const uint32_t oc = tmem + ((uint32_t)((warp & 3) * 32) << 16) + kColO + 128 * acc;
        const int my0 = two ? tiles : (tiles + 1) >> 1, my1 = two ? tiles : tiles >> 1;
        float m = -INFINITY, sum = 0.0f, f0 = 1.0f, f1 = 0.0f;
        if (has_row) {
            m = s_m[row];
            sum = s_l[row];
            if (!two && my1 > 0) {
                const float m1 = s_m[128 + row], mm = fmaxf(m, m1);
                f0 = m == -INFINITY ? 0.0f : ex2(m - mm);
                f1 = m1 == -INFINITY ? 0.0f : ex2(m1 - mm);
                sum = sum * f0 + s_l[128 + row] * f1;
                m = mm;
            }
        }
        (void)my0;
        const float *second = reinterpret_cast<const float *>(sm + 2 * kT);
        const bool merge = !two && my1 > 0;
        float *part = p.partial + (int64_t)(2 * blockIdx.x + (u == r.begin ? 0 : 1)) * tile_slot_floats<D>();
        const bool out_row = has_row && row < rows && s_live[node >= 0 ? node - node0 : 0];
        const int64_t out_at = out_row ? ((int64_t)sg.b * p.N + node) * p.out_row +
                                             (int64_t)(sg.head * p.group + (row0 + row) % p.group) * p.out_head : 0;
        const float vscale = p.scales[p.kv.kv_heads + sg.head];
        if (has_row) {
            const float norm = vscale / sum;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                float v[32];
                tc_ld32(oc + c * 32, v);
                if (merge) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = v[k] * f0 + second[(c * 32 + k) * 128 + row] * f1;
                }
                if (!whole) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) part[(c * 32 + k) * TileShape::M + row] = v[k];
                } else if (out_row) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] *= norm;
#pragma unroll
                    for (int k = 0; k < 32; k += 8) store_out8<DT>(p.out, out_at + c * 32 + k, v + k);
                }
            }
            if (!whole) {
                part[D * TileShape::M + row] = m;
                part[(D + 1) * TileShape::M + row] = sum;
            }
        }
        if (!whole) {
            const int c0 = (int)(sg.item / r.per), c1 = (int)((sg.item + sg.units - 1) / r.per);
            __threadfence();
            __syncthreads();
            if (tid == 0) s_last = atomicAdd(p.counters + c0, 1u) == (unsigned)(c1 - c0);
            __syncthreads();
            if (s_last) {
                __threadfence();
                if (has_row) {
                    auto slot = [&](int c) { return p.partial + (int64_t)(2 * c + (r.per * c >= sg.item ? 0 : 1)) * tile_slot_floats<D>(); };
                    m = -INFINITY;
                    for (int c = c0; c <= c1; ++c) m = fmaxf(m, __ldcg(slot(c) + D * TileShape::M + row));
                    sum = 0.0f;
                    for (int c = c0; c <= c1; ++c) {
                        const float pm = __ldcg(slot(c) + D * TileShape::M + row);
                        sum += (pm == -INFINITY ? 0.0f : ex2(pm - m)) * __ldcg(slot(c) + (D + 1) * TileShape::M + row);
                    }
                    const float norm = vscale / sum;
#pragma unroll 1
                    for (int d0 = 0; d0 < D; d0 += 32) {
                        float v[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = 0.0f;
                        for (int c = c0; c <= c1; ++c) {
                            const float *src = slot(c);
                            const float pm = __ldcg(src + D * TileShape::M + row);
                            const float f = pm == -INFINITY ? 0.0f : ex2(pm - m);
#pragma unroll
                            for (int k = 0; k < 32; ++k) v[k] += __ldcg(src + (d0 + k) * TileShape::M + row) * f;
                        }
                        if (out_row) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) v[k] *= norm;
#pragma unroll
                            for (int k = 0; k < 32; k += 8) store_out8<DT>(p.out, out_at + d0 + k, v + k);
                        }
                    }
                }
                if (tid == 0) p.counters[c0] = 0u;
            }
        }
        tc_fence_before();
        __syncthreads();                  // Q, masks, K stages, accumulators free for the next segment
        tc_fence_after();
        u += sg.unit1 - sg.unit0;
    }

    if (warp == 12 && lane == 0) {
        // all MMAs of this thread must retire before tensor memory is freed
        tc_commit(drain);
        const long long t0 = clock64();
        while (!mbar_try_wait(drain, 0) && clock64() - t0 < kWaitCycles) {}
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemAll) : "memory");
    }
}

size_t attn_tile_partial_bytes(int d)
{
    return sizeof(float) * 2 * kAttnSms * (size_t)(d == 128 ? tile_slot_floats<128>() : tile_slot_floats<64>());
}

template <int D, int DT>
static mars_status_t tile_launch(const AttnParams &p, cudaStream_t st)
{
    cudaError_t e = cudaFuncSetAttribute(attn_tile_kernel<D, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tile_smem_bytes<D>());
    if (e == cudaSuccess)
        e = launch_pdl(hook(kHookNoOverlap) == 0, attn_tile_kernel<D, DT>, dim3(kAttnSms), dim3(kTileThreads), tile_smem_bytes<D>(), st, p);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return MARS_ERR_CUDA; }
    return MARS_OK;
}

mars_status_t attn_tile_launch(const AttnParams &p, int d, int dt, cudaStream_t st)
{
    if (d == 128) return dt == MARS_BF16 ? tile_launch<128, MARS_BF16>(p, st) : tile_launch<128, MARS_FP16>(p, st);
    return dt == MARS_BF16 ? tile_launch<64, MARS_BF16>(p, st) : tile_launch<64, MARS_FP16>(p, st);
}

}  // namespace mars
