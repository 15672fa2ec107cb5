// libmars: attention of draft nodes over the paged 4-bit cache, many query rows per KV head.
//
// The products run on tcgen05.mma (kind::f16, 128 x 128 x 16 steps, fp32 accumulators in tensor
// memory); see mars_attention.cu for the arithmetic.  Up to 256 query rows of one KV head -- a whole
// tree of 60 nodes with four heads to a KV head -- share every key that is unpacked.  One block per SM:
//
//   warps 0-3   softmax of accumulator 0 (thread = query row): Q into shared memory, score scale, mask,
//   warps 4-7   running maximum and sum, P back into tensor memory, the result; same for accumulator 1
//   warps 8-11  unpack: code * scale in fp16 from the ring into two stages of K and of V tiles
//               [128 keys][d] (128-byte swizzle)
//   warp 12     tensor memory, and the MMAs: S = Q K^T (both operands in shared memory), O += P V (P in
//               tensor memory over the columns of S; V's tile read with d as its leading dimension,
//               so that neither K nor V is ever transposed)
//   warp 13     page blocks into a ring of three half tiles (64 keys) with bulk copies.  A separate
//               engine on purpose: loads by the unpacking threads would be waited for by the proxy
//               fence that hands each tile to the tensor cores (measured: half of their time).
//
// Two accumulators keep the tensor cores busy while a softmax runs: with more than 128 rows they hold
// the two halves of the rows and both see every key tile; with fewer they hold the same rows and take
// the key tiles in turn, and their results (same lanes of tensor memory) are merged at the end.
// The step order of the issuing warp is S(0) S(1) | P V(0) S(2) | P V(1) S(3) | ...: tensor operations
// execute in issue order, so S(u + 2) may overwrite the P that P V(u) has read.
//
// Each role walks the block's segments by itself; loader, unpacking and MMA run ahead into the next one.
//
// Every wait is bounded.  One that gives up raises the block's abort flag; all roles fall through to
// the common end, the sequence's status becomes MARS_SEQ_TIMEOUT, tensor memory is freed.
#include "mars_attention.cuh"
#include "mars_hooks.cuh"
#include "mars_tcgen05.cuh"

#include <cuda_runtime.h>

#include "mars_kv.h"

namespace mars {

constexpr int kTileThreads = 512;
constexpr int kTileKeys = 128;
constexpr int kHalfKeys = 64;                          // keys of a ring slot
constexpr int kRingSlots = 3;
constexpr uint32_t kTmemAll = 512;
constexpr uint32_t kColS = 0, kColO = 256;             // accumulator i: S at 128 i, O at 256 + 128 i

template <int D> constexpr uint32_t tile_bytes() { return 128u * D * 2; }    // 128 rows of d fp16
template <int D> constexpr uint32_t slot_bytes() { return (kHalfKeys / kKvBlock) * kv_block_bytes(D); }
template <int D> constexpr int tile_slot_floats() { return TileShape::M * (D + 2); }

constexpr int kMaskWords = kTileMaxTree / 32;

// shared memory: Q (2 tiles) | K (2 stages) | V (2 stages) | ring | masks | parents | live | m, l of
// accumulator 1 | block flags | barriers
struct TileSmem {
    uint32_t mask[kTileMaxTree * kMaskWords];
    int par[kTileMaxTree];
    unsigned char live[kTileMaxTree];
    float m1[128], l1[128];
    int page[kRingSlots][4];                            // of a slot's 16-key blocks: -1 not in the pool, -2 no key
    uint64_t kfull[2], kempty[2], vfull[2], vempty[2], sfull[2], pfull[2], odone[2];
    uint64_t rfull[kRingSlots], rempty[kRingSlots], qfull, drain;
    uint32_t tmem;
    int abort, bad, last, ok;
    unsigned word;
};

template <int D> constexpr size_t tile_smem_bytes()
{
    const size_t need = 1024 + 6 * (size_t)tile_bytes<D>() + kRingSlots * slot_bytes<D>() + sizeof(TileSmem);
    return need > 120 * 1024 ? need : 120 * 1024;      // one block per SM: each takes all of tensor memory
}
static_assert(tile_smem_bytes<128>() <= 227 * 1024 - 1024, "shared memory of one SM, with room for the static part");

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
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// (a0, a1) * (m, m) + (c, c) and (a0, a1) + (b0, b1), both halves rounded as by themselves
__device__ __forceinline__ void fma2(float &a0, float &a1, float m, float c)
{
    asm("{\n\t.reg .b64 a, m, c;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 m, {%2, %2};\n\tmov.b64 c, {%3, %3};\n\t"
        "fma.rn.f32x2 a, a, m, c;\n\tmov.b64 {%0, %1}, a;\n\t}" : "+f"(a0), "+f"(a1) : "f"(m), "f"(c));
}
__device__ __forceinline__ void add2(float &a0, float &a1, float b0, float b1)
{
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\t"
        "add.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}" : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1));
}

__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// Instruction descriptors: D fp32, A and B fp16, M = 128; S: N = 128 keys, both operands K-major;
// O: N = d, B with d as its leading dimension.
constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kTileKeys >> 3) << 17) | ((128u >> 4) << 24);
template <int D> constexpr uint32_t idesc_o() { return (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((128u >> 4) << 24); }

// The 32 keys from position p0 on that node `node` may see, as bits (node -1: a row behind the last).
__device__ __forceinline__ uint32_t visible32(int p0, int len, int node, bool tree, const uint32_t *mask, int words)
{
    const int m0 = p0 - len;
    if (m0 <= -32) return 0xffffffffu;
    if (!tree || node < 0) {
        const int cnt = node + 1 - m0;                  // first cnt keys
        return cnt >= 32 ? 0xffffffffu : cnt <= 0 ? 0u : (1u << cnt) - 1u;
    }
    if (m0 < 0) return ((1u << -m0) - 1u) | (mask[0] << -m0);      // 1..31 committed tokens, then nodes 0, 1, ...
    const int w = m0 >> 5;
    const uint32_t lo = w < words ? mask[w] : 0u, hi = w + 1 < words ? mask[w + 1] : 0u;
    return __funnelshift_r(lo, hi, m0 & 31);
}

// A segment as this kernel sees it.
struct TileSegment : AttnSegment {
    int rows, row0;          // query rows of the tile, its first one
    int key0, tiles, steps;  // first key, key tiles, S / P V steps
    bool two;                // the accumulators hold different rows (else they take turns on the keys)
    bool whole;
};

__device__ __forceinline__ TileSegment tile_segment(const AttnParams &p, AttnRange &r, int64_t u)
{
    TileSegment s;
    static_cast<AttnSegment &>(s) = attn_segment<TileShape>(p, r, u);
    s.rows = attn_tile_rows<TileShape>(p, s.n, s.tile);
    s.row0 = s.tile * TileShape::M;
    s.two = s.rows > 128;
    const int uk = TileShape::unit_keys(s.rows);
    s.key0 = s.unit0 * uk;
    s.tiles = (min(s.keys, s.unit1 * uk) - s.key0 + kTileKeys - 1) / kTileKeys;
    s.steps = s.two ? 2 * s.tiles : s.tiles;
    s.whole = s.unit0 == 0 && s.unit1 == s.units;
    return s;
}

// ------------------------------------------------------------------------------------- warp 13

template <int D>
__device__ __forceinline__ void tile_load(const AttnParams &p, AttnRange r, TileSmem *sh, uint32_t ring)
{
    const int lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh->abort;
    uint32_t slot = 0, phase = 0, issued = 0;
    bool ok = true;
    for (int64_t u = r.begin; u < r.end && ok;) {
        const TileSegment sg = tile_segment(p, r, u);
        const int halves = 2 * sg.tiles, valid = sg.len + sg.n;     // keys from `valid` on were never written
        // lane 4h + c: page id of block c of half tile h0 + h
        auto ids_from = [&](int h0) {
            const int hh = h0 + (lane >> 2), pos = sg.key0 + hh * kHalfKeys + (lane & 3) * kKvBlock;
            return hh < halves && pos < valid ? kv_page_id(p.kv, sg.b, pos) : -2;
        };
        int ids = ids_from(0), next = ids_from(8);
        for (int h = 0; h < halves; ++h) {
            if (h && (h & 7) == 0) { ids = next; next = ids_from(h + 8); }
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh->rempty[slot]), phase ^ 1u, abort_flag, &sh->word));
            if (!ok) break;
            const int id = __shfl_sync(0xffffffffu, ids, (h & 7) * 4 + (lane & 3));
            const bool have = lane < 4 && id >= 0;
            const int n = __popc(__ballot_sync(0xffffffffu, have));
            if (lane < 4) sh->page[slot][lane] = id;
            __syncwarp();
            const uint32_t bar = smem_u32(&sh->rfull[slot]);
            if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n * kv_block_bytes(D)));
            __syncwarp();
            if (have)
                bulk_load(ring + slot * slot_bytes<D>() + lane * kv_block_bytes(D),
                          kv_block<D>(p.kv, p.layer, id, sg.head, sg.key0 + h * kHalfKeys + lane * kKvBlock),
                          kv_block_bytes(D), bar);
            ++issued;
            if (++slot == kRingSlots) { slot = 0; phase ^= 1u; }
        }
        u += sg.unit1 - sg.unit0;
    }
    if (!ok && lane == 0) {
        // copies in flight must land before the block may end (bounded)
        for (uint32_t i = 0; i < kRingSlots && i < issued; ++i) {
            if (slot == 0) { slot = kRingSlots; phase ^= 1u; }
            --slot;
            const long long t0 = clock64();
            while (!mbar_try_wait(smem_u32(&sh->rfull[slot]), phase) && clock64() - t0 < 20000000ll) {}
        }
    }
}

// ------------------------------------------------------------------------------------- warps 8-11

// K (v = 0) or V (v = 1) of the slot's 64 keys into rows key0 .. key0+63 of a tile.  Thread ut: key ut/2;
// 16-byte chunks of 32 codes, the order of a row's halves alternating with the key so that both the
// reads (rows d/2 bytes apart) and the swizzled writes are free of bank conflicts.
template <int D>
__device__ __forceinline__ void tile_unpack(const unsigned char *slot, int key0, int page, unsigned char *tile, int v)
{
    const int ut = threadIdx.x & 127, in = ut >> 1, key = key0 + in;
    const unsigned char *blk = slot + (in >> 4) * kv_block_bytes(D) + (v ? 8 * D : 0) + (in & 15) * (D / 2);
    const unsigned char *scl = slot + (in >> 4) * kv_block_bytes(D) + 16 * D + (v ? D : 0) + (in & 15) * (D / 16);
#pragma unroll
    for (int a = 0; a < D / 64; ++a) {
        const int part = ((D == 128 ? a ^ ((in >> 1) & 1) : 0) << 1) | (ut & 1);
        uint4 c = make_uint4(0u, 0u, 0u, 0u);
        uint32_t s = v && page == -1 ? 0x7f7fu : 0u;             // no such page: NaN
        if (page >= 0) {
            c = *reinterpret_cast<const uint4 *>(blk + part * 16);
            s = *reinterpret_cast<const unsigned short *>(scl + part * 2);
        }
        const uint32_t sh = e4m3x2_to_f16x2(s);
        const uint32_t sc[2] = {__byte_perm(sh, sh, 0x1010), __byte_perm(sh, sh, 0x3232)};
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
        unsigned char *dst = tile + (part >> 1) * (128 * 128) + key * 128;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t h[4];
            e2m1x8_to_f16x2(w[k], h);
            const uint32_t f = sc[k >> 1];
            *reinterpret_cast<uint4 *>(dst + ((((part & 1) * 4 + k) ^ (key & 7)) * 16)) =
                make_uint4(hmul2(h[0], f), hmul2(h[1], f), hmul2(h[2], f), hmul2(h[3], f));
        }
    }
}

template <int D>
__device__ __forceinline__ void tile_unpack_role(const AttnParams &p, AttnRange r, TileSmem *sh, unsigned char *k_tiles,
                                                 unsigned char *v_tiles, const unsigned char *ring)
{
    const int lane = threadIdx.x & 31, in = (threadIdx.x & 127) >> 1;
    volatile int *abort_flag = &sh->abort;
    uint32_t n_kv = 0, slot = 0, phase = 0;
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity) {
        return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity, abort_flag, &sh->word)) != 0;
    };
    for (int64_t u = r.begin; u < r.end && ok;) {
        const TileSegment sg = tile_segment(p, r, u);
        const int valid = sg.len + sg.n;
        for (int t = 0; t < sg.tiles && ok; ++t, ++n_kv) {
            const uint32_t st = n_kv & 1u, par = ((n_kv >> 1) & 1u) ^ 1u;
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                ok = wait(&sh->rfull[slot], phase) && (half || wait(&sh->kempty[st], par));
                if (!ok) break;
                const unsigned char *src = ring + slot * slot_bytes<D>();
                int page = sh->page[slot][in >> 4];
                if (sg.key0 + t * kTileKeys + half * kHalfKeys + in >= valid) page = -2;    // slot never written
                tile_unpack<D>(src, half * kHalfKeys, page, k_tiles + st * tile_bytes<D>(), 0);
                if (half) {
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh->kfull[st]));
                } else {
                    ok = wait(&sh->vempty[st], par);
                    if (!ok) break;
                }
                tile_unpack<D>(src, half * kHalfKeys, page, v_tiles + st * tile_bytes<D>(), 1);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->rempty[slot]));
                if (half) {
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh->vfull[st]));
                }
                if (++slot == kRingSlots) { slot = 0; phase ^= 1u; }
            }
        }
        u += sg.unit1 - sg.unit0;
    }
}

// ------------------------------------------------------------------------------------- warp 12

template <int D>
__device__ __forceinline__ void tile_mma(const AttnParams &p, AttnRange r, TileSmem *sh, uint32_t tmem, uint32_t q_at,
                                         uint32_t k_at, uint32_t v_at)
{
    constexpr uint32_t kT = tile_bytes<D>();
    const int lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh->abort;
    uint32_t n_kv = 0, n_seg = 0, n_p[2] = {0, 0};
    bool ok = true;
    for (int64_t u = r.begin; u < r.end && ok; ++n_seg) {
        const TileSegment sg = tile_segment(p, r, u);
        if (lane == 0) {
            auto wait = [&](uint64_t *bar, uint32_t parity) { return mbar_wait(smem_u32(bar), parity, abort_flag, &sh->word); };
            auto issue_s = [&](int s) {
                const int i = s & 1, t = sg.two ? s >> 1 : s;
                const uint32_t st = (n_kv + t) & 1u, par = ((n_kv + t) >> 1) & 1u;
                if ((!sg.two || i == 0) && !wait(&sh->kfull[st], par)) return false;
                tc_fence_after();
                const uint64_t a = umma_desc_k_sw128(q_at + (sg.two ? i * kT : 0)), b = umma_desc_k_sw128(k_at + st * kT);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = (k >> 2) * ((128 * 128) >> 4) + 2 * (k & 3);
                    tc_mma_f16_ss(tmem + kColS + 128 * i, a + off, b + off, kIdescS, k != 0);
                }
                tc_commit(smem_u32(&sh->sfull[i]));
                if (!sg.two || i == 1) tc_commit(smem_u32(&sh->kempty[st]));
                return true;
            };
            ok = wait(&sh->qfull, n_seg & 1u);
            for (int s = 0; s < min(2, sg.steps) && ok; ++s) ok = issue_s(s);
            for (int s = 0; s < sg.steps && ok; ++s) {
                const int i = s & 1, t = sg.two ? s >> 1 : s;
                const uint32_t st = (n_kv + t) & 1u, par = ((n_kv + t) >> 1) & 1u;
                ok = wait(&sh->pfull[i], n_p[i] & 1u);
                ++n_p[i];
                if (ok && (!sg.two || i == 0)) ok = wait(&sh->vfull[st], par);
                if (!ok) break;
                tc_fence_after();
                const uint64_t b = umma_desc_mn_sw128(v_at + st * kT, 128 * 128);
#pragma unroll
                for (int k = 0; k < kTileKeys / 16; ++k)
                    tc_mma_f16_ts(tmem + kColO + 128 * i, tmem + kColS + 128 * i + 8 * k, b + k * (2048 >> 4), idesc_o<D>(),
                                  s >= 2 || k != 0);
                tc_commit(smem_u32(&sh->odone[i]));
                if (!sg.two || i == 1) tc_commit(smem_u32(&sh->vempty[st]));
                if (s + 2 < sg.steps) ok = issue_s(s + 2);
            }
        }
        ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
        n_kv += sg.tiles;
        u += sg.unit1 - sg.unit0;
    }
    if (lane == 0) {
        // all MMAs of this thread must retire before tensor memory is freed
        tc_commit(smem_u32(&sh->drain));
        const long long t0 = clock64();
        while (!mbar_try_wait(smem_u32(&sh->drain), 0) && clock64() - t0 < kWaitCycles) {}
    }
}

// ------------------------------------------------------------------------------------- warps 0-7

template <int D, int DT>
__device__ __forceinline__ void tile_softmax(const AttnParams &p, AttnRange r, TileSmem *sh, uint32_t tmem, unsigned char *q_tiles)
{
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int acc = warp >> 2, rr = tid & 127;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t sc = lanes + kColS + 128 * acc, oc = lanes + kColO + 128 * acc;
    volatile int *abort_flag = &sh->abort;
    uint32_t n_s = 0;                        // S tiles of this accumulator so far
    for (int64_t u = r.begin; u < r.end;) {
        const TileSegment sg = tile_segment(p, r, u);
        const bool tree = p.parent != nullptr;
        const int node0 = attn_node(p, sg.row0);
        const int words = (sg.n + 31) >> 5;
        const int row = (sg.two ? acc * 128 : 0) + rr;
        const int node = row < sg.rows ? attn_node(p, sg.row0 + row) : -1;
        const int head = sg.head * p.group + (node >= 0 ? sg.row0 + row - node * p.group : 0);

        // ---- Q: this thread's row, scaled to fp16, into its swizzled tile
        float rs;                            // score scale of the row in log2 units
        {
            uint4 w[D / 8];
            if (node >= 0) {
                const uint4 *src = reinterpret_cast<const uint4 *>(p.q + 2 * (((int64_t)sg.b * p.N + node) * p.q_row + head * p.q_head));
#pragma unroll
                for (int c = 0; c < D / 8; ++c) w[c] = src[c];
            } else {
#pragma unroll
                for (int c = 0; c < D / 8; ++c) w[c] = make_uint4(0u, 0u, 0u, 0u);
            }
            float m = 0.0f;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint32_t x[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = widen2<DT>(x[j]);
                    m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
            }
            float down, up;
            row_scale(m, &down, &up);
            rs = fmaxf(p.scale_log2 * p.scales[sg.head] * up, 1.17549435e-38f);
            if (sg.two || acc == 0) {
                unsigned char *dst = q_tiles + acc * tile_bytes<D>() + rr * 128;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const uint32_t x[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
                    uint32_t h[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 f = widen2<DT>(x[j]);
                        h[j] = f16x2_from(f.x * down, f.y * down);
                    }
                    *reinterpret_cast<uint4 *>(dst + (c >> 3) * (128 * 128) + (((c & 7) ^ (rr & 7)) * 16)) = make_uint4(h[0], h[1], h[2], h[3]);
                }
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->qfull));
        }
        int status = MARS_SEQ_OK;
        if (tree)
            status = attn_tree_masks(p, sg.b, sg.n, node0, attn_node(p, sg.row0 + sg.rows - 1) - node0 + 1, sh->par, sh->mask,
                                     words, sh->live, &sh->bad, tid, 256, softmax_sync);
        if (tid == 0 && p.status && sg.head == 0 && sg.tile == 0 && sg.unit0 == 0) p.status[sg.b] = status;

        const uint32_t *mask = sh->mask + (tree && node >= 0 ? node - node0 : 0) * words;
        float mref = -INFINITY, l = 0.0f;
        const int my = sg.two ? sg.tiles : (sg.tiles + 1 - acc) >> 1;      // this accumulator's key tiles
        bool ok = true;
        for (int j = 0; j < my; ++j) {
            const int pos0 = sg.key0 + (sg.two ? j : 2 * j + acc) * kTileKeys;
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh->sfull[acc]), n_s & 1u, abort_flag, &sh->word));
            if (!ok) break;
            tc_fence_after();
            float v[kTileKeys];
#pragma unroll
            for (int c = 0; c < kTileKeys; c += 32) tc_ld32_issue(sc + c, v + c);
#pragma unroll
            for (int c = 0; c < kTileKeys; c += 32) tc_ld32_wait(v + c);
            if (pos0 + kTileKeys > sg.len) {
#pragma unroll
                for (int c = 0; c < kTileKeys / 32; ++c) {
                    const uint32_t see = visible32(pos0 + 32 * c, sg.len, node, tree, mask, words);
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[32 * c + k] = (see >> k) & 1u ? v[32 * c + k] : -INFINITY;
                }
            }
            float m4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int k = 4; k < kTileKeys - 4; k += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e) m4[e] = max3(m4[e], v[k + e], v[k + 4 + e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) m4[e] = fmaxf(m4[e], v[kTileKeys - 4 + e]);
            const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * rs;
            // the maximum moves only when it grows by more than 2^8; the first tile just sets it
            const bool grow = mx > mref + 8.0f;
            if (__any_sync(0xffffffffu, grow)) {
                const float to = grow ? mx : mref;
                const float f = to == -INFINITY || mref == to ? 1.0f : ex2(mref - to);
                mref = to;
                l *= f;
                if (j > 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh->odone[acc]), (n_s - 1u) & 1u, abort_flag, &sh->word));
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        float x[32];
                        tc_ld32_issue(oc + c * 32, x);
                        tc_ld32_wait(x);
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] *= f;
                        tc_st32(oc + c * 32, x);
                    }
                }
            }
            // P = 2^(s - mref + 7), see mars_attention.cu; over columns of S, all of which were read
            const float minus = mref == -INFINITY ? 0.0f : 7.0f - mref;
            float l4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < kTileKeys / 32; ++c) {
                uint32_t h[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    float &a = v[32 * c + 2 * k], &b = v[32 * c + 2 * k + 1];
                    fma2(a, b, rs, minus);
                    a = ex2(a);
                    b = ex2(b);
                    add2(l4[2 * (k & 1)], l4[2 * (k & 1) + 1], a, b);
                    h[k] = f16x2_from(a, b);
                }
                tc_st16(sc + c * 16, h);
            }
            l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->pfull[acc]));
            ++n_s;
        }
        if (ok && my > 0) {
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh->odone[acc]), (n_s - 1u) & 1u, abort_flag, &sh->word));
            tc_fence_after();
        }
        if (!sg.two && acc == 1) { sh->m1[rr] = mref; sh->l1[rr] = l; }
        tc_fence_before();
        softmax_sync();
        tc_fence_after();
        if (tid == 0) sh->ok = *abort_flag == 0;
        softmax_sync();
        if (!sh->ok) {
            if (tid == 0 && p.status) p.status[sg.b] = MARS_SEQ_TIMEOUT;
            break;
        }

        // ---- result of the segment: thread = row
        const bool has_row = sg.two || acc == 0;
        const bool merge = !sg.two && sg.tiles > 1;
        float m = mref, sum = l, f0 = 1.0f, f1 = 0.0f;
        if (has_row && merge) {
            const float m1 = sh->m1[rr], mm = fmaxf(m, m1);
            f0 = m == -INFINITY ? 0.0f : ex2(m - mm);
            f1 = m1 == -INFINITY ? 0.0f : ex2(m1 - mm);
            sum = sum * f0 + sh->l1[rr] * f1;
            m = mm;
        }
        const bool out_row = has_row && node >= 0 && (!tree || sh->live[node - node0]);
        const int64_t out_at = out_row ? ((int64_t)sg.b * p.N + node) * p.out_row + (int64_t)head * p.out_head : 0;
        const float vscale = p.scales[p.kv.kv_heads + sg.head];
        constexpr int kF = tile_slot_floats<D>();
        if (has_row) {
            float *part = p.partial + (int64_t)(2 * blockIdx.x + (u == r.begin ? 0 : 1)) * kF;
            const float norm = vscale / sum;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                float v[32];
                tc_ld32_issue(oc + c * 32, v);
                tc_ld32_wait(v);
                if (merge) {
                    float x[32];
                    tc_ld32_issue(oc + 128 + c * 32, x);       // the second accumulator, same lanes
                    tc_ld32_wait(x);
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = v[k] * f0 + x[k] * f1;
                }
                if (!sg.whole) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) part[(c * 32 + k) * TileShape::M + row] = v[k];
                } else if (out_row) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] *= norm;
#pragma unroll
                    for (int k = 0; k < 32; k += 8) store_out8<DT>(p.out, out_at + c * 32 + k, v + k);
                }
            }
            if (!sg.whole) {
                part[D * TileShape::M + row] = m;
                part[(D + 1) * TileShape::M + row] = sum;
            }
        }
        if (!sg.whole) {
            const int c0 = (int)(sg.item / r.per), c1 = (int)((sg.item + sg.units - 1) / r.per);
            __threadfence();
            softmax_sync();
            if (tid == 0) sh->last = atomicAdd(p.counters + c0, 1u) == (unsigned)(c1 - c0);
            softmax_sync();
            if (sh->last) {
                __threadfence();
                if (has_row) {
                    // block order, running maximum; all of a block's values are loaded at once
                    float o[D];
                    m = -INFINITY;
                    sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < D; ++k) o[k] = 0.0f;
#pragma unroll 1
                    for (int c = c0; c <= c1; ++c) {
                        const float *src = p.partial + (int64_t)(2 * c + (r.per * c >= sg.item ? 0 : 1)) * kF + row;
                        const float pm = __ldcg(src + D * TileShape::M), pl = __ldcg(src + (D + 1) * TileShape::M);
                        const float mm = fmaxf(m, pm);
                        const float a = m == -INFINITY ? 0.0f : ex2(m - mm), b = pm == -INFINITY ? 0.0f : ex2(pm - mm);
                        m = mm;
                        sum = sum * a + pl * b;
#pragma unroll
                        for (int k = 0; k < D; ++k) o[k] = o[k] * a + __ldcg(src + k * TileShape::M) * b;
                    }
                    if (out_row) {
                        const float norm = vscale / sum;
#pragma unroll
                        for (int k = 0; k < D; ++k) o[k] *= norm;
#pragma unroll
                        for (int k = 0; k < D; k += 8) store_out8<DT>(p.out, out_at + k, o + k);
                    }
                }
                if (tid == 0) p.counters[c0] = 0u;
            }
        }
        tc_fence_before();
        softmax_sync();                   // masks, m1 / l1 and the accumulators are free for the next segment
        tc_fence_after();
        u += sg.unit1 - sg.unit0;
    }
}

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
    unsigned char *ring = sm + 6 * kT;
    TileSmem *sh = reinterpret_cast<TileSmem *>(ring + kRingSlots * slot_bytes<D>());
    const int tid = threadIdx.x, warp = tid >> 5;

    const AttnRange r = attn_split<TileShape, kTileThreads>(p);
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->kfull[i]), 4);
            mbar_init(smem_u32(&sh->vfull[i]), 4);
            mbar_init(smem_u32(&sh->kempty[i]), 1);
            mbar_init(smem_u32(&sh->vempty[i]), 1);
            mbar_init(smem_u32(&sh->sfull[i]), 1);
            mbar_init(smem_u32(&sh->pfull[i]), 4);
            mbar_init(smem_u32(&sh->odone[i]), 1);
        }
        for (int i = 0; i < kRingSlots; ++i) {
            mbar_init(smem_u32(&sh->rfull[i]), 1);
            mbar_init(smem_u32(&sh->rempty[i]), 4);
        }
        mbar_init(smem_u32(&sh->qfull), 8);
        mbar_init(smem_u32(&sh->drain), 1);
        sh->abort = 0;
        sh->word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&sh->tmem)), "r"(kTmemAll) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;

    // registers go where a thread holds a row of S: 2 * 192 + 72 + 56 = 512 = 4 * 128 per lane at launch
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        tile_softmax<D, DT>(p, r, sh, tmem, sm);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        tile_unpack_role<D>(p, r, sh, sm + 2 * kT, sm + 4 * kT, ring);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 12) tile_mma<D>(p, r, sh, tmem, base, base + 2 * kT, base + 4 * kT);
        else if (warp == 13) tile_load<D>(p, r, sh, smem_u32(ring));
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
