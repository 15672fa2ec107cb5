// libmars: attention of draft nodes over the paged 4-bit cache, many query rows per KV head.
//
// The products run on tcgen05.mma (kind::f16, 128 x 128 x 16 steps, fp32 accumulators in tensor
// memory); see mars_attention.cu for the arithmetic.  Up to 256 query rows of one KV head -- a whole
// tree of 60 nodes with four heads to a KV head -- share every key that is unpacked.  One block per SM:
//
//   warps 20-27 softmax, four warps to an accumulator (thread = query row): Q into shared memory, score
//               scale, mask, maximum, P back into tensor memory, the result
//   warps 4-11  unpack K, 12-19 V: a warp fetches its 16 keys of every tile with 16-byte asynchronous copies
//               a tile ahead, and writes code * scale in fp16 into two stages of tiles [128 keys][d]
//               (128-byte swizzle)
//   warp 3      tensor memory, and the MMAs: S = Q K^T (both operands in shared memory), O += P V (P in
//               tensor memory over the columns of S; V's tile read with d as its leading dimension,
//               so that neither K nor V is ever transposed)
//
// Two accumulators: with more than 128 rows they hold the two halves of the rows and both see every key
// tile; with fewer they hold the same rows and take the key tiles in turn, and their results (same lanes
// of tensor memory) are merged at the end.  The MMA order is S(0) S(1) | P V(0) S(2) | P V(1) S(3) | ...:
// tensor operations execute in issue order, so S(u + 2) may overwrite the P that P V(u) has read.
//
// What bounds it: a key tile of 256 rows takes 4500 cycles, and nothing is full in them (issue slots 43 %, 8000
// warp instructions; tensor pipe 36 %; shared memory about half).  S reads both operands from shared
// memory at its full rate, beside the unpacking warps' stores, so that the MMA warp takes 1400 to 1700 cycles
// for the two products of a step (1026 alone); softmax of a step takes about 3000 of an accumulator's 4500, and
// two accumulators overlap only in part.  64 trees of 60 nodes over contexts of 2000 to 12000 tokens (8 KV heads of
// 4, d 128): 420 us; one tree over 500000 tokens 580 us; four prompts of 2048 (4 KV heads of 4, d 64) 130 us.  Spills at
// d 128 (d 64): 284 (104) bytes stored and 432 (244) loaded, under the split of 136, 48 and 40 registers to the roles.
// Measured and not kept, us for those trees / prompts: S and P in halves of 64 keys, four in flight (503 / 126:
// with 64 columns S reads Q twice as often); 16 softmax warps with 64 scores a thread and 8 unpacking ones (526 /
// 130); P by the old reference in one pass over S, the maximum looked at afterwards (412 / 135); the MMA warp
// waiting for V and the next K before P, with fewer commits (436 / 132); a warp of its own for each accumulator's
// products (519 / 136); copies three tiles ahead for tiles of up to 128 rows, longer suspended waits (both as without).
//
// Each role walks the block's segments by itself; unpacking and MMA run ahead into the next one.
//
// Every wait is bounded.  One that gives up raises the block's abort flag.  Unpacking and MMA then fall
// through to the common end, where tensor memory is freed; the softmax warps walk the rest of the block's
// segments without keys: their rows become NaN, shared items get a partial result of NaN and their arrival,
// so that every counter is back at zero when the call ends, and the sequences say MARS_SEQ_TIMEOUT.
#include "mars_attention.cuh"
#include "mars_hooks.cuh"
#include "mars_tcgen05.cuh"

#include <cuda_runtime.h>

#include "mars_kv.h"

namespace mars {

constexpr int kTileThreads = 896;
constexpr int kSoftThreads = 256;
constexpr int kTileKeys = 128;
constexpr int kUnpackWarps = 8;                        // per K and V: 16 keys each
constexpr uint32_t kTmemAll = 512;
constexpr uint32_t kColO = 256;                        // accumulator i: S at 128 i, O at 256 + 128 i

template <int D> constexpr uint32_t tile_bytes() { return 128u * D * 2; }    // 128 rows of d fp16
template <int D> constexpr uint32_t slot_bytes() { return 9 * D; }           // a block's K or V: codes [16][d/2], scales [16][d/16]
template <int D> constexpr uint32_t ring_bytes() { return 2 * kUnpackWarps * slot_bytes<D>(); }
template <int D> constexpr int tile_slot_floats() { return TileShape::kMost * (D + 2); }

constexpr int kMaskWords = kTileMaxTree / 32;

// shared memory: Q (2 tiles) | K (2 stages) | V (2 stages) | a slot per unpacking warp | the rest
struct TileSmem {
    uint32_t mask[kTileMaxTree * kMaskWords];
    int par[kTileMaxTree];
    unsigned char live[kTileMaxTree];
    AttnSeqs seqs;
    float xm[2][128], xl[2][128];                       // [accumulator][row]: maxima and sums
    uint64_t kfull[2], kempty[2], vfull[2], vempty[2], sfull[2], pfull[2], odone[2];
    uint64_t qfull, drain;
    uint32_t tmem;
    int abort, bad, last;
    int ok;                                             // no wait gave up up to the last segment's end
    unsigned word;
};

template <int D> constexpr size_t tile_smem_bytes()
{
    const size_t need = 1024 + 6 * (size_t)tile_bytes<D>() + ring_bytes<D>() + sizeof(TileSmem);
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

// Issued by the one lane whose `lead` is set, as predicated instructions: in code that the whole warp runs
// the descriptors stay in uniform registers.  (Behind a branch on the lane every operand of every
// MMA is moved there first: 110 cycles apiece, and the issuing warp was what bounded the kernel.)
__device__ __forceinline__ void tc_mma_f16_ss(uint32_t lead, uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc), "r"(lead) : "memory");
}
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t lead, uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(acc), "r"(lead) : "memory");
}
__device__ __forceinline__ void tc_commit_if(uint32_t lead, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 ::"r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ uint32_t elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
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

__device__ __forceinline__ TileSegment tile_segment(const AttnParams &p, const TileSmem *sh, AttnRange &r, int64_t u)
{
    TileSegment s;
    static_cast<AttnSegment &>(s) = attn_segment<TileShape>(p, &sh->seqs, r, u);
    s.rows = attn_tile_rows<TileShape>(p, s.n, s.tile);
    s.row0 = s.tile * p.tile_rows;
    s.two = s.rows > 128;
    const int uk = TileShape::unit_keys(s.rows);
    s.key0 = s.unit0 * uk;
    s.tiles = s.unit1 > s.unit0 ? (min(s.keys, s.unit1 * uk) - s.key0 + kTileKeys - 1) / kTileKeys : 0;
    s.steps = s.two ? 2 * s.tiles : s.tiles;
    s.whole = s.unit1 - s.unit0 == s.units;
    return s;
}

// ------------------------------------------------------------------------------------- warps 4-19

// K (v = 0) or V (v = 1) of the warp's 16 keys (w: which of a tile).  Two threads per key; chunks of 32
// codes, the order of a row's halves alternating with the key so that both the reads (rows d/2 bytes
// apart) and the swizzled writes are free of bank conflicts.  A tile's codes go from the warp's slot to
// registers as soon as they are there; then the slot takes the next tile's, while this one waits for its
// place (until S, or P V, of two tiles ago is done).  Copies are groups of the warp's own: no barriers.
template <int D>
__device__ __forceinline__ void tile_unpack_role(const AttnParams &p, AttnRange r, TileSmem *sh, unsigned char *tiles,
                                                 unsigned char *slot, int v, int w)
{
    constexpr int kN = D / 64;
    const int lane = threadIdx.x & 31, in = lane >> 1, odd = lane & 1, key = w * kKvBlock + in;
    const int swap = D == 128 ? (in >> 1) & 1 : 0;
    const unsigned char *blk = slot + in * (D / 2), *scl = slot + 8 * D + in * (D / 16);
    volatile int *abort_flag = &sh->abort;
    uint64_t *full = v ? sh->vfull : sh->kfull, *empty = v ? sh->vempty : sh->kempty;
    const uint32_t slot_u32 = smem_u32(slot) + lane * 16;
    constexpr uint64_t kNoPage = 1;          // address that stands for a page outside the pool; 0: no key
    uint32_t n = 0;                          // tiles unpacked
    bool ok = true;
    for (int64_t u = r.begin; u < r.end && ok;) {
        const TileSegment sg = tile_segment(p, sh, r, u);
        if (sg.tiles == 0) { u += sg.span; continue; }
        const int valid = sg.len + sg.n, first = sg.key0 + w * kKvBlock;   // keys from `valid` on were never written
        // lane i: where the warp's block of tile i0 + i is
        auto locate = [&](int i0) -> uint64_t {
            const int pos = first + (i0 + lane) * kTileKeys;
            if (i0 + lane >= sg.tiles || pos >= valid) return 0;
            const int id = kv_page_id(p.kv, sg.b, pos);
            return id < 0 ? kNoPage : (uint64_t)(kv_block<D>(p.kv, p.layer, id, sg.head, pos) + v * 8 * D);
        };
        uint64_t here = locate(0), next = sg.tiles > 32 ? locate(32) : 0;
        uint64_t from = 0;                   // of the tile in the slot
        auto issue = [&](int t) {
            if (t && (t & 31) == 0) { here = next; next = locate(t + 32); }
            from = t < sg.tiles ? __shfl_sync(0xffffffffu, here, t & 31) : 0;
            if (from > kNoPage) {
                const unsigned char *src = (const unsigned char *)from + lane * 16;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) cp_async16(slot_u32 + i * 512, src + i * 512);
                // the scales follow K's codes by 16d bytes, V's by 9d
                if (lane < D / 16) cp_async16(slot_u32 + 8 * D, src + 16 * D - v * 7 * D);
            }
        };
        issue(0);
        for (int t = 0; t < sg.tiles; ++t, ++n) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
            uint4 c[kN];
            uint32_t s[kN];
            const bool have = from > kNoPage && first + t * kTileKeys + in < valid;
#pragma unroll
            for (int a = 0; a < kN; ++a) {
                const int part = ((a ^ swap) << 1) | odd;
                c[a] = make_uint4(0u, 0u, 0u, 0u);
                s[a] = v && from == kNoPage ? 0x7f7fu : 0u;       // V of a page outside the pool: NaN
                if (have) {
                    c[a] = *reinterpret_cast<const uint4 *>(blk + part * 16);
                    s[a] = *reinterpret_cast<const unsigned short *>(scl + part * 2);
                    // slots of absent nodes may hold anything: NaN scales among the draft nodes count as 0
                    if (first + t * kTileKeys + in >= sg.len) s[a] &= ~(((((s[a] & 0x7f7fu) + 0x0101u) >> 7) & 0x0101u) * 0xffu);
                }
            }
            __syncwarp();
            issue(t + 1);
            const uint32_t st = n & 1u;
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&empty[st]), ((n >> 1) & 1u) ^ 1u, abort_flag, &sh->word)) != 0;
            if (!ok) break;
#pragma unroll
            for (int a = 0; a < kN; ++a) {
                const uint32_t sb = e4m3x2_to_f16x2(s[a]);
                const uint32_t sc[2] = {__byte_perm(sb, sb, 0x1010), __byte_perm(sb, sb, 0x3232)};
                const uint32_t cw[4] = {c[a].x, c[a].y, c[a].z, c[a].w};
                unsigned char *dst = tiles + st * tile_bytes<D>() + (a ^ swap) * (128 * 128) + key * 128;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t h[4];
                    e2m1x8_to_f16x2(cw[k], h);
                    const uint32_t f = sc[k >> 1];
                    *reinterpret_cast<uint4 *>(dst + (((odd * 4 + k) ^ (key & 7)) * 16)) =
                        make_uint4(hmul2(h[0], f), hmul2(h[1], f), hmul2(h[2], f), hmul2(h[3], f));
                }
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&full[st]));
        }
        u += sg.span;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");         // nothing in flight when the block ends
}

// ------------------------------------------------------------------------------------- warp 3

template <int D>
__device__ __forceinline__ void tile_mma(const AttnParams &p, AttnRange r, TileSmem *sh, uint32_t tmem_any, uint32_t q_at,
                                         uint32_t k_at, uint32_t v_at)
{
    constexpr uint32_t kT = tile_bytes<D>();
    volatile int *abort_flag = &sh->abort;
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_any, 0);
    const uint32_t lead = elect_one();
    const uint64_t qdesc = umma_desc_k_sw128(q_at), kdesc = umma_desc_k_sw128(k_at), vdesc = umma_desc_mn_sw128(v_at, 128 * 128);
    uint32_t kst = 0, kpar = 0, vst = 0, vpar = 0;   // K and V stage in use, its phase
    uint32_t ppar[2] = {0, 0}, n_seg = 0;
    bool ok = __all_sync(0xffffffffu, *abort_flag == 0) != 0;
    auto wait = [&](uint64_t *bar, uint32_t parity) {
        return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity, abort_flag, &sh->word)) != 0;
    };
    // S of accumulator i; `opens`, `closes`: the first and the last to read the K tile
    auto issue_s = [&](int i, bool two) {
        const bool opens = !two || i == 0, closes = !two || i == 1;
        if (opens && !wait(&sh->kfull[kst], kpar)) return false;
        tc_fence_after();
        const uint64_t a = qdesc + (two ? i * (kT >> 4) : 0), b = kdesc + kst * (kT >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = (k >> 2) * ((128 * 128) >> 4) + 2 * (k & 3);
            tc_mma_f16_ss(lead, tmem + 128 * i, a + off, b + off, kIdescS, k != 0);
        }
        tc_commit_if(lead, smem_u32(&sh->sfull[i]));
        if (closes) {
            tc_commit_if(lead, smem_u32(&sh->kempty[kst]));
            kpar ^= kst;
            kst ^= 1u;
        }
        return true;
    };
    for (int64_t u = r.begin; u < r.end && ok;) {
        const TileSegment sg = tile_segment(p, sh, r, u);
        if (sg.tiles == 0) { u += sg.span; continue; }
        const int steps = __shfl_sync(0xffffffffu, sg.steps, 0);
        const bool two = __shfl_sync(0xffffffffu, (int)sg.two, 0) != 0;
        ok = wait(&sh->qfull, n_seg & 1u);
        ++n_seg;
        for (int s = 0; s < min(2, steps) && ok; ++s) ok = issue_s(s, two);
        for (int s = 0; s < steps && ok; ++s) {
            const int i = s & 1;
            const bool opens = !two || i == 0, closes = !two || i == 1;
            ok = (!opens || wait(&sh->vfull[vst], vpar)) && wait(&sh->pfull[i], ppar[i]);
            if (!ok) break;
            ppar[i] ^= 1u;
            tc_fence_after();
            const uint64_t b = vdesc + vst * (kT >> 4);
#pragma unroll
            for (int k = 0; k < kTileKeys / 16; ++k)
                tc_mma_f16_ts(lead, tmem + kColO + 128 * i, tmem + 128 * i + 8 * k, b + k * (2048 >> 4), idesc_o<D>(), k != 0 || s >= 2);
            tc_commit_if(lead, smem_u32(&sh->odone[i]));
            if (closes) {
                tc_commit_if(lead, smem_u32(&sh->vempty[vst]));
                vpar ^= vst;
                vst ^= 1u;
            }
            if (s + 2 < steps) ok = issue_s(i, two);
        }
        u += sg.span;
    }
    // all MMAs of this warp must retire before tensor memory is freed
    tc_commit_if(lead, smem_u32(&sh->drain));
    const long long t0 = clock64();
    while (!mbar_try_wait(smem_u32(&sh->drain), 0) && clock64() - t0 < kWaitCycles) {}
}

// ------------------------------------------------------------------------------------- warps 20-27

// 32 scores at tensor memory column `at`, masked where the tile reaches behind the committed tokens.
__device__ __forceinline__ void mask32(float *v, uint32_t see)
{
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] = (see >> k) & 1u ? v[k] : -INFINITY;
}
__device__ __forceinline__ float max32(const float *v)
{
    float a = fmaxf(v[0], v[1]), b = fmaxf(v[2], v[3]);
#pragma unroll
    for (int k = 4; k < 32; k += 4) { a = max3(a, v[k], v[k + 1]); b = max3(b, v[k + 2], v[k + 3]); }
    return fmaxf(a, b);
}
// P of 64 scores into 32 columns; adds them to l4.
__device__ __forceinline__ void exp64(float *v, float rs, float minus, uint32_t at, float (&l4)[4])
{
    uint32_t h[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        float &a = v[2 * k], &b = v[2 * k + 1];
        fma2(a, b, rs, minus);
        a = ex2(a);
        b = ex2(b);
        add2(l4[2 * (k & 1)], l4[2 * (k & 1) + 1], a, b);
        h[k] = f16x2_from(a, b);
    }
    tc_st32(at, h);
}

template <int D, int DT>
__device__ __forceinline__ void tile_softmax(const AttnParams &p, AttnRange r, TileSmem *sh, uint32_t tmem, unsigned char *q_tiles)
{
    const int tid = threadIdx.x - 640, warp = tid >> 5, lane = tid & 31;
    const int acc = warp >> 2, quarter = warp & 3;
    const int rr = quarter * 32 + lane;      // row of the accumulator, lane of tensor memory
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t sc = lanes + 128 * acc, oc = lanes + kColO;
    volatile int *abort_flag = &sh->abort;
    uint32_t n_s = 0;                        // S tiles of this accumulator so far
    int mask_b = -1, status = MARS_SEQ_OK;   // sequence whose masks are in shared memory, its status
    auto wait = [&](uint64_t *bar, uint32_t parity) {
        return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity, abort_flag, &sh->word)) != 0;
    };
    for (int64_t u = r.begin; u < r.end;) {
        const TileSegment sg = tile_segment(p, sh, r, u);
        if (sg.tiles == 0) { u += sg.span; continue; }
        const bool tree = p.parent != nullptr;
        const int words = (sg.n + 31) >> 5;
        const int row = (sg.two ? acc * 128 : 0) + rr;
        const int node = row < sg.rows ? attn_node(p, sg.row0 + row) : -1;
        const int head = sg.head * p.group + (node >= 0 ? sg.row0 + row - node * p.group : 0);
        const bool idle = row - lane >= sg.rows;             // no query row in this warp

        // ---- Q: this thread's row, scaled to fp16, into its swizzled tile
        float rs = 0.0f;                     // score scale of the row in log2 units
        if (sh->ok) {
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + 2 * (((int64_t)sg.b * p.N + (node >= 0 ? node : 0)) * p.q_row + head * p.q_head));
            uint4 w[D / 8];
#pragma unroll
            for (int c = 0; c < D / 8; ++c) w[c] = node >= 0 ? src[c] : make_uint4(0u, 0u, 0u, 0u);
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
            rs = row_log2(p, sg.head, up);
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
        if (tree && sg.b != mask_b) {
            mask_b = sg.b;
            status = attn_tree_masks(p, sg.b, sg.n, 0, sg.n, sh->par, sh->mask, words, sh->live, &sh->bad, tid, kSoftThreads,
                                     softmax_sync);
        }
        if (tid == 0 && p.status && status != MARS_SEQ_OK) atomicMax(p.status + sg.b, status);

        const uint32_t *mask = sh->mask + (tree && node >= 0 ? node : 0) * words;
        float mref = -INFINITY, l = 0.0f;    // reference maximum of the row in this accumulator, its sum
        float minus = 0.0f;
        bool far = false;                    // the row's scores are beyond the fused step
        const int my = !sh->ok ? 0 : sg.two ? sg.tiles : (sg.tiles + 1 - acc) >> 1;   // this accumulator's key tiles
        bool ok = true;
        for (int j = 0; j < my; ++j, ++n_s) {
            const int pos0 = sg.key0 + (sg.two ? j : 2 * j + acc) * kTileKeys;
            ok = wait(&sh->sfull[acc], n_s & 1u);
            if (!ok) break;
            if (idle) {
                // rows without a query: whatever S holds may stand for their P
                if (lane == 0) mbar_arrive(smem_u32(&sh->pfull[acc]));
                continue;
            }
            tc_fence_after();
            // the first 64 scores stay in registers, the others are read twice
            float v[64], x[32];
            float mx = -INFINITY;
            const bool edge = pos0 + kTileKeys > sg.len;
            tc_ld32_issue(sc, v);
            tc_ld32_issue(sc + 32, v + 32);
            tc_ld32_wait(v);
            tc_ld32_wait(v + 32);
            tc_ld32_issue(sc + 64, x);
            if (edge) {
                mask32(v, visible32(pos0, sg.len, node, tree, mask, words));
                mask32(v + 32, visible32(pos0 + 32, sg.len, node, tree, mask, words));
            }
            mx = fmaxf(max32(v), max32(v + 32));
            tc_ld32_wait(x);
            if (edge) mask32(x, visible32(pos0 + 64, sg.len, node, tree, mask, words));
            mx = fmaxf(mx, max32(x));
            tc_ld32_issue(sc + 96, x);
            tc_ld32_wait(x);
            if (edge) mask32(x, visible32(pos0 + 96, sg.len, node, tree, mask, words));
            mx = fmaxf(mx, max32(x));
            // the reference moves only when a score exceeds it by more than 2^8; the first tile just sets it
            const bool grow = (mx - mref) * rs > 8.0f;
            if (__any_sync(0xffffffffu, grow || far)) {
                const float f = grow ? ex2((mref - mx) * rs) : 1.0f;
                if (grow) {
                    mref = mx;
                    far = fabsf(mx * rs) > 4096.0f;
                    minus = far ? 7.0f : 7.0f - mx * rs;
                }
                l *= f;
                if (j > 0) {
                    // P V of the accumulator's tile before is complete: the S that was just read came after it
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        float y[16];
                        uint32_t z[8];
                        tc_ld16(oc + 128 * acc + c, y);
#pragma unroll
                        for (int k = 0; k < 8; ++k) z[k] = __float_as_uint(y[k] * f);
                        tc_st8(oc + 128 * acc + c, z);
#pragma unroll
                        for (int k = 0; k < 8; ++k) z[k] = __float_as_uint(y[8 + k] * f);
                        tc_st8(oc + 128 * acc + c + 8, z);
                    }
                }
                if (__any_sync(0xffffffffu, far)) {
                    const float less = far ? mref : 0.0f;
#pragma unroll
                    for (int k = 0; k < 64; ++k) v[k] -= less;
#pragma unroll 1
                    for (int c = 64; c < 128; c += 8) {
                        float y[8];
                        uint32_t z[8];
                        tc_ld8(sc + c, y);
#pragma unroll
                        for (int k = 0; k < 8; ++k) z[k] = __float_as_uint(y[k] - less);
                        tc_st8(sc + c, z);
                    }
                    tc_wait_st();
                }
            }
            // P = 2^((s - mref) * rs + 7), see mars_attention.cu; over columns of S that were read for good.  A fused
            // step per score, s * rs + minus with minus = 7 - mref * rs, off by 2^-13 at most below scores of 2^12; of
            // rows beyond that (`far`) mref is off S already
            float l4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            exp64(v, rs, minus, sc, l4);
            tc_ld32_issue(sc + 64, v);
            tc_ld32_issue(sc + 96, v + 32);
            tc_ld32_wait(v);
            tc_ld32_wait(v + 32);
            if (edge) {
                mask32(v, visible32(pos0 + 64, sg.len, node, tree, mask, words));
                mask32(v + 32, visible32(pos0 + 96, sg.len, node, tree, mask, words));
            }
            exp64(v, rs, minus, sc + 32, l4);
            l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->pfull[acc]));
        }
        if (ok && my > 0) ok = wait(&sh->odone[acc], (n_s - 1u) & 1u);
        sh->xm[acc][rr] = mref;
        sh->xl[acc][rr] = l;
        tc_fence_before();
        softmax_sync();                      // both accumulators complete
        tc_fence_after();
        if (tid == 0) sh->ok = *abort_flag == 0;
        softmax_sync();
        if (!sh->ok && tid == 0 && p.status) atomicMax(p.status + sg.b, MARS_SEQ_TIMEOUT);

        // ---- result of the segment: with two halves a thread has its row, else half of d of it
        const bool merge = !sg.two && sg.tiles > 1;
        float m = mref, sum = l, f0 = 1.0f, f1 = 0.0f;
        if (!sg.two) {
            m = sh->xm[0][rr];
            sum = sh->xl[0][rr];
            if (merge) {
                const float m1 = sh->xm[1][rr], mm = fmaxf(m, m1);
                f0 = m == -INFINITY ? 0.0f : ex2((m - mm) * rs);
                f1 = m1 == -INFINITY ? 0.0f : ex2((m1 - mm) * rs);
                sum = sum * f0 + sh->xl[1][rr] * f1;
                m = mm;
            }
        }
        if (!sh->ok) { m = -INFINITY; sum = NAN; }           // NaN rows here, and in whoever merges this
        const int d0 = sg.two ? 0 : acc * (D / 2), d1 = sg.two ? D : d0 + D / 2;
        const uint32_t o0 = oc + (sg.two ? 128 * acc : 0);
        const bool out_row = node >= 0 && (!tree || sh->live[node]);
        const int64_t out_at = out_row ? ((int64_t)sg.b * p.N + node) * p.out_row + (int64_t)head * p.out_head : 0;
        const float vscale = p.scales[p.kv.kv_heads + sg.head];
        constexpr int kF = tile_slot_floats<D>();
        if (!idle) {
            float *dst = p.partial + (int64_t)(2 * blockIdx.x + (u == r.begin ? 0 : 1)) * kF + row;
            const float norm = vscale / sum;
#pragma unroll 1
            for (int c = d0; c < d1; c += 32) {
                float v[32];
                tc_ld32_issue(o0 + c, v);
                tc_ld32_wait(v);
                if (!sh->ok) {               // products may still be in flight
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = 0.0f;
                } else if (merge) {
                    float x[32];
                    tc_ld32_issue(o0 + 128 + c, x);        // the second accumulator, same lanes
                    tc_ld32_wait(x);
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = v[k] * f0 + x[k] * f1;
                }
                if (!sg.whole) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) dst[(c + k) * TileShape::kMost] = v[k];
                } else if (out_row) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] *= norm;
#pragma unroll
                    for (int k = 0; k < 32; k += 8) store_out8<DT>(p.out, out_at + c + k, v + k);
                }
            }
            if (!sg.whole && d0 == 0) {
                dst[D * TileShape::kMost] = m;
                dst[(D + 1) * TileShape::kMost] = sum;
            }
        }
        if (!sg.whole) {
            const int c0 = sg.c0, c1 = sg.c1;
            __threadfence();
            softmax_sync();
            if (tid == 0) sh->last = atomicAdd(p.counters + c0, 1u) == (unsigned)(c1 - c0);
            softmax_sync();
            if (sh->last) {
                __threadfence();
                if (!idle) {
                    // block order, running maximum; 32 of a block's values at once
#pragma unroll 1
                    for (int c32 = d0; c32 < d1; c32 += 32) {
                        float o[32];
                        m = -INFINITY;
                        sum = 0.0f;
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = 0.0f;
#pragma unroll 2
                        for (int c = c0; c <= c1; ++c) {
                            const float *src = p.partial + (int64_t)(2 * c + (r.per * c >= sg.item ? 0 : 1)) * kF + row;
                            const float pm = __ldcg(src + D * TileShape::kMost), pl = __ldcg(src + (D + 1) * TileShape::kMost);
                            src += c32 * TileShape::kMost;
                            float x[32];
#pragma unroll
                            for (int k = 0; k < 32; ++k) x[k] = __ldcg(src + k * TileShape::kMost);
                            const float mm = fmaxf(m, pm);
                            const float a = m == -INFINITY ? 0.0f : ex2((m - mm) * rs), b = pm == -INFINITY ? 0.0f : ex2((pm - mm) * rs);
                            m = mm;
                            sum = sum * a + pl * b;
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = o[k] * a + x[k] * b;
                        }
                        if (out_row) {
                            const float norm = vscale / sum;
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] *= norm;
#pragma unroll
                            for (int k = 0; k < 32; k += 8) store_out8<DT>(p.out, out_at + c32 + k, o + k);
                        }
                    }
                }
                if (tid == 0) p.counters[c0] = 0u;
            }
        }
        tc_fence_before();
        softmax_sync();                   // masks, exchange arrays and accumulators are free for the next segment
        tc_fence_after();
        u += sg.span;
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
    TileSmem *sh = reinterpret_cast<TileSmem *>(ring + ring_bytes<D>());
    const int tid = threadIdx.x, warp = tid >> 5;

    const AttnRange r = attn_split<TileShape, kTileThreads>(p, &sh->seqs);
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->kfull[i]), 8);
            mbar_init(smem_u32(&sh->vfull[i]), 8);
            mbar_init(smem_u32(&sh->kempty[i]), 1);
            mbar_init(smem_u32(&sh->vempty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh->sfull[i]), 1);
            mbar_init(smem_u32(&sh->pfull[i]), 4);
            mbar_init(smem_u32(&sh->odone[i]), 1);
        }
        mbar_init(smem_u32(&sh->qfull), 8);
        mbar_init(smem_u32(&sh->drain), 1);
        sh->abort = blockIdx.x >= p.give_up;
        sh->ok = 1;
        sh->word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&sh->tmem)), "r"(kTmemAll) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;

    // registers go where a thread holds scores: 2 * 136 + 4 * 48 + 40 = 504 = 7 * 72 per lane at launch
    if (warp >= 20) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
        tile_softmax<D, DT>(p, r, sh, tmem, sm);
    } else if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        const int v = warp >= 4 + kUnpackWarps;
        tile_unpack_role<D>(p, r, sh, sm + (v ? 4 : 2) * kT, ring + (warp - 4) * slot_bytes<D>(), v, (warp - 4) & (kUnpackWarps - 1));
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 3) tile_mma<D>(p, r, sh, tmem, base, base + 2 * kT, base + 4 * kT);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemAll) : "memory");
    }
}

constexpr int kTileFewItems = kAttnSms / 2;

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

// Tiles of 256 rows share what is unpacked; of 128 rows there are twice as many, which a batch with
// fewer items than half of the SMs is better off with (lengths are not known here).  Measured, us with
// 128 / 256 rows, 60-node trees over 4000 tokens (8 KV heads): 1 tree 35 / 47, 4 trees 45 / 53, 10 trees
// 80 / 78, 16 trees 116 / 107, 48 trees 290 / 267; one prompt of 512 (4 KV heads) 20 / 24, of 2048 55 / 50.
mars_status_t attn_tile_launch(const AttnParams &q, int d, int dt, cudaStream_t st)
{
    AttnParams p = q;
    // Blocks come to a sequence in any order, so none of them may write OK: the statuses begin there, and each
    // block only raises what it has to say (OK < BAD_TREE < TIMEOUT)
    static_assert(MARS_SEQ_OK == 0 && MARS_SEQ_BAD_TREE < MARS_SEQ_TIMEOUT, "statuses in rising order");
    if (p.status && cudaMemsetAsync(p.status, 0, sizeof(int32_t) * p.B, st) != cudaSuccess) {
        (void)cudaGetLastError();
        return MARS_ERR_CUDA;
    }
    p.tile_rows = (int64_t)p.B * p.kv.kv_heads * (((int64_t)p.N * p.group + 255) / 256) < kTileFewItems ? 128 : 256;
    if (d == 128) return dt == MARS_BF16 ? tile_launch<128, MARS_BF16>(p, st) : tile_launch<128, MARS_FP16>(p, st);
    return dt == MARS_BF16 ? tile_launch<64, MARS_BF16>(p, st) : tile_launch<64, MARS_FP16>(p, st);
}

}  // namespace mars
