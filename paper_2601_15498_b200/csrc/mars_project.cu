// libmars: the output projection in 8-bit integers.
//
// y[m, v] = (sum_k q[m, k] w[v, k]) s[m] u[v] (+ b[v]), q and w signed 8-bit with |.| <= 127: the sum is an
// exact integer below 2^31 for K <= 2^17, so neither the order of the products nor a split of K changes a
// result, and the only roundings are the ones of the epilogue in fp32 and of the output type.
//
// The weights are the 256-row operand of tcgen05.mma.cta_group::2 (kind::i8, 128 rows in each block of a
// pair), up to 256 tokens the other: a few tokens then cost a narrow MMA and not a mostly empty one, and a
// warp's 32 lanes hold 32 neighbouring logits of a token, so stores are whole lines whatever the logits'
// alignment.  Tiles go round by round over the pairs, token tiles first, so that the pairs that run together
// share weight tiles in L2.  The tiles that are left for no whole round are cut along K: laid end to end in
// 128-byte blocks of K, every pair takes an equal contiguous range.  The holders of a cut tile leave their
// int32 sums in the workspace, and the last one to arrive adds them up.  Every holder arrives, one that gave up
// with a mark that makes the tile NaN, so the counters are zero after every call.
//   warp 0      TMA: 128 weight rows and half of the tokens per K block into a shared-memory ring
//   warp 1      allocates tensor memory, issues the MMAs (the leader's, for both blocks)
//   warps 2..17 epilogue, from one of two accumulators while the next tile is computed
// Waits on mbarriers are bounded; a block that gives up writes NaN where it owes logits, and a status word.
//
// Bound by reading the weights for few tokens (1 token, 151936 x 4096: 100 us, 6.2 TB/s; ranges of neighbouring tiles for
// each pair instead of rounds 102), by operands from L2 for many (64 KB per K block of a 256 x 256 tile, 0.43 us: 12 TB/s;
// tensor pipe 77 %), and by the power cap in long runs: 3840 x 151936 x 4096 takes 1.53 ms once and 1.77 ms for good, at
// 1350 MHz.  The epilogue has 16 warps because it has to hide under the MMAs: with 4 warps the same product took 2.30 ms,
// with 8 of them 1.61, and 2048 x 18944 x 1024 73 us against 46; it
// is what bounds short K (3840 x 151936 x 64 315 us, 3.7 TB/s of logits).  Sums of cut tiles added up by atomics instead of stores
// and loads were slower where tiles are few (256 x 4096 x 4096: 40 us against 25): int32 atomics run at 200 G/s.
#include "mars_fp32.cuh"
#include "mars_hooks.cuh"
#include "mars_stream.cuh"
#include "mars_tcgen05.cuh"
#include "mars_tensormap.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <climits>
#include <cmath>
#include <mutex>

#include "mars_scores.h"

namespace mars {

// ------------------------------------------------------------------------------ quantisation of rows

constexpr int kQzThreads = 256;
constexpr int kQzKeep = 4;             // 16-byte vectors per thread kept in registers between the two passes
constexpr int kQzMaxColumns = 1 << 17;
constexpr float kQzLeast = 0x1p-119f;  // rows whose largest magnitude is below this are zeros (127 * (1 / a) stays finite)
constexpr int kPjFp16 = 2;             // value of MARS_FP16 (mars_kv.h) in the dtype argument

template <int DT> struct QzElem;
template <> struct QzElem<MARS_BF16> {
    typedef unsigned short raw_t;
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float value(raw_t r) { return __uint_as_float((uint32_t)r << 16); }
};
template <> struct QzElem<kPjFp16> {
    typedef unsigned short raw_t;
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float value(raw_t r) { return __half2float(__ushort_as_half(r)); }
};
template <> struct QzElem<MARS_FP32> {
    typedef float raw_t;
    static constexpr int kVec = 4;
    static __device__ __forceinline__ float value(raw_t r) { return r; }
};

template <int DT>
struct QzVec {
    union {
        uint4 v;
        typename QzElem<DT>::raw_t e[QzElem<DT>::kVec];
    };
};

// Largest magnitude, NaN wherever there is one: the bits of |x| order like integers, NaN above infinity.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

__device__ __forceinline__ int quantise(float x, float r) { return __float2int_rn(x * r); }

// kGroup threads (a warp or the block) per row: one pass for the largest magnitude, one for the codes, the first
// kQzKeep vectors of a thread read once.  Bound by memory: 3840 rows of 4096 (bf16) 10 us, 4.7 TB/s; 20000 rows of 512
// 26.6 us by blocks, 7.8 by warps.
template <int DT, int kGroup>
__global__ void __launch_bounds__(kQzThreads) quantize_rows_kernel(const void *x, long long ldx, long long rows, int K, int8_t *q,
                                                                   long long ldq, float *scale)
{
    typedef QzElem<DT> E;
    __shared__ uint32_t s_max[kQzThreads / 32];
    pdl_begin();
    const int tid = threadIdx.x % kGroup;
    const long long row = (long long)blockIdx.x * (kQzThreads / kGroup) + threadIdx.x / kGroup;
    if (row >= rows) return;             // the same for a whole group
    const typename E::raw_t *src = (const typename E::raw_t *)x + row * ldx;
    int8_t *dst = q + row * ldq;
    const bool wide = ((uintptr_t)src & 15) == 0;        // the codes' rows always are 16-byte aligned
    const int nvec = wide ? K / E::kVec : 0;
    const uint4 *vsrc = (const uint4 *)src;
    QzVec<DT> keep[kQzKeep];
    uint32_t m = 0;
    int n = 0;
#pragma unroll
    for (int u = 0; u < kQzKeep; ++u)
        if (tid + u * kGroup < nvec) keep[u].v = vsrc[tid + u * kGroup];
#pragma unroll
    for (int u = 0; u < kQzKeep; ++u)
        if (tid + u * kGroup < nvec)
#pragma unroll
            for (int e = 0; e < E::kVec; ++e) m = max(m, magnitude(E::value(keep[u].e[e])));
    for (n = tid + kQzKeep * kGroup; n < nvec; n += kGroup) {
        QzVec<DT> t;
        t.v = vsrc[n];
#pragma unroll
        for (int e = 0; e < E::kVec; ++e) m = max(m, magnitude(E::value(t.e[e])));
    }
    for (int i = nvec * E::kVec + tid; i < K; i += kGroup) m = max(m, magnitude(E::value(src[i])));
    m = __reduce_max_sync(0xffffffffu, m);
    if constexpr (kGroup > 32) {
        if ((tid & 31) == 0) s_max[tid >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQzThreads / 32; ++w) m = max(m, s_max[w]);
    }
    const float a = __uint_as_float(m);
    const bool zero = a < kQzLeast, bad = !(a < INFINITY);
    const float r = zero || bad ? 0.0f : 127.0f * __frcp_rn(a);
    if (tid == 0) scale[row] = bad ? NAN : zero ? 0.0f : __fdiv_rn(a, 127.0f);

    auto code = [&](float v) { return bad ? 0 : quantise(v, r); };     // (infinity * 0 has no code)
    auto put = [&](int at, const QzVec<DT> &t) {
        uint32_t w[E::kVec / 4];
#pragma unroll
        for (int i = 0; i < E::kVec / 4; ++i) {
            w[i] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[i] |= (uint32_t)(code(E::value(t.e[4 * i + e])) & 0xff) << (8 * e);
        }
        if constexpr (E::kVec == 8) *reinterpret_cast<uint2 *>(dst + (size_t)at * 8) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(dst + (size_t)at * 4) = w[0];
    };
#pragma unroll
    for (int u = 0; u < kQzKeep; ++u)
        if (tid + u * kGroup < nvec) put(tid + u * kGroup, keep[u]);
    for (n = tid + kQzKeep * kGroup; n < nvec; n += kGroup) {
        QzVec<DT> t;
        t.v = vsrc[n];
        put(n, t);
    }
    for (int i = nvec * E::kVec + tid; i < K; i += kGroup) dst[i] = (int8_t)code(E::value(src[i]));
}

// ------------------------------------------------------------------------------ product

constexpr int kPjRows = 128;                // weight rows per block: tensor memory lanes
constexpr int kPjMaxTokens = 256;           // tokens per tile: columns of an accumulator
constexpr int kPjBK = 128;                  // bytes of K per block: one 128-byte swizzle row
constexpr int kPjWarps = 16;                 // epilogue warps: four per quarter of the lanes, hiding one another's latencies
constexpr int kPjGroup = 16;                 // tokens that an epilogue warp takes at a time
constexpr int kPjStride = kPjGroup * kPjWarps / 4;
constexpr int kPjThreads = 64 + 32 * kPjWarps;
constexpr int kPjMaxStages = 10;
constexpr int kPjPairs = 74;                // pairs of blocks that fill a B200
constexpr int kPjHolders = 4;               // parts that a cut tile goes to (or one more): 16 of them, 500 x 151936 x 4096
                                            // 367 us against 260, since one holder reads what all others wrote
constexpr uint32_t kPjABytes = kPjRows * kPjBK;
constexpr uint32_t kPjTmemCols = 512;
constexpr size_t kPjRing = 200 * 1024;
constexpr size_t kPjSmemBytes = kPjRing + 1024 /*align*/ + 256 /*barriers*/;
constexpr size_t kPjHead = MARS_PROJECT_COUNTER_BYTES;   // workspace: status word, then a counter per (pair, block, warp)
constexpr unsigned kPjLost = 1u << 16;      // in a counter of holders: one of them has no sums

struct ProjectParams {
    int M, V, kblocks;
    int tokens;                 // per tile, a multiple of 32
    int n_ttiles, n_tiles;      // token tiles, all tiles
    int stages;
    int rounds;                 // whole tiles per pair, dealt round by round
    long long per;              // K blocks of the remaining, cut tiles per pair
    const float *xs, *ws, *bias;
    void *out;
    long long ldo;
    unsigned *status, *counters;
    int *partial;               // [pair][2][tokens][2 * kPjRows]
    int packed;                 // bf16 logits may be written two at a time
    int give_up;                // pairs from this one on give up (test hook; the status is then cleared by the host)
};

// A pair's work: its part of the cut tiles first, so that what their holders wait for one another lies under
// the whole tiles that follow.
struct ProjectWalk {
    int round, pair, pairs;
    long long u, end;           // K blocks of the cut tiles
    __device__ __forceinline__ ProjectWalk(const ProjectParams &p)
    {
        round = 0;
        pair = (int)(blockIdx.x >> 1);
        pairs = (int)(gridDim.x >> 1);
        const long long total = (long long)(p.n_tiles - p.rounds * pairs) * p.kblocks;
        u = min(p.per * pair, total);
        end = min(u + p.per, total);
    }
};
struct ProjectSegment {
    int tile, k0, k1;           // K blocks k0 .. k1 - 1 of the tile
    int cut;                    // which of the cut tiles, -1: a whole one
};
__device__ __forceinline__ bool project_next(const ProjectParams &p, ProjectWalk &w, ProjectSegment &s)
{
    if (w.u < w.end) {
        s.cut = (int)(w.u / p.kblocks);
        s.tile = p.rounds * w.pairs + s.cut;
        s.k0 = (int)(w.u - (long long)s.cut * p.kblocks);
        s.k1 = (int)min((long long)p.kblocks, s.k0 + (w.end - w.u));
        if (s.k1 - s.k0 == p.kblocks) s.cut = -1;
        w.u += s.k1 - s.k0;
        return true;
    }
    if (w.round == p.rounds) return false;
    s.tile = w.round * w.pairs + w.pair;
    s.k0 = 0;
    s.k1 = p.kblocks;
    s.cut = -1;
    ++w.round;
    return true;
}

__device__ __forceinline__ void tc_mma_i8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

template <int DT>
__device__ __forceinline__ void put_logit(void *out, long long at, float y)
{
    if (DT == MARS_BF16) ((__nv_bfloat16 *)out)[at] = __float2bfloat16_rn(y);
    else ((float *)out)[at] = y;
}

// How the logits lie, out of the parameters' memory.
struct ProjectOut {
    char *out;
    long long ldo;              // bytes
    int V;
    bool packed;
};

// Logits of a group of tokens (n of them exist) from the sums of one weight row per lane.
template <int DT>
__device__ __forceinline__ void project_emit(const ProjectOut &o, const int (&sum)[kPjGroup], const float4 *xs, float u, float b,
                                             int v, int tok, int n)
{
    constexpr int es = DT == MARS_BF16 ? 2 : 4;
    const float2 u2 = make_float2(u, u), b2 = make_float2(b, b);
    float y[kPjGroup];
#pragma unroll
    for (int j = 0; j < kPjGroup; j += 4) {
        const float4 x = xs[j / 4];
        const float2 t = fma2(mul2(make_float2((float)sum[j], (float)sum[j + 1]), make_float2(x.x, x.y)), u2, b2);
        const float2 w = fma2(mul2(make_float2((float)sum[j + 2], (float)sum[j + 3]), make_float2(x.z, x.w)), u2, b2);
        y[j] = t.x; y[j + 1] = t.y; y[j + 2] = w.x; y[j + 3] = w.y;
    }
    if (DT == MARS_BF16 && o.packed) {
        // neighbouring lanes swap: the even one takes both rows of the even token, the odd one of the odd
        const int odd = threadIdx.x & 1;
        const uint32_t pick = odd ? 0x3276u : 0x5410u;
        uint32_t w[kPjGroup / 2];
#pragma unroll
        for (int j = 0; j < kPjGroup; j += 2) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j / 2]) : "f"(y[j + 1]), "f"(y[j]));
#pragma unroll
        for (int j = 0; j < kPjGroup / 2; ++j) w[j] = __byte_perm(w[j], __shfl_xor_sync(0xffffffffu, w[j], 1), pick);
        if (v >= o.V) return;
        char *dst = o.out + (tok + odd) * o.ldo + (long long)(v - odd) * es;
        if (n >= kPjGroup) {
#pragma unroll
            for (int j = 0; j < kPjGroup / 2; ++j, dst += 2 * o.ldo) *reinterpret_cast<uint32_t *>(dst) = w[j];
        } else {
#pragma unroll
            for (int j = 0; j < kPjGroup / 2; ++j, dst += 2 * o.ldo)
                if (2 * j + odd < n) *reinterpret_cast<uint32_t *>(dst) = w[j];
        }
        return;
    }
    if (v >= o.V) return;
    char *dst = o.out + tok * o.ldo + (long long)v * es;
    if (n >= kPjGroup) {
#pragma unroll
        for (int j = 0; j < kPjGroup; ++j, dst += o.ldo) put_logit<DT>(dst, 0, y[j]);
    } else {
#pragma unroll
        for (int j = 0; j < kPjGroup; ++j, dst += o.ldo)
            if (j < n) put_logit<DT>(dst, 0, y[j]);
    }
}

// Where a tile lies, and what its epilogue needs besides its sums: the scales of this lane's weight row and of two of
// the warp's tokens.
struct ProjectPlace {
    int v, tok0, n;             // the lane's weight row, the first of n tokens
    float u, b, x0, x1;
};

template <int DT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPjThreads, 1)
project_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const ProjectParams p)
{
    extern __shared__ unsigned char smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t stage_bytes = kPjABytes + (uint32_t)(p.tokens / 2) * kPjBK;
    const uint32_t bars = ring + (uint32_t)kPjRing;
    const uint32_t full0 = bars, empty0 = full0 + 8 * kPjMaxStages;
    const uint32_t tfull0 = empty0 + 8 * kPjMaxStages, tempty0 = tfull0 + 16, drain = tempty0 + 16;
    __shared__ uint32_t s_tmem_base;
    __shared__ int s_abort;
    __shared__ __align__(16) float s_xs[kPjWarps][kPjMaxTokens * 4 / kPjWarps];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();            // 0 = leader
    ProjectWalk walk(p);
    ProjectSegment s;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull0 + 8 * a, 1); mbar_init(tempty0 + 8 * a, 2 * kPjWarps); }
        mbar_init(drain, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&s_tmem_base)), "r"(kPjTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    __syncwarp();                  // (single lanes worked above; what follows is for whole warps)
    tc_fence_before();
    cluster_sync_all();            // both blocks' barriers exist before anything signals them
    tc_fence_after();
    const uint32_t tmem_base = s_tmem_base;
    volatile int *abort_flag = &s_abort;
    pdl_begin();                   // the set-up above lies under the predecessor's end
    const bool sound = walk.pair < p.give_up;
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0 && p.give_up == INT_MAX) *p.status = 0;      // (a wait gives up after a second at the earliest)
        if (!sound) atomicExch(p.status, (unsigned)MARS_SEQ_TIMEOUT);
    }

    if (warp == 0) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0;
            bool ok = sound;
            while (ok && project_next(p, walk, s)) {
                const int w_row = (s.tile / p.n_ttiles) * 2 * kPjRows + (int)rank * kPjRows;
                const int x_row = (s.tile % p.n_ttiles) * p.tokens + (int)rank * (p.tokens / 2);
                for (int kb = s.k0; kb < s.k1; ++kb) {
                    if (!mbar_wait(empty0 + 8 * stage, phase ^ 1u, abort_flag, p.status)) { ok = false; break; }
                    const uint32_t leader_full = mapa_shared(full0 + 8 * stage, 0);
                    if (rank == 0) mbar_expect_tx_cluster(leader_full, 2 * stage_bytes);
                    const uint32_t dst = ring + stage * stage_bytes;
                    tma_load_2d_pair(dst, &map_w, kb * kPjBK, w_row, leader_full);
                    tma_load_2d_pair(dst + kPjABytes, &map_x, kb * kPjBK, x_row, leader_full);
                    if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
                }
            }
            if (*abort_flag) {     // let copies already issued by this block land (bounded)
                const long long t0 = clock64();
                while (clock64() - t0 < 20000000ll) {}
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            // D int32, A and B signed 8-bit, both K-major, M = 256, N = tokens
            const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(p.tokens >> 3) << 17) |
                                   ((uint32_t)((2 * kPjRows) >> 4) << 24);
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
            bool ok = sound;
            while (ok && project_next(p, walk, s)) {
                if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1u, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + acc * kPjMaxTokens;
                for (int kb = s.k0; kb < s.k1; ++kb) {
                    if (!mbar_wait(full0 + 8 * stage, phase, abort_flag, p.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a_addr = ring + stage * stage_bytes;
                    const uint64_t adesc = umma_desc_k_sw128(a_addr);
                    const uint64_t bdesc = umma_desc_k_sw128(a_addr + kPjABytes);
#pragma unroll
                    for (int k = 0; k < kPjBK / 32; ++k)     // 32 bytes along K per step
                        tc_mma_i8_pair(d_tmem, adesc + 2 * k, bdesc + 2 * k, idesc, (kb != s.k0 || k != 0) ? 1u : 0u);
                    tc_commit_pair(empty0 + 8 * stage);      // frees the stage in both blocks
                    if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                tc_commit_pair(tfull0 + 8 * acc);            // accumulator complete in both blocks
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
            tc_commit_pair_local(drain);
        }
    } else {
        const int quarter = warp & 3, mine = warp - 2;       // TMEM lanes this warp may read
        const int first = kPjGroup * (mine >> 2);            // its groups: tokens first, first + kPjStride, ...
        const int in_tile = (int)rank * kPjRows + quarter * 32 + lane;
        const long long slot = (long long)p.tokens * 2 * kPjRows;
        float *xs = s_xs[mine];
        ProjectOut o;
        o.out = (char *)p.out; o.ldo = p.ldo * (DT == MARS_BF16 ? 2 : 4); o.V = p.V; o.packed = p.packed != 0;
        uint32_t acc = 0, acc_phase = 0;
        bool ok = sound;
        static_assert(kPjMaxTokens * 4 / kPjWarps == 64, "two scales of tokens per lane");
        const int t0 = first + (lane / kPjGroup) * kPjStride + lane % kPjGroup, t1 = t0 + 2 * kPjStride;
        auto place = [&](const ProjectSegment &g) {
            ProjectPlace r;
            const int row = g.tile / p.n_ttiles;
            r.v = row * 2 * kPjRows + in_tile;
            r.tok0 = (g.tile - row * p.n_ttiles) * p.tokens;
            r.n = min(p.tokens, p.M - r.tok0);
            r.u = r.v < p.V ? p.ws[r.v] : 0.0f;
            r.b = (p.bias && r.v < p.V) ? p.bias[r.v] : 0.0f;
            r.x0 = t0 < r.n ? p.xs[r.tok0 + t0] : 0.0f;
            r.x1 = t1 < r.n ? p.xs[r.tok0 + t1] : 0.0f;
            return r;
        };
        ProjectSegment next;
        bool more = project_next(p, walk, s);
        ProjectPlace now = {}, then = {};
        if (more) now = place(s);
        for (; more; s = next, now = then) {
            more = project_next(p, walk, next);
            if (more) then = place(next);                    // its scales are on their way while this tile is written
            const int v = now.v, tok0 = now.tok0, n = now.n;
            // lanes without a weight row leave a group early and have to be back before the next load from tensor memory
            const bool ragged = v - lane + 31 >= p.V;
            __syncwarp();
            xs[lane] = now.x0;
            xs[lane + 32] = now.x1;
            __syncwarp();
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, acc_phase, abort_flag, p.status));
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * kPjMaxTokens;
            const bool whole = s.cut < 0;
            bool last = true, lost = !ok;                    // a block that gave up owes NaN
            int c0 = 0, c1 = 0;                              // first and last pair that hold a part of the tile
            if (!whole) {
                const long long t0 = (long long)s.cut * p.kblocks;
                c0 = (int)(t0 / p.per);
                c1 = (int)((t0 + p.kblocks - 1) / p.per);
                // the first holder has the tile at its range's end, the others at their begin
                int *dst = p.partial + (2ll * walk.pair + (walk.pair == c0 ? 1 : 0)) * slot + in_tile;
#pragma unroll 1
                for (int c = first; c < n && ok; c += kPjStride) {
                    float x[kPjGroup];
                    tc_ld16(taddr + c, x);
#pragma unroll
                    for (int j = 0; j < kPjGroup; ++j) __stcg(dst + (c + j) * (2 * kPjRows), __float_as_int(x[j]));
                }
                // every lane's sums, then the warp's arrival: lane 0 orders both for all of them, before and behind
                __syncwarp();
                unsigned *counter = p.counters + (c0 * 2 + (int)rank) * kPjWarps + mine;
                unsigned seen = 0;
                if (lane == 0) {
                    __threadfence();
                    seen = atomicAdd(counter, ok ? 1u : kPjLost + 1u);   // also without sums: the others count on it
                    if (seen % kPjLost == (unsigned)(c1 - c0)) *counter = 0;     // as it was found: the workspace serves the next call
                    __threadfence();
                }
                __syncwarp();
                seen = __shfl_sync(0xffffffffu, seen, 0);
                last = seen % kPjLost == (unsigned)(c1 - c0);
                lost = lost || seen >= kPjLost;
            }
            // (two copies of the loop: sums that may still change would be moved between registers once more)
            if (lost) {
                if (last && v < p.V)
                    for (int c = first; c < n; c += kPjStride)
                        for (int j = 0; j < kPjGroup && c + j < n; ++j)
                            put_logit<DT>(p.out, (long long)(tok0 + c + j) * p.ldo + v, NAN);
                if (!ok) continue;
            } else if (whole) {
#pragma unroll 1
                for (int c = first, i = 0; c < n; c += kPjStride, i += kPjGroup) {
                    int sum[kPjGroup];
                    if (ragged) __syncwarp();
                    tc_ld16(taddr + c, reinterpret_cast<float (&)[kPjGroup]>(sum));
                    project_emit<DT>(o, sum, reinterpret_cast<const float4 *>(xs + i), now.u, now.b, v, tok0 + c, n - c);
                }
            } else if (last) {
#pragma unroll 1
                for (int c = first, i = 0; c < n; c += kPjStride, i += kPjGroup) {
                    int sum[kPjGroup];
                    if (ragged) __syncwarp();
                    tc_ld16(taddr + c, reinterpret_cast<float (&)[kPjGroup]>(sum));
                    // two holders' parts at a time: 32 loads of a line each in flight
                    const int *src = p.partial + in_tile + (long long)c * (2 * kPjRows);
#pragma unroll 1
                    for (int h = c0; h <= c1; h += 2) {
                        const int *part = src + (2ll * h + (h == c0 ? 1 : 0)) * slot, *other = src + 2ll * (h + 1) * slot;
                        const bool one = h != walk.pair, two = h + 1 <= c1 && h + 1 != walk.pair;
                        int x[kPjGroup], y[kPjGroup];
#pragma unroll
                        for (int j = 0; j < kPjGroup; ++j) {
                            x[j] = one ? __ldcg(part + j * (2 * kPjRows)) : 0;
                            y[j] = two ? __ldcg(other + j * (2 * kPjRows)) : 0;
                        }
#pragma unroll
                        for (int j = 0; j < kPjGroup; ++j) sum[j] += x[j] + y[j];
                    }
                    project_emit<DT>(o, sum, reinterpret_cast<const float4 *>(xs + i), now.u, now.b, v, tok0 + c, n - c);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_shared(tempty0 + 8 * acc, 0));   // leader's barrier
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
    }

    // The leader's MMAs write both blocks' TMEM: wait for them to retire, then meet the peer.
    if (warp == 1 && lane == 0 && rank == 0) {
        const long long t0 = clock64();
        while (!mbar_try_wait(drain, 0) && clock64() - t0 < kWaitCycles) {}
    }
    tc_fence_before();
    // Single lanes of warps 0 and 1 come from loops of their own, so every thread arrives for itself (a __syncwarp() here,
    // where 31 lanes wait for the whole kernel, made 3840 x 151936 x 4096 1.7 % slower).
    cluster_sync_threads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kPjTmemCols) : "memory");
    }
}

// How a product is cut up.  `tokens` per tile; `rounds` whole tiles for each of `pairs`; the remaining tiles are dealt in
// shares of `per` K blocks, which may end inside a tile, or (per = kblocks) as whole tiles to the first pairs.
struct ProjectPlan {
    int tokens, rounds, pairs;
    long long per;
};

static int project_widest(int64_t M) { return M < kPjMaxTokens ? (int)((M + 31) / 32 * 32) : kPjMaxTokens; }

// The plan of least time by this estimate, in us: a K block of a tile takes what its bytes take from L2, 43 a clock and
// SM (measured: 0.43 us at 256 tokens, 0.35 at 192, 12 TB/s in all; the MMA's own 2 clocks a token lie below), the whole
// no less than the weights take from HBM; a tile's epilogue 1 us and 1 us for 64 tokens; a cut tile 2 us and 1 us for 24
// tokens more, for the sums that its holders exchange.  Narrower tiles than the widest are tried where tiles are few.
// 333 x 32001 x 5000, us whole / cut: 192 tokens 64.5 / 69.8 (the plan's choice is the first, 30 of 74 pairs busy in its
// last round), 128 tokens 75.6 / 73.1, 96 tokens 86.1 / 91.8.
static ProjectPlan project_plan(int64_t M, int V, int K, int pairs)
{
    const int kb = (K + kPjBK - 1) / kPjBK;
    const int64_t rows = (V + 2 * kPjRows - 1) / (2 * kPjRows), fewest = (M + kPjMaxTokens - 1) / kPjMaxTokens;
    const int64_t most = rows * fewest >= 4 * pairs ? fewest : (M + 31) / 32 < 8 * fewest ? (M + 31) / 32 : 8 * fewest;
    const double hbm = (double)V * K / 6.3e6;
    ProjectPlan best = {};
    double least = 0;
    for (int64_t t = fewest; t <= most; ++t) {
        const int n = (int)(((M + t - 1) / t + 31) / 32 * 32), used = M < n ? (int)M : n;
        const int64_t tiles = rows * ((M + n - 1) / n);
        const double unit = fmax(2.0 * n, (kPjABytes + 64.0 * n) / 43) / 1900, edge = 1 + n / 64.0, join = 2 + used / 24.0;
        for (int cut = 0; cut < 2; ++cut) {
            ProjectPlan p;
            p.tokens = n;
            p.rounds = (int)(tiles / pairs);
            const int64_t rest = tiles - (int64_t)p.rounds * pairs, units = rest * kb;
            if (cut && rest == 0) continue;
            p.per = cut ? (units + pairs - 1) / pairs : kb;
            if (p.per < (kb + kPjHolders - 1) / kPjHolders) p.per = (kb + kPjHolders - 1) / kPjHolders;
            p.pairs = p.rounds ? pairs : (int)((units + p.per - 1) / p.per);
            const double work = ((double)p.rounds * kb + (rest ? (double)p.per : 0)) * unit;
            // in the last, ragged round few pairs pull
            const double stream = hbm * p.rounds * pairs / tiles + (rest ? p.per * 0.2 : 0);
            const double us = fmax(work, stream) + edge + (cut ? join : 0);
            if (least == 0 || us < least) { least = us; best = p; }
        }
    }
    return best;
}

static bool project_supported(int64_t M, int64_t V, int64_t K)
{
    return M >= 1 && V >= 1 && K >= 1 && M <= (1ll << 24) && V <= (1ll << 28) && K <= kQzMaxColumns &&
           ((M + 31) / 32) * ((V + 255) / 256) <= 0x7fffffffll;
}

// Resident pairs of a device, asked for once with that device current.
constexpr int kPjMaxDevices = 64;
static std::mutex g_pj_mu;
static int g_pj_pairs[kPjMaxDevices] = {};

static int project_pairs()
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kPjMaxDevices) return 0;
    std::lock_guard<std::mutex> lock(g_pj_mu);
    if (g_pj_pairs[dev]) return g_pj_pairs[dev];
    for (auto k : {(const void *)project_kernel<MARS_BF16>, (const void *)project_kernel<MARS_FP32>})
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPjSmemBytes) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * kPjPairs); cfg.blockDim = dim3(kPjThreads); cfg.dynamicSmemBytes = kPjSmemBytes;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, project_kernel<MARS_BF16>, &cfg) != cudaSuccess || n < 1) return 0;
    return g_pj_pairs[dev] = n < kPjPairs ? n : kPjPairs;
}

// The runtime's record of the error is cleared, so that no later call takes it for its own.
static mars_status_t project_failed()
{
    (void)cudaGetLastError();
    return MARS_ERR_CUDA;
}

}  // namespace mars

extern "C" {

mars_status_t mars_quantize_rows(const void *x, int64_t ldx, int dt, int64_t rows, int K, void *q, int64_t ldq, float *scale,
                                 void *cuda_stream)
{
    using namespace mars;
    if (!x || !q || !scale || rows < 1 || K < 1 || ldx < K || ldq < K) return MARS_ERR_INVALID_ARG;
    if (((uintptr_t)q & 15) || (ldq & 15)) return MARS_ERR_INVALID_ARG;
    if ((dt != MARS_BF16 && dt != MARS_FP32 && dt != kPjFp16) || K > kQzMaxColumns || rows > 0x7fffffffll)
        return MARS_ERR_UNSUPPORTED;
    if ((uintptr_t)x % (dt == MARS_FP32 ? 4 : 2)) return MARS_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool overlap = hook(kHookNoOverlap) == 0;
    // a warp holds rows of up to 32 * kQzKeep vectors in registers; longer ones get a block
    const bool warps = (int64_t)K * (dt == MARS_FP32 ? 4 : 2) <= 32 * kQzKeep * 16;
    void (*kernel)(const void *, long long, long long, int, int8_t *, long long, float *) =
        dt == MARS_BF16   ? (warps ? quantize_rows_kernel<MARS_BF16, 32> : quantize_rows_kernel<MARS_BF16, kQzThreads>)
        : dt == MARS_FP32 ? (warps ? quantize_rows_kernel<MARS_FP32, 32> : quantize_rows_kernel<MARS_FP32, kQzThreads>)
                          : (warps ? quantize_rows_kernel<kPjFp16, 32> : quantize_rows_kernel<kPjFp16, kQzThreads>);
    const int64_t blocks = warps ? (rows + kQzThreads / 32 - 1) / (kQzThreads / 32) : rows;
    const cudaError_t e = launch_pdl(overlap, kernel, dim3((unsigned)blocks), dim3(kQzThreads), 0, st, x, (long long)ldx,
                                     (long long)rows, K, (int8_t *)q, (long long)ldq, scale);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return MARS_ERR_CUDA; }
    return MARS_OK;
}

size_t mars_project_int8_workspace_bytes(int64_t M, int V, int K)
{
    if (!mars::project_supported(M, V, K)) return 0;
    return mars::kPjHead + (size_t)mars::kPjPairs * 2 * mars::project_widest(M) * (2 * mars::kPjRows) * sizeof(int);
}

mars_status_t mars_project_int8(const void *xq, int64_t ldx, const float *x_scale, const void *wq, int64_t ldw,
                                const float *w_scale, const float *bias, int64_t M, int V, int K, void *out, int64_t ldo,
                                mars_dtype_t dt, uint32_t flags, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace mars;
    if (!xq || !x_scale || !wq || !w_scale || !out || M < 1 || V < 1 || K < 1) return MARS_ERR_INVALID_ARG;
    if (ldx < K || ldw < K || ldo < V || (ldx & 15) || (ldw & 15)) return MARS_ERR_INVALID_ARG;
    if (((uintptr_t)xq & 15) || ((uintptr_t)wq & 15)) return MARS_ERR_INVALID_ARG;
    if ((dt != MARS_BF16 && dt != MARS_FP32) || (flags & ~MARS_COUNTERS_ZERO) || !project_supported(M, V, K))
        return MARS_ERR_UNSUPPORTED;
    if ((uintptr_t)out % (dt == MARS_BF16 ? 2 : 4)) return MARS_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < mars_project_int8_workspace_bytes(M, V, K))
        return MARS_ERR_WORKSPACE;
    ProjectParams p;
    p.M = (int)M; p.V = V;
    p.kblocks = (K + kPjBK - 1) / kPjBK;
    const int resident = project_pairs();
    if (resident < 1) return project_failed();
    const ProjectPlan plan = project_plan(M, V, K, resident);
    p.tokens = plan.tokens;
    p.n_ttiles = (int)((M + p.tokens - 1) / p.tokens);
    p.n_tiles = p.n_ttiles * ((V + 2 * kPjRows - 1) / (2 * kPjRows));
    p.rounds = plan.rounds;
    p.per = plan.per;
    const size_t stage = kPjABytes + (size_t)(p.tokens / 2) * kPjBK;
    p.stages = (int)(kPjRing / stage < (size_t)kPjMaxStages ? kPjRing / stage : kPjMaxStages);
    p.xs = x_scale; p.ws = w_scale; p.bias = bias; p.out = out; p.ldo = ldo;
    p.status = (unsigned *)workspace;
    p.counters = (unsigned *)((char *)workspace + 256);
    p.partial = (int *)((char *)workspace + kPjHead);
    p.packed = dt == MARS_BF16 && V % 2 == 0 && ldo % 2 == 0 && (uintptr_t)out % 4 == 0;
    CUtensorMap map_w, map_x;
    if (!tensor_map_2d(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, wq, (uint64_t)V, (uint64_t)K, (uint64_t)ldw, kPjRows, kPjBK) ||
        !tensor_map_2d(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, xq, (uint64_t)M, (uint64_t)K, (uint64_t)ldx, (uint32_t)p.tokens / 2, kPjBK))
        return project_failed();
    const int give_up = hook(kHookProjectGiveUp);
    p.give_up = give_up ? give_up - 1 : INT_MAX;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (give_up && cudaMemsetAsync(workspace, 0, 4, st) != cudaSuccess) return project_failed();
    if (!(flags & MARS_COUNTERS_ZERO) && cudaMemsetAsync(workspace, 0, kPjHead, st) != cudaSuccess) return project_failed();
    void (*kernel)(const CUtensorMap, const CUtensorMap, const ProjectParams) =
        dt == MARS_BF16 ? project_kernel<MARS_BF16> : project_kernel<MARS_FP32>;
    const cudaError_t e = launch_pdl(hook(kHookNoOverlap) == 0, kernel, dim3(2 * plan.pairs), dim3(kPjThreads), kPjSmemBytes, st,
                                     map_w, map_x, p);
    if (e != cudaSuccess) return project_failed();
    return MARS_OK;
}

}  // extern "C"
