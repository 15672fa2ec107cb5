// libmars: log probabilities of tokens with entropy and best alternatives, and their gradient.
//
// With m the row's largest logit, c = log2(e) / T and x_v = (z_v - m) c:
//   s = sum 2^x,  u = sum 2^x x,  ln p_v = (z_v - m) / T - ln s,  entropy = ln s - ln2 u / s,
// so one pass suffices: every thread keeps (m, s, u) of what it has seen and rescales them when its
// maximum rises by d (in units of x): s 2^d, (u + s d) 2^d.  Maxima are kept unscaled and differences of them
// taken before the scaling (after it where they pass fp32's range), so logits of any size keep their distances.  The gradient of g = sum_j grad_logprob_j and
// h = grad_entropy is, without the tokens' own terms,
//   -p (g + h (ln p + entropy)) / T = 2^x (a + b x),  a = -(g + h (entropy - ln s)) / (T s),  b = -h ln2 / (T s).
//
// Forward: bound by reading the logits, with the exponential unit (one 2^x a logit, 16 a clock and SM) and instruction
// issue close behind: bf16 rows 6.5 TB/s (3840 of 151936 in 180 us), fp32 6.8 (2000 in 179 us), with ten alternatives 205
// to 213 us.  Batches of 8 vectors a thread at 4 blocks per SM; also measured (before the last step, at 190 us / 34 us), us
// for 3840 rows / 512 rows: 4 vectors at 6 blocks 184 / 46, at 5 199 / 43; two buffers of 4 vectors at 4 blocks 193 / 35,
// at 3 194 / 38; two of 8 at 2 blocks 210 / 37.
// Gradient: bound by the copy, 6.1 TB/s (2048 rows of 151936 in 204 us).
#include "mars_fp32.cuh"
#include "mars_hooks.cuh"
#include "mars_topk_select.cuh"

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <cmath>
#include <type_traits>

#include "mars_scores.h"

namespace mars {

namespace cg = cooperative_groups;

constexpr int kScWarps = kTkThreads / 32;
constexpr int kScMaxSplit = 8;                  // blocks per row = blocks per cluster
constexpr float kLn2 = 0.693147180559945309f;

struct LogprobParams {
    const void *logits;
    long long ld, n;
    const int32_t *row_ids;     // or null
    int V, S, L;                // blocks per row, columns per block
    float temperature, c;       // c = log2(e) / temperature
    float reach;                // 200 / c
    const int32_t *tok;
    int J, k;
    float *logprob, *entropy, *stats;
    int32_t *top_id;
    float *top_logprob;
};

// Largest logit, sum of 2^x and sum of 2^x x over a set of logits, x = (z - ref) c.
struct Soft {
    float ref, sum, dot;
};

// The same set seen from a reference that lies d <= 0 below in units of x.
__device__ __forceinline__ void soft_move(Soft &a, float d)
{
    const float f = ex2f(d);
    a.dot = fmaf(a.sum, d, a.dot) * f;
    a.sum *= f;
}

// Distance of a reference to a larger one; 2^-1000 is 0, and 0 * 1000 is, unlike 0 * infinity.  A difference that passes
// fp32's range is one of opposite signs (or of an infinity), so scaling its parts first loses nothing.
__device__ __forceinline__ float soft_distance(float from, float to, float c)
{
    const float d = from - to;
    return from == to ? 0.0f : fmaxf(d > -INFINITY ? d * c : fmaf(from, c, -(to * c)), -1000.0f);
}

// The union of a warp's 32 sets, in all lanes: everybody moves to the largest reference, then plain sums.
__device__ __forceinline__ Soft soft_warp(Soft a, float c)
{
    const float r = tk_dec(__reduce_max_sync(0xffffffffu, tk_enc(a.ref)));
    soft_move(a, soft_distance(a.ref, r, c));
    a.ref = r;
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) {
        a.sum += __shfl_xor_sync(0xffffffffu, a.sum, m);
        a.dot += __shfl_xor_sync(0xffffffffu, a.dot, m);
    }
    return a;
}

// The fast form of x: one fma with R = fl(ref c), which gives x + d with d = ref c - R exactly (below 2^-4); a
// thread's sums are kept with that offset and freed of it at the end.  Logits far below the reference are raised
// to a floor where 2^x = 0 (x <= -199), so that -inf and NaN need no test of their own: 2^x x is then 0 and not
// 0 * infinity.  Where |ref c| passes 2^20, or no such floor exists in fp32, `fast` is false, d = 0, and the
// elements are taken one by one, their differences before the scaling.
struct SoftState {
    Soft a;
    float R, d;
    uint32_t floor;          // packed as the logits are
    bool fast;
};

// max(z, floor) of a packed word; the floor as a bf16 pair is rounded down.
template <int DT>
__device__ __forceinline__ uint32_t soft_floor_word(float z)
{
    const uint32_t b = __float_as_uint(z);
    if (DT == MARS_FP32) return b;
    const uint32_t h = (b >> 31 ? b + 0xffffu : b) >> 16;
    return h | h << 16;
}

template <int DT>
__device__ __forceinline__ void soft_reference(SoftState &t, float ref, float c, float reach)
{
    const float floor = ref - fmaxf(reach, fabsf(ref) * 0x1p-6f);
    t.a.ref = ref;
    t.R = ref * c;
    t.fast = floor > -3e38f && fabsf(t.R) <= 0x1p20f;
    t.d = t.fast ? fmaf(ref, c, -t.R) : 0.0f;
    t.floor = soft_floor_word<DT>(floor);
}

template <int DT>
__device__ __forceinline__ uint4 soft_clamp(uint4 v, uint32_t w)
{
    if constexpr (DT == MARS_BF16) return make_uint4(bmax2(v.x, w), bmax2(v.y, w), bmax2(v.z, w), bmax2(v.w, w));
    const float f = __uint_as_float(w);
    return make_uint4(__float_as_uint(fmaxf(__uint_as_float(v.x), f)), __float_as_uint(fmaxf(__uint_as_float(v.y), f)),
                      __float_as_uint(fmaxf(__uint_as_float(v.z), f)), __float_as_uint(fmaxf(__uint_as_float(v.w), f)));
}

// Terms of one logit against a reference that is at least as large; NaN counts as -inf.
__device__ __forceinline__ void soft_term(float z, float ref, float c, float &sum, float &dot)
{
    if (!(z > -INFINITY)) return;
    const float x = soft_distance(z, ref, c), e = ex2f(x);
    sum += e;
    dot = fmaf(e, x, dot);
}

// The elements of a batch one by one, read again; kept out of the fast path's registers.
template <int DT>
__device__ __noinline__ float2 soft_batch_slow(const uint4 *vbase, int v0, int nvec, int U, float ref, float c)
{
    typedef Elem<DT> E;
    float sum = 0.0f, dot = 0.0f;
    for (int u = 0; u < U; ++u) {
        const int vi = v0 + u * kTkThreads;
        for (int e = 0; vi < nvec && e < E::kVec; ++e) soft_term(E::scalar(vbase, vi * E::kVec + e), ref, c, sum, dot);
    }
    return make_float2(sum, dot);
}

// Something with the maximum m joins: the reference moves up to it.
template <int DT>
__device__ __forceinline__ void soft_rise(SoftState &t, float m, float c, float reach)
{
    if (!(m > t.a.ref)) return;
    const float move = soft_distance(t.a.ref, m, c), d = t.d;
    soft_reference<DT>(t, m, c, reach);
    soft_move(t.a, move + (t.d - d));
}

template <int DT>
__device__ __forceinline__ void soft_single(SoftState &t, float z, float c, float reach)
{
    soft_rise<DT>(t, z, c, reach);
    if (!(z > -INFINITY)) return;
    const float x = soft_distance(z, t.a.ref, c) + t.d, e = ex2f(x);
    t.a.sum += e;
    t.a.dot = fmaf(e, x, t.a.dot);
}

// The state's sums without the offset.
__device__ __forceinline__ Soft soft_free(SoftState t)
{
    soft_move(t.a, -t.d);
    return t.a;
}

// A batch with the maximum bm joins; vectors from `live` on (the same for all threads) are empty.  Skipping those of the
// last batch of 9.3 is worth 5 % of the time of rows of 151936 (bf16).
template <int DT, int U>
__device__ __forceinline__ void soft_batch(SoftState &t, const uint4 (&v)[U], float bm, float c, float reach, const uint4 *vbase,
                                           int v0, int nvec, int live)
{
    typedef Elem<DT> E;
    soft_rise<DT>(t, bm, c, reach);
    if (!t.fast) {
        if (!(fabsf(t.a.ref) < INFINITY)) return;          // nothing above -inf so far, or no softmax
        const float2 s = soft_batch_slow<DT>(vbase, v0, nvec, U, t.a.ref, c);
        t.a.sum += s.x;
        t.a.dot += s.y;
        return;
    }
    const float2 nr = make_float2(-t.R, -t.R), c2 = make_float2(c, c);
    float2 s0 = make_float2(0.0f, 0.0f), d0 = s0, s1 = s0, d1 = s0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u >= live) break;
        const uint4 w = soft_clamp<DT>(v[u], t.floor);
#pragma unroll
        for (int e = 0; e < E::kVec; e += 2) {
            const float2 x = fma2(make_float2(E::elem(w, e), E::elem(w, e + 1)), c2, nr);
            const float2 y = make_float2(ex2f(x.x), ex2f(x.y));
            if (e & 2) { s1 = add2(s1, y); d1 = fma2(y, x, d1); }
            else { s0 = add2(s0, y); d0 = fma2(y, x, d0); }
        }
    }
    s0 = add2(s0, s1);
    d0 = add2(d0, d1);
    t.a.sum += s0.x + s0.y;
    t.a.dot += d0.x + d0.y;
}

// A batch of vectors (-inf where there is none), and its maximum.
template <int DT, int U>
__device__ __forceinline__ void load_raw(const uint4 *vbase, int bi, int nvec, uint4 (&v)[U])
{
    const int v0 = bi * kTkThreads * U + threadIdx.x;
    if ((bi + 1) * kTkThreads * U <= nvec) {          // a full batch (the same for all threads) needs no guards
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = ld_stream(vbase + v0 + u * kTkThreads);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = v0 + u * kTkThreads < nvec ? ld_stream(vbase + v0 + u * kTkThreads) : Elem<DT>::neg_inf();
    }
}
template <int DT, int U>
__device__ __forceinline__ float batch_maximum(const uint4 (&v)[U])
{
    typedef Elem<DT> E;
    typename E::packed_t m = E::vred(v[0]);
#pragma unroll
    for (int u = 1; u < U; ++u) m = E::pmax(m, E::vred(v[u]));
    return E::to_float(m);
}

// The slice's best k.  While the slice streams by, a thread keeps the largest element that it has seen, the batch that
// it was in, and the largest of its other batches' maxima.  The k-th largest of the threads' maxima is a floor under the
// slice's k-th best, and what reaches it lies with the threads whose maximum does, k of them where values differ: the
// block reads that batch of those threads once more (a thread's whole column where another batch reaches the floor too),
// and what reaches the floor, some more than k elements, is ranked.  Order does not matter to it; slices in which very
// many elements tie at the floor are selected again by topk_slice_exact.
// (Whole columns for all of them cost 16 % more DRAM traffic: 3840 rows, k = 10, 221 us against 205.)
struct TopBest {
    float best, other;
    int batch;
    __device__ __forceinline__ void add(float bm, int bi)
    {
        other = fmaxf(other, fminf(best, bm));
        batch = bm > best ? bi : batch;
        best = fmaxf(best, bm);
    }
};

// The k best of n candidates, in order; empty ones (kNoId) lose against every other.
__device__ __forceinline__ void select_rank(const Cand *from, int n, int k, Cand *list)
{
    for (int i = threadIdx.x; i < n; i += kTkThreads) {
        const Cand c = from[i];
        int ahead = 0;
        for (int j = 0; j < n; ++j) ahead += beats(from[j].z, from[j].id, c.z, c.id) ? 1 : 0;
        if (ahead < k && c.id != kNoId) list[ahead] = c;
    }
}

struct TopSelect {
    __align__(8) Cand cand[kTkCap];
    __align__(8) Cand xlist[kScWarps * kTkMaxK];    // exact fallback only
    int xqn[kScWarps];
    unsigned xfloor;
    unsigned top[kScWarps * kTkMaxK];               // tk_enc of the warps' largest maxima
    unsigned floor;
    int n, hits, columns;
    int hit[kTkThreads];                            // thread + batch * kTkThreads
    int column[kTkThreads];

    __device__ __forceinline__ void append(float z, int id)
    {
        const int at = atomicAdd(&n, 1);
        if (at < kTkCap) { cand[at].z = z; cand[at].id = id; }
    }

    // A table of each warp's m largest maxima: its k-th largest never exceeds theirs, and falls short of it only
    // where one warp holds more than m of the block's k largest.  All threads, `best` the thread's maximum; the
    // caller synchronises before finish().
    __device__ __forceinline__ void table(int k, float best, Cand *list)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, m = min(k, 4 + (k >> 2));
        unsigned left = best > -INFINITY ? tk_enc(best) : 0u;
        for (int i = 0; i < m; ++i) {
            const unsigned most = __reduce_max_sync(0xffffffffu, left);
            const unsigned who = __ballot_sync(0xffffffffu, left == most);
            if (lane == __ffs(who) - 1) { top[warp * m + i] = most; left = 0u; }
        }
        if (tid == 0) { floor = 1u; hits = 0; columns = 0; }
        if (tid < kTkMaxK) { list[tid].z = -INFINITY; list[tid].id = kNoId; }
    }

    // All threads, after table(); list gets the slice's best k in order (the caller synchronises).
    template <int DT, int U>
    __device__ __forceinline__ void finish(int k, const TopBest &b, const char *rowp, int lo, int hi, int vlo, int nvec, Cand *list)
    {
        typedef Elem<DT> E;
        const int tid = threadIdx.x, nt = kScWarps * min(k, 4 + (k >> 2));
        const unsigned mine = b.best > -INFINITY ? tk_enc(b.best) : 0u;
        for (int i = tid; i < nt; i += kTkThreads) {
            const unsigned t = top[i];
            int ahead = 0;
            for (int j = 0; j < nt; ++j) ahead += (top[j] > t || (top[j] == t && j < i)) ? 1 : 0;
            if (ahead == k - 1 && t > 1u) floor = t;
        }
        __syncthreads();
        const float f = floor > 1u ? tk_dec(floor) : -INFINITY;
        if (mine >= floor) {
            if (b.other >= f && b.other > -INFINITY) column[atomicAdd(&columns, 1)] = tid;
            else hit[atomicAdd(&hits, 1)] = tid + b.batch * kTkThreads;
        }
        __syncthreads();
        const uint4 *vbase = (const uint4 *)(rowp + (size_t)vlo * E::kBytes);
        auto look = [&](int vi) {
            if (vi >= nvec) return;
            const uint4 v = ld_stream(vbase + vi);
            if (!(E::to_float(E::vred(v)) >= f)) return;
#pragma unroll
            for (int e = 0; e < E::kVec; ++e) {
                const float x = E::elem(v, e);
                if (x >= f && x > -INFINITY) append(x, vlo + vi * E::kVec + e);
            }
        };
        for (int i = tid; i < hits * U; i += kTkThreads) {
            const int h = hit[i / U];
            look((h / kTkThreads * U + i % U) * kTkThreads + h % kTkThreads);
        }
        for (int c = tid >> 5; c < columns; c += kScWarps)
            for (int vi = column[c] + (tid & 31) * kTkThreads; vi < nvec; vi += 32 * kTkThreads) look(vi);
        __syncthreads();
        const int found = n;
        if (found > kTkCap) {
            topk_slice_exact<DT>(rowp, lo, hi, k, list, cand, xlist, xqn, &xfloor);
            return;
        }
        select_rank(cand, found, k, list);
    }
};

// What a row comes to.
struct RowScore {
    float m, ln_s;
    bool ok;
};
__device__ __forceinline__ float row_logprob(const RowScore &r, float z, float temperature)
{
    if (!r.ok) return NAN;
    if (!(z > -INFINITY)) return -INFINITY;
    const float d = z - r.m;             // (beyond fp32's range: see soft_distance)
    return (d > -INFINITY ? __fdiv_rn(d, temperature) : __fdiv_rn(z, temperature) - __fdiv_rn(r.m, temperature)) - r.ln_s;
}

// Forward: a cluster of S blocks (S = 1: a block) streams one row, each block a contiguous slice; the
// block of rank 0 joins the slices' (m, s, u) and lists through distributed shared memory and writes.
// Four blocks per SM leave 64 registers; fp32 with alternatives spills 18 bytes at that.
template <int DT, bool TOP>
__global__ void __launch_bounds__(kTkThreads, 4) logprob_kernel(const LogprobParams p)
{
    typedef Elem<DT> E;
    constexpr int U = kTkU;
    struct Select { TopSelect s; };
    struct None {};
    __shared__ typename std::conditional<TOP, Select, None>::type s_sel;
    __shared__ Soft s_soft[kScWarps];
    __shared__ Soft s_block;
    __shared__ Cand s_list[kTkMaxK];
    __shared__ Cand s_all[TOP ? kTkMaxK * kScMaxSplit : 1];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, k = p.k;
    const long long out_row = blockIdx.x / p.S;
    const int rank = (int)(blockIdx.x - out_row * p.S);
    pdl_begin();
    const long long row = p.row_ids ? (long long)p.row_ids[out_row] : out_row;
    if (row < 0 || row >= p.n) {
        // absent: the whole cluster leaves here
        if (rank == 0) {
            for (int j = tid; j < p.J; j += kTkThreads) p.logprob[out_row * p.J + j] = 0.0f;
            for (int j = tid; j < k; j += kTkThreads) { p.top_id[out_row * k + j] = -1; p.top_logprob[out_row * k + j] = -INFINITY; }
            if (tid == 0) {
                if (p.entropy) p.entropy[out_row] = 0.0f;
                if (p.stats) { p.stats[2 * out_row] = -INFINITY; p.stats[2 * out_row + 1] = 0.0f; }
            }
        }
        return;
    }
    const int lo = min(rank * p.L, p.V), hi = min(p.V, lo + p.L);
    const char *rowp = (const char *)p.logits + (size_t)row * (size_t)p.ld * E::kBytes;
    const uintptr_t a0 = (uintptr_t)(rowp + (size_t)lo * E::kBytes);
    const int nhead = min((int)(((16 - (a0 & 15)) & 15) / E::kBytes), hi - lo);
    const int vlo = lo + nhead;
    const int nvec = (hi - vlo) / E::kVec;
    const int tlo = vlo + nvec * E::kVec;
    const int ntail = hi - tlo;
    const uint4 *vbase = (const uint4 *)(rowp + (size_t)vlo * E::kBytes);
    constexpr int kBatchVecs = kTkThreads * U;
    const float c = p.c;

    uint4 v[U];
    load_raw<DT, U>(vbase, 0, nvec, v);
    // the first tokens' logits are fetched beside the stream
    float zt = -INFINITY;
    bool inside = false;
    if (rank == 0 && tid < p.J) {
        const int t = p.tok[out_row * p.J + tid];
        inside = t >= 0 && t < p.V;
        if (inside) zt = E::scalar(rowp, t);
    }
    const float reach = p.reach;
    SoftState t;
    t.a.ref = -INFINITY; t.a.sum = 0.0f; t.a.dot = 0.0f; t.d = 0.0f; t.fast = false;
    TopBest best = {-INFINITY, -INFINITY, 0};
    if constexpr (TOP) {
        if (tid == 0) s_sel.s.n = 0;
        __syncthreads();
    }
    auto single = [&](int at) {
        const float z = E::scalar(rowp, at);
        soft_single<DT>(t, z, c, reach);
        if constexpr (TOP) { if (z > -INFINITY) s_sel.s.append(z, at); }
    };
    if (tid < nhead) single(lo + tid);
    if (tid < ntail) single(tlo + tid);
    const int nbatch = (nvec + kBatchVecs - 1) / kBatchVecs;
    auto batch = [&](const uint4 (&x)[U], int bi) {
        const float bm = batch_maximum<DT, U>(x);
        if constexpr (TOP) best.add(bm, bi);
        soft_batch<DT, U>(t, x, bm, c, reach, vbase, bi * kBatchVecs + tid, nvec, (nvec - bi * kBatchVecs + kTkThreads - 1) / kTkThreads);
    };
    for (int bi = 0; bi < nbatch; ++bi) {
        if (bi) load_raw<DT, U>(vbase, bi, nvec, v);
        batch(v, bi);
    }

    // ---- the block's (m, s, u) and list ----
    Soft a = soft_warp(soft_free(t), c);
    if (lane == 0) s_soft[warp] = a;
    if constexpr (TOP) s_sel.s.table(k, best.best, s_list);
    __syncthreads();
    if (warp == kScWarps - 1) {
        a.ref = -INFINITY; a.sum = 0.0f; a.dot = 0.0f;
        if (lane < kScWarps) a = s_soft[lane];
        a = soft_warp(a, c);
        if (lane == 0) s_block = a;
    }
    if constexpr (TOP) s_sel.s.template finish<DT, U>(k, best, rowp, lo, hi, vlo, nvec, s_list);

    // ---- the row's ----
    if (p.S > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (rank == 0) {
            if (warp == kScWarps - 1) {
                a.ref = -INFINITY; a.sum = 0.0f; a.dot = 0.0f;
                if (lane < p.S) a = *cluster.map_shared_rank(&s_block, lane);
                a = soft_warp(a, c);
                if (lane == 0) s_block = a;
            }
            if constexpr (TOP)
                if (tid < p.S * k) s_all[tid] = *(cluster.map_shared_rank(s_list, tid / k) + tid % k);
        }
        cluster.sync();          // the other blocks' shared memory was read
        if (rank != 0) return;
        if constexpr (TOP) {
            if (tid < k) { s_list[tid].z = -INFINITY; s_list[tid].id = kNoId; }
            __syncthreads();
            select_rank(s_all, p.S * k, k, s_list);
        }
    }
    __syncthreads();
    RowScore r;
    r.m = s_block.ref;
    r.ok = fabsf(r.m) < INFINITY;
    // s holds the largest logit's 1: what rounding leaves below it would make probabilities above 1
    const float s = fmaxf(s_block.sum, 1.0f);
    r.ln_s = logf(s);
    if (tid == 0) {
        if (p.entropy) p.entropy[out_row] = r.ok ? fmaxf(r.ln_s - kLn2 * (s_block.dot / s), 0.0f) : NAN;
        if (p.stats) { p.stats[2 * out_row] = r.m; p.stats[2 * out_row + 1] = r.ok ? s : NAN; }
    }
    for (int j = tid; j < p.J; j += kTkThreads) {
        if (j >= kTkThreads) {
            const int t = p.tok[out_row * p.J + j];
            inside = t >= 0 && t < p.V;
            zt = inside ? E::scalar(rowp, t) : 0.0f;
        }
        p.logprob[out_row * p.J + j] = inside ? row_logprob(r, zt, p.temperature) : 0.0f;
    }
    if constexpr (TOP) {
        if (warp == kScWarps - 1) {
            float *ov = p.top_logprob + out_row * k;
            int32_t *oi = p.top_id + out_row * k;
            const Cand mine = s_list[lane];              // ordered; entries from `found` on are empty
            const bool real = lane < k && mine.id != kNoId;
            if (real) { ov[lane] = row_logprob(r, mine.z, p.temperature); oi[lane] = mine.id; }
            const int found = __popc(__ballot_sync(0xffffffffu, real));
            __syncwarp();
            if (lane == 0 && found < k) {
                complete_row(ov, oi, found, k);
                if (!r.ok)
                    for (int j = found; j < k; ++j) ov[j] = NAN;
            }
        }
    }
}

struct GradParams {
    const void *logits;
    void *grad;
    long long ld, ld_grad;
    int V, S, L;                // blocks per row, columns per block
    float temperature, c, reach;
    const int32_t *tok;
    int J;
    const float *stats, *entropy, *g, *h;
};

// Vectors per thread at a time, blocks per SM.  2048 rows of 151936 (bf16), us: 2 at 6 blocks 205, at 5 209, at 7 216;
// 4 at 6 blocks 210, at 5 (47 registers) 217; 1 at 6 blocks 234, at 8 224.  Stores that stay in L2 228.  Six blocks leave
// 40 registers, at which 4 bytes are spilled.
constexpr int kGrU = 2, kGrBlocks = 6;

template <int DT>
__device__ __forceinline__ void store_scalar(void *row, int at, float x)
{
    if (DT == MARS_BF16) ((__nv_bfloat16 *)row)[at] = __float2bfloat16_rn(x);
    else ((float *)row)[at] = x;
}

// Gradient of one logit without the tokens' own terms, by the arithmetic of the vector form where there is one, so
// that a result does not depend on where its row begins.
struct GradLine {
    SoftState f;
    float m, c, a, b, fa, fb;        // a + b x, and the same line in x + d times 2^-d
};
template <int DT>
__device__ __forceinline__ float grad_term(float z, const GradLine &l)
{
    if (l.f.fast) {
        const float x = fmaf(fmaxf(z, DT == MARS_BF16 ? __uint_as_float(l.f.floor & 0xffff0000u) : __uint_as_float(l.f.floor)), l.c, -l.f.R);
        return ex2f(x) * fmaf(l.fb, x, l.fa);
    }
    if (!(z > -INFINITY)) return 0.0f;
    const float x = soft_distance(z, l.m, l.c);
    return ex2f(x) * fmaf(l.b, x, l.a);
}

// Backward: a block takes a contiguous piece of one row.
template <int DT>
__global__ void __launch_bounds__(kTkThreads, kGrBlocks) logprob_grad_kernel(const GradParams p)
{
    typedef Elem<DT> E;
    __shared__ float s_z[MARS_SCORES_MAX_TOKENS];
    pdl_begin();
    const int tid = threadIdx.x, lane = tid & 31;
    // the last rows first: a forward pass that came just before has left them in L2
    const long long block = (long long)gridDim.x - 1 - blockIdx.x, row = block / p.S;
    const int lo = min((int)(block - row * p.S) * p.L, p.V), hi = min(p.V, lo + p.L);
    const char *zrow = (const char *)p.logits + (size_t)row * (size_t)p.ld * E::kBytes;
    char *grow = (char *)p.grad + (size_t)row * (size_t)p.ld_grad * E::kBytes;
    const int32_t *tok = p.tok + row * p.J;
    const float *gj = p.g + row * p.J;
    const float m = p.stats[2 * row], s = p.stats[2 * row + 1], c = p.c;

    float g = 0.0f;
    for (int j = lane; j < p.J; j += 32) {
        const int t = tok[j];
        if (t >= 0 && t < p.V) g += gj[j];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) g += __shfl_xor_sync(0xffffffffu, g, o);
    const bool ok = fabsf(m) < INFINITY && s > 0.0f;
    const float ts = p.temperature * s;
    const float h = p.h ? p.h[row] : 0.0f;
    float a = -g, b = 0.0f;
    if (p.h) { a = -fmaf(h, p.entropy[row] - logf(s), g); b = -(h * kLn2); }
    const float as = a / s, bs = b / s;
    if (ts < INFINITY) { a /= ts; b /= ts; }
    else { a = as / p.temperature; b = bs / p.temperature; }             // T s passes fp32's range, the quotient need not
    if (!ok) { a = 0.0f; b = 0.0f; }
    // factors near the range's end (tiny T): 2^x (a + b x) is divided by T after the product, since infinity * 0 is no 0
    const bool far = !(fabsf(a) < 0x1p100f && fabsf(b) < 0x1p100f);
    if (far) { a = as; b = bs; }

    // the tokens' logits, before anything is overwritten
    bool hit = false;
    for (int j = tid; j < p.J; j += kTkThreads) {
        const int t = tok[j];
        if (t >= lo && t < hi) { s_z[j] = E::scalar(zrow, t); hit = true; }
    }
    hit = __syncthreads_or(hit);

    GradLine line;
    soft_reference<DT>(line.f, m, c, p.reach);
    if (far) { line.f.fast = false; line.f.d = 0.0f; }
    const SoftState &f = line.f;
    const float fd = ex2f(-f.d);
    line.m = m; line.c = c; line.a = a; line.b = b;
    line.fa = fd * fmaf(-b, f.d, a); line.fb = fd * b;
    const uintptr_t a0 = (uintptr_t)(zrow + (size_t)lo * E::kBytes), b0 = (uintptr_t)(grow + (size_t)lo * E::kBytes);
    if (((a0 ^ b0) & 15) || !ok || !f.fast) {
        // rows that lie differently on 16-byte boundaries, and rows without fast form: one by one.  The former are 7 of 8
        // bf16 rows where logits of odd stride get a dense gradient: 2048 rows of 151936 756 us, 1000 fp32 rows 385; with
        // the logits' own stride 209 and 199
        for (int i = lo + tid; i < hi; i += kTkThreads)
            store_scalar<DT>(grow, i, ok ? grad_term<DT>(E::scalar(zrow, i), line) / (far ? p.temperature : 1.0f) : 0.0f);
    } else {
        const int nhead = min((int)(((16 - (a0 & 15)) & 15) / E::kBytes), hi - lo);
        const int vlo = lo + nhead, nvec = (hi - vlo) / E::kVec, tlo = vlo + nvec * E::kVec, ntail = hi - tlo;
        if (tid < nhead) store_scalar<DT>(grow, lo + tid, grad_term<DT>(E::scalar(zrow, lo + tid), line));
        if (tid < ntail) store_scalar<DT>(grow, tlo + tid, grad_term<DT>(E::scalar(zrow, tlo + tid), line));
        const uint4 *src = (const uint4 *)(zrow + (size_t)vlo * E::kBytes);
        uint4 *dst = (uint4 *)(grow + (size_t)vlo * E::kBytes);
        const float2 nr = make_float2(-f.R, -f.R), c2 = make_float2(c, c), a2 = make_float2(line.fa, line.fa), b2 = make_float2(line.fb, line.fb);
        auto one = [&](const uint4 &v) {
            const uint4 t = soft_clamp<DT>(v, f.floor);
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < E::kVec; e += 2) {
                const float2 x = fma2(make_float2(E::elem(t, e), E::elem(t, e + 1)), c2, nr);
                const float2 y = mul2(make_float2(ex2f(x.x), ex2f(x.y)), fma2(b2, x, a2));
                if constexpr (DT == MARS_BF16) {
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[e / 2]) : "f"(y.y), "f"(y.x));
                } else {
                    o[e] = __float_as_uint(y.x);
                    o[e + 1] = __float_as_uint(y.y);
                }
            }
            return make_uint4(o[0], o[1], o[2], o[3]);
        };
        int v0 = tid;
        // (plain loads: the gradient may overwrite the logits; stores that leave L2 to them)
        for (; v0 + (kGrU - 1) * kTkThreads < nvec; v0 += kGrU * kTkThreads) {
            uint4 v[kGrU];
#pragma unroll
            for (int u = 0; u < kGrU; ++u) v[u] = src[v0 + u * kTkThreads];
#pragma unroll
            for (int u = 0; u < kGrU; ++u) __stcs(dst + v0 + u * kTkThreads, one(v[u]));
        }
        for (; v0 < nvec; v0 += kTkThreads) __stcs(dst + v0, one(src[v0]));
    }
    if (!hit) return;
    __syncthreads();
    // a token's own logit: everything that names it, in order, by the first place that does
    for (int j = tid; j < p.J; j += kTkThreads) {
        const int t = tok[j];
        if (t < lo || t >= hi || !ok) continue;
        bool first = true;
        for (int i = 0; i < j; ++i) first &= tok[i] != t;
        if (!first) continue;
        float own = 0.0f;
        for (int i = j; i < p.J; ++i) own += tok[i] == t ? gj[i] : 0.0f;
        const float term = grad_term<DT>(s_z[j], line);
        store_scalar<DT>(grow, t, far ? (term + own) / p.temperature : term + own / p.temperature);
    }
}

static bool scores_sizes_ok(int64_t rows, int V) { return rows <= (1ll << 27) && V <= (1 << 30); }

// Blocks per row: rows are split while the GPU is not full.  How full it has to be depends on what is left of a slice,
// since a block also takes some microseconds whatever its slice.  us split into 1 / 2 / 4 / 8 (bf16): 8 rows of 151936
// 12.0 / 8.2 / 5.8 / 4.8, 60 rows 16.4 / 11.4 / 10.4 / 9.3, 120 rows 21.9 / 19.7 / 16.9 / 21.8, 300 rows 29.6 / 25.0 /
// 25.1 / 30.6, 700 rows 44.8 / 42.8 / 48.2 / 63.2, 1000 rows 61.6 / 69.2; 200 rows of 32000 7.6 / 7.9 / 9.3 / 12.8.  Joining
// eight lists of many alternatives costs more than the split gains: 60 rows with 32 of them, split into 4 / 8, 18.4 / 24.7.
static int logprob_split(int64_t rows, int V, int es, int k)
{
    const int force = hook(kHookForceSplit);
    int S = 1;
    for (; S < kScMaxSplit; S *= 2) {
        const int64_t blocks = rows * S * 2, slice = (int64_t)V * es / (S * 2);
        const bool more = force >= 1 ? 2 * S <= force
                                     : slice >= 24 * 1024 && blocks <= 148 * (slice >= 128 * 1024 ? 8 : slice >= 64 * 1024 || k <= 16 ? 4 : 2);
        if (!more) break;
    }
    return S;
}

static int slice_columns(int V, int S)
{
    const long long L = ((long long)V + S - 1) / S;
    return (int)((L + 15) / 16 * 16);
}

template <int DT>
static cudaError_t logprob_launch(const LogprobParams &p, unsigned rows, cudaStream_t st)
{
    void (*kernel)(const LogprobParams) = p.k ? logprob_kernel<DT, true> : logprob_kernel<DT, false>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(rows * (unsigned)p.S); cfg.blockDim = dim3(kTkThreads); cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = hook(kHookNoOverlap) == 0 ? 1 : 0;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)p.S; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = p.S > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace mars

extern "C" {

mars_status_t mars_token_logprobs(const void *logits, int64_t ld, mars_dtype_t dt, int64_t n, const int32_t *row_ids,
                                  int64_t rows, int V, float temperature, const int32_t *tok, int J, int k,
                                  float *logprob, float *entropy, float *stats, int32_t *top_id, float *top_logprob,
                                  void *cuda_stream)
{
    using namespace mars;
    if (!logits || rows < 1 || n < 1 || V < 1 || ld < V || J < 0 || k < 0 || k > V) return MARS_ERR_INVALID_ARG;
    if (!row_ids && rows != n) return MARS_ERR_INVALID_ARG;
    if (!(temperature > 0.0f) || temperature > 3.40282347e38f) return MARS_ERR_INVALID_ARG;
    if (J > 0 && (!tok || !logprob)) return MARS_ERR_INVALID_ARG;
    if (k > 0 && (!top_id || !top_logprob)) return MARS_ERR_INVALID_ARG;
    if (J > MARS_SCORES_MAX_TOKENS || k > MARS_SCORES_MAX_TOP) return MARS_ERR_UNSUPPORTED;
    if ((dt != MARS_BF16 && dt != MARS_FP32) || !scores_sizes_ok(rows, V)) return MARS_ERR_UNSUPPORTED;
    const int es = dt == MARS_BF16 ? 2 : 4;
    if ((uintptr_t)logits % es) return MARS_ERR_INVALID_ARG;
    LogprobParams p;
    p.logits = logits; p.ld = ld; p.n = n; p.row_ids = row_ids; p.V = V;
    p.S = logprob_split(rows, V, es, k);
    p.L = slice_columns(V, p.S);
    p.temperature = temperature;
    p.c = (float)(1.4426950408889634 / (double)temperature);
    if (!(p.c > 0.0f) || p.c > 3.40282347e38f) return MARS_ERR_UNSUPPORTED;
    p.reach = 200.0f / p.c;
    p.tok = tok; p.J = J; p.k = k;
    p.logprob = logprob; p.entropy = entropy; p.stats = stats; p.top_id = top_id; p.top_logprob = top_logprob;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = dt == MARS_BF16 ? logprob_launch<MARS_BF16>(p, (unsigned)rows, st)
                                          : logprob_launch<MARS_FP32>(p, (unsigned)rows, st);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return MARS_ERR_CUDA; }
    return MARS_OK;
}

mars_status_t mars_token_logprobs_backward(const void *logits, int64_t ld, mars_dtype_t dt, int64_t rows, int V,
                                           float temperature, const int32_t *tok, int J, const float *stats,
                                           const float *entropy, const float *grad_logprob, const float *grad_entropy,
                                           void *grad, int64_t ld_grad, void *cuda_stream)
{
    using namespace mars;
    if (!logits || !grad || !tok || !stats || !grad_logprob || (grad_entropy && !entropy)) return MARS_ERR_INVALID_ARG;
    if (rows < 1 || V < 1 || ld < V || ld_grad < V || J < 1) return MARS_ERR_INVALID_ARG;
    if (!(temperature > 0.0f) || temperature > 3.40282347e38f) return MARS_ERR_INVALID_ARG;
    if (J > MARS_SCORES_MAX_TOKENS || (dt != MARS_BF16 && dt != MARS_FP32) || !scores_sizes_ok(rows, V))
        return MARS_ERR_UNSUPPORTED;
    const int es = dt == MARS_BF16 ? 2 : 4;
    if ((uintptr_t)logits % es || (uintptr_t)grad % es) return MARS_ERR_INVALID_ARG;
    if (grad == logits && ld_grad != ld) return MARS_ERR_INVALID_ARG;
    GradParams p;
    p.logits = logits; p.grad = grad; p.ld = ld; p.ld_grad = ld_grad; p.V = V;
    // Batches per block: each block spends about 300 instructions a thread before its first logit, so as many as leave
    // the GPU full, up to eight (2048 rows of 151936: 205 us; 16 and 32 batches 209 and 211).
    const int64_t batch = kTkThreads * kGrU * 16 / es, batches = (V + batch - 1) / batch;
    int64_t each = rows * batches / (148 * 8);
    each = each < 1 ? 1 : each > 8 ? 8 : each;
    p.S = (int)((batches + each - 1) / each);
    p.L = slice_columns(V, p.S);
    if (rows * p.S > 0x7fffffffll) return MARS_ERR_UNSUPPORTED;
    p.temperature = temperature;
    p.c = (float)(1.4426950408889634 / (double)temperature);
    if (!(p.c > 0.0f) || p.c > 3.40282347e38f) return MARS_ERR_UNSUPPORTED;
    p.reach = 200.0f / p.c;
    p.tok = tok; p.J = J; p.stats = stats; p.entropy = entropy; p.g = grad_logprob; p.h = grad_entropy;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool overlap = hook(kHookNoOverlap) == 0;
    const dim3 grid((unsigned)(rows * p.S)), block(kTkThreads);
    const cudaError_t e = dt == MARS_BF16 ? launch_pdl(overlap, logprob_grad_kernel<MARS_BF16>, grid, block, 0, st, p)
                                          : launch_pdl(overlap, logprob_grad_kernel<MARS_FP32>, grid, block, 0, st, p);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return MARS_ERR_CUDA; }
    return MARS_OK;
}

}  // extern "C"
