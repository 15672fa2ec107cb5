// libmars: log probabilities of tokens with entropy and best alternatives, and their gradient.
//
// With m the row's largest logit, c = log2(e) / T and x_v = (z_v - m) c:
//   s = sum 2^x,  u = sum 2^x x,  ln p_v = (z_v - m) / T - ln s,  entropy = ln s - ln2 u / s,
// so one pass suffices: every thread keeps (m, s, u) of what it has seen and rescales them when its
// maximum rises by d (in units of x): s 2^d, (u + s d) 2^d.  Differences are taken before the scaling,
// so logits of any size keep their exact distances.  The gradient of g = sum_j grad_logprob_j and
// h = grad_entropy is, without the tokens' own terms,
//   -p (g + h (ln p + entropy)) / T = 2^x (a + b x),  a = -(g + h (entropy - ln s)) / (T s),  b = -h ln2 / (T s).
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

constexpr int kScMaxSplit = 8;                  // blocks per row = blocks per cluster
constexpr int kScTargetBlocks = 148 * 4;        // resident blocks of the forward kernel
constexpr int kScMinSliceBytes = 24 * 1024;     // three quarters of a batch of one block
constexpr float kLn2 = 0.693147180559945309f;

struct LogprobParams {
    const void *logits;
    long long ld, n;
    const int32_t *row_ids;     // or null
    int V, S, L;                // blocks per row, columns per block
    float temperature, c;       // c = log2(e) / temperature
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

// Distance of a reference to a larger one; 2^-1000 is 0, and 0 * 1000 is, unlike 0 * infinity.
__device__ __forceinline__ float soft_distance(float from, float to, float c)
{
    return from == to ? 0.0f : fmaxf((from - to) * c, -1000.0f);
}

__device__ __forceinline__ Soft soft_union(Soft a, Soft b, float c)
{
    const float r = fmaxf(a.ref, b.ref);
    soft_move(a, soft_distance(a.ref, r, c));
    soft_move(b, soft_distance(b.ref, r, c));
    Soft o;
    o.ref = r; o.sum = a.sum + b.sum; o.dot = a.dot + b.dot;
    return o;
}

__device__ __forceinline__ Soft soft_shfl_xor(const Soft &a, int m)
{
    Soft o;
    o.ref = __shfl_xor_sync(0xffffffffu, a.ref, m);
    o.sum = __shfl_xor_sync(0xffffffffu, a.sum, m);
    o.dot = __shfl_xor_sync(0xffffffffu, a.dot, m);
    return o;
}

// Logits this far below the reference have 2^x = 0 (x <= -200) and are raised to it, so that -inf and NaN
// need no test of their own: 2^x x is then 0 and not 0 * infinity.  Where a reference is so large, or c so
// extreme, that no such level exists in fp32, `ok` is false and the elements are taken one by one.
struct SoftFloor {
    float z;
    bool ok;
};
__device__ __forceinline__ SoftFloor soft_floor(float ref, float c)
{
    SoftFloor f;
    f.z = ref - fmaxf(200.0f / c, fabsf(ref) * 0x1p-6f);
    f.ok = f.z > -3e38f && fabsf(ref) * c < 1e38f;
    return f;
}

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

__device__ __forceinline__ void soft_add(Soft &a, float z, float c)
{
    if (z > a.ref) { soft_move(a, soft_distance(a.ref, z, c)); a.ref = z; }
    soft_term(z, a.ref, c, a.sum, a.dot);
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

// A batch with the maximum bm joins.
template <int DT, int U>
__device__ __forceinline__ void soft_batch(Soft &a, const uint4 (&v)[U], float bm, float c, const uint4 *vbase, int v0, int nvec)
{
    typedef Elem<DT> E;
    if (bm > a.ref) { soft_move(a, soft_distance(a.ref, bm, c)); a.ref = bm; }
    if (!(fabsf(a.ref) < INFINITY)) return;          // nothing above -inf so far, or no softmax
    const SoftFloor f = soft_floor(a.ref, c);
    if (!f.ok) {
        const float2 t = soft_batch_slow<DT>(vbase, v0, nvec, U, a.ref, c);
        a.sum += t.x;
        a.dot += t.y;
        return;
    }
    const uint32_t w = soft_floor_word<DT>(f.z);
    const float2 nref = make_float2(-a.ref, -a.ref), c2 = make_float2(c, c);
    float2 s0 = make_float2(0.0f, 0.0f), d0 = s0, s1 = s0, d1 = s0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint4 t = soft_clamp<DT>(v[u], w);
#pragma unroll
        for (int e = 0; e < E::kVec; e += 2) {
            const float2 x = mul2(add2(make_float2(E::elem(t, e), E::elem(t, e + 1)), nref), c2);
            const float2 y = make_float2(ex2f(x.x), ex2f(x.y));
            if (e & 2) { s1 = add2(s1, y); d1 = fma2(y, x, d1); }
            else { s0 = add2(s0, y); d0 = fma2(y, x, d0); }
        }
    }
    s0 = add2(s0, s1);
    d0 = add2(d0, d1);
    a.sum += s0.x + s0.y;
    a.dot += d0.x + d0.y;
}

// What a row comes to.
struct RowScore {
    float m, ln_s;
    bool ok;
};
__device__ __forceinline__ float row_logprob(const RowScore &r, float z, float temperature)
{
    if (!r.ok) return NAN;
    return (z > -INFINITY) ? __fdiv_rn(z - r.m, temperature) - r.ln_s : -INFINITY;
}

// Forward: a cluster of S blocks (S = 1: a block) streams one row, each block a contiguous slice; the
// block of rank 0 joins the slices' (m, s, u) and lists through distributed shared memory and writes.
template <int DT, int U, int MINB, bool TOP>
__global__ void __launch_bounds__(kTkThreads, MINB) logprob_kernel(const LogprobParams p)
{
    typedef Elem<DT> E;
    struct Select { TopkSelect s; };
    struct None {};
    __shared__ typename std::conditional<TOP, Select, None>::type s_sel;
    __shared__ Soft s_soft[kTkThreads / 32];
    __shared__ Soft s_block;
    __shared__ RowScore s_row;
    __shared__ Cand s_list[TOP ? kTkMaxK : 1];
    __shared__ Cand s_all[TOP ? kTkMaxK * kScMaxSplit : 1];
    __shared__ int s_found;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, k = p.k;
    const long long out_row = blockIdx.x / p.S;
    const int rank = (int)(blockIdx.x - out_row * p.S);
    pdl_launch_dependents();
    pdl_wait();
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
    const int nfull = nvec / kBatchVecs;
    const float c = p.c;

    uint4 v[U];
    typename E::packed_t q[U];
    float bm = (nfull > 0) ? load_batch<DT, U, false>(vbase, tid, nvec, v, q)
                           : load_batch<DT, U, true>(vbase, tid, nvec, v, q);
    // the first tokens' logits are fetched beside the stream
    float zt = -INFINITY;
    bool inside = false;
    if (rank == 0 && tid < p.J) {
        const int t = p.tok[out_row * p.J + tid];
        inside = t >= 0 && t < p.V;
        if (inside) zt = E::scalar(rowp, t);
    }
    Soft a;
    a.ref = -INFINITY; a.sum = 0.0f; a.dot = 0.0f;
    if constexpr (TOP) {
        s_sel.s.clear();
        __syncthreads();
    }
    auto single = [&](int at) {
        const float z = E::scalar(rowp, at);
        soft_add(a, z, c);
        if constexpr (TOP) { if (z > -INFINITY) s_sel.s.append(z, at); }
    };
    if (tid < nhead) single(lo + tid);
    if (tid < ntail) single(tlo + tid);
    if constexpr (TOP) s_sel.s.first_floor(k, bm);

    auto batch = [&](int v0) {
        if constexpr (TOP) s_sel.s.template scan<DT, U>(k, v, q, bm, vlo + v0 * E::kVec);
        soft_batch<DT, U>(a, v, bm, c, vbase, v0, nvec);
    };
    batch(tid);
    for (int bi = 1; bi < nfull; ++bi) {
        bm = load_batch<DT, U, false>(vbase, bi * kBatchVecs + tid, nvec, v, q);
        batch(bi * kBatchVecs + tid);
    }
    if (nfull > 0 && nfull * kBatchVecs < nvec) {
        bm = load_batch<DT, U, true>(vbase, nfull * kBatchVecs + tid, nvec, v, q);
        batch(nfull * kBatchVecs + tid);
    }

    // ---- the block's (m, s, u) and list ----
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) a = soft_union(a, soft_shfl_xor(a, m), c);
    if (lane == 0) s_soft[warp] = a;
    __syncthreads();
    if (warp == 0) {
        a.ref = -INFINITY; a.sum = 0.0f; a.dot = 0.0f;
        if (lane < kTkThreads / 32) a = s_soft[lane];
#pragma unroll
        for (int m = kTkThreads / 64; m > 0; m >>= 1) a = soft_union(a, soft_shfl_xor(a, m), c);
        if (lane == 0) s_block = a;
    }
    if constexpr (TOP) {
        if (s_sel.s.overflow) {
            topk_slice_exact<DT>(rowp, lo, hi, k, s_list, s_sel.s.cand, s_sel.s.xlist, s_sel.s.xqn, &s_sel.s.floor);
        } else if (warp == 0) {
            s_sel.s.drain(k, true);
            __syncwarp();
            s_list[lane] = s_sel.s.list[lane];
        }
    }

    // ---- the row's ----
    int n_all = k;
    if (p.S > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (rank == 0) {
            if (warp == 0) {
                a.ref = -INFINITY; a.sum = 0.0f; a.dot = 0.0f;
                if (lane < p.S) a = *cluster.map_shared_rank(&s_block, lane);
#pragma unroll
                for (int m = kScMaxSplit / 2; m > 0; m >>= 1) a = soft_union(a, soft_shfl_xor(a, m), c);
                if (lane == 0) s_block = a;
            }
            n_all = p.S * k;
            if constexpr (TOP)
                if (tid < n_all) s_all[tid] = *(cluster.map_shared_rank(s_list, tid / k) + tid % k);
        }
        cluster.sync();          // the other blocks' shared memory was read
        if (rank != 0) return;
    } else {
        __syncthreads();
        if constexpr (TOP) { if (tid < k) s_all[tid] = s_list[tid]; }
    }
    if (tid == 0) {
        const Soft t = s_block;
        RowScore r;
        r.m = t.ref;
        r.ok = fabsf(t.ref) < INFINITY;
        r.ln_s = logf(t.sum);
        s_row = r;
        s_found = 0;
        if (p.entropy) p.entropy[out_row] = r.ok ? r.ln_s - kLn2 * (t.dot / t.sum) : NAN;
        if (p.stats) { p.stats[2 * out_row] = t.ref; p.stats[2 * out_row + 1] = r.ok ? t.sum : NAN; }
    }
    __syncthreads();
    const RowScore r = s_row;
    for (int j = tid; j < p.J; j += kTkThreads) {
        if (j >= kTkThreads) {
            const int t = p.tok[out_row * p.J + j];
            inside = t >= 0 && t < p.V;
            zt = inside ? E::scalar(rowp, t) : 0.0f;
        }
        p.logprob[out_row * p.J + j] = inside ? row_logprob(r, zt, p.temperature) : 0.0f;
    }
    if constexpr (TOP) {
        float *ov = p.top_logprob + out_row * k;
        int32_t *oi = p.top_id + out_row * k;
        if (tid < n_all) {
            const Cand mine = s_all[tid];
            if (mine.id != kNoId) {
                int ahead = 0;
                for (int j = 0; j < n_all; ++j) ahead += beats(s_all[j].z, s_all[j].id, mine.z, mine.id) ? 1 : 0;
                if (ahead < k) {
                    ov[ahead] = row_logprob(r, mine.z, p.temperature);
                    oi[ahead] = mine.id;
                    atomicAdd(&s_found, 1);
                }
            }
        }
        __syncthreads();
        if (tid == 0 && s_found < k) {
            const int found = s_found;
            complete_row(ov, oi, found, k);
            if (!r.ok)
                for (int j = found; j < k; ++j) ov[j] = NAN;
        }
    }
}

struct GradParams {
    const void *logits;
    void *grad;
    long long ld, ld_grad;
    int V, S, L;                // blocks per row, columns per block
    float temperature, c;
    const int32_t *tok;
    int J;
    const float *stats, *entropy, *g, *h;
};

constexpr int kGrU = 4;

template <int DT>
__device__ __forceinline__ void store_scalar(void *row, int at, float x)
{
    if (DT == MARS_BF16) ((__nv_bfloat16 *)row)[at] = __float2bfloat16_rn(x);
    else ((float *)row)[at] = x;
}

// Gradient of one logit without the tokens' own terms.
__device__ __forceinline__ float grad_term(float z, float m, float c, float a, float b)
{
    if (!(z > -INFINITY)) return 0.0f;
    const float x = soft_distance(z, m, c);
    return ex2f(x) * fmaf(b, x, a);
}

// Backward: a block takes a contiguous piece of one row.
template <int DT>
__global__ void __launch_bounds__(kTkThreads) logprob_grad_kernel(const GradParams p)
{
    typedef Elem<DT> E;
    __shared__ float s_z[MARS_SCORES_MAX_TOKENS];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31;
    const long long row = blockIdx.x / p.S;
    const int lo = min((int)(blockIdx.x - row * p.S) * p.L, p.V), hi = min(p.V, lo + p.L);
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
    float a = -g / ts, b = 0.0f;
    if (p.h) { a = -fmaf(h, p.entropy[row] - logf(s), g) / ts; b = -(h * kLn2) / ts; }
    if (!ok) { a = 0.0f; b = 0.0f; }

    // the tokens' logits, before anything is overwritten
    bool hit = false;
    for (int j = tid; j < p.J; j += kTkThreads) {
        const int t = tok[j];
        if (t >= lo && t < hi) { s_z[j] = E::scalar(zrow, t); hit = true; }
    }
    hit = __syncthreads_or(hit);

    const SoftFloor f = soft_floor(m, c);
    const uintptr_t a0 = (uintptr_t)(zrow + (size_t)lo * E::kBytes), b0 = (uintptr_t)(grow + (size_t)lo * E::kBytes);
    if (((a0 ^ b0) & 15) || !ok || !f.ok) {
        // rows that lie differently on 16-byte boundaries, and rows without fast form: one by one
        for (int i = lo + tid; i < hi; i += kTkThreads)
            store_scalar<DT>(grow, i, ok ? grad_term(E::scalar(zrow, i), m, c, a, b) : 0.0f);
    } else {
        const int nhead = min((int)(((16 - (a0 & 15)) & 15) / E::kBytes), hi - lo);
        const int vlo = lo + nhead, nvec = (hi - vlo) / E::kVec, tlo = vlo + nvec * E::kVec, ntail = hi - tlo;
        if (tid < nhead) store_scalar<DT>(grow, lo + tid, grad_term(E::scalar(zrow, lo + tid), m, c, a, b));
        if (tid < ntail) store_scalar<DT>(grow, tlo + tid, grad_term(E::scalar(zrow, tlo + tid), m, c, a, b));
        const uint4 *src = (const uint4 *)(zrow + (size_t)vlo * E::kBytes);
        uint4 *dst = (uint4 *)(grow + (size_t)vlo * E::kBytes);
        const uint32_t w = soft_floor_word<DT>(f.z);
        const float2 nm = make_float2(-m, -m), c2 = make_float2(c, c), a2 = make_float2(a, a), b2 = make_float2(b, b);
        for (int v0 = tid; v0 < nvec; v0 += kTkThreads * kGrU) {
            uint4 v[kGrU];
#pragma unroll
            for (int u = 0; u < kGrU; ++u)
                if (v0 + u * kTkThreads < nvec) v[u] = src[v0 + u * kTkThreads];   // (plain loads: the gradient may overwrite)
#pragma unroll
            for (int u = 0; u < kGrU; ++u) {
                if (v0 + u * kTkThreads >= nvec) break;
                const uint4 t = soft_clamp<DT>(v[u], w);
                float y[E::kVec];
#pragma unroll
                for (int e = 0; e < E::kVec; e += 2) {
                    const float2 x = mul2(add2(make_float2(E::elem(t, e), E::elem(t, e + 1)), nm), c2);
                    const float2 r = mul2(make_float2(ex2f(x.x), ex2f(x.y)), fma2(b2, x, a2));
                    y[e] = r.x; y[e + 1] = r.y;
                }
                uint4 o;
                if constexpr (DT == MARS_BF16) {
                    uint32_t q[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q[i]) : "f"(y[2 * i + 1]), "f"(y[2 * i]));
                    o = make_uint4(q[0], q[1], q[2], q[3]);
                } else {
                    o = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
                }
                dst[v0 + u * kTkThreads] = o;
            }
        }
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
        store_scalar<DT>(grow, t, grad_term(s_z[j], m, c, a, b) + own / p.temperature);
    }
}

static bool scores_sizes_ok(int64_t rows, int V) { return rows <= (1ll << 27) && V <= (1 << 30); }

// Blocks per row: as many as fill the GPU, while a slice is worth a block.
static int logprob_split(int64_t rows, int V, int es)
{
    const int force = hook(kHookForceSplit);
    int S = 1;
    while (S < kScMaxSplit && (force >= 1 ? 2 * S <= force
                                          : rows * S * 2 <= kScTargetBlocks && (int64_t)V * es >= (int64_t)2 * S * kScMinSliceBytes))
        S *= 2;
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
    void (*kernel)(const LogprobParams) = p.k ? logprob_kernel<DT, kTkU, 3, true> : logprob_kernel<DT, kTkU, 4, false>;
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
    p.S = logprob_split(rows, V, es);
    p.L = slice_columns(V, p.S);
    p.temperature = temperature;
    p.c = (float)(1.4426950408889634 / (double)temperature);
    if (!(p.c > 0.0f) || p.c > 3.40282347e38f) return MARS_ERR_UNSUPPORTED;
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
    const int piece = kTkThreads * kGrU * 16 / es;       // columns that a block holds in registers at once
    p.S = (V + piece - 1) / piece;
    p.L = slice_columns(V, p.S);
    if (rows * p.S > 0x7fffffffll) return MARS_ERR_UNSUPPORTED;
    p.temperature = temperature;
    p.c = (float)(1.4426950408889634 / (double)temperature);
    if (!(p.c > 0.0f) || p.c > 3.40282347e38f) return MARS_ERR_UNSUPPORTED;
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
