// Pieces shared by the kernels that select the best k <= 32 of a logits row: candidates, ordered lists held
// by warps, the exact selection of a slice, and the completion of rows with fewer than k entries above -inf.
#pragma once

#include "mars_common.cuh"
#include "mars_top2_stream.cuh"

namespace mars {

constexpr int kTkThreads = 256;
constexpr int kTkU = 8;
constexpr int kTkMaxK = 32;
constexpr int kTkCap = kTkThreads * 8;   // slots of a slice's queue of candidates (the exact selection reuses
                                         // them: one vector step per thread)

struct Cand {
    float z;
    int id;
};

// Order-preserving float <-> uint encoding for the block-wide bound (atomicMax on shared memory).
__device__ __forceinline__ unsigned tk_enc(float x)
{
    unsigned b = __float_as_uint(x + 0.0f);
    return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float tk_dec(unsigned e)
{
    return __uint_as_float(e ^ ((e & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}

// A warp keeps its k best elements so far spread over its lanes: lane i < k holds the i-th best
// (value wz, token id wid), the other lanes hold {-inf, kNoId}.  Inserting one candidate is a
// ballot (how many entries beat it) and one shuffle; the candidate is the same in all lanes.
__device__ __forceinline__ void warp_list_insert(float &wz, int &wid, int lane, int k, float x, int id)
{
    const unsigned ahead = __ballot_sync(0xffffffffu, beats(wz, wid, x, id));
    const int pos = __popc(ahead);              // entries are sorted: exactly lanes 0..pos-1 beat it
    const float uz = __shfl_up_sync(0xffffffffu, wz, 1);
    const int uid = __shfl_up_sync(0xffffffffu, wid, 1);
    if (pos < k) {
        if (lane == pos) { wz = x; wid = id; }
        else if (lane > pos && lane < k) { wz = uz; wid = uid; }
    }
}

// Exact slice selection with per-warp lists; always correct, used when a streaming kernel's queue
// runs out of room.  Called by all threads of the block.  The caller lends its shared memory:
//   queue_mem  kTkThreads * 8 candidates (per warp: the candidates of one vector step)
//   s_list     (kTkThreads / 32) * kTkMaxK candidates (the warps' lists for the final ranking)
//   s_qn       kTkThreads / 32 counters;  s_bound  block-wide lower bound on the slice's k-th value
template <int DT>
__device__ __noinline__ void topk_slice_exact(const char *rowp, const int lo, const int hi, const int k,
                                              Cand *out, Cand *queue_mem, Cand *s_list, int *s_qn,
                                              unsigned *s_bound_p)
{
    typedef Elem<DT> E;
    constexpr int kWarps = kTkThreads / 32;
    unsigned &s_bound = *s_bound_p;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    const uintptr_t a0 = (uintptr_t)(rowp + (size_t)lo * E::kBytes);
    int nhead = (int)(((16 - (a0 & 15)) & 15) / E::kBytes);
    nhead = min(nhead, max(hi - lo, 0));
    const int vlo = lo + nhead;
    const int nvec = max(hi - vlo, 0) / E::kVec;
    const int tlo = vlo + nvec * E::kVec;
    const int ntail = max(hi - tlo, 0);
    const uint4 *vbase = (const uint4 *)(rowp + (size_t)vlo * E::kBytes);

    __syncthreads();             // shared arrays may still be in use from a previous slice
    if (tid == 0) s_bound = tk_enc(-INFINITY);
    if (lane == 0) s_qn[warp] = 0;
    __syncthreads();

    float wz = -INFINITY;       // this lane's entry of the warp's list
    int wid = kNoId;
    float kth = -INFINITY;      // value / id of the warp's k-th best (entry of lane k-1)
    int kth_id = kNoId;
    float warp_floor = -INFINITY;   // value-only bound from the warp's first batch
    Cand *queue = queue_mem + warp * (32 * 8);

    // Drain the warp's queue into its list (all lanes), then publish the warp's k-th value.
    auto drain = [&]() {
        __syncwarp();
        const int n = s_qn[warp];
        for (int i = 0; i < n; ++i) {
            const Cand c = queue[i];
            if (beats(c.z, c.id, kth, kth_id)) {
                warp_list_insert(wz, wid, lane, k, c.z, c.id);
                kth = __shfl_sync(0xffffffffu, wz, k - 1);
                kth_id = __shfl_sync(0xffffffffu, wid, k - 1);
            }
        }
        __syncwarp();
        if (lane == 0) {
            s_qn[warp] = 0;
            if (kth > -INFINITY) atomicMax(&s_bound, tk_enc(kth));
        }
        __syncwarp();
    };
    // One element of this lane: queue it if it can still be among the slice's k best.
    auto offer = [&](float x, int idx, float floor_v) {
        if (x >= floor_v && x > -INFINITY && beats(x, idx, kth, kth_id)) {
            const int pos = atomicAdd(&s_qn[warp], 1);
            queue[pos].z = x;
            queue[pos].id = idx;
        }
    };

    // head and tail scalars (at most 15 elements) go through the same queue
    if (nhead > 0 || ntail > 0) {
        if (warp == 0) {
            if (lane < nhead) offer(E::scalar(rowp, lo + lane), lo + lane, -INFINITY);
            if (lane < ntail) offer(E::scalar(rowp, tlo + lane), tlo + lane, -INFINITY);
            drain();
        }
    }

    constexpr int kBatchVecs = kTkThreads * kTkU;
    const int nbatches = (nvec + kBatchVecs - 1) / kBatchVecs;
    for (int bi = 0; bi < nbatches; ++bi) {
        uint4 v[kTkU];
        typename E::packed_t q[kTkU];
        const int v0 = bi * kBatchVecs + tid;
#pragma unroll
        for (int u = 0; u < kTkU; ++u) {
            int vi = v0 + u * kTkThreads;
            v[u] = vi < nvec ? ld_stream(vbase + vi) : E::neg_inf();
        }
        typename E::packed_t m = E::vred(v[0]);
        q[0] = m;
#pragma unroll
        for (int u = 1; u < kTkU; ++u) { q[u] = E::vred(v[u]); m = E::pmax(m, q[u]); }
        const float bm = E::to_float(m);
        if (bi == 0) {
            // value-only bound for the warp: the k-th largest of its lanes' first-batch maxima
            // (maxima of distinct elements); rank by (value, lane).
            const float mine = (bm == bm) ? bm : -INFINITY;
            int rank = 0;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float o = __shfl_sync(0xffffffffu, mine, j);
                rank += (o > mine || (o == mine && j < lane)) ? 1 : 0;
            }
            const unsigned who = __ballot_sync(0xffffffffu, rank == k - 1);
            warp_floor = __shfl_sync(0xffffffffu, mine, __ffs(who) - 1);
        }
        float floor_v = fmaxf(warp_floor, tk_dec(*(volatile unsigned *)&s_bound));
        floor_v = fmaxf(floor_v, kth);
        if (__any_sync(0xffffffffu, bm >= floor_v)) {
#pragma unroll
            for (int u = 0; u < kTkU; ++u) {
                const float qf = E::to_float(q[u]);
                if (__any_sync(0xffffffffu, qf >= floor_v)) {
                    if (qf >= floor_v) {
                        const int base = vlo + (v0 + u * kTkThreads) * E::kVec;
#pragma unroll
                        for (int e = 0; e < E::kVec; ++e) offer(E::elem(v[u], e), base + e, floor_v);
                    }
                    drain();
                    floor_v = fmaxf(floor_v, kth);
                }
            }
        }
    }

    // ---- block: the k best of the warps' lists by rank counting ----
    if (lane < kTkMaxK) { s_list[warp * kTkMaxK + lane].z = lane < k ? wz : -INFINITY;
                          s_list[warp * kTkMaxK + lane].id = lane < k ? wid : kNoId; }
    for (int i = tid; i < k; i += kTkThreads) { out[i].z = -INFINITY; out[i].id = kNoId; }
    __syncthreads();
    constexpr int kAll = kWarps * kTkMaxK;
    for (int i = tid; i < kAll; i += kTkThreads) {
        const Cand c = s_list[i];
        if (c.id == kNoId) continue;
        int rank = 0;
        for (int j = 0; j < kAll; ++j)
            rank += (s_list[j].id != kNoId && beats(s_list[j].z, s_list[j].id, c.z, c.id)) ? 1 : 0;
        if (rank < k) out[rank] = c;
    }
}

// Fewer than k entries above -inf in a row: the remaining places go to the lowest unused ids at
// -inf (every -inf / NaN entry ties, lowest id first).  One thread.
__device__ inline void complete_row(float *ov, int32_t *oi, int found, int k)
{
    int next = 0;
    while (found < k) {
        bool used = false;
        for (int j = 0; j < found; ++j) used |= (oi[j] == next);
        if (!used) { ov[found] = -INFINITY; oi[found] = next; ++found; }
        ++next;
    }
}

}  // namespace mars
