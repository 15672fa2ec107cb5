// Exact top-k (k <= 32) of a slice of a logits row while a block streams it: the selection shared by
// mars_topk_rows and the calls that report alternatives beside other results of the same pass.
#pragma once

#include "mars_common.cuh"
#include "mars_top2_stream.cuh"

namespace mars {

constexpr int kTkThreads = 256;
constexpr int kTkU = 8;
constexpr int kTkMaxK = 32;
constexpr int kTkWarps = kTkThreads / 32;
constexpr int kTkCap = kTkThreads * 8;   // slots of the slice's queue of elements at or above the floor
                                         // (the exact fallback reuses them: one vector step per thread)

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

// Exact slice selection with per-warp lists; always correct, used when the streaming kernel below
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

// Slice selection.  A block streams its slice once, like the top-2 kernel (batches of 8 vectors
// per thread reduced with packed max instructions).  A batch is looked at more closely only if
// its maximum reaches the floor, a lower bound on the slice's k-th value:
//   - the floor starts as the k-th largest of the threads' first-batch maxima (values of distinct
//     elements): every warp orders its lanes' maxima, the k best of each warp go to a small
//     table, and the table's k-th entry is found by rank counting;
//   - a thread whose batch reaches the floor appends the elements that do to a queue in shared
//     memory (one atomicAdd each), nothing more;
//   - the slice's k best so far live in one ordered list in shared memory.  After appending, a
//     warp TRIES to take the list (one compare-and-swap, no waiting): if it gets it, it holds
//     the list in its lanes (lane i = entry i), feeds the queued elements into it one by one (a
//     ballot and a shuffle each), stores it back and publishes the k-th entry's value as the new
//     floor; if another warp has it, that warp or a later one will pick the elements up.
// So nobody ever waits, the floor trails the stream by at most a few elements, about
// k (1 + ln(batches)) elements reach the queue on unordered data, and the list is the result.
// If the queue fills up (adversarially ordered rows), the block redoes its slice with
// topk_slice_exact.
struct TopkSelect {
    __align__(8) Cand cand[kTkCap];
    __align__(8) Cand list[kTkMaxK];
    __align__(8) Cand xlist[kTkWarps * kTkMaxK];    // exact fallback only
    float top[kTkWarps * kTkMaxK];
    unsigned floor;
    int tail, head, lock, overflow;
    int xqn[kTkWarps];

    // Empty queue and list (all threads; the caller synchronises before the first append).
    __device__ __forceinline__ void clear()
    {
        // empty slots carry kNoId so that a reader can tell a reserved slot from a written one
        Cand e; e.z = -INFINITY; e.id = kNoId;
        for (int i = threadIdx.x; i < kTkCap; i += kTkThreads) cand[i] = e;
        if (threadIdx.x < kTkMaxK) list[threadIdx.x] = e;
        if (threadIdx.x == 0) { floor = tk_enc(-INFINITY); tail = 0; head = 0; lock = 0; overflow = 0; }
    }

    __device__ __forceinline__ void append(float x, int idx)
    {
        const int pos = atomicAdd(&tail, 1);
        if (pos < kTkCap) {
            Cand e; e.z = x; e.id = idx;     // one 8-byte store: value and id become visible together
            *reinterpret_cast<volatile unsigned long long *>(&cand[pos]) = *reinterpret_cast<unsigned long long *>(&e);
        } else {
            overflow = 1;
        }
    }

    // Feed the queued elements into the list.  Called by whole warps; `force` skips the
    // compare-and-swap (used once at the end, when no other warp can be in here).
    __device__ __forceinline__ void drain(int k, bool force)
    {
        const int lane = threadIdx.x & 31;
        int got = 1;
        if (!force) {
            if (lane == 0) got = atomicCAS(&lock, 0, 1) == 0 ? 1 : 0;
            got = __shfl_sync(0xffffffffu, got, 0);
        }
        if (!got) return;
        __threadfence_block();
        // one lane reads the queue's bounds for all: the tail moves while other warps append
        int i = 0, end = 0;
        if (lane == 0) { i = *(volatile int *)&head; end = min(*(volatile int *)&tail, kTkCap); }
        i = __shfl_sync(0xffffffffu, i, 0);
        end = __shfl_sync(0xffffffffu, end, 0);
        unsigned long long raw = *reinterpret_cast<volatile unsigned long long *>(&list[lane]);
        Cand mine = *reinterpret_cast<Cand *>(&raw);
        // 32 slots at a time, one per lane.  Lanes do not read at the same instant, so what is
        // "written" is settled by a ballot: every decision below is the same in all lanes.
        while (i < end) {
            Cand c; c.z = -INFINITY; c.id = kNoId;
            if (i + lane < end) {
                raw = *reinterpret_cast<volatile unsigned long long *>(&cand[i + lane]);
                c = *reinterpret_cast<Cand *>(&raw);
            }
            const unsigned written = __ballot_sync(0xffffffffu, c.id != kNoId);
            const int n = written == 0xffffffffu ? 32 : __ffs(~written) - 1;    // leading written slots
            for (int t = 0; t < n; ++t) {
                const float cz = __shfl_sync(0xffffffffu, c.z, t);
                const int cid = __shfl_sync(0xffffffffu, c.id, t);
                warp_list_insert(mine.z, mine.id, lane, k, cz, cid);
            }
            i += n;
            if (n < 32) break;       // a slot that is reserved but not written yet: a later round takes it
        }
        *reinterpret_cast<volatile unsigned long long *>(&list[lane]) = *reinterpret_cast<unsigned long long *>(&mine);
        if (lane == k - 1 && mine.id != kNoId) atomicMax(&floor, tk_enc(mine.z));
        __syncwarp();
        if (lane == 0) {
            *(volatile int *)&head = i;
            __threadfence_block();
            if (!force) atomicExch(&lock, 0);
        }
    }

    // First floor: the k-th largest of the threads' first-batch maxima, or a value just below it.
    // Each warp enters its m = min(k, 4 + k/4) largest maxima, ordered, into a table and the
    // k-th largest table entry is taken: the table is a subset of the maxima (8 m >= k entries),
    // so its k-th largest never exceeds theirs, and it falls short of it only when one warp
    // holds more than m of the block's k largest (k = 32: 12 of 32 in one of 8 warps).
    __device__ __forceinline__ void first_floor(int k, float bm)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        const int m = min(k, 4 + (k >> 2));
        const float mine = (bm == bm) ? bm : -INFINITY;
        int wrank = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float o = __shfl_sync(0xffffffffu, mine, j);
            wrank += (o > mine || (o == mine && j < lane)) ? 1 : 0;
        }
        if (wrank < m) top[warp * m + wrank] = mine;
        __syncthreads();
        const int nt = kTkWarps * m;
        if (tid < nt) {
            const float t = top[tid];
            int rank = 0;
            for (int j = 0; j < nt; ++j) {
                const float o = top[j];
                rank += (o > t || (o == t && j < tid)) ? 1 : 0;
            }
            if (rank == k - 1 && t > -INFINITY) atomicMax(&floor, tk_enc(t));
        }
        __syncthreads();
    }

    // One batch of the thread (its vectors, their maxima and the batch's): element e of vector u has
    // the id base0 + u * kTkThreads * kVec + e.
    template <int DT, int U>
    __device__ __forceinline__ void scan(int k, const uint4 (&v)[U], const typename Elem<DT>::packed_t (&q)[U],
                                         float bm, int base0)
    {
        typedef Elem<DT> E;
        const float floor_v = tk_dec(*(volatile unsigned *)&floor);
        bool appended = false;
        if (bm >= floor_v) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (E::to_float(q[u]) >= floor_v) {
                    unsigned em = 0;
#pragma unroll
                    for (int e = 0; e < E::kVec; ++e) {
                        const float x = E::elem(v[u], e);
                        em |= (x >= floor_v && x > -INFINITY) ? (1u << e) : 0u;
                    }
                    const int base = base0 + u * kTkThreads * E::kVec;
                    while (em) {
                        const int e = __ffs(em) - 1;
                        em &= em - 1;
                        append(E::elem(v[u], e), base + e);
                        appended = true;
                    }
                }
            }
        }
        if (__any_sync(0xffffffffu, appended)) drain(k, false);
    }
};

}  // namespace mars
