// libmars: the calls that write, move and hand out the pages of the 4-bit KV cache.
//
// All of them move bytes; none computes enough to matter.  append and gather are one pass over
// their rows with a thread per 16 values (one scale); commit and fork move packed rows with 16-byte
// loads; resize and fork's bookkeeping run in one thread block cluster / block, since the page
// tables are a few hundred kilobytes at most and a grid-wide step would cost more than it moves.
// Measured: append and gather of 49300 ragged rows of 8 heads of 128 (259 MB moved each) 65 and
// 52 us: 4.0 and 5.0 TB/s; 67 and 75 % of the issue slots are taken (conversions and quotients).  In fp32 (461 MB)
// 70 and 80 us: 6.6 and 5.8 TB/s.  The rows of
// 64 forks' last pages 21 us for 150 MB (7.1 TB/s, partly in L2), their tables 12 us; the page decisions of 2048 sequences
// 24 us, of 64 11 us (latency of dependent steps: 5 % of the issue slots, nothing of DRAM); the paths out of 64
// trees in four layers 6 us.
#include "mars_kv.cuh"
#include "mars_stream.cuh"
#include "mars_hooks.cuh"

#include <cuda_runtime.h>
#include <math.h>

#include "mars_kv.h"

namespace mars {

__host__ __device__ constexpr int elem_bytes(int dt) { return dt == MARS_FP32 ? 4 : 2; }

inline bool kv_dtype_ok(int dt) { return dt == MARS_BF16 || dt == MARS_FP32 || dt == MARS_FP16; }

// --------------------------------------------------------------------------------- append

struct AppendParams {
    KvView kv;
    unsigned char *layer;
    const float *scales;       // this layer's [2][kv_heads]
    const unsigned char *src[2];
    int64_t row[2], head[2];   // elements
    const int32_t *count;
    int32_t *status;
    int N, iters;
    bool wide;                 // every group of 16 values on a 32-byte boundary
};

// 32 bytes at p; `wide`: p is 32-byte aligned and one load does (two 16-byte loads of a warp would each
// touch half of every 32-byte sector).
__device__ __forceinline__ void load32(const unsigned char *p, bool wide, uint32_t (&w)[8])
{
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
            : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
    } else {
        const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
}
__device__ __forceinline__ void store32(unsigned char *p, bool wide, const uint32_t (&w)[8])
{
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
            ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// 16 values of `DT`, widened exactly.
template <int DT>
__device__ __forceinline__ void load16(const unsigned char *p, bool wide, float (&x)[16])
{
    uint32_t w[8];
    load32(p, wide, w);
    if constexpr (DT == MARS_FP32) {
        uint32_t v[8];
        load32(p + 32, wide, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[i] = __uint_as_float(w[i]); x[8 + i] = __uint_as_float(v[i]); }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (DT == MARS_BF16) {
                x[2 * j] = __uint_as_float(w[j] << 16);
                x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            } else {
                const float2 f = f16x2_to_float2(w[j]);
                x[2 * j] = f.x;
                x[2 * j + 1] = f.y;
            }
        }
    }
}

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ uint32_t e4m3_from(float x)   // nearest even, saturating; x >= 0, not NaN
{
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(x));
    return r & 0xffu;
}

// Eight values -> eight E2M1 codes, element 0 in the lowest nibble; nearest even, saturating.
__device__ __forceinline__ uint32_t e2m1x8_from(const float *t)
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(t[0]), "f"(t[1]), "f"(t[2]), "f"(t[3]), "f"(t[4]), "f"(t[5]), "f"(t[6]), "f"(t[7]));
    return r;
}

// Sixteen values against their scale: the negated IEEE quotients -(x / sg), as the definition has them, in
// place.  With 8-bit significands and a power of two as g many quotients lie exactly on the border of
// two codes, where a reciprocal's last bit would decide.  Fast form: x * r and one residual correction
// (Markstein 1990: with r the rounded reciprocal, fma(fma(-q, sg, x), r, q) is the rounded quotient
// while nothing over- or underflows), two values at a time.  The scale did not saturate, so |x / sg| <= 6.4 for
// a normal s; for a subnormal one, off by up to a third, it reaches 9, and the conversion to codes saturates.
// The sign is turned since fma(0, r, -0) is +0 and a zero would lose its sign bit.
__device__ __forceinline__ void quotients16(float (&x)[16], float sg, bool plain)
{
    if (plain) {
        const float r = -__frcp_rn(sg);
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            asm("{\n\t.reg .b64 x, r, d, q, e;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 r, {%2, %2};\n\tmov.b64 d, {%3, %3};\n\t"
                "mul.rn.f32x2 q, x, r;\n\tfma.rn.f32x2 e, q, d, x;\n\tfma.rn.f32x2 q, e, r, q;\n\tmov.b64 {%0, %1}, q;\n\t}"
                : "+f"(x[i]), "+f"(x[i + 1]) : "f"(r), "f"(sg));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = sg > 0.0f ? -__fdiv_rn(x[i], sg) : -0.0f;
    }
}

// Rows that a thread of append / gather goes through: four in long calls, where the blocks' start-up
// counts, two where about all blocks are resident at once and the latency of a row does.  Measured, us
// with 1 / 2 / 4: 64 trees into four layers and the path out of them (one graph) 40.8 / 39.3 / 47.3; 16
// prompts of up to 4096 rows in and out 167 / 135 / 121.
inline int row_iters(int64_t blocks) { return blocks <= 16 * 148 ? 2 : 4; }

// Rows a block of 256 threads covers at once when a row takes per_row threads.
__host__ __device__ inline int rows_at_once(int per_row) { return per_row >= 256 ? 1 : 256 / per_row; }

// A thread per 16 values and row (p.iters rows one after the other): grid.y = sequence.
// Bound by memory from a few thousand rows on; below that by its latency.
template <int D, int DT>
__global__ void __launch_bounds__(256) kv_append_kernel(const AppendParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kG = D / 16;   // groups of a row
    const int b = blockIdx.y;
    const int count = p.count ? p.count[b] : p.N, len = p.kv.seq_len[b], cap = kv_capacity(p.kv, b);
    const int n = min(max(count, 0), p.N);
    const bool room = n == 0 || (len >= 0 && (int64_t)len + n <= cap);
    if (blockIdx.x == 0 && threadIdx.x == 0 && p.status) p.status[b] = room ? MARS_SEQ_OK : MARS_SEQ_NO_ROOM;
    if (!room) return;
    const int per_row = p.kv.kv_heads * 2 * kG, at_once = rows_at_once(per_row);
    const int lane_row = per_row >= 256 ? 0 : (int)threadIdx.x / per_row;
    if (lane_row >= at_once) return;
    const int row0 = blockIdx.x * at_once * p.iters + lane_row;
    // a thread keeps its head and place in the row and goes down the rows
#pragma unroll 1
    for (int c = (int)threadIdx.x - lane_row * per_row; c < per_row; c += 256) {
        const int h = c / (2 * kG), kv = (c / kG) & 1, grp = c % kG;
        const int64_t stride = kv ? p.row[1] : p.row[0];
        const unsigned char *src0 = (kv ? p.src[1] : p.src[0]) + ((int64_t)b * p.N * stride + h * (kv ? p.head[1] : p.head[0]) + grp * 16) * elem_bytes(DT);
        const float g = p.scales[kv * p.kv.kv_heads + h];
        int row = row0;
#pragma unroll 1
        for (int it = 0; it < p.iters && row < n; ++it, row += at_once) {
            const int pos = len + row, id = kv_page_id(p.kv, b, pos), slot = pos & 15;
            if (id < 0) continue;
            float x[16];
            load16<DT>(src0 + row * stride * elem_bytes(DT), p.wide, x);
            float a = fabsf(x[0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) a = max_nan(a, fabsf(x[i]));
            if (a != a) {                    // NaN counts as 0
                a = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[i] = x[i] == x[i] ? x[i] : 0.0f;
                    a = fmaxf(a, fabsf(x[i]));
                }
            }
            const uint32_t s8 = e4m3_from(__fdiv_rn(__fdiv_rn(a, 6.0f), g));
            const float sg = __fmul_rn(f16x2_to_float2(e4m3x2_to_f16x2(s8)).x, g);
            quotients16(x, sg, s8 != 0x7eu && sg > 1e-30f && sg < 1e30f);
            unsigned char *blk = kv_block<D>(p.kv, p.layer, id, h, pos);
            *reinterpret_cast<uint2 *>(blk + 8 * D * kv + slot * (D / 2) + grp * 8) = make_uint2(e2m1x8_from(x) ^ 0x88888888u, e2m1x8_from(x + 8) ^ 0x88888888u);
            blk[16 * D + D * kv + slot * kG + grp] = (unsigned char)s8;
        }
    }
}

// --------------------------------------------------------------------------------- gather

struct GatherParams {
    KvView kv;
    int layer0;
    const int32_t *start, *count;
    unsigned char *dst[2];
    int B, rows, iters;
    bool wide;                 // outputs on 32-byte boundaries
};

// f * g (f a code times its scale: at most 6 bits, 2^-10 or more unless 0) so that a conversion to a 16-bit type
// rounds the exact product: cut off to 24 bits, the last bit set if anything was lost (rounding to odd, Boldo and
// Melquiond 2008).  Rounded to nearest first, a product just off a border of two 16-bit values can land on it.
// `last` (odd_bit) is that bit for all f of a head, without a remainder.  A g of at most 18 bits has exact products: 0.
// Another g has 19 bits or more and ends within 6 of its last place, as the product does: too low for it to be a
// border itself, and off a border the bit may be set whether or not something was lost.  (Subnormal g below 2^18
// units have at most 18 bits wherever they end.  All of it holds while the product does not underflow in fp32; it does
// for bf16 results below 2^-126 only.)  16 prompts in and out 117 us, with products to nearest 115, from remainders 135.
__device__ __forceinline__ uint32_t odd_bit(float g) { return (__float_as_uint(g) & 63u) != 0u && g >= 0x1p-131f; }
__device__ __forceinline__ float product_to_odd(float f, float g, uint32_t last)
{
    return __uint_as_float(__float_as_uint(__fmul_rz(f, g)) | last);
}

// A thread per 16 values and row, as in append: grid.y = sequence, grid.z = layer.
template <int D, int DT>
__global__ void __launch_bounds__(256) kv_gather_kernel(const GatherParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kG = D / 16;
    const int b = blockIdx.y, lay = blockIdx.z, H = p.kv.kv_heads;
    const int count = p.count ? p.count[b] : p.rows, start = p.start ? p.start[b] : 0, cap = kv_capacity(p.kv, b);
    const int n = min(max(count, 0), p.rows);
    const int per_row = H * 2 * kG, at_once = rows_at_once(per_row);
    const int lane_row = per_row >= 256 ? 0 : (int)threadIdx.x / per_row;
    if (lane_row >= at_once) return;
    unsigned char *layer = p.kv.pages + (int64_t)(p.layer0 + lay) * p.kv.layer_bytes;
    const float *scales = p.kv.scales + (int64_t)(p.layer0 + lay) * 2 * H;
    const int row0 = blockIdx.x * at_once * p.iters + lane_row;
#pragma unroll 1
    for (int c = (int)threadIdx.x - lane_row * per_row; c < per_row; c += 256) {
        const int kv = c >= H * kG, h = (c / kG) - kv * H, grp = c % kG;
        const float g = scales[kv * H + h];
        const uint32_t last = odd_bit(g);
        unsigned char *dst = (kv ? p.dst[1] : p.dst[0]) + ((((int64_t)lay * p.B + b) * p.rows * H + h) * D + grp * 16) * elem_bytes(DT);
        const int64_t dst_row = (int64_t)H * D * elem_bytes(DT);
        int row = row0;
#pragma unroll 1
        for (int it = 0; it < p.iters && row < n; ++it, row += at_once) {
            const int64_t pos64 = (int64_t)start + row;
            if (pos64 < 0 || pos64 >= cap) continue;
            const int pos = (int)pos64, id = kv_page_id(p.kv, b, pos), slot = pos & 15;
            if (id < 0) continue;
            const unsigned char *blk = kv_block<D>(p.kv, layer, id, h, pos);
            const uint2 codes = *reinterpret_cast<const uint2 *>(blk + 8 * D * kv + slot * (D / 2) + grp * 8);
            const uint32_t s = e4m3x2_to_f16x2(blk[16 * D + D * kv + slot * kG + grp] * 0x101u);
            // code * scale is exact in fp16, so the product with g is the one thing to round
            float x[16];
            uint32_t hh[4];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                e2m1x8_to_f16x2(w ? codes.y : codes.x, hh);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = f16x2_to_float2(hmul2(hh[j], s));
                    x[8 * w + 2 * j] = DT == MARS_FP32 ? f.x * g : product_to_odd(f.x, g, last);
                    x[8 * w + 2 * j + 1] = DT == MARS_FP32 ? f.y * g : product_to_odd(f.y, g, last);
                }
            }
            unsigned char *o = dst + row * dst_row;
            uint32_t w[8];
            if constexpr (DT == MARS_FP32) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[8 * half + i]);
                    store32(o + 32 * half, p.wide, w);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[i] = DT == MARS_BF16 ? bf16x2_from(x[2 * i], x[2 * i + 1]) : f16x2_from(x[2 * i], x[2 * i + 1]);
                store32(o, p.wide, w);
            }
        }
    }
}

// --------------------------------------------------------------------------------- commit

struct CommitParams {
    KvView kv;
    const int32_t *path;       // or null
    const int32_t *accept_len;
    int32_t *new_len;
    int32_t *status;
    int path_width, B, layers;
};

// Whether sequence b's path is sound (warp-uniform), and its accepted drafts a (-1: none).
__device__ bool commit_path_ok(const CommitParams &p, int b, int lane, int *a_out)
{
    const int a = p.accept_len[b], len = p.kv.seq_len[b];
    const int64_t cap = kv_capacity(p.kv, b);
    *a_out = a;
    if (a == -1) return true;
    bool ok = a >= 0 && len >= 0 && (p.path ? a < p.path_width : (int64_t)len + a < cap);
    if (ok && p.path) {
        const int32_t *path = p.path + (int64_t)b * p.path_width;
        for (int j = lane; j <= a; j += 32) {
            const int x = path[j], prev = j ? path[j - 1] : -1;
            if (x <= prev || (j == 0 && x != 0) || (int64_t)len + x >= cap) ok = false;
        }
    }
    return __all_sync(0xffffffffu, ok) != 0;
}

// A warp per (sequence, layer, head).  Node numbers rise along the path, so path[j] >= j and row j's
// source is never a row that an earlier step wrote: a batch of rows is read into registers before any
// of it is written, and later batches read behind everything written so far.
template <int D>
__global__ void __launch_bounds__(128) kv_commit_kernel(const CommitParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t w = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int64_t per_seq = (int64_t)p.layers * p.kv.kv_heads;
    const int b = (int)(w / per_seq);
    if (b >= p.B) return;
    const int rest = (int)(w - b * per_seq), lay = rest / p.kv.kv_heads, h = rest % p.kv.kv_heads;
    int a;
    const bool ok = commit_path_ok(p, b, lane, &a);
    const int len = p.kv.seq_len[b];
    if (rest == 0 && lane == 0) {
        if (p.new_len && p.new_len != p.kv.seq_len) p.new_len[b] = ok ? len + a + 1 : len;
        if (p.status) p.status[b] = ok ? MARS_SEQ_OK : MARS_SEQ_BAD_PATH;
    }
    if (!ok || a < 1 || !p.path) return;
    const int32_t *path = p.path + (int64_t)b * p.path_width;
    unsigned char *layer = p.kv.pages + lay * p.kv.layer_bytes;
    // a row: 2 * D/32 pieces of 16 code bytes and 2 pieces of D/16 scale bytes
    constexpr int kCode = D / 16, kPieces = kCode + 2, kPer = 4;
    constexpr int kRows = 32 * kPer / kPieces;   // rows per batch
    for (int j0 = 1; j0 <= a; j0 += kRows) {
        const int rows = min(kRows, a + 1 - j0);
        // lane r: block of row j0 + r's source and destination and its slots there, 0 where nothing moves
        uint64_t from = 0, into = 0;
        int slots = 0;
        if (lane < rows) {
            const int src = len + path[j0 + lane], dst = len + j0 + lane;
            const int ids = kv_page_id(p.kv, b, src), idd = kv_page_id(p.kv, b, dst);
            if (src != dst && ids >= 0 && idd >= 0) {
                from = (uint64_t)kv_block<D>(p.kv, layer, ids, h, src);
                into = (uint64_t)kv_block<D>(p.kv, layer, idd, h, dst);
                slots = (src & 15) | (dst & 15) << 4;
            }
        }
        uint4 v[kPer];
        unsigned char *to[kPer];
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int i = u * 32 + lane, r = i / kPieces, c = i - r * kPieces;
            const unsigned char *sb = (const unsigned char *)__shfl_sync(0xffffffffu, from, r & 31);
            unsigned char *db = (unsigned char *)__shfl_sync(0xffffffffu, into, r & 31);
            const int sl = __shfl_sync(0xffffffffu, slots, r & 31), ss = sl & 15, ds = sl >> 4;
            to[u] = nullptr;
            if (r < rows && sb) {
                if (c < kCode) {
                    const int off = 8 * D * (c / (kCode / 2)), in = (c % (kCode / 2)) * 16;
                    v[u] = *reinterpret_cast<const uint4 *>(sb + off + ss * (D / 2) + in);
                    to[u] = db + off + ds * (D / 2) + in;
                } else {
                    const int off = 16 * D + D * (c - kCode);
                    if constexpr (D == 128) {
                        const uint2 t = *reinterpret_cast<const uint2 *>(sb + off + ss * 8);
                        v[u].x = t.x; v[u].y = t.y;
                    } else {
                        v[u].x = *reinterpret_cast<const uint32_t *>(sb + off + ss * 4);
                    }
                    to[u] = db + off + ds * (D / 16);
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            if (!to[u]) continue;
            const int i = u * 32 + lane, c = i % kPieces;
            if (c < kCode) *reinterpret_cast<uint4 *>(to[u]) = v[u];
            else if constexpr (D == 128) *reinterpret_cast<uint2 *>(to[u]) = make_uint2(v[u].x, v[u].y);
            else *reinterpret_cast<uint32_t *>(to[u]) = v[u].x;
        }
        __syncwarp();
    }
}

// Lengths in place: only after every warp of the kernel above has read the old ones.
__global__ void __launch_bounds__(256) kv_commit_len_kernel(const CommitParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, b = (int)((blockIdx.x * blockDim.x + threadIdx.x) >> 5);
    if (b >= p.B) return;
    int a;
    const bool ok = commit_path_ok(p, b, lane, &a);
    const int len = p.kv.seq_len[b];
    __syncwarp();
    if (lane == 0 && ok) p.new_len[b] = len + a + 1;
}

// --------------------------------------------------------------------------------- page bookkeeping

constexpr int kPoolThreads = 1024;
constexpr int kPoolCluster = 8;

// Exclusive prefix sums of need[0..n) in place (one thread block); returns the total.
__device__ int block_exclusive_scan(int *need, int n, int *s_warp)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (n + kPoolThreads - 1) / kPoolThreads;
    const int lo = min(tid * per, n), hi = min(lo + per, n);
    int sum = 0;
    for (int i = lo; i < hi; ++i) sum += need[i];
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int w = s_warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    const int total = s_warp[31];
    int at = inc - sum + (warp ? s_warp[warp - 1] : 0);
    for (int i = lo; i < hi; ++i) {
        const int x = need[i];
        need[i] = at;
        at += x;
    }
    __syncthreads();
    return total;
}

// Number of free pages, at least up to `enough` (one thread block; scans the set in order).
__device__ int count_free(const uint32_t *bits, int words, int enough, int *s_warp)
{
    int have = 0;
    for (int w0 = 0; w0 < words && have < enough; w0 += 4 * kPoolThreads) {
        int c = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int w = w0 + u * kPoolThreads + threadIdx.x;
            if (w < words) c += __popc(__ldcg(bits + w));
        }
        c = __reduce_add_sync(0xffffffffu, c);
        if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = c;
        __syncthreads();
        int t = s_warp[threadIdx.x & 31];
        have += __reduce_add_sync(0xffffffffu, t);
        __syncthreads();
    }
    return have;
}

// The k-th (from 0) set bit of w, which has more than k.
__device__ __forceinline__ int nth_bit(uint32_t w, int k)
{
    int at = 0;
#pragma unroll
    for (int half = 16; half; half >>= 1) {
        const int c = __popc((w >> at) & ((1u << half) - 1u));
        if (k >= c) { k -= c; at += half; }
    }
    return at;
}

struct FreeTile {                // 1024 words of the free set: exclusive prefix counts and the words
    int first[kPoolThreads];
    uint32_t word[kPoolThreads];
    int warp[32];
};

// The lowest free pages 0, 1, ... of the set go, in order, to `give(rank, page)` for rank < total, and
// leave the set (one thread block).  Ranks, not words, are spread over the threads: free pages tend to
// lie together, and a word's 32 pages would otherwise be given by one thread.
template <class Give>
__device__ void take_free(uint32_t *bits, int words, int total, FreeTile *f, Give give)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int base = 0;
    for (int w0 = 0; w0 < words && base < total; w0 += kPoolThreads) {
        const int w = w0 + tid;
        uint32_t word = w < words ? __ldcg(bits + w) : 0u;
        const int c = __popc(word);
        int inc = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += t;
        }
        if (lane == 31) f->warp[warp] = inc;
        __syncthreads();
        const int sums = f->warp[lane];
        const int before = __reduce_add_sync(0xffffffffu, lane < warp ? sums : 0);
        const int all = __reduce_add_sync(0xffffffffu, sums);
        const int first = before + inc - c;
        f->first[tid] = first;
        f->word[tid] = word;
        __syncthreads();
        const int here = min(all, total - base);
        for (int r = tid; r < here; r += kPoolThreads) {
            int lo = 0, hi = kPoolThreads;           // last word with first <= r
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (f->first[mid] <= r) lo = mid;
                else hi = mid;
            }
            give(base + r, (w0 + lo) * 32 + nth_bit(f->word[lo], r - f->first[lo]));
        }
        // what stays of this thread's word
        if (c && first < here) {
            int gone = min(c, here - first);
            if (gone == c) word = 0u;
            for (; word && gone; --gone) word &= word - 1;
            bits[w] = word;
        }
        base += all;
        __syncthreads();
    }
}

// Request that rank r falls to: the last i with first[i] <= r (first = exclusive prefix sums).
__device__ __forceinline__ int owner_of(const int *first, int n, int r)
{
    int lo = 0, hi = n;          // first[lo] <= r
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct PoolParams {
    int32_t *table, *seq_len, *seq_pages, *refs;
    uint32_t *bits;
    const int32_t *extra;        // resize
    const int32_t *src, *dst;    // fork
    int32_t *status;
    int n;                       // sequences (resize) or pairs (fork)
    int seqs, num_pages, table_width, page_size, page_log2;
};

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Pages that a sequence with `held` pages shall hold; -1: the request does not fit its table row.
__device__ __forceinline__ int resize_want(const PoolParams &p, int extra, int len, int held)
{
    if (extra < -1) return held;
    if (extra == -1) return 0;
    const int64_t pages = ((int64_t)max(len, 0) + extra + p.page_size - 1) >> p.page_log2;
    return pages > p.table_width ? -1 : (int)pages;
}

// One cluster of eight blocks.  First all of it gives pages back (counts and free
// bits are changed by commutative integer atomics, so the order is immaterial); the cluster barrier
// makes that visible; then its first block serves the growing requests from the lowest free pages,
// found by a prefix sum over the bit set.  No order of threads shows in the result.
__global__ void __cluster_dims__(kPoolCluster, 1, 1) __launch_bounds__(kPoolThreads) kv_resize_kernel(const PoolParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ int s_first[];   // [n]
    __shared__ int s_warp[32];
    __shared__ FreeTile s_free;
    const int lane = threadIdx.x & 31;
    // a lane per sequence decides, then the warp gives back the pages of one sequence after the other
    constexpr int kLanes = 8;           // sequences per warp and round: more warps share the rows of a round
    const int warps = kPoolCluster * (kPoolThreads / 32), warp = blockIdx.x * (kPoolThreads / 32) + (threadIdx.x >> 5);
    for (int b0 = warp * kLanes; b0 < p.n; b0 += warps * kLanes) {
        const int b = b0 + lane;
        int held = 0, want = 0;
        bool drop = false;
        if (lane < kLanes && b < p.n) {
            const int ex = p.extra[b], pages = p.seq_pages[b], len = p.seq_len[b];
            held = min(max(pages, 0), p.table_width);
            want = resize_want(p, ex, len, held);
            drop = want >= 0 && want < held;
            if (drop) p.seq_pages[b] = want;
            if (ex == -1) p.seq_len[b] = 0;
            if (p.status && want <= held) p.status[b] = want < 0 ? MARS_SEQ_NO_ROOM : MARS_SEQ_OK;
        }
        for (unsigned left = __ballot_sync(0xffffffffu, drop); left; left &= left - 1) {
            const int i = __ffs((int)left) - 1;
            const int from = __shfl_sync(0xffffffffu, want, i), upto = __shfl_sync(0xffffffffu, held, i);
            int32_t *row = p.table + (int64_t)(b0 + i) * p.table_width;
#pragma unroll 8
            for (int c = from + lane; c < upto; c += 32) {
                const int id = row[c];
                row[c] = -1;
                if ((unsigned)id < (unsigned)p.num_pages && atomicSub(p.refs + id, 1) == 1)
                    atomicOr(p.bits + (id >> 5), 1u << (id & 31));
            }
        }
    }
    __threadfence();
    cluster_barrier();
    if (blockIdx.x != 0) return;

    for (int b = threadIdx.x; b < p.n; b += kPoolThreads) {
        const int ex = p.extra[b], pages = __ldcg(p.seq_pages + b), len = __ldcg(p.seq_len + b);
        const int held = min(max(pages, 0), p.table_width), want = ex >= 0 ? resize_want(p, ex, len, held) : held;
        s_first[b] = max(want - held, 0);
    }
    __syncthreads();
    const int total = block_exclusive_scan(s_first, p.n, s_warp);
    if (total == 0) return;
    const int words = (p.num_pages + 31) >> 5;
    const int have = count_free(p.bits, words, total, s_warp);
    // requests are served in order while they fit: those whose pages end at or before `have`
    auto need_of = [&](int i) { return (i + 1 < p.n ? s_first[i + 1] : total) - s_first[i]; };
    int taken = total;
    if (have < total) {      // the last request that fits ends the list
        const int i = owner_of(s_first, p.n, have);          // have < total: i is the request that breaks off
        taken = s_first[i];
        // rank `have` may be the first of request i, or inside it; in both cases i is not served
    }
    take_free(p.bits, words, taken, &s_free, [&](int rank, int page) {
        if (page >= p.num_pages) return;
        const int i = owner_of(s_first, p.n, rank);
        const int held = min(max(__ldcg(p.seq_pages + i), 0), p.table_width);
        p.table[(int64_t)i * p.table_width + held + (rank - s_first[i])] = page;
        p.refs[page] = 1;
    });
    __syncthreads();
    for (int b = threadIdx.x; b < p.n; b += kPoolThreads) {
        const int need = need_of(b);
        if (need == 0) continue;
        const bool ok = s_first[b] + need <= taken;
        if (ok) p.seq_pages[b] = min(max(__ldcg(p.seq_pages + b), 0), p.table_width) + need;
        if (p.status) p.status[b] = ok ? MARS_SEQ_OK : MARS_SEQ_OUT_OF_PAGES;
    }
}

constexpr int kForkEmpty = -1;   // status inside the kernel: a sound pair whose source has no tokens

// One block: validate and claim, find the new last pages, write tables and counts.
__global__ void __launch_bounds__(kPoolThreads) kv_fork_kernel(const PoolParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ int s_first[];   // [n]
    __shared__ int s_warp[32];
    __shared__ FreeTile s_free;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarps = kPoolThreads / 32;
    // 1. what is wrong with a pair taken by itself (a warp per pair); sources as they stand
    for (int i = warp; i < p.n; i += kWarps) {
        const int s = p.src[i], d = p.dst[i];
        bool ok = (unsigned)s < (unsigned)p.seqs && (unsigned)d < (unsigned)p.seqs && s != d;
        int len = 0;
        if (ok) {
            const int held = p.seq_pages[s], there = p.seq_pages[d];
            len = p.seq_len[s];
            const int64_t pages = ((int64_t)len + p.page_size - 1) >> p.page_log2;
            ok = len >= 0 && pages <= held && pages <= p.table_width && there == 0;
            if (ok) {
                const int32_t *row = p.table + (int64_t)s * p.table_width;
#pragma unroll 4
                for (int c = lane; c < (int)pages; c += 32)
                    if ((unsigned)row[c] >= (unsigned)p.num_pages) ok = false;
            }
        }
        ok = __all_sync(0xffffffffu, ok);
        if (lane == 0) p.status[i] = !ok ? MARS_SEQ_BAD_FORK : len == 0 ? kForkEmpty : MARS_SEQ_OK;
    }
    __syncthreads();
    // 2. of several pairs with one destination the first claims it: its page count, 0 so far, takes
    //    the smallest of the (negative) claim numbers
    for (int i = threadIdx.x; i < p.n; i += kPoolThreads)
        if (p.status[i] != MARS_SEQ_BAD_FORK) atomicMin(p.seq_pages + p.dst[i], i - 0x7fffffff);
    __syncthreads();
    for (int i = threadIdx.x; i < p.n; i += kPoolThreads) {
        int need = 0;
        if (p.status[i] != MARS_SEQ_BAD_FORK) {
            if (__ldcg(p.seq_pages + p.dst[i]) != i - 0x7fffffff) p.status[i] = MARS_SEQ_BAD_FORK;
            else if (p.status[i] != kForkEmpty) need = (p.seq_len[p.src[i]] & (p.page_size - 1)) != 0;
        }
        s_first[i] = need;
    }
    __syncthreads();
    const int total = block_exclusive_scan(s_first, p.n, s_warp);
    const int words = (p.num_pages + 31) >> 5;
    const int have = total ? count_free(p.bits, words, total, s_warp) : 0;
    auto need_of = [&](int i) { return (i + 1 < p.n ? s_first[i + 1] : total) - s_first[i]; };
    const int taken = min(have, total);    // needs are 0 or 1: every rank below `have` ends its request
    take_free(p.bits, words, taken, &s_free, [&](int rank, int page) {
        if (page >= p.num_pages) return;
        const int i = owner_of(s_first, p.n, rank);
        const int len = p.seq_len[p.src[i]];
        p.table[(int64_t)p.dst[i] * p.table_width + (len >> p.page_log2)] = page;
        p.refs[page] = 1;
    });
    __syncthreads();
    // 3. shared pages: table entries and counts.  A source that is also a destination holds no pages,
    //    so its pair is refused or marked empty, and nothing of it is read while it is written here.
    for (int i = warp; i < p.n; i += kWarps) {
        const int st = p.status[i];
        if (st == MARS_SEQ_BAD_FORK) continue;
        const int s = p.src[i], d = p.dst[i], need = need_of(i);
        __syncwarp();
        if (st == kForkEmpty) {
            if (lane == 0) { p.status[i] = MARS_SEQ_OK; p.seq_len[d] = 0; p.seq_pages[d] = 0; }
            continue;
        }
        if (need && s_first[i] >= taken) {
            __syncwarp();
            if (lane == 0) { p.status[i] = MARS_SEQ_OUT_OF_PAGES; p.seq_pages[d] = 0; }
            continue;
        }
        const int len = p.seq_len[s], full = len >> p.page_log2;
        __syncwarp();
#pragma unroll 4
        for (int c = lane; c < full; c += 32) {
            const int id = p.table[(int64_t)s * p.table_width + c];
            p.table[(int64_t)d * p.table_width + c] = id;
            atomicAdd(p.refs + id, 1);
        }
        if (lane == 0) {
            p.seq_len[d] = len;
            p.seq_pages[d] = full + need;
        }
    }
}

struct ForkCopyParams {
    KvView kv;
    const int32_t *src, *dst, *status;
    int pairs;
};

// The ragged last page's rows, a block per (pair, layer), a warp per 16-token block of a head at a
// time; partly filled blocks are copied row by row so that no byte behind the rows is touched.
template <int D>
__global__ void __launch_bounds__(256) kv_fork_copy_kernel(const ForkCopyParams p)
{
    pdl_launch_dependents();
    pdl_wait();
    const int i = blockIdx.x, lay = blockIdx.y;
    if (p.status[i] != MARS_SEQ_OK) return;
    const int s = p.src[i], d = p.dst[i], len = p.kv.seq_len[d];
    const int page = 1 << p.kv.page_log2, tail = len & (page - 1), first = len - tail;
    if (!tail) return;
    const int ids = kv_page_id(p.kv, s, first), idd = kv_page_id(p.kv, d, first);
    if (ids < 0 || idd < 0) return;
    unsigned char *layer = p.kv.pages + lay * p.kv.layer_bytes;
    const int blocks = (tail + 15) >> 4;
    const int lane = threadIdx.x & 31;
    constexpr int kChunks = kv_block_bytes(D) / 16, kPer = (kChunks + 31) / 32;
    for (int w = threadIdx.x >> 5; w < blocks * p.kv.kv_heads; w += blockDim.x >> 5) {
        const int h = w / blocks, blk = w % blocks, rows = min(16, tail - 16 * blk);
        const unsigned char *from = kv_block<D>(p.kv, layer, ids, h, first + 16 * blk);
        unsigned char *to = kv_block<D>(p.kv, layer, idd, h, first + 16 * blk);
        uint4 v[kPer];
#pragma unroll
        for (int u = 0; u < kPer; ++u)
            if (u * 32 + lane < kChunks) v[u] = reinterpret_cast<const uint4 *>(from)[u * 32 + lane];
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int at = (u * 32 + lane) * 16;
            if (at >= kv_block_bytes(D)) continue;
            // rows that the 16 bytes belong to: codes D/2 bytes a row, scales D/16
            const bool code = at < 16 * D;
            const int in = code ? at % (8 * D) : (at - 16 * D) % D, width = code ? D / 2 : D / 16;
            const int r0 = in / width, r1 = (in + 15) / width;
            if (r1 < rows) {
                *reinterpret_cast<uint4 *>(to + at) = v[u];
            } else if (r0 < rows) {        // scales: 2 or 4 rows share 16 bytes
                const uint32_t q[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
                constexpr int kWords = D / 64;   // words of a row's scales
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (r0 + k / kWords < rows) reinterpret_cast<uint32_t *>(to + at)[k] = q[k];
            }
        }
    }
}

template <class K, class P>
static mars_status_t kv_launch(K kernel, dim3 grid, int block, size_t smem, cudaStream_t st, const P &p)
{
    const cudaError_t e = launch_pdl(hook(kHookNoOverlap) == 0, kernel, grid, dim3(block), smem, st, p);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return MARS_ERR_CUDA; }
    return MARS_OK;
}

// Rows and heads of a caller's tensor on 16-byte boundaries.
static bool kv_rows_aligned(const void *p, int64_t row, int64_t head, int dt)
{
    const int es = elem_bytes(dt);
    return !((uintptr_t)p & 15) && !((row * es) & 15) && !((head * es) & 15);
}

}  // namespace mars

using namespace mars;

extern "C" {

size_t mars_kv_pool_bytes(int layers, int num_pages, int kv_heads, int head_dim, int page_size)
{
    if (layers < 1 || num_pages < 1 || kv_heads < 1 || (head_dim != 64 && head_dim != 128) || kv_page_log2(page_size) < 0 ||
        num_pages > (1 << 30) || kv_heads > 1024 || layers > 4096)
        return 0;
    return (size_t)kv_pool_bytes(layers, num_pages, kv_heads, head_dim, page_size);
}

mars_status_t mars_kv_append(const mars_kv_cache_t *cache, int layer, const void *k, int64_t k_row, int64_t k_head,
                             const void *v, int64_t v_row, int64_t v_head, int dt, int B, int N, const int32_t *count,
                             int32_t *seq_status, void *cuda_stream)
{
    const mars_status_t cs = kv_check(cache);
    if (cs != MARS_OK) return cs;
    if (!k || !v || B < 1 || N < 1 || B > cache->seqs || layer < 0 || layer >= cache->layers) return MARS_ERR_INVALID_ARG;
    if (!kv_dtype_ok(dt) || N > (1 << 24)) return MARS_ERR_UNSUPPORTED;
    if (!kv_rows_aligned(k, k_row, k_head, dt) || !kv_rows_aligned(v, v_row, v_head, dt)) return MARS_ERR_INVALID_ARG;
    AppendParams p;
    p.kv = kv_view(cache);
    p.layer = p.kv.pages + layer * p.kv.layer_bytes;
    p.scales = cache->scales + (int64_t)layer * 2 * cache->kv_heads;
    p.src[0] = (const unsigned char *)k; p.src[1] = (const unsigned char *)v;
    p.row[0] = k_row; p.row[1] = v_row; p.head[0] = k_head; p.head[1] = v_head;
    p.count = count; p.status = seq_status; p.N = N;
    const int es = elem_bytes(dt);
    p.wide = !(((uintptr_t)k | (uintptr_t)v | (uintptr_t)(k_row * es) | (uintptr_t)(k_head * es) | (uintptr_t)(v_row * es) |
                (uintptr_t)(v_head * es)) & 31);
    int rows = rows_at_once(cache->kv_heads * 2 * (cache->head_dim / 16));
    p.iters = row_iters((int64_t)B * ((N + rows - 1) / rows));
    rows *= p.iters;
    const dim3 grid((unsigned)((N + rows - 1) / rows), B);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (cache->head_dim == 128)
        return dt == MARS_BF16   ? kv_launch(kv_append_kernel<128, MARS_BF16>, grid, 256, 0, st, p)
               : dt == MARS_FP32 ? kv_launch(kv_append_kernel<128, MARS_FP32>, grid, 256, 0, st, p)
                                 : kv_launch(kv_append_kernel<128, MARS_FP16>, grid, 256, 0, st, p);
    return dt == MARS_BF16   ? kv_launch(kv_append_kernel<64, MARS_BF16>, grid, 256, 0, st, p)
           : dt == MARS_FP32 ? kv_launch(kv_append_kernel<64, MARS_FP32>, grid, 256, 0, st, p)
                             : kv_launch(kv_append_kernel<64, MARS_FP16>, grid, 256, 0, st, p);
}

mars_status_t mars_kv_commit(const mars_kv_cache_t *cache, const int32_t *path_nodes, int path_width,
                             const int32_t *accept_len, int B, int32_t *new_len, int32_t *seq_status, void *cuda_stream)
{
    const mars_status_t cs = kv_check(cache);
    if (cs != MARS_OK) return cs;
    if (!accept_len || !new_len || B < 1 || B > cache->seqs || (path_nodes && path_width < 1)) return MARS_ERR_INVALID_ARG;
    CommitParams p;
    p.kv = kv_view(cache);
    p.path = path_nodes; p.path_width = path_width; p.accept_len = accept_len;
    p.new_len = new_len; p.status = seq_status; p.B = B; p.layers = path_nodes ? cache->layers : 1;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int64_t warps = (int64_t)B * p.layers * cache->kv_heads, blocks = (warps + 3) / 4;
    if (blocks > 0x7fffffff) return MARS_ERR_UNSUPPORTED;
    const mars_status_t r = cache->head_dim == 128
                                ? kv_launch(kv_commit_kernel<128>, dim3((unsigned)blocks), 128, 0, st, p)
                                : kv_launch(kv_commit_kernel<64>, dim3((unsigned)blocks), 128, 0, st, p);
    if (r != MARS_OK || new_len != cache->seq_len) return r;
    return kv_launch(kv_commit_len_kernel, dim3((B + 7) / 8), 256, 0, st, p);
}

static PoolParams pool_params(const mars_kv_cache_t *c)
{
    PoolParams p = {};
    p.table = c->block_table; p.seq_len = c->seq_len; p.seq_pages = c->seq_pages; p.refs = c->page_refs;
    p.bits = c->free_bits; p.seqs = c->seqs; p.num_pages = c->num_pages; p.table_width = c->table_width;
    p.page_size = c->page_size; p.page_log2 = kv_page_log2(c->page_size);
    return p;
}

mars_status_t mars_kv_resize(const mars_kv_cache_t *cache, const int32_t *extra, int32_t *seq_status, void *cuda_stream)
{
    const mars_status_t cs = kv_check(cache);
    if (cs != MARS_OK) return cs;
    if (!extra) return MARS_ERR_INVALID_ARG;
    PoolParams p = pool_params(cache);
    p.extra = extra; p.status = seq_status; p.n = cache->seqs;
    return kv_launch(kv_resize_kernel, dim3(kPoolCluster), kPoolThreads, sizeof(int) * cache->seqs, (cudaStream_t)cuda_stream, p);
}

mars_status_t mars_kv_fork(const mars_kv_cache_t *cache, const int32_t *src, const int32_t *dst, int pairs, int32_t *status,
                           void *cuda_stream)
{
    const mars_status_t cs = kv_check(cache);
    if (cs != MARS_OK) return cs;
    if (!src || !dst || !status || pairs < 1) return MARS_ERR_INVALID_ARG;
    if (pairs > MARS_KV_MAX_SEQS) return MARS_ERR_UNSUPPORTED;
    PoolParams p = pool_params(cache);
    p.src = src; p.dst = dst; p.status = status; p.n = pairs;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const mars_status_t r = kv_launch(kv_fork_kernel, dim3(1), kPoolThreads, sizeof(int) * pairs, st, p);
    if (r != MARS_OK) return r;
    ForkCopyParams c;
    c.kv = kv_view(cache); c.src = src; c.dst = dst; c.status = status; c.pairs = pairs;
    const dim3 grid(pairs, cache->layers);
    return cache->head_dim == 128 ? kv_launch(kv_fork_copy_kernel<128>, grid, 256, 0, st, c)
                                  : kv_launch(kv_fork_copy_kernel<64>, grid, 256, 0, st, c);
}

mars_status_t mars_kv_gather(const mars_kv_cache_t *cache, int layer0, int layers, int B, const int32_t *start,
                             const int32_t *count, int rows, void *k_out, void *v_out, int dt, void *cuda_stream)
{
    const mars_status_t cs = kv_check(cache);
    if (cs != MARS_OK) return cs;
    if (!k_out || !v_out || B < 1 || B > cache->seqs || rows < 1 || layer0 < 0 || layers < 1 || layers > cache->layers - layer0)
        return MARS_ERR_INVALID_ARG;
    if (((uintptr_t)k_out & 15) || ((uintptr_t)v_out & 15)) return MARS_ERR_INVALID_ARG;
    if (!kv_dtype_ok(dt) || rows > (1 << 24)) return MARS_ERR_UNSUPPORTED;
    GatherParams p;
    p.kv = kv_view(cache);
    p.layer0 = layer0; p.start = start; p.count = count; p.B = B; p.rows = rows;
    p.dst[0] = (unsigned char *)k_out; p.dst[1] = (unsigned char *)v_out;
    p.wide = !(((uintptr_t)k_out | (uintptr_t)v_out) & 31);
    int per_block = rows_at_once(cache->kv_heads * 2 * (cache->head_dim / 16));
    p.iters = row_iters((int64_t)B * layers * ((rows + per_block - 1) / per_block));
    per_block *= p.iters;
    const dim3 grid((unsigned)((rows + per_block - 1) / per_block), B, layers);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (cache->head_dim == 128)
        return dt == MARS_BF16   ? kv_launch(kv_gather_kernel<128, MARS_BF16>, grid, 256, 0, st, p)
               : dt == MARS_FP32 ? kv_launch(kv_gather_kernel<128, MARS_FP32>, grid, 256, 0, st, p)
                                 : kv_launch(kv_gather_kernel<128, MARS_FP16>, grid, 256, 0, st, p);
    return dt == MARS_BF16   ? kv_launch(kv_gather_kernel<64, MARS_BF16>, grid, 256, 0, st, p)
           : dt == MARS_FP32 ? kv_launch(kv_gather_kernel<64, MARS_FP32>, grid, 256, 0, st, p)
                             : kv_launch(kv_gather_kernel<64, MARS_FP16>, grid, 256, 0, st, p);
}

}  // extern "C"
