// Layout and number formats of the paged 4-bit KV cache, shared by the kernels that write it, move
// it and attend over it, and the host checks of the cache descriptor.
//
// A block is 16 tokens of one KV head, 18*d bytes:
//   K codes [16][d/2] | V codes [16][d/2] | K scales [16][d/16] | V scales [16][d/16]
// Keeping 16 tokens' codes and scales in one run of 2304 (1152) bytes makes a page one contiguous
// run per head and lets a warp fetch everything it needs for 16 keys with five 16-byte copies a lane.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "mars_kv.h"

namespace mars {

constexpr int kKvBlock = 16;   // tokens per block

__host__ __device__ constexpr int kv_block_bytes(int d) { return 18 * d; }

inline int kv_page_log2(int page_size)
{
    return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : page_size == 128 ? 7 : -1;
}

// Bytes of one layer of the pool for sizes that each are in range (below 2^55), and of all of it; 0: no 63-bit count.
inline int64_t kv_layer_bytes(int num_pages, int kv_heads, int head_dim, int page_size)
{
    return (int64_t)num_pages * kv_heads * (page_size / kKvBlock) * kv_block_bytes(head_dim);
}
inline int64_t kv_pool_bytes(int layers, int num_pages, int kv_heads, int head_dim, int page_size)
{
    const int64_t layer = kv_layer_bytes(num_pages, kv_heads, head_dim, page_size);
    return layer <= INT64_MAX / layers ? layer * layers : 0;
}

// Host check of a descriptor: what every call needs of it.
inline mars_status_t kv_check(const mars_kv_cache_t *c)
{
    if (!c || !c->pages || !c->scales || !c->block_table || !c->seq_len || !c->seq_pages || !c->page_refs ||
        !c->free_bits)
        return MARS_ERR_INVALID_ARG;
    if (c->layers < 1 || c->num_pages < 1 || c->kv_heads < 1 || c->seqs < 1 || c->table_width < 1)
        return MARS_ERR_INVALID_ARG;
    if (((uintptr_t)c->pages & 15) || ((uintptr_t)c->scales & 3) || ((uintptr_t)c->block_table & 3) ||
        ((uintptr_t)c->seq_len & 3) || ((uintptr_t)c->seq_pages & 3) || ((uintptr_t)c->page_refs & 3) ||
        ((uintptr_t)c->free_bits & 3))
        return MARS_ERR_INVALID_ARG;
    if ((c->head_dim != 64 && c->head_dim != 128) || kv_page_log2(c->page_size) < 0) return MARS_ERR_UNSUPPORTED;
    // positions (table_width * page_size) stay below 2^30, page ids below 2^30; the pages that all sequences
    // together may ask for (seqs * table_width) below 2^31, since the prefix sums over them are 32-bit
    if (c->seqs > MARS_KV_MAX_SEQS || c->num_pages > (1 << 30) || c->kv_heads > 1024 || c->layers > 4096 ||
        (long long)c->table_width * c->page_size > (1ll << 30) || (long long)c->seqs * c->table_width >= (1ll << 31))
        return MARS_ERR_UNSUPPORTED;
    if (kv_pool_bytes(c->layers, c->num_pages, c->kv_heads, c->head_dim, c->page_size) == 0) return MARS_ERR_UNSUPPORTED;
    return MARS_OK;
}

// What the kernels need to find a token's block; by value in kernel parameters.
struct KvView {
    unsigned char *pages;      // of layer 0
    const int32_t *table;
    const int32_t *seq_len;
    const int32_t *seq_pages;
    const float *scales;       // [layers][2][kv_heads]
    int64_t layer_bytes;
    int num_pages, kv_heads, table_width, page_log2;
};

inline KvView kv_view(const mars_kv_cache_t *c)
{
    KvView v;
    v.pages = (unsigned char *)c->pages;
    v.table = c->block_table;
    v.seq_len = c->seq_len;
    v.seq_pages = c->seq_pages;
    v.scales = c->scales;
    v.page_log2 = kv_page_log2(c->page_size);
    v.layer_bytes = kv_layer_bytes(c->num_pages, c->kv_heads, c->head_dim, c->page_size);
    v.num_pages = c->num_pages;
    v.kv_heads = c->kv_heads;
    v.table_width = c->table_width;
    return v;
}

// Tokens that sequence b's pages hold (its table row never reaches beyond table_width entries).
__device__ __forceinline__ int kv_capacity(const KvView &v, int b)
{
    return min(max(v.seq_pages[b], 0), v.table_width) << v.page_log2;
}

// Page id of the block that holds position pos, or -1 if the table names no page of the pool there.
__device__ __forceinline__ int kv_page_id(const KvView &v, int b, int pos)
{
    const int id = v.table[(int64_t)b * v.table_width + (pos >> v.page_log2)];
    return (unsigned)id < (unsigned)v.num_pages ? id : -1;
}

// First byte of the block of position pos (64-bit: a pool passes 2^32 bytes easily).
template <int D>
__device__ __forceinline__ unsigned char *kv_block(const KvView &v, unsigned char *layer, int page_id, int head, int pos)
{
    const int blocks = 1 << (v.page_log2 - 4);
    const int64_t blk = ((int64_t)page_id * v.kv_heads + head) * blocks + ((pos >> 4) & (blocks - 1));
    return layer + blk * kv_block_bytes(D);
}

// ---- number formats (sm_100a conversions)

// Four bytes of E2M1 pairs -> four f16x2 (low nibble in the low half).
__device__ __forceinline__ void e2m1x8_to_f16x2(uint32_t w, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}

// Two E4M3 bytes -> f16x2 (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
    return r;
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// fp32 pair -> f16x2, nearest even (lo in the low half)
__device__ __forceinline__ uint32_t f16x2_from(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float2 f16x2_to_float2(uint32_t h)
{
    float2 f;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
        : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}

__device__ __forceinline__ uint32_t bf16x2_from(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace mars
