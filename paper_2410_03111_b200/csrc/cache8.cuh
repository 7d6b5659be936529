// Uncompressed layers in 8 bits: where rows and scales live, and how codes become numbers.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

#define LORC_BLOCK8 LORC_CACHE8_BLOCK

// Mirrors lorc_cache8, device-usable.  Contiguous caches have page_size 0; rows are n bytes, scales n_kv floats per block.
struct Cache8View {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    const int32_t* page_table;
    const int32_t* seq_lens;
    int batch, max_seq_len, page_size, max_pages_per_seq, n_pages, type, n, n_kv;
    long long seq_stride, capacity;
};

// Number of the block (of 16 rows) that holds positions 16 blk .. of sequence s, in the cache's order of blocks; -1: it lies
// outside the capacity or its page outside the pool.  Row i of the block is row 16 * number + i of the codes, and its scales
// start at number * n_kv.
// FROM_L2: for a kernel that asks before it has waited for the one in front (and knows that nothing is being written there).
template <bool FROM_L2 = false>
__device__ __forceinline__ long long lorc_block8(const Cache8View& c, int s, int blk) {
    const long long pos = (long long)blk * LORC_BLOCK8;
    if (blk < 0 || pos >= c.capacity) return -1;
    if (c.page_table == nullptr) return (long long)s * (c.seq_stride / LORC_BLOCK8) + blk;
    const int per = c.page_size / LORC_BLOCK8, lp = blk / per;
    const int32_t* at = c.page_table + (long long)s * c.max_pages_per_seq + lp;
    const int page = FROM_L2 ? __ldcg(at) : *at;
    if (page < 0 || page >= c.n_pages) return -1;
    return (long long)page * per + (blk - lp * per);
}

// Cached tokens of sequence s that count: a sequence that is too long for anything that bounds it is empty (and reported).
__device__ __forceinline__ int lorc_len8(const Cache8View& c, int s, int max_pos, int* status) {
    const int len = c.seq_lens[s];
    if (len > c.max_seq_len || len > max_pos || len > c.capacity) {
        if (status) lorc_set_status(status, LORC_ERR_CAPACITY);
        return 0;
    }
    return len < 0 ? 0 : len;
}

// Four codes (the bytes of x, lowest first) as fp16, exactly: a = codes I0, I1, b = codes I2, I3.  Integers: the byte with its
// sign bit turned over is code + 128; behind the byte 0x64 it is the fp16 number 1024 + code + 128.
template <bool E4M3, int I0, int I1, int I2, int I3>
__device__ __forceinline__ void lorc_codes_half(uint32_t x, uint32_t& a, uint32_t& b) {
    if (E4M3) {
        const uint32_t y = (I0 == 0 && I1 == 1 && I2 == 2 && I3 == 3) ? x : __byte_perm(x, 0, I0 | I1 << 4 | I2 << 8 | I3 << 12);
        asm("{\n\t"
            ".reg .b16 l, h;\n\t"
            "mov.b32 {l, h}, %2;\n\t"
            "cvt.rn.f16x2.e4m3x2 %0, l;\n\t"
            "cvt.rn.f16x2.e4m3x2 %1, h;\n\t"
            "}\n"
            : "=r"(a), "=r"(b)
            : "r"(y));
    } else {
        x ^= 0x80808080u;
        const __half2 bias = __half2half2(__ushort_as_half(0x6480));        // 1024 + 128
        uint32_t u = __byte_perm(x, 0x64646464u, I0 | 4 << 4 | I1 << 8 | 4 << 12);
        uint32_t w = __byte_perm(x, 0x64646464u, I2 | 4 << 4 | I3 << 8 | 4 << 12);
        const __half2 p = __hsub2(*reinterpret_cast<__half2*>(&u), bias), q = __hsub2(*reinterpret_cast<__half2*>(&w), bias);
        a = *reinterpret_cast<const uint32_t*>(&p);
        b = *reinterpret_cast<const uint32_t*>(&q);
    }
}

// Two fp32 numbers, rounded to the nearest codes (ties to even), the first one in the lower byte.  They do not exceed the largest
// code (a NaN becomes 0, what is larger the largest code).
template <bool E4M3>
__device__ __forceinline__ uint32_t lorc_to_codes2(float x, float y) {
    x = x == x ? x : 0.f;
    y = y == y ? y : 0.f;
    if (E4M3) {
        uint16_t r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(x), "f"(y));
        return r;
    }
    const int a = __float2int_rn(fminf(fmaxf(x, -127.f), 127.f)), b = __float2int_rn(fminf(fmaxf(y, -127.f), 127.f));
    return (uint32_t)(a & 0xff) | (uint32_t)(b & 0xff) << 8;
}

// Smallest power of two 2^e, -100 <= e <= 100, with most <= largest * 2^e; most >= 0 and finite.  The largest code is
// 1.984375 * 2^6 (127) or 1.75 * 2^8 (448): with most = f * 2^k, 1 <= f < 2, e is k - 6 (k - 8) where f does not exceed its
// factor, else one more.
template <bool E4M3>
__device__ __forceinline__ float lorc_scale8(float most) {
    const uint32_t b = __float_as_uint(most), f = b & 0x7fffffu;
    int e = (int)(b >> 23) - 127 - (E4M3 ? 8 : 6) + (f > (E4M3 ? 0x600000u : 0x7e0000u) ? 1 : 0);
    e = e < -100 ? -100 : e > 100 ? 100 : e;            // (zero and subnormal numbers have the lowest exponent)
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// ---- host side ----------------------------------------------------------------------------------------------------------
// Projection and quantisation (append8.cu): x [batch, T, D] -> codes.  Scratch of a call, and of any call with at most as many
// sequences and tokens.
enum Append8Way { APPEND8_MMA, APPEND8_SPLIT, APPEND8_TC };
Append8Way lorc_append8_way(const lorc_ctx* ctx, int batch, int T);
size_t lorc_append8_scratch_bytes(const lorc_ctx* ctx, int batch, int T);
size_t lorc_append8_scratch_most(const lorc_ctx* ctx, int batch, int T);
cudaError_t lorc_append8_launch(lorc_ctx* ctx, const LorcLayer& L, const Cache8View& cv, const bf16* x, int T, void* scratch,
                                cudaStream_t st, int* launches);

// Attention of T >= 1 queries per sequence on mma.sync (decode8.cu): query t of a sequence is the decode query of the sequence cut
// after that token, and lorc_decode8_queries of them share a pass over the sequence.
int lorc_decode8_queries(const lorc_ctx* ctx, int T);
bool lorc_decode8_fits(const lorc_ctx* ctx, const Cache8View& cv, int T);      // the list of its work has fewer than 2^30 units
size_t lorc_decode8_scratch_bytes(const lorc_ctx* ctx, int batch, int max_seq_len, int T);
cudaError_t lorc_decode8_launch(lorc_ctx* ctx, const Cache8View& cv, const bf16* q, bf16* out, int T, void* scratch,
                                cudaStream_t st, int* launches);

// Attention of prompt chunks on tcgen05 (prefill8.cu).  Scratch of a call, and of any call with at most as many sequences, tokens and
// queries.
bool lorc_prefill8_supported(const lorc_ctx* ctx, const Cache8View& cv, int T);
size_t lorc_prefill8_scratch_bytes(const lorc_ctx* ctx, int batch, int max_seq_len, int T);
size_t lorc_prefill8_scratch_most(const lorc_ctx* ctx, int batch, int max_seq_len, int T);
cudaError_t lorc_prefill8_launch(lorc_ctx* ctx, const Cache8View& cv, const bf16* q, bf16* out, int T, void* scratch,
                                 cudaStream_t st, int* launches);
