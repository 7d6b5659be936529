// Where the rows of an 8-bit cache write go, and how numbers become codes there.
#pragma once

#include "cache8.cuh"

struct Append8Params {
    Cache8View cv;
    const float2* rope_table;
    int* status;
    int T, n_blocks, max_pos, interleaved;      // n_blocks: blocks of a sequence that T new tokens can reach
};

// One row (token) of a block.
struct Append8Row {
    long long at;                // number of the block in the cache, -1: there is nothing to write
    int pos;
    bool fresh, old, has_old;    // a new token, an earlier one; whether the block has earlier ones
};

// Row r of the i-th block that the new tokens of sequence s reach (s < 0: none); thread r = 0 reports what is wrong with it.
template <bool FROM_L2 = false>
__device__ __forceinline__ void append8_row(const Append8Params& p, int s, int i, int r, Append8Row& row) {
    row.at = -1;
    row.pos = 0;
    row.fresh = row.old = row.has_old = false;
    if (s < 0) return;
    const int len = FROM_L2 ? __ldcg(p.cv.seq_lens + s) : p.cv.seq_lens[s];
    const bool fits = len >= 0 && len <= p.cv.max_seq_len && len <= p.max_pos && len <= p.cv.capacity;
    // a sequence that is too long, or shorter than what is written to it, is reported; of the latter the tokens that have a place
    // are written
    if ((!fits || len < p.T) && r == 0) lorc_set_status(p.status, LORC_ERR_CAPACITY);
    if (!fits) return;
    const int begin = max(len - p.T, 0), blk = begin / LORC_BLOCK8 + i;
    if (blk * LORC_BLOCK8 >= len) return;
    row.at = lorc_block8<FROM_L2>(p.cv, s, blk);
    if (row.at < 0) {
        if (r == 0) lorc_set_status(p.status, LORC_ERR_CAPACITY);
        return;
    }
    row.pos = blk * LORC_BLOCK8 + r;
    row.fresh = row.pos >= begin && row.pos < len;
    row.old = row.pos < begin;
    row.has_old = begin > blk * LORC_BLOCK8;
}

// The scale of a block and head from the largest magnitude of its new numbers and the scale that its earlier tokens stand under, which
// may be any finite number: the larger one in magnitude.
template <bool E4M3>
__device__ __forceinline__ float append8_scale(float most, float before) {
    const float scale = lorc_scale8<E4M3>(most), m = fabsf(before);
    return m > scale && m <= 3.4028234663852886e38f ? before : scale;
}
// What the codes of the earlier tokens are multiplied by.
__device__ __forceinline__ float append8_keep(float before, float scale) {
    return fabsf(before) <= 3.4028234663852886e38f ? before / scale : 0.f;
}

// Magnitudes of finite numbers for the block's maximum; odd: one of them is not finite.
template <int N>
__device__ __forceinline__ float append8_most(const float (&x)[N], bool& odd) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float m = fabsf(x[i]);
        if (m <= 3.4028234663852886e38f) most = fmaxf(most, m);
        else odd = true;
    }
    return most;
}

// Sixteen numbers (times `inv`) as codes; clean: they are finite and none exceeds the largest code.  Adding 1.5 * 2^23 to a number
// below 2^22 leaves its nearest integer (ties to even) in the lowest bits.
template <bool E4M3>
__device__ __forceinline__ uint4 append8_codes(const float* x, float inv, bool clean) {
    uint32_t w[4];
    if (clean && E4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint16_t lo, hi;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(lo) : "f"(x[4 * i] * inv), "f"(x[4 * i + 1] * inv));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(hi) : "f"(x[4 * i + 2] * inv), "f"(x[4 * i + 3] * inv));
            w[i] = (uint32_t)lo | (uint32_t)hi << 16;
        }
    } else if (clean) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = __float_as_uint(x[4 * i + j] * inv + 12582912.f);
            w[i] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = lorc_to_codes2<E4M3>(x[4 * i] * inv, x[4 * i + 1] * inv) | lorc_to_codes2<E4M3>(x[4 * i + 2] * inv, x[4 * i + 3] * inv) << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Sixteen codes under another scale.
template <bool E4M3>
__device__ __forceinline__ uint4 append8_recode(const uint4& c, float keep) {
    const uint32_t in[4] = {c.x, c.y, c.z, c.w};
    float x[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t a, b;
        lorc_codes_half<E4M3, 0, 1, 2, 3>(in[i], a, b);
        const float2 u = __half22float2(*reinterpret_cast<__half2*>(&a)), v = __half22float2(*reinterpret_cast<__half2*>(&b));
        x[4 * i] = u.x;
        x[4 * i + 1] = u.y;
        x[4 * i + 2] = v.x;
        x[4 * i + 3] = v.y;
    }
    return append8_codes<E4M3>(x, keep, false);
}

// Few tokens, D split over a cluster (append8_split.cu).
bool lorc_append8_split_supported(const lorc_ctx* ctx, int batch, int T);
long long lorc_append8_split_time(const lorc_ctx* ctx, int batch, int T);
cudaError_t lorc_append8_split_launch(lorc_ctx* ctx, const LorcLayer& L, const Append8Params& q, const bf16* x, cudaStream_t st, int* launches);

// Prompt-sized launches (append8_tc.cu).
bool lorc_append8_tc_supported(const lorc_ctx* ctx);
long long lorc_append8_tc_time(const lorc_ctx* ctx, int batch, int T);
cudaError_t lorc_append8_tc_launch(lorc_ctx* ctx, const LorcLayer& L, const Append8Params& q, const bf16* x, cudaStream_t st, int* launches);
