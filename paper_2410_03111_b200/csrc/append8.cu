// Cache write of uncompressed layers in 8 bits: [K | V] = x [W_k | W_v], keys rotated, both rounded to codes with one scale per
// block of 16 tokens and KV head.  Here are the kernels for a handful of tokens, the plain ones, and the choice; batches of steps and
// short prompts run in append8_split.cu, others in append8_tc.cu.
//
// Two kernels.  The projection leaves fp32 numbers [tokens][2 n] in the workspace; the second kernel has a block of threads for each
// (block of tokens, KV head, keys or values), which sees all numbers that share a scale.  16 sequences, D 4096, 8 KV heads of 128
// dimensions: 7.8 us, of which 2.6 are the factor's bytes at the rate of a copy; the rest is two launches in a row, and x through L2
// once per eight columns.
#include <math.h>

#include "append8.cuh"
#include "sm100_ptx.cuh"
#include "tc_kernels.cuh"

using namespace sm100;

namespace {

// ---------------------------------------------------------------------------------------------
// projection for a handful of tokens: grid (2 n / 8, tiles of 16 tokens), eight warps = eight slices of D.  Bound by the stream of
// the factor (in fragment order, see retile_factor_kernel), which is requested before the kernel in front has finished.
// The MMAs sum 128 products at a time, and ordinary additions the pieces: an MMA loses more of its running sum than rounding would.
// (D 8192, products of one sign: off by 2^-19.1 of their sum with 1024 at a time, by 2^-23.3 so; codes that are not the fp64
// projection's 2.5e-4 and 3e-5.  16 x 1 tokens take as long, 1 x 1 5.40 us instead of 5.33.)
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256, 2)
project8_mma_kernel(const bf16* __restrict__ x, const bf16* __restrict__ A_tiled, float* __restrict__ proj, int D, int R,
                    long long n_tok) {
    __shared__ float red[8][32][4];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * 8;
    const long long m0 = (long long)blockIdx.y * 16;
    const int kspan = D / 8, k_begin = warp * kspan, steps = kspan / 32;
    const bool row_lo = m0 + g < n_tok, row_hi = m0 + g + 8 < n_tok;
    const uint4* xa = reinterpret_cast<const uint4*>(x + (m0 + g) * D + k_begin) + t;
    const uint4* xb = reinterpret_cast<const uint4*>(x + (m0 + g + 8) * D + k_begin) + t;
    const uint4* wb = reinterpret_cast<const uint4*>(A_tiled) + ((long long)blockIdx.x * (D / 32) + k_begin / 32) * 32 + lane;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    float c[4] = {0.f, 0.f, 0.f, 0.f};
    uint4 w[16];
    auto load_factor = [&](int kb0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            w[i] = zero;
            if (kb0 + i < steps)
                asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                             : "l"(wb + (kb0 + i) * 32));
        }
    };
    load_factor(0);
    grid_dep_wait();
    grid_dep_launch();
    for (int kb0 = 0; kb0 < steps; kb0 += 16) {
        if (kb0 > 0) load_factor(kb0);
#pragma unroll
        for (int i0 = 0; i0 < 16; i0 += 4) {
            uint4 lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = zero;
                hi[i] = zero;
                if (kb0 + i0 + i < steps) {
                    if (row_lo) lo[i] = xa[(kb0 + i0 + i) * 4];
                    if (row_hi) hi[i] = xb[(kb0 + i0 + i) * 4];
                }
            }
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (kb0 + i0 + i < steps) {
                    mma_bf16_16816(part, lo[i].x, hi[i].x, lo[i].y, hi[i].y, w[i0 + i].x, w[i0 + i].y);
                    mma_bf16_16816(part, lo[i].z, hi[i].z, lo[i].w, hi[i].w, w[i0 + i].z, w[i0 + i].w);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] += part[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[warp][lane][i] = c[i];
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c[i] = ((red[0][lane][i] + red[1][lane][i]) + (red[2][lane][i] + red[3][lane][i])) +
               ((red[4][lane][i] + red[5][lane][i]) + (red[6][lane][i] + red[7][lane][i]));
    const int col = n0 + 2 * t;
    if (row_lo) *reinterpret_cast<float2*>(proj + (m0 + g) * R + col) = make_float2(c[0], c[1]);
    if (row_hi) *reinterpret_cast<float2*>(proj + (m0 + g + 8) * R + col) = make_float2(c[2], c[3]);
}

// The same without conditions on D: thread = column, eight tokens, columns of W as they are.
__global__ void __launch_bounds__(128)
project8_plain_kernel(const bf16* __restrict__ x, const bf16* __restrict__ A_cat, float* __restrict__ proj, int D, int R,
                      long long n_tok) {
    constexpr int TT = 8, CH = 512;
    __shared__ float xs[TT][CH];
    const int tid = threadIdx.x, col = blockIdx.x * 128 + tid;
    const long long tok0 = (long long)blockIdx.y * TT;
    float acc[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t] = 0.f;
    grid_dep_wait();
    grid_dep_launch();
    for (int d0 = 0; d0 < D; d0 += CH) {
        const int dn = min(CH, D - d0);
        for (int i = tid; i < TT * CH; i += 128) {
            const int t = i / CH, d = i - t * CH;
            xs[t][d] = tok0 + t < n_tok && d < dn ? __bfloat162float(x[(tok0 + t) * D + d0 + d]) : 0.f;
        }
        __syncthreads();
        if (col < R)
            for (int d = 0; d < dn; ++d) {
                const float a = __bfloat162float(A_cat[(long long)(d0 + d) * R + col]);
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[t] = fmaf(xs[t][d], a, acc[t]);
            }
        __syncthreads();
    }
    if (col < R)
#pragma unroll
        for (int t = 0; t < TT; ++t)
            if (tok0 + t < n_tok) proj[(tok0 + t) * R + col] = acc[t];
}

// ---------------------------------------------------------------------------------------------
// rotation and quantisation: grid (batch * blocks a chunk can reach, KV heads, keys / values), DH threads.  A thread owns 16 dimensions
// of one of the 16 rows: one 16-byte store.
// ---------------------------------------------------------------------------------------------
template <int DH, bool E4M3>
__global__ void __launch_bounds__(DH)
quantize8_kernel(const Append8Params p, const float* __restrict__ proj, int pairs_adjacent) {
    constexpr int TPR = DH / 16, WARPS = DH / 32;
    __shared__ float most_s[WARPS];
    __shared__ int odd_s[WARPS];
    const Cache8View& cv = p.cv;
    const int tid = threadIdx.x, r = tid / TPR, d0 = (tid % TPR) * 16;
    const int s = (int)blockIdx.x / p.n_blocks, head = blockIdx.y;
    const bool val = blockIdx.z != 0;
    // What does not depend on the projection is looked up while that runs (16 x 1 tokens 8.8 us, now 7.8).  Each of its blocks has waited
    // for the kernels in front of it before it lets this kernel start, and it writes nothing but `proj`; from L2, since what this
    // SM may hold of an earlier kernel's reads is not known to be given up before the wait.
    Append8Row row;
    append8_row<true>(p, s, (int)blockIdx.x % p.n_blocks, r, row);
    float* scale_at = (val ? cv.v_scale : cv.k_scale) + (row.at < 0 ? 0 : row.at) * cv.n_kv + head;
    const float before = row.at >= 0 && row.has_old ? __ldcg(scale_at) : 0.f;
    const bool second = d0 >= DH / 2;
    float2 cs[16];                               // of this thread's dimensions (interleaved: pairs, eight of them)
    if (!val && row.fresh) {
        const float2* at = p.rope_table + (long long)row.pos * (DH / 2) + (p.interleaved ? d0 / 2 : second ? d0 - DH / 2 : d0);
#pragma unroll
        for (int i = 0; i < 16; ++i) cs[i] = i < 8 || !p.interleaved ? at[i] : make_float2(0.f, 0.f);
    }
    grid_dep_wait();
    grid_dep_launch();
    if (row.at < 0) return;                      // (the whole block of threads)
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    if (row.fresh) {
        const float* src = proj + ((long long)s * p.T + (row.pos - (cv.seq_lens[s] - p.T))) * (2 * cv.n) + (val ? cv.n : 0) + head * DH;
        if (val) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(x + i) = *reinterpret_cast<const float4*>(src + d0 + i);
        } else {
            if (p.interleaved) {
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float2 ab = *reinterpret_cast<const float2*>(src + d0 + i), c = cs[i / 2];
                    x[i] = ab.x * c.x - ab.y * c.y;
                    x[i + 1] = ab.x * c.y + ab.y * c.x;
                }
            } else {
                const int j0 = second ? d0 - DH / 2 : d0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = j0 + i;
                    const float a = src[pairs_adjacent ? 2 * j : j], b = src[pairs_adjacent ? 2 * j + 1 : j + DH / 2];
                    const float2 c = cs[i];
                    x[i] = second ? a * c.y + b * c.x : a * c.x - b * c.y;
                }
            }
        }
    }
    bool odd = false;
    float most = append8_most(x, odd);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    const int any_odd = __any_sync(0xffffffffu, odd);
    if ((tid & 31) == 0) {
        most_s[tid >> 5] = most;
        odd_s[tid >> 5] = any_odd;
    }
    __syncthreads();                             // (`before` has been read by all threads: one writes its place)
    int bad = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        most = fmaxf(most, most_s[w]);
        bad |= odd_s[w];
    }
    const float scale = append8_scale<E4M3>(most, before);
    if (tid == 0) {
        *scale_at = scale;
        if (bad) lorc_set_status(p.status, LORC_ERR_ARG);
    }
    uint4* dst = reinterpret_cast<uint4*>((val ? cv.v : cv.k) + (row.at * LORC_BLOCK8 + r) * cv.n + head * DH + d0);
    if (row.fresh) *dst = append8_codes<E4M3>(x, 1.f / scale, false);
    else if (row.old && scale != before) *dst = append8_recode<E4M3>(*dst, append8_keep(before, scale));
}

}  // namespace

// Expected time of the kernels of this file in tenths of a microsecond: every tile of 16 tokens streams the factor.
static long long mma_time(const lorc_ctx* ctx, long long tiles) {
    return 40 + tiles * (2 * ctx->n) * (15 + 28 * ctx->desc.d_model / 4096) / 2048;
}

constexpr long long MMA_TILES = 64;      // (beyond them every way is faster)

// The kernels for a call: those that should take least.  Measured, us, 8 KV heads of 128 dimensions, D 4096 (sequences x tokens), these
// kernels / D split over clusters / prompts: 1 x 1 5.4 / 8.8 / 21, 16 x 1 7.8 / 9.3 / 21, 32 x 1 11.8 / 9.5 / 22, 64 x 1 19 / 10.6 / 22,
// 256 x 1 64 / 16 / 55, 512 x 1 - / 31 / 118, 64 x 4 61 / 16 / 32, 1 x 48 16 / 11 / 21, 1 x 120 35 / 16 / 22, 1 x 250 60 / 25 / 22,
// 16 x 20 - / 48 / 23; D 8192: 16 x 1 12.3 / 12.3 / 37, 32 x 1 21.7 / 13.2 / 37, 128 x 1 59 / 18 / 52; 32 KV heads: 16 x 1 24 / 27 / 24,
// 32 x 1 39 / 28 / 33; 8 KV heads of 64, D 2048: 16 x 1 5.5 / 6.8 / 14, 64 x 1 10.0 / 7.1 / 14.
// (D that is no multiple of 512, or above 8192, has no kernel for split D: batches of single tokens run here once per 16 of
// them, or on the prompts' kernel with one new row in sixteen.)
Append8Way lorc_append8_way(const lorc_ctx* ctx, int batch, int T) {
    const long long tiles = ((long long)batch * T + 15) / 16;
    const bool split = lorc_append8_split_supported(ctx, batch, T), tc = lorc_append8_tc_supported(ctx);
    Append8Way way = APPEND8_MMA;
    long long least = (split || tc) && tiles > MMA_TILES ? 1ll << 62 : mma_time(ctx, tiles);
    if (tc && tiles > 1 && lorc_append8_tc_time(ctx, batch, T) < least) {
        way = APPEND8_TC;
        least = lorc_append8_tc_time(ctx, batch, T);
    }
    if (split && lorc_append8_split_time(ctx, batch, T) < least) way = APPEND8_SPLIT;
    return way;
}

size_t lorc_append8_scratch_bytes(const lorc_ctx* ctx, int batch, int T) {
    if (lorc_append8_way(ctx, batch, T) != APPEND8_MMA) return 0;
    return lorc_align_up((size_t)batch * T * 2 * ctx->n * sizeof(float), 256);
}

size_t lorc_append8_scratch_most(const lorc_ctx* ctx, int batch, int T) {
    // a call with fewer tokens may run on the kernels that need scratch
    long long n = (long long)batch * T;
    if (lorc_append8_tc_supported(ctx) && n > MMA_TILES * 16) n = MMA_TILES * 16;
    return lorc_align_up((size_t)n * 2 * ctx->n * sizeof(float), 256);
}

cudaError_t lorc_append8_launch(lorc_ctx* ctx, const LorcLayer& L, const Cache8View& cv, const bf16* x, int T, void* scratch,
                                cudaStream_t st, int* launches) {
    const int D = ctx->desc.d_model, R = 2 * ctx->n;
    const long long n_tok = (long long)cv.batch * T;
    float* proj = (float*)scratch;
    Append8Params p;
    p.cv = cv; p.rope_table = ctx->rope_table; p.status = ctx->status_dev; p.T = T; p.max_pos = ctx->desc.max_pos;
    p.n_blocks = (T + LORC_BLOCK8 - 2) / LORC_BLOCK8 + 1;
    p.interleaved = ctx->pair_style == LORC_ROPE_INTERLEAVED;
    const Append8Way way = lorc_append8_way(ctx, cv.batch, T);
    if (way == APPEND8_SPLIT) return lorc_append8_split_launch(ctx, L, p, x, st, launches);
    if (way == APPEND8_TC) return lorc_append8_tc_launch(ctx, L, p, x, st, launches);
    const bool mma = D % 256 == 0 && L.A_tiled != nullptr && !(ctx->desc.flags & LORC_FLAG_DEBUG_FP32);
    // grid rows are limited to 65535: chunks of as many tokens
    const int tile = mma ? 16 : 8;
    const long long most = 65535ll * tile;
    for (long long t0 = 0; t0 < n_tok; t0 += most) {
        const long long cnt = n_tok - t0 < most ? n_tok - t0 : most;
        const unsigned y = (unsigned)((cnt + tile - 1) / tile);
        cudaError_t e =
            mma ? lorc_launch_dependent(project8_mma_kernel, dim3(R / 8, y), dim3(256), 0, st, x + t0 * D, (const bf16*)L.A_tiled,
                                        proj + t0 * R, D, R, cnt)
                : lorc_launch_dependent(project8_plain_kernel, dim3((R + 127) / 128, y), dim3(128), 0, st, x + t0 * D,
                                        (const bf16*)L.A_cat, proj + t0 * R, D, R, cnt);
        *launches += 1;
        if (e != cudaSuccess) return e;
    }
    const int adjacent = mma && ctx->pair_style == LORC_ROPE_HALF_SPLIT;
    const dim3 grid((unsigned)((long long)cv.batch * p.n_blocks), (unsigned)cv.n_kv, 2);
    const int DH = ctx->desc.d_head;
    const bool e4m3 = cv.type == LORC_CACHE8_E4M3;
    auto kernel = DH == 128 ? (e4m3 ? quantize8_kernel<128, true> : quantize8_kernel<128, false>)
                            : (e4m3 ? quantize8_kernel<64, true> : quantize8_kernel<64, false>);
    *launches += 1;
    return lorc_launch_dependent(kernel, grid, dim3(DH), 0, st, p, (const float*)proj, adjacent);
}
