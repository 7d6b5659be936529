// Prompt chunks over the 8-bit cache of uncompressed layers: keys and values of the cached tokens are brought to fp16 once per
// call (code x scale has seven significant bits: exact where the scale is a power of two and the number within fp16's normal range),
// then the tcgen05 attention kernel of the latent mode runs over them.  With T queries per sequence each number of the buffer enters up to
// T G products, so the pass over it is small for chunks.
#include <math.h>

#include "cache8.cuh"
#include "sm100_ptx.cuh"
#include "tc_kernels.cuh"

using namespace sm100;

namespace {

struct Expand8Params {
    Cache8View cv;
    uint4 *khat, *vbuf;              // [batch][rows][n] fp16
    int* status;
    long long rows;
    int dh_shift, max_pos, T;
};

// A block of threads per (block of 16 tokens, keys / values): 16 codes per thread and step.  Rows of the buffer behind the
// sequence's end, up to a multiple of 128, become zero: the attention kernel reads whole tiles.
template <bool E4M3>
__global__ void __launch_bounds__(256)
expand8_kernel(const Expand8Params p) {
    const Cache8View& cv = p.cv;
    const int blk = blockIdx.x, s = blockIdx.y;
    const bool val = blockIdx.z != 0;
    grid_dep_wait();
    grid_dep_launch();
    const int len = cv.seq_lens[s];
    // (what the attention kernel treats as empty has no rows to read)
    if (len < p.T || len > cv.max_seq_len || len > p.max_pos) return;
    if (blk * LORC_BLOCK8 >= (len + 127) / 128 * 128) return;
    long long at = -1;
    if (blk * LORC_BLOCK8 < len) {
        at = lorc_block8(cv, s, blk);
        if (at < 0 && threadIdx.x == 0) lorc_set_status(p.status, LORC_ERR_CAPACITY);
    }
    const int per_row = cv.n / 16;                               // pieces of 16 codes
    const uint4* src = reinterpret_cast<const uint4*>(val ? cv.v : cv.k) + at * LORC_BLOCK8 * per_row;
    const float* scale = (val ? cv.v_scale : cv.k_scale) + at * cv.n_kv;
    uint4* dst = (val ? p.vbuf : p.khat) + ((long long)s * p.rows + (long long)blk * LORC_BLOCK8) * per_row * 2;
    __half2 most = __floats2half2_rn(0.f, 0.f);
    for (int i = threadIdx.x; i < LORC_BLOCK8 * per_row; i += 256) {
        const int r = i / per_row, c = i - r * per_row;
        uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
        if (at >= 0 && blk * LORC_BLOCK8 + r < len) {
            const uint4 x = src[i];
            const float f = scale[(c * 16) >> p.dh_shift];
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t a, b;
                lorc_codes_half<E4M3, 0, 1, 2, 3>(in[j], a, b);
                const float2 u = __half22float2(*reinterpret_cast<__half2*>(&a)), v = __half22float2(*reinterpret_cast<__half2*>(&b));
                const __half2 y = __floats2half2_rn(u.x * f, u.y * f), z = __floats2half2_rn(v.x * f, v.y * f);
                most = __hmax2(most, __hmax2(__habs2(y), __habs2(z)));
                w[2 * j] = *reinterpret_cast<const uint32_t*>(&y);
                w[2 * j + 1] = *reinterpret_cast<const uint32_t*>(&z);
            }
            lo = make_uint4(w[0], w[1], w[2], w[3]);
            hi = make_uint4(w[4], w[5], w[6], w[7]);
        }
        dst[2 * i] = lo;
        dst[2 * i + 1] = hi;
    }
    // numbers that fp16 does not hold
    if (fmaxf(__low2float(most), __high2float(most)) > 65504.f) lorc_set_status(p.status, LORC_ERR_ARG);
}

size_t expand8_rows(int max_seq_len) { return ((size_t)max_seq_len + 127) / 128 * 128; }

constexpr int MAX_SPLIT = 16;

// How the units of the attention kernel run: the first `whole` ones on a CTA each, of the others S CTAs share the keys.
struct Split8 {
    long long units, whole;
    int S;
    long long time;              // tenths of a microsecond
};

// A CTA takes 2.2 us per tile of 128 keys and 4 us before and after, whatever runs beside it; the merge 3 us and its traffic.  Either
// all units share their keys among S CTAs, or those that the full rounds of the SMs leave over.  (Whole calls, 8 KV heads of 128
// dimensions in groups of four: the last 128 of 8000 tokens took 144 us with one CTA per unit and 47 as chosen here, 512 of them 146 and
// 99.  8 x 512 tokens behind 3584, 512 units on 148 SMs: 325 us in four rounds, 309 with the last 68 units shared by two CTAs each; 3 to 8 %
// more when calls go on and the power cap lowers the clock.)
Split8 prefill8_split(const lorc_ctx* ctx, int batch, int max_seq_len, int T) {
    const int qp = 2 * (128 / ctx->group);
    const long long P = ctx->sm_count, tiles = ((long long)max_seq_len + 127) / 128;
    Split8 best;
    best.units = best.whole = (long long)batch * ctx->desc.n_kv_heads * ((T + qp - 1) / qp);
    best.S = 1;
    best.time = (best.units + P - 1) / P * (tiles * 22 + 40);
    for (int full = 0; full < 2; ++full) {
        const long long whole = full ? best.units / P * P : 0, rest = best.units - whole;
        if (rest == 0 || (full && whole == 0)) continue;
        for (int S = 2; S <= MAX_SPLIT && 2 * S <= tiles && rest * S <= 2 * P; ++S) {
            const long long time = whole / P * (tiles * 22 + 40) + (rest * S + P - 1) / P * ((tiles + S - 1) / S * 22 + 40) + 30 +
                                   rest * S * LORC_PREFILL_PART_FLOATS * 8 / 500000;
            if (time < best.time) {
                best.whole = whole;
                best.S = S;
                best.time = time;
            }
        }
    }
    return best;
}

size_t expand8_bytes(const lorc_ctx* ctx, int batch, int max_seq_len) {
    return 2 * lorc_align_up((size_t)batch * expand8_rows(max_seq_len) * ctx->n * 2, 256);
}

}  // namespace

// Few queries per sequence are better served by the streaming kernel, which reads the codes once per lorc_decode8_queries of them (from
// L2, mostly) and is then bound by its arithmetic: 0.33 us per 64 tokens, pass and KV head on an SM, against 1.3 us to expand them for
// all queries.  (8 KV heads of 128 dimensions in groups of four, us here and there: 8 x 4096 tokens, 4 queries 31 and 85, 16 queries
// 89 and 85, 32 queries 163 and 87; one sequence of 1000 tokens, 32 queries 15 and 18; of 8000, 32 queries 50 and 39.  8 x 512 queries
// of 4096 tokens 2306 and 309, heads of 64 in groups of four, 1510 and 246; heads of 128 in groups of five 4292 and 432, ungrouped 1171
// and 226.)
bool lorc_prefill8_supported(const lorc_ctx* ctx, const Cache8View& cv, int T) {
    if (T == 1 || cv.batch > 65535 || (ctx->desc.flags & LORC_FLAG_DEBUG_FP32)) return false;
    const long long units = (long long)cv.batch * cv.n_kv * ((cv.max_seq_len + 63) / 64), P = ctx->sm_count;
    const int Q = lorc_decode8_queries(ctx, T);
    const long long stream = 80 + 33 * units * ((T + Q - 1) / Q) / (10 * P);
    const long long expand = 100 + 13 * units / P + prefill8_split(ctx, cv.batch, cv.max_seq_len, T).time;
    return expand < stream;
}

size_t lorc_prefill8_scratch_bytes(const lorc_ctx* ctx, int batch, int max_seq_len, int T) {
    const Split8 split = prefill8_split(ctx, batch, max_seq_len, T);
    return expand8_bytes(ctx, batch, max_seq_len) + (size_t)(split.units - split.whole) * split.S * LORC_PREFILL_PART_FLOATS * sizeof(float);
}

size_t lorc_prefill8_scratch_most(const lorc_ctx* ctx, int batch, int max_seq_len, int T) {
    // a call with fewer sequences or tokens may share more units' keys, among more CTAs: two per SM at most, and MAX_SPLIT per unit
    const size_t qp = 2 * (128 / ctx->group), all = (size_t)batch * ctx->desc.n_kv_heads * ((T + qp - 1) / qp) * MAX_SPLIT;
    const size_t cap = 2 * (size_t)ctx->sm_count;
    return expand8_bytes(ctx, batch, max_seq_len) + (all < cap ? all : cap) * LORC_PREFILL_PART_FLOATS * sizeof(float);
}

cudaError_t lorc_prefill8_launch(lorc_ctx* ctx, const Cache8View& cv, const bf16* q, bf16* out, int T, void* scratch,
                                 cudaStream_t st, int* launches) {
    static bool attr[64] = {false};
    const bool known = ctx->device >= 0 && ctx->device < 64;
    cudaError_t e = cudaSuccess;
    if (!known || !attr[ctx->device]) {
        e = lorc_tc_prefill_set_attrs();
        if (e != cudaSuccess) return e;
        if (known) attr[ctx->device] = true;
    }
    const size_t rows = expand8_rows(cv.max_seq_len);
    Expand8Params p;
    p.cv = cv; p.status = ctx->status_dev; p.rows = (long long)rows; p.max_pos = ctx->desc.max_pos; p.T = T;
    p.khat = (uint4*)scratch;
    const size_t kv = expand8_bytes(ctx, cv.batch, cv.max_seq_len);
    p.vbuf = (uint4*)((char*)scratch + kv / 2);
    p.dh_shift = ctx->desc.d_head == 128 ? 7 : 6;
    const dim3 grid((unsigned)(rows / LORC_BLOCK8), (unsigned)cv.batch, 2);
    e = cv.type == LORC_CACHE8_E4M3 ? lorc_launch_dependent(expand8_kernel<true>, grid, dim3(256), 0, st, p)
                                    : lorc_launch_dependent(expand8_kernel<false>, grid, dim3(256), 0, st, p);
    *launches += 1;
    if (e != cudaSuccess) return e;
    const Split8 split = prefill8_split(ctx, cv.batch, cv.max_seq_len, T);
    return lorc_tc_prefill_attend(ctx, cv.seq_lens, cv.batch, rows, cv.max_seq_len, p.khat, p.vbuf, q, out, T, true, split.whole, split.S,
                                  (float*)((char*)scratch + kv), st, launches);
}
