// Attention over the 8-bit cache of uncompressed layers, one query per sequence and head, on the warp-level tensor cores.
//
// One pass over 2 n bytes per token, bound by HBM: a block streams (sequence, KV head) pairs; a producer warp keeps
// D8_STAGES 64-token stages of codes in flight by TMA, each of four consumer warps owns 16 of a stage's tokens, which is one block of
// the cache: one scale for its keys, one for its values.  Scores and outputs are computed transposed (tokens, then dimensions on
// the M side of the m16n8k16 tiles, the G <= 8 query heads on the N side).  Codes become fp16 numbers exactly, in registers:
//
//   S^T[16 tok x 8] = K[16 tok x d] . Q^^T      Q^ = RoPE(q, N-1) brought to [1, 2) by a power of two per head, in two fp16 parts
//                                               (22 bits); the scale of the keys, 1 / sqrt(d) and log2 e multiply the fp32 sums
//   p = 2^(S - m), l += p                       m is raised when a score exceeds it by more than 2^8
//   O^T[d x 8]     += V^T[d x 16 tok] . (c p)^T c = scale of the values / largest one so far, c p in two fp16 parts
//
// A 16-bit word of a row is two dimensions.  Key fragments take the dimensions in the order in which ldmatrix delivers bytes, and the
// query fragments take the same order; for the values a transposed 8 x 8 matrix of words holds two dimensions of two tokens per
// register, whose bytes are paired by token: fragment row g is dimension 2 g of the 16, row g + 8 dimension 2 g + 1.
//
// The steps (64 tokens) of all sequences form one list, cut into equal parts for the blocks of a KV head that are resident at
// once: all of them stream from the start to the end of the launch whatever the lengths are.  A part may begin and end inside
// a sequence; what it computes of a sequence that it does not hold alone goes to memory, un-normalised, for a merge kernel.
#include <math.h>

#include "cache8.cuh"
#include "sm100_ptx.cuh"
#include "tc_kernels.cuh"

using namespace sm100;

namespace {

constexpr int D8_TILE = 128;         // tokens per stage (32 per consumer warp)
constexpr int D8_UNIT = 64;          // tokens by which work is dealt out
constexpr int D8_STAGES = 3;
constexpr int D8_THREADS = 160;      // warps 0..3 consumers, warp 4 TMA
constexpr int D8_BLOCKS_PER_SM = 2;
constexpr float D8_RAISE = 8.f;
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
// transpose of an 8 x 8 matrix of 16-bit elements spread over the warp (row lane / 4, columns 2 (lane % 4), + 1)
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                              uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_half(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
// 2^x for x <= D8_RAISE (relative error 2^-22)
__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int DH>
struct D8Smem {
    uint8_t kv[D8_STAGES][2][D8_TILE * DH];     // keys, values of a stage: rows of DH bytes, swizzled (128 or 64 bytes)
    float o[4][4][DH + 4];                      // at the end of a sequence's part: every warp's un-normalised output, four heads at a time
    float qs[8][DH];                            // rotated queries of the G heads (rows G..7 zero)
    float m[4][8], l[4][8], vs[4];
    uint64_t full[D8_STAGES], empty[D8_STAGES];
    uint32_t dead[D8_STAGES];                   // boxes of the stage whose page lies outside the pool, one bit each
};

struct D8Params {
    const bf16* q;
    bf16* out;
    Cache8View cv;
    const float2* rope_table;
    float* part_ml;                             // [n_kv][parts + rows][G][2]: reference (log2 units), sum
    float* part_o;                              // [n_kv][parts + rows][G][DH]
    int* status;
    int G, n_kv, T, interleaved, max_pos, box_rows;
    int rows;                                   // batch * T
    int parts, least;                           // 0: a block per row and KV head; else parts of the list, of `least` steps at least
};

// Row r = s T + t stands for query t of sequence s: the tokens up to that query's own (0: nothing to attend to).
__device__ __forceinline__ int d8_len(const D8Params& p, int r, int* status) {
    const int s = r / p.T, len = lorc_len8(p.cv, s, p.max_pos, status);
    if (p.T == 1) return len;
    if (len < p.T) {
        if (len > 0 && status) lorc_set_status(status, LORC_ERR_ARG);
        return 0;
    }
    return len - (p.T - 1 - (r - s * p.T));
}
// Units of a row on the list; a row without tokens has one, in which its zeros are written.
__device__ __forceinline__ int d8_weight(int len) { return len <= 0 ? 1 : (len - 1) / D8_UNIT + 1; }

// Sum of the weights of rows [0, n); whole warps.
__device__ __forceinline__ long long d8_total(const D8Params& p, int n, int lane) {
    long long sum = 0;
    for (int i = lane; i < n; i += 32) sum += d8_weight(d8_len(p, i, nullptr));
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}
__device__ __forceinline__ long long d8_per(const D8Params& p, long long total) {
    const long long per = (total + p.parts - 1) / p.parts;
    return per < p.least ? p.least : per;
}

// The row that holds step f of the list and the first step of that row; whole warps.
__device__ __forceinline__ void d8_locate(const D8Params& p, long long f, int lane, int& row, long long& first) {
    long long before = 0;
    for (int i0 = 0; i0 < p.rows; i0 += 32) {
        const int i = i0 + lane, w = i < p.rows ? d8_weight(d8_len(p, i, nullptr)) : 0;
        long long end = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, end, o);
            if (lane >= o) end += x;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, f < before + end);
        if (hit) {
            const int l = __ffs(hit) - 1;
            row = i0 + l;
            first = before + __shfl_sync(0xffffffffu, end - w, l);
            return;
        }
        before += __shfl_sync(0xffffffffu, end, 31);
    }
    row = p.rows;
    first = before;
}

// What a block works on: steps [f, end) of the list, beginning in row `row`, whose first step is `first`.
struct D8Range {
    long long f, end, first;
    int row;
};
__device__ __forceinline__ D8Range d8_range(const D8Params& p, int part, int lane) {
    D8Range r;
    if (p.parts == 0) {
        r.row = part;
        r.f = r.first = 0;
        r.end = d8_weight(d8_len(p, part, nullptr));
        return r;
    }
    const long long total = d8_total(p, p.rows, lane), per = d8_per(p, total);
    r.f = part * per;
    r.end = r.f + per < total ? r.f + per : total;
    r.row = p.rows;
    r.first = 0;
    if (r.f < r.end) d8_locate(p, r.f, lane, r.row, r.first);
    return r;
}

template <int DH, bool E4M3>
__global__ void __launch_bounds__(D8_THREADS, D8_BLOCKS_PER_SM)
decode8_mma_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const D8Params p) {
    constexpr int KS = DH / 16;                  // pieces of 16 dimensions
    extern __shared__ uint8_t d8_raw[];
    D8Smem<DH>& sm = *reinterpret_cast<D8Smem<DH>*>((reinterpret_cast<uintptr_t>(d8_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;       // fragment row / column group of this lane
    const int kvh = (int)blockIdx.x % p.n_kv, part = (int)blockIdx.x / p.n_kv;
    const Cache8View& cv = p.cv;
    const int G = p.G, H_q = G * p.n_kv;
    if (tid == 0) {
        for (int i = 0; i < D8_STAGES; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 4);
        }
        fence_barrier_init();
        prefetch_tensormap(&mapK);
        prefetch_tensormap(&mapV);
    }
    grid_dep_wait();
    grid_dep_launch();
    const D8Range range = d8_range(p, part, lane);
    __syncthreads();                             // the barriers are initialised
    bool ok = true;
    int st = 0;                                  // place in the ring of stages
    uint32_t par = 0;                            // and the parity of this round

    if (warp == 4) {
        // ------------------------------------------------------------------ producer (one elected lane issues)
        const int nbox = D8_TILE / p.box_rows;   // boxes per tile: 2, or up to 8 on small pages
        int fetched = 0;                         // stages that may have copies under way
        long long f = range.f, first = range.first;
        for (int row = range.row; f < range.end && ok; ++row) {
            const int s = row / p.T, len = d8_len(p, row, nullptr), w = d8_weight(len);
            const long long stop = first + w < range.end ? first + w : range.end;
            if (len <= 0) {
                f = first += w;
                continue;
            }
            // lane i < nbox: the page of the tile's i-th box, -1 for a table entry outside the pool (reported).  Such a box,
            // and one past the end of the sequence, is fetched from behind the pool, where it reads as zero.
            auto lookup = [&](int t0) {
                int page = cv.page_table ? cv.n_pages : 0;
                if (cv.page_table != nullptr && lane < nbox && t0 + lane * p.box_rows < len) {
                    page = cv.page_table[(long long)s * cv.max_pages_per_seq + (t0 + lane * p.box_rows) / cv.page_size];
                    if (page < 0 || page >= cv.n_pages) {
                        lorc_set_status(p.status, LORC_ERR_CAPACITY);
                        page = -1;
                    }
                }
                return page;
            };
            int t0 = (int)(f - first) * D8_UNIT;
            const int t_end = min(len, (int)(stop - first) * D8_UNIT);
            int mine = lookup(t0);
            for (; t0 < t_end; t0 += D8_TILE) {
                int pages[8];
                const uint32_t dead = __ballot_sync(0xffffffffu, mine < 0);
                if (mine < 0) mine = cv.n_pages;
#pragma unroll
                for (int j = 0; j < 8; ++j) pages[j] = __shfl_sync(0xffffffffu, mine, j);
                if (t0 + D8_TILE < t_end) mine = lookup(t0 + D8_TILE);
                ok = __all_sync(0xffffffffu, mbar_wait(&sm.empty[st], par ^ 1));
                if (!ok) break;
                if (elect_one()) {
                    // boxes wholly behind the part's end are not fetched
                    const int live = min(nbox, (t_end - t0 + p.box_rows - 1) / p.box_rows);
                    sm.dead[st] = dead;
                    mbar_arrive_expect_tx(&sm.full[st], 2 * DH * p.box_rows * live);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (j >= live) break;
                        const int tok = t0 + j * p.box_rows;
                        const int y = cv.page_table ? tok % cv.page_size : tok, z = cv.page_table ? pages[j] : s;
                        tma_load_3d(sm.kv[st][0] + j * p.box_rows * DH, &mapK, &sm.full[st], kvh * DH, y, z);
                        tma_load_3d(sm.kv[st][1] + j * p.box_rows * DH, &mapV, &sm.full[st], kvh * DH, y, z);
                    }
                }
                __syncwarp();
                if (++st == D8_STAGES) { st = 0; par ^= 1; }
                if (fetched < D8_STAGES) ++fetched;
            }
            f = stop;
            first += w;
        }
        // The block stays until the copies into its shared memory have landed, also when a wait has run out.
        for (; fetched > 0; --fetched) {
            if (--st < 0) { st = D8_STAGES - 1; par ^= 1; }
            if (!mbar_wait(&sm.full[st], par)) ok = false;
        }
        if (!ok && lane == 0) lorc_set_status(p.status, LORC_ERR_TIMEOUT);
        return;
    }

    // ---------------------------------------------------------------------- consumers
    // byte offset of this lane's row in a stage and the row's swizzle; ldmatrix.x4 takes four 8 x 8 matrices of words, lane
    // mi = lane / 8 addresses a row of matrix mi: (tokens 0..7 | 8..15) x piece, then the same x the next piece
    const int mi = lane >> 3, lr = lane & 7;
    const uint32_t my_row = (uint32_t)(warp * 32 + (mi & 1) * 8 + lr);
    const uint32_t row_off = my_row * DH, sw = DH == 128 ? my_row & 7 : (my_row >> 1) & 3;
    const int box0 = warp * 32 / p.box_rows, box1 = (warp * 32 + 16) / p.box_rows;      // the boxes of this warp's tokens
    long long f = range.f, first = range.first;
    for (int row = range.row; f < range.end; ++row) {
        const int s = row / p.T, len = d8_len(p, row, tid == 0 ? p.status : nullptr), w = d8_weight(len);
        const long long stop = first + w < range.end ? first + w : range.end;
        const bool whole = f == first && stop == first + w;
        const int t_begin = (int)(f - first) * D8_UNIT, t_end = min(len, (int)(stop - first) * D8_UNIT);

        // the scales of this warp's blocks, two a step, 16 steps at a time: lane 2 j + u holds block u of step j
        auto scales = [&](int t0, float& ks, float& vs) {
            const int pos = t0 + (lane >> 1) * D8_TILE + warp * 32 + (lane & 1) * 16;
            ks = vs = 0.f;
            if (pos < t_end) {
                const long long at = lorc_block8(cv, s, pos / LORC_BLOCK8);
                if (at >= 0) {
                    ks = cv.k_scale[at * p.n_kv + kvh];
                    vs = cv.v_scale[at * p.n_kv + kvh];
                }
            }
        };
        float ks_now, vs_now, ks_next = 0.f, vs_next = 0.f;
        scales(t_begin, ks_now, vs_now);

        // RoPE(q, position) for the G heads of this KV head
        for (int i = tid; i < 8 * (DH / 2); i += 128) {
            const int h = i / (DH / 2), jj = i - h * (DH / 2);
            const int ia = p.interleaved ? 2 * jj : jj, ib = p.interleaved ? 2 * jj + 1 : jj + DH / 2;
            float ra = 0.f, rb = 0.f;
            if (h < G && len > 0) {
                const bf16* qp = p.q + ((long long)row * H_q + kvh * G + h) * DH;
                const float a = __bfloat162float(qp[ia]), b = __bfloat162float(qp[ib]);
                const float2 cs = p.rope_table[(long long)(len - 1) * (DH / 2) + jj];
                ra = a * cs.x - b * cs.y;
                rb = a * cs.y + b * cs.x;
            }
            sm.qs[h][ia] = ra;
            sm.qs[h][ib] = rb;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        // Query fragments of head g: piece ks, dimensions 4 t .. 4 t + 3 of its 16.
        uint32_t qhi[KS][2], qlo[KS][2];
        float factor[2];                         // heads 2 t, 2 t + 1: what brings a sum of code products to log2 units
        {
            float most = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const float4 v = *reinterpret_cast<const float4*>(&sm.qs[g][16 * ks + 4 * t]);
                most = fmaxf(most, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
            }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // its power of two, between 2^-100 and 2^100
            const uint32_t e = min(max(__float_as_uint(most) >> 23, 27u), 227u);
            const float up = __uint_as_float(e << 23), down = __uint_as_float((254u - e) << 23);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                float4 v = *reinterpret_cast<const float4*>(&sm.qs[g][16 * ks + 4 * t]);
                v.x *= down; v.y *= down; v.z *= down; v.w *= down;
                qhi[ks][0] = pack_half(v.x, v.y);
                qhi[ks][1] = pack_half(v.z, v.w);
                const float2 a = unpack_half(qhi[ks][0]), b = unpack_half(qhi[ks][1]);
                qlo[ks][0] = pack_half(v.x - a.x, v.y - a.y);
                qlo[ks][1] = pack_half(v.z - b.x, v.w - b.y);
            }
            const float base = rsqrtf((float)DH) * LOG2E;
            factor[0] = __shfl_sync(0xffffffffu, up, 8 * t) * base;
            factor[1] = __shfl_sync(0xffffffffu, up, 8 * t + 4) * base;
        }
        float o[KS][4];                          // dimensions 16 ks + 2 g (+ 1: [2], [3]), heads 2 t, 2 t + 1
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) o[ks][0] = o[ks][1] = o[ks][2] = o[ks][3] = 0.f;
        float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};   // heads 2 t, 2 t + 1 (l: this lane's tokens)
        float v_ref = 0.f, v_inv = 0.f;          // largest scale of values so far: o is in units of it

        int turn = 0;
        for (int t0 = t_begin; t0 < t_end && ok; t0 += D8_TILE, turn = (turn + 2) & 31) {
            const int tw = t0 + warp * 32;       // first token of this warp
            if (turn == 0) {
                if (t0 > t_begin) { ks_now = ks_next; vs_now = vs_next; }
                if (t0 + 16 * D8_TILE < t_end) scales(t0 + 16 * D8_TILE, ks_next, vs_next);
            }
            float k_scale[2], v_scale[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                k_scale[u] = __shfl_sync(0xffffffffu, ks_now, turn + u);
                v_scale[u] = __shfl_sync(0xffffffffu, vs_now, turn + u);
            }
            ok = __all_sync(0xffffffffu, mbar_wait(&sm.full[st], par));
            if (!ok) break;
            const uint32_t k0 = smem_u32(sm.kv[st][0]) + row_off, v0 = smem_u32(sm.kv[st][1]) + row_off;
            // scores of tokens g, g + 8 of both blocks against heads 2 t, 2 t + 1
            float x[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float sc[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j) sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
#pragma unroll
                for (int k2 = 0; k2 < KS / 2; ++k2) {
                    uint32_t a[4];
                    ldmatrix_x4(a, k0 + u * 16 * DH + (((2 * k2 + (mi >> 1)) ^ sw) << 4));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t a0, a1, a2, a3;
                        lorc_codes_half<E4M3, 0, 1, 2, 3>(a[2 * e], a0, a2);
                        lorc_codes_half<E4M3, 0, 1, 2, 3>(a[2 * e + 1], a1, a3);
                        mma_f16_16816(sc[0], a0, a1, a2, a3, qhi[2 * k2 + e][0], qhi[2 * k2 + e][1]);
                        mma_f16_16816(sc[1], a0, a1, a2, a3, qlo[2 * k2 + e][0], qlo[2 * k2 + e][1]);
                    }
                }
                const float f0 = factor[0] * k_scale[u], f1 = factor[1] * k_scale[u];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[u][j] = (sc[0][j] + sc[1][j]) * (j & 1 ? f1 : f0);
            }
            const uint32_t dead = sm.dead[st];
            if (tw + 32 > t_end || dead) {       // tokens past the end, or in pages that do not exist
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int live = (dead >> (u ? box1 : box0)) & 1 ? 0 : t_end - tw - 16 * u;
                    if (live <= 0) v_scale[u] = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (g + (j >> 1) * 8 >= live) x[u][j] = -INFINITY;
                }
                if (E4M3) {
                    // such rows have the factor zero, but their bytes may be codes of NaN
                    for (int r = max(t_end - tw, 0); r < 32; ++r)
                        if (lane < DH / 8) *reinterpret_cast<uint2*>(sm.kv[st][1] + (warp * 32 + r) * DH + lane * 8) = make_uint2(0u, 0u);
                    fence_proxy_async_smem();    // before the stage's next copy
                    __syncwarp();
                }
            }
            // running softmax over this warp's tokens: the reference is raised when a score exceeds it by more than 2^8, which
            // after the first steps is rare, so the maximum is looked for only then
            const float top0 = fmaxf(fmaxf(x[0][0], x[0][2]), fmaxf(x[1][0], x[1][2]));
            const float top1 = fmaxf(fmaxf(x[0][1], x[0][3]), fmaxf(x[1][1], x[1][3]));
            const float v_mag = fmaxf(fabsf(v_scale[0]), fabsf(v_scale[1]));
            if (__any_sync(0xffffffffu, top0 > m_run[0] + D8_RAISE || top1 > m_run[1] + D8_RAISE || v_mag > v_ref)) {
                float shrink = 1.f;
                if (v_mag > v_ref) {
                    const float now = fmaxf(v_mag, 1e-35f);
                    v_inv = 1.f / now;
                    shrink = v_ref * v_inv;
                    v_ref = now;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = e ? top1 : top0;
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    float alpha = 1.f;
                    if (mx > m_run[e] + D8_RAISE) {
                        alpha = m_run[e] == -INFINITY ? 0.f : ex2_approx(m_run[e] - mx);
                        m_run[e] = mx;
                    }
                    l_run[e] *= alpha;
                    alpha *= shrink;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        o[ks][e] *= alpha;
                        o[ks][2 + e] *= alpha;
                    }
                }
            }
            // p = 2^(x - m); c p as fp16, pairs of heads
            const float m0 = m_run[0] == -INFINITY ? 0.f : m_run[0], m1 = m_run[1] == -INFINITY ? 0.f : m_run[1];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float c = v_scale[u] * v_inv;
                uint32_t ph[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float p0 = ex2_approx(x[u][2 * j] - m0), p1 = ex2_approx(x[u][2 * j + 1] - m1);
                    l_run[0] += p0;
                    l_run[1] += p1;
                    ph[j] = pack_half(p0 * c, p1 * c);
                }
                const uint32_t b0 = movmatrix_trans(ph[0]), b1 = movmatrix_trans(ph[1]);
                // O^T += V^T (c P)^T
#pragma unroll
                for (int k2 = 0; k2 < KS / 2; ++k2) {
                    uint32_t a[4];
                    ldmatrix_x4_trans(a, v0 + u * 16 * DH + (((2 * k2 + (mi >> 1)) ^ sw) << 4));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t a0, a1, a2, a3;
                        lorc_codes_half<E4M3, 0, 2, 1, 3>(a[2 * e], a0, a1);
                        lorc_codes_half<E4M3, 0, 2, 1, 3>(a[2 * e + 1], a2, a3);
                        mma_f16_16816(o[2 * k2 + e], a0, a1, a2, a3, b0, b1);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.empty[st]);
            if (++st == D8_STAGES) { st = 0; par ^= 1; }
        }
        // what the four warps have, four heads at a time
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], d);
            if (g == 0) {
                sm.m[warp][2 * t + e] = m_run[e];
                sm.l[warp][2 * t + e] = l_run[e];
            }
        }
        if (lane == 0) sm.vs[warp] = v_ref;
        for (int h0 = 0; h0 < G; h0 += 4) {
            if (2 * t >= h0 && 2 * t < h0 + 4)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        *reinterpret_cast<float2*>(&sm.o[warp][2 * t + e - h0][16 * ks + 2 * g]) = make_float2(o[ks][e], o[ks][2 + e]);
            __syncwarp();
            asm volatile("bar.sync 1, 128;" ::: "memory");
            const int heads = min(G - h0, 4);
            for (int i = tid; i < heads * DH; i += 128) {
                const int h = h0 + i / DH, d = i % DH;
                float M = -INFINITY;
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (sm.l[x][h] != 0.f) M = fmaxf(M, sm.m[x][h]);
                float L = 0.f, acc = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float wgt = sm.l[x][h] != 0.f ? exp2f(sm.m[x][h] - M) : 0.f;
                    L += wgt * sm.l[x][h];
                    acc += wgt * sm.vs[x] * sm.o[x][h - h0][d];
                }
                if (whole) {
                    p.out[((long long)row * H_q + kvh * G + h) * DH + d] = __float2bfloat16_rn(L != 0.f ? acc / L : 0.f);
                    if (L == 0.f && d == 0) lorc_set_status(p.status, LORC_ERR_EMPTY);
                } else {
                    const long long unit = ((long long)kvh * (p.parts + p.rows) + part + row) * G + h;
                    if (d == 0) *reinterpret_cast<float2*>(p.part_ml + unit * 2) = make_float2(M, L);
                    p.part_o[unit * DH + d] = acc;
                }
            }
            if (h0 + 4 < G) asm volatile("bar.sync 1, 128;" ::: "memory");
        }
        first += w;
        f = stop;
    }
    if (!ok && lane == 0) lorc_set_status(p.status, LORC_ERR_TIMEOUT);
}

// Sequences that were cut: piece i of row r came from part c0 + i and lies in slot c0 + i + r.  One block per (head, row).
template <int DH>
__global__ void __launch_bounds__(DH)
decode8_merge_kernel(const D8Params p) {
    const int tid = threadIdx.x, lane = tid & 31;
    const int H_q = p.G * p.n_kv, hq = (int)blockIdx.x % H_q, row = (int)blockIdx.x / H_q, kvh = hq / p.G, h = hq - kvh * p.G;
    grid_dep_wait();
    grid_dep_launch();
    const long long per = d8_per(p, d8_total(p, p.rows, lane)), first = d8_total(p, row, lane);
    const int w = d8_weight(d8_len(p, row, nullptr));
    const int c0 = (int)(first / per), c1 = (int)((first + w - 1) / per);
    if (c0 == c1) return;                        // one block had it all and has written the result
    const long long unit0 = ((long long)kvh * (p.parts + p.rows) + c0 + row) * p.G + h;
    const int n = c1 - c0 + 1;
    float M = -INFINITY;
    for (int c = lane; c < n; c += 32) {
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + (unit0 + (long long)c * p.G) * 2);
        if (ml.y != 0.f) M = fmaxf(M, ml.x);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    float L = 0.f, acc = 0.f;
#pragma unroll 4
    for (int c = 0; c < n; ++c) {
        const long long unit = unit0 + (long long)c * p.G;
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + unit * 2);
        const float x = p.part_o[unit * DH + tid];
        const float wgt = ml.y != 0.f ? exp2f(ml.x - M) : 0.f;
        L += wgt * ml.y;
        acc += wgt != 0.f ? wgt * x : 0.f;
    }
    p.out[((long long)row * H_q + hq) * DH + tid] = __float2bfloat16_rn(L != 0.f ? acc / L : 0.f);
    if (L == 0.f && tid == 0) lorc_set_status(p.status, LORC_ERR_EMPTY);
}

// 8-bit rows in boxes of d_head bytes x box_rows tokens.
bool make_map8(CUtensorMap* map, const void* base, const Cache8View& cv, int dh, int box_rows) {
    lorc_tmap_encode_fn enc = lorc_get_tmap_encode();
    if (!enc) return false;
    const uint64_t rows = cv.page_table ? (uint64_t)cv.page_size : (uint64_t)cv.seq_stride;
    const cuuint64_t dims[3] = {(cuuint64_t)cv.n, rows, (cuuint64_t)(cv.page_table ? cv.n_pages : cv.batch)};
    const cuuint64_t strides[2] = {(cuuint64_t)cv.n, rows * cv.n};
    const cuuint32_t box[3] = {(cuuint32_t)dh, (cuuint32_t)box_rows, 1}, ones[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
               dh == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How the rows of a call are dealt out.  Parts: the blocks of a KV head that are resident at once.  A block per row where rows are
// at most four steps long, or, with several queries per sequence, where there are more rows than parts (they are about equally
// long then, and the list would be long to search).
void d8_plan(const lorc_ctx* ctx, int rows, int max_seq_len, int T, int* parts, int* least) {
    const int slots = D8_BLOCKS_PER_SM * ctx->sm_count / ctx->desc.n_kv_heads;
    *parts = slots > 1 ? slots : 1;
    *least = 2;
    if (max_seq_len <= 4 * D8_UNIT || (T > 1 && rows >= *parts)) *parts = 0;
}

size_t d8_ml_bytes(const lorc_ctx* ctx, long long slots) {
    return lorc_align_up((size_t)slots * ctx->desc.n_q_heads * 2 * sizeof(float), 256);
}

template <int DH, bool E4M3>
cudaError_t d8_launch(lorc_ctx* ctx, const CUtensorMap& mapK, const CUtensorMap& mapV, const D8Params& p, cudaStream_t st) {
    const size_t smem = sizeof(D8Smem<DH>) + 1024;
    // the attribute belongs to a device's copy of the kernel: one flag per device
    static bool attr[64] = {false};
    const bool known = ctx->device >= 0 && ctx->device < 64;
    if (!known || !attr[ctx->device]) {
        cudaError_t e = cudaFuncSetAttribute(decode8_mma_kernel<DH, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (known) attr[ctx->device] = true;
    }
    const long long blocks = (long long)p.n_kv * (p.parts ? p.parts : p.rows);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    return lorc_launch_dependent(decode8_mma_kernel<DH, E4M3>, dim3((unsigned)blocks), dim3(D8_THREADS), smem, st, mapK, mapV, p);
}

}  // namespace

size_t lorc_decode8_scratch_bytes(const lorc_ctx* ctx, int batch, int max_seq_len, int T) {
    // a call may have fewer tokens or shorter sequences than stated here: room for the list in any case
    int parts, least;
    const long long rows = (long long)batch * T;
    d8_plan(ctx, 1, max_seq_len > 4 * D8_UNIT ? max_seq_len : 4 * D8_UNIT + 1, 1, &parts, &least);
    const long long slots = parts + (batch > parts || rows <= batch ? batch : rows < parts ? rows : parts);
    return d8_ml_bytes(ctx, slots) + lorc_align_up((size_t)slots * ctx->desc.n_q_heads * ctx->desc.d_head * sizeof(float), 256);
}

cudaError_t lorc_decode8_launch(lorc_ctx* ctx, const Cache8View& cv, const bf16* q, bf16* out, int T, void* scratch,
                                cudaStream_t st, int* launches) {
    const lorc_model_desc& d = ctx->desc;
    // a box never leaves its page: page sizes are multiples of 16
    const int box_rows = !cv.page_table || cv.page_size % 64 == 0 ? 64 : cv.page_size % 32 == 0 ? 32 : 16;
    CUtensorMap mapK, mapV;
    if (!make_map8(&mapK, cv.k, cv, d.d_head, box_rows) || !make_map8(&mapV, cv.v, cv, d.d_head, box_rows)) return cudaErrorInvalidValue;
    D8Params p;
    p.q = q; p.out = out; p.cv = cv; p.rope_table = ctx->rope_table; p.status = ctx->status_dev;
    p.G = ctx->group; p.n_kv = d.n_kv_heads; p.T = T; p.interleaved = ctx->pair_style == LORC_ROPE_INTERLEAVED;
    p.max_pos = d.max_pos; p.box_rows = box_rows; p.rows = cv.batch * T;
    d8_plan(ctx, p.rows, cv.max_seq_len, T, &p.parts, &p.least);
    p.part_ml = (float*)scratch;
    p.part_o = (float*)((char*)scratch + d8_ml_bytes(ctx, p.parts + p.rows));
    const bool e4m3 = cv.type == LORC_CACHE8_E4M3;
    cudaError_t e;
    {
        LorcStageTimer timer(ctx, LORC_STAGE_SCORE, st);
        e = d.d_head == 128 ? (e4m3 ? d8_launch<128, true>(ctx, mapK, mapV, p, st) : d8_launch<128, false>(ctx, mapK, mapV, p, st))
                            : (e4m3 ? d8_launch<64, true>(ctx, mapK, mapV, p, st) : d8_launch<64, false>(ctx, mapK, mapV, p, st));
        *launches += 1;
    }
    if (e != cudaSuccess || p.parts == 0) return e;
    LorcStageTimer timer(ctx, LORC_STAGE_COMBINE, st);
    const long long blocks = (long long)p.rows * d.n_q_heads;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    *launches += 1;
    return d.d_head == 128 ? lorc_launch_dependent(decode8_merge_kernel<128>, dim3((unsigned)blocks), dim3(128), 0, st, p)
                           : lorc_launch_dependent(decode8_merge_kernel<64>, dim3((unsigned)blocks), dim3(64), 0, st, p);
}
