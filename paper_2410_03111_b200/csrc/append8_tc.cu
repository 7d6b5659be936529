// Cache write of uncompressed layers in 8 bits for prompt-sized token counts, on the tensor cores (sm_100a: TMA + tcgen05 + TMEM):
// projection, rotation and quantisation in one kernel.
//
// The rows of a tile are blocks of 16 tokens as the cache has them (aligned by position), so that the numbers which share a
// scale are 16 neighbouring lanes of tensor memory and the columns of one head: the largest magnitude of a block takes four
// shuffles, and a thread stores its row's codes.  The fp32 projection never goes to memory.
//
// Persistent CTA pairs (cta_group::2) walk units of 256 rows x 256 (or 128) columns of [W_k | W_v], K = D in 64-wide TMA
// stages.  The tensor cores' fp32 sums lose more than rounding would as they grow longer, and a number near the border between
// two codes may then fall on the other side; so the MMAs sum 512 products at a time, in two accumulators in TMEM by turns, and
// sixteen epilogue warps add these up in registers.  (D 4096, codes that are not the fp64 projection's: 1.2e-5 of them, as with a
// plain fp32 projection; with one sum of 4096 1.0e-4, in 7 % less time, with sums of 256 0.6e-5, in 13 % more.  Products of one sign
// are off by 2^-20.1 of their sum at most.)  Rows of a block that
// are not new (earlier tokens, or behind the end) lie outside x and read as zero.
#include <math.h>

#include "append8.cuh"
#include "sm100_pair.cuh"
#include "sm100_ptx.cuh"
#include "tc_kernels.cuh"

using namespace sm100;

namespace {

constexpr int TILE = 128;            // rows per CTA
constexpr int KC = 64;               // D elements per stage
constexpr int NB_MAX = 256;          // columns per unit
constexpr int A8_STAGES = 6;          // 32 KiB each
constexpr int A8_THREADS = 640;      // warp 0 TMA, warp 1 MMA (leader CTA issues), warps 4..19 epilogue
constexpr int A8_SUM = 8;            // stages per accumulator
constexpr int PER_TILE = TILE / LORC_BLOCK8;

struct A8Smem {
    bf16 X[A8_STAGES][TILE * KC];          // [128 rows][64]                                                 16 KiB
    bf16 A[A8_STAGES][2][KC * KC];         // this CTA's half of the columns: two blocks of [64 D rows][64]  16 KiB
    float4 near[LORC_BLOCK8][33];          // (cos, sin) of the positions 0 .. 15, DH / 4 pairs of pairs each
    float most[2][2][4][TILE];             // what the epilogue warps of a row exchange: [turn][piece][group][row]
    uint64_t full[A8_STAGES], empty[A8_STAGES], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
};

// The four epilogue warps that read the same lanes of tensor memory: whether all of them say so.
__device__ __forceinline__ bool quarter_all(int quarter, bool mine) {
    int all;
    asm volatile(
        "{\n\t"
        ".reg .pred p, q;\n\t"
        "setp.ne.s32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, 128, p;\n\t"
        "selp.s32 %0, 1, 0, q;\n\t"
        "}\n"
        : "=r"(all)
        : "r"((int)mine), "r"(quarter + 1)
        : "memory");
    return all != 0;
}

// A piece of a head of this thread's row: 32 of its DH columns, as two runs of 16 in which both members of every rotary pair meet.
// Piece c: columns 16 c .. and DH / 2 + 16 c .., or 32 c .. and 32 c + 16 .. (interleaved pairs).
template <int DH>
__device__ __forceinline__ int piece_column(int c, bool interleaved, int run) {
    return interleaved ? 32 * c + 16 * run : 16 * c + run * (DH / 2);
}

// Piece c of a key, rotated: the row's position is that of the block's first row plus r, and R(16 b + r) = R(16 b) R(r), with R(16 b)
// from the table (`far`, one address for the 16 lanes of a block) and R(r), r < 16, from the copy of the table's first rows in
// shared memory (`near`).  (With a table row of its own for every lane, 32 lines per access, this took three times as long.)
__device__ __forceinline__ void append8_rotate(int c, bool interleaved, const float4* far, const float4* near, float (&a)[16], float (&b)[16]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float4 f = __ldg(far + 8 * c + j), n = near[8 * c + j];
        const float c0 = f.x * n.x - f.y * n.y, s0 = f.x * n.y + f.y * n.x, c1 = f.z * n.z - f.w * n.w, s1 = f.z * n.w + f.w * n.z;
        if (interleaved) {
            float* x = j < 4 ? a + 4 * j : b + 4 * (j - 4);
            const float u = x[0], v = x[1], w = x[2], z = x[3];
            x[0] = u * c0 - v * s0;
            x[1] = u * s0 + v * c0;
            x[2] = w * c1 - z * s1;
            x[3] = w * s1 + z * c1;
        } else {
            const float u = a[2 * j], v = b[2 * j], w = a[2 * j + 1], z = b[2 * j + 1];
            a[2 * j] = u * c0 - v * s0;
            b[2 * j] = u * s0 + v * c0;
            a[2 * j + 1] = w * c1 - z * s1;
            b[2 * j + 1] = w * s1 + z * c1;
        }
    }
}

struct A8Params {
    Append8Params q;
    int D, R, m_units, n_units, total_blocks;
};

// NP: pieces per epilogue thread, that is columns of a unit / 128.
template <int DH, bool E4M3, int NP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(A8_THREADS, 1)
append8_tc_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapX16,
                  const __grid_constant__ CUtensorMap mapA, const A8Params p) {
    extern __shared__ uint8_t raw[];
    A8Smem& sm = *reinterpret_cast<A8Smem*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = (int)cluster_ctarank();           // 0 = leader (issues the MMAs, owns the full / acc_empty barriers)
    const int pair_id = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    constexpr int NB = 128 * NP;                       // columns of a unit
    const int nkc = p.D / KC, sums = (nkc + A8_SUM - 1) / A8_SUM, total = p.m_units * p.n_units;
    const Cache8View& cv = p.q.cv;

    if (tid == 0) {
        for (int i = 0; i < A8_STAGES; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.acc_full[i], 1);
            mbar_init(&sm.acc_empty[i], 2 * 16);            // one arrival per epilogue warp, both CTAs
        }
        fence_barrier_init();
        prefetch_tensormap(&mapX);
        prefetch_tensormap(&mapA);
    }
    grid_dep_wait();
    for (int i = tid; i < min(LORC_BLOCK8, p.q.max_pos) * (DH / 4); i += A8_THREADS)
        sm.near[i / (DH / 4)][i % (DH / 4)] = reinterpret_cast<const float4*>(p.q.rope_table)[i];
    if (warp == 1) {
        tmem_alloc_pair(&sm.tmem_base, 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive_release();                            // the peer's barriers are initialised before anyone signals them
    cluster_wait_acquire();
    tc_fence_after_sync();
    grid_dep_launch();
    const uint32_t tmem = sm.tmem_base;
    bool ok = true;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer (both CTAs)
        const uint32_t x_base = smem_u32(sm.X[0]), a_base = smem_u32(sm.A[0][0]);
        const uint32_t empty0 = smem_u32(&sm.empty[0]), full0 = smem_u32(&sm.full[0]);
        const uint32_t lead_full0 = mapa_shared(full0, 0);   // all bytes of a stage are counted on the leader's barrier
        constexpr int half = NB / 2, boxes = half / KC;
        const uint32_t bytes = 2 * (TILE + half) * KC * 2;
        uint32_t st = 0, par = 1;
        for (int u = pair_id; u < total && ok; u += n_pairs) {
            const int mt = u / p.n_units, acol = (u - mt * p.n_units) * NB + rank * half;
            // the tile's first block, and where its rows are in x; lane i < 8: the same for block i
            const int q0 = (mt * 2 + rank) * PER_TILE, mine = q0 + (lane & 7);
            const int s = min(mine, p.total_blocks - 1) / p.q.n_blocks;
            const int begin = max(cv.seq_lens[s] - p.q.T, 0) / LORC_BLOCK8 * LORC_BLOCK8;
            int y = p.q.T;                                   // behind the end: reads as zero
            if (mine < p.total_blocks)
                y = begin + (mine - s * p.q.n_blocks) * LORC_BLOCK8 - (cv.seq_lens[s] - p.q.T);
            // (a length that is out of range is dealt with in the epilogue; coordinates stay near the tensor)
            y = max(min(y, p.q.T), -LORC_BLOCK8);
            int ys[PER_TILE], ss[PER_TILE];
#pragma unroll
            for (int i = 0; i < PER_TILE; ++i) {
                ys[i] = __shfl_sync(0xffffffffu, y, i);
                ss[i] = __shfl_sync(0xffffffffu, s, i);
            }
            const bool one = __all_sync(0xffffffffu, lane >= PER_TILE || mine >= p.total_blocks ||
                                                         (s == ss[0] && y == min(ys[0] + lane * LORC_BLOCK8, p.q.T)));
            for (int kc = 0; kc < nkc; ++kc) {
                ok = __all_sync(0xffffffffu, mbar_wait_addr(empty0 + st * 8, par));
                if (!ok) break;
                const uint32_t lead_bar = lead_full0 + st * 8, a_dst = a_base + st * (2 * KC * KC * 2);
                const uint32_t x_dst = x_base + st * (TILE * KC * 2);
                if (elect_one()) {
                    if (rank == 0) mbar_arrive_expect_tx_addr(full0 + st * 8, bytes);
                    tma_load_2d_pair_addr(a_dst, &mapA, lead_bar, acol, kc * KC);
                    if (boxes > 1) tma_load_2d_pair_addr(a_dst + KC * KC * 2, &mapA, lead_bar, acol + KC, kc * KC);
                    if (one) {
                        tma_load_3d_pair_addr(x_dst, &mapX, lead_bar, kc * KC, ys[0], ss[0]);
                    } else {
#pragma unroll
                        for (int i = 0; i < PER_TILE; ++i)
                            tma_load_3d_pair_addr(x_dst + i * LORC_BLOCK8 * KC * 2, &mapX16, lead_bar, kc * KC, ys[i], ss[i]);
                    }
                }
                __syncwarp();
                if (++st == A8_STAGES) { st = 0; par ^= 1; }
            }
        }
        if (!ok) {
            // copies may be under way into either CTA: neither leaves before they must have landed
            if (lane == 0) lorc_set_status(p.q.status, LORC_ERR_TIMEOUT);
            for (const uint64_t since = global_timer_ns(); global_timer_ns() - since < 1000000ull;) {}
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (leader CTA only)
        // A: x rows (K-major), a k-step is 32 bytes.  B: factor blocks (MN-major: a D row's 64 columns are contiguous),
        // 64-column blocks 8 KiB apart, 16 D rows (one k-step) 2 KiB apart.
        if (rank == 0) {
            const uint64_t da0 = make_smem_desc_sw128(smem_u32(sm.X[0]), 0, 1024);
            const uint64_t db0 = make_smem_desc_sw128(smem_u32(sm.A[0][0]), KC * KC * 2, 1024);
            const uint32_t a_lo0 = (uint32_t)da0, a_hi = (uint32_t)(da0 >> 32);
            const uint32_t b_lo0 = (uint32_t)db0, b_hi = (uint32_t)(db0 >> 32);
            const uint32_t full0 = smem_u32(&sm.full[0]), empty0 = smem_u32(&sm.empty[0]);
            const uint32_t idesc = make_idesc_bf16(256, NB, 0, 1);
            uint32_t st = 0, par = 0, sc = 0;
            for (int u = pair_id; u < total && ok; u += n_pairs) {
                for (int kc = 0; kc < nkc; ++kc) {
                    const int buf = sc & 1;
                    if (kc % A8_SUM == 0) {
                        ok = __all_sync(0xffffffffu, mbar_wait(&sm.acc_empty[buf], ((sc >> 1) & 1) ^ 1));
                        if (!ok) break;
                        tc_fence_after_sync();
                    }
                    const uint32_t d = tmem + buf * NB_MAX;
                    ok = __all_sync(0xffffffffu, mbar_wait_addr(full0 + st * 8, par));
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t a_lo = a_lo0 + st * (TILE * KC * 2 / 16), b_lo = b_lo0 + st * (2 * KC * KC * 2 / 16);
                    const bool last = kc % A8_SUM == A8_SUM - 1 || kc == nkc - 1;
                    if (elect_one()) {
                        if (kc % A8_SUM == 0)
                            tc_mma_bf16_pair_set(d, a_lo, a_hi, b_lo, b_hi, idesc);
                        else
                            tc_mma_bf16_pair_acc(d, a_lo, a_hi, b_lo, b_hi, idesc);
#pragma unroll
                        for (int k = 1; k < 4; ++k)
                            tc_mma_bf16_pair_acc(d, a_lo + 2 * k, a_hi, b_lo + 128 * k, b_hi, idesc);
                        tc_commit_pair_addr(empty0 + st * 8);        // frees the stage in both CTAs
                        if (last) tc_commit_pair(&sm.acc_full[buf]);
                    }
                    __syncwarp();
                    if (last) ++sc;
                    if (++st == A8_STAGES) { st = 0; par ^= 1; }
                }
            }
            if (!ok && lane == 0) lorc_set_status(p.q.status, LORC_ERR_TIMEOUT);
        }
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ epilogue (both CTAs): this CTA's 128 rows
        // A warp's 32 rows (two blocks) are its tensor-memory lanes; of the unit's columns it has the pieces k * 4 + group, k < NP.
        const int quarter = warp % 4, group = (warp - 4) >> 2;
        const uint32_t lead_acc_empty[2] = {mapa_shared(smem_u32(&sm.acc_empty[0]), 0), mapa_shared(smem_u32(&sm.acc_empty[1]), 0)};
        const uint32_t tlane = tmem + ((uint32_t)(quarter * 32) << 16);
        const float4* near = sm.near[lane & 15];
        const bool il = p.q.interleaved;
        constexpr int PIECES = DH / 32, SHARE = PIECES < 4 ? PIECES : 4;      // pieces of a head, and groups that have them
        const int c = group % PIECES;                                         // (the same piece of different heads)
        uint32_t sc = 0, turn = 0;
        for (int u = pair_id; u < total; u += n_pairs, turn ^= 1) {
            const int mt = u / p.n_units, col0 = (u - mt * p.n_units) * NB;
            Append8Row row;
            const int q = (mt * 2 + rank) * PER_TILE + quarter * 2 + (lane >> 4);
            append8_row(p.q, q < p.total_blocks ? q / p.q.n_blocks : -1, q % p.q.n_blocks, lane & 15, row);
            float a[NP][16], b[NP][16];
            for (int sum = 0; sum < sums && ok; ++sum, ++sc) {
                const int buf = sc & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(&sm.acc_full[buf], (sc >> 1) & 1));
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const uint32_t at = tlane + buf * NB_MAX + (k * 4 + group) / PIECES * DH;
#pragma unroll
                    for (int run = 0; run < 2; ++run) {
                        uint32_t r[16];
                        tmem_ld16(at + piece_column<DH>(c, il, run), r);
                        tmem_wait_ld();
                        float (&to)[16] = run ? b[k] : a[k];
#pragma unroll
                        for (int i = 0; i < 16; ++i) to[i] = sum == 0 ? __uint_as_float(r[i]) : to[i] + __uint_as_float(r[i]);
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(lead_acc_empty[buf]);      // this warp has read its part of the accumulator
            }
            // rotation, and the largest magnitudes; a sign bit stands for a number that is not finite (and does not count)
            float most[NP], before[NP];
            // (rows that are not to be written are rotated as position 0; their numbers are zero)
            const float4* far = reinterpret_cast<const float4*>(p.q.rope_table + (long long)(row.pos & ~(LORC_BLOCK8 - 1)) * (DH / 2));
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const int head = col0 / DH + (k * 4 + group) / PIECES;
                const bool val = head >= cv.n_kv;
                if (!val && ok) append8_rotate(c, il, far, near, a[k], b[k]);
                bool odd = false;
                most[k] = fmaxf(append8_most(a[k], odd), append8_most(b[k], odd));
                if (odd && row.fresh) most[k] = -most[k];
                sm.most[turn][k][group][quarter * 32 + lane] = most[k];
                before[k] = row.at >= 0 && row.has_old ? (val ? cv.v_scale : cv.k_scale)[row.at * cv.n_kv + (val ? head - cv.n_kv : head)] : 0.f;
            }
            ok = quarter_all(quarter, ok);                       // (behind the loads of `before`)
            if (!ok) break;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const int head = col0 / DH + (k * 4 + group) / PIECES, h = head >= cv.n_kv ? head - cv.n_kv : head;
                const bool val = head >= cv.n_kv;
                bool odd = signbit(most[k]);
                most[k] = fabsf(most[k]);
#pragma unroll
                for (int x = 1; x < SHARE; ++x) {
                    const float other = sm.most[turn][k][group / SHARE * SHARE + (group + x) % SHARE][quarter * 32 + lane];
                    odd |= signbit(other);
                    most[k] = fmaxf(most[k], fabsf(other));
                }
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) most[k] = fmaxf(most[k], __shfl_xor_sync(0xffffffffu, most[k], o));
                const bool any_odd = __ballot_sync(0xffffffffu, odd) >> (lane & 16) & 0xffff;
                const float scale = append8_scale<E4M3>(most[k], before[k]), inv = 1.f / scale;
                if ((lane & 15) == 0 && row.at >= 0 && c == 0) {
                    (val ? cv.v_scale : cv.k_scale)[row.at * cv.n_kv + h] = scale;
                    if (any_odd) lorc_set_status(p.q.status, LORC_ERR_ARG);
                }
                const bool clean = __all_sync(0xffffffffu, !any_odd && most[k] * inv <= (E4M3 ? 448.f : 127.f));
                uint8_t* dst = (val ? cv.v : cv.k) + (row.at * LORC_BLOCK8 + (row.pos & (LORC_BLOCK8 - 1))) * cv.n + h * DH;
                uint4* at[2] = {reinterpret_cast<uint4*>(dst + piece_column<DH>(c, il, 0)), reinterpret_cast<uint4*>(dst + piece_column<DH>(c, il, 1))};
                if (row.fresh) {
                    *at[0] = append8_codes<E4M3>(a[k], inv, clean);
                    *at[1] = append8_codes<E4M3>(b[k], inv, clean);
                } else if (row.old && scale != before[k]) {
                    const float keep = append8_keep(before[k], scale);
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) *at[i] = append8_recode<E4M3>(*at[i], keep);
                }
            }
        }
        if (!ok && lane == 0) lorc_set_status(p.q.status, LORC_ERR_TIMEOUT);
    }
    // both CTAs are done with tensor memory and with each other's barriers before either lets go
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive_release();
    cluster_wait_acquire();
    if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

}  // namespace

bool lorc_append8_tc_supported(const lorc_ctx* ctx) {
    return ctx->desc.d_model % KC == 0 && lorc_get_tmap_encode() && !(ctx->desc.flags & LORC_FLAG_DEBUG_FP32);
}

// Expected time in tenths of a microsecond: rounds of the persistent pairs over units of 256 rows x 128 columns.
long long lorc_append8_tc_time(const lorc_ctx* ctx, int batch, int T) {
    const long long blocks = (long long)batch * ((T + LORC_BLOCK8 - 2) / LORC_BLOCK8 + 1), units = (blocks + 15) / 16 * (2 * ctx->n / 128);
    const long long slots = ctx->sm_count / 2;
    return 80 + (units + slots - 1) / slots * 125 * ctx->desc.d_model / 4096;
}

cudaError_t lorc_append8_tc_launch(lorc_ctx* ctx, const LorcLayer& L, const Append8Params& q, const bf16* x, cudaStream_t st, int* launches) {
    const int D = ctx->desc.d_model, R = 2 * ctx->n, DH = ctx->desc.d_head;
    const bool e4m3 = q.cv.type == LORC_CACHE8_E4M3;
    CUtensorMap mapX, mapX16, mapA;
    {
        uint64_t xd[3] = {(uint64_t)D, (uint64_t)q.T, (uint64_t)q.cv.batch}, xs[2] = {(uint64_t)D * 2, (uint64_t)q.T * D * 2};
        uint32_t xb[3] = {KC, TILE, 1};
        if (!lorc_make_tmap_bf16(&mapX, x, 3, xd, xs, xb)) return cudaErrorInvalidValue;
        xb[1] = LORC_BLOCK8;
        if (!lorc_make_tmap_bf16(&mapX16, x, 3, xd, xs, xb)) return cudaErrorInvalidValue;
        uint64_t ad[2] = {(uint64_t)R, (uint64_t)D}, as[1] = {(uint64_t)R * 2};
        uint32_t ab[2] = {KC, KC};
        if (!lorc_make_tmap_bf16(&mapA, L.A_cat, 2, ad, as, ab)) return cudaErrorInvalidValue;
    }
    A8Params p;
    p.q = q; p.D = D; p.R = R;
    p.total_blocks = q.cv.batch * q.n_blocks;
    p.m_units = (p.total_blocks + 2 * PER_TILE - 1) / (2 * PER_TILE);
    // Width of a unit: the widest (fewest operand bytes per product), unless narrower ones finish the rounds of the persistent pairs
    // in less time: a unit's time goes with its width, and in part with the rows.
    const int slots = ctx->sm_count / 2;
    int nb = 128;
    if (R % NB_MAX == 0) {
        const long long wide = (long long)p.m_units * (R / NB_MAX), narrow = 2 * wide;
        if ((wide + slots - 1) / slots * (NB_MAX + 32) <= (narrow + slots - 1) / slots * (128 + 32)) nb = NB_MAX;
    }
    p.n_units = R / nb;
    const long long total = (long long)p.m_units * p.n_units;
    if (total > 0x7fffffffll - slots) return cudaErrorInvalidValue;      // (units are counted in 32 bits)
    const int pairs = total < slots ? (int)total : slots;
    const bool two = nb == NB_MAX;
    auto kernel = DH == 128 ? (e4m3 ? (two ? append8_tc_kernel<128, true, 2> : append8_tc_kernel<128, true, 1>)
                                    : (two ? append8_tc_kernel<128, false, 2> : append8_tc_kernel<128, false, 1>))
                            : (e4m3 ? (two ? append8_tc_kernel<64, true, 2> : append8_tc_kernel<64, true, 1>)
                                    : (two ? append8_tc_kernel<64, false, 2> : append8_tc_kernel<64, false, 1>));
    // the attribute belongs to a device's copy of the kernel: one flag per device and kernel
    static bool attr[64][8] = {};
    const bool known = ctx->device >= 0 && ctx->device < 64;
    const int which = (DH == 128 ? 4 : 0) + (e4m3 ? 2 : 0) + (two ? 1 : 0);
    if (!known || !attr[ctx->device][which]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(A8Smem) + 1024);
        if (e != cudaSuccess) return e;
        if (known) attr[ctx->device][which] = true;
    }
    *launches += 1;
    return lorc_launch_dependent(kernel, dim3(2 * pairs), dim3(A8_THREADS), sizeof(A8Smem) + 1024, st, mapX, mapX16, mapA, p);
}
