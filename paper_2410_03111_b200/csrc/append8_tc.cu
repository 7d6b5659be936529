// Cache write of uncompressed layers in 8 bits for prompt-sized token counts, on the tensor cores (sm_100a: TMA + tcgen05 + TMEM):
// projection, rotation and quantisation in one kernel.
//
// The rows of a tile are blocks of 16 tokens as the cache has them (aligned by position), so that the numbers which share a
// scale are 16 neighbouring lanes of tensor memory and the columns of one head: the largest magnitude of a block takes four
// shuffles, and a thread stores its row's codes.  The fp32 projection never goes to memory.
//
// Persistent CTA pairs (cta_group::2) walk units of 256 rows x 256 (or 128) columns of [W_k | W_v], K = D in 64-wide TMA
// stages; two accumulators in TMEM, so the epilogue of a unit runs under the MMAs of the next.  Rows of a block that are not new (earlier tokens, or behind the end) lie outside x and read as zero.
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
constexpr int A8_THREADS = 384;      // warp 0 TMA, warp 1 MMA (leader CTA issues), warps 4..11 epilogue
constexpr int PER_TILE = TILE / LORC_BLOCK8;

struct A8Smem {
    bf16 X[A8_STAGES][TILE * KC];          // [128 rows][64]                                                 16 KiB
    bf16 A[A8_STAGES][2][KC * KC];         // this CTA's half of the columns: two blocks of [64 D rows][64]  16 KiB
    float4 near[LORC_BLOCK8][33];          // (cos, sin) of the positions 0 .. 15, DH / 4 pairs of pairs each
    float most[2][8][32];                  // what the epilogue groups exchange, two heads in turn
    uint64_t full[A8_STAGES], empty[A8_STAGES], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
};

// The two epilogue warps that read the same lanes of tensor memory.
__device__ __forceinline__ void pair_sync(int quarter) { asm volatile("bar.sync %0, 64;" ::"r"(quarter + 1) : "memory"); }
// ... and whether both of them say so.
__device__ __forceinline__ bool pair_all(int quarter, bool mine) {
    int both;
    asm volatile(
        "{\n\t"
        ".reg .pred p, q;\n\t"
        "setp.ne.s32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, 64, p;\n\t"
        "selp.s32 %0, 1, 0, q;\n\t"
        "}\n"
        : "=r"(both)
        : "r"((int)mine), "r"(quarter + 1)
        : "memory");
    return both != 0;
}

// Piece c of a head of this thread's row: 32 of its DH columns (tensor-memory address `col0`), as two runs of 16 in which both
// members of every rotary pair meet: columns 16 c .. and DH / 2 + 16 c .., or 32 c .. and 32 c + 16 .. (interleaved pairs).  Keys are
// rotated: the row's position is that of the block's first row plus r, and R(16 b + r) = R(16 b) R(r), with R(16 b) from the
// table (`far`, one address for the 16 lanes of a block) and R(r), r < 16, from the copy of the table's first rows in shared memory
// (`near`).
template <int DH>
__device__ __forceinline__ void append8_piece(uint32_t col0, int c, bool key, bool interleaved, const float4* far, const float4* near,
                                              float (&a)[16], float (&b)[16]) {
    uint32_t ra[16], rb[16];
    tmem_ld16(col0 + (interleaved ? 32 * c : 16 * c), ra);
    tmem_ld16(col0 + (interleaved ? 32 * c + 16 : DH / 2 + 16 * c), rb);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        a[i] = __uint_as_float(ra[i]);
        b[i] = __uint_as_float(rb[i]);
    }
    if (!key) return;
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

// Half of a row of one head, by the thread whose tensor-memory lane it is; the block's rows are 16 neighbouring lanes, and the warp of
// the other epilogue group that reads the same lanes has the other half (`mine`, `theirs`: where the two leave their largest
// magnitudes; -1 stands for a number that is not finite).
template <int DH, bool E4M3>
__device__ __forceinline__ void append8_head(const Append8Params& p, const Append8Row& row, uint32_t col0, const float4* near, bool val,
                                             int head, int lane, int group, int quarter, float* mine, const float* theirs) {
    constexpr int PIECES = DH / 64;
    const Cache8View& cv = p.cv;
    float* scale_at = (val ? cv.v_scale : cv.k_scale) + row.at * cv.n_kv + head;
    const float before = row.at >= 0 && row.has_old ? *scale_at : 0.f;
    // (rows that are not to be written are rotated as position 0; their numbers are zero)
    const float4* far = reinterpret_cast<const float4*>(p.rope_table + (long long)(row.pos & ~(LORC_BLOCK8 - 1)) * (DH / 2));
    float a[PIECES][16], b[PIECES][16], most = 0.f;
    bool odd = false;
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
        append8_piece<DH>(col0, group * PIECES + c, !val, p.interleaved, far, near, a[c], b[c]);
        most = fmaxf(most, fmaxf(append8_most(a[c], odd), append8_most(b[c], odd)));
    }
    mine[lane] = odd && row.fresh ? -1.f : most;
    pair_sync(quarter);                                          // (behind the loads of `before`)
    const float other = theirs[lane];
    odd = (odd && row.fresh) || other < 0.f;
    most = fmaxf(most, other);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    const bool any_odd = __ballot_sync(0xffffffffu, odd) >> (lane & 16) & 0xffff;
    const float scale = append8_scale<E4M3>(most, before), inv = 1.f / scale;
    if ((lane & 15) == 0 && row.at >= 0 && group == 0) {
        *scale_at = scale;
        if (any_odd) lorc_set_status(p.status, LORC_ERR_ARG);
    }
    const bool clean = __all_sync(0xffffffffu, !any_odd && most * inv <= (E4M3 ? 448.f : 127.f));
    uint8_t* dst = (val ? cv.v : cv.k) + (row.at * LORC_BLOCK8 + (row.pos & (LORC_BLOCK8 - 1))) * cv.n + head * DH;
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
        const int pc = group * PIECES + c;
        uint4* at[2] = {reinterpret_cast<uint4*>(dst + (p.interleaved ? 32 * pc : 16 * pc)),
                        reinterpret_cast<uint4*>(dst + (p.interleaved ? 32 * pc + 16 : DH / 2 + 16 * pc))};
        if (row.fresh) {
            *at[0] = append8_codes<E4M3>(a[c], inv, clean);
            *at[1] = append8_codes<E4M3>(b[c], inv, clean);
        } else if (row.old && scale != before) {
            const float keep = (before > 0.f ? before : 0.f) / scale;
#pragma unroll 1
            for (int i = 0; i < 2; ++i) *at[i] = append8_recode<E4M3>(*at[i], keep);
        }
    }
}

struct A8Params {
    Append8Params q;
    int D, R, nb, m_units, n_units, total_blocks;
};

template <int DH, bool E4M3>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(A8_THREADS, 1)
append8_tc_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapX16,
                  const __grid_constant__ CUtensorMap mapA, const A8Params p) {
    extern __shared__ uint8_t raw[];
    A8Smem& sm = *reinterpret_cast<A8Smem*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = (int)cluster_ctarank();           // 0 = leader (issues the MMAs, owns the full / acc_empty barriers)
    const int pair_id = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int nkc = p.D / KC, total = p.m_units * p.n_units;
    const Cache8View& cv = p.q.cv;

    if (tid == 0) {
        for (int i = 0; i < A8_STAGES; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.acc_full[i], 1);
            mbar_init(&sm.acc_empty[i], 2 * 8);             // one arrival per epilogue warp, both CTAs
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
        const int half = p.nb / 2, boxes = half / KC;
        const uint32_t bytes = 2 * (TILE + half) * KC * 2;
        uint32_t st = 0, par = 1;
        for (int u = pair_id; u < total && ok; u += n_pairs) {
            const int mt = u / p.n_units, acol = (u - mt * p.n_units) * p.nb + rank * half;
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
            const uint32_t idesc = make_idesc_bf16(256, p.nb, 0, 1);
            uint32_t st = 0, par = 0, uc = 0;
            for (int u = pair_id; u < total && ok; u += n_pairs, ++uc) {
                const int buf = uc & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(&sm.acc_empty[buf], ((uc >> 1) & 1) ^ 1));
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t d = tmem + buf * NB_MAX;
                for (int kc = 0; kc < nkc; ++kc) {
                    ok = __all_sync(0xffffffffu, mbar_wait_addr(full0 + st * 8, par));
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t a_lo = a_lo0 + st * (TILE * KC * 2 / 16), b_lo = b_lo0 + st * (2 * KC * KC * 2 / 16);
                    if (elect_one()) {
                        if (kc == 0)
                            tc_mma_bf16_pair_set(d, a_lo, a_hi, b_lo, b_hi, idesc);
                        else
                            tc_mma_bf16_pair_acc(d, a_lo, a_hi, b_lo, b_hi, idesc);
#pragma unroll
                        for (int k = 1; k < 4; ++k)
                            tc_mma_bf16_pair_acc(d, a_lo + 2 * k, a_hi, b_lo + 128 * k, b_hi, idesc);
                        tc_commit_pair_addr(empty0 + st * 8);        // frees the stage in both CTAs
                    }
                    __syncwarp();
                    if (++st == A8_STAGES) { st = 0; par ^= 1; }
                }
                if (!ok) break;
                if (elect_one()) tc_commit_pair(&sm.acc_full[buf]);
                __syncwarp();
            }
            if (!ok && lane == 0) lorc_set_status(p.q.status, LORC_ERR_TIMEOUT);
        }
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ epilogue (both CTAs): this CTA's 128 rows
        // A warp's 32 rows (two blocks) are its tensor-memory lanes; warps 4..7 take one half of every head's columns, warps 8..11 the
        // other.  (With a group of four warps for each accumulator the epilogue of a launch's last units, which nothing hides, took
        // up to 14 us.)
        const int quarter = warp % 4, group = (warp - 4) >> 2;
        const uint32_t lead_acc_empty[2] = {mapa_shared(smem_u32(&sm.acc_empty[0]), 0), mapa_shared(smem_u32(&sm.acc_empty[1]), 0)};
        const float4* near = sm.near[lane & 15];
        uint32_t uc = 0, turn = 0;
        for (int u = pair_id; u < total; u += n_pairs, ++uc) {
            const int buf = uc & 1;
            const int mt = u / p.n_units, col0 = (u - mt * p.n_units) * p.nb;
            Append8Row row;
            const int q = (mt * 2 + rank) * PER_TILE + quarter * 2 + (lane >> 4);
            append8_row(p.q, q < p.total_blocks ? q / p.q.n_blocks : -1, q % p.q.n_blocks, lane & 15, row);
            ok = pair_all(quarter, mbar_wait(&sm.acc_full[buf], (uc >> 1) & 1));
            if (!ok) break;
            tc_fence_after_sync();
            const uint32_t tbase = tmem + ((uint32_t)(quarter * 32) << 16) + buf * NB_MAX;
#pragma unroll 1
            for (int c0 = 0; c0 < p.nb; c0 += DH, turn ^= 1) {
                const int head = (col0 + c0) / DH;
                const bool val = head >= cv.n_kv;
                append8_head<DH, E4M3>(p.q, row, tbase + c0, near, val, val ? head - cv.n_kv : head, lane, group, quarter,
                                       sm.most[turn][warp - 4], sm.most[turn][(warp - 4) ^ 4]);
            }
            // this warp has read its part of the accumulator
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(lead_acc_empty[buf]);
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

// Whether a launch runs here: see lorc_tc_append_gemm_supported, whose kernels have the same balance.
bool lorc_append8_tc_supported(const lorc_ctx* ctx, int batch, int T) {
    if (ctx->desc.d_model % KC || !lorc_get_tmap_encode() || (ctx->desc.flags & LORC_FLAG_DEBUG_FP32)) return false;
    const long long n_tok = (long long)batch * T;
    return 2 * ctx->n / 8 * ((n_tok + 15) / 16) > 6ll * ctx->sm_count;
}

cudaError_t lorc_append8_tc_launch(lorc_ctx* ctx, const LorcLayer& L, const Append8Params& q, const bf16* x, cudaStream_t st, int* launches) {
    const int D = ctx->desc.d_model, R = 2 * ctx->n, DH = ctx->desc.d_head;
    const bool e4m3 = q.cv.type == LORC_CACHE8_E4M3;
    auto kernel = DH == 128 ? (e4m3 ? append8_tc_kernel<128, true> : append8_tc_kernel<128, false>)
                            : (e4m3 ? append8_tc_kernel<64, true> : append8_tc_kernel<64, false>);
    // the attribute belongs to a device's copy of the kernel: one flag per device and kernel
    static bool attr[64][4] = {};
    const bool known = ctx->device >= 0 && ctx->device < 64;
    const int which = (DH == 128 ? 2 : 0) + (e4m3 ? 1 : 0);
    if (!known || !attr[ctx->device][which]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(A8Smem) + 1024);
        if (e != cudaSuccess) return e;
        if (known) attr[ctx->device][which] = true;
    }
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
    long long best = 0;
    for (int nb = R % NB_MAX ? NB_MAX / 2 : NB_MAX; nb >= 128; nb /= 2) {
        const long long rounds = ((long long)p.m_units * (R / nb) + slots - 1) / slots, cost = rounds * (nb + 32);
        if (!best || cost < best) {
            best = cost;
            p.nb = nb;
        }
    }
    p.n_units = R / p.nb;
    const long long total = (long long)p.m_units * p.n_units;
    const int pairs = total < slots ? (int)total : slots;
    *launches += 1;
    return lorc_launch_dependent(kernel, dim3(2 * pairs), dim3(A8_THREADS), sizeof(A8Smem) + 1024, st, mapX, mapX16, mapA, p);
}
