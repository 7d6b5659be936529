// Cache write of uncompressed layers in 8 bits for few tokens, in one launch: projection on the tensor cores with D split over a
// cluster, rotation and quantisation where the slices meet.
//
// With few tokens the time is that of the factor's stream, and a CTA that walks all of D (4096: 64 loads in a row) takes longer than
// memory does.  So a cluster of eight CTAs takes 128 rows x 128 columns (one or two heads), each an eighth of D, and every SM has some
// 256 KB to fetch.  The partial products (fp32, tensor memory) go to the CTA that owns the rows, sixteen of the 128 each, through
// distributed shared memory: that CTA adds them up in the order of the slices and has whole heads of whole groups, which is what a
// scale needs.  Nothing passes through the workspace.
//
// Two CTAs fit an SM, not for more in flight but because clusters of eight large ones do not fill the GPU (15 of them, where 16 tiles
// of columns want to run; the second round doubled the time).  8 KV heads of 128 dimensions, D 4096: 32 tokens 9.5 us, 64 10.6, 256 15.5;
// the factor's bytes take 2.6 at the rate of a copy, the rest is the chain of launch, three rounds of loads, two cluster barriers.
//
// Rows.  A group of 16 rows holds every number that shares a scale with one of its own: T <= 16 new tokens of 16 / T sequences (a
// token's block may have rows of earlier tokens, which are re-expressed in memory if the scale grows), or, with more tokens per
// sequence, one block of 16 positions as the cache has it.
#include <math.h>

#include "append8.cuh"
#include "sm100_pair.cuh"
#include "sm100_ptx.cuh"
#include "tc_kernels.cuh"

using namespace sm100;

namespace {

constexpr int TILE = 128;            // rows and columns of a cluster
constexpr int KC = 64;               // D elements per stage
constexpr int CTAS = 8;              // slices of D
constexpr int THREADS = 384;         // warp 0 TMA, warp 1 MMA, warps 4..11 epilogue
constexpr int SUM = 8;               // stages per accumulator (sums of 512 products, as in the kernel for prompts)
constexpr int MAX_SUMS = 2;          // accumulators of a slice (half of the tensor memory: two CTAs on an SM never wait for one another)
constexpr int GROUPS = TILE / LORC_BLOCK8;

constexpr int STAGES_MAX = 6;
constexpr int A_BYTES = KC * TILE * 2;           // of a stage: two blocks of [64 D rows][64 columns]
constexpr int GROUP_BYTES = LORC_BLOCK8 * KC * 2;

struct SpSmem {
    float most[LORC_BLOCK8][2];
    long long block[LORC_BLOCK8];                // block that a row's token goes to, -1: none
    uint64_t full[STAGES_MAX], empty[STAGES_MAX], acc_full;
    uint32_t tmem_base;
};
// Dynamic shared memory: the factor's stages, the rows' stages (the groups that tiles have; the MMAs read 128 rows all the same, what
// stands behind the groups is nobody's), and afterwards, in their place, the partial products of the owned rows by slice.
typedef float SpPart[LORC_BLOCK8][TILE + 4];     // (padded: the lanes of a warp write rows)
constexpr int RING_BYTES = 110 * 1024;           // two CTAs fit an SM
static_assert(CTAS * sizeof(SpPart) <= 3 * A_BYTES + 3 * GROUPS * GROUP_BYTES, "the partial products fit the stages");

struct SpParams {
    Append8Params q;
    int D, n_groups, per;            // per: sequences of a group, 0: groups are blocks
    int whole_boxes;                 // one box holds all groups of a tile
    int tile_groups, stages;         // groups of a tile, stages of 16 KB + 2 KB per group
};

__device__ __forceinline__ void st_cluster_f4(uint32_t cluster_addr, float x, float y, float z, float w) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}

// Row i of a group of whole sequences: as append8_row, with `fresh` for rows that stand for a token.
__device__ __forceinline__ void token_row(const Append8Params& p, int s, int t, Append8Row& row, bool report) {
    row.at = -1;
    row.pos = 0;
    row.fresh = row.old = row.has_old = false;
    const int len = p.cv.seq_lens[s];
    const bool fits = len >= 0 && len <= p.cv.max_seq_len && len <= p.max_pos && len <= p.cv.capacity;
    if ((!fits || len < p.T) && report) lorc_set_status(p.status, LORC_ERR_CAPACITY);
    const int pos = len - p.T + t;
    if (!fits || pos < 0) return;
    row.at = lorc_block8(p.cv, s, pos / LORC_BLOCK8);
    if (row.at < 0) {
        if (report) lorc_set_status(p.status, LORC_ERR_CAPACITY);
        return;
    }
    row.pos = pos;
    row.fresh = true;
    row.has_old = max(len - p.T, 0) > pos / LORC_BLOCK8 * LORC_BLOCK8;
}

template <int DH, bool E4M3>
__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(THREADS, 2)
append8_split_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapX16,
                     const __grid_constant__ CUtensorMap mapA, const SpParams p) {
    extern __shared__ uint8_t raw[];
    __shared__ SpSmem sm;
    uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    SpPart* const part = reinterpret_cast<SpPart*>(ring);
    const int stages = p.stages, x_bytes = p.tile_groups * GROUP_BYTES;
    uint8_t* const x_ring = ring + stages * A_BYTES;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = (int)cluster_ctarank();
    const int col0 = (int)blockIdx.x / CTAS * TILE, g0 = (int)blockIdx.y * GROUPS;
    const int groups = min(GROUPS, p.n_groups - g0);   // of this tile
    const int nkc = p.D / (CTAS * KC), k0 = rank * nkc * KC;
    const int sums = nkc > SUM ? 2 : 1;
    const Cache8View& cv = p.q.cv;
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 1);
        }
        mbar_init(&sm.acc_full, 1);
        fence_barrier_init();
        prefetch_tensormap(&mapX);
        prefetch_tensormap(&mapA);
    }
    if (warp == 1) {
        tmem_alloc(&sm.tmem_base, sums * TILE);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sm.tmem_base;
    bool ok = true;

    // What the epilogue's threads know of their row: row i of the group that this CTA owns, columns `cols` .. + 3 and DH / 2 behind
    constexpr int LANES = DH / 8;                      // threads that share a row of a head
    const int et = tid - 128, i = et / 16, c = et % LANES, sub = et % 16 / LANES;
    const int heads = col0 / DH + sub;                 // keys of all heads, then values
    const bool val = heads >= cv.n_kv;
    const int head = val ? heads - cv.n_kv : heads, cols = sub * DH + 4 * c;
    float* const scales = val ? cv.v_scale : cv.k_scale;
    Append8Row row;
    row.at = -1;
    row.pos = 0;
    row.fresh = row.old = row.has_old = false;
    float before = 0.f;
    float2 cs[4];

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer: the factor does not depend on the kernel in front
        const uint32_t bytes = (p.whole_boxes ? x_bytes : groups * (p.per ? p.per * p.q.T : LORC_BLOCK8) * KC * 2) + A_BYTES;
        auto load_factor = [&](int kc, int st) {
            mbar_arrive_expect_tx(&sm.full[st], bytes);
            tma_load_2d(ring + st * A_BYTES, &mapA, &sm.full[st], col0, k0 + kc * KC);
            tma_load_2d(ring + st * A_BYTES + A_BYTES / 2, &mapA, &sm.full[st], col0 + KC, k0 + kc * KC);
        };
        const bool issues = elect_one();
        if (issues)
            for (int kc = 0; kc < min(stages, nkc); ++kc) load_factor(kc, kc);
        __syncwarp();
        grid_dep_wait();
        grid_dep_launch();
        // where the groups' rows are in x; lane gi < 8: group gi
        int y = 0, s = 0;
        if (p.per) {
            s = (g0 + (lane & 7)) * p.per;
        } else {
            const int mine = min(g0 + (lane & 7), p.n_groups - 1);
            s = mine / p.q.n_blocks;
            const int len = cv.seq_lens[s], begin = max(len - p.q.T, 0) / LORC_BLOCK8 * LORC_BLOCK8;
            // (a length that is out of range is dealt with in the epilogue; coordinates stay near the tensor)
            y = max(min(begin + (mine - s * p.q.n_blocks) * LORC_BLOCK8 - (len - p.q.T), p.q.T), -LORC_BLOCK8);
        }
        int ys[GROUPS], ss[GROUPS];
#pragma unroll
        for (int gi = 0; gi < GROUPS; ++gi) {
            ys[gi] = __shfl_sync(0xffffffffu, y, gi);
            ss[gi] = __shfl_sync(0xffffffffu, s, gi);
        }
        uint32_t st = 0, par = 1;
        for (int kc = 0; kc < nkc; ++kc) {
            ok = __all_sync(0xffffffffu, mbar_wait(&sm.empty[st], par));
            if (!ok) break;
            if (issues) {
                if (kc >= stages) load_factor(kc, st);
                if (p.whole_boxes) {
                    tma_load_3d(x_ring + st * x_bytes, &mapX, &sm.full[st], k0 + kc * KC, 0, ss[0]);
                } else {
#pragma unroll
                    for (int gi = 0; gi < GROUPS; ++gi)
                        if (gi < groups)
                            tma_load_3d(x_ring + st * x_bytes + gi * GROUP_BYTES, &mapX16, &sm.full[st], k0 + kc * KC, ys[gi], ss[gi]);
                }
            }
            __syncwarp();
            if (++st == stages) { st = 0; par ^= 1; }
        }
        if (!ok) {
            // copies may be under way: the CTA does not leave before they must have landed
            if (lane == 0) lorc_set_status(p.q.status, LORC_ERR_TIMEOUT);
            for (const uint64_t since = global_timer_ns(); global_timer_ns() - since < 1000000ull;) {}
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA: A x rows (K-major), B factor blocks (MN-major)
        grid_dep_wait();
        grid_dep_launch();
        const uint32_t idesc = make_idesc_bf16(TILE, TILE, 0, 1);
        uint32_t st = 0, par = 0;
        for (int kc = 0; kc < nkc; ++kc) {
            ok = __all_sync(0xffffffffu, mbar_wait(&sm.full[st], par));
            if (!ok) break;
            tc_fence_after_sync();
            if (elect_one()) {
                const uint32_t x0 = smem_u32(x_ring + st * x_bytes), a0 = smem_u32(ring + st * A_BYTES);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    tc_mma_bf16(tmem + kc / SUM * TILE, make_smem_desc_sw128(x0 + k * 32, 0, 1024),
                                make_smem_desc_sw128(a0 + k * 2048, KC * KC * 2, 1024), idesc, kc % SUM != 0 || k != 0);
                tc_commit(&sm.empty[st]);
                if (kc == nkc - 1) tc_commit(&sm.acc_full);
            }
            __syncwarp();
            if (++st == stages) { st = 0; par ^= 1; }
        }
        if (!ok && lane == 0) lorc_set_status(p.q.status, LORC_ERR_TIMEOUT);
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ epilogue: where the owned rows go, while the products are formed
        grid_dep_wait();
        grid_dep_launch();
        const int g = g0 + rank;
        if (g < p.n_groups) {
            if (p.per) {
                const int sq = i / p.q.T, s = g * p.per + sq;
                if (sq < p.per && s < cv.batch) token_row(p.q, s, i - sq * p.q.T, row, et % 16 == 0);
            } else {
                append8_row(p.q, g / p.q.n_blocks, g % p.q.n_blocks, i, row);
            }
        }
        // (loads that nothing here waits for)
        if (row.fresh && row.has_old) before = scales[row.at * cv.n_kv + head];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            cs[e] = val || !row.fresh ? make_float2(1.f, 0.f)
                                      : p.q.rope_table[(long long)row.pos * (DH / 2) + (p.q.interleaved ? (e < 2 ? 2 * c + e : DH / 4 + 2 * c + e - 2) : 4 * c + e)];
        ok = __all_sync(0xffffffffu, mbar_wait(&sm.acc_full, 0));
        if (!ok && lane == 0) lorc_set_status(p.q.status, LORC_ERR_TIMEOUT);
    } else {
        grid_dep_wait();
        grid_dep_launch();
    }
    cluster_arrive_release();
    cluster_wait_acquire();                            // no CTA of the cluster needs its stages any more
    if (warp >= 4) {
        // this slice's products to the CTAs that own the rows: a thread has half of a row's columns
        const int quarter = warp % 4, half = (warp - 4) / 4, r = quarter * 32 + lane, owner = r / LORC_BLOCK8;
        if (ok) {
            tc_fence_after_sync();
            const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + half * 64;
            const uint32_t to = mapa_shared(smem_u32(&part[rank][r % LORC_BLOCK8][half * 64]), owner);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint32_t x[16];
                tmem_ld16(from + 16 * h, x);
                tmem_wait_ld();
                if (sums > 1) {
                    uint32_t z[16];
                    tmem_ld16(from + TILE + 16 * h, z);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) + __uint_as_float(z[j]));
                }
                if (owner < groups)
#pragma unroll
                    for (int j = 0; j < 16; j += 4)
                        st_cluster_f4(to + (16 * h + j) * 4, __uint_as_float(x[j]), __uint_as_float(x[j + 1]), __uint_as_float(x[j + 2]),
                                      __uint_as_float(x[j + 3]));
            }
            tc_fence_before_sync();
        }
    }
    cluster_arrive_release();
    cluster_wait_acquire();                            // every slice of the owned rows has arrived
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, sums * TILE);
    }
    if (warp < 4 || rank >= groups) return;
    float x[8];
#pragma unroll
    for (int run = 0; run < 2; ++run) {
        float4 y[CTAS];
#pragma unroll
        for (int k = 0; k < CTAS; ++k) y[k] = *reinterpret_cast<const float4*>(&part[k][i][cols + run * (DH / 2)]);
#pragma unroll
        for (int n = CTAS / 2; n > 0; n /= 2)
#pragma unroll
            for (int k = 0; k < n; ++k) {
                y[k].x += y[k + n].x;
                y[k].y += y[k + n].y;
                y[k].z += y[k + n].z;
                y[k].w += y[k + n].w;
            }
        x[4 * run] = y[0].x;
        x[4 * run + 1] = y[0].y;
        x[4 * run + 2] = y[0].z;
        x[4 * run + 3] = y[0].w;
    }
    if (!val) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (p.q.interleaved) {
                const float a = x[2 * e], b = x[2 * e + 1];
                x[2 * e] = a * cs[e].x - b * cs[e].y;
                x[2 * e + 1] = a * cs[e].y + b * cs[e].x;
            } else {
                const float a = x[e], b = x[4 + e];
                x[e] = a * cs[e].x - b * cs[e].y;
                x[4 + e] = a * cs[e].y + b * cs[e].x;
            }
        }
    }
    bool odd = false;
    float most = append8_most(x, odd);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    const uint32_t same = (LANES == 16 ? 0xffffu : 0xffu) << (lane & (32 - LANES));
    odd = (__ballot_sync(0xffffffffu, odd) & same) != 0;
    if (c == 0) sm.most[i][sub] = odd ? -most : most;              // (a sign bit: some are not finite)
    if (et % 16 == 0) sm.block[i] = row.fresh ? row.at : -1;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (!row.fresh) return;
    most = 0.f;
    odd = false;
#pragma unroll
    for (int j = 0; j < LORC_BLOCK8; ++j)
        if (sm.block[j] == row.at) {
            most = fmaxf(most, fabsf(sm.most[j][sub]));
            odd |= signbit(sm.most[j][sub]);
        }
    const float scale = append8_scale<E4M3>(most, before), inv = 1.f / scale;
    const int in_block = row.pos % LORC_BLOCK8;
    uint8_t* dst = (val ? cv.v : cv.k) + row.at * LORC_BLOCK8 * cv.n + head * DH;
#pragma unroll
    for (int run = 0; run < 2; ++run)
        *reinterpret_cast<uint32_t*>(dst + (long long)in_block * cv.n + 4 * c + run * (DH / 2)) =
            lorc_to_codes2<E4M3>(x[4 * run] * inv, x[4 * run + 1] * inv) | lorc_to_codes2<E4M3>(x[4 * run + 2] * inv, x[4 * run + 3] * inv) << 16;
    // the first new token of the block: its scale, and the earlier tokens under it
    const bool first = i == 0 || sm.block[i - 1] != row.at;
    if (!first) return;
    if (c == 0) {
        scales[row.at * cv.n_kv + head] = scale;
        if (odd) lorc_set_status(p.q.status, LORC_ERR_ARG);
    }
    if (!row.has_old || scale == before) return;
    const float keep = append8_keep(before, scale);
    for (int r = c; r < in_block; r += LANES)
#pragma unroll 1
        for (int j = 0; j < DH; j += 16) {
            uint4* at = reinterpret_cast<uint4*>(dst + (long long)r * cv.n + j);
            *at = append8_recode<E4M3>(*at, keep);
        }
}

}  // namespace

// Groups of 16 rows that a launch has.
static long long split_groups(int batch, int T) {
    if (T > LORC_BLOCK8) return (long long)batch * ((T + LORC_BLOCK8 - 2) / LORC_BLOCK8 + 1);
    const int per = LORC_BLOCK8 / T;
    return ((long long)batch + per - 1) / per;
}

bool lorc_append8_split_supported(const lorc_ctx* ctx, int batch, int T) {
    const int D = ctx->desc.d_model;
    if (D % (CTAS * KC) || D > CTAS * KC * SUM * MAX_SUMS || !lorc_get_tmap_encode() || (ctx->desc.flags & LORC_FLAG_DEBUG_FP32)) return false;
    return (split_groups(batch, T) + GROUPS - 1) / GROUPS <= 65535;
}

// Expected time in tenths of a microsecond.  (Two CTAs per SM, but a cluster lies within a part of the GPU: 33 of the 37 that 148 SMs
// could hold.)
long long lorc_append8_split_time(const lorc_ctx* ctx, int batch, int T) {
    const long long groups = split_groups(batch, T), tiles = (groups + GROUPS - 1) / GROUPS, clusters = tiles * (2 * ctx->n / TILE);
    const long long slots = 2 * ctx->sm_count / (CTAS + 1), D = ctx->desc.d_model;
    if (clusters <= slots / 4) return 52 + 24 * D / 4096 + 2 * (groups < GROUPS ? groups : GROUPS);
    if (clusters <= slots / 2) return 62 + 24 * D / 4096 + 6 * (groups < GROUPS ? groups : GROUPS);
    return (clusters + slots - 1) / slots * (105 + 50 * D / 4096);
}

cudaError_t lorc_append8_split_launch(lorc_ctx* ctx, const LorcLayer& L, const Append8Params& q, const bf16* x, cudaStream_t st, int* launches) {
    const int D = ctx->desc.d_model, R = 2 * ctx->n, DH = ctx->desc.d_head, T = q.T, batch = q.cv.batch;
    SpParams p;
    p.q = q; p.D = D;
    p.per = T <= LORC_BLOCK8 ? LORC_BLOCK8 / T : 0;
    p.n_groups = (int)split_groups(batch, T);
    p.whole_boxes = p.per && LORC_BLOCK8 % T == 0;
    p.tile_groups = p.n_groups < GROUPS ? p.n_groups : GROUPS;
    const int behind = (GROUPS - p.tile_groups) * GROUP_BYTES;       // what the MMAs of the last stage read behind its groups
    p.stages = (RING_BYTES - behind) / (A_BYTES + p.tile_groups * GROUP_BYTES);
    if (p.stages > STAGES_MAX) p.stages = STAGES_MAX;
    CUtensorMap mapX, mapX16, mapA;
    {
        uint64_t xd[3] = {(uint64_t)D, (uint64_t)T, (uint64_t)batch}, xs[2] = {(uint64_t)D * 2, (uint64_t)T * D * 2};
        uint32_t xb[3] = {KC, (uint32_t)(p.per ? T : LORC_BLOCK8), (uint32_t)(p.per ? p.per : 1)};
        if (!lorc_make_tmap_bf16(&mapX16, x, 3, xd, xs, xb)) return cudaErrorInvalidValue;
        if (p.whole_boxes) xb[2] *= p.tile_groups;
        if (!lorc_make_tmap_bf16(&mapX, x, 3, xd, xs, xb)) return cudaErrorInvalidValue;
        uint64_t ad[2] = {(uint64_t)R, (uint64_t)D}, as[1] = {(uint64_t)R * 2};
        uint32_t ab[2] = {KC, KC};
        if (!lorc_make_tmap_bf16(&mapA, L.A_cat, 2, ad, as, ab)) return cudaErrorInvalidValue;
    }
    const bool e4m3 = q.cv.type == LORC_CACHE8_E4M3;
    auto kernel = DH == 128 ? (e4m3 ? append8_split_kernel<128, true> : append8_split_kernel<128, false>)
                            : (e4m3 ? append8_split_kernel<64, true> : append8_split_kernel<64, false>);
    const size_t smem = RING_BYTES + 1024;
    // the attribute belongs to a device's copy of the kernel: one flag per device and kernel
    static bool attr[64][4] = {};
    const bool known = ctx->device >= 0 && ctx->device < 64;
    const int which = (DH == 128 ? 2 : 0) + (e4m3 ? 1 : 0);
    if (!known || !attr[ctx->device][which]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (known) attr[ctx->device][which] = true;
    }
    *launches += 1;
    return lorc_launch_dependent(kernel, dim3(R / TILE * CTAS, (unsigned)((p.n_groups + GROUPS - 1) / GROUPS)), dim3(THREADS), smem, st, mapX,
                                 mapX16, mapA, p);
}
