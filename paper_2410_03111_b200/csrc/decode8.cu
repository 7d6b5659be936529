// Attention over the 8-bit cache of uncompressed layers, one or few queries per sequence, on the warp-level tensor cores.
//
// One pass over 2 n bytes per token, bound by HBM: a block streams (sequence, KV head) pairs; a producer warp keeps D8_STAGES
// 128-token stages of codes in flight by TMA, and each of four consumer warps takes 32 of a stage's tokens, two blocks of the cache
// with a scale each for their keys and values.  A warp of its own rotates the queries of the next sequence.  Scores and outputs are
// computed transposed (tokens, then dimensions on the M side of the m16n8k16 tiles, the G <= 8 query heads on the N side: tiles of
// the tcgen05 kind would be 128 wide there).  Codes become fp16 numbers exactly, in registers:
//
//   S^T[16 tok x 8] = K[16 tok x d] . Q^^T      Q^ = RoPE(q, N-1) brought to [1, 2) by a power of two per head, in two fp16 parts
//                                               (22 bits); the scale of the keys, 1 / sqrt(d) and log2 e multiply the fp32 sums
//   l += 2^(S - m)
//   O^T[d x 8]     += V^T[d x 16 tok] . Y^T     Y = c 2^(S - w) in one fp16 part, c the scale of the values: each weight is
//                                               off by 2^-11 of itself at most, which averages out over tokens; bf16 outputs
//                                               lose 2^-8
//
// m is raised to the largest score when that exceeds it by more than 2^8; w stands 2^7 below the heaviest weight, until one is 2^15
// above it.  fp16 holds 2^15, and the room above 1 is room below: a weight below 2^-21 of the heaviest is off by 2^-32 of that one (with the
// heaviest weight at 1, 2^-25, and tokens of less than that counted in l only).
//
// A 16-bit word of a row is two dimensions.  Key fragments take the dimensions in the order in which ldmatrix delivers bytes, and the
// query fragments take the same order; for the values a transposed 8 x 8 matrix of words holds two dimensions of two tokens per
// register, whose bytes are paired by token: fragment row g is dimension 2 g of the 16, row g + 8 dimension 2 g + 1.
//
// Units of 64 tokens of all sequences form one list, cut into equal parts for the blocks of a KV head that are resident at
// once: all of them stream from the start to the end of the launch whatever the lengths are.  A part may begin and end inside
// a sequence; what it computes of a sequence that it does not hold alone goes to memory, un-normalised, and the last of the
// sequence's parts to get there adds them up.  (A merge kernel of its own cost 6 to 8 us more; the same by the queries' warp, so that
// the others go on, 1 to 3 us more, since one warp takes longer over it at the end of the launch.)
//
// Several queries of a sequence (prompt chunks of few tokens, drafts that are verified) are rows of as many queries as fit the eight
// columns; each column has its own last token.  (8 x 4096 tokens, four heads per KV head: 4 queries 31 us, one by one 43; 16
// queries 90 and 147.)
//
// Measured, 8 KV heads of 128 dimensions: 16 x 4129 tokens 29.4 us (4.6 TB/s), 4 x 32777 48.8 us (5.5), 64 sequences of 512 to
// 16384 185 us (6.0; a copy 6.6), 202 to 217 (5.1 to 5.5) when calls go on and the power cap lowers the clock, 128 x 300 31 us:
// there it is the 1.5 us per sequence and block from its last tile's arrival to the next one's first products.  (Query fragments
// made by the queries' warp save 1 us of the 31 and cost 1 of the 13 of 64 x 200.)
#include <math.h>

#include "cache8.cuh"
#include "sm100_ptx.cuh"
#include "tc_kernels.cuh"

using namespace sm100;

namespace {

constexpr int D8_TILE = 128;         // tokens per stage (32 per consumer warp)
constexpr int D8_UNIT = 6;           // work is dealt out by 64 tokens (2^6),
constexpr int D8_SHORT = 8;          // or, where no sequence has more than 256 (2^8), by whole sequences
constexpr int D8_STAGES = 3;
constexpr int D8_THREADS = 192;      // warps 0..3 consumers, warp 4 TMA and scales, warp 5 queries
constexpr int D8_BLOCKS_PER_SM = 2;
constexpr int D8_LIST = 128;          // rows of a list that are looked at in one go
constexpr float D8_RAISE = 8.f;      // a reference is raised only when it is exceeded by more than this (log2 units)
constexpr float D8_HEAD = 7.f;       // and the heaviest weight then stands at 2^7, so weights reach 2^15 as fp16 numbers
constexpr float D8_BELOW = 118.f, D8_ABOVE = 125.f;    // how far the reference of the weights may lie from that of the scores
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_half(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

// log2 |x| of a scale, -infinity for zero (absolute error below 2^-15, a thirtieth of what a weight loses as an fp16 number)
__device__ __forceinline__ float d8_log2(float x) { return __log2f(fabsf(x)); }

template <int DH>
struct D8Smem {
    uint8_t kv[D8_STAGES][2][D8_TILE * DH];     // keys, values of a stage: rows of DH bytes, swizzled (128 or 64 bytes)
    float o[4][4][DH + 4];                      // at the end of a sequence's part: every warp's un-normalised output, four heads at a time
    float qs[8][DH];                            // rotated queries of the G heads (rows G..7 zero)
    float m[4][8], l[4][8], w[4][8];
    int last;
    alignas(16) float scale[D8_STAGES][2][D8_TILE / 16];    // scales of a stage's blocks, keys and values
    uint64_t full[D8_STAGES], empty[D8_STAGES], q_full, q_empty;
    uint32_t dead[D8_STAGES];                   // blocks of the stage whose page lies outside the pool, one bit each
};

struct D8Params {
    const bf16* q;
    bf16* out;
    Cache8View cv;
    const float2* rope_table;
    float* part_ml;                             // [n_kv][parts + rows][G][2]: reference (log2 units), sum
    float* part_o;                              // [n_kv][parts + rows][G][DH]
    unsigned* count;                            // [n_kv][parts], zero between calls
    int* status;
    int G, n_kv, T, interleaved, max_pos, box_rows;
    int Q, per_seq, cols;                       // queries of a sequence that share a row, rows per sequence, G * Q
    unsigned page_magic;                        // see d8_page_of
    int rows;                                   // batch * per_seq
    int each;                                   // parts / rows, where a list has at most 128 rows
    int unit;                                   // D8_UNIT or D8_SHORT
    int parts, least;                           // 0: a block per row and KV head; else parts of the list, of `least` steps at least
};

// Logical page of block b (of 16 tokens): b divided by the blocks of a page, with page_magic = 2^32 divided by them, rounded up.
// b page_magic / 2^32 exceeds the quotient by less than b / 2^32 < 1.
__device__ __forceinline__ int d8_page_of(const D8Params& p, int b) {
    const int per = p.cv.page_size / LORC_BLOCK8;
    if (per == 1) return b;
    const int q = (int)__umulhi((unsigned)b, p.page_magic);
    return q * per > b ? q - 1 : q;
}

// Row r = s per_seq + j stands for the queries j Q .. j Q + Q - 1 of sequence s (the last row may have fewer): the tokens up to the
// last one's own (0: nothing to attend to).
__device__ __forceinline__ int d8_queries(const D8Params& p, int j) { return min(p.Q, p.T - j * p.Q); }
__device__ __forceinline__ int d8_len(const D8Params& p, int r, int* status) {
    if (p.T == 1) return lorc_len8(p.cv, r, p.max_pos, status);
    const int s = r / p.per_seq, len = lorc_len8(p.cv, s, p.max_pos, status);
    if (len < p.T) {
        if (len > 0 && status) lorc_set_status(status, LORC_ERR_ARG);
        return 0;
    }
    return len - max(p.T - (r - s * p.per_seq + 1) * p.Q, 0);
}
// Units of a row on the list; a row without tokens has one, in which its zeros are written.
__device__ __forceinline__ int d8_weight(const D8Params& p, int len) { return len <= 0 ? 1 : ((len - 1) >> p.unit) + 1; }

// What a block works on: units [f, end) of the list, beginning in row `row`, whose first unit is `first`; `per` units to a part.
// Unit u of the list belongs to part base + u / per.  (The host sees to it that a list has fewer than 2^30 units.)
struct D8Range {
    int f, end, first, row, per, base;
};

// By whole warps.  Up to 128 rows are loaded at once.
__device__ __forceinline__ D8Range d8_range(const D8Params& p, int part, int lane) {
    D8Range r;
    r.base = 0;
    if (p.parts == 0) {
        r.row = part;
        r.f = r.first = 0;
        r.end = r.per = d8_weight(p, d8_len(p, part, nullptr));
        return r;
    }
    int w[4], sum = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = c * 32 + lane < p.rows ? d8_weight(p, d8_len(p, c * 32 + lane, nullptr)) : 0;
    for (int i = 128 + lane; i < p.rows; i += 32) sum += d8_weight(p, d8_len(p, i, nullptr));
    const int total = __reduce_add_sync(0xffffffffu, sum + w[0] + w[1] + w[2] + w[3]);
    r.per = max((int)((unsigned)(total + p.parts - 1) / (unsigned)p.parts), p.least);
    if (p.each > 0) {
        // As many parts for every row, where that gives no block more than a quarter above the even cut: each row is a list of its
        // own, no part ends one row and begins the next.  (8 KV heads of 128 dimensions, us, this and the even cut, in brackets the
        // longest part over the even one: 16 x 1000 14.1 and 17.0, 16 x 4129 29.8 and 32.6, 16 x 16000 85.3 and 87.7 (1.15); 12 x 4129
        // 24.1 and 27.7 (1.0), 8 x 2000 14.2 and 17.2 (1.14), 32 x 8000 82.6 and 86.5 (1.15), 4 x 16000 29.1 and 31.0 (1.0); two to eight
        // sequences of 1000 the same.  Beyond: 24 x 1000 15.8 and 20.1, 24 x 4129 45.3 and 41.1, 24 x 8000 80.1 and 68.6 (1.5).)
        const int most = __reduce_max_sync(0xffffffffu, max(max(w[0], w[1]), max(w[2], w[3])));
        const int longest = (int)((unsigned)(most + p.each - 1) / (unsigned)p.each);
        if (longest <= r.per + max(r.per / 4, 2)) {
            r.row = part / p.each;
            r.base = r.row * p.each;
            r.first = 0;
            r.f = r.end = 0;
            if (r.row < p.rows) {
                const int mine = d8_weight(p, d8_len(p, r.row, nullptr));
                r.per = max((int)((unsigned)(mine + p.each - 1) / (unsigned)p.each), p.least);
                r.f = (part - r.base) * r.per;
                r.end = min(r.f + r.per, mine);
            }
            return r;
        }
    }
    r.f = part * r.per;
    r.end = min(r.f + r.per, total);
    r.row = p.rows;
    r.first = 0;
    if (r.f >= r.end) return r;
    int before = 0;
    bool found = false;
    auto look = [&](int i0, int x) {             // rows i0 .. i0 + 31, lane's weight x
        const int end = warp_scan(x, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, r.f < before + end);
        if (hit) {
            const int l = __ffs(hit) - 1;
            r.row = i0 + l;
            r.first = before + __shfl_sync(0xffffffffu, end - x, l);
            found = true;
        } else {
            before += __shfl_sync(0xffffffffu, end, 31);
        }
    };
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (!found && c * 32 < p.rows) look(c * 32, w[c]);
    for (int i0 = 128; !found && i0 < p.rows; i0 += 32) look(i0, i0 + lane < p.rows ? d8_weight(p, d8_len(p, i0 + lane, nullptr)) : 0);
    if (!found) r.end = r.f;                     // (lengths that change under way)
    return r;
}

// Four numbers of the result: sums divided by the denominator.
__device__ __forceinline__ void d8_store(const D8Params& p, long long at, const float4& acc, float L) {
    const float inv = L != 0.f ? 1.f / L : 0.f;
    const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), hi = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
    *reinterpret_cast<uint2*>(p.out + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    if (L == 0.f) lorc_set_status(p.status, LORC_ERR_EMPTY);
}

// Where column h of a row goes: head h of the KV head, or head h % G of query h / G.
template <bool MULTI>
__device__ __forceinline__ long long d8_out_row(const D8Params& p, int row, int kvh, int h) {
    const int H_q = p.G * p.n_kv;
    if (!MULTI) return (long long)row * H_q + kvh * p.G + h;
    const int s = row / p.per_seq, t = (row - s * p.per_seq) * p.Q + h / p.G;
    return ((long long)s * p.T + t) * H_q + kvh * p.G + h % p.G;
}

// Merge of a row that was cut into n pieces: the `cols` columns of a KV head, by 128 threads, four dimensions each.  Pieces come four at a
// time, and the sums so far are brought to a new reference with each four: one round trip to L2 per four pieces.
template <int DH, bool MULTI>
__device__ __forceinline__ void d8_merge(const D8Params& p, long long unit0, int n, int row, int kvh, int cols, int tid) {
    const int stride = MULTI ? p.cols : p.G;
    for (int i = tid; i < cols * (DH / 4); i += 128) {
        const int h = i / (DH / 4), d = (i - h * (DH / 4)) * 4;
        const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + unit0 + h;
        const float* po = p.part_o + (unit0 + h) * DH + d;
        float M = -INFINITY, L = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c0 = 0; c0 < n; c0 += 4) {
            float2 x[4];
            float4 y[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                x[c] = make_float2(0.f, 0.f);
                y[c] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (c0 + c < n) {
                    x[c] = __ldcg(ml + (long long)(c0 + c) * stride);
                    y[c] = __ldcg(reinterpret_cast<const float4*>(po + (long long)(c0 + c) * stride * DH));
                }
            }
            float now = M;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (x[c].y != 0.f) now = fmaxf(now, x[c].x);
            if (now > M) {
                const float alpha = M == -INFINITY ? 0.f : exp2f(M - now);
                L *= alpha;
                acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
                M = now;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (x[c].y == 0.f) continue;
                const float wgt = exp2f(x[c].x - M);
                L += wgt * x[c].y;
                acc.x += wgt * y[c].x;
                acc.y += wgt * y[c].y;
                acc.z += wgt * y[c].z;
                acc.w += wgt * y[c].w;
            }
        }
        d8_store(p, d8_out_row<MULTI>(p, row, kvh, h) * DH + d, acc, L);
    }
}

// MULTI: rows of several queries.
template <int DH, bool E4M3, bool MULTI>
__global__ void __launch_bounds__(D8_THREADS, D8_BLOCKS_PER_SM)
decode8_mma_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const D8Params p) {
    constexpr int KS = DH / 16;                  // pieces of 16 dimensions
    extern __shared__ uint8_t d8_raw[];
    D8Smem<DH>& sm = *reinterpret_cast<D8Smem<DH>*>((reinterpret_cast<uintptr_t>(d8_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;       // fragment row / column group of this lane
    const int kvh = (int)blockIdx.x % p.n_kv, part = (int)blockIdx.x / p.n_kv;
    const Cache8View& cv = p.cv;
    const int G = p.G;
    if (tid == 0) {
        for (int i = 0; i < D8_STAGES; ++i) {
            mbar_init(&sm.full[i], 2);           // the copies, and the scales
            mbar_init(&sm.empty[i], 4);
        }
        mbar_init(&sm.q_full, 1);
        mbar_init(&sm.q_empty, 4);
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
        // ------------------------------------------------------------------ producer (one elected lane issues the copies)
        // Tiles of 128 tokens, row after row.  Lane b + 8 i looks up the page of block b and loads its scale (i = 0: keys, 1:
        // values; other lanes idle): the page two tiles ahead, the scale while the tile's copies are under way.  A box in a page
        // outside the pool (reported), or behind the end of the sequence, is fetched from behind the pool, where it reads as zero.
        struct Tile {
            int s, t0, t_end, page, y;           // page of this lane's block and the block's first row in it
        };
        const int nbox = D8_TILE / p.box_rows, blk = lane & 7;
        const long long per_page = (cv.page_table ? cv.page_size : cv.seq_stride) / LORC_BLOCK8;
        int f = range.f, first = range.first, row = range.row, len = 0;
        Tile next = {0, 0, 0, 0, 0};
        bool more = true;
        // moves `next` to the tile behind it (before the first call: to the first one); more: there is one
        auto advance = [&]() {
            next.t0 += D8_TILE;
            while (next.t0 >= next.t_end) {
                if (len > 0) {                   // this row is done
                    const int w = d8_weight(p, len);
                    f = min(first + w, range.end);
                    first += w;
                    ++row;
                }
                for (; f < range.end && row < p.rows; ++row) {
                    len = d8_len(p, row, nullptr);
                    if (len > 0) break;
                    f = ++first;
                }
                if (f >= range.end || row >= p.rows) {
                    more = false;
                    return;
                }
                next.s = p.T == 1 ? row : row / p.per_seq;
                next.t0 = (f - first) << p.unit;
                next.t_end = min(len, (min(first + d8_weight(p, len), range.end) - first) << p.unit);
            }
            // (looked at only when the tile's turn comes: the table access is under way until then)
            const int pos = next.t0 + blk * LORC_BLOCK8;
            next.page = next.s;
            next.y = pos;
            if (cv.page_table != nullptr) {
                const int lp = d8_page_of(p, pos / LORC_BLOCK8);
                next.page = cv.n_pages;
                next.y = pos - lp * cv.page_size;
                if (lane < 16 && pos < next.t_end) next.page = cv.page_table[(long long)next.s * cv.max_pages_per_seq + lp];
            }
        };
        Tile now;
        float scale = 0.f, before = 0.f;         // this lane's scale of the tile, and of the one before
        int fetched = 0, prev = -1;              // stages that may have copies under way; the stage that `before` belongs to
        advance();
        bool live = more;
        now = next;
        if (live) advance();
        while (live) {
            // All that a tile needs is known before its stage is free: the time from there to the copies counts.  (With the
            // divisions of the page arithmetic behind the wait, 64 x 8448 tokens in 64-token pages took 219 us, now 174.)
            const bool bad = cv.page_table != nullptr && lane < 16 && now.t0 + blk * LORC_BLOCK8 < now.t_end &&
                             (now.page < 0 || now.page >= cv.n_pages);
            if (bad) lorc_set_status(p.status, LORC_ERR_CAPACITY);
            const uint32_t dead = __ballot_sync(0xffffffffu, bad) & 0xff;
            const int boxes = min(nbox, (now.t_end - now.t0 + p.box_rows - 1) / p.box_rows);      // (the others are not fetched)
            int z[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[j] = __shfl_sync(0xffffffffu, bad ? cv.n_pages : now.page, j * p.box_rows / LORC_BLOCK8 & 7);
                y[j] = __shfl_sync(0xffffffffu, now.y, j * p.box_rows / LORC_BLOCK8 & 7);
            }
            scale = 0.f;
            if (lane < 16 && now.t0 + blk * LORC_BLOCK8 < now.t_end && !bad) {
                const long long at = (long long)now.page * per_page + now.y / LORC_BLOCK8;
                scale = (lane < 8 ? cv.k_scale : cv.v_scale)[at * p.n_kv + kvh];
            }
            ok = __all_sync(0xffffffffu, mbar_wait(&sm.empty[st], par ^ 1));
            if (!ok) break;
            if (elect_one()) {
                sm.dead[st] = dead;
                mbar_arrive_expect_tx(&sm.full[st], 2 * DH * p.box_rows * boxes);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j >= boxes) break;
                    tma_load_3d(sm.kv[st][0] + j * p.box_rows * DH, &mapK, &sm.full[st], kvh * DH, y[j], z[j]);
                    tma_load_3d(sm.kv[st][1] + j * p.box_rows * DH, &mapV, &sm.full[st], kvh * DH, y[j], z[j]);
                }
            }
            __syncwarp();
            if (prev >= 0) {                     // the scales of the tile before have come
                if (lane < 16) sm.scale[prev][lane >> 3][blk] = before;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.full[prev]);
            }
            before = scale;
            prev = st;
            live = more;
            now = next;
            if (more) advance();
            if (++st == D8_STAGES) { st = 0; par ^= 1; }
            if (fetched < D8_STAGES) ++fetched;
        }
        if (prev >= 0) {
            if (lane < 16) sm.scale[prev][lane >> 3][blk] = before;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.full[prev]);
        }
        // The block stays until the copies into its shared memory have landed, also when a wait has run out.
        for (; fetched > 0; --fetched) {
            if (--st < 0) { st = D8_STAGES - 1; par ^= 1; }
            if (!mbar_wait(&sm.full[st], par)) ok = false;
        }
        if (!ok && lane == 0) lorc_set_status(p.status, LORC_ERR_TIMEOUT);
        return;
    }
    if (warp == 5) {
        // ------------------------------------------------------------------ queries: RoPE(q, position) of the row's columns, one row ahead
        constexpr int E = DH / 64;               // rotary pairs per lane
        int f = range.f, first = range.first;
        for (int row = range.row; f < range.end && row < p.rows && ok; ++row) {
            const int len = d8_len(p, row, nullptr), w = d8_weight(p, len);
            if (len > 0) {
                const int nq = MULTI ? d8_queries(p, row % p.per_seq) : 1, cols = nq * G;
                const float2* cs = p.rope_table + (long long)(len - nq) * (DH / 2) + lane * E;      // of the first query
                int ia[E], ib[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    ia[e] = p.interleaved ? 2 * (lane * E + e) : lane * E + e;
                    ib[e] = p.interleaved ? ia[e] + 1 : ia[e] + DH / 2;
                }
                bf16 a[8][E], b[8][E];
                float2 c[MULTI ? 8 : 1][E];
#pragma unroll
                for (int h = 0; h < 8; ++h) {
                    const bf16* q = p.q + d8_out_row<MULTI>(p, row, kvh, h) * DH;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        a[h][e] = b[h][e] = __float2bfloat16_rn(0.f);
                        if (h < cols) {
                            a[h][e] = q[ia[e]];
                            b[h][e] = q[ib[e]];
                        }
                        if (MULTI) c[MULTI ? h : 0][e] = h < cols ? cs[(long long)(h / G) * (DH / 2) + e] : make_float2(0.f, 0.f);
                    }
                }
                if (!MULTI)
#pragma unroll
                    for (int e = 0; e < E; ++e) c[0][e] = cs[e];
                ok = __all_sync(0xffffffffu, mbar_wait(&sm.q_empty, par ^ 1));
                if (!ok) break;
#pragma unroll
                for (int h = 0; h < 8; ++h)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float x = __bfloat162float(a[h][e]), y = __bfloat162float(b[h][e]);
                        const float2 w = c[MULTI ? h : 0][e];
                        sm.qs[h][ia[e]] = x * w.x - y * w.y;
                        sm.qs[h][ib[e]] = x * w.y + y * w.x;
                    }
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.q_full);
                par ^= 1;
            }
            first += w;
            f = min(first, range.end);
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
    uint32_t q_par = 0;
    int f = range.f, first = range.first;
    for (int row = range.row; f < range.end && row < p.rows; ++row) {
        const int len = d8_len(p, row, tid == 0 ? p.status : nullptr), w = d8_weight(p, len);
        const int stop = min(first + w, range.end);
        const bool whole = f == first && stop == first + w;
        const int t_begin = (f - first) << p.unit, t_end = min(len, (stop - first) << p.unit);
        const int nq = MULTI ? d8_queries(p, row % p.per_seq) : 1, cols = nq * G;
        // (of a row of several queries, heads 2 t, 2 t + 1 of the first ones see fewer tokens)
        int seen[2] = {t_end, t_end}, seen_least = t_end;
        if (MULTI) {
            seen_least = min(t_end, len - (nq - 1));
#pragma unroll
            for (int e = 0; e < 2; ++e) seen[e] = min(t_end, len - max(nq - 1 - (2 * t + e) / G, 0));
        }

        if (len > 0) {
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&sm.q_full, q_par));
            q_par ^= 1;
        }
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
            // its power of two, between 2^-100 and 2^126 (the inverse is an ordinary number too; what is divided lies below 4)
            const uint32_t e = min(max(__float_as_uint(most) >> 23, 27u), 253u);
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
            __syncwarp();
            if (len > 0 && lane == 0) mbar_arrive(&sm.q_empty);
            const float base = rsqrtf((float)DH) * LOG2E;
            factor[0] = __shfl_sync(0xffffffffu, up, 8 * t) * base;
            factor[1] = __shfl_sync(0xffffffffu, up, 8 * t + 4) * base;
        }
        float o[KS][4];                          // dimensions 16 ks + 2 g (+ 1: [2], [3]), heads 2 t, 2 t + 1
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) o[ks][0] = o[ks][1] = o[ks][2] = o[ks][3] = 0.f;
        float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};   // heads 2 t, 2 t + 1 (l: this lane's tokens)
        float w_run[2] = {-INFINITY, -INFINITY}, m_to_w[2] = {0.f, 0.f};  // o is in units of 2^w; 2^(m - w)

        for (int t0 = t_begin; t0 < t_end && ok; t0 += D8_TILE) {
            const int tw = t0 + warp * 32;       // first token of this warp
            ok = __all_sync(0xffffffffu, mbar_wait(&sm.full[st], par));
            if (!ok) break;
            const float2 k_scale2 = *reinterpret_cast<const float2*>(&sm.scale[st][0][2 * warp]);
            const float2 v_scale2 = *reinterpret_cast<const float2*>(&sm.scale[st][1][2 * warp]);
            const float k_scale[2] = {k_scale2.x, k_scale2.y};
            float v_scale[2] = {v_scale2.x, v_scale2.y};
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
            if (tw + 32 > seen_least || dead) {  // tokens past the end, or in pages that do not exist
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bool gone = (dead >> (2 * warp + u)) & 1;
                    if (gone || t_end - tw - 16 * u <= 0) v_scale[u] = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (gone || g + (j >> 1) * 8 >= seen[j & 1] - tw - 16 * u) x[u][j] = -INFINITY;
                }
                if (E4M3) {
                    // such rows have the factor zero, but their bytes may be codes of NaN
                    for (int r = max(t_end - tw, 0); r < 32; ++r)
                        if (lane < DH / 8) *reinterpret_cast<uint2*>(sm.kv[st][1] + (warp * 32 + r) * DH + lane * 8) = make_uint2(0u, 0u);
                    fence_proxy_async_smem();    // before the stage's next copy
                    __syncwarp();
                }
            }
            // Running softmax over this warp's tokens.  The sum of p and the weighted values have references of their own (m, w): a
            // token's weight is p times its values' scale, so tokens with small values count in full also beside tokens of little
            // weight with far larger values.  A reference is raised when it is exceeded by more than 2^8 (2^15), which after the
            // first steps is rare, so the maximum over the warp is looked for only then.
            const float lv[2] = {d8_log2(v_scale[0]), d8_log2(v_scale[1])};
            float top[2], heavy[2];              // the largest score, and the largest weight (score + log2 of the scale), heads 2 t, 2 t + 1
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float a = fmaxf(x[0][e], x[0][2 + e]), b = fmaxf(x[1][e], x[1][2 + e]);
                top[e] = fmaxf(a, b);
                heavy[e] = fmaxf(a + lv[0], b + lv[1]);
            }
            if (__any_sync(0xffffffffu, top[0] > m_run[0] + D8_RAISE || top[1] > m_run[1] + D8_RAISE || heavy[0] > w_run[0] + D8_HEAD + D8_RAISE ||
                                            heavy[1] > w_run[1] + D8_HEAD + D8_RAISE)) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], d));
                        heavy[e] = fmaxf(heavy[e], __shfl_xor_sync(0xffffffffu, heavy[e], d));
                    }
                    if (top[e] > m_run[e] + D8_RAISE) {
                        l_run[e] *= m_run[e] == -INFINITY ? 0.f : ex2_approx(m_run[e] - top[e]);
                        m_run[e] = top[e];
                    }
                    // w is at least m - D8_BELOW, so that p 2^(m - w) <= 2^(D8_RAISE + D8_BELOW) stays a number of fp32, and at most
                    // m + D8_ABOVE, so that 2^(m - w) is not flushed to zero (a weight is 2^(D8_RAISE + 128 - D8_ABOVE) at most then)
                    float now = heavy[e] > w_run[e] + D8_HEAD + D8_RAISE ? heavy[e] - D8_HEAD : w_run[e];
                    if (m_run[e] != -INFINITY) now = fminf(fmaxf(now, m_run[e] - D8_BELOW), m_run[e] + D8_ABOVE);
                    const float alpha = w_run[e] == -INFINITY ? 0.f : ex2_approx(w_run[e] - now);
                    w_run[e] = now;
                    m_to_w[e] = m_run[e] == -INFINITY ? 0.f : ex2_approx(m_run[e] - now);
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        o[ks][e] *= alpha;
                        o[ks][2 + e] *= alpha;
                    }
                }
            }
            // p = 2^(x - m), and the weights (p 2^(m - w)) c as fp16, pairs of heads.  (In this order: c 2^(m - w) may exceed fp32 for tokens
            // without weight, whose p is zero.)
            const float m0 = m_run[0] == -INFINITY ? 0.f : m_run[0], m1 = m_run[1] == -INFINITY ? 0.f : m_run[1];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t ph[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float p0 = ex2_approx(x[u][2 * j] - m0), p1 = ex2_approx(x[u][2 * j + 1] - m1);
                    l_run[0] += p0;
                    l_run[1] += p1;
                    ph[j] = pack_half(p0 * m_to_w[0] * v_scale[u], p1 * m_to_w[1] * v_scale[u]);
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
                sm.w[warp][2 * t + e] = w_run[e];
            }
        }
        for (int h0 = 0; h0 < cols; h0 += 4) {
            if (2 * t >= h0 && 2 * t < h0 + 4)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        *reinterpret_cast<float2*>(&sm.o[warp][2 * t + e - h0][16 * ks + 2 * g]) = make_float2(o[ks][e], o[ks][2 + e]);
            __syncwarp();
            asm volatile("bar.sync 1, 128;" ::: "memory");
            const int h = h0 + tid / (DH / 4), d = tid % (DH / 4) * 4;          // a thread takes four dimensions of a head
            if (h < min(cols, h0 + 4)) {
                float M = -INFINITY;
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (sm.l[x][h] != 0.f) M = fmaxf(M, sm.m[x][h]);
                float L = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float wgt = sm.l[x][h] != 0.f ? ex2_approx(sm.m[x][h] - M) : 0.f;
                    const float c = sm.l[x][h] != 0.f ? ex2_approx(sm.w[x][h] - M) : 0.f;
                    const float4 y = *reinterpret_cast<const float4*>(&sm.o[x][h - h0][d]);
                    L += wgt * sm.l[x][h];
                    acc.x += c * y.x;
                    acc.y += c * y.y;
                    acc.z += c * y.z;
                    acc.w += c * y.w;
                }
                if (whole) {
                    d8_store(p, d8_out_row<MULTI>(p, row, kvh, h) * DH + d, acc, L);
                } else {
                    const long long unit = ((long long)kvh * (p.parts + p.rows) + part + row) * (MULTI ? p.cols : G) + h;
                    if (d == 0) *reinterpret_cast<float2*>(p.part_ml + unit * 2) = make_float2(M, L);
                    *reinterpret_cast<float4*>(p.part_o + unit * DH + d) = acc;
                }
            }
            // all have read before a warp writes here again: the other heads, or a short row that comes next
            asm volatile("bar.sync 1, 128;" ::: "memory");
        }
        if (!whole) {
            // The row's parts c0 .. c1 count themselves in (the counter of c0, since a part begins at most one row that it does not
            // end); the last one adds up all pieces, in their order, and leaves the counter at zero.
            const int c0 = range.base + first / range.per, c1 = range.base + (first + w - 1) / range.per, n = c1 - c0 + 1;
            __threadfence();
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (tid == 0) sm.last = atomicInc(p.count + kvh * p.parts + c0, n - 1) == (unsigned)(n - 1);
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (sm.last) {
                __threadfence();
                d8_merge<DH, MULTI>(p, ((long long)kvh * (p.parts + p.rows) + c0 + row) * (MULTI ? p.cols : G), n, row, kvh, cols, tid);
            }
        }
        first += w;
        f = stop;
    }
    if (!ok && lane == 0) lorc_set_status(p.status, LORC_ERR_TIMEOUT);
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

// How the rows of a call are dealt out.  Parts: the blocks of a KV head that are resident at once; 0: a block per row.  That spares the
// search for a block's part, and is taken for short sequences while there are no more of them than parts (16 x 100 tokens 5.0 us, as a
// list 6.1), and, with several queries per sequence, where the list would be long to search.  More short sequences are dealt out
// whole, so that a block fetches the next one while it works on one (a block per row / cut by 64 tokens / whole, us: 256 x 200 tokens
// 44 / 36.4 / 35.5, 512 x 100 66 / 50.7 / 49.9, 64 x 200 12.8 / 17.1 / 11.9).
void d8_plan(const lorc_ctx* ctx, int rows, int max_seq_len, int T, int* parts, int* least, int* unit) {
    const int slots = D8_BLOCKS_PER_SM * ctx->sm_count / ctx->desc.n_kv_heads;      // (lorc_part_counters goes by this)
    const bool few = max_seq_len <= 1 << D8_SHORT;
    *parts = slots > 1 ? slots : 1;
    *least = few ? 1 : 2;
    *unit = few ? D8_SHORT : D8_UNIT;
    if ((few && rows <= *parts) || (T > 1 && rows > D8_LIST && rows >= *parts)) *parts = 0;
}

size_t d8_ml_bytes(const lorc_ctx* ctx, long long slots) {
    return lorc_align_up((size_t)slots * ctx->desc.n_q_heads * 2 * sizeof(float), 256);
}

template <int DH, bool E4M3, bool MULTI>
cudaError_t d8_launch(lorc_ctx* ctx, const CUtensorMap& mapK, const CUtensorMap& mapV, const D8Params& p, cudaStream_t st) {
    const size_t smem = sizeof(D8Smem<DH>) + 1024;
    // the attribute belongs to a device's copy of the kernel: one flag per device
    static bool attr[64] = {false};
    const bool known = ctx->device >= 0 && ctx->device < 64;
    if (!known || !attr[ctx->device]) {
        cudaError_t e = cudaFuncSetAttribute(decode8_mma_kernel<DH, E4M3, MULTI>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (known) attr[ctx->device] = true;
    }
    const long long blocks = (long long)p.n_kv * (p.parts ? p.parts : p.rows);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    return lorc_launch_dependent(decode8_mma_kernel<DH, E4M3, MULTI>, dim3((unsigned)blocks), dim3(D8_THREADS), smem, st, mapK, mapV, p);
}

template <int DH, bool E4M3>
cudaError_t d8_launch(lorc_ctx* ctx, const CUtensorMap& mapK, const CUtensorMap& mapV, const D8Params& p, cudaStream_t st) {
    return p.Q > 1 ? d8_launch<DH, E4M3, true>(ctx, mapK, mapV, p, st) : d8_launch<DH, E4M3, false>(ctx, mapK, mapV, p, st);
}

}  // namespace

int lorc_decode8_queries(const lorc_ctx* ctx, int T) { return T < 8 / ctx->group ? T : 8 / ctx->group; }

bool lorc_decode8_fits(const lorc_ctx* ctx, const Cache8View& cv, int T) {
    const int Q = lorc_decode8_queries(ctx, T);
    const long long rows = (long long)cv.batch * ((T + Q - 1) / Q);
    int parts, least, unit;
    d8_plan(ctx, (int)rows, cv.max_seq_len, T, &parts, &least, &unit);
    if (parts == 0) return rows * ctx->desc.n_kv_heads <= 0x7fffffffll;            // a block per row and KV head
    return rows * (((cv.max_seq_len - 1) >> unit) + 1) < 1ll << 30;
}

size_t lorc_decode8_scratch_bytes(const lorc_ctx* ctx, int batch, int max_seq_len, int T) {
    // a call may have fewer queries or shorter sequences than stated here: room for the list in any case (one query: all sequences
    // are on it; several: at most D8_LIST rows or as many as parts, of Q queries each)
    int parts, least, unit;
    d8_plan(ctx, 1, (1 << D8_SHORT) + 1, 1, &parts, &least, &unit);
    const long long Q = lorc_decode8_queries(ctx, T), one = (long long)parts + batch;
    const long long several = T > 1 ? (parts + (parts > D8_LIST ? parts : (long long)D8_LIST)) * Q : 0;
    const long long slots = one > several ? one : several;
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
    p.count = ctx->part_count;
    p.G = ctx->group; p.n_kv = d.n_kv_heads; p.T = T; p.interleaved = ctx->pair_style == LORC_ROPE_INTERLEAVED;
    p.max_pos = d.max_pos; p.box_rows = box_rows;
    p.Q = lorc_decode8_queries(ctx, T);
    p.per_seq = (T + p.Q - 1) / p.Q;
    p.cols = p.Q * p.G;
    p.rows = cv.batch * p.per_seq;
    const unsigned per = cv.page_table ? cv.page_size / LORC_BLOCK8 : 1;
    p.page_magic = per > 1 ? (unsigned)(((1ull << 32) + per - 1) / per) : 0;
    d8_plan(ctx, p.rows, cv.max_seq_len, T, &p.parts, &p.least, &p.unit);
    p.each = p.rows <= 128 ? p.parts / p.rows : 0;
    p.part_ml = (float*)scratch;
    p.part_o = (float*)((char*)scratch + d8_ml_bytes(ctx, (long long)(p.parts + p.rows) * p.Q));
    const bool e4m3 = cv.type == LORC_CACHE8_E4M3;
    LorcStageTimer timer(ctx, LORC_STAGE_SCORE, st);
    *launches += 1;
    return d.d_head == 128 ? (e4m3 ? d8_launch<128, true>(ctx, mapK, mapV, p, st) : d8_launch<128, false>(ctx, mapK, mapV, p, st))
                           : (e4m3 ? d8_launch<64, true>(ctx, mapK, mapV, p, st) : d8_launch<64, false>(ctx, mapK, mapV, p, st));
}
