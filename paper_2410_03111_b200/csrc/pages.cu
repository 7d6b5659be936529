// Pages of a pool that sequences share: fork, grow, free, compact, all on the device.
//
// A call plans with one block (who needs pages, which are the lowest free ones: prefix sums over the list and over the reference
// counts), and a second kernel with the whole GPU moves the pages' contents in every array and rewrites table entries.  The moves
// are plain copies, bound by HBM: a warp takes 4 KB of one page of one array at a time, eight 16-byte loads per lane in flight.
// (468 MB, half of the pages of a pool of eight layers: 80 us with its plan, 0.89 of the measured copy rate.)  What is left of a small
// call is its chain of launches and round trips.
#include "common.cuh"
#include "sm100_ptx.cuh"

using namespace sm100;

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int BUFS = 128;               // arrays per launch of the copying kernels (the descriptors are kernel arguments)
constexpr int UNIT = 4096;              // bytes of a warp's piece of work
constexpr int SMALL = 256;              // pairs of a fork whose plan stays in shared memory

struct PagesView {
    int n_pages, page_size, per_row, n_rows;
    int32_t *table, *lens, *refs;
};

// Arrays of one launch; first[i]: pieces of a page that lie in the arrays before i.
struct Bufs {
    char* base[BUFS];
    long long bytes[BUFS];
    int first[BUFS + 1];
    int n;
    unsigned wide[BUFS / 32];           // arrays whose pages are 16-byte aligned
};

struct Copy {
    int src, dst;
};

// Pages that a row of `len` tokens holds; a length beyond the table counts as 0 (callers report it).
__device__ __forceinline__ bool row_fits(const PagesView& p, long long len) { return len <= (long long)p.per_row * p.page_size; }
__device__ __forceinline__ int held_pages(const PagesView& p, int len) {
    return len <= 0 || !row_fits(p, len) ? 0 : (len - 1) / p.page_size + 1;
}

// Sums over the block in thread order: the sum of the threads before this one; `all` receives the sum of all.  (All threads.)
template <typename T>
__device__ __forceinline__ T block_scan(T x, T* sums, T& all) {
    static_assert(PLAN_THREADS == 1024, "a warp's lanes are the block's warps");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T incl = warp_scan(x, lane);
    __syncthreads();
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    const T mine = sums[lane], upto = warp_scan(mine, lane);
    all = __shfl_sync(0xffffffffu, upto, 31);
    return __shfl_sync(0xffffffffu, upto - mine, warp) + incl - x;
}

// This thread's four of the 4096 counts from page p0 on: which of them are free.
__device__ __forceinline__ unsigned free_of(const PagesView& p, int p0) {
    const int at = p0 + 4 * (int)threadIdx.x;
    unsigned mask = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < p.n_pages && p.refs[at + i] <= 0) mask |= 1u << i;
    return mask;
}

// Writes the `want` lowest free pages (at most) in ascending order; returns how many there are of them.  `first`: free_of the first
// 4096 pages, which the caller has asked for before it knew `want`.  (All threads.)
__device__ int lowest_free(const PagesView& p, long long want, unsigned first, int32_t* list, int* sums) {
    int found = 0;
    for (int p0 = 0; p0 < p.n_pages && found < want; p0 += 4 * PLAN_THREADS) {
        const unsigned free = p0 == 0 ? first : free_of(p, p0);
        int all, rank = found + block_scan(__popc(free), sums, all);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (free >> i & 1) {
                if (rank < want) list[rank] = p0 + 4 * (int)threadIdx.x + i;
                ++rank;
            }
        found += all;
    }
    __syncthreads();
    return found < want ? found : (int)want;
}

__global__ void __launch_bounds__(256)
pages_free_kernel(const PagesView p, const int32_t* __restrict__ rows, int* status) {
    __shared__ int row_s, len_s;
    grid_dep_wait();
    grid_dep_launch();
    if (threadIdx.x == 0) {
        const int row = rows[blockIdx.x];
        int len = 0;
        if (row < 0 || row >= p.n_rows) lorc_set_status(status, LORC_ERR_ARG);
        else len = atomicExch(p.lens + row, 0);          // whoever sees the length gives the pages back
        if (!row_fits(p, len)) lorc_set_status(status, LORC_ERR_CAPACITY);
        row_s = row;
        len_s = len;
    }
    __syncthreads();
    const int held = held_pages(p, len_s);
    for (int i = threadIdx.x; i < held; i += 256) {
        const int page = p.table[(long long)row_s * p.per_row + i];
        if (page < 0 || page >= p.n_pages) lorc_set_status(status, LORC_ERR_CAPACITY);
        else atomicSub(p.refs + page, 1);
    }
}

// One pair of a fork: len < 0 leaves it out; page >= 0: the child's own last page.
struct ForkPair {
    int parent, child, len, page;
};

__global__ void __launch_bounds__(PLAN_THREADS)
pages_fork_plan_kernel(const PagesView p, const int32_t* __restrict__ parents, const int32_t* __restrict__ children, int n,
                       ForkPair* __restrict__ plan, int32_t* __restrict__ list, int* status) {
    __shared__ int sums[PLAN_THREADS / 32];
    const int tid = threadIdx.x;
    grid_dep_wait();
    grid_dep_launch();
    // lengths as they are when the call begins
    for (int i = tid; i < n; i += PLAN_THREADS) {
        ForkPair f = {parents[i], children[i], -1, -1};
        if (f.parent < 0 || f.parent >= p.n_rows || f.child < 0 || f.child >= p.n_rows || p.lens[f.child] > 0) {
            lorc_set_status(status, LORC_ERR_ARG);
        } else {
            f.len = max(p.lens[f.parent], 0);
            if (!row_fits(p, f.len)) {
                lorc_set_status(status, LORC_ERR_CAPACITY);
                f.len = -1;
            }
        }
        plan[i] = f;
    }
    __syncthreads();
    // A child belongs to the first pair that lists it: the lowest of the numbers i - n, which are all below zero, stays in its
    // length until the end.
    for (int i = tid; i < n; i += PLAN_THREADS)
        if (plan[i].len >= 0) p.lens[plan[i].child] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += PLAN_THREADS)
        if (plan[i].len >= 0) atomicMin(p.lens + plan[i].child, i - n);
    __syncthreads();
    for (int i = tid; i < n; i += PLAN_THREADS)
        if (plan[i].len >= 0 && *(volatile int32_t*)(p.lens + plan[i].child) != i - n) {
            lorc_set_status(status, LORC_ERR_ARG);
            plan[i].len = -1;
        }
    // who needs a page, and which one
    int want = 0;
    for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        const bool need = i < n && plan[i].len > 0 && plan[i].len % p.page_size != 0;
        int all;
        const int rank = want + block_scan((int)need, sums, all);
        if (need) plan[i].page = rank;
        want += all;
    }
    const int found = lowest_free(p, want, free_of(p, 0), list, sums);
    for (int i = tid; i < n; i += PLAN_THREADS) {
        ForkPair f = plan[i];
        if (f.len < 0) continue;
        if (f.page >= 0) {
            const int rank = f.page;
            f.page = rank < found ? list[rank] : -1;
            if (f.page < 0) {
                lorc_set_status(status, LORC_ERR_CAPACITY);
                f.len = -1;
            } else {
                p.refs[f.page] = 1;
            }
            plan[i] = f;
        }
        p.lens[f.child] = f.len > 0 ? f.len : 0;
    }
}

// A warp copies bytes [begin, begin + UNIT) of page `src` of array b to page `dst`.
__device__ __forceinline__ void copy_unit(const Bufs& bufs, int b, long long begin, int src, int dst, int lane) {
    const long long bytes = bufs.bytes[b];
    const char* from = bufs.base[b] + src * bytes + begin;
    char* to = bufs.base[b] + dst * bytes + begin;
    const int left = (int)(bytes - begin < UNIT ? bytes - begin : UNIT);
    if (bufs.wide[b >> 5] >> (b & 31) & 1) {
        // (what is copied is not read again soon)
        uint4 x[UNIT / 512];
#pragma unroll
        for (int i = 0; i < UNIT / 512; ++i)
            if ((i * 32 + lane) * 16 < left) x[i] = __ldcs(reinterpret_cast<const uint4*>(from) + i * 32 + lane);
#pragma unroll
        for (int i = 0; i < UNIT / 512; ++i)
            if ((i * 32 + lane) * 16 < left) __stcs(reinterpret_cast<uint4*>(to) + i * 32 + lane, x[i]);
    } else {
        for (int i = lane * 4; i < left; i += 128) *reinterpret_cast<uint32_t*>(to + i) = *reinterpret_cast<const uint32_t*>(from + i);
    }
}

// Array and first byte of piece u of a page.
__device__ __forceinline__ int find_buf(const Bufs& bufs, int u, long long& begin) {
    int lo = 0, hi = bufs.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (bufs.first[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    begin = (long long)(u - bufs.first[lo]) * UNIT;
    return lo;
}

// Pieces me, me + warps, me + 2 warps, ... of a list of pages with `units` pieces each: page i, piece u.
struct Pieces {
    long long i, di;
    int u, du, units;
    __device__ Pieces(long long me, long long warps, int units) : units(units) {
        i = units ? me / units : 0;
        u = units ? (int)(me - i * units) : 0;
        di = units ? warps / units : 0;
        du = units ? (int)(warps - di * units) : 0;
    }
    __device__ void next() {
        i += di;
        u += du;
        if (u >= units) {
            u -= units;
            ++i;
        }
    }
};

// The rows of the children, and the pages of their own: by `warps` warps, of which this is number `me`.
__device__ __forceinline__ void fork_apply(const Bufs& bufs, const PagesView& p, const ForkPair* plan, int n, bool rows_too, long long me,
                                           long long warps, int lane, int* status) {
    if (rows_too)
        for (long long i = me; i < n; i += warps) {
            const ForkPair f = plan[i];
            if (f.len <= 0) continue;
            const int held = held_pages(p, f.len), shared = f.page >= 0 ? held - 1 : held;
            const int32_t* from = p.table + (long long)f.parent * p.per_row;
            int32_t* to = p.table + (long long)f.child * p.per_row;
            for (int j = lane; j < held; j += 32) {
                const int page = j < shared ? from[j] : f.page;
                to[j] = page;
                if (page < 0 || page >= p.n_pages) lorc_set_status(status, LORC_ERR_CAPACITY);
                else if (j < shared) atomicAdd(p.refs + page, 1);
            }
        }
    if (bufs.first[bufs.n] == 0) return;
    for (Pieces w(me, warps, bufs.first[bufs.n]); w.i < n; w.next()) {
        const ForkPair f = plan[w.i];
        if (f.len <= 0 || f.page < 0) continue;
        const int src = p.table[(long long)f.parent * p.per_row + f.len / p.page_size];
        if (src < 0 || src >= p.n_pages) {
            if (lane == 0) lorc_set_status(status, LORC_ERR_CAPACITY);
            continue;
        }
        long long begin;
        const int b = find_buf(bufs, w.u, begin);
        copy_unit(bufs, b, begin, src, f.page, lane);
    }
}

// The same for at most SMALL pairs: a thread per pair, and the plan stays in shared memory until it is written out.  apply: there is
// so little to do that this block does it all.
__global__ void __launch_bounds__(PLAN_THREADS)
pages_fork_small_kernel(const __grid_constant__ Bufs bufs, const PagesView p, const int32_t* __restrict__ parents,
                        const int32_t* __restrict__ children, int n, ForkPair* __restrict__ plan, int apply, int* status) {
    __shared__ int sums[PLAN_THREADS / 32];
    __shared__ ForkPair pairs[SMALL];
    __shared__ alignas(16) int32_t child_s[SMALL];
    __shared__ int32_t list[SMALL];
    const int tid = threadIdx.x;
    grid_dep_wait();
    grid_dep_launch();
    const unsigned free = free_of(p, 0);
    ForkPair f = {-1, -1, -1, -1};
    if (tid < n) {
        f.parent = parents[tid];
        f.child = children[tid];
        if (f.parent < 0 || f.parent >= p.n_rows || f.child < 0 || f.child >= p.n_rows) {
            lorc_set_status(status, LORC_ERR_ARG);
        } else {
            const int theirs = p.lens[f.child], len = max(p.lens[f.parent], 0);
            if (theirs > 0) lorc_set_status(status, LORC_ERR_ARG);
            else if (!row_fits(p, len)) lorc_set_status(status, LORC_ERR_CAPACITY);
            else f.len = len;
        }
    }
    if (tid < SMALL) child_s[tid] = f.len >= 0 ? f.child : -1;
    __syncthreads();
    if (f.len >= 0) {
        bool again = false;                      // an earlier pair has the same child
        for (int j = 0; j < tid; j += 4) {
            const int4 c = *reinterpret_cast<const int4*>(child_s + j);
            again |= c.x == f.child || (c.y == f.child && j + 1 < tid) || (c.z == f.child && j + 2 < tid) || (c.w == f.child && j + 3 < tid);
        }
        if (again) {
            lorc_set_status(status, LORC_ERR_ARG);
            f.len = -1;
        }
    }
    const bool need = f.len > 0 && f.len % p.page_size != 0;
    int want;
    const int rank = block_scan((int)need, sums, want);
    const int found = lowest_free(p, want, free, list, sums);
    if (f.len >= 0) {
        if (need) {
            if (rank < found) {
                f.page = list[rank];
                p.refs[f.page] = 1;
            } else {
                lorc_set_status(status, LORC_ERR_CAPACITY);
                f.len = 0;
            }
        }
        p.lens[f.child] = f.len;
    }
    if (tid < n) {
        if (apply) pairs[tid] = f;
        else plan[tid] = f;
    }
    if (!apply) return;
    __syncthreads();
    fork_apply(bufs, p, pairs, n, true, tid >> 5, PLAN_THREADS / 32, tid & 31, status);
}

__global__ void __launch_bounds__(256)
pages_fork_kernel(const __grid_constant__ Bufs bufs, const PagesView p, const ForkPair* __restrict__ plan, int n, int rows_too,
                  int* status) {
    grid_dep_wait();
    grid_dep_launch();
    fork_apply(bufs, p, plan, n, rows_too != 0, (long long)blockIdx.x * 8 + (threadIdx.x >> 5), (long long)gridDim.x * 8,
               threadIdx.x & 31, status);
}

__global__ void __launch_bounds__(PLAN_THREADS)
pages_grow_kernel(const PagesView p, const int32_t* __restrict__ grow, long long* __restrict__ start, int32_t* __restrict__ list,
                  int* status) {
    __shared__ long long sums[PLAN_THREADS / 32];
    __shared__ int counts[PLAN_THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31;
    grid_dep_wait();
    grid_dep_launch();
    const unsigned free = free_of(p, 0);
    // start[s]: the rank of the row's first new page, -1 for a row that stays as it is
    long long want = 0;
    for (int s0 = 0; s0 < p.n_rows; s0 += PLAN_THREADS) {
        const int s = s0 + tid;
        int more = 0;
        bool live = false;
        if (s < p.n_rows && grow[s] > 0) {
            const long long len = max(p.lens[s], 0), now = len + grow[s];
            live = row_fits(p, now) && now <= 0x7fffffffll;
            if (live) more = held_pages(p, (int)now) - held_pages(p, (int)len);
            else lorc_set_status(status, LORC_ERR_CAPACITY);
        }
        long long all;
        const long long rank = want + block_scan((long long)more, sums, all);
        if (s < p.n_rows) start[s] = live ? rank : -1;
        want += all;
    }
    const int found = lowest_free(p, want, free, list, counts);
    for (int s = tid >> 5; s < p.n_rows; s += PLAN_THREADS / 32) {
        const long long first = start[s];
        if (first < 0) continue;
        const int len = max(p.lens[s], 0), now = len + grow[s], old = held_pages(p, len), held = held_pages(p, now);
        if (held > old && first + held - old > found) {
            if (lane == 0) lorc_set_status(status, LORC_ERR_CAPACITY);
            continue;
        }
        for (int j = old + lane; j < held; j += 32) {
            const int page = list[first + j - old];
            p.table[(long long)s * p.per_row + j] = page;
            p.refs[page] = 1;
        }
        __syncwarp();
        if (lane == 0) p.lens[s] = now;
    }
}

// moves[i]: a used page at or above the number of used pages, and the free page below it that takes its contents; count[i]: its
// references; to[p]: where page p goes, for p >= *used (-1: it is free).
__global__ void __launch_bounds__(PLAN_THREADS)
pages_compact_plan_kernel(const PagesView p, Copy* __restrict__ moves, int32_t* __restrict__ count, int32_t* __restrict__ to,
                          int32_t* __restrict__ head, int32_t* __restrict__ n_used) {
    __shared__ long long sums[PLAN_THREADS / 32];
    const int tid = threadIdx.x;
    grid_dep_wait();
    grid_dep_launch();
    long long mine = 0, all;
    for (int i = tid; i < p.n_pages; i += PLAN_THREADS) mine += p.refs[i] > 0;
    block_scan(mine, sums, all);
    const int used = (int)all;
    int n_src = 0, n_dst = 0;
    for (int p0 = 0; p0 < p.n_pages; p0 += 4 * PLAN_THREADS) {
        const int at = p0 + 4 * tid;
        int ref[4], src = 0, dst = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ref[i] = at + i < p.n_pages ? p.refs[at + i] : 0;
            if (at + i < used) dst += ref[i] <= 0;
            else src += ref[i] > 0;
        }
        // (both counts in one sum; a block looks at 4096 pages at a time)
        const long long scan = block_scan((long long)src << 32 | dst, sums, all);
        int rs = n_src + (int)(scan >> 32), rd = n_dst + (int)(scan & 0xffffffff);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int page = at + i;
            if (page >= p.n_pages) break;
            if (page < used) {
                if (ref[i] <= 0) moves[rd++].dst = page;
            } else if (ref[i] > 0) {
                moves[rs].src = page;
                count[rs++] = ref[i];
            } else {
                to[page] = -1;
            }
        }
        n_src += (int)(all >> 32);
        n_dst += (int)(all & 0xffffffff);
    }
    __syncthreads();
    for (int i = tid; i < n_src; i += PLAN_THREADS) to[moves[i].src] = moves[i].dst;
    if (tid == 0) {
        head[0] = used;
        head[1] = n_src;
        if (n_used) *n_used = used;
    }
}

__global__ void __launch_bounds__(256)
pages_compact_kernel(const __grid_constant__ Bufs bufs, const PagesView p, const Copy* __restrict__ moves,
                     const int32_t* __restrict__ count, const int32_t* __restrict__ to, const int32_t* __restrict__ head,
                     int32_t* table_out, int32_t* refs_out, int rows_too, int* status) {
    const int lane = threadIdx.x & 31;
    const long long warps = (long long)gridDim.x * 8, me = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    grid_dep_wait();
    grid_dep_launch();
    const int used = head[0], n = head[1];
    if (rows_too) {
        const long long threads = warps * 32, t0 = me * 32 + lane;
        for (long long i = t0; i < p.n_pages; i += threads) {
            // (free pages below `used` are written with the move that fills them)
            if (i >= used) refs_out[i] = 0;
            else if (p.refs[i] > 0 && p.refs != refs_out) refs_out[i] = p.refs[i];
        }
        for (long long i = t0; i < n; i += threads) refs_out[moves[i].dst] = count[i];
        for (long long s = me; s < p.n_rows; s += warps) {
            const int len = p.lens[s], held = held_pages(p, len);
            if (!row_fits(p, len) && lane == 0) lorc_set_status(status, LORC_ERR_CAPACITY);
            for (int j = lane; j < p.per_row; j += 32) {
                const long long at = s * p.per_row + j;
                int page = p.table[at];
                if (j < held) {
                    if (page < 0 || page >= p.n_pages) {
                        lorc_set_status(status, LORC_ERR_CAPACITY);
                    } else if (page >= used) {
                        // a row that holds a page without a reference: the counts are wrong
                        if (to[page] < 0) lorc_set_status(status, LORC_ERR_ARG);
                        else page = to[page];
                    }
                }
                table_out[at] = page;
            }
        }
    }
    if (bufs.first[bufs.n] == 0) return;
    for (Pieces w(me, warps, bufs.first[bufs.n]); w.i < n; w.next()) {
        const Copy m = moves[w.i];
        long long begin;
        const int b = find_buf(bufs, w.u, begin);
        copy_unit(bufs, b, begin, m.src, m.dst, lane);
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------
int fail_p(lorc_ctx* ctx, int code, const char* msg) {
    ctx->err = msg;
    return code;
}

int fail_p_cuda(lorc_ctx* ctx, cudaError_t e, const char* where) {
    ctx->err = std::string(where) + ": " + cudaGetErrorString(e);
    return LORC_ERR_CUDA;
}

bool sizes_ok(const lorc_pages* p) {
    return p && p->n_pages > 0 && p->page_size > 0 && p->max_pages_per_seq > 0 && p->n_rows > 0 && p->n_bufs >= 0 &&
           p->n_bufs <= LORC_PAGES_MAX_BUFS && p->n_pages <= (1 << 30) && p->n_rows <= (1 << 30);
}

struct Layout {
    size_t plan, list, more, total;     // fork: pairs | list; grow: list | starts; compact: moves, counts, targets, head
};

Layout layout(const lorc_pages* p, int n) {
    Layout l;
    const size_t pages = (size_t)p->n_pages, longest = pages > (size_t)n ? pages : (size_t)n;
    l.plan = 0;
    l.list = lorc_align_up((size_t)n * sizeof(ForkPair) > pages * sizeof(Copy) ? (size_t)n * sizeof(ForkPair) : pages * sizeof(Copy), 256);
    l.more = l.list + lorc_align_up(longest * sizeof(int32_t), 256);
    const size_t starts = (size_t)p->n_rows * sizeof(long long), targets = (pages + 2) * sizeof(int32_t);
    l.total = l.more + lorc_align_up(starts > targets ? starts : targets, 256);
    return l;
}

int check_pages(lorc_ctx* ctx, const lorc_pages* p, int n, PagesView* v, bool bufs) {
    if (!sizes_ok(p) || !p->page_table || !p->seq_lens || !p->refs) return fail_p(ctx, LORC_ERR_ARG, "pages: null pointer or size out of range");
    if (((uintptr_t)p->page_table & 3) || ((uintptr_t)p->seq_lens & 3) || ((uintptr_t)p->refs & 3))
        return fail_p(ctx, LORC_ERR_ARG, "pages: page table, lengths and counts must be 4-byte aligned");
    if (n < 0 || n > LORC_PAGES_MAX_LIST) return fail_p(ctx, LORC_ERR_ARG, "pages: the list is longer than LORC_PAGES_MAX_LIST");
    if (bufs) {
        if (p->n_bufs > 0 && !p->bufs) return fail_p(ctx, LORC_ERR_ARG, "pages: bufs is null");
        for (int i = 0; i < p->n_bufs; ++i)
            if (!p->bufs[i].base || ((uintptr_t)p->bufs[i].base & 3) || p->bufs[i].page_bytes <= 0 || p->bufs[i].page_bytes % 4 ||
                p->bufs[i].page_bytes > (1ll << 32))
                return fail_p(ctx, LORC_ERR_ARG, "pages: arrays must be 4-byte aligned, and their pages a positive multiple of 4 bytes");
    }
    if (!ctx->ws || layout(p, n).total > ctx->ws_bytes)
        return fail_p(ctx, LORC_ERR_WORKSPACE, "pages: workspace missing or too small (see lorc_pages_workspace_bytes)");
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail_p_cuda(ctx, e, "pages");
    if (dev != ctx->device) return fail_p(ctx, LORC_ERR_ARG, "pages: the context's device is not the current one");
    v->n_pages = p->n_pages;
    v->page_size = p->page_size;
    v->per_row = p->max_pages_per_seq;
    v->n_rows = p->n_rows;
    v->table = p->page_table;
    v->lens = p->seq_lens;
    v->refs = p->refs;
    return LORC_OK;
}

// Arrays [from, from + BUFS) of the pool as one launch's argument.
void take_bufs(const lorc_pages* p, int from, Bufs* b) {
    b->n = 0;
    b->first[0] = 0;
    for (int i = 0; i < BUFS / 32; ++i) b->wide[i] = 0;
    for (int i = from; i < p->n_bufs && b->n < BUFS; ++i, ++b->n) {
        const lorc_page_buf& x = p->bufs[i];
        b->base[b->n] = (char*)x.base;
        b->bytes[b->n] = x.page_bytes;
        b->first[b->n + 1] = b->first[b->n] + (int)((x.page_bytes + UNIT - 1) / UNIT);
        if (((uintptr_t)x.base & 15) == 0 && x.page_bytes % 16 == 0) b->wide[b->n >> 5] |= 1u << (b->n & 31);
    }
}

// Blocks of a copying kernel: enough warps for `most` pages, at most what the GPU holds at once.
unsigned copy_blocks(const lorc_ctx* ctx, const Bufs& b, long long most, long long least_warps) {
    long long warps = most * b.first[b.n];
    if (warps < least_warps) warps = least_warps;
    long long blocks = (warps + 7) / 8;
    const long long cap = 4ll * ctx->sm_count;
    if (blocks > cap) blocks = cap;
    return blocks < 1 ? 1u : (unsigned)blocks;
}

}  // namespace

extern "C" {

size_t lorc_pages_workspace_bytes(const lorc_pages* pages, int n) {
    if (!sizes_ok(pages) || n < 0 || n > LORC_PAGES_MAX_LIST) return 0;
    return layout(pages, n).total;
}

int lorc_pages_free(lorc_ctx* ctx, const lorc_pages* pages, const int32_t* rows, int n, void* stream) {
    if (!ctx) return LORC_ERR_ARG;
    PagesView v;
    const int rc = check_pages(ctx, pages, n, &v, false);
    if (rc) return rc;
    if (n == 0) return LORC_OK;
    if (!rows) return fail_p(ctx, LORC_ERR_ARG, "pages_free: null list");
    const cudaError_t e = lorc_launch_dependent(pages_free_kernel, dim3(n), dim3(256), 0, (cudaStream_t)stream, v, rows, ctx->status_dev);
    ctx->launches += 1;
    return e == cudaSuccess ? LORC_OK : fail_p_cuda(ctx, e, "lorc_pages_free");
}

int lorc_pages_fork(lorc_ctx* ctx, const lorc_pages* pages, const int32_t* parents, const int32_t* children, int n, void* stream) {
    if (!ctx) return LORC_ERR_ARG;
    PagesView v;
    const int rc = check_pages(ctx, pages, n, &v, true);
    if (rc) return rc;
    if (n == 0) return LORC_OK;
    if (!parents || !children) return fail_p(ctx, LORC_ERR_ARG, "pages_fork: null list");
    const Layout l = layout(pages, n);
    ForkPair* plan = (ForkPair*)((char*)ctx->ws + l.plan);
    int32_t* list = (int32_t*)((char*)ctx->ws + l.list);
    cudaStream_t st = (cudaStream_t)stream;
    Bufs b;
    take_bufs(pages, 0, &b);
    cudaError_t e;
    // One block copies some 250 KB and 16384 table entries in the time that another launch takes.
    const bool all = n <= SMALL && pages->n_bufs <= BUFS && (long long)n * b.first[b.n] <= PLAN_THREADS / 32 && (long long)n * v.per_row <= 16384;
    if (n <= SMALL)
        e = lorc_launch_dependent(pages_fork_small_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, b, v, parents, children, n, plan, (int)all,
                                  ctx->status_dev);
    else
        e = lorc_launch_dependent(pages_fork_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, v, parents, children, n, plan, list,
                                  ctx->status_dev);
    ctx->launches += 1;
    for (int from = 0; !all && e == cudaSuccess && (from == 0 || from < pages->n_bufs); from += BUFS) {
        if (from > 0) take_bufs(pages, from, &b);
        e = lorc_launch_dependent(pages_fork_kernel, dim3(copy_blocks(ctx, b, n, n)), dim3(256), 0, st, b, v, (const ForkPair*)plan, n,
                                  (int)(from == 0), ctx->status_dev);
        ctx->launches += 1;
    }
    return e == cudaSuccess ? LORC_OK : fail_p_cuda(ctx, e, "lorc_pages_fork");
}

int lorc_pages_grow(lorc_ctx* ctx, const lorc_pages* pages, const int32_t* grow, void* stream) {
    if (!ctx) return LORC_ERR_ARG;
    PagesView v;
    const int rc = check_pages(ctx, pages, 0, &v, false);
    if (rc) return rc;
    if (!grow) return fail_p(ctx, LORC_ERR_ARG, "pages_grow: null list");
    const Layout l = layout(pages, 0);
    const cudaError_t e = lorc_launch_dependent(pages_grow_kernel, dim3(1), dim3(PLAN_THREADS), 0, (cudaStream_t)stream, v, grow,
                                                (long long*)((char*)ctx->ws + l.more), (int32_t*)((char*)ctx->ws + l.list), ctx->status_dev);
    ctx->launches += 1;
    return e == cudaSuccess ? LORC_OK : fail_p_cuda(ctx, e, "lorc_pages_grow");
}

int lorc_pages_compact(lorc_ctx* ctx, const lorc_pages* pages, int32_t* page_table_out, int32_t* refs_out, int32_t* n_used,
                       void* stream) {
    if (!ctx) return LORC_ERR_ARG;
    PagesView v;
    const int rc = check_pages(ctx, pages, 0, &v, true);
    if (rc) return rc;
    if (((uintptr_t)page_table_out & 3) || ((uintptr_t)refs_out & 3) || ((uintptr_t)n_used & 3))
        return fail_p(ctx, LORC_ERR_ARG, "pages_compact: outputs must be 4-byte aligned");
    const Layout l = layout(pages, 0);
    Copy* moves = (Copy*)((char*)ctx->ws + l.plan);
    int32_t* count = (int32_t*)((char*)ctx->ws + l.list);
    int32_t* head = (int32_t*)((char*)ctx->ws + l.more);
    int32_t* to = head + 2;
    if (!page_table_out) page_table_out = v.table;
    if (!refs_out) refs_out = v.refs;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = lorc_launch_dependent(pages_compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, v, moves, count, to, head, n_used);
    ctx->launches += 1;
    Bufs b;
    for (int from = 0; e == cudaSuccess && (from == 0 || from < pages->n_bufs); from += BUFS) {
        take_bufs(pages, from, &b);
        // at most half of the pages move
        e = lorc_launch_dependent(pages_compact_kernel, dim3(copy_blocks(ctx, b, v.n_pages / 2, v.n_rows)), dim3(256), 0, st, b, v,
                                  (const Copy*)moves, (const int32_t*)count, (const int32_t*)to, (const int32_t*)head, page_table_out,
                                  refs_out, (int)(from == 0), ctx->status_dev);
        ctx->launches += 1;
    }
    return e == cudaSuccess ? LORC_OK : fail_p_cuda(ctx, e, "lorc_pages_compact");
}

}  // extern "C"
