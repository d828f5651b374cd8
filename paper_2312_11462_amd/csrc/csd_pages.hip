// The pages of a paged cache: page tables, row starts and slots of a step's new rows, from the sequences' lengths; pages of rows that are not kept given back;
// pages of a common prompt shared.
//
// Every call is bound by its trips to memory, a few bytes each.  One workgroup takes the sequences 1024 at a time, a thread each, with running sums over
// them; pages are dealt to all threads by a search in those sums.  The rows' positions and slots are written by the same workgroup where there are
// few, else by a second launch.
#include "csd_internal.h"

static constexpr int kThreads = 1024, kWaves = kThreads / 64;
static constexpr int kRowsHere = 4096;                       // rows that the planning workgroup writes itself

typedef unsigned long long u64;

struct PagesShared {
    u64 part[kWaves];
    int32_t run[kThreads];        // pages up to and with a sequence of the 1024
    int32_t from[kThreads];       // its first one, as an entry of its table
};

// inclusive running sum over the workgroup; `total`: of all
__device__ __forceinline__ u64 group_scan(u64 v, u64 *part, u64 &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const u64 x = __shfl_up(v, o, 64);
        if (lane >= o) v += x;
    }
    __syncthreads();
    if (lane == 63) part[wave] = v;
    __syncthreads();
    total = 0;
    u64 before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
        if (w < wave) before += part[w];
        total += part[w];
    }
    return v + before;
}

// the first of n ascending numbers that is more than x
template <typename P>
__device__ __forceinline__ int first_above(const P *run, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (run[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

struct PlanRows {
    const int32_t *cache_len, *new_rows;
    int32_t rows;
    int32_t *row_start, *sequence, *position;
    long long *slot;
    int32_t *served;
};

__device__ __forceinline__ int held_of(const csd_pages &p, int b) { return min(max(p.held[b], 0), p.table_stride); }

__device__ __forceinline__ void write_row(const csd_pages &p, const PlanRows &r, int shift, int row, int b) {
    int pos = -1;
    long long slot = -1;
    if (b < p.n_sequences) {
        pos = max(r.cache_len[b], 0) + row - r.row_start[b];
        const int i = pos >> shift, page = i < p.table_stride ? p.table[(size_t)b * p.table_stride + i] : -1;
        if ((unsigned)page < (unsigned)p.n_pages) slot = ((long long)page << shift) + (pos & ((1 << shift) - 1));
    } else {
        b = -1;
    }
    r.sequence[row] = b;
    r.position[row] = pos;
    r.slot[row] = slot;
}

__global__ __launch_bounds__(kThreads) void k_pages_plan(csd_pages p, PlanRows r, int shift) {
    __shared__ PagesShared S;
    const int tid = threadIdx.x;
    const int n_free = min(max(p.n_free[0], 0), p.n_pages);
    u64 want_pages = 0, want_rows = 0;                       // of the sequences before, served or not
    int taken = 0, rows = 0;                                 // served
    for (int b0 = 0; b0 < p.n_sequences; b0 += kThreads) {
        const int b = b0 + tid;
        int held = 0, n = 0, need = 0;
        bool fits = false;
        if (b < p.n_sequences) {
            const long long t = max(r.cache_len[b], 0);
            n = max(r.new_rows[b], 0);
            held = held_of(p, b);
            const long long wanted = (t + n + (1 << shift) - 1) >> shift;
            fits = wanted <= p.table_stride;
            need = fits ? max((int)wanted - held, 0) : 0;
            n = fits ? n : 0;
        }
        u64 all_pages, all_rows, all;
        const u64 pages_to = want_pages + group_scan(need, S.part, all_pages), rows_to = want_rows + group_scan(n, S.part, all_rows);
        want_pages += all_pages;
        want_rows += all_rows;
        const bool served = fits && (need == 0 || pages_to <= (u64)n_free) && (n == 0 || rows_to <= (u64)r.rows);
        if (!served) need = n = 0;
        // (served ones have n_free pages and r.rows rows at most)
        const u64 both = group_scan((u64)need << 32 | (uint32_t)n, S.part, all);
        S.run[tid] = (int)(both >> 32);
        S.from[tid] = held;
        if (b < p.n_sequences) {
            r.served[b] = served ? 1 : 0;
            r.row_start[b + 1] = rows + (int)(uint32_t)both;
            p.held[b] = held + need;
        }
        __syncthreads();
        const int count = (int)(all >> 32);
        for (int i = tid; i < count; i += kThreads) {
            const int j = first_above(S.run, kThreads, i), at = S.from[j] + i - (j ? S.run[j - 1] : 0);
            const int page = p.free_pages[n_free - 1 - taken - i];
            p.table[(size_t)(b0 + j) * p.table_stride + at] = page;
            if ((unsigned)page < (unsigned)p.n_pages) p.users[page] = 1;
        }
        taken += count;
        rows += (int)(uint32_t)all;
        __syncthreads();
    }
    if (tid == 0) {
        p.n_free[0] = n_free - taken;
        r.row_start[0] = 0;
    }
    if (r.rows > kRowsHere) return;
    __syncthreads();
    for (int row = tid; row < r.rows; row += kThreads) write_row(p, r, shift, row, first_above(r.row_start + 1, p.n_sequences, row));
}

__global__ __launch_bounds__(256) void k_pages_rows(csd_pages p, PlanRows r, int shift) {
    const int row = blockIdx.x * 256 + threadIdx.x;
    if (row < r.rows) write_row(p, r, shift, row, first_above(r.row_start + 1, p.n_sequences, row));
}

// The pages that leave their sequences are counted through by (sequence, place).  A page that nobody uses any more belongs to the first item that names it (two
// sequences may give up a shared page in one call): it is found by the least item written over the page's count.
__global__ __launch_bounds__(kThreads) void k_pages_release(csd_pages p, const int32_t *keep_len, int shift) {
    __shared__ PagesShared S;
    const int tid = threadIdx.x;
    const int n_free = min(max(p.n_free[0], 0), p.n_pages);
    constexpr int32_t kItem = -0x7FFFFFFF - 1;               // + item: a page that is waiting for its first one
    int back = 0, pushed = 0;
    for (int pass = 0; pass < 4; pass++) {
        int item0 = 0;
        for (int b0 = 0; b0 < p.n_sequences; b0 += kThreads) {
            const int b = b0 + tid;
            int kept = 0, gone = 0;
            if (b < p.n_sequences && keep_len[b] >= 0) {
                const int held = held_of(p, b);
                kept = (int)min(((long long)keep_len[b] + (1 << shift) - 1) >> shift, (long long)held);
                gone = held - kept;
            }
            u64 all;
            S.run[tid] = (int)group_scan(gone, S.part, all);
            S.from[tid] = kept;
            __syncthreads();
            if (pass == 3 && b < p.n_sequences && keep_len[b] >= 0) p.held[b] = kept;
            const int count = (int)all;
            for (int i0 = 0; i0 < count; i0 += kThreads) {
                const int i = i0 + tid;
                int page = -1;
                int32_t *entry = nullptr;
                if (i < count) {
                    const int j = first_above(S.run, kThreads, i), at = S.from[j] + i - (j ? S.run[j - 1] : 0);
                    entry = p.table + (size_t)(b0 + j) * p.table_stride + at;
                    page = *entry;
                    if ((unsigned)page >= (unsigned)p.n_pages) page = -1;
                }
                const int item = item0 + i;
                if (pass == 0) {
                    if (page >= 0) atomicSub(&p.users[page], 1);
                } else if (pass == 1) {
                    const int n = page >= 0 ? __hip_atomic_load(&p.users[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 1;
                    if (n == 0 || n < kItem / 2) atomicMin(&p.users[page], kItem + item);
                } else {
                    const bool mine = page >= 0 && __hip_atomic_load(&p.users[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == kItem + item;
                    u64 n;
                    const int rank = (int)group_scan(mine ? 1 : 0, S.part, n);
                    if (pass == 2) {
                        back += (int)n;
                    } else {
                        // the last one in order comes first, so that the next plan takes them in order
                        const int at = n_free + back - 1 - (pushed + rank - 1);
                        if (mine && at >= 0 && at < p.n_pages) p.free_pages[at] = page;
                        pushed += (int)n;
                        if (mine) p.users[page] = 0;
                        if (entry) *entry = -1;
                    }
                }
            }
            item0 += count;
            __syncthreads();
        }
        __threadfence();                                     // the counts, before the next pass reads them
        __syncthreads();
    }
    if (tid == 0) p.n_free[0] = min(n_free + back, p.n_pages);
}

// One workgroup per sequence.  Only sequences that hold nothing take, and only from ones that take nothing: no one reads what another writes.
__global__ __launch_bounds__(256) void k_pages_share(csd_pages p, const int32_t *source, const int32_t *length, int shift) {
    const int b = blockIdx.x, s = source[b];
    if (s < 0 || s >= p.n_sequences || s == b || p.held[b] > 0 || source[s] >= 0) return;
    const int n = min(max(length[b], 0) >> shift, held_of(p, s));
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 256) {
        const int page = p.table[(size_t)s * p.table_stride + i];
        p.table[(size_t)b * p.table_stride + i] = page;
        if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(&p.users[page], 1);
    }
    if (threadIdx.x == 0) p.held[b] = n;
}

// ------------------------------------------------------------------------------------------ entry points

static int32_t check_pages(const csd_pages *p, int &shift) {
    if (!p || !p->table || !p->held || !p->free_pages || !p->n_free || !p->users) return CSD_ENULL;
    if (p->n_pages < 1 || p->n_sequences < 1 || p->table_stride < 1) return CSD_EINVAL;
    if (p->page_rows < 16 || p->page_rows > 1024 || (p->page_rows & (p->page_rows - 1))) return CSD_EINVAL;
    if ((long long)p->table_stride * p->page_rows > (1ll << 30) || p->n_sequences > (1 << 20) || (long long)p->n_sequences * p->table_stride > (1ll << 30) ||
        p->n_pages > (1 << 30))
        return CSD_ESHAPE;
    shift = 0;
    while ((1 << shift) < p->page_rows) shift++;
    return CSD_OK;
}

extern "C" int32_t csd_pages_plan(const csd_pages *pages, const int32_t *cache_len, const int32_t *new_rows, int32_t rows, int32_t *row_start,
                                  int32_t *sequence, int32_t *position, int64_t *slot, int32_t *served, void *stream) {
    int shift;
    const int32_t rc = check_pages(pages, shift);
    if (rc != CSD_OK) return rc;
    if (rows < 0) return CSD_EINVAL;
    if (rows > (1 << 22)) return CSD_ESHAPE;
    if (!cache_len || !new_rows || !row_start || !served || (rows > 0 && (!sequence || !position || !slot))) return CSD_ENULL;
    if ((uintptr_t)slot % 8) return CSD_EINVAL;
    const PlanRows r{cache_len, new_rows, rows, row_start, sequence, position, (long long *)slot, served};
    hipLaunchKernelGGL(k_pages_plan, dim3(1), dim3(kThreads), 0, (hipStream_t)stream, *pages, r, shift);
    if (rows > kRowsHere) hipLaunchKernelGGL(k_pages_rows, dim3((rows + 255) / 256), dim3(256), 0, (hipStream_t)stream, *pages, r, shift);
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}

extern "C" int32_t csd_pages_release(const csd_pages *pages, const int32_t *keep_len, void *stream) {
    int shift;
    const int32_t rc = check_pages(pages, shift);
    if (rc != CSD_OK) return rc;
    if (!keep_len) return CSD_ENULL;
    hipLaunchKernelGGL(k_pages_release, dim3(1), dim3(kThreads), 0, (hipStream_t)stream, *pages, keep_len, shift);
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}

extern "C" int32_t csd_pages_share(const csd_pages *pages, const int32_t *source, const int32_t *length, void *stream) {
    int shift;
    const int32_t rc = check_pages(pages, shift);
    if (rc != CSD_OK) return rc;
    if (!source || !length) return CSD_ENULL;
    hipLaunchKernelGGL(k_pages_share, dim3(pages->n_sequences), dim3(256), 0, (hipStream_t)stream, *pages, source, length, shift);
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}
