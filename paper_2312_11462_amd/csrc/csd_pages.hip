// The pages of a paged cache: page tables, row starts and slots of a step's new rows, from the sequences' lengths; pages of rows that are not kept given back;
// pages of a common prompt shared.
//
// Every call is bound by its trips to memory, for a few bytes each: one workgroup, a thread per sequence, running sums over them, and what the next
// stage needs in LDS.  A plan has five trips (lengths; of pages that are written on, the tables and the counts of users; the stack; the tables of rows that had their
// page before), a release two (tables; the pages' counts).  64 sequences, plan and release: 9.3 us, 0.55 of them the look at the users.  The
// rows of a step are written by the same workgroup where there are few, else by a second launch.
#include "csd_lanes.h"

static constexpr int kRowsHere = 4096;                       // rows that the planning workgroup writes itself
static constexpr int kFresh = 2048;                          // pages of a plan that are kept in LDS for the rows
static constexpr int kAtOnce = 8;                            // pages that a thread has on their way (4112 pages taken and given back: by four 25 us)

template <int N>
struct PagesShared {
    u64 part[2][N / 64];
    uint32_t odd[N / 64];
    int32_t run[N];               // pages up to and with a sequence
    int32_t from[N];              // its first one of them, as an entry of its table
    int32_t end[N], pos[N];       // plan: where its rows end, and the position of the first
    int32_t fresh[kFresh];
};

// Running sums over the workgroup, inclusive, of two numbers; `totals`: of all; true if `odd` is, anywhere.
template <int N>
__device__ __forceinline__ bool group_scan(PagesShared<N> &S, u64 &a, u64 &b, u64 &all_a, u64 &all_b, bool odd) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    a = wave_scan(a);
    b = wave_scan(b);
    const bool here = __any(odd);
    __syncthreads();
    if (lane == 63) {
        S.part[0][wave] = a;
        S.part[1][wave] = b;
        S.odd[wave] = here ? 1 : 0;
    }
    __syncthreads();
    uint32_t some = 0;
    all_a = all_b = 0;
#pragma unroll
    for (int w = 0; w < N / 64; w++) {
        if (w == wave) {
            a += all_a;
            b += all_b;
        }
        all_a += S.part[0][w];
        all_b += S.part[1][w];
        some |= S.odd[w];
    }
    return some != 0;
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

// The same for N numbers, a power of two, in as many steps whatever they are, so that several searches go side by side.
template <int N>
__device__ __forceinline__ int first_above(const int32_t (&run)[N], int x) {
    int at = 0;
#pragma unroll
    for (int s = N / 2; s > 0; s >>= 1) at += run[at + s - 1] <= x ? s : 0;
    return at;
}

struct PlanRows {
    const int32_t *cache_len, *new_rows;
    int32_t rows;
    int32_t *row_start, *sequence, *position;
    long long *slot;
    int32_t *served;
};

__device__ __forceinline__ int held_of(const csd_pages &p, int b) { return min(max(p.held[b], 0), p.table_stride); }

// Whether one of a sequence's entries [from, to) names a page that others use too: its rows are not this sequence's to write.
__device__ __forceinline__ bool shared_among(const csd_pages &p, int b, int from, int to) {
    constexpr int AHEAD = 4;                                 // (one entry mostly: the page that the sequence's last row is in)
    bool shared = false;
    for (int i0 = from; i0 < to && !shared; i0 += AHEAD) {
        int page[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) page[u] = i0 + u < to ? p.table[(size_t)b * p.table_stride + i0 + u] : -1;
#pragma unroll
        for (int u = 0; u < AHEAD; u++)
            if ((unsigned)page[u] < (unsigned)p.n_pages) shared |= p.users[page[u]] > 1;
    }
    return shared;
}

__device__ __forceinline__ void write_row(const csd_pages &p, const PlanRows &r, int shift, int row, int b, int pos, int page) {
    r.sequence[row] = b;
    r.position[row] = pos;
    r.slot[row] = (unsigned)page < (unsigned)p.n_pages ? ((long long)page << shift) + (pos & ((1 << shift) - 1)) : -1;
}

template <int N>
__global__ __launch_bounds__(N) void k_pages_plan(csd_pages p, PlanRows r, int shift, int rows_here) {
    __shared__ PagesShared<N> S;
    const int tid = threadIdx.x;
    const int n_free = min(max(p.n_free[0], 0), p.n_pages);
    u64 want_pages = 0, want_rows = 0;                       // of the sequences before, served or not
    int taken = 0, rows = 0;                                 // served
    for (int b0 = 0; b0 < p.n_sequences; b0 += N) {
        const int b = b0 + tid;
        int held = 0, n = 0, need = 0, t = 0;
        bool fits = true;
        if (b < p.n_sequences) {
            t = max(r.cache_len[b], 0);
            n = max(r.new_rows[b], 0);
            held = held_of(p, b);
            const long long wanted = ((long long)t + n + (1 << shift) - 1) >> shift;
            fits = wanted <= p.table_stride;
            if (fits && n > 0) fits = !shared_among(p, b, t >> shift, min(held, (int)wanted));
            need = fits ? max((int)wanted - held, 0) : 0;
            n = fits ? n : 0;
        }
        u64 pages_to = need, rows_to = n, all_pages, all_rows;
        const bool some_do_not_fit = group_scan<N>(S, pages_to, rows_to, all_pages, all_rows, !fits);
        pages_to += want_pages;
        rows_to += want_rows;
        const bool served = fits && (need == 0 || pages_to <= (u64)n_free) && (n == 0 || rows_to <= (u64)r.rows);
        u64 mine = pages_to - want_pages, my_rows = rows_to - want_rows, count64 = all_pages, rows64 = all_rows;
        if (some_do_not_fit || want_pages + all_pages > (u64)n_free || want_rows + all_rows > (u64)r.rows) {
            // somebody goes without: the sums over those who do not
            if (!served) need = n = 0;
            mine = need;
            my_rows = n;
            group_scan<N>(S, mine, my_rows, count64, rows64, false);
        }
        want_pages += all_pages;
        want_rows += all_rows;
        // (served ones have n_free pages and r.rows rows at most)
        S.run[tid] = (int)mine;
        S.from[tid] = held;
        S.end[tid] = rows + (int)my_rows;
        S.pos[tid] = t;
        if (b < p.n_sequences) {
            r.served[b] = served ? 1 : 0;
            r.row_start[b + 1] = rows + (int)my_rows;
            if (need) p.held[b] = held + need;
        }
        const int count = (int)count64;
        __syncthreads();
        for (int i0 = tid; i0 < count; i0 += kAtOnce * N) {
            int page[kAtOnce], j[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; u++)
                if (i0 + u * N < count) page[u] = p.free_pages[n_free - 1 - taken - i0 - u * N];
#pragma unroll
            for (int u = 0; u < kAtOnce; u++)
                if (i0 + u * N < count) j[u] = first_above(S.run, i0 + u * N);
#pragma unroll
            for (int u = 0; u < kAtOnce; u++) {
                const int i = i0 + u * N;
                if (i >= count) break;
                p.table[(size_t)(b0 + j[u]) * p.table_stride + S.from[j[u]] + i - (j[u] ? S.run[j[u] - 1] : 0)] = page[u];
                if ((unsigned)page[u] < (unsigned)p.n_pages) p.users[page[u]] = 1;
                if (i < kFresh) S.fresh[i] = page[u];
            }
        }
        taken += count;
        rows += (int)rows64;
        __syncthreads();
    }
    if (tid == 0) {
        p.n_free[0] = n_free - taken;
        r.row_start[0] = 0;
    }
    if (!rows_here) return;                                  // (else all sequences are in LDS)
    for (int row = tid; row < r.rows; row += N) {
        const int b = first_above(S.end, p.n_sequences, row);
        if (b == p.n_sequences) {
            write_row(p, r, shift, row, -1, -1, -1);
            continue;
        }
        const int pos = S.pos[b] + row - (b ? S.end[b - 1] : 0), i = pos >> shift, fresh = (b ? S.run[b - 1] : 0) + i - S.from[b];
        write_row(p, r, shift, row, b, pos, i >= S.from[b] && fresh < kFresh ? S.fresh[fresh] : p.table[(size_t)b * p.table_stride + i]);
    }
}

// The rows of a step, behind its plan.
__global__ __launch_bounds__(256) void k_pages_rows(csd_pages p, PlanRows r, int shift) {
    constexpr int kStarts = 4096;
    __shared__ int32_t s_end[kStarts];
    const int row = blockIdx.x * 256 + threadIdx.x;
    int b;
    if (p.n_sequences <= kStarts) {
        for (int i = threadIdx.x; i < p.n_sequences; i += 256) s_end[i] = r.row_start[i + 1];
        __syncthreads();
        b = first_above(s_end, p.n_sequences, row);
    } else {
        b = first_above(r.row_start + 1, p.n_sequences, row);
    }
    if (row >= r.rows) return;
    if (b == p.n_sequences) return write_row(p, r, shift, row, -1, -1, -1);
    const int pos = max(r.cache_len[b], 0) + row - r.row_start[b], i = pos >> shift;
    write_row(p, r, shift, row, b, pos, i < p.table_stride ? p.table[(size_t)b * p.table_stride + i] : -1);
}

// The pages that leave their sequences, "items", are counted through by (sequence, place).
template <int N>
struct Release {
    const csd_pages &p;
    const int32_t *keep_len;
    int shift;
    PagesShared<N> &S;

    // items of the N sequences from b0 on; S.run, S.from
    __device__ __forceinline__ int items(int b0, int &kept) const {
        const int b = b0 + threadIdx.x;
        int gone = 0;
        kept = -1;                                           // (left alone)
        if (b < p.n_sequences) {
            const int keep = keep_len[b], held = held_of(p, b);
            if (keep >= 0) {
                kept = (int)min(((long long)keep + (1 << shift) - 1) >> shift, (long long)held);
                gone = held - kept;
            }
        }
        u64 run = gone, none = 0, all, all_none;
        group_scan<N>(S, run, none, all, all_none, false);
        S.run[threadIdx.x] = (int)run;
        S.from[threadIdx.x] = max(kept, 0);
        __syncthreads();
        return (int)all;
    }
    // where item i is named
    __device__ __forceinline__ int32_t *entry(int b0, int i) const {
        const int j = first_above(S.run, i), at = S.from[j] + i - (j ? S.run[j - 1] : 0);
        return p.table + (size_t)(b0 + j) * p.table_stride + at;
    }
    __device__ __forceinline__ int page_of(const int32_t *entry) const {
        const int page = *entry;
        return (unsigned)page < (unsigned)p.n_pages ? page : -1;
    }
    __device__ __forceinline__ int users_of(int page) const { return __hip_atomic_load(&p.users[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

    // Any items.  A page that nobody uses any more belongs to the first item that names it (two sequences may give up a shared page in one call): it is found
    // by the least item written over the page's count.  Pass 0: users go down; 1: firsts; 2: how many; 3: back to the stack.
    __device__ __forceinline__ void any(int first_pass, int n_free) const {
        const int tid = threadIdx.x;
        constexpr int32_t kItem = -0x7FFFFFFF - 1;           // + item: a page that is waiting for its first one
        int back = 0, pushed = 0;
        for (int pass = first_pass; pass < 4; pass++) {
            int item0 = 0;
            for (int b0 = 0; b0 < p.n_sequences; b0 += N) {
                int kept;
                const int count = items(b0, kept);
                if (pass == 3 && kept >= 0) p.held[b0 + tid] = kept;
                for (int i0 = 0; i0 < count; i0 += N) {
                    const int i = i0 + tid, item = item0 + i;
                    int32_t *at = i < count ? entry(b0, i) : nullptr;
                    const int page = at ? page_of(at) : -1;
                    if (pass == 0) {
                        if (page >= 0) atomicSub(&p.users[page], 1);
                    } else if (pass == 1) {
                        const int n = page >= 0 ? users_of(page) : 1;
                        if (n == 0 || n < kItem / 2) atomicMin(&p.users[page], kItem + item);
                    } else {
                        const bool mine = page >= 0 && users_of(page) == kItem + item;
                        u64 rank = mine ? 1 : 0, none = 0, n, all_none;
                        group_scan<N>(S, rank, none, n, all_none, false);
                        if (pass == 2) {
                            back += (int)n;
                        } else {
                            // the last one in order comes first, so that the next plan takes them in order
                            const int to = n_free + back - pushed - (int)rank;
                            if (mine && to >= 0 && to < p.n_pages) p.free_pages[to] = page;
                            pushed += (int)n;
                            if (mine) p.users[page] = 0;
                            if (at) *at = -1;
                        }
                    }
                }
                item0 += count;
                __syncthreads();
            }
            __threadfence();                                 // the counts, before the next pass reads them
            __syncthreads();
        }
        if (tid == 0) p.n_free[0] = min(n_free + back, p.n_pages);
    }
};

template <int N>
__global__ __launch_bounds__(N) void k_pages_release(csd_pages p, const int32_t *keep_len, int shift) {
    __shared__ PagesShared<N> S;
    const Release<N> x{p, keep_len, shift, S};
    const int tid = threadIdx.x, n_free = min(max(p.n_free[0], 0), p.n_pages);
    if (p.n_sequences > N) return x.any(0, n_free);
    // Where every item names a page that it alone uses, its place in the stack is its number.  Whether that is so is seen from the counts as they go down.
    int kept;
    const int count = x.items(0, kept);
    bool odd = false;
    int32_t *at[kAtOnce];
    int page[kAtOnce];
    auto request = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kAtOnce; u++) {
            const int i = i0 + u * N + tid;
            at[u] = i < count ? x.entry(0, i) : nullptr;
            page[u] = at[u] ? x.page_of(at[u]) : -1;
        }
    };
    auto put = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kAtOnce; u++)
            if (at[u]) {
                const int to = n_free + count - 1 - (i0 + u * N + tid);
                if (to < p.n_pages) p.free_pages[to] = page[u];
                *at[u] = -1;
            }
    };
    for (int i0 = 0; i0 < count; i0 += kAtOnce * N) {
        request(i0);
        int before[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; u++) before[u] = page[u] >= 0 ? atomicSub(&p.users[page[u]], 1) : at[u] ? 0 : 1;
#pragma unroll
        for (int u = 0; u < kAtOnce; u++) odd |= before[u] != 1;
    }
    if (__syncthreads_or(odd)) {
        __threadfence();
        __syncthreads();
        return x.any(1, n_free);
    }
    for (int i0 = 0; i0 < count; i0 += kAtOnce * N) {
        if (count > kAtOnce * N) request(i0);                // (else they are at hand)
        put(i0);
    }
    if (kept >= 0 && p.held[tid] != kept) p.held[tid] = kept;
    if (tid == 0 && count) p.n_free[0] = min(n_free + count, p.n_pages);
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
    const bool small = pages->n_sequences <= 256 && rows <= 1024, here = pages->n_sequences <= 1024 && rows <= kRowsHere;
    if (small) hipLaunchKernelGGL(k_pages_plan<256>, dim3(1), dim3(256), 0, (hipStream_t)stream, *pages, r, shift, 1);
    else hipLaunchKernelGGL(k_pages_plan<1024>, dim3(1), dim3(1024), 0, (hipStream_t)stream, *pages, r, shift, here ? 1 : 0);
    if (!small && !here && rows > 0) hipLaunchKernelGGL(k_pages_rows, dim3((rows + 255) / 256), dim3(256), 0, (hipStream_t)stream, *pages, r, shift);
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}

extern "C" int32_t csd_pages_release(const csd_pages *pages, const int32_t *keep_len, void *stream) {
    int shift;
    const int32_t rc = check_pages(pages, shift);
    if (rc != CSD_OK) return rc;
    if (!keep_len) return CSD_ENULL;
    hipLaunchKernelGGL(k_pages_release<1024>, dim3(1), dim3(1024), 0, (hipStream_t)stream, *pages, keep_len, shift);
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
