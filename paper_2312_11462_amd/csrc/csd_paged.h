// Shared by the kernels of the paged KV cache (csd_paged.hip: rows in and out, commit; csd_paged_attn.hip: attention).
#pragma once

#include <type_traits>

#include "csd_epilogue.h"
#include "csd_internal.h"

#define CSD_PAGED_COUNTER_BYTES CSD_PAGED_WORKSPACE_ZERO_BYTES      /* the workspace begins with counters, zero between launches */

// The pool of one layer and the page table, by value in the kernels' arguments.
struct PagedPool {
    void *k, *v;                  // this layer's [n_pages][Hkv][page_rows][D]
    uint8_t *ks, *vs;             // e4m3: this layer's scale bytes [n_pages][Hkv][page_rows]
    const int32_t *table;
    int32_t table_stride, n_pages, page_shift, Hkv, D;
};

// The ragged batch of a call.
struct PagedRows {
    const int32_t *row_start, *pos;
    int32_t B, rows;
};

// rows [start, start + m) of the call are sequence b's, from position t on
struct PagedSeq {
    int start, m, t;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedRows &r, int b) {
    const int s = min(max(r.row_start[b], 0), r.rows);
    const int e = min(max(r.row_start[b + 1], s), r.rows);
    return PagedSeq{s, e - s, min(max(r.pos[b], 0), 0x3FFFFFFF)};
}

// Tree blocks (64 rows at most): the rows of the sequence's block that row `lane` continues, and itself, one bit each, by doubling the step up; a parent
// outside [0, row) is row 0.
__device__ __forceinline__ unsigned long long lane_of(unsigned long long v, int lane) {
    return ((unsigned long long)(unsigned)__shfl((unsigned)(v >> 32), lane, 64) << 32) | (unsigned)__shfl((unsigned)v, lane, 64);
}
__device__ __forceinline__ unsigned long long paged_ancestors(const int32_t *parent, const PagedSeq &s, int lane) {
    unsigned long long anc = 1ull << lane;
    int up = 0;
    if (lane < s.m && lane > 0) {
        up = parent[s.start + lane];
        if (up < 0 || up >= lane) up = 0;
    }
    anc |= 1ull << up;
#pragma unroll
    for (int k = 0; k < 6; k++) {
        anc |= lane_of(anc, up);
        up = __shfl(up, up, 64);
    }
    return anc;
}

// page of a position, -1: there is none
__device__ __forceinline__ int paged_page(const PagedPool &p, int b, int pos) {
    const int i = pos >> p.page_shift;
    if (pos < 0 || i >= p.table_stride) return -1;
    const int page = p.table[(size_t)b * p.table_stride + i];
    return (unsigned)page < (unsigned)p.n_pages ? page : -1;
}
// row index of (page, head, position) in a layer's pool
__device__ __forceinline__ size_t paged_row(const PagedPool &p, int page, int head, int pos) {
    return (((size_t)page * p.Hkv + head) << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
}

__device__ __forceinline__ float pow2_of_byte(unsigned s) { return __uint_as_float(s << 23); }   // 2^(s - 127), s in 1 .. 254

// Eight consecutive elements as floats, from fp32, bf16 or (unscaled) e4m3 memory.
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<float>(const float *p, float (&x)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x[i] = a[i];
        x[4 + i] = b[i];
    }
}
template <> __device__ __forceinline__ void load8<bf16_t>(const bf16_t *p, float (&x)[8]) {
    const u32x4 a = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x[2 * i] = __uint_as_float(a[i] << 16);
        x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
}
template <> __device__ __forceinline__ void load8<uint8_t>(const uint8_t *p, float (&x)[8]) {
    const u32x2 a = *reinterpret_cast<const u32x2 *>(p);
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[i], true);
        x[4 * i] = lo[0];
        x[4 * i + 1] = lo[1];
        x[4 * i + 2] = hi[0];
        x[4 * i + 3] = hi[1];
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&x)[8]);
template <> __device__ __forceinline__ void store8<float>(float *p, const float (&x)[8]) {
    *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
template <> __device__ __forceinline__ void store8<bf16_t>(bf16_t *p, const float (&x)[8]) {
    *reinterpret_cast<u32x4 *>(p) =
        u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
}

// Values that are not finite.  Rows of a block differ in what they attend, and on the matrix cores 0 * inf = NaN would reach the rows that do
// not attend such a value.  Where rows differ, the kernels take these values out of the products and remember that there were some;
// in that rare case they go through the keys once more and add the values themselves to the outputs of the rows that attend them.
// Bits of a pair of bf16 that are not finite, as masks of 16 ones.
__device__ __forceinline__ uint32_t odd_halves(uint32_t v) {
    return ((v & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((v & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}
// what element c of a row adds to the output of a row that attends it (or does not): the value if it is not finite, else 0
template <bool F8>
__device__ __forceinline__ float odd_value(const void *row, int c, bool attends) {
    float v;
    if constexpr (F8) v = __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t *>(row)[c], 0);
    else v = bf16_to_f32(reinterpret_cast<const bf16_t *>(row)[c]);
    return fabsf(v) < INFINITY || !attends ? 0.f : v;
}

// A pair of weights as two bf16 planes {hi, lo}, w = hi + lo, off by at most 2^-15 of w.  An infinite value has to stay one under both: so hi is w cut
// off, and lo not negative; and where the pool's type has infinities (INF), lo is at least 2^-16 of hi, so not zero either (a weight below 2^-110 may have 0).
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
template <bool INF>
__device__ __forceinline__ u32x2 two_planes(float w0, float w1) {
    const uint32_t h0 = __float_as_uint(w0) & 0xFFFF0000u, h1 = __float_as_uint(w1) & 0xFFFF0000u;
    const uint32_t hi = __builtin_amdgcn_perm(h1, h0, 0x07060302u);
    uint32_t lo = pack_bf16x2(w0 - __uint_as_float(h0), w1 - __uint_as_float(h1));
    if constexpr (INF) {
        const u16x2 least = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, hi), u16x2{16 << 7, 16 << 7});
        lo = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, lo), least));
    }
    return u32x2{hi, lo};
}

// Blocks of tokens to review, trees among them, and single tokens are weighed in two planes, whatever else is in the call, and so is all cross-attention; the chunks
// of more rows than this in one: bf16, off by half a step (2^-8 of a weight, random in sign; the sum of the weights is kept in fp32).
#define CSD_PAGED_FINE_ROWS 64

// The shares: T tiles over n workgroups, the first T % n of them one tile longer.
struct PagedShares {
    int q, r;
    __device__ __forceinline__ PagedShares(int T, int n) : q(T / n), r(T % n) {}
    __device__ __forceinline__ int first(int w) const { return w * q + min(w, r); }
    __device__ __forceinline__ int owner(int tile) const {
        const int wide = r * (q + 1);
        return tile < wide ? tile / (q + 1) : r + (tile - wide) / q;
    }
};

// One attention call.
struct PagedAttn {
    PagedPool p;
    PagedRows r;
    const int32_t *parent;        // tree blocks, or null
    int max_rows, group;          // rows of a sequence at most; query heads per key-value head
    const void *q;
    long long q_stride;
    void *out;
    float scale;
    void *ws;
    int32_t cross;                // the sequences' positions are an encoder's rows (pos[b] of them): every row attends them all, and no row of the call is one
};
// The kernels are made for either (a look at `cross` in one kernel for both: chunks of 2048 rows 417 us, 412 without).
template <bool CROSS>
struct PagedAttnOf : PagedAttn {
    // the last position that row i of a sequence at t attends, and (cross: there may be none) the positions up to it
    __device__ __forceinline__ int last(int t, int i) const { return CROSS ? t - 1 : t + i; }
    __device__ __forceinline__ int keys(int t, int i) const { return min(last(t, i) + 1, p.table_stride << p.page_shift); }
};
// launch(PagedAttnOf<..>) for the call's own
template <typename F>
static inline void csd_paged_by_cross(const PagedAttn &a, F launch) {
    if (a.cross) launch(PagedAttnOf<true>{a});
    else launch(PagedAttnOf<false>{a});
}
// Parts of items.  A workgroup has two at most that are not whole items: one that others began (its slot 0) and one that others end (slot 1).  A slot
// holds R rows of DH outputs (weighted sums), their maximum and the sum of weights.  Slots are written and read within a launch by workgroups on
// different compute dies: device scope (the stores write through).
template <int DH> constexpr int part_stride() { return DH + 4; }     // floats per row, 16-byte pieces
template <int DH, int R>
struct PagedParts {
    __amdgpu_buffer_rsrc_t r;
    int w_first, parts;                                      // the workgroup that has the item's first part; how many there are
    __device__ __forceinline__ PagedParts(void *ws, int wgs, int w_first_, int parts_) : w_first(w_first_), parts(parts_) {
        r = ch_rsrc(reinterpret_cast<char *>(ws) + CSD_PAGED_COUNTER_BYTES, (size_t)2 * wgs * R * part_stride<DH>() * 4);
    }
    __device__ __forceinline__ int at(int part, int row, int c) const {
        return (((2 * (w_first + part) + (part == 0 ? 1 : 0)) * R + row) * part_stride<DH>() + c) * 4;
    }
    __device__ __forceinline__ void store(int part, int row, int c, f32x4 v) const {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, at(part, row, c), 0, CH_SC1);
    }
    __device__ __forceinline__ f32x4 load(int part, int row, int c) const {
        return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at(part, row, c), 0, CH_SC1));
    }
    // Behind the stores of this workgroup's part: true in the workgroup that finishes last.  `flag`: LDS.
    __device__ __forceinline__ bool arrive(void *ws, int *flag) const {
        __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): the stores are acknowledged before the counter moves
        __syncthreads();
        if (threadIdx.x == 0)
            *flag = __hip_atomic_fetch_add(reinterpret_cast<unsigned *>(ws) + w_first, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(parts - 1);
        __syncthreads();
        return *flag != 0;
    }
    // The last one joins the parts, in their order: out = sum f_k o_k / sum f_k l_k with f_k = 2^(m_k - max m).  lds: (2 * parts + 1) * R floats.  `out` of a row:
    // 256 threads, four features each.  P such places of a thread and K parts are requested at once, the first of them along with the maxima:
    // each round of requests is a trip to memory (two rows of 4 heads of 64 over 3000 keys, up to twenty parts: 11.6 us by fours, 10.5 by sixteen; as
    // many in flight again spill).
    template <typename OUT>
    __device__ __forceinline__ void join(void *ws, float *lds, int rows, OUT out) const {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                        // (what follows from it is made here, not kept in registers from the kernel's start on)
        float *fade = lds, *sum = lds + parts * R, *inv = lds + 2 * parts * R;
        constexpr int C = DH / 4, P = R * C / 256 < 1 ? 1 : R * C / 256 > 4 ? 4 : R * C / 256, K = 16 / P;
        f32x4 v[P][K];
        auto request = [&](int x0, int k0) {
            const int voff = ((x0 + tid) / C * part_stride<DH>() + 4 * (tid % C)) * 4;
#pragma unroll
            for (int k = 0; k < K; k++) {
                if (k0 + k >= parts) break;
                const int soff = __builtin_amdgcn_readfirstlane(at(k0 + k, 0, 0));
#pragma unroll
                for (int i = 0; i < P; i++)
                    if (x0 + 256 * i + tid < rows * C)
                        v[i][k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff + i * (256 / C) * part_stride<DH>() * 4, CH_SC1));
            }
        };
        request(0, 0);
        for (int x = tid; x < parts * rows; x += 256) {
            const int k = x / rows, row = x - k * rows;
            const f32x4 ml = load(k, row, DH);
            fade[k * R + row] = ml[0];
            sum[k * R + row] = ml[1];
        }
        __syncthreads();
        if (tid < rows) {
            float m = -INFINITY, l = 0.f;
            for (int k = 0; k < parts; k++) m = fmaxf(m, fade[k * R + tid]);
            const float ref = m == -INFINITY ? 0.f : m;
            for (int k = 0; k < parts; k++) {
                const float f = __builtin_amdgcn_exp2f(fade[k * R + tid] - ref);
                l += f * sum[k * R + tid];
                fade[k * R + tid] = f;
            }
            inv[tid] = m == -INFINITY ? -1.f : 1.f / l;      // (-1: the row has nothing to attend)
        }
        __syncthreads();
        for (int x0 = 0; x0 < rows * C; x0 += 256 * P) {
            f32x4 o[P];
#pragma unroll
            for (int i = 0; i < P; i++) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int row0 = (x0 + tid) / C;
            for (int k0 = 0; k0 < parts; k0 += K) {
                if (x0 + k0 > 0) request(x0, k0);
#pragma unroll
                for (int k = 0; k < K; k++) {
                    if (k0 + k >= parts) break;
#pragma unroll
                    for (int i = 0; i < P; i++) o[i] += v[i][k] * fade[(k0 + k) * R + min(row0 + i * (256 / C), R - 1)];
                }
            }
#pragma unroll
            for (int i = 0; i < P; i++) {
                if (x0 + 256 * i + tid >= rows * C) continue;
                const int row = row0 + i * (256 / C), c = 4 * (tid % C);
                const float f = inv[row];
                *reinterpret_cast<u32x2 *>(out(row) + c) =
                    f == -1.f ? u32x2{0u, 0u} : u32x2{pack_bf16x2(o[i][0] * f, o[i][1] * f), pack_bf16x2(o[i][2] * f, o[i][3] * f)};
            }
        }
        if (tid == 0) __hip_atomic_store(reinterpret_cast<unsigned *>(ws) + w_first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next launch
    }
};

int32_t csd_paged_attention_enqueue(const PagedAttn &a, int32_t pool_dtype, int32_t q_dtype, hipStream_t st);

// csd_paged_few.hip: sequences of up to 32 rows per key-value head.
#define CSD_PAGED_FEW_GRID 512       /* two workgroups per compute unit */
#define CSD_PAGED_FEW_SHARE 4        /* tiles of 32 keys per workgroup at least */
#define CSD_PAGED_FEW_COST 8         /* what an item costs besides its keys, in such tiles */
#define CSD_PAGED_FEW_PARTS 64       /* parts of an item at most */
#define CSD_PAGED_FEW_ROWS 32
static_assert(CSD_PAGED_COUNTER_BYTES + 2ull * CSD_PAGED_FEW_GRID * CSD_PAGED_FEW_ROWS * 132 * 4 <= CSD_PAGED_WORKSPACE_BYTES, "");
// the types and head sizes of the kernels that split their work over workgroups
static inline bool csd_paged_few_types(int32_t head_dim, int32_t pool_dtype, int32_t q_dtype) {
    return q_dtype == CSD_DTYPE_BF16 && pool_dtype != CSD_DTYPE_FP32 && (head_dim == 64 || head_dim == 128);
}
bool csd_paged_few_fits(const PagedAttn &a, int32_t pool_dtype, int32_t q_dtype);
void csd_paged_few_enqueue(const PagedAttn &a, int rows, int32_t pool_dtype, hipStream_t st);

// csd_paged_many.hip: the others, in the same types and head sizes, 128 rows per workgroup and item.
#define CSD_PAGED_MANY_ROWS 128
#define CSD_PAGED_MANY_SHARE 4       /* tiles of 64 keys per part of an item at least */
#define CSD_PAGED_MANY_COST 4        /* what an item costs besides its keys, in such tiles */
#define CSD_PAGED_MANY_PARTS 14      /* parts of an item at most */
#define CSD_PAGED_MANY_GRID 512      /* two workgroups per compute unit */
#define CSD_PAGED_MANY_BATCH 512     /* sequences that take part at most */
// With more items (row tiles times key-value heads, as far as the host can tell) than this, and sequences of as many rows as the second (times the query heads that share keys; fewer leave more than
// a quarter of the workgroups' rows idle), csd_paged_chunk.hip takes over, a workgroup of 256 rows per item; but not for blocks of up to CSD_PAGED_FINE_ROWS rows.  us here and there, heads of
// 128 in bf16: 5 sequences of 300 rows over 0 to 1400 keys, 32 heads, 512 items, 66 and 76; 2 of 2048 rows over 2048 and 8191, 8 x 4 heads, 1040 items, 519 and 418; 42 of 328 rows over 0 to
// 1000, 8 heads, 1200 items, 104 and 119; 8 of 512 rows over 0 to 700, 32 heads, 1280 items, 103 and 88; blocks: 40 of 64 rows over 0 to 3000, 8 x 4 heads, 960 items, 137 and 178; 44 trees of 41 rows
// over 0 to 1400, 32 heads, 1856 items, 149 and 247; 150 of 48 rows over 100 to 400, 4 x 8 heads, 2400 items, 116 and 127 (e4m3 107 and 122, heads of 64 71 and 92).
#define CSD_PAGED_MANY_ITEMS 1024
#define CSD_PAGED_CHUNK_ROWS 384
static_assert(CSD_PAGED_COUNTER_BYTES + 2ull * CSD_PAGED_MANY_GRID * CSD_PAGED_MANY_ROWS * 132 * 4 <= CSD_PAGED_WORKSPACE_BYTES, "");
// min_rows: sequences of so many rows (times the query heads that share keys) or fewer are another kernel's.  How many can have more:
static inline long long csd_paged_batch(const PagedAttn &a, int min_rows) {
    const long long most = (long long)a.r.rows * a.group / (min_rows + 1);
    return most < a.r.B ? most : a.r.B;
}
void csd_paged_many_enqueue(const PagedAttn &a, int min_rows, int32_t pool_dtype, hipStream_t st);
void csd_paged_chunk_enqueue(const PagedAttn &a, int min_rows, int32_t pool_dtype, hipStream_t st);
