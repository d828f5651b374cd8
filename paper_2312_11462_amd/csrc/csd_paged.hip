// The paged KV cache: rows in (with quantisation), rows out, the commit of a tree's path, and the entry points' checks.
//
// All three move rows of D elements between dense rows and pages; they read and write each byte once and are bound by memory, or,
// with few rows, by the chain row -> sequence -> page -> place of dependent reads.
#include "csd_paged.h"

static constexpr int kPagedThreads = 256;

// e4m3: the byte e + 127 of a row with largest finite magnitude a: a = f * 2^x, f in [1, 2), and 448 = 1.75 * 2^8, so e = x - 8 while
// f <= 1.75, else x - 7; at least -126 (then a < 448 * 2^e holds too).
__device__ __forceinline__ int scale_byte(float a) {
    const uint32_t u = __float_as_uint(a);
    return max((int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), 1);
}

// 8 codes of x * 2^(127 - s).  The factor is a power of two, so the only rounding is the conversion's own, to nearest even.  With
// the largest scale (s = 247) a code of 256 would stand for 2^128, which no fp32 value reaches: 240 is the largest there.
__device__ __forceinline__ u32x2 quantise8(const float (&x)[8], int s) {
    const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
    uint32_t c[2];
    bool odd = s >= 247;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h] * inv, x[4 * h + 1] * inv, 0, false);
        c[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2] * inv, x[4 * h + 3] * inv, w, true);
    }
#pragma unroll
    for (int i = 0; i < 8; i++) odd |= !(fabsf(x[i]) < INFINITY);
    if (odd) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int at = 8 * (i & 3);
            if (!(fabsf(x[i]) < INFINITY)) c[i >> 2] |= 0x7Fu << at;
            else if (s >= 247 && ((c[i >> 2] >> at) & 0x7Fu) == 0x78u) c[i >> 2] -= 1u << at;
        }
    }
    return u32x2{c[0], c[1]};
}

// maximum over the 2^log_w neighbouring lanes of a row, in each of them (register moves up to sixteen lanes; a shuffle goes through LDS)
template <int CTRL>
__device__ __forceinline__ float max_dpp(float a) {
    return fmaxf(a, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(a), CTRL, 0xF, 0xF, false)));
}
__device__ __forceinline__ float row_max(float a, int log_w) {
    if (log_w > 0) a = max_dpp<0xB1>(a);                     // lane ^ 1
    if (log_w > 1) a = max_dpp<0x4E>(a);                     // lane ^ 2
    if (log_w > 2) a = max_dpp<0x141>(a);                    // 7 - lane, of eight
    if (log_w > 3) a = max_dpp<0x140>(a);                    // 15 - lane, of sixteen
    if (log_w > 4) a = fmaxf(a, __shfl_xor(a, 16, 64));
    return a;
}

// Eight elements of a dense row as they are in memory: bf16 one 16-byte piece, fp32 two.
template <typename T> struct Raw8 {
    u32x4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; i++) w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p) + i);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(w[i / 4][i % 4]);
            else x[i] = __uint_as_float(i & 1 ? w[0][i / 2] & 0xFFFF0000u : w[0][i / 2] << 16);
        }
    }
};

// Stores past the caches, for many dense rows: they are more than a cache level holds, and kept there they push out the pages still to be read (36004
// rows of 8 heads of 128, e4m3 to bf16: 57 -> 34 us; with the loads of the pages past them too 52).
template <typename T>
__device__ __forceinline__ void store8_past(T *p, const float (&x)[8]) {
    alignas(16) T t[8];
    store8<T>(t, x);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; i++) __builtin_nontemporal_store(reinterpret_cast<u32x4 *>(t)[i], reinterpret_cast<u32x4 *>(p) + i);
}

// Where to begin to look for the sequence of a row, 64 sequences at a time: all those before end at or before it (4096 sequences a step; uniform in the
// wave; 1024 single rows in, 8 heads of 128: 8.2 -> 6.4 us).
__device__ __forceinline__ int paged_block(const PagedRows &r, int row) {
    const int lane = threadIdx.x & 63;
    int b0 = 0;
    for (int g = 0; g + 64 < r.B; g += 4096) {
        const int e = g + (lane + 1) * 64;
        const int n = __popcll(__ballot(e <= r.B && r.row_start[min(e, r.B)] <= row));
        b0 = g + 64 * n;
        if (n < 64) break;
    }
    return b0;
}

// How the moves of rows are laid out.  A row of one head belongs to W lanes (W = 2^log_w: the power of two from D / 8 up), eight elements per lane, so its
// maximum stays inside the lanes.  A wave takes 64 / W consecutive rows of U heads: in the pool consecutive rows of a head lie one behind
// the other, their scale bytes too (with a wave on one row of 64 / W heads every scale byte was a store of its own: a prompt of 8198 rows of 32 heads of
// 128 56 -> 45 us).  Everything that a lane loads is requested before anything is looked up or used.
struct RowPlace {
    bool ok;          // the lane holds eight elements of a row of some sequence
    int page;         // -1: a place without a row
    size_t at;        // row index in the layer's pool, of head 0
};

__device__ __forceinline__ RowPlace row_place(const PagedPool &p, const PagedRows &r, int first, int row, bool active, int log_w) {
    const int lane = threadIdx.x & 63;
    // the sequence of each row of the wave: how many sequences end at or before it (64 ends at a time; the sequences of a wave's rows are
    // mostly the same)
    int b = paged_block(r, first);
    for (int b0 = b; b0 < r.B; b0 += 64) {
        const int end = b0 + lane < r.B ? r.row_start[b0 + lane + 1] : 0x7FFFFFFF;
        const int before = __popcll(__ballot(end <= first));
        b += before;
        for (int j = 1; j < 64 >> log_w; j++) {              // rows that begin another sequence than the wave's first one
            const int n = __popcll(__ballot(end <= first + j)) - before;
            if (row - first == j) b += n;
        }
        if (__popcll(__ballot(end <= first + (64 >> log_w) - 1)) < 64) break;
    }
    RowPlace o{false, -1, 0};
    if (!active || b >= r.B) return o;
    const PagedSeq s = paged_seq(r, b);
    if (row < s.start) return o;
    o.ok = true;
    const int pos = s.t + (row - s.start);
    o.page = paged_page(p, b, pos);
    if (o.page >= 0) o.at = paged_row(p, o.page, 0, pos);
    return o;
}

// TR: type of the dense rows, TP: of the pool (uint8_t: e4m3), U: heads per wave.
template <typename TR, typename TP, int U>
__global__ __launch_bounds__(kPagedThreads) void k_paged_write(PagedPool p, PagedRows r, const TR *__restrict__ k, long long k_stride,
                                                               const TR *__restrict__ v, long long v_stride, int log_w, int head_blocks) {
    const int wave = blockIdx.x * (kPagedThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int first = (wave / head_blocks) * (64 >> log_w), head0 = wave % head_blocks * U;
    if (first >= r.rows) return;
    const int row = first + (lane >> log_w), c = 8 * (lane & ((1 << log_w) - 1));
    const bool active = row < r.rows && c < p.D;
    Raw8<TR> raw[U][2];
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int side = 0; side < 2; side++) {
            raw[u][side] = Raw8<TR>{};
            if (active && head0 + u < p.Hkv) raw[u][side].load((side ? v + row * v_stride : k + row * k_stride) + (size_t)(head0 + u) * p.D + c);
        }
    const RowPlace o = row_place(p, r, first, row, active, log_w);
#pragma unroll
    for (int u = 0; u < U; u++) {
        if (head0 + u >= p.Hkv) break;
        const size_t at = o.at + ((size_t)(head0 + u) << p.page_shift);
#pragma unroll
        for (int side = 0; side < 2; side++) {
            float x[8];
            raw[u][side].get(x);
            TP *to = reinterpret_cast<TP *>(side ? p.v : p.k) + at * p.D + c;
            if constexpr (sizeof(TP) == 1) {
                float a = 0.f;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float f = fabsf(x[i]);
                    a = f < INFINITY ? fmaxf(a, f) : a;
                }
                a = row_max(a, log_w);
                const int s = scale_byte(a);
                if (o.page >= 0) {
                    *reinterpret_cast<u32x2 *>(to) = quantise8(x, s);
                    if (c == 0) (side ? p.vs : p.ks)[at] = (uint8_t)s;
                }
            } else {
                if (o.page >= 0) store8<TP>(to, x);
            }
        }
    }
}

template <typename TR, typename TP, int U>
__global__ __launch_bounds__(kPagedThreads) void k_paged_read(PagedPool p, PagedRows r, TR *__restrict__ k, long long k_stride,
                                                              TR *__restrict__ v, long long v_stride, int log_w, int head_blocks) {
    const int wave = blockIdx.x * (kPagedThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int first = (wave / head_blocks) * (64 >> log_w), head0 = wave % head_blocks * U;
    if (first >= r.rows) return;
    const int row = first + (lane >> log_w), c = 8 * (lane & ((1 << log_w) - 1));
    const RowPlace o = row_place(p, r, first, row, row < r.rows && c < p.D, log_w);
    if (!o.ok) return;
    float x[U][2][8], f[U][2];
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int side = 0; side < 2; side++) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[u][side][i] = 0.f;
            f[u][side] = 1.f;
            if (o.page >= 0 && head0 + u < p.Hkv) {
                const size_t at = o.at + ((size_t)(head0 + u) << p.page_shift);
                load8<TP>(reinterpret_cast<const TP *>(side ? p.v : p.k) + at * p.D + c, x[u][side]);
                if constexpr (sizeof(TP) == 1) f[u][side] = pow2_of_byte((side ? p.vs : p.ks)[at]);
            }
        }
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int side = 0; side < 2; side++) {
            if (head0 + u >= p.Hkv) break;
            if constexpr (sizeof(TP) == 1) {
#pragma unroll
                for (int i = 0; i < 8; i++) x[u][side][i] *= f[u][side];
            }
            TR *to = (side ? v + row * v_stride : k + row * k_stride) + (size_t)(head0 + u) * p.D + c;
            if constexpr (U > 1) store8_past<TR>(to, x[u][side]);
            else store8<TR>(to, x[u][side]);
        }
}

// The kept rows of a tree block to where a plain block would have put them.  A thread owns eight elements of one head of one
// layer, keys or values, and moves them row by row in order: path is increasing with path[j] >= j + 1, so row j + 1, which move j fills,
// is no source of a later move.
// E: bytes of an element (sources and places are moved as they are).
template <int E>
__global__ __launch_bounds__(kPagedThreads) void k_paged_commit(PagedPool p, size_t layer_rows, const int32_t *__restrict__ cache_len,
                                                                const int32_t *__restrict__ path, const int32_t *__restrict__ n_accepted,
                                                                int m) {
    __shared__ long long s_src[64], s_dst[64];    // row index of head 0, without the layer's part; -1: nothing to move
    __shared__ int s_n;
    const int b = blockIdx.y, layer = blockIdx.z;
    if (threadIdx.x < 64) {
        const int j = threadIdx.x, t = min(max(cache_len[b], 0), 0x3FFFFFFF);
        const int n = min(max(n_accepted[b], 0), m - 1);
        const int src = j < n ? path[(size_t)b * m + j] : 0, prev = j > 0 && j < n ? path[(size_t)b * m + j - 1] : 0;
        const bool good = j < n && src > prev && src >= j + 1 && src < m;
        const unsigned long long bad = __ballot(j < n && !good);
        const int kept = bad ? __ffsll((long long)bad) - 1 : n;
        long long from = -1, to = -1;
        if (j < kept && src != j + 1) {
            const int sp = paged_page(p, b, t + src), dp = paged_page(p, b, t + 1 + j);
            if (sp >= 0 && dp >= 0) {
                from = (long long)paged_row(p, sp, 0, t + src);
                to = (long long)paged_row(p, dp, 0, t + 1 + j);
            }
        }
        s_src[j] = from;
        s_dst[j] = to;
        if (j == 0) s_n = kept;
    }
    __syncthreads();
    const int per_head = p.D / 8, unit = blockIdx.x * kPagedThreads + threadIdx.x;
    const int side = unit / (p.Hkv * per_head);
    if (side > 1) return;
    const int head = (unit - side * p.Hkv * per_head) / per_head, c = unit % per_head;
    const size_t head_rows = (size_t)head << p.page_shift, base = (size_t)layer * layer_rows;
    char *pool = reinterpret_cast<char *>(side ? p.v : p.k);
    uint8_t *scale = side ? p.vs : p.ks;
    for (int j = 0; j < s_n; j++) {
        if (s_src[j] < 0) continue;
        const size_t from = base + s_src[j] + head_rows, to = base + s_dst[j] + head_rows;
        const char *f = pool + (from * p.D + c * 8) * E;
        char *g = pool + (to * p.D + c * 8) * E;
        if constexpr (E == 1) {
            *reinterpret_cast<u32x2 *>(g) = *reinterpret_cast<const u32x2 *>(f);
            if (c == 0) scale[to] = scale[from];
        } else {
#pragma unroll
            for (int i = 0; i < E / 2; i++) reinterpret_cast<u32x4 *>(g)[i] = reinterpret_cast<const u32x4 *>(f)[i];
        }
    }
}

// ------------------------------------------------------------------------------------------ entry points

static int ilog2(int x) {
    int n = 0;
    while ((1 << n) < x) n++;
    return n;
}

static int32_t check_pool(const csd_paged_kv *kv) {
    if (!kv || !kv->k || !kv->v || !kv->table) return CSD_ENULL;
    if (kv->dtype != CSD_DTYPE_FP32 && kv->dtype != CSD_DTYPE_BF16 && kv->dtype != CSD_DTYPE_FP8) return CSD_EINVAL;
    if (kv->dtype == CSD_DTYPE_FP8 && (!kv->k_scale || !kv->v_scale)) return CSD_ENULL;
    if (kv->n_layers < 1 || kv->n_pages < 1 || kv->n_kv_heads < 1 || kv->table_stride < 1) return CSD_EINVAL;
    if (kv->head_dim < 8 || kv->head_dim > 256 || kv->head_dim % 8) return CSD_EINVAL;
    if (kv->page_rows < 16 || kv->page_rows > 1024 || (kv->page_rows & (kv->page_rows - 1))) return CSD_EINVAL;
    if (((uintptr_t)kv->k | (uintptr_t)kv->v) % 16 || ((uintptr_t)kv->k_scale | (uintptr_t)kv->v_scale) % 8) return CSD_EINVAL;
    if ((long long)kv->table_stride * kv->page_rows > (1ll << 30) || kv->n_kv_heads > 4096) return CSD_ESHAPE;
    return CSD_OK;
}

static int32_t check_rows(const csd_paged_kv *kv, int32_t layer, const int32_t *row_start, const int32_t *pos, int32_t B, int32_t rows,
                          int32_t dtype) {
    const int32_t rc = check_pool(kv);
    if (rc != CSD_OK) return rc;
    if (!row_start || !pos) return CSD_ENULL;
    if (B < 1 || rows < 0 || layer < 0 || layer >= kv->n_layers) return CSD_EINVAL;
    if (dtype != CSD_DTYPE_FP32 && dtype != CSD_DTYPE_BF16) return CSD_EINVAL;
    if (rows > (1 << 22) || B > (1 << 20)) return CSD_ESHAPE;
    return CSD_OK;
}

static size_t pool_rows(const csd_paged_kv *kv) { return (size_t)kv->n_pages * kv->n_kv_heads * kv->page_rows; }

PagedPool csd_paged_layer(const csd_paged_kv *kv, int32_t layer) {
    const size_t rows = pool_rows(kv) * layer, esz = kv->dtype == CSD_DTYPE_FP32 ? 4 : kv->dtype == CSD_DTYPE_BF16 ? 2 : 1;
    PagedPool p;
    p.k = (char *)kv->k + rows * kv->head_dim * esz;
    p.v = (char *)kv->v + rows * kv->head_dim * esz;
    p.ks = kv->dtype == CSD_DTYPE_FP8 ? kv->k_scale + rows : nullptr;
    p.vs = kv->dtype == CSD_DTYPE_FP8 ? kv->v_scale + rows : nullptr;
    p.table = kv->table;
    p.table_stride = kv->table_stride;
    p.n_pages = kv->n_pages;
    p.page_shift = ilog2(kv->page_rows);
    p.Hkv = kv->n_kv_heads;
    p.D = kv->head_dim;
    return p;
}

static bool row_stride_ok(const csd_paged_kv *kv, int heads, int64_t stride, const void *p) {
    return stride >= (int64_t)heads * kv->head_dim && stride % 8 == 0 && (uintptr_t)p % 16 == 0;
}

// calls f(dense type, pool type) with null pointers of the two types
template <typename F>
static void by_types(int32_t dense, int32_t pool, F f) {
    if (dense == CSD_DTYPE_FP32) {
        if (pool == CSD_DTYPE_FP32) f((float *)nullptr, (float *)nullptr);
        else if (pool == CSD_DTYPE_BF16) f((float *)nullptr, (bf16_t *)nullptr);
        else f((float *)nullptr, (uint8_t *)nullptr);
    } else {
        if (pool == CSD_DTYPE_FP32) f((bf16_t *)nullptr, (float *)nullptr);
        else if (pool == CSD_DTYPE_BF16) f((bf16_t *)nullptr, (bf16_t *)nullptr);
        else f((bf16_t *)nullptr, (uint8_t *)nullptr);
    }
}

// Launches f for the types of a move of rows: four heads per wave where there are waves enough to fill the chip all the same, else one.
template <typename F>
static int32_t move_rows(const csd_paged_kv *kv, int32_t dtype, int32_t rows, F f) {
    const int log_w = ilog2(kv->head_dim / 8), per_wave = 64 >> log_w;
    const long long row_blocks = ((long long)rows + per_wave - 1) / per_wave;
    const bool wide = row_blocks * kv->n_kv_heads >= 4 * 256 * 16;      // 16 waves per compute unit
    const int head_blocks = wide ? (kv->n_kv_heads + 3) / 4 : kv->n_kv_heads;
    const long long grid = (row_blocks * head_blocks + kPagedThreads / 64 - 1) / (kPagedThreads / 64);
    if (grid > 0xFFFFFF) return CSD_ESHAPE;                  // (work items of a launch are counted in 32 bits)
    by_types(dtype, kv->dtype, [&](auto *dense, auto *pool) {
        if (wide) f(dense, pool, std::integral_constant<int, 4>{}, (unsigned)grid, log_w, head_blocks);
        else f(dense, pool, std::integral_constant<int, 1>{}, (unsigned)grid, log_w, head_blocks);
    });
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}

extern "C" int32_t csd_paged_write(const csd_paged_kv *kv, int32_t layer, const int32_t *row_start, const int32_t *pos, int32_t B,
                                   int32_t rows, const void *k_rows, int64_t k_stride, const void *v_rows, int64_t v_stride,
                                   int32_t dtype, void *stream) {
    int32_t rc = check_rows(kv, layer, row_start, pos, B, rows, dtype);
    if (rc != CSD_OK) return rc;
    if (rows == 0) return CSD_OK;
    if (!k_rows || !v_rows) return CSD_ENULL;
    if (!row_stride_ok(kv, kv->n_kv_heads, k_stride, k_rows) || !row_stride_ok(kv, kv->n_kv_heads, v_stride, v_rows)) return CSD_EINVAL;
    const PagedPool p = csd_paged_layer(kv, layer);
    const PagedRows r{row_start, pos, B, rows};
    return move_rows(kv, dtype, rows, [&](auto *dense, auto *pool, auto u, unsigned grid, int log_w, int head_blocks) {
        using TR = std::remove_pointer_t<decltype(dense)>;
        using TP = std::remove_pointer_t<decltype(pool)>;
        hipLaunchKernelGGL((k_paged_write<TR, TP, decltype(u)::value>), dim3(grid), dim3(kPagedThreads), 0, (hipStream_t)stream, p, r, (const TR *)k_rows,
                           (long long)k_stride, (const TR *)v_rows, (long long)v_stride, log_w, head_blocks);
    });
}

extern "C" int32_t csd_paged_read(const csd_paged_kv *kv, int32_t layer, const int32_t *row_start, const int32_t *pos, int32_t B,
                                  int32_t rows, void *k_rows, int64_t k_stride, void *v_rows, int64_t v_stride, int32_t dtype,
                                  void *stream) {
    int32_t rc = check_rows(kv, layer, row_start, pos, B, rows, dtype);
    if (rc != CSD_OK) return rc;
    if (rows == 0) return CSD_OK;
    if (!k_rows || !v_rows) return CSD_ENULL;
    if (!row_stride_ok(kv, kv->n_kv_heads, k_stride, k_rows) || !row_stride_ok(kv, kv->n_kv_heads, v_stride, v_rows)) return CSD_EINVAL;
    const PagedPool p = csd_paged_layer(kv, layer);
    const PagedRows r{row_start, pos, B, rows};
    return move_rows(kv, dtype, rows, [&](auto *dense, auto *pool, auto u, unsigned grid, int log_w, int head_blocks) {
        using TR = std::remove_pointer_t<decltype(dense)>;
        using TP = std::remove_pointer_t<decltype(pool)>;
        hipLaunchKernelGGL((k_paged_read<TR, TP, decltype(u)::value>), dim3(grid), dim3(kPagedThreads), 0, (hipStream_t)stream, p, r, (TR *)k_rows,
                           (long long)k_stride, (TR *)v_rows, (long long)v_stride, log_w, head_blocks);
    });
}

extern "C" int32_t csd_paged_commit(const csd_paged_kv *kv, const int32_t *cache_len, const int32_t *path, const int32_t *n_accepted,
                                    int32_t B, int32_t m, void *stream) {
    const int32_t rc = check_pool(kv);
    if (rc != CSD_OK) return rc;
    if (!cache_len || !path || !n_accepted) return CSD_ENULL;
    if (B < 1 || m < 1) return CSD_EINVAL;
    if (m > 64 || B > 65535 || kv->n_layers > 65535) return CSD_ESHAPE;
    const PagedPool p = csd_paged_layer(kv, 0);
    const int units = 2 * kv->n_kv_heads * (kv->head_dim / 8);
    const dim3 grid((units + kPagedThreads - 1) / kPagedThreads, B, kv->n_layers);
    const auto kernel = kv->dtype == CSD_DTYPE_FP32 ? k_paged_commit<4> : kv->dtype == CSD_DTYPE_BF16 ? k_paged_commit<2> : k_paged_commit<1>;
    hipLaunchKernelGGL(kernel, grid, dim3(kPagedThreads), 0, (hipStream_t)stream, p, pool_rows(kv), cache_len, path, n_accepted, m);
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}

static int32_t attention(const csd_paged_kv *kv, int32_t layer, const int32_t *row_start, const int32_t *cache_len, const int32_t *parent, int32_t cross, int32_t B,
                         int32_t rows, int32_t max_rows, const void *q, int64_t q_stride, int32_t n_heads, int32_t dtype, float scale, void *out,
                         void *workspace, void *stream) {
    int32_t rc = check_rows(kv, layer, row_start, cache_len, B, rows, dtype);
    if (rc != CSD_OK) return rc;
    if (max_rows < 1 || n_heads < 1 || n_heads % kv->n_kv_heads || !(fabsf(scale) < INFINITY)) return CSD_EINVAL;
    const int32_t most = max_rows < rows ? max_rows : rows;
    if (n_heads > 65535 || (parent && most > 64)) return CSD_ESHAPE;
    if (rows == 0) return CSD_OK;
    if (!q || !out || (!workspace && csd_paged_few_types(kv->head_dim, kv->dtype, dtype))) return CSD_ENULL;
    if (!row_stride_ok(kv, n_heads, q_stride, q) || (uintptr_t)out % 16 || (uintptr_t)workspace % 256) return CSD_EINVAL;
    const PagedAttn a{csd_paged_layer(kv, layer), PagedRows{row_start, cache_len, B, rows}, parent, most,
                      n_heads / kv->n_kv_heads, q, (long long)q_stride, out, scale, workspace, cross};
    return csd_paged_attention_enqueue(a, kv->dtype, dtype, (hipStream_t)stream);
}

extern "C" int32_t csd_paged_attention(const csd_paged_kv *kv, int32_t layer, const int32_t *row_start, const int32_t *cache_len,
                                       const int32_t *parent, int32_t B, int32_t rows, int32_t max_rows, const void *q,
                                       int64_t q_stride, int32_t n_heads, int32_t dtype, float scale, void *out, void *workspace,
                                       void *stream) {
    return attention(kv, layer, row_start, cache_len, parent, 0, B, rows, max_rows, q, q_stride, n_heads, dtype, scale, out, workspace, stream);
}

extern "C" int32_t csd_paged_cross_attention(const csd_paged_kv *kv, int32_t layer, const int32_t *row_start, const int32_t *enc_len, int32_t B,
                                             int32_t rows, int32_t max_rows, const void *q, int64_t q_stride, int32_t n_heads, int32_t dtype,
                                             float scale, void *out, void *workspace, void *stream) {
    return attention(kv, layer, row_start, enc_len, nullptr, 1, B, rows, max_rows, q, q_stride, n_heads, dtype, scale, out, workspace, stream);
}
