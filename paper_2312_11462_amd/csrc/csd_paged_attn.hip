// Attention of new rows over a paged KV cache.
#include "csd_paged.h"

// Four consecutive elements of a pool's row as they are in memory.
template <typename T> struct Raw4 {
    uint32_t w[sizeof(T)];
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<u32x4 *>(w) = *reinterpret_cast<const u32x4 *>(p);
        else if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2 *>(w) = *reinterpret_cast<const u32x2 *>(p);
        else w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
    __device__ __forceinline__ void get(float (&x)[4]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = __uint_as_float(w[e]);
        } else if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        } else {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], true);
            x[0] = lo[0];
            x[1] = lo[1];
            x[2] = hi[0];
            x[3] = hi[1];
        }
    }
};

// sum over the 2^log_w neighbouring lanes, in each of them
template <int CTRL>
__device__ __forceinline__ float add_dpp(float a) {
    return a + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(a), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lanes_sum(float a, int log_w) {
    if (log_w > 0) a = add_dpp<0xB1>(a);                     // lane ^ 1
    if (log_w > 1) a = add_dpp<0x4E>(a);                     // lane ^ 2
    if (log_w > 2) a = add_dpp<0x141>(a);                    // 7 - lane, of eight
    if (log_w > 3) a = add_dpp<0x140>(a);                    // 15 - lane, of sixteen
    if (log_w > 4) a += __shfl_xor(a, 16, 64);
    if (log_w > 5) a += __shfl_xor(a, 32, 64);
    return a;
}

// Any types and head sizes: one workgroup per (row, query head).  Its waves take 64 keys in turn.  For the products the lanes are W = 2^log_w pieces of four
// features (the power of two from D / 4 up) of 64 / W keys at a time, eight such steps of keys and the first eight of values requested at once; for the
// softmax a lane is a key.  Running maximum, sum and output per wave are joined at the end.  Only keys that the row attends are looked at.  All
// arithmetic is in fp32.  Small models' calls are bound by the chain rows -> page table -> keys and values: so as many waves as the page table has
// room for 64 keys each, four or eight.  (fp32: twelve rows of 4 heads of 64 over 761 keys 18 us, a tree of 41 rows over 445 11; with a lane per key in the scores and a
// feature per lane behind them 63 and 38.  Five rows of 4 heads of 16 over 32 keys 7.4.)
static constexpr int kAnyWaves = 8;

template <typename TQ, typename TP, bool CROSS>
__global__ __launch_bounds__(64 * kAnyWaves) void k_paged_attn_any(PagedAttnOf<CROSS> a, int log_w) {
    __shared__ float s_o[kAnyWaves][256], s_m[kAnyWaves], s_l[kAnyWaves], s_w[kAnyWaves][64];
    __shared__ size_t s_at[kAnyWaves][64];
    __shared__ bool s_any[kAnyWaves];                        // the wave has met a key that the row attends
    const int row = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int waves = blockDim.x >> 6;
    const PagedPool &p = a.p;
    const int D = p.D, kvh = head / a.group;
    const int per_step = 64 >> log_w, key_in = lane >> log_w, c = 4 * (lane & ((1 << log_w) - 1));
    float q[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < D) {
        const TQ *qp = reinterpret_cast<const TQ *>(a.q) + (size_t)row * a.q_stride + (size_t)head * D + c;
        Raw4<TQ> raw;
        raw.load(qp);
        raw.get(q);
    }
    // ---- the row's sequence
    PagedSeq s{0, 0, 0};
    int b = -1;
    for (int b0 = 0; b0 < a.r.B; b0 += 64) {
        const bool there = b0 + lane < a.r.B;
        PagedSeq mine{0, 0, 0};
        int end = 0x7FFFFFFF;
        if (there) {
            mine = paged_seq(a.r, b0 + lane);
            end = a.r.row_start[b0 + lane + 1];
        }
        const int n = __popcll(__ballot(end <= row));
        if (n < 64) {
            b = b0 + n;
            s = PagedSeq{__builtin_amdgcn_readlane(mine.start, n), __builtin_amdgcn_readlane(mine.m, n), __builtin_amdgcn_readlane(mine.t, n)};
            break;
        }
    }
    if (b < 0 || b >= a.r.B) return;
    const int i = row - s.start;
    if (i < 0 || i >= min(s.m, a.max_rows)) return;
    const unsigned long long above = a.parent ? lane_of(paged_ancestors(a.parent, s, lane), i) : ~0ull;      // (trees: max_rows <= 64)
    constexpr float kLog2e = 1.44269504088896f;
    float m_run = -INFINITY, l_run = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    bool any = false;
    const int keys = a.keys(s.t, i);
    for (int key0 = wave * 64; key0 < keys; key0 += 64 * waves) {
        const int key = key0 + lane;
        int page = key < keys ? paged_page(p, b, key) : -1;
        if (a.parent && key >= s.t && !((above >> min(key - s.t, 63)) & 1ull)) page = -1;
        const size_t at = page >= 0 ? paged_row(p, page, kvh, key) : 0;
        const unsigned long long seen = __ballot(page >= 0);
        if (!seen) continue;
        any = true;
        s_at[wave][lane] = at;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        // step j: keys j * per_step + key_in of the 64
        const int steps = (min(64, keys - key0) + per_step - 1) >> (6 - log_w);
        auto has = [&](int j) { return j < steps && ((seen >> (j * per_step + key_in)) & 1ull); };
        Raw4<TP> k[8], v[8];
        auto request = [&](Raw4<TP> (&r)[8], const void *pool, int first) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                r[j] = Raw4<TP>{};
                if (has(first + j) && c < D) r[j].load(reinterpret_cast<const TP *>(pool) + s_at[wave][(first + j) * per_step + key_in] * D + c);
            }
        };
        request(k, p.k, 0);
        request(v, p.v, 0);
        float k_scale = 1.f, v_scale = 1.f;
        if constexpr (sizeof(TP) == 1)
            if (page >= 0) {
                k_scale = pow2_of_byte(p.ks[at]);
                v_scale = pow2_of_byte(p.vs[at]);
            }
        for (int first = 0; first < steps; first += 8) {
            if (first) request(k, p.k, first);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                float x[4];
                k[j].get(x);
                const float dot = lanes_sum(fmaf(x[0], q[0], fmaf(x[1], q[1], fmaf(x[2], q[2], x[3] * q[3]))), log_w);
                if (c == 0 && has(first + j)) s_w[wave][(first + j) * per_step + key_in] = dot;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const float score = page >= 0 ? s_w[wave][lane] * k_scale * a.scale : -INFINITY;
        const float m_new = fmaxf(m_run, wave_max(score)), m_ref = m_new == -INFINITY ? 0.f : m_new;
        const float w = page >= 0 ? exp2f((score - m_ref) * kLog2e) : 0.f, fade = exp2f((m_run - m_ref) * kLog2e);
        l_run = l_run * fade + wave_sum(w);
        m_run = m_new;
        s_w[wave][lane] = w * v_scale;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] *= fade;
        for (int first = 0; first < steps; first += 8) {
            if (first) request(v, p.v, first);
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (has(first + j)) {
                    const float f = s_w[wave][(first + j) * per_step + key_in];
                    float x[4];
                    v[j].get(x);
#pragma unroll
                    for (int e = 0; e < 4; e++) o[e] = fmaf(f, x[e], o[e]);
                }
        }
    }
    for (int x = 32; x >= 1 << log_w; x >>= 1)               // (the lanes that hold the same features)
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] += __shfl_xor(o[e], x, 64);
    if (key_in == 0)
#pragma unroll
        for (int e = 0; e < 4; e++) s_o[wave][c + e] = o[e];
    if (lane == 0) {
        s_m[wave] = m_run;
        s_l[wave] = l_run;
        s_any[wave] = any;
    }
    __syncthreads();
    if (tid >= D) return;
    float m_all = s_m[0];
    for (int w = 1; w < waves; w++) m_all = fmaxf(m_all, s_m[w]);
    if (m_all == -INFINITY) m_all = 0.f;
    float l = 0.f, x = 0.f;
    any = false;
    for (int w = 0; w < waves; w++) {
        const float f = exp2f((s_m[w] - m_all) * kLog2e);
        l += f * s_l[w];
        x += f * s_o[w][tid];
        any |= s_any[w];
    }
    // nothing to attend: zeros (0 / 0 where there are keys but all scores are -inf, as the formula has it)
    TQ *out = reinterpret_cast<TQ *>(a.out) + ((size_t)row * p.Hkv * a.group + head) * D;
    out[tid] = from_f32<TQ>(any ? x / l : 0.f);
}

template <typename TQ, typename TP>
static void any_launch(const PagedAttn &a, hipStream_t st) {
    int log_w = 0;
    while (4 << log_w < a.p.D) log_w++;
    const int keys = a.p.table_stride << a.p.page_shift, waves = keys > 4 * 64 ? 8 : 4;
    csd_paged_by_cross(a, [&](auto x) {
        constexpr bool CROSS = std::is_same<decltype(x), PagedAttnOf<true>>::value;
        hipLaunchKernelGGL((k_paged_attn_any<TQ, TP, CROSS>), dim3(a.r.rows, a.p.Hkv * a.group), dim3(64 * waves), 0, st, x, log_w);
    });
}

int32_t csd_paged_attention_enqueue(const PagedAttn &a, int32_t pool_dtype, int32_t q_dtype, hipStream_t st) {
    if (csd_paged_few_fits(a, pool_dtype, q_dtype)) {
        // Sequences of few rows are bound by the cache's bytes, others by the products.  A batch that may hold both takes both kernels, and
        // the first one only for up to 16 rows (single tokens, mostly), where it has no second row tile to carry.
        const long long rows = (long long)a.max_rows * a.group;
        const bool many = rows > CSD_PAGED_FEW_ROWS;
        // (one sequence, or as many rows as B sequences of max_rows have: no sequence needs the other kernel)
        const bool few = !many || (a.r.B > 1 && a.r.rows < (long long)a.r.B * a.max_rows);
        if (many) csd_paged_many_enqueue(a, few ? 16 : 0, pool_dtype, st);
        if (few) csd_paged_few_enqueue(a, (int)(many ? 16 : rows), pool_dtype, st);
        CSD_LAUNCH_CHECK();
        return CSD_OK;
    }
    if (q_dtype == CSD_DTYPE_FP32) {
        if (pool_dtype == CSD_DTYPE_FP32) any_launch<float, float>(a, st);
        else if (pool_dtype == CSD_DTYPE_BF16) any_launch<float, bf16_t>(a, st);
        else any_launch<float, uint8_t>(a, st);
    } else {
        if (pool_dtype == CSD_DTYPE_FP32) any_launch<bf16_t, float>(a, st);
        else if (pool_dtype == CSD_DTYPE_BF16) any_launch<bf16_t, bf16_t>(a, st);
        else any_launch<bf16_t, uint8_t>(a, st);
    }
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}
