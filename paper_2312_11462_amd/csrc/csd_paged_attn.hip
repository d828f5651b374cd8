// Attention of new rows over a paged KV cache.
#include "csd_paged.h"

// Any types and head sizes: one workgroup per (row, query head).  The four waves take 64 keys in turn, a key per lane for the scores;
// for the products with the values the lanes are W features (the power of two from D up, 64 at most) of 64 / W keys at a time, eight such steps
// requested together, the first eight along with the keys.  Running maximum, sum and output per wave are joined at the end.  Only keys
// that the row attends are looked at in the second half, so that nothing else reaches it.  All arithmetic is in fp32.  Small models' calls are bound by
// the chain rows -> page table -> keys and values (five rows of 4 heads of 16 over 32 cached keys, fp32: 10.1 -> 7.1 us with each of these
// asked for at once).
template <typename TQ, typename TP>
__global__ __launch_bounds__(256) void k_paged_attn_any(PagedAttn a, int log_w) {
    __shared__ float s_q[256], s_o[4][256], s_m[4], s_l[4], s_w[4][64];
    __shared__ size_t s_at[4][64];
    const int row = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PagedPool &p = a.p;
    const int D = p.D, kvh = head / a.group;
    const TQ *q = reinterpret_cast<const TQ *>(a.q) + (size_t)row * a.q_stride + (size_t)head * D;
    const float q_mine = tid < D ? to_f32<TQ>(q[tid]) : 0.f;
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
    // the row's ancestors in its block, one bit each
    unsigned long long above = ~0ull;
    if (a.parent) {
        above = 1ull << i;
        for (int x = i; x > 0;) {
            const int up = a.parent[s.start + x];
            x = up >= 0 && up < x ? up : 0;
            above |= 1ull << x;
        }
    }
    if (tid < D) s_q[tid] = q_mine;
    __syncthreads();
    constexpr float kLog2e = 1.44269504088896f;
    const int per_step = 64 >> log_w, key_in = lane >> log_w, feature = lane & ((1 << log_w) - 1);
    float m_run = -INFINITY, l_run = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    const int keys = min(s.t + i + 1, p.table_stride << p.page_shift);
    for (int key0 = wave * 64; key0 < keys; key0 += 256) {
        const int key = key0 + lane;
        int page = key < keys ? paged_page(p, b, key) : -1;
        if (a.parent && key >= s.t && !((above >> min(key - s.t, 63)) & 1ull)) page = -1;
        const size_t at = page >= 0 ? paged_row(p, page, kvh, key) : 0;
        const unsigned long long seen = __ballot(page >= 0);
        if (!seen) continue;
        s_at[wave][lane] = at;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        // values of steps st .. st + 7: element e of step j is feature 64 e + `feature` of key (st + j) * per_step + key_in
        const int steps = min(64, keys - key0 + per_step - 1) >> (6 - log_w);
        float v[8][4];
        auto values = [&](int st) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int x = (st + j) * per_step + key_in;
                const bool there = st + j < steps && x < 64 && ((seen >> (x & 63)) & 1ull);
                const TP *vp = reinterpret_cast<const TP *>(p.v) + s_at[wave][x & 63] * D;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    v[j][e] = 0.f;
                    if (there && (e == 0 || D > 64 * e) && 64 * e + feature < D) {
                        if constexpr (sizeof(TP) == 1) v[j][e] = __builtin_amdgcn_cvt_f32_fp8((int)vp[64 * e + feature], 0);
                        else v[j][e] = to_f32<TP>(vp[64 * e + feature]);
                    }
                }
            }
        };
        values(0);
        float v_scale = 1.f, score = -INFINITY;
        if (page >= 0) {
            const TP *kp = reinterpret_cast<const TP *>(p.k) + at * D;
            float k_scale = 1.f;
            if constexpr (sizeof(TP) == 1) {
                k_scale = pow2_of_byte(p.ks[at]);
                v_scale = pow2_of_byte(p.vs[at]);
            }
            float dot = 0.f;
#pragma unroll 4
            for (int c = 0; c < D; c += 8) {
                float x[8];
                load8<TP>(kp + c, x);
#pragma unroll
                for (int e = 0; e < 8; e++) dot = fmaf(x[e], s_q[c + e], dot);
            }
            score = dot * k_scale * a.scale;
        }
        const float m_new = fmaxf(m_run, wave_max(score)), m_ref = m_new == -INFINITY ? 0.f : m_new;
        const float w = page >= 0 ? exp2f((score - m_ref) * kLog2e) : 0.f, fade = exp2f((m_run - m_ref) * kLog2e);
        l_run = l_run * fade + wave_sum(w);
        m_run = m_new;
        s_w[wave][lane] = w * v_scale;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] *= fade;
        for (int st = 0; st < steps; st += 8) {
            if (st) values(st);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int x = (st + j) * per_step + key_in;
                if (st + j < steps && x < 64 && ((seen >> x) & 1ull)) {
                    const float f = s_w[wave][x];
#pragma unroll
                    for (int e = 0; e < 4; e++) o[e] = fmaf(f, v[j][e], o[e]);
                }
            }
        }
    }
    for (int x = 32; x >= 1 << log_w; x >>= 1)               // (the lanes that hold the same feature)
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] += __shfl_xor(o[e], x, 64);
    if (key_in == 0)
#pragma unroll
        for (int e = 0; e < 4; e++) s_o[wave][e * 64 + feature] = o[e];
    if (lane == 0) {
        s_m[wave] = m_run;
        s_l[wave] = l_run;
    }
    __syncthreads();
    if (tid >= D) return;
    float m_all = s_m[0];
    for (int w = 1; w < 4; w++) m_all = fmaxf(m_all, s_m[w]);
    if (m_all == -INFINITY) m_all = 0.f;
    float l = 0.f, x = 0.f;
    for (int w = 0; w < 4; w++) {
        const float f = exp2f((s_m[w] - m_all) * kLog2e);
        l += f * s_l[w];
        x += f * s_o[w][tid];
    }
    // nothing to attend: zeros (0 / 0 where there are keys but all scores are -inf, as the formula has it)
    bool any = l != 0.f;
    if (!any)
        for (int key = 0; key < keys && !any; key++)
            any = paged_page(p, b, key) >= 0 && (!a.parent || key < s.t || ((above >> min(key - s.t, 63)) & 1ull));
    TQ *out = reinterpret_cast<TQ *>(a.out) + ((size_t)row * p.Hkv * a.group + head) * D;
    out[tid] = from_f32<TQ>(any ? x / l : 0.f);
}

template <typename TQ, typename TP>
static void any_launch(const PagedAttn &a, hipStream_t st) {
    int log_w = 0;
    while (log_w < 6 && (1 << log_w) < a.p.D) log_w++;
    hipLaunchKernelGGL((k_paged_attn_any<TQ, TP>), dim3(a.r.rows, a.p.Hkv * a.group), dim3(256), 0, st, a, log_w);
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
