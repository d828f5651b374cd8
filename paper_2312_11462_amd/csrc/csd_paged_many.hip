// Attention of many rows (chunks of a prompt, large trees, many query heads per key-value head) over a paged KV cache: bf16 queries, heads of
// 64 or 128, bf16 or e4m3 pools.
//
// The products of the scores and the weights bound this.  A workgroup of four waves takes 128 rows (rows of a sequence times the query heads that
// share its keys) of one key-value head, 32 rows per wave, and goes through the keys in tiles of 64 that it stages in LDS as bf16, two tiles
// deep: while a tile is worked on, the next one's loads are in flight to registers, from where it is stored (e4m3: converted, with its
// scale, exactly) behind the work.  Two workgroups share a compute unit, so that one's matrix products run beside the other's exponentials.
// Products are transposed:
//   S^T = K q^T    A = K (32 keys x 16 features, one 16-byte read), B = q^T, in registers throughout
//   O^T = V^T P^T  A = V^T (32 features x 16 keys, by LDS's transposing reads), B = P^T: a lane's scores of 16 keys are, in
//                  order, keys 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 (h = lane / 32), and A's columns are read in that order
// so that the weights never move between lanes.  The weights enter as bf16 (half a step: 2^-8 of a weight, random in sign; the sum of the weights
// is kept in fp32): a second plane of them would be a third more matrix instructions, which bound this kernel.
// Rows of 16-byte pieces are stored with the piece index xored by the row, K and V in different ways, so that each kind of read
// spreads over all banks.
#include "csd_paged.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

static constexpr int kKeys = 64;                             // keys per tile

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float halves_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ void store_dev2(float *p, float a, float b) {
    const uint64_t x = ((uint64_t)__float_as_uint(b) << 32) | __float_as_uint(a);
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_dev2(const float *p) {
    const uint64_t x = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return float2{__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32))};
}

// 16-byte piece c of row `row` in a staged tile
template <int DH> __device__ __forceinline__ int k_piece(int row, int c) { return row * (DH / 8) + (c ^ (row & (DH / 8 - 1))); }
template <int DH> __device__ __forceinline__ int v_piece(int row, int c) {
    return row * (DH / 8) + (c ^ (DH == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2));
}

template <int DH, bool F8>
__global__ __launch_bounds__(256, 2) void k_paged_attn_many(PagedAttn a, int min_rows, int splits) {
    constexpr int ES = F8 ? 1 : 2, LPR = DH * ES / 16;       // lanes that load a row
    constexpr int RPP = 256 / LPR, NP = kKeys / RPP;         // rows per pass of the workgroup, passes per tile
    constexpr int PIECES = kKeys * DH / 8;                   // 16-byte pieces of a staged tile
    constexpr int ST = DH / 16, DT = DH / 32, PS = DH + 2, BM = CSD_PAGED_MANY_ROWS;
    __shared__ u32x4 s_k[2][PIECES], s_v[2][PIECES];
    __shared__ int s_odd, s_last;
    const PagedPool &p = a.p;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, h = lane >> 5;
    const int cap = p.table_stride << p.page_shift;

    // ---- which rows: key-value heads follow one another (workgroups of a die, every eighth, read the same keys), then the parts of an item,
    // then the row tiles, the late ones with the most keys first
    const int kvh = blockIdx.x % p.Hkv, part_no = (blockIdx.x / p.Hkv) % splits, tile_no = blockIdx.x / p.Hkv / splits;
    int b = -1, rt = 0, total = 0, n_tiles = 0;
    PagedSeq seq{0, 0, 0};
    for (int pass = 0; pass < 2; pass++) {                   // count the tiles of all sequences, then find this one
        int before = 0;
        const int want = pass ? total - 1 - tile_no : 0;
        if (pass && want < 0) return;
        for (int b0 = 0; b0 < a.r.B; b0 += 64) {
            PagedSeq s{0, 0, 0};
            int n = 0;
            if (b0 + lane < a.r.B) {
                s = paged_seq(a.r, b0 + lane);
                s.m = min(s.m, a.max_rows);
                const int rows = s.m * a.group;
                n = rows > min_rows ? (rows + BM - 1) / BM : 0;
            }
            int incl = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int x = __shfl_up(incl, o, 64);
                if (lane >= o) incl += x;
            }
            if (pass) {
                const unsigned long long past = __ballot(before + incl > want);
                if (past) {
                    const int j = __ffsll((long long)past) - 1;
                    b = b0 + j;
                    n_tiles = __builtin_amdgcn_readlane(n, j);
                    rt = want - (before + __builtin_amdgcn_readlane(incl, j) - n_tiles);
                    seq = PagedSeq{__builtin_amdgcn_readlane(s.start, j), __builtin_amdgcn_readlane(s.m, j), __builtin_amdgcn_readlane(s.t, j)};
                    break;
                }
            }
            before += __builtin_amdgcn_readlane(incl, 63);
        }
        total = before;
    }
    if (b < 0) return;
    const int rows = min(seq.m * a.group - rt * BM, BM);     // of this item
    const int i_first = rt * BM / a.group, i_last = (rt * BM + rows - 1) / a.group;
    const int len = min(seq.t + i_last + 1, cap);            // keys that some row attends
    const int n_kt = (len + kKeys - 1) / kKeys;
    // an item's keys in equal parts of at least CSD_PAGED_MANY_SHARE tiles
    const int parts = min(splits, max(1, n_kt / CSD_PAGED_MANY_SHARE));
    if (part_no >= parts) return;
    const int kt0 = (int)((long long)n_kt * part_no / parts), kt1 = (int)((long long)n_kt * (part_no + 1) / parts);

    // ---- this lane's row
    const int r = rt * BM + wave * 32 + col, i = r / a.group, hq = r - i * a.group;
    const bool live = wave * 32 + col < rows;
    const int limit = seq.t + i;                             // last position it attends
    unsigned long long above = 0;
    if (a.parent) {                                          // ancestors of block row `lane`, by doubling the step up; then those of this lane's row
        unsigned long long anc = 1ull << lane;
        int up = 0;
        if (lane < seq.m && lane > 0) {
            up = a.parent[seq.start + lane];
            if (up < 0 || up >= lane) up = 0;
        }
        anc |= 1ull << up;
#pragma unroll
        for (int k = 0; k < 6; k++) {
            const unsigned lo = __shfl((unsigned)anc, up, 64), hi = __shfl((unsigned)(anc >> 32), up, 64);
            anc |= ((unsigned long long)hi << 32) | lo;
            up = __shfl(up, up, 64);
        }
        const int src = min(i, 63);
        above = ((unsigned long long)(unsigned)__shfl((unsigned)(anc >> 32), src, 64) << 32) | (unsigned)__shfl((unsigned)anc, src, 64);
    }
    u32x4 qf[ST];
    {
        const bf16_t *q = reinterpret_cast<const bf16_t *>(a.q) + (size_t)(seq.start + i) * a.q_stride + (size_t)(kvh * a.group + hq) * DH + 8 * h;
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;      // a negative scale turns the queries around: the maximum below needs scale >= 0
#pragma unroll
        for (int s = 0; s < ST; s++) {
            qf[s] = u32x4{0u, 0u, 0u, 0u};
            if (live) qf[s] = *reinterpret_cast<const u32x4 *>(q + 16 * s);
#pragma unroll
            for (int w = 0; w < 4; w++) qf[s][w] ^= flip;
        }
    }
    // scores in units of log2 (at least 1e-30: a masked score of -inf has to stay one)
    const float scale = fmaxf(fabsf(a.scale) * 1.44269504088896f, 1e-30f);
    f32x16 acc[DT];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[d][e] = 0.f;

    // ---- staging: in pass x a wave's rows lie in one group of 16 keys, so in one page
    const int row_in = tid / LPR, c_in = tid % LPR;
    u32x4 kr[NP], vr[NP];
    uint8_t ksr[NP], vsr[NP];
    auto group_of = [&](int x) { return (x * RPP + wave * (64 / LPR)) >> 4; };
    auto load = [&](int kt) {
#pragma unroll
        for (int x = 0; x < NP; x++) {
            const int page = max(paged_page(p, b, kt * kKeys + 16 * group_of(x)), 0);     // (no page: rows of page 0, which the masks leave out)
            const size_t row = paged_row(p, page, kvh, kt * kKeys + x * RPP + row_in);
            kr[x] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(p.k) + row * (DH * ES) + c_in * 16);
            vr[x] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(p.v) + row * (DH * ES) + c_in * 16);
            if constexpr (F8) {
                ksr[x] = p.ks[row];
                vsr[x] = p.vs[row];
            }
        }
    };
    auto here_mask = [&](int kt) {                           // bit g: keys 16 g .. 16 g + 15 of the tile have a page
        unsigned m = 0;
#pragma unroll
        for (int g = 0; g < 4; g++) m |= (unsigned)(paged_page(p, b, kt * kKeys + 16 * g) >= 0) << g;
        return (unsigned)__builtin_amdgcn_readfirstlane((int)m);
    };
    auto stage = [&](int kt, int buf, unsigned here) {
        const bool edge = kt * kKeys + kKeys > seq.t || here != 0xFu;     // rows of the block, or places without a row, among the keys
#pragma unroll
        for (int x = 0; x < NP; x++) {
            const int row = x * RPP + row_in;
            u32x4 vv[F8 ? 2 : 1];
            if constexpr (F8) {
                const float fk = pow2_of_byte(ksr[x]), fv = pow2_of_byte(vsr[x]);
#pragma unroll
                for (int w = 0; w < 2; w++) {
                    u32x4 kk;
#pragma unroll
                    for (int y = 0; y < 2; y++) {
                        kk[2 * y] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kr[x][2 * w + y], fk, false));
                        kk[2 * y + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kr[x][2 * w + y], fk, true));
                        vv[w][2 * y] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vr[x][2 * w + y], fv, false));
                        vv[w][2 * y + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vr[x][2 * w + y], fv, true));
                    }
                    s_k[buf][k_piece<DH>(row, 2 * c_in + w)] = kk;
                }
            } else {
                s_k[buf][k_piece<DH>(row, c_in)] = kr[x];
                vv[0] = vr[x];
            }
            if (edge) {
                // values that no row attends are taken out, and those that are not finite (see odd_halves)
                bool odd = false;
                const bool out = kt * kKeys + row >= len || !((here >> group_of(x)) & 1u);
#pragma unroll
                for (int w = 0; w < (F8 ? 2 : 1); w++)
#pragma unroll
                    for (int y = 0; y < 4; y++) {
                        if (out) vv[w][y] = 0u;
                        const uint32_t o = odd_halves(vv[w][y]);
                        odd |= o != 0u;
                        vv[w][y] &= ~o;
                    }
                if (odd) s_odd = 1;
            }
#pragma unroll
            for (int w = 0; w < (F8 ? 2 : 1); w++) s_v[buf][v_piece<DH>(row, (F8 ? 2 : 1) * c_in + w)] = vv[w];
        }
    };
    // V^T operand: features 32 d .. 32 d + 31 of keys 16 u .. 16 u + 15, in the order of the weights
    const int l16 = lane & 15;
    auto v_operand = [&](int buf, int d, int u) {
        uint64_t w[2];
#pragma unroll
        for (int y = 0; y < 2; y++) {
            const int row = 16 * u + 8 * y + 4 * h + (l16 >> 2), piece = 4 * d + 2 * ((lane >> 4) & 1) + ((l16 >> 1) & 1);
            char *at = reinterpret_cast<char *>(&s_v[buf][v_piece<DH>(row, piece)]) + 8 * (l16 & 1);
            w[y] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at));
        }
        return u32x4{(uint32_t)w[0], (uint32_t)(w[0] >> 32), (uint32_t)w[1], (uint32_t)(w[1] >> 32)};
    };

    if (tid == 0) s_odd = 0;
    load(kt0);
    unsigned here = here_mask(kt0);
    __syncthreads();
    stage(kt0, 0, here);
    __syncthreads();
    const int wave_first = seq.t + (rt * BM + wave * 32) / a.group;      // last position that the wave's first row attends
    const bool wave_live = wave * 32 < rows;
#pragma unroll 1
    for (int kt = kt0; kt < kt1; kt++) {
        const int buf = (kt - kt0) & 1, key0 = kt * kKeys;
        const bool more = kt + 1 < kt1;
        unsigned here_next = 0xFu;
        if (more) {
            load(kt + 1);
            here_next = here_mask(kt + 1);
        }
        if (wave_live) {
            f32x16 st[2];
#pragma unroll
            for (int T2 = 0; T2 < 2; T2++) {
#pragma unroll
                for (int e = 0; e < 16; e++) st[T2][e] = 0.f;
#pragma unroll
                for (int s = 0; s < ST; s++) st[T2] = mfma32(s_k[buf][k_piece<DH>(32 * T2 + col, 2 * s + h)], qf[s], st[T2]);
            }
            // element e of half T2 is key 32 T2 + 8 (e / 4) + 4 h + e % 4
            uint32_t sees = ~0u;
            const bool whole = (a.parent ? key0 + kKeys <= seq.t : key0 + kKeys - 1 <= wave_first) && key0 + kKeys <= len && here == 0xFu;
            if (!whole) {
                const int n = min(limit, len - 1) - key0;    // attended: keys 0 .. n of the tile
                unsigned long long m = n >= 63 ? ~0ull : n < 0 ? 0ull : (2ull << n) - 1;
#pragma unroll
                for (int g = 0; g < 4; g++)
                    if (!((here >> g) & 1u)) m &= ~(0xFFFFull << (16 * g));
                if (a.parent) {
                    const int d = key0 - seq.t;              // rows of the block lie at d .. of `above`; keys before them are cached
                    m &= d >= 0 ? (d < 64 ? above >> d : 0ull) : -d >= 64 ? ~0ull : (above << -d) | ((1ull << -d) - 1);
                }
                m >>= 4 * h;
                sees = 0;
#pragma unroll
                for (int q = 0; q < 8; q++) sees |= (uint32_t)((m >> (8 * q)) & 0xFull) << (4 * q);
#pragma unroll
                for (int e = 0; e < 32; e++)
                    if (!((sees >> e) & 1u)) st[e >> 4][e & 15] = -INFINITY;
            }
            float top = st[0][0];
#pragma unroll
            for (int e = 1; e < 32; e++) top = fmaxf(top, st[e >> 4][e & 15]);
            top = halves_max(sees ? fmaxf(top * scale, -3.0e38f) : -INFINITY);   // -inf: nothing to attend yet (a score of -inf is something)
            // weights up to 2^8 are as good as weights up to 1: the outputs are rescaled only when the maximum has moved by more
            if (__any(top > m_run + 8.f)) {
                const float m_new = fmaxf(m_run, top), fade = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
                l_run *= fade;
#pragma unroll
                for (int d = 0; d < DT; d++) acc[d] *= fade;
                m_run = m_new;
            }
            const float ref = m_run == -INFINITY ? 0.f : m_run;
            u32x4 pw[4];                                     // weights of keys 16 u .. 16 u + 15
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float w0 = __builtin_amdgcn_exp2f(fmaf(st[e >> 4][e & 15], scale, -ref)), w1 = __builtin_amdgcn_exp2f(fmaf(st[e >> 4][(e + 1) & 15], scale, -ref));
                l_run += w0;
                l_run += w1;
                pw[e >> 3][(e & 7) >> 1] = pack_bf16x2(w0, w1);
            }
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int u = 0; u < 4; u++) acc[d] = mfma32(v_operand(buf, d, u), pw[u], acc[d]);
        }
        if (more) {
            stage(kt + 1, buf ^ 1, here_next);               // (that buffer was last read a turn ago)
            __syncthreads();
            here = here_next;
        }
    }

    if (s_odd) {                                             // (uniform; the last tile was staged in front of a barrier)
        for (int kt = kt0; kt < kt1; kt++) {
            const unsigned m = here_mask(kt);
            if (kt * kKeys + kKeys <= seq.t && m == 0xFu) continue;
            for (int key = kt * kKeys; key < min(kt * kKeys + kKeys, len); key++) {
                const int page = paged_page(p, b, key);
                if (page < 0) continue;
                const bool attends = live && key <= limit && (!a.parent || key < seq.t || ((above >> min(key - seq.t, 63)) & 1ull));
                const char *row = reinterpret_cast<const char *>(p.v) + paged_row(p, page, kvh, key) * (DH * ES);
#pragma unroll
                for (int d = 0; d < DT; d++)
#pragma unroll
                    for (int e = 0; e < 16; e++) acc[d][e] += odd_value<F8>(row, 32 * d + 8 * (e / 4) + 4 * h + e % 4, attends);
            }
        }
    }

    // ---- results: element e of acc[d] is feature 32 d + 8 (e / 4) + 4 h + e % 4 of the lane's row
    l_run = halves_sum(l_run);
    const size_t out_row = ((size_t)(seq.start + i) * p.Hkv + kvh) * a.group + hq;
    if (parts == 1) {
        if (live) {
            const float inv = 1.f / l_run;
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    u32x2 o = u32x2{pack_bf16x2(acc[d][4 * y] * inv, acc[d][4 * y + 1] * inv), pack_bf16x2(acc[d][4 * y + 2] * inv, acc[d][4 * y + 3] * inv)};
                    if (m_run == -INFINITY) o = u32x2{0u, 0u};
                    *reinterpret_cast<u32x2 *>(reinterpret_cast<bf16_t *>(a.out) + out_row * DH + 32 * d + 8 * y + 4 * h) = o;
                }
        }
        return;
    }
    const int item = tile_no * p.Hkv + kvh;
    float *part = reinterpret_cast<float *>(reinterpret_cast<char *>(a.ws) + CSD_PAGED_COUNTER_BYTES) + (size_t)item * splits * BM * PS;
    if (live) {
        float *mine = part + ((size_t)part_no * BM + wave * 32 + col) * PS;
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
            for (int y = 0; y < 4; y++) {
                store_dev2(mine + 32 * d + 8 * y + 4 * h, acc[d][4 * y], acc[d][4 * y + 1]);
                store_dev2(mine + 32 * d + 8 * y + 4 * h + 2, acc[d][4 * y + 2], acc[d][4 * y + 3]);
            }
        if (h == 0) store_dev2(mine + DH, m_run, l_run);
    }
    // the stores above are acknowledged before the counter moves; whoever arrives last joins the parts, in their order
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0)
    __syncthreads();
    unsigned *count = reinterpret_cast<unsigned *>(a.ws) + item;
    if (tid == 0) s_last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(parts - 1);
    __syncthreads();
    if (!s_last) return;
    float *weight = reinterpret_cast<float *>(&s_k[0][0]);   // [parts][BM], then the rows' maxima and sums
    float *sums = weight + CSD_PAGED_MANY_PARTS * BM;
    if (tid < rows) {
        float m = -INFINITY, l = 0.f;
        float2 ml[CSD_PAGED_MANY_PARTS];
#pragma unroll
        for (int k = 0; k < CSD_PAGED_MANY_PARTS; k++) ml[k] = k < parts ? load_dev2(part + ((size_t)k * BM + tid) * PS + DH) : float2{-INFINITY, 0.f};
#pragma unroll
        for (int k = 0; k < CSD_PAGED_MANY_PARTS; k++) m = fmaxf(m, ml[k].x);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int k = 0; k < CSD_PAGED_MANY_PARTS; k++)
            if (k < parts) {
                const float f = __builtin_amdgcn_exp2f(ml[k].x - ref);
                l += f * ml[k].y;
                weight[k * BM + tid] = f;
            }
        sums[2 * tid] = m;
        sums[2 * tid + 1] = l;
    }
    __syncthreads();
    for (int x = tid; x < rows * (DH / 2); x += 256) {
        const int rr = x / (DH / 2), c = 2 * (x % (DH / 2));
        float o0 = 0.f, o1 = 0.f;
        float2 v[CSD_PAGED_MANY_PARTS];
#pragma unroll
        for (int k = 0; k < CSD_PAGED_MANY_PARTS; k++) v[k] = load_dev2(part + ((size_t)min(k, parts - 1) * BM + rr) * PS + c);
#pragma unroll
        for (int k = 0; k < CSD_PAGED_MANY_PARTS; k++)
            if (k < parts) {
                const float f = weight[k * BM + rr];
                o0 += f * v[k].x;
                o1 += f * v[k].y;
            }
        const int ro = rt * BM + rr, io = ro / a.group, ho = ro - io * a.group;
        const float inv = 1.f / sums[2 * rr + 1];
        uint32_t *out = reinterpret_cast<uint32_t *>(a.out) + (((size_t)(seq.start + io) * p.Hkv + kvh) * a.group + ho) * (DH / 2);
        out[c / 2] = sums[2 * rr] == -INFINITY ? 0u : pack_bf16x2(o0 * inv, o1 * inv);
    }
    if (tid == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);     // ready for the next launch
}

// min_rows: sequences of so many rows or fewer are another kernel's.
void csd_paged_many_enqueue(const PagedAttn &a, int min_rows, int32_t pool_dtype, hipStream_t st) {
    // row tiles at most: full ones, and a last one per sequence
    const long long tiles = (long long)a.r.rows * a.group / CSD_PAGED_MANY_ROWS + a.r.B, items = tiles * a.p.Hkv;
    // few items: their keys are split, as far as the chip (two workgroups per compute unit) and the workspace have room
    int splits = 1;
    while (splits * 2 <= CSD_PAGED_MANY_PARTS && items * splits * 2 <= CSD_PAGED_MANY_SLOTS) splits *= 2;
    const dim3 grid((unsigned)(items * splits));
    if (a.p.D == 128) {
        if (pool_dtype == CSD_DTYPE_FP8) hipLaunchKernelGGL((k_paged_attn_many<128, true>), grid, dim3(256), 0, st, a, min_rows, splits);
        else hipLaunchKernelGGL((k_paged_attn_many<128, false>), grid, dim3(256), 0, st, a, min_rows, splits);
    } else {
        if (pool_dtype == CSD_DTYPE_FP8) hipLaunchKernelGGL((k_paged_attn_many<64, true>), grid, dim3(256), 0, st, a, min_rows, splits);
        else hipLaunchKernelGGL((k_paged_attn_many<64, false>), grid, dim3(256), 0, st, a, min_rows, splits);
    }
}
