// Attention of few rows (a token, a drafted block, a small tree) over a paged KV cache: bf16 queries, heads of 64 or 128, bf16 or e4m3 pools,
// up to 32 rows per key-value head (rows of a sequence times the query heads that share its keys).
//
// Every cached row is read once and takes part in few products, so the cache's bytes bound this: what matters is that all compute units
// read all the time.  The tiles of 32 keys of all sequences and key-value heads are counted through, and every workgroup takes an
// equal, contiguous share of them (sequences of very different length share the chip evenly, and nobody outside the device has to know the
// lengths).  An item (sequence, key-value head) counts CSD_PAGED_FEW_COST tiles more than it has, for the trips to memory before its first key and behind
// its last (5 rows of 16 ragged sequences, 8 heads of 128, e4m3: 112 us without, 104 for 4 tiles, 102 for 8 and for 12).  A share ends inside an
// item in general; the parts of such an item are joined by the workgroup that finishes last.
//
// The four waves of a workgroup take the tiles of its share in turn.  Both
// products are transposed so that nothing passes through LDS:
//   S^T = K q^T    A = K (16 keys x 32 features), B = q^T.  Key of A-row r of tile half T: 8 (r / 4) + 4 T + r % 4, so that lane group g
//                  (lane / 16) ends up with the scores of keys 8 g .. 8 g + 7 of the tile, all in one page
//   O^T = V^T P^T  A = V^T (16 features x 32 keys), B = P^T, which those scores are already.  A lane loads DH / 16 consecutive features of
//                  eight keys (a row of V is read by 16 neighbouring lanes) and transposes them in registers by byte permutations; A-row i of
//                  product j is then feature DH / 16 * i + j.
// e4m3 keys and values become bf16 without loss; the keys' scales multiply the scores, the values' scales the weights (powers of
// two: exact).  The weights enter the second product as two bf16 planes (w = hi + lo, 16 bits): the matrix cores have time to spare (20 rows of 16 ragged
// sequences, 8 heads of 128: bf16 100 us with either, e4m3 100 with one plane and 101 to 103 with two; heads of 64, e4m3: 61 and 67).
#include "csd_paged.h"

static constexpr int kFewPages = 1024;      // entries of the page table held in LDS at a time

template <int DH, bool F8>
struct FewTile {
    static constexpr int F = DH / 16;                        // features per lane of a V row
    static constexpr int VW = F8 ? F / 4 : F / 2;            // dwords that hold them
    static constexpr int KV = F8 ? DH / 64 : DH / 32;        // 16-byte pieces of a K row per lane
    u32x4 k[2][KV];
    uint32_t v[8][VW];
    u32x2 ks, vs;                                            // e4m3: scale bytes of the lane group's eight keys
    bool here;                                               // the group's keys have a page
};

template <int VW>
__device__ __forceinline__ void load_words(const void *p, uint32_t (&w)[VW]) {
    if constexpr (VW == 4) {
        const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = x[i];
    } else if constexpr (VW == 2) {
        const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(p));
        w[0] = x[0];
        w[1] = x[1];
    } else {
        w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(p));
    }
}

// two e4m3 codes (the low or the high half of w) times `scale`, a power of two, as bf16, exact
template <bool HI>
__device__ __forceinline__ uint32_t bf16x2_of_fp8(uint32_t w, float scale = 1.0f) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// Weights are multiplied by their values' scales, 2^-126 to 2^120, before they are rounded to bf16.  So that products with the smallest scales do not end below bf16's
// normal values, the weights get 2^kUp more (2^127 at most) and the codes as much less (20 rows over e4m3
// caches: heads of 128 as before, heads of 64 66.5 -> 67.3 us).
static constexpr int kUp = 7;

// V^T operands of features y .. y + 3 (of the lane's DH / 16) from the eight keys' words: dword i holds keys 2 i, 2 i + 1
template <int DH, bool F8>
__device__ __forceinline__ void v_operands(const uint32_t (&v)[8][FewTile<DH, F8>::VW], u32x4 (&f)[4], int y) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t *a = v[2 * i], *b = v[2 * i + 1];
        if constexpr (F8) {
            const int w = y / 4;
            const uint32_t lo = __builtin_amdgcn_perm(b[w], a[w], 0x05010400u), hi = __builtin_amdgcn_perm(b[w], a[w], 0x07030602u);
            constexpr float down = 1.0f / (1 << kUp);
            f[0][i] = bf16x2_of_fp8<false>(lo, down);
            f[1][i] = bf16x2_of_fp8<true>(lo, down);
            f[2][i] = bf16x2_of_fp8<false>(hi, down);
            f[3][i] = bf16x2_of_fp8<true>(hi, down);
        } else {
#pragma unroll
            for (int w = 0; w < 2; w++) {
                f[2 * w][i] = __builtin_amdgcn_perm(b[y / 2 + w], a[y / 2 + w], 0x05040100u);
                f[2 * w + 1][i] = __builtin_amdgcn_perm(b[y / 2 + w], a[y / 2 + w], 0x07060302u);
            }
        }
    }
}

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// RT: 16-row tiles of queries.
template <int DH, bool F8, int RT>
__global__ __launch_bounds__(256, 2) void k_paged_attn_few(PagedAttn a) {
    using Tile = FewTile<DH, F8>;
    constexpr int F = DH / 16, R = 16 * RT;
    constexpr int NB = (F8 && (RT == 1 || DH == 64) ? 2 : 1) + (DH == 64 ? 1 : 0);     // tiles in flight per wave, as registers allow
    constexpr int ES = F8 ? 1 : 2, kGrid = CSD_PAGED_FEW_GRID, kCost = CSD_PAGED_FEW_COST;
    __shared__ int s_pages[kFewPages];
    __shared__ __align__(16) float s_o[4][R][DH + 4];
    __shared__ float s_m[4][R], s_l[4][R];
    __shared__ int s_limit[R];                               // last position a row attends
    __shared__ unsigned long long s_above[R];                // tree: its ancestors in the block
    static_assert((2 * CSD_PAGED_FEW_PARTS + 1) * R <= 4 * R * (DH + 4) && RT * (DH / 32) * 64 * 16 <= 4 * R * (DH + 4) * 4, "");
    __shared__ int s_last;
    const PagedPool &p = a.p;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
    const int cap = p.table_stride << p.page_shift;
    const float per_group = 1.f / (float)a.group;
    auto token_of = [&](int r) { return (int)(((float)r + 0.5f) * per_group); };     // r / group, r < 32: at least 1 / 64 from the next whole number

    // ---- the tiles of every sequence, counted from what an item costs besides them
    auto seq_of = [&](int b, PagedSeq &s) -> int {
        s = PagedSeq{0, 0, 0};
        if (b >= a.r.B) return 0;
        s = paged_seq(a.r, b);
        s.m = min(s.m, a.max_rows);
        const int rows = s.m * a.group;
        return rows >= 1 && rows <= R ? kCost + ((min(s.t + s.m, cap) + 31) >> 5) : 0;
    };
    PagedSeq s0;
    const int n0 = seq_of(lane, s0);                         // the first 64 sequences stay in registers
    int sum = n0, longest = n0;
#pragma unroll 4
    for (int b0 = 64; b0 < a.r.B; b0 += 64) {
        PagedSeq s;
        const int n = seq_of(b0 + lane, s);
        sum += n;
        longest = max(longest, n);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o, 64);
        longest = max(longest, __shfl_xor(longest, o, 64));
    }
    longest = __builtin_amdgcn_readfirstlane(longest);
    const int T = __builtin_amdgcn_readfirstlane(sum) * p.Hkv;
    if (T == 0) return;
    // a share is at least CSD_PAGED_FEW_SHARE tiles, and so long that no item has more parts than the join has room for
    const int least = max(CSD_PAGED_FEW_SHARE, (longest + CSD_PAGED_FEW_PARTS - 3) / (CSD_PAGED_FEW_PARTS - 2));
    const int n_wg = min((int)kGrid, max(1, T / least));
    if ((int)blockIdx.x >= n_wg) return;
    const PagedShares shares(T, n_wg);
    const int u_end = shares.first(blockIdx.x + 1);

    // The sequences of a share follow one another: 64 of them are held (lane x: sequence block + x), lane j is the one at hand, whose tiles begin at `before`.
    int u = shares.first(blockIdx.x), block = 0, j = 0, before = 0, n = 0;
    PagedSeq held = s0;
    int held_n = n0;
    for (;; block += 64) {
        if (block >= a.r.B) return;                          // (the lengths changed while they were read)
        if (block) held_n = seq_of(block + lane, held);
        int incl = held_n * p.Hkv;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(incl, o, 64);
            if (lane >= o) incl += x;
        }
        const unsigned long long past = __ballot(before + incl > u);
        if (past) {
            j = __ffsll((long long)past) - 1;
            n = __builtin_amdgcn_readlane(held_n, j);
            before += __builtin_amdgcn_readlane(incl, j) - n * p.Hkv;
            break;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }

    while (u < u_end) {
        // ---- the item of tile u: sequence b, key-value head kvh, tiles t0 .. t1 of its n
        while (u >= before + n * p.Hkv) {                    // the next sequence that has tiles
            before += n * p.Hkv;
            const unsigned long long next = __ballot(held_n > 0) & ~((2ull << j) - 1);
            if (next) {
                j = __ffsll((long long)next) - 1;
            } else {
                block += 64;
                if (block >= a.r.B) return;
                held_n = seq_of(block + lane, held);
                j = 0;
            }
            n = __builtin_amdgcn_readlane(held_n, j);
        }
        const int b = block + j;
        const PagedSeq seq{__builtin_amdgcn_readlane(held.start, j), __builtin_amdgcn_readlane(held.m, j), __builtin_amdgcn_readlane(held.t, j)};
        const int u0 = u, kvh = (u - before) / n, item = before + kvh * n + kCost, tiles = n - kCost;      // (where its tiles begin, how many there are)
        u = min(item + tiles, u_end);
        const int t0 = max(u0 - item, 0), t1 = u - item;
        if (t0 >= t1) continue;                              // (the share ends before the item's tiles begin)
        const int len = min(seq.t + seq.m, cap), rows = seq.m * a.group;

        // ---- the first pages and the queries are requested together; row r = token r / group, head r % group of the group
        const int first_page = paged_page(p, b, ((((t0 * 32) >> p.page_shift) + tid)) << p.page_shift);
        u32x4 qf[RT == 1 ? DH / 32 : 1];                      // (two row tiles: in LDS, where the waves' results will be; the registers are needed)
        u32x4 *s_q = reinterpret_cast<u32x4 *>(&s_o[0][0][0]) + lane;
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
        const unsigned long long anc = a.parent ? paged_ancestors(a.parent, seq, lane) : 0ull;
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            const int r = rt * 16 + col, i = token_of(r), h = r - i * a.group;
            const unsigned long long above = a.parent ? lane_of(anc, min(i, 63)) : 0ull;
            if (wave == 0 && g == 0) {                       // (needed where rows differ only: not worth registers)
                s_limit[r] = seq.t + i;
                s_above[r] = above;
            }
            const bf16_t *q = reinterpret_cast<const bf16_t *>(a.q) + (size_t)(seq.start + min(i, seq.m - 1)) * a.q_stride + (size_t)(kvh * a.group + h) * DH;
#pragma unroll
            for (int s = 0; s < DH / 32; s++) {
                const int at = F8 ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;      // features of the K operand's step s
                u32x4 x = *reinterpret_cast<const u32x4 *>(q + at);
#pragma unroll
                for (int w = 0; w < 4; w++) x[w] = r < rows && a.scale != 0.f ? x[w] ^ flip : 0u;
                if constexpr (RT == 1) qf[s] = x;
                else if (wave == 0) s_q[(rt * (DH / 32) + s) * 64] = x;
            }
        }
        const bool second = RT > 1 && rows > 16;             // the second row tile holds rows
        // scores in units of log2; the sign is the queries' (the maximum needs scale >= 0), and so is a scale of 0 (a masked score of -inf has to stay one)
        const float scale = fmaxf(fabsf(a.scale) * 1.44269504088896f, 1e-37f);
        f32x4 acc[RT][F];
        float m_run[RT], l_run[RT];
        uint32_t odd = 0;                                    // the wave took values out of its products
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            m_run[rt] = -INFINITY;
            l_run[rt] = 0.f;
#pragma unroll
            for (int j = 0; j < F; j++) acc[rt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        for (int c0 = t0; c0 < t1;) {
            // ---- the pages of tiles c0 .. c1
            const int page0 = (c0 * 32) >> p.page_shift;
            const long long fits = ((long long)(page0 + kFewPages) << p.page_shift) >> 5;
            const int c1 = fits >= t1 ? t1 : t0 + (((int)fits - t0) & ~3);      // (a wave keeps its turn from piece to piece)
            const int n_pages = (((c1 * 32 - 1) >> p.page_shift) - page0) + 1;
            __syncthreads();
            if (c0 == t0) {
                if (tid < n_pages) s_pages[tid] = first_page;
                for (int i = tid + 256; i < n_pages; i += 256) s_pages[i] = paged_page(p, b, (page0 + i) << p.page_shift);
            } else {
                for (int i = tid; i < n_pages; i += 256) s_pages[i] = paged_page(p, b, (page0 + i) << p.page_shift);
            }
            __syncthreads();
            // The queries have come too (before the table's entries, in order); said here, as otherwise the first product below waits for them, and
            // with them for every load in flight, at every turn.
            __builtin_amdgcn_s_waitcnt(0x0F70);              // vmcnt(0)

            // A wave has NB tiles' loads in flight, and the next one's as parts of a tile become free: its keys when the scores are made, its values
            // when the products are.
            Tile ring[NB];
            auto load_k = [&](Tile &t, int tile) {
                const int key = tile * 32 + 8 * (col >> 2);
                const int page = max(s_pages[(key >> p.page_shift) - page0], 0);      // (no page: rows of page 0, which the masks leave out)
                const char *kp = reinterpret_cast<const char *>(p.k) + paged_row(p, page, kvh, key + (col & 3)) * (DH * ES) + 16 * g;
#pragma unroll
                for (int T2 = 0; T2 < 2; T2++)
#pragma unroll
                    for (int s = 0; s < Tile::KV; s++) t.k[T2][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kp + T2 * 4 * DH * ES + s * 64));
                if constexpr (F8) {
                    const int key8 = tile * 32 + 8 * g;
                    t.ks = *reinterpret_cast<const u32x2 *>(p.ks + paged_row(p, max(s_pages[(key8 >> p.page_shift) - page0], 0), kvh, key8));
                }
            };
            auto load_v = [&](Tile &t, int tile) {
                const int key = tile * 32 + 8 * g;
                const int page = s_pages[(key >> p.page_shift) - page0];
                t.here = page >= 0;
                const size_t row = paged_row(p, max(page, 0), kvh, key);
                const char *vp = reinterpret_cast<const char *>(p.v) + row * (DH * ES) + col * (F * ES);
#pragma unroll
                for (int e = 0; e < 8; e++) load_words<Tile::VW>(vp + e * DH * ES, t.v[e]);
                if constexpr (F8) t.vs = *reinterpret_cast<const u32x2 *>(p.vs + row);
            };

            auto step = [&](Tile &t, int tile, auto always) {
                const int key0 = tile * 32, key = key0 + 8 * g;
                const bool whole = key0 + 32 <= seq.t && __all(t.here);      // (uniform) every row attends all 32 keys
                float x[RT][8];
                int q_off = 0;
                if constexpr (RT > 1) asm volatile("" : "+v"(q_off));   // (read here, at every tile)
                {
                    // (a half of the keys at a time, and below half of the features: the operands of a whole tile at once would not leave room for
                    // two waves per SIMD)
#pragma unroll
                    for (int T2 = 0; T2 < 2; T2++) {
                        u32x4 kf[DH / 32];
#pragma unroll
                        for (int s = 0; s < DH / 32; s++) {
                            if constexpr (F8) {
                                const uint32_t lo = t.k[T2][s / 2][2 * (s & 1)], hi = t.k[T2][s / 2][2 * (s & 1) + 1];
                                kf[s] = u32x4{bf16x2_of_fp8<false>(lo), bf16x2_of_fp8<true>(lo), bf16x2_of_fp8<false>(hi), bf16x2_of_fp8<true>(hi)};
                            } else {
                                kf[s] = t.k[T2][s];
                            }
                        }
#pragma unroll
                        for (int rt = 0; rt < RT; rt++) {
                            if (rt > 0 && !second) break;
                            f32x4 st = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int s = 0; s < DH / 32; s++) st = mfma16(kf[s], RT == 1 ? qf[s] : s_q[q_off + (rt * (DH / 32) + s) * 64], st);
#pragma unroll
                            for (int e = 0; e < 4; e++) x[rt][4 * T2 + e] = F8 ? st[e] * pow2_of_byte((t.ks[T2] >> (8 * e)) & 0xFFu) : st[e];
                        }
                    }
                }
                if (decltype(always)::value || tile + 4 * NB < c1) load_k(t, tile + 4 * NB);

                if constexpr (F8) {                          // values' scales of places that no row attends: 1 (the bytes may be anything)
                    if (!whole) {
                        const int n_in = t.here ? min(max(len - key, 0), 8) : 0;
                        const uint64_t in = n_in == 8 ? ~0ull : (1ull << (8 * n_in)) - 1, ones = 0x7F7F7F7F7F7F7F7Full;
                        const uint64_t v = (((uint64_t)t.vs[1] << 32 | t.vs[0]) & in) | (ones & ~in);
                        t.vs = u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
                    }
                }
                u32x4 hi[RT], lo[RT];
                uint32_t sees[RT];                           // bit e: the lane's row attends key + e
#pragma unroll
                for (int rt = 0; rt < RT; rt++) {
                    if (rt > 0 && !second) break;
                    sees[rt] = 0xFFu;
                    if (!whole) {
                        const int n_see = t.here ? min(max(min(s_limit[rt * 16 + col] + 1, len) - key, 0), 8) : 0;
                        sees[rt] = (1u << n_see) - 1u;
                        if (a.parent) {
                            const int d = key - seq.t;       // rows of the block lie at d .. d + 7 of `up`; keys before them are cached
                            const unsigned long long up = s_above[rt * 16 + col];
                            const unsigned long long m = d >= 0 ? (d < 64 ? up >> d : 0ull) : (up << min(-d, 8)) | ((1ull << min(-d, 8)) - 1);
                            sees[rt] &= (uint32_t)m;
                        }
#pragma unroll
                        for (int e = 0; e < 8; e++)
                            if (!((sees[rt] >> e) & 1u)) x[rt][e] = -INFINITY;
                    }
                    float top = fmaxf(fmaxf(fmaxf(x[rt][0], x[rt][1]), fmaxf(x[rt][2], x[rt][3])),
                                      fmaxf(fmaxf(x[rt][4], x[rt][5]), fmaxf(x[rt][6], x[rt][7])));
                    top = groups_max(sees[rt] ? fmaxf(top * scale, -3.0e38f) : -INFINITY);   // -inf: nothing to attend yet (a score of -inf is something)
                    // The reference of the weights is 8 above the maximum when it is set, and moves when a score passes it: the outputs are seldom rescaled, and
                    // no weight is above 1 (a sum of large values has the room that the formula's has).
                    if (__any(top > m_run[rt])) {
                        const float m_new = top > m_run[rt] ? top + 8.f : m_run[rt], fade = __builtin_amdgcn_exp2f(m_run[rt] - (m_new == -INFINITY ? 0.f : m_new));
                        l_run[rt] *= fade;
#pragma unroll
                        for (int j = 0; j < F; j++) acc[rt][j] *= fade;
                        m_run[rt] = m_new;
                    }
                    const float ref = m_run[rt] == -INFINITY ? 0.f : m_run[rt];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        float w[2];
#pragma unroll
                        for (int o = 0; o < 2; o++) {
                            const int e = 2 * i + o;
                            w[o] = __builtin_amdgcn_exp2f(fmaf(x[rt][e], scale, -ref));
                            l_run[rt] += w[o];
                            if constexpr (F8) w[o] *= pow2_of_byte(((t.vs[e >> 2] >> (8 * (e & 3))) & 0xFFu) + kUp);
                        }
                        const u32x2 planes = two_planes<!F8>(w[0], w[1]);
                        hi[rt][i] = planes[0];
                        lo[rt][i] = planes[1];
                    }
                }

#pragma unroll
                for (int y = 0; y < F; y += 4) {
                    u32x4 vf[4];
                    v_operands<DH, F8>(t.v, vf, y);
                    if (!whole) {
                        // keys behind the sequence's last are whatever the page holds, keys without a page somebody else's; and values that are not finite
                        const int n_in = t.here ? min(max(len - key, 0), 8) : 0;
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            const uint32_t keep = (2 * i < n_in ? 0xFFFFu : 0u) | (2 * i + 1 < n_in ? 0xFFFF0000u : 0u);
#pragma unroll
                            for (int j = 0; j < 4; j++) {
                                vf[j][i] &= keep;
                                const uint32_t o = odd_halves(vf[j][i]);
                                odd |= o;
                                vf[j][i] &= ~o;
                            }
                        }
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; rt++) {
                        if (rt > 0 && !second) break;
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            acc[rt][y + j] = mfma16(vf[j], hi[rt], acc[rt][y + j]);
                            acc[rt][y + j] = mfma16(vf[j], lo[rt], acc[rt][y + j]);
                        }
                    }
                }
                if (decltype(always)::value || tile + 4 * NB < c1) load_v(t, tile + 4 * NB);
            };
            // (behind a load under a condition, the wait for an earlier one is a wait for all: the main part has none)
            int tile = c0 + wave;
            if (tile + 4 * (2 * NB - 1) < c1) {
#pragma unroll
                for (int x = 0; x < NB; x++) {
                    load_k(ring[x], tile + 4 * x);
                    load_v(ring[x], tile + 4 * x);
                }
#pragma unroll 1
                do {
#pragma unroll
                    for (int x = 0; x < NB; x++) step(ring[x], tile + 4 * x, std::true_type{});
                    tile += 4 * NB;
                } while (tile + 4 * (2 * NB - 1) < c1);
            } else {
#pragma unroll
                for (int x = 0; x < NB; x++)
                    if (tile + 4 * x < c1) {
                        load_k(ring[x], tile + 4 * x);
                        load_v(ring[x], tile + 4 * x);
                    }
            }
#pragma unroll 1
            for (; tile < c1; tile += 4 * NB) {
#pragma unroll
                for (int x = 0; x < NB; x++)
                    if (tile + 4 * x < c1) step(ring[x], tile + 4 * x, std::false_type{});
            }
            c0 = c1;
        }

        if (__any(odd != 0u)) {
            for (int tile = t0 + wave; tile < t1; tile += 4)
                for (int key = tile * 32; key < min(tile * 32 + 32, len); key++) {
                    const int page = paged_page(p, b, key);
                    if (page < 0) continue;
                    const char *row = reinterpret_cast<const char *>(p.v) + paged_row(p, page, kvh, key) * (DH * ES);
#pragma unroll
                    for (int rt = 0; rt < RT; rt++) {
                        const bool attends = key <= s_limit[rt * 16 + col] && (!a.parent || key < seq.t || ((s_above[rt * 16 + col] >> min(key - seq.t, 63)) & 1ull));
#pragma unroll
                        for (int j = 0; j < F; j++)
#pragma unroll
                            for (int i = 0; i < 4; i++) acc[rt][j][i] += odd_value<F8>(row, F * (4 * g + i) + j, attends);
                    }
                }
        }

        // ---- the four waves' results
        if constexpr (RT > 1) __syncthreads();               // (the queries are no longer read)
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            l_run[rt] = groups_sum(l_run[rt]);
            if (g == 0) {
                s_m[wave][rt * 16 + col] = m_run[rt];
                s_l[wave][rt * 16 + col] = l_run[rt];
            }
#pragma unroll
            for (int j = 0; j < F; j++)                      // product j, A-row 4 g + i: feature F (4 g + i) + j
#pragma unroll
                for (int i = 0; i < 4; i++) s_o[wave][rt * 16 + col][F * (4 * g + i) + j] = acc[rt][j][i];
        }
        __syncthreads();
        const int w_first = shares.owner(item), w_last = shares.owner(item + tiles - 1);
        const bool split = w_first != w_last;
        const PagedParts<DH, R> parts(a.ws, CSD_PAGED_FEW_GRID, w_first, w_last - w_first + 1);
        auto out_row = [&](int r) {
            const int i = token_of(r), h = r - i * a.group;
            return reinterpret_cast<bf16_t *>(a.out) + (((size_t)(seq.start + i) * p.Hkv + kvh) * a.group + h) * DH;
        };
        for (int x = tid; x < rows * (DH / 4); x += 256) {
            const int r = x / (DH / 4), c = 4 * (x % (DH / 4));
            float m = s_m[0][r];
#pragma unroll
            for (int w = 1; w < 4; w++) m = fmaxf(m, s_m[w][r]);
            const float ref = m == -INFINITY ? 0.f : m;
            float l = 0.f;
            f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float f = __builtin_amdgcn_exp2f(s_m[w][r] - ref);
                l += f * s_l[w][r];
                o += *reinterpret_cast<const f32x4 *>(&s_o[w][r][c]) * f;
            }
            if (!split) {
                const float inv = 1.f / l;
                *reinterpret_cast<u32x2 *>(out_row(r) + c) =
                    m == -INFINITY ? u32x2{0u, 0u} : u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
            } else {
                parts.store(blockIdx.x - w_first, r, c, o);
                if (c == 0) parts.store(blockIdx.x - w_first, r, DH, f32x4{m, l, 0.f, 0.f});
            }
        }
        if (split && parts.arrive(a.ws, &s_last)) parts.join(a.ws, &s_o[0][0][0], rows, out_row);
        __syncthreads();
    }
}

template <int DH, bool F8, int RT>
static void few_launch(const PagedAttn &a, hipStream_t st) {
    hipLaunchKernelGGL((k_paged_attn_few<DH, F8, RT>), dim3(CSD_PAGED_FEW_GRID), dim3(256), 0, st, a);
}

template <int DH, bool F8>
static void few_rows(const PagedAttn &a, int rows, hipStream_t st) {
    if (rows <= 16) few_launch<DH, F8, 1>(a, st);
    else few_launch<DH, F8, 2>(a, st);
}

bool csd_paged_few_fits(const PagedAttn &a, int32_t pool_dtype, int32_t q_dtype) {
    if (!csd_paged_few_types(a.p.D, pool_dtype, q_dtype)) return false;
    // tiles are counted in 32 bits, and so are the work items of a launch
    const long long tiles = (((long long)a.p.table_stride << a.p.page_shift) + 31) / 32, heads = (long long)a.p.Hkv * a.group;
    return (tiles + CSD_PAGED_FEW_COST) * a.p.Hkv * a.r.B < (1ll << 30) && (long long)a.r.rows * heads / 128 + (long long)a.r.B * a.p.Hkv < (1ll << 23);
}

void csd_paged_few_enqueue(const PagedAttn &a, int rows, int32_t pool_dtype, hipStream_t st) {
    if (a.p.D == 128) {
        if (pool_dtype == CSD_DTYPE_FP8) few_rows<128, true>(a, rows, st);
        else few_rows<128, false>(a, rows, st);
    } else {
        if (pool_dtype == CSD_DTYPE_FP8) few_rows<64, true>(a, rows, st);
        else few_rows<64, false>(a, rows, st);
    }
}
