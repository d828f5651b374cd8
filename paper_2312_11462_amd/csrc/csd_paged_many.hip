// Attention of many rows (chunks of prompts beside other sequences, large trees, many query heads per key-value head) over a paged KV cache: bf16 queries, heads of
// 64 or 128, bf16 or e4m3 pools.
//
// The products of the scores and the weights bound this.  A workgroup of four waves takes 128 rows (rows of a sequence times the query heads that
// share its keys) of one key-value head, 32 rows per wave, and goes through the keys in tiles of 64 that it stages in LDS as bf16, two tiles
// deep: while a tile is worked on, the next one's loads are in flight to registers, from where it is stored (e4m3: converted, with its
// scale, exactly) between the second products.  Two workgroups share a compute unit, so that one's matrix products run beside the other's exponentials.
// Products are transposed:
//   S^T = K q^T    A = K (32 keys x 16 features, one 16-byte read), B = q^T, in registers throughout
//   O^T = V^T P^T  A = V^T (32 features x 16 keys, by LDS's transposing reads), B = P^T: a lane's scores of 16 keys are, in
//                  order, keys 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 (h = lane / 32), and A's columns are read in that order
// so that the weights never move between lanes.  The weights of sequences of up to 64 rows, and of cross-attention, enter as two bf16 planes, those of longer chunks as one:
// a second plane is half as many matrix instructions more, which bound this kernel (with it and without: a tree of 41 rows 22.4 and 21.4 us; 50 trees 112 and 105; 5 rows of 12 ragged
// sequences over up to 30000 keys, 8 x 8 heads of 128, e4m3 150 and 125; 4 chunks of 250 rows, 8 x 4 heads of 64, and 20 tokens 100 and 88).
// Rows of 16-byte pieces are stored with the piece index xored by the row, K and V in different ways, so that each kind of read
// spreads over all banks.
#include "csd_paged_tiles.h"

// The grid is a fixed number of workgroups, which take equal, contiguous shares of all items' key tiles (as k_paged_attn_few does; the parts of an item
// are joined by the workgroup that finishes last).
template <int DH, bool F8, bool CROSS>
__global__ __launch_bounds__(256, 2) void k_paged_attn_many(PagedAttnOf<CROSS> a, int min_rows) {
    constexpr int ES = F8 ? 1 : 2, LPR = DH * ES / 16;       // lanes that load a row
    constexpr int RPP = 256 / LPR, NP = kKeys / RPP;         // rows per pass of the workgroup, passes per tile
    constexpr int PIECES = kKeys * DH / 8;                   // 16-byte pieces of a staged tile
    constexpr int ST = DH / 16, DT = DH / 32, BM = CSD_PAGED_MANY_ROWS, PARTS = CSD_PAGED_MANY_PARTS;
    // what an item costs besides its keys, in tiles: the round trips to memory in front of its first tile and behind its last one
    constexpr int COST = CSD_PAGED_MANY_COST;
    __shared__ u32x4 s_tiles[4][PIECES];
    u32x4(&s_k)[2][PIECES] = *reinterpret_cast<u32x4(*)[2][PIECES]>(&s_tiles[0]), (&s_v)[2][PIECES] = *reinterpret_cast<u32x4(*)[2][PIECES]>(&s_tiles[2]);
    __shared__ float s_max[BM], s_sum[BM];
    __shared__ int s_odd, s_last;
    __shared__ int s_b[CSD_PAGED_MANY_BATCH], s_start[CSD_PAGED_MANY_BATCH], s_m[CSD_PAGED_MANY_BATCH], s_t[CSD_PAGED_MANY_BATCH], s_units[CSD_PAGED_MANY_BATCH];
    __shared__ int s_count[4];
    const PagedPool &p = a.p;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, h = lane >> 5;

    auto seq_of = [&](int b, PagedSeq &s) -> int {           // row tiles of a sequence
        s = PagedSeq{0, 0, 0};
        if (b >= a.r.B) return 0;
        s = paged_seq(a.r, b);
        s.m = min(s.m, a.max_rows);
        const int rows = s.m * a.group;
        return rows > min_rows ? (rows + BM - 1) / BM : 0;
    };
    auto scan = [&](int x) {                                 // inclusive, over the wave
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(x, o, 64);
            if (lane >= o) x += y;
        }
        return x;
    };

    // ---- the sequences that take part, in order
    int batch = 0;
    for (int b0 = 0; b0 < a.r.B; b0 += 256) {
        PagedSeq s;
        const bool in = seq_of(b0 + tid, s) > 0;
        const unsigned long long all = __ballot(in);
        if (lane == 0) s_count[wave] = __popcll(all);
        __syncthreads();
        int at = batch + __popcll(all & ((1ull << lane) - 1));
        for (int w = 0; w < 4; w++) {
            if (w < wave) at += s_count[w];
            batch += s_count[w];
        }
        if (in && at < CSD_PAGED_MANY_BATCH) {
            s_b[at] = b0 + tid;
            s_m[at] = s.m;
            s_t[at] = s.t;
            s_start[at] = s.start;
        }
        __syncthreads();
    }
    batch = min(__builtin_amdgcn_readfirstlane(batch), CSD_PAGED_MANY_BATCH);

    // ---- this workgroup's share
    for (int b = tid / 8; b < batch; b += 32) {              // eight lanes per sequence
        const int m = s_m[b], t = s_t[b], n = (m * a.group + BM - 1) / BM;
        int sum = 0;
        for (int rt = tid % 8; rt < n; rt += 8) sum += COST + row_tile_keys(a, rt, m, t);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        if (tid % 8 == 0) s_units[b] = sum;
    }
    __syncthreads();
    int sum = 0, longest = 0;
    for (int b = lane; b < batch; b += 64) {
        sum += s_units[b];
        longest = max(longest, COST + tiles_of<CROSS>(a.keys(s_t[b], s_m[b] - 1)));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o, 64);
        longest = max(longest, __shfl_xor(longest, o, 64));
    }
    const int T = __builtin_amdgcn_readfirstlane(sum) * p.Hkv;
    if (T == 0) return;
    longest = __builtin_amdgcn_readfirstlane(longest);
    const int least = max(CSD_PAGED_MANY_SHARE, (longest + PARTS - 3) / (PARTS - 2));
    const int n_wg = min(CSD_PAGED_MANY_GRID, max(1, T / least));
    // workgroups go to the compute dies in turn: a die's take neighbouring shares, which read the same keys
    const int per_die = (n_wg + 7) / 8;
    const int me = (int)(blockIdx.x % 8) * per_die + (int)(blockIdx.x / 8);
    if ((int)blockIdx.x / 8 >= per_die || me >= n_wg) return;
    const PagedShares shares(T, n_wg);
    int u = shares.first(me);
    const int u_end = shares.first(me + 1);

    while (u < u_end) {
    // ---- the item: rows rt * BM .. of sequence b, key-value head kvh, key tiles kt0 .. kt1 of its n_kt
    int at = -1, before = 0;
    for (int b0 = 0; b0 < batch; b0 += 64) {
        const int x = b0 + lane < batch ? s_units[b0 + lane] * p.Hkv : 0, incl = scan(x);
        const unsigned long long past = __ballot(before + incl > u);
        if (past) {
            const int j = __ffsll((long long)past) - 1;
            at = b0 + j;
            before += __builtin_amdgcn_readlane(incl, j) - __builtin_amdgcn_readlane(x, j);
            break;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    if (at < 0) return;                                      // (the lengths changed while they were read)
    const PagedSeq seq{__builtin_amdgcn_readfirstlane(s_start[at]), __builtin_amdgcn_readfirstlane(s_m[at]), __builtin_amdgcn_readfirstlane(s_t[at])};
    const int b = __builtin_amdgcn_readfirstlane(s_b[at]);
    const int units = __builtin_amdgcn_readfirstlane(s_units[at]), n = (seq.m * a.group + BM - 1) / BM;
    const int kvh = (u - before) / units;
    if (kvh >= p.Hkv) return;
    int left = u - before - kvh * units;
    int rt = -1, kt0 = 0;
    for (int r0 = 0; r0 < n; r0 += 64) {
        const int x = r0 + lane < n ? COST + row_tile_keys(a, r0 + lane, seq.m, seq.t) : 0, incl = scan(x);
        const unsigned long long past = __ballot(incl > left);
        if (past) {
            const int j = __ffsll((long long)past) - 1;
            rt = r0 + j;
            kt0 = left - (__builtin_amdgcn_readlane(incl, j) - __builtin_amdgcn_readlane(x, j));
            break;
        }
        left -= __builtin_amdgcn_readlane(incl, 63);
    }
    if (rt < 0) return;
    const int item = u - kt0 + COST;                         // where its keys begin
    kt0 -= COST;
    const int rows = min(seq.m * a.group - rt * BM, BM);     // of this item
    const int n_kt = row_tile_keys(a, rt, seq.m, seq.t);
    const int kt1 = min(n_kt, kt0 + u_end - u);
    u += kt1 - kt0;
    kt0 = max(kt0, 0);
    if (kt1 <= 0) continue;                                  // (the share ends before the keys begin)
    const int len = a.keys(seq.t, (rt * BM + rows - 1) / a.group);      // keys that some row attends

    // The page table, 16 tiles at a time: lane x holds where the x-th group of 16 keys from tile `base` on lies in the pools (bytes; one without a
    // page: in page 0, which the masks leave out), and bit x of `here` says that it has a page.
    struct Pages {
        size_t at;
        unsigned long long here;
    };
    auto pages_from = [&](int base) {
        const int key = (base * 4 + lane) * 16;
        const int page = paged_page(p, b, key);
        return Pages{paged_row(p, max(page, 0), kvh, key) * (DH * ES), __ballot(page >= 0)};
    };
    Pages pages = pages_from(kt0), pages_next = pages_from(kt0 + 16);

    // ---- this lane's row
    const int r = rt * BM + wave * 32 + col, i = r / a.group, hq = r - i * a.group;
    const bool live = wave * 32 + col < rows;
    const int limit = a.last(seq.t, i);                             // last position it attends
    unsigned long long above = 0;
    if (a.parent) above = lane_of(paged_ancestors(a.parent, seq, lane), min(i, 63));
    u32x4 qf[ST];
    {
        const bf16_t *q = reinterpret_cast<const bf16_t *>(a.q) + (size_t)(seq.start + i) * a.q_stride + (size_t)(kvh * a.group + hq) * DH + 8 * h;
#pragma unroll
        for (int s = 0; s < ST; s++) {
            qf[s] = u32x4{0u, 0u, 0u, 0u};
            if (live && a.scale != 0.f) qf[s] = *reinterpret_cast<const u32x4 *>(q + 16 * s);
        }
    }
    // scores in units of log2 (more than 0, so that a masked score of -inf stays one; with a scale of 0 the queries are)
    const float scale = fmaxf(fabsf(a.scale) * 1.44269504088896f, 1e-37f);
    f32x16 acc[DT];
    float m_run = -INFINITY;
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[d][e] = 0.f;

    // ---- staging: in pass x a wave's rows lie in one group of 16 keys, so in one page
    const int row_in = tid / LPR, c_in = tid % LPR;
    auto group_of = [&](int x) { return (x * RPP + wave * (64 / LPR)) >> 4; };
    auto here_mask = [&](int kt) { return (unsigned)(pages.here >> (((kt - kt0) & 15) * 4)) & 0xFu; };
    // A side (0: keys, 1: values) of a tile, pass by pass: to registers, then, converted, to LDS.
    constexpr std::integral_constant<int, 0> K{};
    constexpr std::integral_constant<int, 1> V{};
    constexpr int SIDES = F8 ? 2 : 1;                        // bf16: both sides in the same registers, one after the other
    u32x4 regs[SIDES][NP];
    uint8_t scales[F8 ? 2 : 1][NP];
    const unsigned lane_at = ((wave * (64 / LPR)) & 15) * (DH * ES) + lane * 16;       // a lane's place in the 16 keys of its pass
    auto load = [&](int kt, int x, auto side) {
        constexpr int S = decltype(side)::value;
        const int from = ((kt - kt0) & 15) * 4 + group_of(x);
        const size_t at = ((size_t)(unsigned)__builtin_amdgcn_readlane((int)(pages.at >> 32), from) << 32) | (unsigned)__builtin_amdgcn_readlane((int)pages.at, from);
        regs[S % SIDES][x] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(S ? p.v : p.k) + at + lane_at);
        if constexpr (F8) scales[S][x] = ((S ? p.vs : p.ks) + at / DH)[lane_at / DH];
    };
    auto stage = [&](int x, int buf, auto side) {
        constexpr int S = decltype(side)::value, W = F8 ? 2 : 1;
        const int row = x * RPP + row_in;
        const u32x4 raw = regs[S % SIDES][x];
        u32x4 v[W];
        if constexpr (F8) {
            const float f = pow2_of_byte(scales[S][x]);
#pragma unroll
            for (int w = 0; w < 2; w++)
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    v[w][2 * y] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[2 * w + y], f, false));
                    v[w][2 * y + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[2 * w + y], f, true));
                }
        } else {
            v[0] = raw;
        }
#pragma unroll
        for (int w = 0; w < W; w++) {
            if constexpr (S == 1) s_v[buf][v_piece<DH>(row, W * c_in + w)] = v[w];
            else s_k[buf][k_piece<DH>(row, W * c_in + w)] = v[w];
        }
    };
    // Where rows of the block, or places without a row, are among a tile's keys: values that no row attends are taken out of LDS again, and those
    // that are not finite (see odd_halves).  A thread looks at what it stored.
    auto mend = [&](int kt, int buf) {
        const unsigned here = here_mask(kt);
        if (kt * kKeys + kKeys <= seq.t && here == 0xFu) return;
        constexpr int W = F8 ? 2 : 1;
        bool odd = false;
#pragma unroll
        for (int x = 0; x < NP; x++) {
            const int row = x * RPP + row_in;
            const bool out = kt * kKeys + row >= len || !((here >> group_of(x)) & 1u);
#pragma unroll
            for (int w = 0; w < W; w++) {
                u32x4 v = s_v[buf][v_piece<DH>(row, W * c_in + w)];
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    if (out) v[y] = 0u;
                    const uint32_t o = odd_halves(v[y]);
                    odd |= o != 0u;
                    v[y] &= ~o;
                }
                s_v[buf][v_piece<DH>(row, W * c_in + w)] = v;
            }
        }
        if (odd) s_odd = 1;
    };
    if (tid == 0) s_odd = 0;
    __syncthreads();
    {
        u32x4 first[NP];                                     // (both sides in flight)
#pragma unroll
        for (int x = 0; x < NP; x++) load(kt0, x, V);
#pragma unroll
        for (int x = 0; x < NP; x++) first[x] = regs[1 % SIDES][x];
#pragma unroll
        for (int x = 0; x < NP; x++) load(kt0, x, K);
#pragma unroll
        for (int x = 0; x < NP; x++) stage(x, 0, K);
#pragma unroll
        for (int x = 0; x < NP; x++) regs[1 % SIDES][x] = first[x];
#pragma unroll
        for (int x = 0; x < NP; x++) stage(x, 0, V);
        mend(kt0, 0);
    }
    __syncthreads();

    if (a.scale < 0.f)                                       // a negative scale turns the queries around: the maximum below needs scale >= 0
#pragma unroll
        for (int s = 0; s < ST; s++) qf[s] ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
    const int wave_first = a.last(seq.t, (rt * BM + wave * 32) / a.group);      // last position that the wave's first row attends
    // where a lane reads: K row `col` (+ 32), pieces 2 s + h; V as LDS's transposing read wants it (the place of 4 features of a key), pieces 4 d + ..
    const int l16 = lane & 15;
    const int k_at = k_piece<DH>(col, h) * 16, v_row = 4 * h + (l16 >> 2);
    const int v_at = v_piece<DH>(v_row, 2 * ((lane >> 4) & 1) + ((l16 >> 1) & 1)) * 16 + 8 * (l16 & 1);
    float l_run = 0.f, l_more = 0.f;                         // the sum of weights, in two chains
    int kt = kt0;
    auto turn = [&](auto which, auto planes) {
        constexpr int buf = decltype(which)::value;
        constexpr bool TWO = decltype(planes)::value;        // weights in two bf16 planes
        const int key0 = kt * kKeys, next = min(kt + 1, kt1 - 1);        // (the last turn brings its own tile once more: no branches)
        const unsigned here = here_mask(kt);
        if (((next - kt0) & 15) == 0 && next != kt) {
            pages = pages_next;
            pages_next = pages_from(next + 16);
        }
        // What is issued between the matrix instructions, which take as long as several others, is set down one by one: operands are read two
        // products ahead; the next tile's values are requested first and stored (to the other buffer, last read a turn ago) beside the second
        // products, its keys requested as registers become free and stored at the end.
        int ka_at = k_at, va_at = v_at;
        asm volatile("" : "+v"(ka_at), "+v"(va_at));         // (the xors below are made here, not kept in a register each)
        f32x16 st[2];
#pragma unroll
        for (int e = 0; e < 16; e++) st[0][e] = st[1][e] = 0.f;
        u32x4 ka[3][2];
        auto read_k = [&](int s) {
#pragma unroll
            for (int T2 = 0; T2 < 2; T2++)
                ka[s % 3][T2] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(&s_k[buf][0]) + (ka_at ^ (32 * s)) + T2 * 32 * DH * 2);
        };
        read_k(0);
        read_k(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < ST; s++) {
            if (s + 2 < ST) read_k(s + 2);
            st[0] = mfma32(ka[s % 3][0], qf[s], st[0]);
            if (s < NP) load(next, s, V);
            __builtin_amdgcn_sched_barrier(0);
            st[1] = mfma32(ka[s % 3][1], qf[s], st[1]);
            if (F8 && s < NP) load(next, s, K);
            __builtin_amdgcn_sched_barrier(0);
        }
        // element e of half T2 is key 32 T2 + 8 (e / 4) + 4 h + e % 4
        const bool whole = (a.parent ? key0 + kKeys <= seq.t : key0 + kKeys - 1 <= wave_first) && key0 + kKeys <= len && here == 0xFu;
        bool sees = true;
        if (!whole) {
            const int n = min(limit, len - 1) - key0;        // attended: keys 0 .. n of the tile
            unsigned long long m = n >= 63 ? ~0ull : n < 0 ? 0ull : (2ull << n) - 1;
#pragma unroll
            for (int g = 0; g < 4; g++)
                if (!((here >> g) & 1u)) m &= ~(0xFFFFull << (16 * g));
            if (a.parent) {
                const int d = key0 - seq.t;                  // rows of the block lie at d .. of `above`; keys before them are cached
                m &= d >= 0 ? (d < 64 ? above >> d : 0ull) : -d >= 64 ? ~0ull : (above << -d) | ((1ull << -d) - 1);
            }
            sees = m != 0;
            m >>= 4 * h;
#pragma unroll
            for (int e = 0; e < 32; e++)
                if (!((m >> (8 * (e / 4) + e % 4)) & 1u)) st[e >> 4][e & 15] = -INFINITY;
        }
        auto read_v = [&](int x) {                           // features 32 d .. of keys 16 u .., in the order of the weights
            const int u = x / DT, d = x % DT;
            uint64_t w[2];
#pragma unroll
            for (int y = 0; y < 2; y++) {
                char *at = reinterpret_cast<char *>(&s_v[buf][0]) + (va_at ^ (64 * d)) + (16 * u + 8 * y) * DH * 2;
                w[y] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at));
            }
            return u32x4{(uint32_t)w[0], (uint32_t)(w[0] >> 32), (uint32_t)w[1], (uint32_t)(w[1] >> 32)};
        };
        u32x4 va[3];
        va[0] = read_v(0);
        va[1] = read_v(1);
        float top = st[0][0];
#pragma unroll
        for (int e = 1; e < 31; e += 2) top = fmaxf(fmaxf(st[e >> 4][e & 15], st[(e + 1) >> 4][(e + 1) & 15]), top);
        // (both halves of the lanes have the row's maximum; -inf: nothing to attend yet, a score of -inf is something)
        top = halves_max(sees ? fmaxf(fmaxf(top, st[1][15]) * scale, -3.0e38f) : -INFINITY);
        // The reference of the weights is 8 above the maximum when it is set, and moves when a score passes it: the outputs are seldom rescaled, and no
        // weight is above 1 (a sum of large values has the room that the formula's has).
        if (__any(top > m_run)) {
            const float m_new = top > m_run ? top + 8.f : m_run, fade = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
            l_run *= fade;
            l_more *= fade;
#pragma unroll
            for (int d = 0; d < DT; d++) acc[d] *= fade;
            m_run = m_new;
        }
        const float ref = m_run == -INFINITY ? 0.f : -m_run;
        u32x4 pw[2], pl[2];                                  // weights of keys 16 u .. 16 u + 15 at u % 2
        auto weigh = [&](int e) {                            // elements e, e + 1
            const float w0 = __builtin_amdgcn_exp2f(fmaf(st[e >> 4][e & 15], scale, ref)), w1 = __builtin_amdgcn_exp2f(fmaf(st[e >> 4][(e + 1) & 15], scale, ref));
            l_run += w0;
            l_more += w1;
            if constexpr (TWO) {
                const u32x2 w = two_planes<!F8>(w0, w1);
                pw[(e >> 3) & 1][(e & 7) >> 1] = w[0];
                pl[(e >> 3) & 1][(e & 7) >> 1] = w[1];
            } else {
                pw[(e >> 3) & 1][(e & 7) >> 1] = pack_bf16x2(w0, w1);
            }
        };
#pragma unroll
        for (int e = 0; e < 8; e += 2) weigh(e);
        __builtin_amdgcn_sched_barrier(0);
        // The next 16 keys' weights are made beside the products of these.  (A wave here goes first: the matrix cores wait for nothing else; 4 chunks of 250 rows
        // and 20 tokens, 8 x 4 heads of 64, 94.7 -> 87.5 us, 300 rows over 8000 keys, heads of 128, 76.9 -> 74.2.)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int x = 0; x < 4 * DT; x++) {
            const int u = x / DT, d = x % DT;
            if (x + 2 < 4 * DT) va[(x + 2) % 3] = read_v(x + 2);
            acc[d] = mfma32(va[x % 3], pw[u & 1], acc[d]);
            if constexpr (TWO) acc[d] = mfma32(va[x % 3], pl[u & 1], acc[d]);
            if (u < 3)
#pragma unroll
                for (int e = 0; e < 8 / DT; e += 2) weigh(8 * (u + 1) + 8 / DT * d + e);
            __builtin_amdgcn_sched_barrier(0);
            if (x < NP) {
                stage(x, buf ^ 1, V);
                if (!F8) load(next, x, K);
            }
            if (F8 && x >= 4 * DT - NP) stage(x - (4 * DT - NP), buf ^ 1, K);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (!F8)
#pragma unroll
            for (int x = 0; x < NP; x++) stage(x, buf ^ 1, K);
        mend(next, buf ^ 1);
    };
    auto turns = [&](auto planes) {
#pragma unroll 1
        while (true) {
            turn(std::integral_constant<int, 0>{}, planes);
            __syncthreads();
            if (++kt == kt1) break;
            turn(std::integral_constant<int, 1>{}, planes);
            __syncthreads();
            if (++kt == kt1) break;
        }
    };
    if constexpr (CROSS) turns(std::true_type{});
    else if (seq.m <= CSD_PAGED_FINE_ROWS) turns(std::true_type{});
    else turns(std::false_type{});
    l_run = halves_sum(l_run + l_more);

    if (s_odd) {                                             // (uniform; the last tile was staged in front of a barrier)
        for (kt = kt0; kt < kt1; kt++) {
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

    // ---- results: element e of acc[d] is feature 32 d + 8 (e / 4) + 4 h + e % 4 of the lane's row.  Turned in LDS, where the key tiles were (16-byte pieces,
    // their index xored by the row), so that whole rows are written one behind the other (with the join by 4 x 4 pieces, against 16-byte stores from here and
    // a join by fours: a tree of 41 rows over 1024 keys, 32 heads of 128, 23.9 -> 21.5 us; 22.6 with weights in two planes).
    constexpr int C = DH / 4;
    auto piece = [&](int row, int c) { return row * C + (c ^ (row & (C - 1))); };
    u32x4 *s_o = &s_tiles[0][0];
    {
        int row = wave * 32 + col;
        asm volatile("" : "+v"(row));
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
            for (int y = 0; y < 4; y++)
                s_o[piece(row, 8 * d + 2 * y + h)] = __builtin_bit_cast(u32x4, f32x4{acc[d][4 * y], acc[d][4 * y + 1], acc[d][4 * y + 2], acc[d][4 * y + 3]});
        if (h == 0) {
            s_max[row] = m_run;
            s_sum[row] = l_run;
        }
    }
    __syncthreads();
    int id = tid;
    asm volatile("" : "+v"(id));                             // (what follows from it is made here, not kept in registers all along)
    auto out_row = [&](int row) {
        const int r_ = rt * BM + row, i_ = r_ / a.group, h_ = r_ - i_ * a.group;
        return reinterpret_cast<bf16_t *>(a.out) + (((size_t)(seq.start + i_) * p.Hkv + kvh) * a.group + h_) * DH;
    };
    const int w_first = shares.owner(item), w_last = shares.owner(item + n_kt - 1), parts = w_last - w_first + 1;
    if (parts == 1) {
        for (int x = id; x < rows * (C / 2); x += 256) {
            const int row = x / (C / 2), c = x % (C / 2);
            const float inv = 1.f / s_sum[row];
            u32x4 o;
#pragma unroll
            for (int y = 0; y < 2; y++) {
                const f32x4 v = __builtin_bit_cast(f32x4, s_o[piece(row, 2 * c + y)]) * inv;
                o[2 * y] = pack_bf16x2(v[0], v[1]);
                o[2 * y + 1] = pack_bf16x2(v[2], v[3]);
            }
            if (s_max[row] == -INFINITY) o = u32x4{0u, 0u, 0u, 0u};
            *reinterpret_cast<u32x4 *>(out_row(row) + 8 * c) = o;
        }
        __syncthreads();
        continue;
    }
    const PagedParts<DH, BM> split(a.ws, CSD_PAGED_MANY_GRID, w_first, parts);
    for (int x = id; x < rows * (C + 1); x += 256) {
        const int row = x / (C + 1), c = x % (C + 1);
        split.store(me - w_first, row, 4 * c, c < C ? __builtin_bit_cast(f32x4, s_o[piece(row, c)]) : f32x4{s_max[row], s_sum[row], 0.f, 0.f});
    }
    if (!split.arrive(a.ws, &s_last)) continue;
    static_assert((2 * PARTS + 1) * BM * 4 <= 4 * PIECES * 16 && BM * C <= 4 * PIECES, "");
    split.join(a.ws, reinterpret_cast<float *>(s_o), rows, out_row);
    __syncthreads();
    }
}

void csd_paged_many_enqueue(const PagedAttn &a, int min_rows, int32_t pool_dtype, hipStream_t st) {
    // row tiles at most: full ones, and a last one per sequence that takes part
    const long long rows = (long long)a.r.rows * a.group, batch = csd_paged_batch(a, min_rows), items = (rows / CSD_PAGED_MANY_ROWS + batch) * a.p.Hkv;
    const long long keys = ((long long)a.p.table_stride << a.p.page_shift) / kKeys + 1 + CSD_PAGED_MANY_COST;      // (all key tiles are counted in 32 bits)
    const bool fits = batch <= CSD_PAGED_MANY_BATCH && items * keys < (1ll << 30);
    // row tiles if some sequences have max_rows rows and the others one
    const long long most = a.max_rows, full = most > 1 ? (a.r.rows - (long long)a.r.B + most - 2) / (most - 1) : a.r.B;
    const long long likely = (full * most * a.group / CSD_PAGED_MANY_ROWS + full) * a.p.Hkv;
    if (!fits || (likely > CSD_PAGED_MANY_ITEMS && most > CSD_PAGED_FINE_ROWS && most * a.group >= CSD_PAGED_CHUNK_ROWS))
        return csd_paged_chunk_enqueue(a, min_rows, pool_dtype, st);
    const bool f8 = pool_dtype == CSD_DTYPE_FP8;
    csd_paged_by_cross(a, [&](auto x) {
        constexpr bool CROSS = std::is_same<decltype(x), PagedAttnOf<true>>::value;
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(CSD_PAGED_MANY_GRID), dim3(256), 0, st, x, min_rows); };
        if (a.p.D == 128) f8 ? launch(k_paged_attn_many<128, true, CROSS>) : launch(k_paged_attn_many<128, false, CROSS>);
        else f8 ? launch(k_paged_attn_many<64, true, CROSS>) : launch(k_paged_attn_many<64, false, CROSS>);
    });
}
