// Attention of so many rows that whole workgroups of them fill the chip (chunks of long prompts), in the types and head sizes of csd_paged_many.hip,
// whose tiles and products these are.
//
// A workgroup of eight waves takes 256 rows of one key-value head, 32 rows per wave, two waves per SIMD.  A wave issues an instruction every five cycles
// or so whatever it is, and a matrix instruction keeps the matrix core busy for 32: what bounds this is how well the two waves of a SIMD
// fill each other's gaps.  So waves 4 .. 7 work half a tile behind waves 0 .. 3: between two barriers
//   waves 0-3:  scores of tile k, weights and products of tile k
//   waves 4-7:  weights and products of tile k - 1, scores of tile k
// and each stages its part of tile k + 1 beside its scores, from registers that were requested a tile earlier.  Values of three tiles and keys of two are in LDS.
// (2 chunks of 2048 rows, 8 x 4 heads of 128, 10239 and 4096 keys, bf16: 415 us, 993 TFLOP/s; two independent workgroups of four waves and 128 rows
// per compute unit took 455; e4m3 406 against 433; heads of 64 256 against 284; a barrier behind each half of a tile instead: 411, but one fresh prompt of
// 4099 rows, 32 heads, 215 instead of 193.)  Weights in two planes, as those of blocks of up to 64 rows are, would take 542 us, e4m3 531, heads of 64 348.
// Cross-attention has them: as near to 64 bits as its output's rounding lets it be, however many rows there are (4 x 1024 rows over 1000 to 4096 encoder rows, 32 heads
// of 128: 255 to 274 us by the card, off by 1.66e-3 of the outputs' size; in one plane 196 to 202, off by 2.32e-3).
#include "csd_paged_tiles.h"

static constexpr int kChunkRows = 256;
template <int DH, bool F8, bool CROSS>
__global__ __launch_bounds__(512, 2) void k_paged_attn_chunk(PagedAttnOf<CROSS> a, int min_rows) {
    constexpr int ES = F8 ? 1 : 2, LB = F8 && DH == 64 ? 8 : 16;         // bytes that a lane loads
    constexpr int LPR = DH * ES / LB;                        // lanes that load a row
    constexpr int RPP = 512 / LPR, NP = kKeys / RPP;         // rows per pass of the workgroup, passes per tile
    constexpr int PIECES = kKeys * DH / 8, W = F8 ? LB / 8 : 1;          // 16-byte pieces of a staged tile, of what a lane stages
    constexpr int ST = DH / 16, DT = DH / 32, BM = kChunkRows;
    typedef typename std::conditional<LB == 16, u32x4, u32x2>::type raw_t;
    __shared__ u32x4 s_tiles[5][PIECES];                     // keys of two tiles, values of three
    __shared__ int s_odd;
    const PagedPool &p = a.p;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, h = lane >> 5;
    const bool late = wave >= 4;                             // half a tile behind
    const int cap = p.table_stride << p.page_shift;

    // ---- the item: key-value heads follow one another (workgroups of a die, every eighth, read the same keys), then the row tiles, the late ones with
    // the most keys first
    const int kvh = blockIdx.x % p.Hkv;
    int b = -1, rt = 0, total = 0;
    PagedSeq seq{0, 0, 0};
    const bool by_length = CROSS && a.r.B <= 64;
    if (by_length) {
        // Every row tile of a sequence has all of its encoder's keys: the sequences with the most keys first, so that the last workgroups are short ones (4 x 1024 rows
        // over 1000 to 4096 encoder rows, 32 heads of 128: 267 us, in the order of the sequences 303).
        PagedSeq s{0, 0, 0};
        int n = 0;
        if (lane < a.r.B) {
            s = paged_seq(a.r, lane);
            s.m = min(s.m, a.max_rows);
            if (s.m * a.group > min_rows) n = (s.m * a.group + BM - 1) / BM;
        }
        const int keys = n ? min(s.t, cap) : -1;
        int before = 0;                                      // row tiles of the sequences ahead
        for (int o = 0; o < a.r.B; o++) {
            const int other = __builtin_amdgcn_readlane(keys, o);
            const bool first = other > keys || (other == keys && o < lane);
            before += first ? __builtin_amdgcn_readlane(n, o) : 0;
        }
        const int want = (int)(blockIdx.x / p.Hkv);
        const unsigned long long mine = __ballot(n > 0 && before <= want && want < before + n);
        if (!mine) return;
        b = __ffsll((long long)mine) - 1;
        rt = want - __builtin_amdgcn_readlane(before, b);
        seq = PagedSeq{__builtin_amdgcn_readlane(s.start, b), __builtin_amdgcn_readlane(s.m, b), __builtin_amdgcn_readlane(s.t, b)};
    }
    for (int pass = by_length ? 2 : 0; pass < 2; pass++) {   // count the row tiles of all sequences, then find this one
        int before = 0;
        const int want = total - 1 - (int)(blockIdx.x / p.Hkv);
        if (pass && want < 0) return;
        for (int b0 = 0; b0 < a.r.B; b0 += 64) {
            PagedSeq s{0, 0, 0};
            int n = 0;
            if (b0 + lane < a.r.B) {
                s = paged_seq(a.r, b0 + lane);
                s.m = min(s.m, a.max_rows);
                if (s.m * a.group > min_rows) n = (s.m * a.group + BM - 1) / BM;
            }
            int incl = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(incl, o, 64);
                if (lane >= o) incl += y;
            }
            if (pass) {
                const unsigned long long past = __ballot(before + incl > want);
                if (past) {
                    const int j = __ffsll((long long)past) - 1;
                    b = b0 + j;
                    rt = want - (before + __builtin_amdgcn_readlane(incl, j) - __builtin_amdgcn_readlane(n, j));
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
    const int len = a.keys(seq.t, (rt * BM + rows - 1) / a.group);      // keys that some row attends
    const int n_kt = tiles_of<CROSS>(len);

    // The page table, 16 tiles at a time: lane x holds where the x-th group of 16 keys from tile `base` on lies in the pools (bytes; one without a
    // page: in page 0, which the masks leave out), and bit x of `here` says that it has a page.  The window moves by eight tiles.
    struct Pages {
        size_t at;
        unsigned long long here;
    };
    auto pages_from = [&](int tile) {
        const int key = (tile * 4 + lane) * 16;              // (behind the table's end, which a sequence may be said to reach, there is no page)
        const int page = paged_page(p, b, key);
        return Pages{paged_row(p, max(page, 0), kvh, key) * (DH * ES), __ballot(page >= 0)};
    };
    int base = 0;
    Pages pages = pages_from(0), pages_next = pages_from(8);

    // ---- this lane's row
    const int r = rt * BM + wave * 32 + col, i = r / a.group, hq = r - i * a.group;
    const bool live = wave * 32 + col < rows;
    const int limit = a.last(seq.t, i);                             // last position it attends
    unsigned long long above = 0;
    if (a.parent) above = lane_of(paged_ancestors(a.parent, seq, lane), min(i, 63));
    u32x4 qf[ST];
    {
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;          // (a negative scale turns the queries around: the maximum below needs scale >= 0)
        const bf16_t *q = reinterpret_cast<const bf16_t *>(a.q) + (size_t)(seq.start + i) * a.q_stride + (size_t)(kvh * a.group + hq) * DH + 8 * h;
#pragma unroll
        for (int s = 0; s < ST; s++) {
            qf[s] = u32x4{0u, 0u, 0u, 0u};
            if (live && a.scale != 0.f) qf[s] = *reinterpret_cast<const u32x4 *>(q + 16 * s) ^ flip;
        }
    }
    // scores in units of log2 (more than 0, so that a masked score of -inf stays one; with a scale of 0 the queries are)
    const float scale = fmaxf(fabsf(a.scale) * 1.44269504088896f, 1e-37f);
    f32x16 acc[DT];
    float m_run = -INFINITY, l_run = 0.f, l_more = 0.f;      // the sum of weights, in two chains
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[d][e] = 0.f;

    // ---- staging: in pass x a wave's rows lie in one group of 16 keys, so in one page
    const int row_in = tid / LPR, c_in = tid % LPR;
    auto group_of = [&](int x) { return (x * RPP + wave * (64 / LPR)) >> 4; };
    auto here_mask = [&](int kt) { return (unsigned)(pages.here >> ((kt - base) * 4)) & 0xFu; };
    constexpr std::integral_constant<int, 0> K{};
    constexpr std::integral_constant<int, 1> V{};
    raw_t regs[2][NP];
    uint8_t scales[2][NP];
    const unsigned lane_at = ((wave * (64 / LPR)) & 15) * (DH * ES) + lane * LB;       // a lane's place in the 16 keys of its pass
    auto load = [&](int kt, auto side) {
        constexpr int S = decltype(side)::value;
        const int tile = min(kt, n_kt - 1);
#pragma unroll
        for (int x = 0; x < NP; x++) {
            const int from = (tile - base) * 4 + group_of(x);
            const size_t at = ((size_t)(unsigned)__builtin_amdgcn_readlane((int)(pages.at >> 32), from) << 32) | (unsigned)__builtin_amdgcn_readlane((int)pages.at, from);
            regs[S][x] = *reinterpret_cast<const raw_t *>(reinterpret_cast<const char *>(S ? p.v : p.k) + at + lane_at);
            if constexpr (F8) scales[S][x] = ((S ? p.vs : p.ks) + at / DH)[lane_at / DH];
        }
    };
    auto stage = [&](int buf, auto side) {
        constexpr int S = decltype(side)::value;
#pragma unroll
        for (int x = 0; x < NP; x++) {
            const int row = x * RPP + row_in;
            u32x4 v[W];
            if constexpr (F8) {
                const float f = pow2_of_byte(scales[S][x]);
#pragma unroll
                for (int w = 0; w < W; w++)
#pragma unroll
                    for (int y = 0; y < 2; y++) {
                        v[w][2 * y] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(regs[S][x][2 * w + y], f, false));
                        v[w][2 * y + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(regs[S][x][2 * w + y], f, true));
                    }
            } else {
                v[0] = regs[S][x];
            }
#pragma unroll
            for (int w = 0; w < W; w++) s_tiles[buf][S ? v_piece<DH>(row, W * c_in + w) : k_piece<DH>(row, W * c_in + w)] = v[w];
        }
    };
    // Where rows of the block, or places without a row, are among a tile's keys: values that no row attends are taken out of LDS again, and those
    // that are not finite (see odd_halves).  A thread looks at what it stored.
    auto mend = [&](int kt, int buf) {
        const int tile = min(kt, n_kt - 1);
        const unsigned here = here_mask(tile);
        if (tile * kKeys + kKeys <= seq.t && here == 0xFu) return;
        bool odd = false;
#pragma unroll
        for (int x = 0; x < NP; x++) {
            const int row = x * RPP + row_in;
            const bool out = tile * kKeys + row >= len || !((here >> group_of(x)) & 1u);
#pragma unroll
            for (int w = 0; w < W; w++) {
                u32x4 v = s_tiles[buf][v_piece<DH>(row, W * c_in + w)];
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    if (out) v[y] = 0u;
                    const uint32_t o = odd_halves(v[y]);
                    odd |= o != 0u;
                    v[y] &= ~o;
                }
                s_tiles[buf][v_piece<DH>(row, W * c_in + w)] = v;
            }
        }
        if (odd) s_odd = 1;
    };
    if (tid == 0) s_odd = 0;
    __syncthreads();
    load(0, K);
    load(0, V);
    stage(0, K);
    stage(2, V);
    mend(0, 2);
    load(1, K);
    load(1, V);

    const int wave_first = a.last(seq.t, (rt * BM + wave * 32) / a.group);      // last position that the wave's first row attends
    // where a lane reads: K row `col` (+ 32), pieces 2 s + h; V as LDS's transposing read wants it (the place of 4 features of a key), pieces 4 d + ..
    const int l16 = lane & 15;
    const int k_at = k_piece<DH>(col, h) * 16, v_row = 4 * h + (l16 >> 2);
    const int v_at = v_piece<DH>(v_row, 2 * ((lane >> 4) & 1) + ((l16 >> 1) & 1)) * 16 + 8 * (l16 & 1);
    // (said here, as otherwise the loop's first waits are for these loads, at every turn)
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0)
    __syncthreads();

    f32x16 st[2];
    bool sees = true;
    // the scores of tile kt, masked; the next tile to LDS
    auto scores = [&](int kt, int v_next) __attribute__((always_inline)) {
        const int key0 = kt * kKeys;
        if ((kt & 7) == 0 && kt != 0) {
            pages = pages_next;
            base = kt;
            pages_next = pages_from(kt + 8);
        }
        int ka_at = k_at + (kt & 1) * PIECES * 16;
        asm volatile("" : "+v"(ka_at));                      // (the xors below are made here, not kept in a register each)
        u32x4 ka[3][2];
        auto read_k = [&](int s) {
#pragma unroll
            for (int T2 = 0; T2 < 2; T2++)
                ka[s % 3][T2] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(&s_tiles[0][0]) + (ka_at ^ (32 * s)) + T2 * 32 * DH * 2);
        };
        read_k(0);
        read_k(1);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);                       // (nothing but matrix instructions: 415 us, without 421)
#pragma unroll
        for (int s = 0; s < ST; s++) {
            if (s + 2 < ST) read_k(s + 2);
            st[0] = mfma32(ka[s % 3][0], qf[s], s ? st[0] : f32x16{});
            __builtin_amdgcn_sched_barrier(0);
            st[1] = mfma32(ka[s % 3][1], qf[s], s ? st[1] : f32x16{});
            __builtin_amdgcn_sched_barrier(0);
            if (s == ST - 2) {
                stage((kt + 1) & 1, K);
                stage(2 + v_next, V);
                load(kt + 2, K);
                load(kt + 2, V);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        mend(kt + 1, 2 + v_next);
        // element e of half T2 is key 32 T2 + 8 (e / 4) + 4 h + e % 4
        const unsigned here = here_mask(kt);
        const bool whole = (a.parent ? key0 + kKeys <= seq.t : key0 + kKeys - 1 <= wave_first) && key0 + kKeys <= len && here == 0xFu;
        sees = true;
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
    };
    // its weights, and their products with the values
    auto products = [&](int v_this, auto planes) __attribute__((always_inline)) {
        constexpr bool TWO = decltype(planes)::value;        // weights in two bf16 planes
        int va_at = v_at + (2 + v_this) * PIECES * 16;
        asm volatile("" : "+v"(va_at));
        auto read_v = [&](int x) {                           // features 32 d .. of keys 16 u .., in the order of the weights
            const int u = x / DT, d = x % DT;
            uint64_t w[2];
#pragma unroll
            for (int y = 0; y < 2; y++) {
                char *at = reinterpret_cast<char *>(&s_tiles[0][0]) + (va_at ^ (64 * d)) + (16 * u + 8 * y) * DH * 2;
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
#pragma unroll
        for (int x = 0; x < 4 * DT; x++) {                   // the next 16 keys' weights are made beside the products of these
            const int u = x / DT, d = x % DT;
            if (x + 2 < 4 * DT) va[(x + 2) % 3] = read_v(x + 2);
            acc[d] = mfma32(va[x % 3], pw[u & 1], acc[d]);
            if constexpr (TWO) acc[d] = mfma32(va[x % 3], pl[u & 1], acc[d]);
            if (u < 3)
#pragma unroll
                for (int e = 0; e < 8 / DT; e += 2) weigh(8 * (u + 1) + 8 / DT * d + e);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int v_this = 0, v_next = 1;                              // tile kt modulo three, and kt + 1
    auto on = [&] {
        v_this = v_next;
        v_next = v_next == 2 ? 0 : v_next + 1;
    };
    auto tiles = [&](auto planes) __attribute__((always_inline)) {
        if (!late) {
#pragma unroll 1
            for (int kt = 0; kt < n_kt; kt++, on()) {
                scores(kt, v_next);
                products(v_this, planes);
                __syncthreads();
            }
        } else {
            scores(0, 1);
            __syncthreads();
#pragma unroll 1
            for (int kt = 1; kt < n_kt; kt++, on()) {
                products(v_this, planes);
                scores(kt, v_next == 2 ? 0 : v_next + 1);
                __syncthreads();
            }
            products(v_this, planes);
        }
    };
    if constexpr (CROSS) tiles(std::true_type{});
    else if (seq.m <= CSD_PAGED_FINE_ROWS) tiles(std::true_type{});
    else tiles(std::false_type{});
    __syncthreads();
    l_run = halves_sum(l_run + l_more);

    if (s_odd) {                                             // (uniform: the last tile was staged in front of a barrier)
        for (int key = 0; key < len; key++) {
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

    // ---- results: element e of acc[d] is feature 32 d + 8 (e / 4) + 4 h + e % 4 of the lane's row.  Turned in LDS, where the key tiles were (16-byte
    // pieces, their index xored by the row), so that whole rows are written one behind the other; each wave its own.
    constexpr int C = DH / 8;
    static_assert(BM * C <= 5 * PIECES, "");
    u32x4 *s_o = &s_tiles[0][0] + wave * 32 * C;
    int id = lane;
    asm volatile("" : "+v"(id));                             // (what follows from it is made here, not kept in registers all along)
    {
        const float inv = 1.f / l_run;
        const int row = id & 31;
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
            for (int y = 0; y < 4; y++) {
                u32x2 o = u32x2{pack_bf16x2(acc[d][4 * y] * inv, acc[d][4 * y + 1] * inv), pack_bf16x2(acc[d][4 * y + 2] * inv, acc[d][4 * y + 3] * inv)};
                if (m_run == -INFINITY) o = u32x2{0u, 0u};
                reinterpret_cast<u32x2 *>(&s_o[row * C + ((4 * d + y) ^ (row & (C - 1)))])[id >> 5] = o;
            }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int x = 0; x < 32 * C / 64; x++) {
        const int row = (x * 64 + id) / C, c = id % C;
        if (wave * 32 + row >= rows) continue;
        const int r_ = rt * BM + wave * 32 + row, i_ = r_ / a.group, h_ = r_ - i_ * a.group;
        *reinterpret_cast<u32x4 *>(reinterpret_cast<bf16_t *>(a.out) + (((size_t)(seq.start + i_) * p.Hkv + kvh) * a.group + h_) * DH + 8 * c) =
            s_o[row * C + (c ^ (row & (C - 1)))];
    }
}

void csd_paged_chunk_enqueue(const PagedAttn &a, int min_rows, int32_t pool_dtype, hipStream_t st) {
    // row tiles at most: full ones, and a last one per sequence that takes part
    const long long items = ((long long)a.r.rows * a.group / kChunkRows + csd_paged_batch(a, min_rows)) * a.p.Hkv;
    const bool f8 = pool_dtype == CSD_DTYPE_FP8;
    csd_paged_by_cross(a, [&](auto x) {
        constexpr bool CROSS = std::is_same<decltype(x), PagedAttnOf<true>>::value;
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)items), dim3(512), 0, st, x, min_rows); };
        if (a.p.D == 128) f8 ? launch(k_paged_attn_chunk<128, true, CROSS>) : launch(k_paged_attn_chunk<128, false, CROSS>);
        else f8 ? launch(k_paged_attn_chunk<64, true, CROSS>) : launch(k_paged_attn_chunk<64, false, CROSS>);
    });
}
