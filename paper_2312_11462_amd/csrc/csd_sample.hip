// Draws from logits by temperature, top-k, top-p and min-p, and the probabilities of such draws.
//
// With M the largest logit of a row and w_v = 2^((l_v - M) log2(e) / T), every weight is the whole number round(w_v 2^45): sums do not depend on their
// order, so neither do the sets that they bound nor the tokens (2^18 of them make 2^63, so sums have no sign; what weights of 64 bits would add to the sums decides
// for uniform numbers within 2^-38 or so of a border).  Tokens are ranked by (logit, lowest token first), which is the order of one 64-bit number, key << 32 | ~token.
// Each parameter keeps a start of the ranking, so together they keep the tokens from a least such number on:
//   top-k   the first k
//   top-p   of those the shortest start with at least p of their weight
//   min-p   of those the ones with w >= p
//
// A workgroup per row.  Three ways, by what a row asks for:
//   few tokens   a logit that all tokens that stay reach is known beforehand: the k-th largest of the lanes' own largest ones, or M + T ln(min-p).  The
//                tokens that reach it go to a list and are ranked, weighed and drawn there, each against each; no other weight is ever made.
//   a share      the weights of all tokens are added up in steps of 1/32 octave; the step that holds the border is ranked, or divided again by the bits of
//                its logits until few tokens are left or all are equal.  What stays is then a list as above or, if there are too many, goes
//   all          by the sum over the row, and the draw descends it: the wave's range that holds the border, a range of each wave in it, a tile.
// Memory bounds the first (656 rows of 50001 in bf16 into probabilities 46 us, 4.3 TB/s) or, for a row alone, its barriers and trips (one of 32000: 9 us, 6 of
// them in the workgroup: 1 to read it, 0.8 for the cut, 1.5 for the list, 2.7 to rank and draw).  The others are bound by the instructions of the weights, 24 a
// token in the histogram: of 256 rows of 32000 with top-p (36 us) 7.8 us are the histogram, 7 the border, 6 the sum, 2.6 the draw; of 131072 in bf16 (103 us, for the
// rows in which most tokens stay) 26, 26, 28 and 5.
#include "csd_epilogue.h"
#include "csd_lanes.h"

static constexpr int kList = 256;                            // tokens that are ranked against one another at most
static constexpr int kBins = 2048;                           // counters of a histogram
static constexpr int kPerOctave = 32, kSteps = 46 * kPerOctave + 1;      // steps of the weight, from M down (lower weights round to 0)
static constexpr float kMost = 3.402823466e38f;

struct SampleRows {
    const void *logits;
    long long stride;             // elements from one row to the next
    int V, each;                  // each: rows that share a set of parameters
    const float *u;
    int32_t *tokens;
    float *probs;
    const float *temperature, *top_p, *min_p;      // by set, or null: the numbers below
    const int32_t *top_k;
    float temperature_all, top_p_all, min_p_all;
    int32_t top_k_all;
    // Probabilities are stored past the caches where these would not hold what a review uses: p and q with the logits of both, so from 144 MiB of logits and
    // probabilities on.  us past and through them of p, q and accept, MiB of p, fp32, top-k and top-p: 16.6 33.0 and 33.4, 33 47 and 44, 54 56 and 51, 66 67.2 and 65.3,
    // 73 73 and 77, 87 78 and 99, 129 117 and 133; top-p alone: 33 94 and 92, 66 149 and 150, 73 163 and 171, 129 240 and 258; bf16 logits, top-k and top-p: 45 130 and 107,
    // 104 169 and 168, 114 177 and 180, 201 232 and 253.
    bool past;
};

// ---------------------------------------------------------------------------------------- numbers

// Logits are used as they are: NaN fails every comparison and has no weight, inf has that of the largest number of its type.
template <typename T> static constexpr float kLargest = sizeof(T) == 4 ? kMost : 3.3895313892515355e38f;
template <typename T>
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(fminf(v, kLargest<T>) + 0.f);     // (-0 is 0)
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
__device__ __forceinline__ u64 rank_of(uint32_t key, int v) { return (u64)key << 32 | (uint32_t)~v; }

__device__ __forceinline__ double fma_of(double a, double b, double c) {      // (the compiler makes two instructions of it, with c moved to the result first)
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
    return r;
}

// Weights of a row.  x = (l - M) c, c = log2(e) / T, is cut to [-48, 0] (NaN: -48); n = round(32 x) is minus the token's step, and with f = x - n / 32,
// |f| <= 1 / 64, 2^x = 2^(n / 32) 2^f: a table of 2^(i / 32) and the powers of ln 2 over the factorials up to the fifth (off by 2^-48).  About twenty instructions,
// five cycles each whatever they are, and they bound the passes that weigh every token.
struct Weights {
    double top, c;                // (c is at least 10^-300: -inf times it is -inf)
    const double *roots;          // 2^(i / 32), in LDS
    __device__ __forceinline__ double exponent(float l) const { return fmin(fmax(((double)l - top) * c, -48.0), 0.0); }
    static constexpr double kRound = 1.5 * (1ull << 47);     // a number of this size has steps of 1 / 32
    // -32 x, rounded: the low half of x + kRound
    static __device__ __forceinline__ int step(double x) { return -(int)(uint32_t)__double_as_longlong(x + kRound); }
    // 2^f, and 2^(n / 32)
    __device__ __forceinline__ void factors(double x, double &p, double &root) const {
        const double t = x + kRound, f = x - (t - kRound);
        const int n = (int)(uint32_t)__double_as_longlong(t);
        root = ldexp(roots[n & (kPerOctave - 1)], n >> 5);
        p = fma_of(f, 0.0013333558146428443, 0.009618129107628477);
        p = fma_of(p, f, 0.05550410866482158);
        p = fma_of(p, f, 0.2402265069591007);
        p = fma_of(p, f, 0.6931471805599453);
        p = fma(p, f, 1.0);
    }
    __device__ __forceinline__ double real(double x) const {
        double p, root;
        factors(x, p, root);
        return p * root;
    }
    // times 2^45, to the nearest whole number: 128 + w has steps of 2^-45
    static __device__ __forceinline__ u64 bits_of(double w) { return (u64)__double_as_longlong(w) & ((1ull << 52) - 1); }
    static __device__ __forceinline__ u64 whole(double w) { return bits_of(w + 128.0); }
    __device__ __forceinline__ u64 at(double x) const {
        double p, root;
        factors(x, p, root);
        return bits_of(fma(p, root, 128.0));
    }
    __device__ __forceinline__ u64 operator()(float l) const { return at(exponent(l)); }
    // A logit that every token within x octaves of M reaches, and few others; one that no token further down than x octaves passes.
    __device__ __forceinline__ float reach(float x) const {
        const double l = top - (double)x / c;
        return fmaxf((float)(l - fmax(fabs(l), fabs(top)) * 0x1p-20), -kMost);
    }
    __device__ __forceinline__ float below(float x) const {
        const double l = x > 0.f ? top - (double)x / c : top;
        return fminf((float)(l + fmax(fabs(l), fabs(top)) * 0x1p-20), kMost);
    }
};

// floor(a z) or, `up`, ceil(a z), for a in [0, 1)
__device__ __forceinline__ u64 share_of(float a, u64 z, bool up) {
    if (!(a > 0.f)) return 0;
    const uint32_t b = __float_as_uint(a), e = b >> 23;
    const uint32_t m = e ? (b & 0x7FFFFFu) | 0x800000u : b;
    const int s = 150 - (int)(e ? e : 1);                    // a = m 2^-s, s >= 24
    const unsigned __int128 y = (unsigned __int128)m * z;
    if (s >= 120) return up && z ? 1 : 0;
    const u64 q = (u64)(y >> s);
    return q + (up && ((unsigned __int128)q << s) != y ? 1 : 0);
}

// ---------------------------------------------------------------------------------------- lanes

__device__ __forceinline__ float wave_largest(float v) {
    auto step = [&](float o) { v = fmaxf(v, o); };
#define CSD_MOVED(CTRL, ROWS) __uint_as_float(moved<CTRL, ROWS>(__float_as_uint(v), __float_as_uint(v)))
    step(CSD_MOVED(0x111, 0xF));
    step(CSD_MOVED(0x112, 0xF));
    step(CSD_MOVED(0x114, 0xF));
    step(CSD_MOVED(0x118, 0xF));
    step(CSD_MOVED(0x142, 0xA));
    step(CSD_MOVED(0x143, 0xC));
#undef CSD_MOVED
    return __uint_as_float(from_lane(__float_as_uint(v), 63));
}

// ---------------------------------------------------------------------------------------- a row, by N threads

// Wave w has the w-th range of the row, tile by tile (a tile: 16 bytes of each lane).  NV tiles of a wave stay in registers, for the first passes, which do little with a
// token; the others read the row again.  (What a pass does is in the code once for each token of a tile, where the row is read, or of all NV: instructions that are not in
// their cache cost more than all of the row's bytes.)  NV = 0: all passes read.  V is at least VE, or the row is TINY.
template <typename T, int N, int NV, bool TINY = false>
struct Row {
    static constexpr int VE = 16 / sizeof(T), W = N / 64, TILE = 64 * VE;
    static constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;      // -inf
    const T *x;
    int V;
    u32x4 kept[NV ? NV : 1];

    // rows start at any element
    struct __attribute__((packed, aligned(sizeof(T)))) Raw {
        u32x4 v;
    };
    // This lane's piece of the tile that begins at `base`; -inf for tokens from V on.  (The wave's own branch: what the last tile takes would be four times the rest.)
    __device__ __forceinline__ u32x4 load(int base) const {
        const int at = base + (threadIdx.x & 63) * VE;
        if (!TINY && base + TILE <= V) return raw(at);
        u32x4 r{kNone, kNone, kNone, kNone};
        if (at >= V) return r;
        if constexpr (TINY) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (sizeof(T) == 4) {
                    r[i] = at + i < V ? __float_as_uint(x[at + i]) : 0xFF800000u;
                } else {
                    const uint32_t lo = at + 2 * i < V ? x[at + 2 * i] : 0xFF80u, hi = at + 2 * i + 1 < V ? x[at + 2 * i + 1] : 0xFF80u;
                    r[i] = lo | hi << 16;
                }
            }
            return r;
        }
        const int from = min(at, V - VE), s = at - from;     // the last piece is read from further ahead, and moved down
        r = raw(from);
        constexpr int D = 4 / (int)sizeof(T);                // tokens of a dword
        if (s & (2 * D)) r = u32x4{r[2], r[3], kNone, kNone};
        if (s & D) r = u32x4{r[1], r[2], r[3], kNone};
        if (D == 2 && (s & 1)) r = u32x4{r[0] >> 16 | r[1] << 16, r[1] >> 16 | r[2] << 16, r[2] >> 16 | r[3] << 16, r[3] >> 16 | kNone << 16};
        return r;
    }
    __device__ __forceinline__ u32x4 raw(int at) const { return reinterpret_cast<const Raw *>(reinterpret_cast<const char *>(x) + (uint32_t)at * (uint32_t)sizeof(T))->v; }
    static __device__ __forceinline__ float get(const u32x4 &r, int e) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(r[e]);
        else return __uint_as_float(e & 1 ? r[e / 2] & 0xFFFF0000u : r[e / 2] << 16);
    }
    // f(first token, piece) for this lane's pieces of VE tokens of the tiles from lo to hi, the next one on its way; lo and hi are the wave's
    template <typename F>
    __device__ __forceinline__ void pieces(int lo, int hi, F f) const {
        if (lo >= hi) return;
        u32x4 next = load(lo);
#pragma unroll 1
        for (; lo < hi; lo += TILE) {
            const u32x4 r = next;
            if (lo + TILE < hi) next = load(lo + TILE);
            f(lo + (int)(threadIdx.x & 63) * VE, r);
        }
    }
    // f(token, logit); tokens from V on have -inf
    template <typename F>
    __device__ __forceinline__ void tokens(int lo, int hi, F f) const {
        pieces(lo, hi, [&](int at, const u32x4 &r) {
#pragma unroll
            for (int e = 0; e < VE; e++) f(at + e, get(r, e));
        });
    }
    // tokens of a wave's range of n
    static __device__ __forceinline__ int range(int n) { return (n + W * TILE - 1) / (W * TILE) * TILE; }
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    template <typename F>
    __device__ __forceinline__ void all(F f) const {
        const int c = range(V);
        tokens(min(wave() * c, V), min(wave() * c + c, V), f);
    }
    __device__ __forceinline__ void keep() {
        if constexpr (NV > 0) {
            const int c = range(V);
#pragma unroll
            for (int j = 0; j < NV; j++) {
                kept[j] = u32x4{kNone, kNone, kNone, kNone};
                if (j * TILE < c && wave() * c + j * TILE < V) kept[j] = load(wave() * c + j * TILE);
            }
        }
    }
    // passes that do little with a token: from registers, or with four tiles on their way
    template <typename F>
    __device__ __forceinline__ void all_pieces(F f) const {
        const int c = range(V), lo = wave() * c;
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; j++) {
                u32x4 r = kept[j];
                asm volatile("" : "+v"(r));                  // (nothing that one pass makes of them is kept for the next)
                if (j * TILE < c) f(lo + j * TILE + (int)(threadIdx.x & 63) * VE, r);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            constexpr int AHEAD = 4;
            const int hi = min(lo + c, V);
#pragma unroll 1
            for (int base = lo; base < hi; base += AHEAD * TILE) {
                u32x4 r[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; j++)
                    if (base + j * TILE < hi) r[j] = load(base + j * TILE);
#pragma unroll
                for (int j = 0; j < AHEAD; j++)
                    if (base + j * TILE < hi) f(base + j * TILE + (int)(threadIdx.x & 63) * VE, r[j]);
            }
        }
    }
};

struct Ranked {
    u64 rank, mass;
};

struct SampleShared {
    Ranked list[kList];
    u64 mass[kBins];
    uint32_t count[kBins], octave[64];
    u64 stay_mass[kList];
    double roots[kPerOctave];
    u64 part[16];
    uint32_t part32[16], about[16];
    float top[16];
    uint32_t n_list;
    u64 least, sum, stay;
    int token;
};

template <int N>
__device__ __forceinline__ void clear_counters(SampleShared &S) {
    for (int i = threadIdx.x; i < kBins / 4; i += N) reinterpret_cast<u32x4 *>(S.count)[i] = u32x4{0u, 0u, 0u, 0u};
    for (int i = threadIdx.x; i < kBins / 2; i += N) reinterpret_cast<u32x4 *>(S.mass)[i] = u32x4{0u, 0u, 0u, 0u};
    if (threadIdx.x < 64) S.octave[threadIdx.x] = 0;
}

// A counter of the histogram: what it has, and what lies before it.
struct Found {
    int bin;                      // kBins: none
    uint32_t base_count, count;
    u64 base_mass, mass;
    uint32_t about;               // a histogram of weights: sixteen times the tokens that there are likely up to the end of its lane's counters
};
// About how many tokens a step of so much weight has (within a percent or so: their weights are).
__device__ __forceinline__ float likely(u64 mass, int step) { return (float)mass * __builtin_amdgcn_exp2f((float)step / kPerOctave - 45.f); }

// The waves' sums of the counters (wave w: its kBins / W ones); a barrier behind it.
template <int N>
__device__ __forceinline__ void sum_counters(SampleShared &S) {
    constexpr int B = kBins / N;
    uint32_t n = 0;
    u64 m = 0;
    float some = 0.f;
#pragma unroll
    for (int i = 0; i < B; i++) {
        const u64 mass = S.mass[threadIdx.x * B + i];
        n += S.count[threadIdx.x * B + i];
        m += mass;
        some += likely(mass, threadIdx.x * B + i);
    }
    n = wave_total(n);
    m = wave_total(m);
    const uint32_t about = wave_total((uint32_t)(some * 16.f));      // (in sixteenths)
    if ((threadIdx.x & 63) == 0) {
        S.part32[threadIdx.x >> 6] = n;
        S.part[threadIdx.x >> 6] = m;
        S.about[threadIdx.x >> 6] = about;
    }
    __syncthreads();
}
// The first counter at which k tokens, or m of weight, are reached; every wave finds it by itself.
template <int N>
__device__ __forceinline__ Found find(const SampleShared &S, uint32_t k, u64 m) {
    constexpr int B = kBins / N, W = N / 64;
    const int lane = threadIdx.x & 63;
    Found f{kBins, 0, 0, 0, 0, 0};
    int w = 0;
    for (; w < W; w++) {
        const uint32_t n = uniform(S.part32[w]);
        const u64 x = uniform(S.part[w]);
        if (f.base_count + n >= k || f.base_mass + x >= m) break;
        f.base_count += n;
        f.base_mass += x;
        f.about += uniform(S.about[w]);
    }
    if (w == W) return f;
    uint32_t count[B], n = 0;
    u64 mass[B], x = 0;
    float some = 0.f;
#pragma unroll
    for (int i = 0; i < B; i++) {
        count[i] = S.count[(w * 64 + lane) * B + i];
        mass[i] = S.mass[(w * 64 + lane) * B + i];
        n += count[i];
        x += mass[i];
        some += likely(mass[i], (w * 64 + lane) * B + i);
    }
    const uint32_t part = (uint32_t)(some * 16.f);
    const uint32_t to = f.base_count + wave_scan(n);
    const u64 mass_to = f.base_mass + wave_scan(x);
    const int hit = __ffsll((long long)__ballot(to >= k || mass_to >= m)) - 1;
    uint32_t before = to - n, at = 0, mine = 0;
    u64 mass_before = mass_to - x, mass_mine = 0;
    bool there = false;
#pragma unroll
    for (int i = 0; i < B; i++)
        if (!there) {
            there = before + count[i] >= k || mass_before + mass[i] >= m;
            if (there) {
                at = i;
                mine = count[i];
                mass_mine = mass[i];
            } else {
                before += count[i];
                mass_before += mass[i];
            }
        }
    return Found{(w * 64 + hit) * B + (int)from_lane(at, hit), from_lane(before, hit), from_lane(mine, hit), from_lane(mass_before, hit), from_lane(mass_mine, hit),
                 f.about + from_lane(wave_scan(part), hit)};
}

// The lowest token of [lo, hi) at which the running sum of value(token, logit), from lo on, passes `target`; the sum over the range is more than that.
template <typename R, typename F>
__device__ __forceinline__ int descend(const R &row, SampleShared &S, u64 target, int lo, int hi, F value) {
    using U = decltype(value(0, 0.f));
    const int lane = threadIdx.x & 63, wave = R::wave();
    while (hi - lo > R::TILE) {
        const int c = R::range(hi - lo), a = min(lo + wave * c, hi), b = min(a + c, hi);
        U sum = 0;
        row.tokens(a, b, [&](int v, float l) { sum += value(v, l); });
        sum = wave_total(sum);
        __syncthreads();
        if (lane == 0) S.part[wave] = sum;
        __syncthreads();
        int w = 0;
        for (; w < R::W - 1 && uniform(S.part[w]) <= target; w++) target -= uniform(S.part[w]);
        lo = min(lo + w * c, hi - 1);
        hi = min(lo + c, hi);
    }
    __syncthreads();
    if (wave == 0) {
        u64 mine[R::VE], sum = 0;
        const int at = lo + lane * R::VE;
        const u32x4 r = row.load(lo);
#pragma unroll
        for (int e = 0; e < R::VE; e++) {
            mine[e] = value(at + e, R::get(r, e));
            sum += mine[e];
        }
        const u64 incl = wave_scan(sum), past = __ballot(incl > target);
        if (past && lane == __ffsll((long long)past) - 1) {
            u64 run = incl - sum;
            int e = 0;
#pragma unroll
            for (int i = 0; i < R::VE - 1; i++) {
                run += mine[i];
                e += run <= target ? 1 : 0;
            }
            S.token = at + e;
        }
    }
    __syncthreads();
    return S.token;
}

// a && b without a branch between them
__device__ __forceinline__ bool both(bool a, bool b) { return ((int)a & (int)b) != 0; }

// The tokens with logits of [from, to] for which in(logit) holds to the list, by no order: how many; more than kList: too many.
template <typename T, typename R, typename F>
__device__ __forceinline__ uint32_t collect(const R &row, SampleShared &S, float from, float to, F in) {
    __syncthreads();
    if (threadIdx.x == 0) S.n_list = 0;
    __syncthreads();
    row.all_pieces([&](int at, const u32x4 &r) {
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < R::VE; e++) hits |= both(R::get(r, e) >= from, R::get(r, e) <= to) ? 1u << e : 0u;
        while (hits) {
            const int e = __ffs(hits) - 1;
            hits &= hits - 1;
            constexpr int D = 4 / (int)sizeof(T);
            const int d = e / D;
            const uint32_t w = d & 2 ? d & 1 ? r[3] : r[2] : d & 1 ? r[1] : r[0];
            const float l = __uint_as_float(D == 1 ? w : e & 1 ? w & 0xFFFF0000u : w << 16);
            if (!in(l)) continue;
            const uint32_t i = atomicAdd(&S.n_list, 1u);
            if (i < (uint32_t)kList) S.list[i].rank = rank_of(key_of<T>(l), at + e);
        }
    });
    __syncthreads();
    return uniform(S.n_list);
}

// f(token, logit) for the tokens of the waves' ranges for which stays(first token of the piece, place in it, logit) holds, 64 at a time: a weight takes two to three
// times what the look and a queue in LDS take, and of a vocabulary with a border few tokens stay (256 rows of 131072 in bf16, top-p: the sum 19 us, 28 over all
// tokens).  The queues lie where the counters were.
template <typename R, typename STAYS, typename F>
__device__ __forceinline__ void gather(const R &row, SampleShared &S, STAYS stays, F f) {
    static_assert(sizeof(S.mass) >= R::W * 128 * sizeof(u64), "");
    const int lane = threadIdx.x & 63, wave = R::wave(), c = R::range(row.V);
    u64 *queue = S.mass + wave * 128;                        // a ring: from `head` on, `n` tokens
    int head = 0, n = 0;
    auto one = [&](u64 t) { f((int)(uint32_t)(t >> 32), __uint_as_float((uint32_t)t)); };
    row.pieces(min(wave * c, row.V), min(wave * c + c, row.V), [&](int at, const u32x4 &r) {
#pragma unroll
        for (int e = 0; e < R::VE; e++) {
            const float l = R::get(r, e);
            const bool in = stays(at, e, l);
            const u64 mask = __builtin_amdgcn_ballot_w64(in);
            const int place = head + n + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
            if (in) queue[place & 127] = (u64)(uint32_t)(at + e) << 32 | __float_as_uint(l);
            n += __popcll(mask);
            if (n >= 64) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                one(queue[(head + lane) & 127]);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                head = (head + 64) & 127;
                n -= 64;
            }
        }
    });
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (lane < n) one(queue[(head + lane) & 127]);
}

// A token of the list, by N / kList neighbouring lanes: its weight (which goes to the list), and how many tokens and how much weight rank ahead of it.
template <int N>
struct Listed {
    static constexpr int G = N / kList;
    u64 rank, mass, run;
    double real;
    uint32_t ahead;
    bool there, first;
    __device__ __forceinline__ int token() const { return (int)~(uint32_t)rank; }
    template <typename F>
    static __device__ __forceinline__ void others(uint32_t n, F f) {
#pragma unroll 4
        for (uint32_t j = threadIdx.x % G; j < n; j += G) f(j);
    }
    template <typename U>
    static __device__ __forceinline__ void join(U &v) {
#pragma unroll
        for (int o = 1; o < G; o <<= 1) v += __shfl_xor(v, o, 64);
    }
    __device__ __forceinline__ Listed(SampleShared &S, const Weights &weight, uint32_t n) {
        const int i = threadIdx.x / G;
        there = i < (int)n;
        first = threadIdx.x % G == 0;
        rank = there ? S.list[i].rank : 0;
        real = there ? weight.real(weight.exponent(logit_of((uint32_t)(rank >> 32)))) : 0.0;
        mass = Weights::whole(real);
        if (there && first) S.list[i].mass = mass;
        if (threadIdx.x == 0) {
            S.sum = S.stay = 0;
            S.least = ~0ull;
        }
        __syncthreads();
        ahead = 0;
        run = 0;
        others(n, [&](uint32_t j) {
            const Ranked o = S.list[j];
            const bool higher = o.rank > rank;
            ahead += higher ? 1 : 0;
            run += higher ? o.mass : 0;
        });
        join(ahead);
        join(run);
    }
};

// sum += v of all lanes, by every wave
__device__ __forceinline__ void add(u64 &sum, u64 v) {
    v = wave_total(v);
    if (v && (threadIdx.x & 63) == 0) atomicAdd(&sum, v);
}

// Parameters of a row, as the ranking takes them.
struct Limits {
    uint32_t k;                   // tokens
    float p;                      // by_mass: share of the weight of the first k
    bool by_mass;
    u64 w_min;
};

// The draw's place in the sum of weights.
__device__ __forceinline__ u64 place_of(float u, u64 sum) { return min(share_of(fminf(u, 0.99999994f), sum, false), sum - 1); }

// The list holds all tokens that stay: their probabilities (over zeros) and the draw.  `all`: the weight that top-p is a share of, 0: that of the first k.
template <int N>
__device__ __forceinline__ void finish(SampleShared &S, const Weights &weight, const Limits &lim, u64 all, uint32_t n, float *out, float u, int32_t *token) {
    const Listed<N> t(S, weight, n);
    bool stays = t.there && t.ahead < lim.k;
    if (lim.by_mass) {
        if (!all) {
            add(S.sum, stays && t.first ? t.mass : 0);
            __syncthreads();
            all = S.sum;
        }
        stays = stays && (t.ahead == 0 || t.run < share_of(lim.p, all, true));
    }
    stays = stays && t.mass >= lim.w_min;
    if (t.first) S.stay_mass[threadIdx.x / Listed<N>::G] = stays ? t.mass : 0;
    add(S.stay, stays && t.first ? t.mass : 0);
    __syncthreads();
    const u64 sum = S.stay;
    if (out && stays && t.first) out[t.token()] = (float)(t.real * (1.0 / ((double)sum * 0x1p-45)));
    if (token) {
        const u64 target = place_of(u, sum);
        u64 before = 0;
        Listed<N>::others(n, [&](uint32_t j) { before += (uint32_t)S.list[j].rank > (uint32_t)t.rank ? S.stay_mass[j] : 0; });
        Listed<N>::join(before);
        if (stays && t.first && before <= target && target < before + t.mass) *token = t.token();
    }
}

// The border of the first k tokens, or of m of weight, lies in step f.bin: the rank of the last token inside, and the weight inside.
// True: the counters have been used.
template <typename T, int N, typename R>
__device__ __forceinline__ bool border(const R &row, SampleShared &S, const Weights &weight, uint32_t k, u64 m, Found f, u64 &least, u64 &inside) {
    // its logits lie between two keys; those of bf16 logits are their upper halves
    constexpr int LOW = sizeof(T) == 4 ? 0 : 16;
    const int step = f.bin;
    uint32_t lo = uniform(key_of<T>(weight.reach(((float)step + 0.5f) / kPerOctave)) >> LOW), hi = uniform(key_of<T>(weight.below(((float)step - 0.5f) / kPerOctave)) >> LOW);
    auto full_key = [&](uint32_t key) { return LOW && !(key >> 15) ? key << LOW | 0xFFFFu : key << LOW; };       // (keys of negative numbers are turned around)
    float from, to;
    auto between = [&] {
        if (hi == 0x7FFFFFFFu >> LOW) hi--;                  // (-0, which no token's key is)
        lo = min(lo, hi);
        from = logit_of(full_key(lo));
        to = logit_of(full_key(hi));
        if (to == kLargest<T>) to = INFINITY;
    };
    bool all_in = false;                                     // all numbers between them are the step's
    auto in = [&](float l) { return all_in || Weights::step(weight.exponent(l)) == step; };
    // (bf16: a step has few numbers in it, if not one)
    if (hi - lo < 64) {
        const uint32_t key = lo + (threadIdx.x & 63);
        const u64 some = __ballot(key <= hi && Weights::step(weight.exponent(logit_of(full_key(key)))) == step);
        if (some) {
            hi = uniform(lo + 63 - __clzll((long long)some));
            lo = uniform(lo + __ffsll((long long)some) - 1);
            all_in = true;
        }
    }
    between();
    uint32_t base = f.base_count;
    u64 base_mass = f.base_mass;
    // (as many as are likely, if they were not counted)
    uint32_t n = uniform(f.count ? f.count : (uint32_t)likely(f.mass, step));
    if (n <= (uint32_t)kList) n = collect<T>(row, S, from, to, in);
    const bool used = n > (uint32_t)kList;
    if (used && hi - lo < 3 && to < INFINITY) {
        // Many tokens of three numbers at most (bf16, mostly): how many each wave has of each is known after one pass, and so where the border lies among equal ones
        // (256 rows of 131072 in bf16, top-p: 25 us by the keys as below).
        float number[3];
        uint32_t have[3] = {0, 0, 0};
#pragma unroll
        for (int i = 0; i < 3; i++) number[i] = uniform(hi - lo >= (uint32_t)i && hi - i != 0x7FFFFFFFu >> LOW ? logit_of(full_key(hi - i)) : NAN);      // (-0 is 0)
        row.all_pieces([&](int, const u32x4 &r) {
#pragma unroll
            for (int e = 0; e < R::VE; e++)
#pragma unroll
                for (int i = 0; i < 3; i++) have[i] += __popcll(__builtin_amdgcn_ballot_w64(R::get(r, e) == number[i]));
        });
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 3; i++)
            if ((threadIdx.x & 63) == 0) S.count[i * R::W + R::wave()] = have[i];
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < 3 && hi - lo >= (uint32_t)i; i++) {
            const float l = logit_of(full_key(hi - i));
            const u64 w = weight(l);
            uint32_t all = 0;
            for (int x = 0; x < R::W; x++) all += uniform(S.count[i * R::W + x]);
            if (base + all < k && base_mass + all * w < m) {
                base += all;
                base_mass += all * w;
                continue;
            }
            u64 keep = k - base;
            if (w) keep = min(keep, (m - base_mass - 1) / w + 1);      // (m is more than base_mass)
            keep = uniform(max(keep, (u64)1));
            uint32_t before = 0;
            int x = 0;
            for (; x < R::W - 1 && before + uniform(S.count[i * R::W + x]) < keep; x++) before += uniform(S.count[i * R::W + x]);
            const int c = R::range(row.V);
            const int last = descend(row, S, keep - 1 - before, min(x * c, row.V - 1), min(x * c + c, row.V), [&](int, float v) { return v == l ? 1u : 0u; });
            least = uniform(rank_of(full_key(hi - i), last));
            inside = uniform(base_mass + keep * w);
            return true;
        }
    }
    while (n > (uint32_t)kList) {
        if (lo == hi) {
            // all equal: the first of them by token
            const u64 w = weight(from);
            u64 keep = k - base;
            if (w) keep = min(keep, (m - base_mass - 1) / w + 1);      // (m is more than base_mass)
            keep = max(keep, (u64)1);
            const int last = descend(row, S, keep - 1, 0, row.V, [&](int, float l) { return both(l >= from, l <= to) ? 1u : 0u; });
            least = uniform(rank_of(full_key(lo), last));
            inside = uniform(base_mass + keep * w);
            return true;
        }
        const int shift = max(0, 32 - __clz(hi - lo) - 11);  // 2^11 steps of keys at most
        __syncthreads();
        clear_counters<N>(S);
        __syncthreads();
        row.all([&](int, float l) {
            if (both(l >= from, l <= to) && in(l)) {
                const uint32_t key = key_of<T>(l) >> LOW;    // (between lo and hi, so less than 2^11 steps from it)
                if (key < lo || key > hi) return;
                atomicAdd(&S.count[(hi - key) >> shift], 1u);
                if (shift) atomicAdd(&S.mass[(hi - key) >> shift], weight(l));
            }
        });
        __syncthreads();
        if (shift == 0) {                                    // (a number each: its tokens weigh alike)
            for (uint32_t i = threadIdx.x; i <= hi - lo; i += N) S.mass[i] = S.count[i] ? S.count[i] * weight(logit_of(full_key(hi - i))) : 0;
            __syncthreads();
        }
        sum_counters<N>(S);
        f = find<N>(S, k - base, m - base_mass);
        if (f.bin == kBins) break;                           // (the logits changed while they were read)
        base += f.base_count;
        base_mass += f.base_mass;
        hi -= (uint32_t)f.bin << shift;
        lo = max(lo, hi - min(hi, (1u << shift) - 1));
        between();
        n = f.count;
        if (n <= (uint32_t)kList) n = collect<T>(row, S, from, to, in);
    }
    const Listed<N> t(S, weight, min(n, (uint32_t)kList));
    if (t.there && t.first && base + t.ahead < k && base_mass + t.run < m) {
        atomicMin(&S.least, t.rank);
        atomicAdd(&S.sum, t.mass);
    }
    __syncthreads();
    least = uniform(S.least);
    inside = uniform(base_mass + S.sum);
    return used;
}

// Four probabilities of a row from token v on; `past`: past the caches.
__device__ __forceinline__ void store_quad(__amdgpu_buffer_rsrc_t row, int v, f32x4 p, bool past) {
    if (past) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, p), row, 4 * v, 0, 2);      // (2: not to be kept)
    else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, p), row, 4 * v, 0, 0);
}

template <typename T, int N, int NV, bool TINY>
__global__ __launch_bounds__(N, 4) void k_sample(SampleRows a) {
    __shared__ __align__(16) SampleShared S;
    using R = Row<T, N, NV, TINY>;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = R::wave(), set = r / a.each;
    R row;
    row.x = reinterpret_cast<const T *>(a.logits) + (size_t)r * a.stride;
    row.V = a.V;
    row.keep();
    const float temperature = uniform(a.temperature ? a.temperature[set] : a.temperature_all), p = uniform(a.top_p ? a.top_p[set] : a.top_p_all),
                p_min = uniform(a.min_p ? a.min_p[set] : a.min_p_all), u = uniform(a.tokens ? a.u[r] : 0.f);
    const bool greedy = !(temperature > 0.f);
    int k = greedy ? 1 : __builtin_amdgcn_readfirstlane(a.top_k ? a.top_k[set] : a.top_k_all);
    if (k <= 0 || k > a.V) k = a.V;
    clear_counters<N>(S);
    if (tid < kPerOctave) S.roots[tid] = exp2((double)tid / kPerOctave);

    float mine = -INFINITY;
    row.all_pieces([&](int, const u32x4 &piece) {
#pragma unroll
        for (int e = 0; e < R::VE; e++) mine = fmaxf(mine, __builtin_canonicalizef(R::get(piece, e)));      // (a signalling NaN would be what v_max_f32 gives)
    });
    mine = fminf(mine, kLargest<T>);
    float top = wave_largest(mine);
    if (lane == 0) S.top[wave] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N / 64; i++) top = fmaxf(top, S.top[i]);
    top = uniform(top);
    float *out = a.probs ? a.probs + (size_t)r * a.V : nullptr;
    const __amdgpu_buffer_rsrc_t out_row = ch_rsrc(out, (size_t)a.V * 4);
    int32_t *token = a.tokens ? a.tokens + r : nullptr;
    auto clear = [&] {
        for (int i = 4 * tid; i < a.V; i += 4 * N)
            if (i + 4 <= a.V) store_quad(out_row, i, f32x4{0.f, 0.f, 0.f, 0.f}, a.past);
            else
                for (int e = i; e < a.V; e++) out[e] = 0.f;
    };
    if (top == -INFINITY) {                                  // nothing to draw from
        if (out) clear();
        if (token && tid == 0) *token = -1;
        return;
    }
    const Weights weight{(double)top, fmax(1.4426950408889634 / (greedy ? 1.0 : (double)temperature), 1e-300), S.roots};
    Limits lim{(uint32_t)k, p, p < 1.f && k > 1, 1};
    if (p_min > 0.f) lim.w_min = uniform(max((u64)ceil((double)fminf(p_min, 1.f) * (double)(1ull << 45)), (u64)1));

    // ---- few tokens at most
    // (What the list takes in is k tokens and some more: the others of k's step, and of the lanes whose largest ones were counted.  For larger k it would overflow
    // too often, and the row starts over: us for top-k 180, 192 and 193 of a row of 32000 13.8, 14.0 and 23.5, of 656 of 50001 in bf16 46, 75 and 84.)
    const bool few = k <= kList * 3 / 4;
    if (few || (k == a.V && !lim.by_mass && p_min > 0.f)) {
        float cut = -kMost;
        if (k == 1) {
            cut = top;
        } else if (few) {
            const int i = Weights::step(weight.exponent(mine));
            if (i < kSteps) {
                atomicAdd(&S.count[i], 1u);
                atomicAdd(&S.octave[i >> 5], 1u);
            }
            __syncthreads();
            // (every wave finds the k-th by itself: the octave, then the step)
            const uint32_t o = S.octave[lane], to = wave_scan(o);
            const u64 past = __ballot(to >= (uint32_t)k);
            if (past) {
                const int at = __ffsll((long long)past) - 1;
                const uint32_t before = from_lane(to - o, at), in = before + wave_scan(lane < 32 ? S.count[at * 32 + lane] : 0u);
                const int step = at * 32 + __ffsll((long long)__ballot(in >= (uint32_t)k)) - 1;
                cut = weight.reach(((float)step + 0.5f) / kPerOctave);
            } else {
                cut = weight.reach(46.5f);                   // (fewer lanes have a token with a weight)
            }
        }
        if (!lim.by_mass && p_min > 0.f) cut = fmaxf(cut, weight.reach(-__builtin_amdgcn_logf(fminf(p_min, 1.f)) * 1.0001f + 0.001f));      // (log2)
        if (out) clear();
        const uint32_t n = collect<T>(row, S, cut, INFINITY, [](float) { return true; });
        if (n <= (uint32_t)kList) return finish<N>(S, weight, lim, 0, n, out, u, token);
        clear_counters<N>(S);
        __syncthreads();
    }

    // ---- by many tokens, or by a share of the weight (from here on the row is read again; what is kept of it would cost the registers of these passes)
    const Row<T, N, 0, TINY> again{row.x, row.V, {}};
    u64 least = 0, sum = 0;
    const bool counted = k < a.V;
    bool stand = false;                                      // the counters hold the histogram
    uint32_t likely_stay = (uint32_t)a.V;
#pragma unroll 1
    for (int pass = 0; pass < 2; pass++) {
        if (pass ? !lim.by_mass : !counted) continue;
        if (!stand) {
            again.all([&](int, float l) {
                const double x = weight.exponent(l);
                const int i = Weights::step(x);
                const u64 w = weight.at(x);
                if (i < kSteps) {
                    if (counted) atomicAdd(&S.count[i], 1u);
                    atomicAdd(&S.mass[i], w);
                }
            });
            __syncthreads();
            sum_counters<N>(S);
            stand = true;
            if (!sum)
#pragma unroll
                for (int i = 0; i < N / 64; i++) sum += uniform(S.part[i]);
        }
        const uint32_t first = pass ? ~0u : (uint32_t)k;
        const u64 m = pass ? uniform(max(share_of(p, sum, true), (u64)1)) : ~0ull;
        const Found f = find<N>(S, first, m);
        if (f.bin >= kSteps) continue;                       // (all tokens with a weight)
        // what stays may fit the list: all tokens down to the end of the step
        const float cut = weight.reach(((float)f.bin + 0.5f) / kPerOctave);
        const uint32_t about = counted ? f.base_count + f.count : f.about / 16;
        likely_stay = about;
        if (about <= (uint32_t)kList + kList / 8) {
            const uint32_t n = collect<T>(again, S, cut, INFINITY, [](float) { return true; });
            if (n <= (uint32_t)kList) {
                if (out) clear();
                __syncthreads();
                return finish<N>(S, weight, lim, pass ? sum : 0, n, out, u, token);
            }
        }
        stand = !border<T, N>(again, S, weight, first, m, f, least, sum);
        if (!stand) {
            __syncthreads();
            clear_counters<N>(S);
            __syncthreads();
        }
    }

    // ---- all
    const float l_least = least ? logit_of((uint32_t)(least >> 32)) : -INFINITY;
    const float l_above = l_least == kLargest<T> ? INFINITY : l_least;   // (inf counts as that)
    const int v_last = (int)~(uint32_t)least;                // of the tokens with the least logit
    auto stays = [&](int at, int e, float l) { return !both(!(l > l_above), !both(l >= l_least, e <= v_last - at)); };
    const bool bounded = lim.w_min > 1;
    auto value = [&](int v, float l) -> u64 {
        const u64 w = weight(l);
        if (bounded) return both(stays(v, 0, l), w >= lim.w_min) ? w : 0;
        return stays(v, 0, l) ? w : 0;
    };
    const bool seldom = least && likely_stay * 3 < (uint32_t)a.V;      // (one in three: as fast either way)
    const int range = R::range(a.V);
    if (token || !sum || bounded) {
        u64 of_wave = 0;
        auto weigh = [&](int, float l) {
            const u64 w = weight(l);
            of_wave += w >= lim.w_min ? w : 0;
        };
        if (seldom) {
            __syncthreads();                                 // (the counters have been read)
            gather(again, S, stays, weigh);
        } else if (least || bounded) {
            again.all([&](int v, float l) { of_wave += value(v, l); });
        } else {
            again.all([&](int, float l) { of_wave += weight(l); });
        }
        of_wave = wave_total(of_wave);
        __syncthreads();
        if (lane == 0) S.part[wave] = of_wave;
        __syncthreads();
        sum = 0;
#pragma unroll
        for (int i = 0; i < N / 64; i++) sum += uniform(S.part[i]);
    }
    const double inv = 1.0 / ((double)sum * 0x1p-45);
    if (out && seldom) {
        clear();
        __syncthreads();                                     // (zeros before probabilities; and the counters have been read)
        gather(again, S, stays, [&](int v, float l) {
            const double w = weight.real(weight.exponent(l));
            if (Weights::whole(w) >= lim.w_min) out[v] = (float)(w * inv);
        });
    } else if (out) {
        again.pieces(min(wave * range, a.V), min(wave * range + range, a.V), [&](int at, const u32x4 &raw) {
            float y[R::VE];
#pragma unroll
            for (int e = 0; e < R::VE; e++) {
                const float l = R::get(raw, e);
                const double w = weight.real(weight.exponent(l));
                y[e] = both(stays(at, e, l), Weights::whole(w) >= lim.w_min) ? (float)(w * inv) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < R::VE; e += 4)
                if (at + e + 4 <= a.V) store_quad(out_row, at + e, f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]}, a.past);
                else
#pragma unroll
                    for (int i = 0; i < 3; i++)
                        if (at + e + i < a.V) out[at + e + i] = y[e + i];
        });
    }
    if (token) {
        u64 target = uniform(place_of(u, sum));
        int w = 0;
        for (; w < N / 64 - 1 && uniform(S.part[w]) <= target; w++) target -= uniform(S.part[w]);
        const int found = descend(again, S, target, min(w * range, a.V - 1), min(w * range + range, a.V), value);
        if (tid == 0) *token = found;
    }
}

// ---------------------------------------------------------------------------------------- entry points

template <typename T, int N, int NV, bool TINY = false>
static void sample_launch_as(const SampleRows &a, int rows, hipStream_t st) {
    hipLaunchKernelGGL((k_sample<T, N, NV, TINY>), dim3(rows), dim3(N), 0, st, a);
}

// The row stays in registers where it fits them.  A workgroup of 1024 threads has a compute unit to itself, of 512 and 256 two and four share one: the more threads the sooner a
// row is done, the more rows at once the less of the chip waits at a row's barriers.  us by 1024 threads and by 512, rows of 32000: 200 with top-k 14.2 and 16.3, 300 22.2 and 20.5,
// 200 with top-p 35.5 and 40.6, 400 61.3 and 57.3, 500 67.4 and 59.1.  By 256 and by 512, short rows: one of 512 10.4 and 7.9, 64 of 4000 22.2 and 14.9, 300 of 2000 26.3 and
// 17.4, 1000 of 512 23.4 and 25.9, 3000 of 2000 56 and 68 (1000 of 4000 35.9 and 30.9).
template <typename T>
static void sample_launch(const SampleRows &a, int rows, hipStream_t st) {
    constexpr int VE = 16 / sizeof(T);
    if (a.V < VE) sample_launch_as<T, 256, 1, true>(a, rows, st);
    else if (a.V <= 256 * 4 * VE && rows > 512) sample_launch_as<T, 256, 4>(a, rows, st);
    else if (a.V <= 256 * 4 * VE) sample_launch_as<T, 512, 8>(a, rows, st);
    else if (a.V <= 512 * 16 * VE && rows > 256) sample_launch_as<T, 512, 16>(a, rows, st);
    else if (a.V <= 1024 * 8 * VE) sample_launch_as<T, 1024, 8>(a, rows, st);
    else if (a.V <= 1024 * 16 * VE) sample_launch_as<T, 1024, 16>(a, rows, st);
    else sample_launch_as<T, 1024, 0>(a, rows, st);
}

static int32_t sample_enqueue(const csd_filter *f, const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t V, const float *u,
                              int32_t *tokens, float *probs, void *stream) {
    if (!f || (f->rows_each < 1)) return f ? CSD_EINVAL : CSD_ENULL;
    if (dtype != CSD_DTYPE_FP32 && dtype != CSD_DTYPE_BF16) return CSD_EINVAL;
    if (rows < 0 || V < 1 || stride < V) return CSD_EINVAL;
    // (the arrays end with the last whole set)
    if ((f->temperature || f->top_k || f->top_p || f->min_p) && rows % f->rows_each) return CSD_EINVAL;
    if (!f->temperature && !(f->temperature_all >= 0.f)) return CSD_EINVAL;
    if (!f->top_p && !(f->top_p_all >= 0.f)) return CSD_EINVAL;
    if (!f->min_p && !(f->min_p_all >= 0.f && f->min_p_all <= 1.f)) return CSD_EINVAL;
    if (V > (1 << 18) || rows > (1 << 21)) return CSD_ESHAPE;       // (work items of a launch are counted in 32 bits)
    if (rows == 0) return CSD_OK;
    if (!logits) return CSD_ENULL;
    const size_t size = dtype == CSD_DTYPE_FP32 ? 4 : 2;
    if ((uintptr_t)logits % size || ((uintptr_t)probs | (uintptr_t)u | (uintptr_t)tokens) % 4) return CSD_EINVAL;
    // rows are read again behind the first probabilities
    const char *from = (const char *)logits, *to = from + ((size_t)(rows - 1) * stride + V) * size;
    if (probs && (const char *)probs < to && from < (const char *)(probs + (size_t)rows * V)) return CSD_EINVAL;
    const SampleRows a{logits, (long long)stride, V, f->rows_each, u, tokens, probs, f->temperature, f->top_p, f->min_p, f->top_k,
                       f->temperature_all, f->top_p_all, f->min_p_all, f->top_k_all, (long long)rows * V * (long long)(size + 4) >= 144ll << 20};
    if (dtype == CSD_DTYPE_FP32) sample_launch<float>(a, rows, (hipStream_t)stream);
    else sample_launch<bf16_t>(a, rows, (hipStream_t)stream);
    CSD_LAUNCH_CHECK();
    return CSD_OK;
}

extern "C" int32_t csd_sample(const csd_filter *f, const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t V, const float *u,
                              int32_t *tokens, float *probs, void *stream) {
    if (rows > 0 && (!u || !tokens)) return CSD_ENULL;
    return sample_enqueue(f, logits, stride, dtype, rows, V, u, tokens, probs, stream);
}

extern "C" int32_t csd_filter_probs(const csd_filter *f, const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t V, float *probs,
                                    void *stream) {
    if (rows > 0 && !probs) return CSD_ENULL;
    return sample_enqueue(f, logits, stride, dtype, rows, V, nullptr, nullptr, probs, stream);
}
