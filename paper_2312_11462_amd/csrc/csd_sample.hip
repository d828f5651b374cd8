// Draws from logits by temperature, top-k, top-p and min-p, and the probabilities of such draws.
//
// With M the largest logit of a row and w_v = 2^((l_v - M) log2(e) / T), every weight is the whole number round(w_v 2^45): sums do not depend on their
// order, so neither do the sets that they bound nor the tokens (2^18 of them fit 63 bits; what a weight of 64 bits would add to the sums decides
// for uniform numbers within 2^-38 or so of a border).  Tokens are ranked by (logit, lowest token first), which is the order of one 64-bit number, key << 32 | ~token.
// Each parameter keeps a start of the ranking, so together they keep the tokens from a least such number on:
//   top-k   the first k
//   top-p   of those the shortest start with at least p of their weight
//   min-p   of those the ones with w >= p
// The least number is found by a histogram of counts and weights over 2048 steps of the logit (46 octaves of weight below M; lower ones have weight 0), and in
// the step that holds the border by ranking its tokens against one another.  Steps with too many for that are divided again by their keys, until
// few are left or all are equal.  The draw descends the row: sixteen ranges, the one that holds the border, sixteen ranges of that.
//
// A workgroup per row, which goes over it four to six times.
#include "csd_internal.h"

static constexpr int kBins = 2048, kList = 256;              // steps of the histogram; tokens that are ranked against one another at most

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
};

typedef unsigned long long u64;

// ---------------------------------------------------------------------------------------- numbers

// NaN counts as -inf, -0 as 0
__device__ __forceinline__ float plain_logit(float v) { return fmaxf(v, -INFINITY) + 0.f; }
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ u64 rank_of(uint32_t key, int v) { return (u64)key << 32 | (uint32_t)~v; }

// 2^x for x in [-46, 0] to 2^-47 of itself: the powers of ln 2 over the factorials, for the part of x within half of a whole number
__device__ __forceinline__ double exp2_of(double x) {
    const double n = rint(x), f = x - n;
    double p = 4.4455382718708116e-10;
    p = fma(p, f, 7.054911620801123e-09);
    p = fma(p, f, 1.01780860092397e-07);
    p = fma(p, f, 1.321548679014431e-06);
    p = fma(p, f, 1.5252733804059841e-05);
    p = fma(p, f, 0.0001540353039338161);
    p = fma(p, f, 0.0013333558146428443);
    p = fma(p, f, 0.009618129107628477);
    p = fma(p, f, 0.05550410866482158);
    p = fma(p, f, 0.2402265069591007);
    p = fma(p, f, 0.6931471805599453);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}

// Weights of a row.
struct Weights {
    float top;                    // M
    double c;                     // log2(e) / T
    __device__ __forceinline__ double real(float v) const {
        const double x = v == top ? 0.0 : ((double)v - (double)top) * c;
        return x >= -46.0 ? exp2_of(x) : 0.0;                // (also for NaN: 0 times -inf)
    }
    // times 2^45, to the nearest whole number: 128 + w has steps of 2^-45
    static __device__ __forceinline__ u64 whole(double w) { return (u64)__double_as_longlong(w + 128.0) & ((1ull << 52) - 1); }
    __device__ __forceinline__ u64 operator()(float v) const { return whole(real(v)); }
};

// floor(a z) and ceil(a z) for a in [0, 1)
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

// ---------------------------------------------------------------------------------------- a row, by N threads

template <typename T, int N>
struct Row {
    static constexpr int VE = 16 / sizeof(T), W = N / 64, TILE = 64 * VE, AHEAD = 4;
    const T *x;
    int V;

    // rows start at any element
    struct __attribute__((packed, aligned(sizeof(T)))) Raw {
        u32x4 v;
    };
    __device__ __forceinline__ u32x4 load(int at) const {
        if (at + VE <= V) return reinterpret_cast<const Raw *>(x + at)->v;
        u32x4 r;
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
    static __device__ __forceinline__ float get(const u32x4 &r, int e) {
        if constexpr (sizeof(T) == 4) return plain_logit(__uint_as_float(r[e]));
        else return plain_logit(__uint_as_float(e & 1 ? r[e / 2] & 0xFFFF0000u : r[e / 2] << 16));
    }
    // f(first token, piece) for the pieces of VE tokens of [lo, hi) that are this lane's; lo and hi are the wave's
    template <typename F>
    __device__ __forceinline__ void pieces(int lo, int hi, F f) const {
        const int lane = threadIdx.x & 63;
        for (int base = lo; base < hi; base += AHEAD * TILE) {
            u32x4 r[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; j++) {
                const int at = base + j * TILE + lane * VE;
                if (at < hi) r[j] = load(at);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; j++) {
                const int at = base + j * TILE + lane * VE;
                if (at < hi) f(at, r[j]);
            }
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
    // the ranges of the waves
    static __device__ __forceinline__ int range(int n) { return (n + W * TILE - 1) / (W * TILE) * TILE; }
    template <typename F>
    __device__ __forceinline__ void all(F f) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = range(V);
        tokens(min(wave * c, V), min(wave * c + c, V), f);
    }
};

struct SampleShared {
    uint32_t count[kBins];
    u64 mass[kBins];
    u64 list_rank[kList], list_mass[kList];
    u64 part[32];
    uint32_t part32[32];
    float top[16];
    uint32_t bin, base_count, n_list, key_lo, key_hi;
    u64 base_mass, least, sum;
    int token;
};

__device__ __forceinline__ u64 wave_sum64(u64 v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ u64 wave_scan64(u64 v) {      // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const u64 x = __shfl_up(v, o, 64);
        if (lane >= o) v += x;
    }
    return v;
}
// sum over the workgroup, in every thread
template <int N>
__device__ __forceinline__ u64 group_sum64(SampleShared &S, u64 v) {
    v = wave_sum64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) S.part[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 t = 0;
#pragma unroll
    for (int i = 0; i < N / 64; i++) t += S.part[i];
    return t;
}

// What the threads know of the histogram: thread t has kBins / N neighbouring steps, what they hold and what lies before them.
template <int N>
struct Steps {
    static constexpr int B = kBins / N;
    uint32_t count[B], before;
    u64 mass[B], mass_before;

    __device__ __forceinline__ void read(SampleShared &S) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        uint32_t n = 0;
        u64 m = 0;
#pragma unroll
        for (int i = 0; i < B; i++) {
            count[i] = S.count[tid * B + i];
            mass[i] = S.mass[tid * B + i];
            n += count[i];
            m += mass[i];
        }
        const u64 ni = wave_scan64(n), mi = wave_scan64(m);
        __syncthreads();
        if (lane == 63) {
            S.part32[wave] = (uint32_t)ni;
            S.part[wave] = mi;
        }
        __syncthreads();
        before = (uint32_t)ni - n;
        mass_before = mi - m;
        for (int i = 0; i < wave; i++) {
            before += S.part32[i];
            mass_before += S.part[i];
        }
    }
    // The first step at which k tokens, or m of weight, are reached, into S (all threads; S.bin is kBins where there is none).
    __device__ __forceinline__ void find(SampleShared &S, uint32_t k, u64 m) const {
        __syncthreads();
        if (threadIdx.x == 0) S.bin = kBins;
        __syncthreads();
        uint32_t n = before;
        u64 w = mass_before;
#pragma unroll
        for (int i = 0; i < B; i++) {
            if (n < k && w < m && (n + count[i] >= k || w + mass[i] >= m)) {
                S.bin = threadIdx.x * B + i;
                S.base_count = n;
                S.base_mass = w;
                S.n_list = count[i];
            }
            n += count[i];
            w += mass[i];
        }
        __syncthreads();
    }
};

// The lowest token of [0, V) at which the running sum of value(token, logit) passes `target`; the sum over the row is more than that.
template <typename T, int N, typename F>
__device__ __forceinline__ int descend(const Row<T, N> &row, SampleShared &S, u64 target, F value) {
    using R = Row<T, N>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int lo = 0, hi = row.V;
    while (hi - lo > R::TILE) {
        const int c = R::range(hi - lo), a = min(lo + wave * c, hi), b = min(a + c, hi);
        u64 sum = 0;
        row.tokens(a, b, [&](int v, float l) { sum += value(v, l); });
        sum = wave_sum64(sum);
        __syncthreads();
        if (lane == 0) S.part[wave] = sum;
        __syncthreads();
        int w = 0;
        for (; w < N / 64 - 1 && S.part[w] <= target; w++) target -= S.part[w];
        lo = min(lo + w * c, hi - 1);
        hi = min(lo + c, hi);
    }
    __syncthreads();
    if (wave == 0) {
        u64 mine[R::VE], sum = 0;
#pragma unroll
        for (int e = 0; e < R::VE; e++) mine[e] = 0;
        row.pieces(lo, hi, [&](int at, const u32x4 &r) {
#pragma unroll
            for (int e = 0; e < R::VE; e++) {
                mine[e] = at + e < hi ? value(at + e, R::get(r, e)) : 0;
                sum += mine[e];
            }
        });
        const u64 incl = wave_scan64(sum), past = __ballot(incl > target);
        if (past && lane == __ffsll((long long)past) - 1) {
            u64 run = incl - sum;
            int e = 0;
#pragma unroll
            for (int i = 0; i < R::VE - 1; i++) {
                run += mine[i];
                e += run <= target ? 1 : 0;
            }
            S.token = lo + lane * R::VE + e;
        }
    }
    __syncthreads();
    return S.token;
}

// The step of `steps` that holds the border of the first k tokens, or of m of weight, has been found (S): the rank of the last token inside, and the weight inside.
// in_step(v, l): whether a token is in the step.
template <typename T, int N, typename F>
__device__ __forceinline__ void border(const Row<T, N> &row, SampleShared &S, const Weights &weight, uint32_t k, u64 m, F in_step, u64 &least, u64 &inside) {
    const int tid = threadIdx.x;
    uint32_t base = S.base_count, n = S.n_list;
    u64 base_mass = S.base_mass;
    uint32_t key_lo = 0, key_hi = 0xFFFFFFFFu;
    auto in = [&](int v, float l) {
        const uint32_t key = key_of(l);
        return v < row.V && key >= key_lo && key <= key_hi && in_step(l);
    };
    while (n > (uint32_t)kList) {
        __syncthreads();
        if (tid == 0) {
            S.key_lo = 0xFFFFFFFFu;
            S.key_hi = 0;
        }
        __syncthreads();
        uint32_t lo = 0xFFFFFFFFu, hi = 0;
        row.all([&](int v, float l) {
            if (in(v, l)) {
                lo = min(lo, key_of(l));
                hi = max(hi, key_of(l));
            }
        });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            lo = min(lo, (uint32_t)__shfl_xor(lo, o, 64));
            hi = max(hi, (uint32_t)__shfl_xor(hi, o, 64));
        }
        if ((tid & 63) == 0) {
            atomicMin(&S.key_lo, lo);
            atomicMax(&S.key_hi, hi);
        }
        for (int i = tid; i < kBins; i += N) {
            S.count[i] = 0;
            S.mass[i] = 0;
        }
        __syncthreads();
        key_lo = S.key_lo;
        key_hi = S.key_hi;
        if (key_lo >= key_hi) break;
        const int shift = max(0, 32 - __clz(key_hi - key_lo) - 11);      // 2^11 steps of keys
        row.all([&](int v, float l) {
            if (in(v, l)) {
                const uint32_t i = (key_hi - key_of(l)) >> shift;
                atomicAdd(&S.count[i], 1u);
                atomicAdd(&S.mass[i], weight(l));
            }
        });
        __syncthreads();
        Steps<N> steps;
        steps.read(S);
        steps.find(S, k - base, m - base_mass);
        base += S.base_count;
        base_mass += S.base_mass;
        n = S.n_list;
        const uint32_t top = key_hi - (S.bin << shift);
        key_lo = max(key_lo, top - min(top, (1u << shift) - 1));
        key_hi = top;
    }
    __syncthreads();
    if (tid == 0) {
        S.n_list = 0;
        S.least = ~0ull;
        S.sum = 0;
    }
    __syncthreads();
    if (n > (uint32_t)kList) {
        // all equal: the first of them by token
        const uint32_t key = key_lo;
        u64 w = 0;
        if (tid == 0) {
            const float l = __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
            S.sum = weight(l);
        }
        __syncthreads();
        w = S.sum;
        u64 keep = k - base;
        if (w) keep = min(keep, (m - base_mass - 1) / w + 1);      // (m is more than base_mass)
        keep = min(max(keep, (u64)1), (u64)n);
        const int last = descend(row, S, keep - 1, [&](int v, float l) { return (u64)(v < row.V && key_of(l) == key ? 1 : 0); });
        least = rank_of(key, last);
        inside = base_mass + keep * w;
        return;
    }
    row.all([&](int v, float l) {
        if (in(v, l)) {
            const uint32_t i = atomicAdd(&S.n_list, 1u);
            if (i < (uint32_t)kList) {
                S.list_rank[i] = rank_of(key_of(l), v);
                S.list_mass[i] = weight(l);
            }
        }
    });
    __syncthreads();
    n = min(S.n_list, (uint32_t)kList);
    if (tid < (int)n) {
        const u64 mine = S.list_rank[tid];
        uint32_t ahead = base;
        u64 run = base_mass;
        for (uint32_t i = 0; i < n; i++)
            if (S.list_rank[i] > mine) {
                ahead++;
                run += S.list_mass[i];
            }
        if (ahead < k && run < m) {
            atomicMin(&S.least, mine);
            atomicAdd(&S.sum, S.list_mass[tid]);
        }
    }
    __syncthreads();
    least = S.least;
    inside = base_mass + S.sum;
}

template <typename T, int N>
__global__ __launch_bounds__(N) void k_sample(SampleRows a) {
    __shared__ SampleShared S;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, set = r / a.each;
    const Row<T, N> row{reinterpret_cast<const T *>(a.logits) + (size_t)r * a.stride, a.V};
    const float temperature = a.temperature ? a.temperature[set] : a.temperature_all, p = a.top_p ? a.top_p[set] : a.top_p_all,
                p_min = a.min_p ? a.min_p[set] : a.min_p_all;
    const bool greedy = !(temperature > 0.f);
    int k = greedy ? 1 : a.top_k ? a.top_k[set] : a.top_k_all;
    if (k <= 0 || k > a.V) k = a.V;

    float top = -INFINITY;
    row.all([&](int, float l) { top = fmaxf(top, l); });
    top = wave_max(top);
    if (lane == 0) S.top[wave] = top;
    for (int i = tid; i < kBins; i += N) {
        S.count[i] = 0;
        S.mass[i] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N / 64; i++) top = fmaxf(top, S.top[i]);
    float *out = a.probs ? a.probs + (size_t)r * a.V : nullptr;
    if (top == -INFINITY) {                                  // nothing to draw from
        if (out)
            for (int i = tid; i < a.V; i += N) out[i] = 0.f;
        if (a.tokens && tid == 0) a.tokens[r] = -1;
        return;
    }
    const double c = 1.4426950408889634 / (greedy ? 1.0 : (double)temperature);
    const Weights weight{top, c};
    const bool by_mass = p < 1.f && k > 1;
    u64 least = 0;
    if (k < a.V || by_mass) {
        const float per = (float)((double)(kBins / 46.0) * c);
        auto step_of = [&](float l) {
            const float t = l == top ? 0.f : (top - l) * per;
            return t < (float)kBins ? (int)t : kBins;        // (kBins: no weight; also for NaN)
        };
        row.all([&](int v, float l) {
            const int i = v < a.V ? step_of(l) : kBins;
            if (i < kBins) {
                atomicAdd(&S.count[i], 1u);
                if (by_mass) atomicAdd(&S.mass[i], weight(l));
            }
        });
        __syncthreads();
        Steps<N> steps;
        steps.read(S);
        u64 all = steps.mass_before;
#pragma unroll
        for (int i = 0; i < Steps<N>::B; i++) all += steps.mass[i];
        __syncthreads();
        if (tid == N - 1) S.sum = all;
        __syncthreads();
        all = S.sum;
        if (k < a.V) {
            steps.find(S, k, ~0ull);
            const int at = S.bin;
            if (at < kBins) border(row, S, weight, k, ~0ull, [&](float l) { return step_of(l) == at; }, least, all);
        }
        if (by_mass) {
            const u64 m = max(share_of(p, all, true), (u64)1);
            steps.find(S, ~0u, m);
            const int at = S.bin;
            if (at < kBins) border(row, S, weight, ~0u, m, [&](float l) { return step_of(l) == at; }, least, all);
        }
    }
    const u64 w_min = p_min > 0.f ? max((u64)ceil((double)fminf(p_min, 1.f) * (double)(1ull << 45)), (u64)1) : 1;
    auto value = [&](int v, float l) -> u64 {
        if (v >= a.V || rank_of(key_of(l), v) < least) return 0;
        const u64 w = weight(l);
        return w >= w_min ? w : 0;
    };
    u64 sum = 0;
    row.all([&](int v, float l) { sum += value(v, l); });
    sum = group_sum64<N>(S, sum);
    if (out) {
        const double inv = 1.0 / ((double)sum * 0x1p-45);
        row.all([&](int v, float l) {
            if (v < a.V) out[v] = value(v, l) ? (float)(weight.real(l) * inv) : 0.f;
        });
    }
    if (a.tokens) {
        const u64 target = min(share_of(fminf(a.u[r], 0.99999994f), sum, false), sum - 1);
        const int token = descend(row, S, target, value);
        if (tid == 0) a.tokens[r] = token;
    }
}

// ---------------------------------------------------------------------------------------- entry points

static int32_t sample_enqueue(const csd_filter *f, const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t V, const float *u,
                              int32_t *tokens, float *probs, void *stream) {
    if (!f || (f->rows_each < 1)) return f ? CSD_EINVAL : CSD_ENULL;
    if (dtype != CSD_DTYPE_FP32 && dtype != CSD_DTYPE_BF16) return CSD_EINVAL;
    if (rows < 0 || V < 1 || stride < V) return CSD_EINVAL;
    if (!f->temperature && !(f->temperature_all >= 0.f)) return CSD_EINVAL;
    if (!f->top_p && !(f->top_p_all >= 0.f)) return CSD_EINVAL;
    if (!f->min_p && !(f->min_p_all >= 0.f && f->min_p_all <= 1.f)) return CSD_EINVAL;
    if (V > (1 << 18) || rows > (1 << 22)) return CSD_ESHAPE;
    if (rows == 0) return CSD_OK;
    if (!logits) return CSD_ENULL;
    if ((uintptr_t)logits % (dtype == CSD_DTYPE_FP32 ? 4 : 2) || (uintptr_t)probs % 4) return CSD_EINVAL;
    const SampleRows a{logits, (long long)stride, V, f->rows_each, u, tokens, probs, f->temperature, f->top_p, f->min_p, f->top_k,
                       f->temperature_all, f->top_p_all, f->min_p_all, f->top_k_all};
    if (dtype == CSD_DTYPE_FP32) hipLaunchKernelGGL((k_sample<float, 1024>), dim3(rows), dim3(1024), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((k_sample<bf16_t, 1024>), dim3(rows), dim3(1024), 0, (hipStream_t)stream, a);
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
