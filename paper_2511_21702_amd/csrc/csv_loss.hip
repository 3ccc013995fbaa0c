// Log-probabilities of given tokens from rows of logits, their gradient, and the clipped policy loss with its gradient.
//
//   row_kernel     one block per row: the largest logit m and s = sum exp(c (x - m)), the log-probability of the row's token, and for the
//                  policy loss the row's term and its gradient row, from a second read while the row is still in a cache
//   part_kernel    m and s of a part of a row, for few rows; then
//   join_kernel    the log-probabilities from the parts, or
//   policy_kernel  the policy loss from the parts: every block joins its row's parts and writes its part of the gradient, the block that
//                  finishes last adds the loss up
//   grad_kernel    gradient rows from given m, s and coefficients
//   sum_kernel     the loss: the rows' terms in float64, in one order
//
// A row starts wherever its stride puts it: it is read as up to E - 1 single elements, 16-byte pieces of E elements, and up to
// E - 1 single elements (E = 4 or 8); the single ones go to the first threads, one each.
//
// Exponentials.  exp(c (x - m)) = 2^(d c2) with d = x - m and c2 = c log2(e).  c2 as one float32 is off by up to 2^-25 of itself, and with it every
// log-probability of every row, the same way, by that part of c (m - E[x]).  It is kept as the sum of two floats: fma(d, hi, d lo) rounds once (mean error of
// 2048 rows of 64007 float32 logits, c = 1 / 0.7: -5.8e-8 / -9.5e-8 with one float, below 1e-8 with two; 64 rows of 128256, bound by instructions, 9.8 ->
// 11.5 us, many rows, bound by memory, within 1 percent).  The low part cannot be added to a rounded d hi, or to m c2 before it: most of it is
// lost in their last digit.  A thread adds up in float32; threads and parts are added in float64, because what those last sums lose is
// not averaged over anything.
//
// Times here and below: on the GPU, inputs changing from pass to pass where they fit, unless another measure is named.
#include "csv_common.h"

#include <math.h>

#define LOG2E 1.4426950408889634
#define LOWEST (-3.402823466e38f)
#define MAX_PARTS 64                // parts of a row: one per lane of the wave that joins them
#define PART_MIN 2048               // logits of a part, at least

struct RowArgs {
    const void* x;
    int64_t ld;
    int N, V, parts;
    const int32_t* tokens;
    double c;                // inverse temperature
    float2 c2;               // c log2(e), see split()
    const float* old_logp;   // policy loss
    const float* ref_logp;
    const float* adv;
    const float* weights;
    double clip_low, clip_high, beta;
    const float* stats_in;   // gradient alone
    const float* grad_logp;
    float* logp;
    float* stats;
    double* terms;           // scratch: [N]
    float2* part;            // [N * parts] (m, s) of a part of a row
    float* xt;               // [N] the logit of the row's token
    int* arrived;            // rows whose term is there
    void* grad;
    int64_t ld_grad;
};

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4;
    float v[4];
    __device__ __forceinline__ void widen(const v4u& u) {
        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(u[j]);
    }
    __device__ __forceinline__ void load(const float* p) { widen(*(const v4u*)p); }
    __device__ __forceinline__ void load_last(const float* p) { widen(__builtin_nontemporal_load((const v4u*)p)); }
    __device__ __forceinline__ void store(float* p) const {
        __builtin_nontemporal_store(v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, (v4u*)p);
    }
};
template <> struct Vec<uint16_t> {
    static constexpr int E = 8;
    float v[8];
    __device__ __forceinline__ void widen(const v4u& u) {
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo(u[j]);
            v[2 * j + 1] = bf16_hi(u[j]);
        }
    }
    __device__ __forceinline__ void load(const uint16_t* p) { widen(*(const v4u*)p); }
    __device__ __forceinline__ void load_last(const uint16_t* p) { widen(__builtin_nontemporal_load((const v4u*)p)); }
    __device__ __forceinline__ void store(uint16_t* p) const {
        v4u w;
        for (int j = 0; j < 4; ++j)
            w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j + 1]) << 16;
        __builtin_nontemporal_store(w, (v4u*)p);
    }
};
__device__ __forceinline__ float get(const float* p) { return *p; }
__device__ __forceinline__ float get(const uint16_t* p) { return bf16_lo(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

// How a row of V elements falls into single elements and 16-byte pieces.
template <typename T> struct Row {
    const T* p;
    int head, pieces, tail;
    __device__ __forceinline__ Row(const T* row, int V) : p(row) {
        constexpr int E = Vec<T>::E;
        head = min(V, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));
        pieces = (V - head) / E;
        tail = V - head - pieces * E;
    }
    // the single element of thread t, or -1
    __device__ __forceinline__ int single(int t) const {
        return t < head ? t : t < head + tail ? t + pieces * Vec<T>::E : -1;
    }
};

// A double as two floats, x below it and y > 0: minus infinity times either one is minus infinity, and so is their sum.
static float2 split(double c2) {
    float hi = (float)c2;
    if ((double)hi >= c2) hi = nextafterf(hi, 0.f);
    const float lo = (float)(c2 - (double)hi);
    return make_float2(hi, lo > 0.f ? lo : 1.4013e-45f);
}
// 2^((x - m) c2)
__device__ __forceinline__ float exp_of(float x, float m, float2 c2) {
    const float d = x - m;
    return __builtin_amdgcn_exp2f(fmaf(d, c2.x, d * c2.y));
}

struct Stat {
    float m;
    double s;
};

// Sums of doubles: a wave's by lane exchanges without LDS, the waves' in one order for all threads.
template <int CTRL, int ROW_MASK, bool ZERO>
__device__ __forceinline__ double dpp_add(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const int lo = (int)(unsigned)u, hi = (int)(unsigned)(u >> 32);
    const unsigned a = (unsigned)dpp_move<CTRL, ROW_MASK>(ZERO ? 0 : lo, lo), b = (unsigned)dpp_move<CTRL, ROW_MASK>(ZERO ? 0 : hi, hi);
    return v + __builtin_bit_cast(double, (unsigned long long)b << 32 | a);
}
__device__ __forceinline__ double wave_sum(double v) {
    v = dpp_add<0xB1, 0xf, false>(v);      // quad_perm [1,0,3,2]
    v = dpp_add<0x4E, 0xf, false>(v);      // quad_perm [2,3,0,1]
    v = dpp_add<0x141, 0xf, false>(v);     // row_half_mirror
    v = dpp_add<0x140, 0xf, false>(v);     // row_mirror
    v = dpp_add<0x142, 0xa, true>(v);      // row_bcast15 into rows 1 and 3
    v = dpp_add<0x143, 0xc, true>(v);      // row_bcast31 into rows 2 and 3
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, 63), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), 63);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* red) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < THREADS / 64; ++w) v += red[w];
    return v;
}

// m and s of the single elements and the pieces lo .. hi - 1 of a row, by the whole block.  A thread keeps its own maximum and its sum relative to it.
// The maximum starts at the lowest number, not at minus infinity, which less itself would be NaN: logits of minus infinity add 0 to any of them.
// red: >= 16 doubles of LDS
template <int THREADS, typename T>
__device__ __forceinline__ Stat fold(const Row<T>& row, int lo, int hi, bool singles, float2 c2, double* red) {
    constexpr int E = Vec<T>::E, U = 4;
    const int one = singles ? row.single(threadIdx.x) : -1;
    float m = LOWEST, s = 0.f;
    if (one >= 0) {
        const float x = get(row.p + one);
        m = fmaxf(m, x);
        s = exp_of(x, m, c2);
    }
    const T* base = row.p + row.head;
    auto take = [&](const auto& x, int n) {
        float top = m;
        for (int u = 0; u < n; ++u)
            for (int j = 0; j < E; ++j) top = fmaxf(top, x[u].v[j]);
        float add = 0.f;
        for (int u = 0; u < n; ++u) {
            float e[E];
            for (int j = 0; j < E; ++j) e[j] = exp_of(x[u].v[j], top, c2);
            for (int w = E / 2; w > 0; w >>= 1)         // pairs: a likely token's term is rounded as often as the tree is high, not E times
                for (int j = 0; j < w; ++j) e[j] += e[j + w];
            add += e[0];
        }
        s = fmaf(s, exp_of(m, top, c2), add);
        m = top;
    };
    int i = lo + threadIdx.x;
    for (; i + (U - 1) * THREADS < hi; i += U * THREADS) {
        Vec<T> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].load(base + (int64_t)(i + u * THREADS) * E);
        take(x, U);
    }
    for (; i < hi; i += THREADS) {
        Vec<T> x[1];
        x[0].load(base + (int64_t)i * E);
        take(x, 1);
    }
    Stat r;
    r.m = block_max(m, (float*)red);
    r.s = block_sum<THREADS>((double)(s * exp_of(m, r.m, c2)), red);
    if (r.s == 0.0) r.m = -INFINITY;       // the largest logit itself adds 1, unless it is minus infinity
    return r;
}

// c g ([j = t] - p_j) over the single elements and the pieces lo .. hi - 1 of a row; eg = c g
template <int THREADS, typename T>
__device__ __forceinline__ void write_grad(const Row<T>& row, T* out, int lo, int hi, bool singles, int token, float m, double s, float2 c2, float eg) {
    constexpr int E = Vec<T>::E, U = 4;
    const float f = (float)((double)eg / s);
    // where the result is rounded to bfloat16, 2^-9 of it, what one float32 of c2 loses (2^-23 of the exponent) is not seen
    auto value = [&](float x) { return -f * (sizeof(T) == 4 ? exp_of(x, m, c2) : __builtin_amdgcn_exp2f((x - m) * c2.x)); };
    const int one = singles ? row.single(threadIdx.x) : -1;
    if (one >= 0) put(out + one, (one == token ? eg : 0.f) + value(get(row.p + one)));
    const T* from = row.p + row.head;
    T* to = out + row.head;
    const bool aligned = ((uintptr_t)to & 15) == 0;
    const int special = token >= row.head ? (token - row.head) / E : -1;      // the piece with the token
    auto give = [&](Vec<T>& x, int i) {
        for (int j = 0; j < E; ++j) x.v[j] = value(x.v[j]);
        if (i == special)
            for (int j = 0; j < E; ++j) x.v[j] += row.head + i * E + j == token ? eg : 0.f;
        if (aligned) x.store(to + (int64_t)i * E);
        else
            for (int j = 0; j < E; ++j) put(to + (int64_t)i * E + j, x.v[j]);
    };
    int i = lo + threadIdx.x;
    for (; i + (U - 1) * THREADS < hi; i += U * THREADS) {
        Vec<T> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].load_last(from + (int64_t)(i + u * THREADS) * E);
#pragma unroll
        for (int u = 0; u < U; ++u) give(x[u], i + u * THREADS);
    }
    for (; i < hi; i += THREADS) {
        Vec<T> x;
        x.load_last(from + (int64_t)i * E);
        give(x, i);
    }
}
template <int THREADS, typename T>
__device__ __forceinline__ void write_zeros(T* out, int V, int part, int parts) {
    const Row<T> row(out, V);
    const int one = part == 0 ? row.single(threadIdx.x) : -1;
    if (one >= 0) put(out + one, 0.f);
    const int hi = (int)((int64_t)row.pieces * (part + 1) / parts);
    for (int i = (int)((int64_t)row.pieces * part / parts) + threadIdx.x; i < hi; i += THREADS) __builtin_nontemporal_store(v4u{0, 0, 0, 0}, (v4u*)(out + row.head + (int64_t)i * Vec<T>::E));
}

__device__ __forceinline__ double log_prob(Stat r, float xt, double c) {
    return r.s == 0.0 ? -INFINITY : c * ((double)xt - (double)r.m) - log(r.s);
}

// The loss term of a row and its derivative by the log-probability, in float64: one thread per row does this, and close to a clip border
// the digits decide which branch holds.  A log-probability of minus infinity is that of a masked token, which no other logit changes: ratio 0, no
// derivative.  What would be a difference of equal infinities or 0 times a ratio beyond the largest number is taken for 0.
__device__ __forceinline__ double policy_term(const RowArgs& a, int i, double logp, double& g) {
    const bool masked = isinf(logp);
    const double A = a.adv[i], w = a.weights[i], old = a.old_logp[i], r = masked && isinf(old) ? 0.0 : exp(logp - old);
    const double lo = 1.0 - a.clip_low, hi = 1.0 + a.clip_high, whole = A == 0.0 && isinf(r) ? 0.0 : r * A, cut = fmin(fmax(r, lo), hi) * A;
    double term = cut < whole ? -cut : -whole;
    double d = (A >= 0.0 ? r > hi : r < lo) ? 0.0 * A : -whole;      // a NaN of the inputs is one of the gradient too
    if (a.beta > 0.0) {
        const double ref = a.ref_logp[i], k = ref == logp ? 0.0 : ref - logp, em = expm1(k);
        term += a.beta * (isinf(em) ? em : em - k);
        d -= a.beta * em;
    }
    g = masked ? 0.0 : w * d;
    return w * term;
}

__device__ __forceinline__ bool left_out(const RowArgs& a, int i, int token, bool policy) {
    return token < 0 || token >= a.V || (policy && a.weights[i] == 0.f);
}

// Bound by memory, two blocks per compute unit: one reads while the other reduces or writes.  The second read finds the row in a cache, so the gradient
// costs a read and a write: 4096 x 128256 bf16, a fifth of the rows left out, 402 us (4.7 TB/s, the rate of a copy); the log-probabilities alone,
// 2048 x 128256: 171 us in float32 (6.1 TB/s), 88 us in bf16 (6.0 TB/s).
template <typename T, bool POLICY>
__global__ __launch_bounds__(1024, 8) void row_kernel(RowArgs a) {
    __shared__ double red[16];
    __shared__ float coef;
    const int i = blockIdx.x, tid = threadIdx.x, token = a.tokens[i];
    T* grad = POLICY && a.grad ? (T*)a.grad + (int64_t)i * a.ld_grad : nullptr;
    if (left_out(a, i, token, POLICY)) {
        if (tid == 0) {
            if (a.logp) a.logp[i] = 0.f;
            if (POLICY) a.terms[i] = 0.0;
            else a.stats[2 * i] = a.stats[2 * i + 1] = 0.f;
        }
        if (grad) write_zeros<1024>(grad, a.V, 0, 1);
        return;
    }
    const Row<T> row((const T*)a.x + (int64_t)i * a.ld, a.V);
    const float xt = get(row.p + token);
    const Stat r = fold<1024>(row, 0, row.pieces, true, a.c2, red);
    if (tid == 0) {
        const double logp = log_prob(r, xt, a.c);
        if (a.logp) a.logp[i] = (float)logp;
        if (POLICY) {
            double g = 0.0;
            a.terms[i] = r.s == 0.0 ? 0.0 : policy_term(a, i, logp, g);
            coef = (float)(g * a.c);
        } else {
            a.stats[2 * i] = r.m;
            a.stats[2 * i + 1] = (float)r.s;
        }
    }
    if (!POLICY || !grad) return;
    __syncthreads();                            // the row's token has been read by now: the gradient may replace the logits
    if (r.s == 0.0) write_zeros<1024>(grad, a.V, 0, 1);
    else write_grad<1024>(row, grad, 0, row.pieces, true, token, r.m, r.s, a.c2, coef);
}

// A part's m and s in 8 bytes.  s is 0 (m minus infinity then), not a number (m neither then), or 1 and more, the largest logit's term: 5 bits of
// exponent and 27 below the leading one, because 24 of a float32 would be the largest error of a row that is cut.
__device__ __forceinline__ float2 pack(Stat r) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, r.s) - (1023ull << 52) + (1ull << 24);
    return make_float2(isnan(r.s) ? NAN : r.m, __uint_as_float((uint32_t)(u >> 25)));
}
__device__ __forceinline__ double unpack(float2 v) {
    const double s = __builtin_bit_cast(double, ((unsigned long long)__float_as_uint(v.y) << 25) + (1023ull << 52));
    return isnan(v.x) ? NAN : v.x == -INFINITY ? 0.0 : s;
}

// Short blocks, bound by the latency of a chain of loads and a reduction: 7 x 32003 float32 3.8 us, 64 x 128256 bf16 6.9 us.
template <typename T, bool POLICY>
__global__ __launch_bounds__(256, 8) void part_kernel(RowArgs a) {
    __shared__ double red[16];
    const int i = blockIdx.x / a.parts, p = blockIdx.x % a.parts, token = a.tokens[i];
    if (POLICY && blockIdx.x == 0 && threadIdx.x == 0) *a.arrived = 0;
    if (left_out(a, i, token, POLICY)) return;
    const Row<T> row((const T*)a.x + (int64_t)i * a.ld, a.V);
    const Stat r = fold<256>(row, (int)((int64_t)row.pieces * p / a.parts), (int)((int64_t)row.pieces * (p + 1) / a.parts), p == 0, a.c2, red);
    if (threadIdx.x == 0) {
        a.part[(int64_t)i * a.parts + p] = pack(r);
        if (p == 0) a.xt[i] = get(row.p + token);
    }
}

// m and s of row i from its parts, by a whole wave
__device__ __forceinline__ Stat join(const RowArgs& a, int i) {
    const int lane = threadIdx.x & 63;
    float2 v = make_float2(-INFINITY, 0.f);
    if (lane < a.parts) v = a.part[(int64_t)i * a.parts + lane];
    Stat r;
    r.m = wave_max(v.x);
    const double s = unpack(v);
    r.s = wave_sum(s == 0.0 ? 0.0 : s * (double)exp_of(v.x, r.m, a.c2));
    return r;
}

__global__ __launch_bounds__(256) void join_kernel(RowArgs a) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= a.N) return;
    Stat r = {0.f, 0.0};
    float logp = 0.f;
    if (!left_out(a, i, a.tokens[i], false)) {
        r = join(a, i);
        logp = (float)log_prob(r, a.xt[i], a.c);
    }
    if ((threadIdx.x & 63) == 0) {
        a.logp[i] = logp;
        a.stats[2 * i] = r.m;
        a.stats[2 * i + 1] = (float)r.s;
    }
}

// The sum of the rows' terms, every thread in steps of the block, then a tree: one order for a given N.
template <int THREADS>
__device__ __forceinline__ double sum_terms(const double* terms, int N, double* part) {
    double s = 0.0;
    for (int i = threadIdx.x; i < N; i += THREADS)
        s += __builtin_bit_cast(double, __hip_atomic_load((const unsigned long long*)terms + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < THREADS / 64; ++w) s += part[w];
    return s;
}

// Every block of a row takes the same scalars from the same parts; only the first one writes them.  7 x 32003 float32 5.7 us, 64 x 128256 bf16 8.8 us.
template <typename T>
__global__ __launch_bounds__(256) void policy_kernel(RowArgs a, int parts, float* loss) {
    __shared__ float coef;
    __shared__ int last;
    __shared__ double sums[4];
    const int i = blockIdx.x / parts, p = blockIdx.x % parts, token = a.tokens[i];
    T* grad = a.grad ? (T*)a.grad + (int64_t)i * a.ld_grad : nullptr;
    const bool out = left_out(a, i, token, true);
    Stat r = {0.f, 0.0};
    if (!out) r = join(a, i);
    if (threadIdx.x == 0) {
        double logp = 0.0, g = 0.0, term = 0.0;
        if (!out) {
            logp = log_prob(r, a.xt[i], a.c);
            if (r.s != 0.0) term = policy_term(a, i, logp, g);
        }
        coef = (float)(g * a.c);
        last = 0;
        if (p == 0) {
            if (a.logp) a.logp[i] = (float)logp;
            // The term goes out as an atomic store, past this die's cache, and has arrived before it is counted; a fence would write all of the
            // cache's gradient rows back first (64 rows of 128256: 23 us against 10).
            __hip_atomic_store((unsigned long long*)a.terms + i, __builtin_bit_cast(unsigned long long, term), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            last = __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.N - 1;
        }
    }
    __syncthreads();
    if (grad) {
        const Row<T> row((const T*)a.x + (int64_t)i * a.ld, a.V);
        if (out || r.s == 0.0) write_zeros<256>(grad, a.V, p, parts);
        else write_grad<256>(row, grad, (int)((int64_t)row.pieces * p / parts), (int)((int64_t)row.pieces * (p + 1) / parts), p == 0, token, r.m, r.s, a.c2, coef);
    }
    if (last) {
        const double s = sum_terms<256>(a.terms, a.N, sums);
        if (threadIdx.x == 0) *loss = (float)s;
    }
}

// Bound by memory: 509 x 151669 bf16, rows at odd addresses, 48 us (6.4 TB/s read and written).
template <typename T>
__global__ __launch_bounds__(256) void grad_kernel(RowArgs a) {
    const int i = blockIdx.x / a.parts, p = blockIdx.x % a.parts, token = a.tokens[i];
    T* grad = (T*)a.grad + (int64_t)i * a.ld_grad;
    const float m = a.stats_in[2 * i], s = a.stats_in[2 * i + 1], g = (float)((double)a.grad_logp[i] * a.c);
    const Row<T> row((const T*)a.x + (int64_t)i * a.ld, a.V);
    if (left_out(a, i, token, false) || g == 0.f || s == 0.f) write_zeros<256>(grad, a.V, p, a.parts);
    else write_grad<256>(row, grad, (int)((int64_t)row.pieces * p / a.parts), (int)((int64_t)row.pieces * (p + 1) / a.parts), p == 0, token, m, s, a.c2, g);
}

__global__ __launch_bounds__(1024) void sum_kernel(const double* __restrict__ terms, int N, float* __restrict__ loss) {
    __shared__ double part[16];
    const double s = sum_terms<1024>(terms, N, part);
    if (threadIdx.x == 0) *loss = (float)s;
}

// ------------------------------------------------------------------------------------------------ entry points
static int check_logits(const void* x, int type, int64_t ld, int N, int V, const int32_t* tokens, double c) {
    if (N < 0 || V < 1) { csv_set_error("need N >= 0 and V >= 1 (N=%d, V=%d)", N, V); return CSV_ESHAPE; }
    if (N > CSV_LOSS_MAX_ROWS) { csv_set_error("N=%d is above %d rows", N, CSV_LOSS_MAX_ROWS); return CSV_ESHAPE; }
    if (type != CSV_F32 && type != CSV_BF16) { csv_set_error("bad element type %d", type); return CSV_EINVAL; }
    if (ld < V) { csv_set_error("row stride %lld is below V=%d", (long long)ld, V); return CSV_ESHAPE; }
    if (!(c > 0.0) || !isfinite((float)(c * LOG2E)) || !(split(c * LOG2E).x > 0.f)) { csv_set_error("inverse temperature %g is not positive and finite in float32", c); return CSV_EINVAL; }
    if (N > 0 && (!x || !tokens)) { csv_set_error("null logits or tokens"); return CSV_EINVAL; }
    if (N > 0 && ((uintptr_t)x & (type == CSV_F32 ? 3 : 1))) { csv_set_error("logits are not aligned to their type"); return CSV_EINVAL; }
    return CSV_OK;
}
static int check_grad(const void* x, int type, int64_t ld, int N, int V, const void* grad, int64_t ld_grad) {
    if (ld_grad < V) { csv_set_error("row stride %lld of the gradient is below V=%d", (long long)ld_grad, V); return CSV_ESHAPE; }
    if (N > 0 && ((uintptr_t)grad & (type == CSV_F32 ? 3 : 1))) { csv_set_error("the gradient is not aligned to its type"); return CSV_EINVAL; }
    if (N > 1 && grad == x && ld_grad != ld) { csv_set_error("a gradient in place of the logits needs their row stride"); return CSV_EINVAL; }
    return CSV_OK;
}

// Memory of a call: rows of `bytes`, `step` bytes apart.
struct Span {
    const char* name;
    uintptr_t at;
    int64_t rows, bytes, step;
    bool in_place;           // logits, and the gradient that may take their place
};
static Span vec(const char* name, const void* p, int64_t bytes) { return {name, (uintptr_t)p, bytes > 0, bytes, bytes, false}; }
static Span matrix(const char* name, const void* p, int type, int64_t ld, int N, int V) {
    const int64_t e = type == CSV_F32 ? 4 : 2;
    return {name, (uintptr_t)p, N, V * e, ld * e, true};
}
static bool row_meets(uintptr_t at, int64_t bytes, const Span& m) {
    if (at + bytes <= m.at || at >= m.at + (m.rows - 1) * m.step + m.bytes) return false;
    const int64_t r = at < m.at ? 0 : (int64_t)((at - m.at) % m.step);      // beyond a row's end there is another row
    return r < m.bytes || r + bytes > m.step;
}
static bool meet(const Span& a, const Span& b) {
    if (!a.at || !b.at || a.rows < 1 || b.rows < 1) return false;
    if (a.rows == 1) return row_meets(a.at, a.bytes, b);
    if (b.rows == 1) return row_meets(b.at, b.bytes, a);
    const uintptr_t a_end = a.at + (a.rows - 1) * a.step + a.bytes, b_end = b.at + (b.rows - 1) * b.step + b.bytes;
    if (a.at >= b_end || b.at >= a_end) return false;
    if (a.step == b.step) {               // row j of b begins r bytes behind the start of row j + q of a
        const int64_t o = (int64_t)(b.at - a.at), r = ((o % a.step) + a.step) % a.step, q = (o - r) / a.step;
        return (r < a.bytes && q > -b.rows && q < a.rows) || (r + b.bytes > a.step && q + 1 > -b.rows && q + 1 < a.rows);
    }
    for (int64_t j = 0; j < b.rows; ++j)
        if (row_meets(b.at + j * b.step, b.bytes, a)) return true;
    return false;
}
// What a call writes is apart from what it reads and from what else it writes: blocks read while others write.  A gradient in place of the logits
// is no such case: an element is read by the thread that writes it, and the row's token and statistics before that.
template <int W, int R>
static int check_apart(const Span (&writes)[W], const Span (&reads)[R]) {
    for (int i = 0; i < W; ++i) {
        for (int j = 0; j < R; ++j) {
            if (writes[i].in_place && reads[j].in_place && writes[i].at == reads[j].at) continue;      // with one stride: check_grad
            if (meet(writes[i], reads[j])) { csv_set_error("%s overlaps %s", writes[i].name, reads[j].name); return CSV_EINVAL; }
        }
        for (int j = i + 1; j < W; ++j)
            if (meet(writes[i], writes[j])) { csv_set_error("%s overlaps %s", writes[i].name, writes[j].name); return CSV_EINVAL; }
    }
    return CSV_OK;
}
static int check_scratch(size_t need, const void* p, size_t have) {
    if (need && (!p || have < need)) { csv_set_error("scratch of %zu bytes, %zu are needed", p ? have : (size_t)0, need); return CSV_ESHAPE; }
    if (need && ((uintptr_t)p & 15)) { csv_set_error("scratch has to be 16-byte aligned"); return CSV_EINVAL; }
    return CSV_OK;
}

// Where the rows alone leave compute units without work, or with too little of it to keep the memory busy, a row is cut into parts: two launches,
// and the logits are read twice.  A policy loss does so below few_rows (with gradient, us on the GPU, parts / row: bf16 rows of 128256, 64 of them
// 16.4 / 25.4, 112 22.6 / 26.0, 143 24.4 / 26.1, 190 32.1 / 28.6, of 80000 112 17.7 / 19.3, 143 19.6 / 19.5, 160 22.7 / 19.8, of 32000 112 13.5 / 13.9,
// 143 15.2 / 14.7;  float32 rows of 128256 64 23.7 / 28.7, 112 33.7 / 34.3, 128 41.3 / 35.7, of 80000 90 21.5 / 22.1, 112 23.5 / 22.5, of 32000 64
// 12.1 / 13.0, 112 15.0 / 14.6).  The loss alone follows, so that it keeps its bits (of 128256 bf16 64 13.0 / 15.9, 112 16.5 / 16.3, 143 17.0 / 16.2,
// float32 64 15.8 / 18.2, 112 19.8 / 19.6, of 32000 bf16 64 9.5 / 9.5, 112 11.4 / 10.4).  Log-probabilities in one block per row are one launch,
// 3.3 us less for a host that waits for each call, and stay ahead up to longer rows the more rows there are (float32, 1 row of 32000 4.9 / 5.4, of
// 80000 4.9 / 8.2, of 128256 4.9 / 10.7, 64 of 80000 10.4 / 11.4, of 128256 12.8 / 15.0, 90 of 128256 14.4 / 15.8, bf16, 64 of 80000 8.9 / 9.2; from
// the host, 1 row of 128256 10.1 / 9.8).
#define FEW_ROWS 112
#define FEW_ROWS_BF16 144           // the larger one, and what scratch is made for
static inline int few_rows(int type) { return type == CSV_BF16 ? FEW_ROWS_BF16 : FEW_ROWS; }
#define LONG_ROW(N) (65000 + 950 * (N))
#define PART_BLOCKS 2048            // blocks of 256 threads that are resident together
#define GRAD_BLOCKS 16384           // gradients from given statistics have nothing to join: short blocks (us for 509 x 151669 bf16, 2048 x
                                    // 128256 float32: 64, 412 with 4096 blocks, 54, 391 with 16384)
static inline int parts_of(int N, int V, int most) {
    const int by_rows = most / (N > 0 ? N : 1), by_length = (V - 1) / PART_MIN + 1;
    const int p = by_rows < by_length ? by_rows : by_length;
    return p < 1 ? 1 : p > MAX_PARTS ? MAX_PARTS : p;
}

static int scratch_bytes(int N, int V, bool parts, size_t* bytes) {
    if (N < 0 || V < 1) { csv_set_error("need N >= 0 and V >= 1 (N=%d, V=%d)", N, V); return CSV_ESHAPE; }
    if (!bytes) { csv_set_error("null bytes"); return CSV_EINVAL; }
    *bytes = (size_t)N * sizeof(double) + (parts && N > 0 ? (size_t)N * (sizeof(float2) * parts_of(N, V, PART_BLOCKS) + 8) + 8 : 0);
    return CSV_OK;
}
static inline bool logprobs_by_parts(int N, int V) { return N < FEW_ROWS && V > LONG_ROW(N); }

extern "C" int csv_policy_loss_scratch(int N, int V, size_t* bytes) { return scratch_bytes(N, V, N < FEW_ROWS_BF16, bytes); }

extern "C" int csv_token_logprobs_scratch(int N, int V, size_t* bytes) {
    const int rc = scratch_bytes(N, V, logprobs_by_parts(N, V), bytes);
    if (!rc && !logprobs_by_parts(N, V)) *bytes = 0;
    return rc;
}

static void place_scratch(RowArgs& a, void* p, bool parts) {
    a.terms = (double*)p;
    if (!parts) return;
    a.parts = parts_of(a.N, a.V, PART_BLOCKS);
    a.part = (float2*)(a.terms + a.N);
    a.xt = (float*)(a.part + (size_t)a.N * a.parts);
    a.arrived = (int*)(a.xt + 2 * (size_t)a.N);
}

extern "C" int csv_token_logprobs(const void* d_logits, int type, int64_t ld, int N, int V, const int32_t* d_tokens, double inv_temperature, float* d_logp,
                                  float* d_stats, void* d_scratch, size_t have, void* stream) {
    int rc = check_logits(d_logits, type, ld, N, V, d_tokens, inv_temperature);
    size_t need = 0;
    if (!rc) rc = csv_token_logprobs_scratch(N, V, &need);
    if (!rc) rc = check_scratch(need, d_scratch, have);
    if (rc || N == 0) return rc;
    if (!d_logp || !d_stats) { csv_set_error("null d_logp or d_stats"); return CSV_EINVAL; }
    const Span writes[] = {vec("d_logp", d_logp, 4ll * N), vec("d_stats", d_stats, 8ll * N), vec("d_scratch", need ? d_scratch : nullptr, (int64_t)need)};
    const Span reads[] = {matrix("d_logits", d_logits, type, ld, N, V), vec("d_tokens", d_tokens, 4ll * N)};
    if ((rc = check_apart(writes, reads))) return rc;
    RowArgs a = {};
    a.x = d_logits; a.ld = ld; a.N = N; a.V = V; a.tokens = d_tokens; a.c = inv_temperature; a.c2 = split(a.c * LOG2E); a.logp = d_logp; a.stats = d_stats;
    const hipStream_t st = (hipStream_t)stream;
    if (logprobs_by_parts(N, V)) {
        place_scratch(a, d_scratch, true);
        if (type == CSV_F32) part_kernel<float, false><<<N * a.parts, 256, 0, st>>>(a);
        else part_kernel<uint16_t, false><<<N * a.parts, 256, 0, st>>>(a);
        CSV_LAUNCH_CHECK("part_kernel");
        join_kernel<<<(N + 3) / 4, 256, 0, st>>>(a);
        CSV_LAUNCH_CHECK("join_kernel");
        return CSV_OK;
    }
    if (type == CSV_F32) row_kernel<float, false><<<N, 1024, 0, st>>>(a);
    else row_kernel<uint16_t, false><<<N, 1024, 0, st>>>(a);
    CSV_LAUNCH_CHECK("row_kernel");
    return CSV_OK;
}

extern "C" int csv_token_logprobs_backward(const void* d_logits, int type, int64_t ld, int N, int V, const int32_t* d_tokens, const float* d_stats,
                                           const float* d_grad_logp, double inv_temperature, void* d_grad, int64_t ld_grad, void* stream) {
    int rc = check_logits(d_logits, type, ld, N, V, d_tokens, inv_temperature);
    if (!rc) rc = check_grad(d_logits, type, ld, N, V, d_grad, ld_grad);
    if (rc || N == 0) return rc;
    if (!d_stats || !d_grad_logp || !d_grad) { csv_set_error("null d_stats, d_grad_logp or d_grad"); return CSV_EINVAL; }
    const Span writes[] = {matrix("d_grad", d_grad, type, ld_grad, N, V)};
    const Span reads[] = {matrix("d_logits", d_logits, type, ld, N, V), vec("d_tokens", d_tokens, 4ll * N), vec("d_stats", d_stats, 8ll * N),
                          vec("d_grad_logp", d_grad_logp, 4ll * N)};
    if ((rc = check_apart(writes, reads))) return rc;
    RowArgs a = {};
    a.x = d_logits; a.ld = ld; a.N = N; a.V = V; a.tokens = d_tokens; a.c = inv_temperature; a.c2 = split(a.c * LOG2E); a.stats_in = d_stats; a.grad_logp = d_grad_logp;
    a.grad = d_grad; a.ld_grad = ld_grad;
    a.parts = parts_of(N, V, GRAD_BLOCKS);
    if (type == CSV_F32) grad_kernel<float><<<N * a.parts, 256, 0, (hipStream_t)stream>>>(a);
    else grad_kernel<uint16_t><<<N * a.parts, 256, 0, (hipStream_t)stream>>>(a);
    CSV_LAUNCH_CHECK("grad_kernel");
    return CSV_OK;
}

extern "C" int csv_policy_loss(const void* d_logits, int type, int64_t ld, int N, int V, const int32_t* d_tokens, const float* d_old_logp,
                               const float* d_ref_logp, const float* d_advantages, const float* d_weights, const csv_policy_params* p, float* d_loss,
                               float* d_logp, void* d_grad, int64_t ld_grad, void* d_scratch, size_t have, void* stream) {
    if (!p || !d_loss) { csv_set_error("null params or d_loss"); return CSV_EINVAL; }
    int rc = check_logits(d_logits, type, ld, N, V, d_tokens, p->inv_temperature);
    if (!rc && d_grad) rc = check_grad(d_logits, type, ld, N, V, d_grad, ld_grad);
    size_t need = 0;
    if (!rc) rc = csv_policy_loss_scratch(N, V, &need);
    if (!rc) rc = check_scratch(need, d_scratch, have);
    if (rc) return rc;
    if (!(p->clip_low >= 0.0 && p->clip_low <= 1.0) || !(p->clip_high >= 0.0)) { csv_set_error("clip range 1 - %g .. 1 + %g", p->clip_low, p->clip_high); return CSV_EINVAL; }
    if (!(p->beta >= 0.0) || !isfinite(p->beta)) { csv_set_error("beta=%g is negative or not finite", p->beta); return CSV_EINVAL; }
    if (N > 0 && (!d_old_logp || !d_advantages || !d_weights)) { csv_set_error("null d_old_logp, d_advantages or d_weights"); return CSV_EINVAL; }
    if (N > 0 && p->beta > 0.0 && !d_ref_logp) { csv_set_error("beta=%g needs d_ref_logp", p->beta); return CSV_EINVAL; }
    const int64_t n4 = 4ll * N;
    const Span writes[] = {vec("d_loss", d_loss, 4), vec("d_logp", d_logp, n4), matrix("d_grad", d_grad, type, ld_grad, N, V), vec("d_scratch", d_scratch, (int64_t)need)};
    const Span reads[] = {matrix("d_logits", d_logits, type, ld, N, V), vec("d_tokens", d_tokens, n4), vec("d_old_logp", d_old_logp, n4),
                          vec("d_ref_logp", p->beta > 0.0 ? d_ref_logp : nullptr, n4), vec("d_advantages", d_advantages, n4), vec("d_weights", d_weights, n4)};
    if ((rc = check_apart(writes, reads))) return rc;
    RowArgs a = {};
    a.x = d_logits; a.ld = ld; a.N = N; a.V = V; a.tokens = d_tokens; a.c = p->inv_temperature; a.c2 = split(a.c * LOG2E);
    a.old_logp = d_old_logp; a.ref_logp = d_ref_logp; a.adv = d_advantages; a.weights = d_weights;
    a.clip_low = p->clip_low; a.clip_high = p->clip_high; a.beta = p->beta;
    a.logp = d_logp; a.grad = d_grad; a.ld_grad = ld_grad;
    const bool by_parts = N > 0 && N < few_rows(type);
    place_scratch(a, d_scratch, by_parts);
    const hipStream_t st = (hipStream_t)stream;
    if (by_parts) {
        if (type == CSV_F32) part_kernel<float, true><<<N * a.parts, 256, 0, st>>>(a);
        else part_kernel<uint16_t, true><<<N * a.parts, 256, 0, st>>>(a);
        CSV_LAUNCH_CHECK("part_kernel");
        const int parts = d_grad ? a.parts : 1;
        if (type == CSV_F32) policy_kernel<float><<<N * parts, 256, 0, st>>>(a, parts, d_loss);
        else policy_kernel<uint16_t><<<N * parts, 256, 0, st>>>(a, parts, d_loss);
        CSV_LAUNCH_CHECK("policy_kernel");
        return CSV_OK;
    }
    if (N > 0) {
        if (type == CSV_F32) row_kernel<float, true><<<N, 1024, 0, st>>>(a);
        else row_kernel<uint16_t, true><<<N, 1024, 0, st>>>(a);
        CSV_LAUNCH_CHECK("row_kernel");
    }
    sum_kernel<<<1, 1024, 0, st>>>(a.terms, N, d_loss);
    CSV_LAUNCH_CHECK("sum_kernel");
    return CSV_OK;
}
