// Log-probabilities of given tokens from rows of logits, their gradient, and the clipped policy loss with its gradient.
//
//   row_kernel    one block per row of logits: the largest logit m and s = sum exp(c (x - m)), the log-probability of the row's token, and
//                 as the call asks the row's loss term and its gradient row
//   grad_kernel   gradient rows from given m, s and coefficients
//   sum_kernel    the loss: the rows' terms in float64, in one order
//
// A row starts wherever its stride puts it: it is read as up to E - 1 single elements, 16-byte pieces of E elements, and up to
// E - 1 single elements (E = 4 or 8); the single ones go to the first threads, one each.
#include "csv_common.h"

#include <math.h>

#define THREADS 1024
#define LOG2E 1.44269504089f
#define LOWEST (-3.402823466e38f)   // start of a running maximum: exp(c (-inf - LOWEST)) is 0, not NaN

struct RowArgs {
    const void* x;
    int64_t ld;
    int N, V;
    const int32_t* tokens;
    float c;                 // inverse temperature
    const float* old_logp;   // policy loss
    const float* ref_logp;
    const float* adv;
    const float* weights;
    float clip_low, clip_high, beta;
    const float* stats_in;   // gradient alone
    const float* grad_logp;
    float* logp;
    float* stats;
    double* terms;
    void* grad;
    int64_t ld_grad;
};

template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4;
    float v[4];
    __device__ __forceinline__ void load(const float* p) { const float4 u = *(const float4*)p; v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w; }
    __device__ __forceinline__ void store(float* p) const { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<uint16_t> {
    static constexpr int E = 8;
    float v[8];
    __device__ __forceinline__ void load(const uint16_t* p) {
        const uint4 u = *(const uint4*)p;
        v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
        v[4] = bf16_lo(u.z); v[5] = bf16_hi(u.z); v[6] = bf16_lo(u.w); v[7] = bf16_hi(u.w);
    }
    __device__ __forceinline__ void store(uint16_t* p) const {
        uint32_t w[4];
        for (int j = 0; j < 4; ++j)
            w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * j + 1]) << 16;
        *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
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

// exp(c (x - m)) as 2^((x - m) c log2(e)); the difference is taken first, so that far logits keep their digits
__device__ __forceinline__ float exp_at(float x, float m, float c2) { return __builtin_amdgcn_exp2f((x - m) * c2); }

// c g ([j = t] - p_j) over a row, eg = c g, k = c g / s
template <typename T>
__device__ __forceinline__ void write_grad(const Row<T>& row, T* out, int V, int token, float m, float c2, float eg, float k) {
    constexpr int E = Vec<T>::E;
    const int tid = threadIdx.x, one = row.single(tid);
    if (one >= 0) put(out + one, (one == token ? eg : 0.f) - k * exp_at(get(row.p + one), m, c2));
    const bool aligned = ((uintptr_t)(out + row.head) & 15) == 0;
    for (int i = tid; i < row.pieces; i += THREADS) {
        Vec<T> x;
        const int e0 = row.head + i * E;
        x.load(row.p + e0);
        for (int j = 0; j < E; ++j) x.v[j] = (e0 + j == token ? eg : 0.f) - k * exp_at(x.v[j], m, c2);
        if (aligned) x.store(out + e0);
        else
            for (int j = 0; j < E; ++j) put(out + e0 + j, x.v[j]);
    }
}
template <typename T>
__device__ __forceinline__ void write_zeros(T* out, int V) {
    const Row<T> row(out, V);
    const int one = row.single(threadIdx.x);
    if (one >= 0) put(out + one, 0.f);
    for (int i = threadIdx.x; i < row.pieces; i += THREADS) *(uint4*)(out + row.head + i * Vec<T>::E) = make_uint4(0, 0, 0, 0);
}

// The loss term of a row and its derivative by the log-probability, in float64: one thread per row does this, and close to a clip border
// the digits decide which branch holds.
__device__ __forceinline__ double policy_term(const RowArgs& a, int i, double logp, double& g) {
    const double A = a.adv[i], w = a.weights[i], r = exp(logp - (double)a.old_logp[i]);
    const double lo = 1.0 - (double)a.clip_low, hi = 1.0 + (double)a.clip_high, whole = r * A, cut = fmin(fmax(r, lo), hi) * A;
    double term = cut < whole ? -cut : -whole;
    double d = (A >= 0.0 ? r <= hi : r >= lo) ? -A * r : 0.0;
    if (a.beta > 0.f) {
        const double k = (double)a.ref_logp[i] - logp, em = expm1(k);
        term += (double)a.beta * (em - k);
        d -= (double)a.beta * em;
    }
    g = w * d;
    return w * term;
}

template <typename T, bool POLICY>
__global__ __launch_bounds__(THREADS) void row_kernel(RowArgs a) {
    __shared__ float red[16];
    __shared__ float coef;
    constexpr int E = Vec<T>::E;
    const int i = blockIdx.x, tid = threadIdx.x, token = a.tokens[i];
    T* grad = POLICY && a.grad ? (T*)a.grad + (int64_t)i * a.ld_grad : nullptr;
    if (token < 0 || token >= a.V || (POLICY && a.weights[i] == 0.f)) {
        if (tid == 0) {
            if (a.logp) a.logp[i] = 0.f;
            if (POLICY) a.terms[i] = 0.0;
            else a.stats[2 * i] = a.stats[2 * i + 1] = 0.f;
        }
        if (grad) write_zeros(grad, a.V);
        return;
    }
    const Row<T> row((const T*)a.x + (int64_t)i * a.ld, a.V);
    const float c2 = a.c * LOG2E;
    float m = LOWEST, s = 0.f;
    const int one = row.single(tid);
    if (one >= 0) {
        const float x = get(row.p + one);
        m = fmaxf(m, x);
        s = exp_at(x, m, c2);
    }
    for (int k = tid; k < row.pieces; k += THREADS) {
        Vec<T> x;
        x.load(row.p + row.head + k * E);
        float top = x.v[0];
        for (int j = 1; j < E; ++j) top = fmaxf(top, x.v[j]);
        top = fmaxf(m, top);
        float add = 0.f;
        for (int j = 0; j < E; ++j) add += exp_at(x.v[j], top, c2);
        s = s * exp_at(m, top, c2) + add;
        m = top;
    }
    const float M = block_max(m, red);
    s = block_sum(s * exp_at(m, M, c2), red);
    const float xt = get(row.p + token);
    if (tid == 0) {
        const double logp = s == 0.f ? -INFINITY : (double)a.c * ((double)xt - (double)M) - log((double)s);
        if (a.logp) a.logp[i] = (float)logp;
        if (POLICY) {
            double g;
            a.terms[i] = policy_term(a, i, logp, g);
            coef = (float)(g * (double)a.c);
        } else {
            a.stats[2 * i] = M;
            a.stats[2 * i + 1] = s;
        }
    }
    if (!POLICY || !grad) return;
    __syncthreads();                            // the row's token has been read by now: the gradient may replace the logits
    if (s == 0.f) write_zeros(grad, a.V);
    else write_grad(row, grad, a.V, token, M, c2, coef, coef / s);
}

template <typename T>
__global__ __launch_bounds__(THREADS) void grad_kernel(RowArgs a) {
    const int i = blockIdx.x, token = a.tokens[i];
    T* grad = (T*)a.grad + (int64_t)i * a.ld_grad;
    const float m = a.stats_in[2 * i], s = a.stats_in[2 * i + 1], g = a.grad_logp[i] * a.c;
    if (token < 0 || token >= a.V || g == 0.f || s == 0.f) write_zeros(grad, a.V);
    else write_grad(Row<T>((const T*)a.x + (int64_t)i * a.ld, a.V), grad, a.V, token, m, a.c * LOG2E, g, g / s);
}

__global__ __launch_bounds__(THREADS) void sum_kernel(const double* __restrict__ terms, int N, float* __restrict__ loss) {
    __shared__ double part[THREADS];
    double s = 0.0;
    for (int i = threadIdx.x; i < N; i += THREADS) s += terms[i];
    part[threadIdx.x] = s;
    for (int h = THREADS / 2; h > 0; h >>= 1) {
        __syncthreads();
        if (threadIdx.x < h) part[threadIdx.x] += part[threadIdx.x + h];
    }
    if (threadIdx.x == 0) *loss = (float)part[0];
}

// ------------------------------------------------------------------------------------------------ entry points
static int check_logits(const void* x, int type, int64_t ld, int N, int V, const int32_t* tokens, float c) {
    if (N < 0 || V < 1) { csv_set_error("need N >= 0 and V >= 1 (N=%d, V=%d)", N, V); return CSV_ESHAPE; }
    if (type != CSV_F32 && type != CSV_BF16) { csv_set_error("bad element type %d", type); return CSV_EINVAL; }
    if (ld < V) { csv_set_error("row stride %lld is below V=%d", (long long)ld, V); return CSV_ESHAPE; }
    if (!(c > 0.f) || !isfinite(c * LOG2E)) { csv_set_error("inverse temperature %g is not positive and finite", (double)c); return CSV_EINVAL; }
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
static int check_scratch(int N, int V, const void* p, size_t have) {
    size_t need = 0;
    const int rc = csv_loss_scratch(N, V, &need);
    if (rc) return rc;
    if (need && (!p || have < need)) { csv_set_error("scratch of %zu bytes, %zu are needed", p ? have : (size_t)0, need); return CSV_ESHAPE; }
    if (need && ((uintptr_t)p & 15)) { csv_set_error("scratch has to be 16-byte aligned"); return CSV_EINVAL; }
    return CSV_OK;
}

extern "C" int csv_loss_scratch(int N, int V, size_t* bytes) {
    if (N < 0 || V < 1) { csv_set_error("need N >= 0 and V >= 1 (N=%d, V=%d)", N, V); return CSV_ESHAPE; }
    if (!bytes) { csv_set_error("null bytes"); return CSV_EINVAL; }
    *bytes = (size_t)N * sizeof(double);
    return CSV_OK;
}

extern "C" int csv_token_logprobs(const void* d_logits, int type, int64_t ld, int N, int V, const int32_t* d_tokens, float inv_temperature, float* d_logp,
                                  float* d_stats, void* d_scratch, size_t scratch_bytes, void* stream) {
    int rc = check_logits(d_logits, type, ld, N, V, d_tokens, inv_temperature);
    if (!rc) rc = check_scratch(N, V, d_scratch, scratch_bytes);
    if (rc || N == 0) return rc;
    if (!d_logp || !d_stats) { csv_set_error("null d_logp or d_stats"); return CSV_EINVAL; }
    RowArgs a = {};
    a.x = d_logits; a.ld = ld; a.N = N; a.V = V; a.tokens = d_tokens; a.c = inv_temperature; a.logp = d_logp; a.stats = d_stats;
    if (type == CSV_F32) row_kernel<float, false><<<N, THREADS, 0, (hipStream_t)stream>>>(a);
    else row_kernel<uint16_t, false><<<N, THREADS, 0, (hipStream_t)stream>>>(a);
    CSV_LAUNCH_CHECK("row_kernel");
    return CSV_OK;
}

extern "C" int csv_token_logprobs_backward(const void* d_logits, int type, int64_t ld, int N, int V, const int32_t* d_tokens, const float* d_stats,
                                           const float* d_grad_logp, float inv_temperature, void* d_grad, int64_t ld_grad, void* stream) {
    int rc = check_logits(d_logits, type, ld, N, V, d_tokens, inv_temperature);
    if (!rc) rc = check_grad(d_logits, type, ld, N, V, d_grad, ld_grad);
    if (rc || N == 0) return rc;
    if (!d_stats || !d_grad_logp || !d_grad) { csv_set_error("null d_stats, d_grad_logp or d_grad"); return CSV_EINVAL; }
    RowArgs a = {};
    a.x = d_logits; a.ld = ld; a.N = N; a.V = V; a.tokens = d_tokens; a.c = inv_temperature; a.stats_in = d_stats; a.grad_logp = d_grad_logp;
    a.grad = d_grad; a.ld_grad = ld_grad;
    if (type == CSV_F32) grad_kernel<float><<<N, THREADS, 0, (hipStream_t)stream>>>(a);
    else grad_kernel<uint16_t><<<N, THREADS, 0, (hipStream_t)stream>>>(a);
    CSV_LAUNCH_CHECK("grad_kernel");
    return CSV_OK;
}

extern "C" int csv_policy_loss(const void* d_logits, int type, int64_t ld, int N, int V, const int32_t* d_tokens, const float* d_old_logp,
                               const float* d_ref_logp, const float* d_advantages, const float* d_weights, const csv_policy_params* p, float* d_loss,
                               float* d_logp, void* d_grad, int64_t ld_grad, void* d_scratch, size_t scratch_bytes, void* stream) {
    if (!p || !d_loss) { csv_set_error("null params or d_loss"); return CSV_EINVAL; }
    int rc = check_logits(d_logits, type, ld, N, V, d_tokens, p->inv_temperature);
    if (!rc && d_grad) rc = check_grad(d_logits, type, ld, N, V, d_grad, ld_grad);
    if (!rc) rc = check_scratch(N, V, d_scratch, scratch_bytes);
    if (rc) return rc;
    if (!(p->clip_low >= 0.f && p->clip_low <= 1.f) || !(p->clip_high >= 0.f)) { csv_set_error("clip range 1 - %g .. 1 + %g", (double)p->clip_low, (double)p->clip_high); return CSV_EINVAL; }
    if (!(p->beta >= 0.f) || !isfinite(p->beta)) { csv_set_error("beta=%g is negative or not finite", (double)p->beta); return CSV_EINVAL; }
    if (N > 0 && (!d_old_logp || !d_advantages || !d_weights)) { csv_set_error("null d_old_logp, d_advantages or d_weights"); return CSV_EINVAL; }
    if (N > 0 && p->beta > 0.f && !d_ref_logp) { csv_set_error("beta=%g needs d_ref_logp", (double)p->beta); return CSV_EINVAL; }
    RowArgs a = {};
    a.x = d_logits; a.ld = ld; a.N = N; a.V = V; a.tokens = d_tokens; a.c = p->inv_temperature;
    a.old_logp = d_old_logp; a.ref_logp = d_ref_logp; a.adv = d_advantages; a.weights = d_weights;
    a.clip_low = p->clip_low; a.clip_high = p->clip_high; a.beta = p->beta;
    a.logp = d_logp; a.terms = (double*)d_scratch; a.grad = d_grad; a.ld_grad = ld_grad;
    const hipStream_t st = (hipStream_t)stream;
    if (N > 0) {
        if (type == CSV_F32) row_kernel<float, true><<<N, THREADS, 0, st>>>(a);
        else row_kernel<uint16_t, true><<<N, THREADS, 0, st>>>(a);
        CSV_LAUNCH_CHECK("row_kernel");
    }
    sum_kernel<<<1, THREADS, 0, st>>>(a.terms, N, d_loss);
    CSV_LAUNCH_CHECK("sum_kernel");
    return CSV_OK;
}
