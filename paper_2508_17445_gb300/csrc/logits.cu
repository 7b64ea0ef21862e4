// logits.cu -- sm_103a kernels of the operators on a policy's logits (treepo.h).
//
// A row of logits x_j gives, with c = log2(e) / T, its maximum m and with
// d_j = c (x_j - m) the sums  s = sum 2^d_j,  t = sum 2^d_j d_j:
//   LSE = m / T + ln 2 log2 s,  ln p_j = ln 2 (d_j - log2 s),
//   H = ln 2 (log2 s - t / s).
// The difference is taken before the product: a row of the type's lowest values
// would overflow in c x_j, and the row's largest terms lose nothing.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "logits.h"

namespace tp {
namespace {

constexpr int kThreads = 512;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -INFINITY;

__device__ __forceinline__ float exp2_approx(float x) {  // 2 ulp; exp2(-inf) = +0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ float load_value(const void* p, int64_t i, int dtype) {
    if (dtype == TP_F32) return ((const float*)p)[i];
    if (dtype == TP_F16) return __half2float(((const __half*)p)[i]);
    return __bfloat162float(((const __nv_bfloat16*)p)[i]);
}

// Running statistics of a part of a row. m = -inf (and s = t = 0) while it
// holds no logit above -inf; a NaN or +inf makes s NaN.
struct Stats {
    float m = kNegInf, s = 0.f, t = 0.f;

    __device__ __forceinline__ void raise(float m2, float c) {  // m2 >= m
        const float d = m == kNegInf ? 0.f : c * (m - m2), f = m == kNegInf ? 0.f : exp2_approx(d);
        t = f * (t + s * fmaxf(d, -1e30f));
        s *= f;
        m = m2;
    }
    __device__ __forceinline__ void add(float x, float c) {
        if (x > m) raise(x, c);
        const float d = c * (x - (m == kNegInf ? 0.f : m)), e = exp2_approx(d);
        s += e;
        t = fmaf(e, fmaxf(d, -1e30f), t);  // (0 times -inf stays 0)
    }
    __device__ __forceinline__ void join(Stats b, float c) {
        if (b.m > m) {
            const Stats x = *this;
            *this = b;
            b = x;
        }
        if (b.m == kNegInf) {  // nothing in b, or only NaN
            s += b.s;
            return;
        }
        b.raise(m, c);
        s += b.s;
        t += b.t;
    }
};

struct RowResult {
    float m, c, inv_t, log2_s, entropy, lse;
    bool empty;  // -inf logits only

    __device__ __forceinline__ RowResult(const Stats& a, float c_, float inv_t_) : c(c_), inv_t(inv_t_) {
        empty = a.m == kNegInf && a.s == 0.f;
        m = empty ? 0.f : a.m;
        log2_s = log2f(a.s);
        entropy = empty ? 0.f : kLn2 * (log2_s - a.t / a.s);
        lse = fmaf(log2_s, kLn2, m * inv_t);
    }
    // ln p of logit x (-inf of an empty row); not by way of log2 p, which overflows for the type's lowest values
    __device__ __forceinline__ float logp(float x) const { return empty ? kNegInf : fmaf(inv_t, x - m, -kLn2 * log2_s); }
};

// Policy term of the loss, and the gradient's factor g of (1[j = token] - p_j), both without the weight.
__device__ __forceinline__ float policy_term(float logp, float a, const float* old, int64_t i, float lo, float hi, float& g) {
    const float r = old ? expf(logp - old[i]) : 1.f;
    g = NAN;
    if (isnan(logp) || isnan(r) || isnan(a)) return NAN;
    const bool clipped = (a > 0.f && r > 1.f + hi) || (a < 0.f && r < 1.f - lo);
    g = clipped || a == 0.f ? 0.f : -r * a;
    return a == 0.f ? 0.f : -fminf(r * a, fminf(fmaxf(r, 1.f - lo), 1.f + hi) * a);
}

template <typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, Op op, V* smem) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int off = 16; off; off >>= 1) {
        V o;
        static_assert(sizeof(V) % 4 == 0);
        uint32_t* d = (uint32_t*)&o;
        const uint32_t* w = (const uint32_t*)&v;
        for (int k = 0; k < (int)sizeof(V) / 4; ++k) d[k] = __shfl_xor_sync(0xffffffffu, w[k], off);
        v = op(v, o);
    }
    __syncthreads();
    if (lane == 0) smem[warp] = v;
    __syncthreads();
    v = smem[0];
    for (int k = 1; k < kThreads / 32; ++k) v = op(v, smem[k]);
    return v;
}

__device__ __forceinline__ uint32_t order_key(float x) {  // ascending with x; -0 as +0
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

enum { OP_LOGPROBS, OP_BACKWARD, OP_POLICY, OP_DISTILL };

// The plainest form: one CTA a row, every pass read from memory.
template <typename T, int OP>
__global__ void __launch_bounds__(kThreads) row_kernel(const RowArgs a) {
    __shared__ Stats sh_stats[kThreads / 32];
    __shared__ unsigned long long sh_key[kThreads / 32];
    __shared__ float sh_f[kThreads / 32];
    const int64_t i = blockIdx.x;
    const int V = a.vocab, tid = threadIdx.x;
    const T* x = (const T*)a.x + i * a.x_stride;
    T* dx = (T*)a.dx + i * a.dx_stride;
    const float c = kLog2e / a.temperature, inv_t = 1.f / a.temperature;
    const int32_t tok = OP != OP_DISTILL && a.tokens ? a.tokens[i] : 0;
    bool live = tok >= 0;
    float q_max = kNegInf, q_sum = 0.f;
    bool q_bad = false;
    if (OP == OP_DISTILL) {
        for (int k = tid; k < a.k; k += kThreads)
            if (a.teacher_ids[i * a.k + k] >= 0) {
                const float v = load_value(a.teacher_logits, i * a.k + k, a.teacher_dtype);
                q_bad |= isnan(v) || v == INFINITY;
                q_max = fmaxf(q_max, v);
            }
        q_max = block_reduce(q_max, [](float p, float q) { return fmaxf(p, q); }, sh_f);
        q_bad = __syncthreads_or(q_bad);
        live = q_bad || q_max > kNegInf;
        if (live && !q_bad) {
            for (int k = tid; k < a.k; k += kThreads)
                if (a.teacher_ids[i * a.k + k] >= 0)
                    q_sum += exp2_approx(c * (load_value(a.teacher_logits, i * a.k + k, a.teacher_dtype) - q_max));
            q_sum = block_reduce(q_sum, [](float p, float q) { return p + q; }, sh_f);
        }
    }
    if (!live) {
        if (a.dx)
            for (int j = tid; j < V; j += kThreads) dx[j] = from_f32<T>(0.f);
        if (tid == 0) {
            if (a.logp) a.logp[i] = 0.f;
            if (a.entropy) a.entropy[i] = 0.f;
            if (a.lse) a.lse[i] = 0.f;
            if (a.loss) a.loss[i] = 0.f;
        }
        if (OP == OP_LOGPROBS)
            for (int k = tid; k < a.k; k += kThreads) {
                a.top_ids[i * a.k + k] = -1;
                a.top_logp[i * a.k + k] = kNegInf;
            }
        return;
    }
    float x_tok = NAN;
    if (OP != OP_DISTILL && a.tokens && tok < V) x_tok = to_f32(x[tok]);
    if (OP == OP_BACKWARD) {
        const float lse = a.lse_in[i], gl = a.dlogp ? a.dlogp[i] : 0.f, gh = a.dentropy ? a.dentropy[i] : 0.f;
        const float h = a.dentropy ? a.entropy_in[i] : 0.f;
        const bool bad = a.dlogp && tok >= V;
        for (int j = tid; j < V; j += kThreads) {
            const float lp = to_f32(x[j]) * inv_t - lse, p = exp2_approx(lp * kLog2e);
            float d = gl * ((a.dlogp && j == tok ? 1.f : 0.f) - p) - gh * p * (fmaxf(lp, -1e30f) + h);
            if (lse == kNegInf) d = 0.f;
            if (bad) d = NAN;
            dx[j] = from_f32<T>(d * inv_t);
        }
        return;
    }
    Stats st;
    for (int j = tid; j < V; j += kThreads) st.add(to_f32(x[j]), c);
    st = block_reduce(st, [c](Stats p, Stats q) { p.join(q, c); return p; }, sh_stats);
    const RowResult r(st, c, inv_t);
    if (OP == OP_LOGPROBS) {
        if (tid == 0) {
            if (a.logp) a.logp[i] = tok < V ? r.logp(x_tok) : NAN;
            if (a.entropy) a.entropy[i] = r.entropy;
            if (a.lse) a.lse[i] = r.lse;
        }
        unsigned long long last = ~0ull;
        for (int k = 0; k < a.k; ++k) {
            unsigned long long best = 0;
            if (!isnan(r.lse))
                for (int j = tid; j < V; j += kThreads) {
                    const float v = to_f32(x[j]);
                    const unsigned long long key = (unsigned long long)order_key(v) << 32 | (0xffffffffu - j);
                    if (v > kNegInf && key < last && key > best) best = key;
                }
            best = block_reduce(best, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; }, sh_key);
            if (tid == 0) {
                const int32_t id = best ? (int32_t)(0xffffffffu - (uint32_t)best) : -1;
                a.top_ids[i * a.k + k] = id;
                a.top_logp[i * a.k + k] = isnan(r.lse) ? NAN : id < 0 ? kNegInf : r.logp(to_f32(x[id]));
            }
            last = best;
        }
        return;
    }
    const float w = a.weight ? a.weight[i] : 1.f;
    if (OP == OP_POLICY) {
        float g;
        const float logp = tok < V ? r.logp(x_tok) : NAN;
        const float term = policy_term(logp, a.advantage[i], a.old_logp, i, a.clip_low, a.clip_high, g);
        const float beta = a.entropy_coef;
        __syncthreads();  // x_tok read by everyone before an in-place gradient
        if (tid == 0) {
            a.loss[i] = w * (term - beta * r.entropy);
            if (a.logp) a.logp[i] = logp;
            if (a.entropy) a.entropy[i] = r.entropy;
        }
        if (!a.dx) return;
        for (int j = tid; j < V; j += kThreads) {
            const float lp = r.logp(to_f32(x[j])), p = exp2_approx(lp * kLog2e);
            float d = g * ((j == tok ? 1.f : 0.f) - p) + beta * p * (fmaxf(lp, -1e30f) + r.entropy);
            dx[j] = from_f32<T>(r.empty && !isnan(g) ? 0.f : d * w * inv_t);
        }
        return;
    }
    // distillation
    float loss = 0.f;
    const float log2_q = log2f(q_sum);
    bool bad = q_bad || isnan(r.lse);
    for (int k = tid; k < a.k; k += kThreads) {
        const int32_t id = a.teacher_ids[i * a.k + k];
        if (id < 0) continue;
        const float lq = c * (load_value(a.teacher_logits, i * a.k + k, a.teacher_dtype) - q_max) - log2_q, q = exp2_approx(lq);
        if (q > 0.f && id >= V) bad = true;
        if (q > 0.f && id < V) loss += q * (kLn2 * lq - r.logp(to_f32(x[id])));
    }
    loss = block_reduce(loss, [](float p, float q) { return p + q; }, sh_f);
    bad = __syncthreads_or(bad);
    if (tid == 0) a.loss[i] = bad ? NAN : w * loss;
    if (!a.dx) return;
    for (int j = tid; j < V; j += kThreads) {
        float p = exp2_approx(r.logp(to_f32(x[j])) * kLog2e);
        for (int k = 0; k < a.k; ++k)
            if (a.teacher_ids[i * a.k + k] == j)
                p -= exp2_approx(c * (load_value(a.teacher_logits, i * a.k + k, a.teacher_dtype) - q_max) - log2_q);
        dx[j] = from_f32<T>(bad ? NAN : r.empty ? 0.f : p * w * inv_t);
    }
}

template <int OP>
cudaError_t launch(const RowArgs& a, cudaStream_t s) {
    if (a.dtype == TP_F32)
        row_kernel<float, OP><<<a.n, kThreads, 0, s>>>(a);
    else if (a.dtype == TP_F16)
        row_kernel<__half, OP><<<a.n, kThreads, 0, s>>>(a);
    else
        row_kernel<__nv_bfloat16, OP><<<a.n, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_token_logprobs(const RowArgs& a, cudaStream_t s) { return launch<OP_LOGPROBS>(a, s); }
cudaError_t launch_token_logprobs_backward(const RowArgs& a, cudaStream_t s) { return launch<OP_BACKWARD>(a, s); }
cudaError_t launch_policy_loss(const RowArgs& a, cudaStream_t s) { return launch<OP_POLICY>(a, s); }
cudaError_t launch_distill_loss(const RowArgs& a, cudaStream_t s) { return launch<OP_DISTILL>(a, s); }

}  // namespace tp
