// Loss that distils a teacher's top logits, with the gradient for the student's logits.  Per row, with p = softmax(teacher / tau) over the row's
// entries, q = softmax(s / tau) and q1 = softmax(s) over the vocabulary:
//   loss = w tau^2 sum_j p_j (log p_j - log q[id_j]) + (1 - w) (-log q1[label])
//   grad_v = scale (w tau (q_v - sum of the p_j with id_j = v) + (1 - w) (q1_v - [v = label]))
// The logits are read, the gradient is written: HBM is the bound, and the exponentials (two an element and temperature) come close to it.
#include "seqops.h"
#include "launch.h"

#include <cuda_bf16.h>

namespace fdg {
namespace {

using bf16 = __nv_bfloat16;
__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

constexpr int THREADS = 256;

struct Max { __device__ float operator()(float a, float b) const { return a != a || a > b ? a : b; } };      // NaN stays
struct Add { __device__ float operator()(float a, float b) const { return a + b; } };
// over the CTA, the same value in every thread
template <typename F>
__device__ float reduce(float v, F f, float* sh) {
    for (int d = 16; d; d >>= 1) v = f(v, __shfl_xor_sync(~0u, v, d));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = sh[0];
    for (int i = 1; i < THREADS / 32; ++i) v = f(v, sh[i]);
    return v;
}

// A CTA per row.
template <typename TI, typename TO>
__global__ void __launch_bounds__(THREADS) distill_k(DistillArgs a) {
    extern __shared__ float dyn[];
    float* const tp = dyn;                          // p of the entries, 0 where an entry is left out
    float* const ts = dyn + a.k;                    // the student's logits there
    int* const tid = (int*)(dyn + 2 * a.k);         // their ids, -1 where one is left out
    __shared__ float sh[THREADS / 32];
    const long row = blockIdx.x;
    const TI* const x = (const TI*)a.logits + row * a.logits_stride;
    TO* const g = a.grad ? (TO*)a.grad + row * a.grad_stride : nullptr;
    const int label = a.labels ? a.labels[row] : 0;
    if (label < 0 || label >= a.V) {                // the row does not count
        if (threadIdx.x == 0) a.loss[row] = 0.f;
        if (g) for (long v = threadIdx.x; v < a.V; v += THREADS) st(g + v, 0.f);
        return;
    }
    const float itau = 1.f / a.tau;
    float m = -INFINITY;
    for (long v = threadIdx.x; v < a.V; v += THREADS) m = Max()(ld(x + v), m);
    m = reduce(m, Max(), sh);
    float zt = 0.f, z1 = 0.f;
    for (long v = threadIdx.x; v < a.V; v += THREADS) {
        const float d = ld(x + v) - m;
        if (a.weight > 0.f) zt += expf(d * itau);
        if (a.weight < 1.f) z1 += expf(d);
    }
    if (a.weight > 0.f) zt = reduce(zt, Add(), sh);
    if (a.weight < 1.f) z1 = reduce(z1, Add(), sh);
    float loss = 0.f;
    bool taught = false;
    if (a.weight > 0.f) {
        const float logz = logf(zt);
        float tm = -INFINITY;
        for (int j = threadIdx.x; j < a.k; j += THREADS) {
            const int id = a.ids[row * a.k + j];
            const bool in = id >= 0 && id < a.V;
            tid[j] = in ? id : -1;
            tp[j] = in ? a.teacher[row * a.k + j] : -INFINITY;
            ts[j] = in ? ld(x + id) : 0.f;
            tm = Max()(tp[j], tm);
        }
        tm = reduce(tm, Max(), sh);
        taught = tm != -INFINITY;                   // without an entry that has any weight the term is nothing
        if (taught) {
            float tz = 0.f;
            for (int j = threadIdx.x; j < a.k; j += THREADS) tz += expf((tp[j] - tm) * itau);
            tz = reduce(tz, Add(), sh);
            const float logtz = logf(tz), inv = 1.f / tz;
            float part = 0.f;
            for (int j = threadIdx.x; j < a.k; j += THREADS) {
                const float t = (tp[j] - tm) * itau, pj = expf(t) * inv;
                if (pj != 0.f) part += pj * ((t - logtz) - ((ts[j] - m) * itau - logz));
                tp[j] = pj;
            }
            loss = a.weight * a.tau * a.tau * reduce(part, Add(), sh);
        }
    }
    if (a.weight < 1.f) loss += (1.f - a.weight) * (logf(z1) - (ld(x + label) - m));
    if (threadIdx.x == 0) a.loss[row] = loss;
    if (!g) return;
    const float ct = taught ? a.weight * a.tau : 0.f, c1 = 1.f - a.weight, it = 1.f / zt, i1 = 1.f / z1;
    // gradient at v, whose logit is s and whose entries' p add up to p
    auto at = [&](long v, float s, float p) {
        float r = 0.f;
        if (ct != 0.f) r += ct * (expf((s - m) * itau) * it - p);
        if (c1 != 0.f) r += c1 * (expf(s - m) * i1 - (v == label ? 1.f : 0.f));
        return r * a.scale;
    };
    __syncthreads();                                // every logit that the loss needs has been read (g may be x)
    for (long v = threadIdx.x; v < a.V; v += THREADS) st(g + v, at(v, ld(x + v), 0.f));
    if (!taught) return;
    __syncthreads();
    for (int j = threadIdx.x; j < a.k; j += THREADS) {
        const int id = tid[j];
        if (id < 0) continue;
        float p = 0.f;                              // an id that occurs more than once is its first entry's
        bool first = true;
        for (int i = 0; i < a.k; ++i) if (tid[i] == id) { if (i < j) first = false; p += tp[i]; }
        if (first) st(g + id, at(id, ts[j], p));
    }
}

}  // namespace

cudaError_t distill(int dti, int dtg, const DistillArgs& a, cudaStream_t s) {
    if (a.M == 0) return cudaSuccess;
    Scope sc(KC_DISTILL, 10.0 * a.M * a.V, (double)a.M * a.V * ((dti ? 2 : 4) + (a.grad ? (dtg ? 2 : 4) : 0)), s);
    const size_t smem = 12u * (size_t)a.k;
    if (dti) return klaunch(distill_k<bf16, bf16>, (unsigned)a.M, THREADS, smem, s, a);
    return dtg ? klaunch(distill_k<float, bf16>, (unsigned)a.M, THREADS, smem, s, a) : klaunch(distill_k<float, float>, (unsigned)a.M, THREADS, smem, s, a);
}

}  // namespace fdg
