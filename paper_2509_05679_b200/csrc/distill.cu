// Loss that distils a teacher's top logits, with the gradient for the student's logits.  Per row, with p = softmax(teacher / tau) over the row's
// entries, q = softmax(s / tau) and q1 = softmax(s) over the vocabulary:
//   loss = w tau^2 sum_j p_j (log p_j - log q[id_j]) + (1 - w) (-log q1[label])
//   grad_v = scale (w tau (q_v - sum of the p_j with id_j = v) + (1 - w) (q1_v - [v = label]))
// The logits are read once and the gradient is written once, which is the bound (HBM): a row stays in shared memory between its maximum, its sums and its
// gradient, cut over a cluster where one CTA's share would keep others from its SM.  The exponentials come close to being a second bound: the special-function
// unit makes 16 a cycle and SM, and an element needs one for either temperature in either pass.  Where tau is 1, 2, 4 or 8, exp(d) is a power of exp(d / tau).
#include "seqops.h"
#include "launch.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>

namespace fdg {
namespace {

namespace cg = cooperative_groups;
using bf16 = __nv_bfloat16;
__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int MAX_CLUSTER = 8;

// Results below 2^-126 are zero: beside the maximum's exponential, which is 1, that is nothing, and subnormal ones cost three instructions more.
__device__ __forceinline__ float exp2_(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
constexpr float LOG2E = 1.4426950408889634f;

struct Max { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };      // a NaN comes back by way of the sums
struct Add { __device__ float operator()(float a, float b) const { return a + b; } };
template <typename F> __device__ __forceinline__ float reduce_warp(float v, F f) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = f(v, __shfl_xor_sync(~0u, v, d));
    return v;
}

// The two exponentials of a logit whose difference to the maximum is d: of d / tau and, where the label's term needs it, of d.  SQ: log2(tau) squarings
// lead from the first to the second; -1: any tau.
template <int SQ, bool HARD> struct Exps {
    float c;                                        // log2(e) / tau
    __device__ __forceinline__ void operator()(float d, float& et, float& e1) const {
        et = exp2_(d * c);
        if (!HARD) { e1 = 0.f; return; }
        if (SQ < 0) e1 = exp2_(d * LOG2E);
        else {
            e1 = et;
#pragma unroll
            for (int i = 0; i < SQ; ++i) e1 *= e1;
        }
    }
};

// What a row's gradient is made of.
struct Terms {
    float m, ct, c1, it, i1, scale;                 // maximum; w tau and 1 - w, where the terms are there; 1 / sums
    // gradient at a logit whose exponentials are et, e1; p: of the entries there; hit: the label
    __device__ __forceinline__ float at(float et, float e1, float p, bool hit) const {
        return scale * (ct * (et * it - p) + c1 * (e1 * i1 - (hit ? 1.f : 0.f)));
    }
};

// ---- a warp per row: small vocabularies, where the row comes out of L1 in the later passes
constexpr long WARP_VOCAB = 1024;
constexpr int WARP_TOP = 128;
template <typename TI, typename TO, int SQ, bool HARD>
__global__ void __launch_bounds__(THREADS) distill_warp_k(DistillArgs a) {
    __shared__ float tp_[WARPS][WARP_TOP], ts_[WARPS][WARP_TOP];
    __shared__ int tid_[WARPS][WARP_TOP];
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, V = (int)a.V;
    float *const tp = tp_[w], *const ts = ts_[w];
    int* const tid = tid_[w];
    const long row = (long)blockIdx.x * WARPS + w;
    if (row >= a.M) return;
    const TI* const x = (const TI*)a.logits + row * a.logits_stride;
    TO* const g = a.grad ? (TO*)a.grad + row * a.grad_stride : nullptr;
    const int label = a.labels ? a.labels[row] : 0;
    if (label < 0 || label >= V) {                  // the row does not count
        if (lane == 0) a.loss[row] = 0.f;
        if (g) for (int v = lane; v < V; v += 32) st(g + v, 0.f);
        return;
    }
    const float itau = 1.f / a.tau;
    const Exps<SQ, HARD> exps{itau * LOG2E};
    Terms t{-INFINITY, 0.f, HARD ? 1.f - a.weight : 0.f, 0.f, 0.f, a.scale};
    float tm = -INFINITY;
    const int k = a.weight > 0.f ? a.k : 0;
    for (int j = lane; j < k; j += 32) {
        const int id = a.ids[row * a.k + j];
        const bool in = id >= 0 && id < V;
        tid[j] = in ? id : -1;
        tp[j] = in ? a.teacher[row * a.k + j] : -INFINITY;
        ts[j] = in ? ld(x + id) : 0.f;
        tm = fmaxf(tm, tp[j]);
    }
    for (int v = lane; v < V; v += 32) t.m = fmaxf(t.m, ld(x + v));
    t.m = reduce_warp(t.m, Max()); tm = reduce_warp(tm, Max());
    const bool taught = tm != -INFINITY;            // without an entry that has any weight the term is nothing
    float zt = 0.f, z1 = 0.f, tz = 0.f;
    for (int v = lane; v < V; v += 32) { float et, e1; exps(ld(x + v) - t.m, et, e1); zt += et; z1 += e1; }
    for (int j = lane; j < k; j += 32) tz += expf((tp[j] - tm) * itau);
    zt = reduce_warp(zt, Add()); z1 = reduce_warp(z1, Add()); tz = reduce_warp(tz, Add());
    float loss = 0.f;
    if (taught) {
        const float logz = logf(zt), logtz = logf(tz), inv = 1.f / tz;
        float part = 0.f;
        for (int j = lane; j < k; j += 32) {
            const float d = (tp[j] - tm) * itau, p = expf(d) * inv;
            if (p != 0.f) part += p * ((d - logtz) - ((ts[j] - t.m) * itau - logz));
            tp[j] = p;
        }
        loss = a.weight * a.tau * a.tau * reduce_warp(part, Add());
    }
    if (HARD) loss += t.c1 * (logf(z1) - (ld(x + label) - t.m));
    if (lane == 0) a.loss[row] = loss;
    if (!g) return;
    t.ct = taught ? a.weight * a.tau : 0.f; t.it = 1.f / zt; t.i1 = HARD ? 1.f / z1 : 0.f;
    __syncwarp();                                   // what the loss needs of the row has been read (g may be x)
    for (int v = lane; v < V; v += 32) { float et, e1; exps(ld(x + v) - t.m, et, e1); st(g + v, t.at(et, e1, 0.f, HARD && v == label)); }
    if (!taught) return;
    __syncwarp();
    for (int j = lane; j < k; j += 32) {
        const int id = tid[j];
        if (id < 0) continue;
        float p = 0.f;                              // an id that occurs more than once is its first entry's
        bool first = true;
        for (int i = 0; i < k; ++i) if (tid[i] == id) { if (i < j) first = false; p += tp[i]; }
        float et, e1;
        exps(ts[j] - t.m, et, e1);
        if (first) st(g + id, t.at(et, e1, p, HARD && id == label));
    }
}

// ---- a CTA or a cluster per row
template <typename T> struct Chunk;                 // 16 bytes of logits
template <> struct Chunk<float> { static constexpr int E = 4; };
template <> struct Chunk<bf16> { static constexpr int E = 8; };
__device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) { x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w); }
__device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ unsigned pair(float a, float b) { const __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *(const unsigned*)&v; }
__device__ __forceinline__ void put(float* p, const float (&x)[4]) { *(float4*)p = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void put(bf16* p, const float (&x)[4]) { *(uint2*)p = make_uint2(pair(x[0], x[1]), pair(x[2], x[3])); }
__device__ __forceinline__ void put(bf16* p, const float (&x)[8]) { *(uint4*)p = make_uint4(pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7])); }
__device__ __forceinline__ void copy16(void* smem, const void* g) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(smem)), "l"(g) : "memory");
}
template <int LEFT> __device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

constexpr int PARTS = 4;                            // of a row's copies, so that the maximum of the first begins while the last are on their way

// A row is cut into chunks of 16 aligned bytes, the first and the last one partly outside the row (there: -infinity).  A thread copies, and in every pass
// handles, the chunks threadIdx.x, + THREADS, ... of its CTA's share.
template <typename TI, typename TO, int SQ, bool HARD, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 3) distill_row_k(DistillArgs a, int ranks, int share) {
    constexpr int E = Chunk<TI>::E;
    extern __shared__ __align__(16) char dyn[];
    uint4* const chunks = (uint4*)dyn;
    TI* const xs = (TI*)dyn;                        // the element of the row at chunk * E + i
    float* const tp = (float*)(chunks + share);     // p of the entries, 0 where an entry is left out
    float* const ts = tp + a.k;                     // the student's logits there (where they are this CTA's)
    int* const tid = (int*)(ts + a.k);              // their places in the row's chunks, -1 where one is left out
    __shared__ float sh[6][WARPS];                  // a row of its own for every sum that is joined
    __shared__ float joined[4][MAX_CLUSTER];
    const int R = CLUSTER ? ranks : 1, rank = CLUSTER ? (int)(blockIdx.x % R) : 0, V = (int)a.V;
    const long row = blockIdx.x / R;
    const TI* const x = (const TI*)a.logits + row * a.logits_stride;
    TO* const g = a.grad ? (TO*)a.grad + row * a.grad_stride : nullptr;
    const int phase = (int)((uintptr_t)x / sizeof(TI) % E);                 // place of the row's first element
    const int first = rank * share, n = max(0, min(share, (V + phase + E - 1) / E - first));        // this CTA's chunks
    const int label = a.labels ? a.labels[row] : 0;
    if (label < 0 || label >= V) {                  // the row does not count
        if (rank == 0 && threadIdx.x == 0) a.loss[row] = 0.f;
        const int lo = max(0, first * E - phase), hi = min(V, (first + n) * E - phase);
        if (g) for (int v = lo + threadIdx.x; v < hi; v += THREADS) st(g + v, 0.f);
        return;
    }
    // over the cluster, the same value everywhere
    auto join = [&](float v, auto f, int slot) {
        v = reduce_warp(v, f);
        if ((threadIdx.x & 31) == 0) sh[slot][threadIdx.x >> 5] = v;
        __syncthreads();
        v = sh[slot][0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) v = f(v, sh[slot][i]);
        if (CLUSTER) {
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < R) *cl.map_shared_rank(&joined[slot][rank], threadIdx.x) = v;
            cl.sync();
            v = joined[slot][0];
            for (int r = 1; r < R; ++r) v = f(v, joined[slot][r]);
        }
        return v;
    };
    const auto inside = [&](int c) { return (first + c) * E >= phase && (first + c + 1) * E <= V + phase; };      // the whole chunk lies in the row
    const int part = (n + PARTS - 1) / PARTS;
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
        for (int c = q * part + threadIdx.x; c < min(n, (q + 1) * part); c += THREADS) {
            const long v = (long)(first + c) * E - phase;
            if (inside(c)) copy16(chunks + c, x + v);
            else
                for (int i = 0; i < E; ++i) {
                    if (v + i >= 0 && v + i < V) xs[c * E + i] = x[v + i];
                    else st(xs + c * E + i, -INFINITY);
                }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (CLUSTER) cg::this_cluster().sync();         // every CTA is there before anyone writes to its shared memory
    const float itau = 1.f / a.tau;
    const Exps<SQ, HARD> exps{itau * LOG2E};
    // the teacher, while the row arrives
    const int k = a.weight > 0.f ? a.k : 0;
    float tm = -INFINITY;
    for (int j = threadIdx.x; j < k; j += THREADS) {
        const int id = a.ids[row * a.k + j];
        const bool in = id >= 0 && id < V;
        tid[j] = in ? id + phase : -1;
        tp[j] = in ? a.teacher[row * a.k + j] : -INFINITY;
        tm = fmaxf(tm, tp[j]);
    }
    auto join_cta = [&](float v, auto f, int slot) {
        v = reduce_warp(v, f);
        if ((threadIdx.x & 31) == 0) sh[slot][threadIdx.x >> 5] = v;
        __syncthreads();
        v = sh[slot][0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) v = f(v, sh[slot][i]);
        return v;
    };
    bool taught = false;
    float logtz = 0.f, inv = 0.f;
    if (k) {
        tm = join_cta(tm, Max(), 4);
        taught = tm != -INFINITY;                   // without an entry that has any weight the term is nothing
        float tz = 0.f;
        for (int j = threadIdx.x; j < k; j += THREADS) tz += expf((tp[j] - tm) * itau);
        tz = join_cta(tz, Add(), 5);
        logtz = logf(tz); inv = 1.f / tz;
    }
    // the row's maximum
    Terms t{-INFINITY, 0.f, HARD ? 1.f - a.weight : 0.f, 0.f, 0.f, a.scale};
    auto scan = [&](int q) {
        for (int c = q * part + threadIdx.x; c < min(n, (q + 1) * part); c += THREADS) {
            float v[E];
            unpack(chunks[c], v);
#pragma unroll
            for (int i = 0; i < E; ++i) t.m = fmaxf(t.m, v[i]);
        }
    };
    copies_arrived<3>(); scan(0);
    copies_arrived<2>(); scan(1);
    copies_arrived<1>(); scan(2);
    copies_arrived<0>(); scan(3);
    t.m = join(t.m, Max(), 0);
    // its sums
    float zt = 0.f, z1 = 0.f;
#pragma unroll 2
    for (int c = threadIdx.x; c < n; c += THREADS) {
        float v[E], st_ = 0.f, s1 = 0.f;
        unpack(chunks[c], v);
#pragma unroll
        for (int i = 0; i < E; ++i) { float et, e1; exps(v[i] - t.m, et, e1); st_ += et; s1 += e1; }
        zt += st_; z1 += s1;
    }
    zt = join(zt, Add(), 1);
    if (HARD) z1 = join(z1, Add(), 2);
    float loss = 0.f;
    if (taught) {
        const float logz = logf(zt);
        for (int j = threadIdx.x; j < k; j += THREADS) {
            const float d = (tp[j] - tm) * itau, p = expf(d) * inv;
            tp[j] = p;
            const int at = tid[j] - first * E;
            if (tid[j] < 0 || at < 0 || at >= n * E) { tid[j] = -1; continue; }     // not this CTA's
            tid[j] = at;
            ts[j] = ld(xs + at);
            if (p != 0.f) loss += p * ((d - logtz) - ((ts[j] - t.m) * itau - logz));
        }
        loss *= a.weight * a.tau * a.tau;
    }
    const int hit = HARD ? label + phase - first * E : -1;                   // the label's place
    const bool own = hit >= 0 && hit < n * E;
    if (HARD && own && threadIdx.x == 0) loss += t.c1 * (logf(z1) - (ld(xs + hit) - t.m));
    loss = join(loss, Add(), 3);
    if (rank == 0 && threadIdx.x == 0) a.loss[row] = loss;
    if (!g) return;
    t.ct = taught ? a.weight * a.tau : 0.f; t.it = 1.f / zt; t.i1 = HARD ? 1.f / z1 : 0.f;
    // the gradient without label and entries
    {
        const float A = t.scale * t.ct * t.it, B = t.scale * t.c1 * t.i1;
        const bool vec = (uintptr_t)(g - phase) % (E * sizeof(TO)) == 0;     // the chunks of g start where those of x do
#pragma unroll 2
        for (int c = threadIdx.x; c < n; c += THREADS) {
            float v[E];
            unpack(chunks[c], v);
#pragma unroll
            for (int i = 0; i < E; ++i) { float et, e1; exps(v[i] - t.m, et, e1); v[i] = HARD ? fmaf(A, et, B * e1) : A * et; }
            const long at = (long)(first + c) * E - phase;
            if (vec && inside(c)) put(g + at, v);
            else
#pragma unroll
                for (int i = 0; i < E; ++i) if (at + i >= 0 && at + i < V) st(g + at + i, v[i]);
        }
    }
    // those, over it
    const long base = (long)first * E - phase;
    auto fix = [&](int at, float s, float p) { float et, e1; exps(s - t.m, et, e1); st(g + base + at, t.at(et, e1, p, HARD && at == hit)); };
    const float hit_s = own ? ld(xs + hit) : 0.f;
    __syncthreads();
    if (own && threadIdx.x == 0) fix(hit, hit_s, 0.f);
    if (!taught) return;
    // Does an id occur twice?  Every entry writes its number to its place of the row, which is not needed any more, and looks which one stayed.
    for (int j = threadIdx.x; j < k; j += THREADS) if (tid[j] >= 0) ((unsigned short*)dyn)[tid[j] * (sizeof(TI) / 2)] = (unsigned short)j;
    __syncthreads();
    int twice = 0;
    for (int j = threadIdx.x; j < k; j += THREADS) if (tid[j] >= 0) twice |= ((unsigned short*)dyn)[tid[j] * (sizeof(TI) / 2)] != j;
    if (!__syncthreads_or(twice)) {
        for (int j = threadIdx.x; j < k; j += THREADS) if (tid[j] >= 0) fix(tid[j], ts[j], tp[j]);
        return;
    }
    for (int j = threadIdx.x; j < k; j += THREADS) {
        if (tid[j] < 0) continue;
        float p = 0.f;                              // an id that occurs more than once is its first entry's
        bool first_ = true;
        for (int i = 0; i < k; ++i) if (tid[i] == tid[j]) { if (i < j) first_ = false; p += tp[i]; }
        if (first_) fix(tid[j], ts[j], p);
    }
}

template <typename TI, typename TO, int SQ, bool HARD>
cudaError_t launch(const DistillArgs& a, cudaStream_t s) {
    if (a.V <= WARP_VOCAB && a.k <= WARP_TOP)
        return klaunch(distill_warp_k<TI, TO, SQ, HARD>, (unsigned)((a.M + WARPS - 1) / WARPS), THREADS, 0, s, a);
    // A CTA's share of a row: at most 64 KB, so that three fit on an SM and one copies while others compute; smaller where there are too few rows for the
    // SMs, down to 16 KB
    constexpr int E = Chunk<TI>::E;
    const long chunks = (a.V + E - 1) / E + 1;      // with one more for a row that starts inside a chunk
    int R = 1;
    while (R < MAX_CLUSTER && chunks > 4096l * R) R *= 2;
    while (R < MAX_CLUSTER && a.M * R < 148 && chunks > 1024l * R) R *= 2;
    const int share = (int)((chunks + R - 1) / R);
    const size_t smem = (size_t)share * 16 + (size_t)a.k * 12;
    constexpr int most = (int)((DISTILL_MAX_VOCAB / E + 1 + MAX_CLUSTER - 1) / MAX_CLUSTER) * 16 + DISTILL_MAX_TOP * 12;
    static_assert(most <= 200 * 1024 && most >= 4096 * 16 + DISTILL_MAX_TOP * 12, "shares fit");
    if (R > 1) {
        static OncePerDevice once;
        const cudaError_t e = allow_smem(once, (const void*)distill_row_k<TI, TO, SQ, HARD, true>, most);
        if (e != cudaSuccess) return e;
        return klaunch_cluster(distill_row_k<TI, TO, SQ, HARD, true>, (unsigned)(a.M * R), THREADS, smem, s, R, a, R, share);
    }
    static OncePerDevice once;
    const cudaError_t e = allow_smem(once, (const void*)distill_row_k<TI, TO, SQ, HARD, false>, most);
    if (e != cudaSuccess) return e;
    return klaunch(distill_row_k<TI, TO, SQ, HARD, false>, (unsigned)a.M, THREADS, smem, s, a, 1, share);
}
template <typename TI, typename TO>
cudaError_t pick(const DistillArgs& a, cudaStream_t s) {
    if (!(a.weight < 1.f)) return launch<TI, TO, -1, false>(a, s);
    return a.tau == 1.f ? launch<TI, TO, 0, true>(a, s) : a.tau == 2.f ? launch<TI, TO, 1, true>(a, s) : a.tau == 4.f ? launch<TI, TO, 2, true>(a, s)
           : a.tau == 8.f ? launch<TI, TO, 3, true>(a, s) : launch<TI, TO, -1, true>(a, s);
}

}  // namespace

cudaError_t distill(int dti, int dtg, const DistillArgs& a, cudaStream_t s) {
    if (a.M == 0) return cudaSuccess;
    Scope sc(KC_DISTILL, 10.0 * a.M * a.V, (double)a.M * a.V * ((dti ? 2 : 4) + (a.grad ? (dtg ? 2 : 4) : 0)), s);
    if (dti) return pick<bf16, bf16>(a, s);
    return dtg ? pick<float, bf16>(a, s) : pick<float, float>(a, s);
}

}  // namespace fdg
