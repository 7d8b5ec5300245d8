// Loss that distils a teacher's top logits, with the gradient for the student's logits.  Per row, with p = softmax(teacher / tau) over the row's
// entries, q = softmax(s / tau) and q1 = softmax(s) over the vocabulary:
//   loss = w tau^2 sum_j p_j (log p_j - log q[id_j]) + (1 - w) (-log q1[label])
//   grad_v = scale (w tau (q_v - sum of the p_j with id_j = v) + (1 - w) (q1_v - [v = label]))
// The logits are read once and the gradient is written once, which is the bound (HBM): a row stays in shared memory between its maximum, its sums and its
// gradient, cut over a cluster where one CTA's share would keep others from its SM.  The exponentials come close to being a second bound: the special-function
// unit makes 16 a cycle and SM, and an element needs one for either temperature in either pass.  Where tau is 1, 2 or 4, exp(d) is a power of exp(d / tau).
#include "seqops.h"
#include "launch.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

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
    // two at once, through the packed fp32 instructions
    __device__ __forceinline__ void operator()(float2 d, float2& et, float2& e1) const {
        const float2 x = __fmul2_rn(d, make_float2(c, c));
        et = make_float2(exp2_(x.x), exp2_(x.y));
        if (!HARD) { e1 = make_float2(0.f, 0.f); return; }
        if (SQ < 0) {
            const float2 z = __fmul2_rn(d, make_float2(LOG2E, LOG2E));
            e1 = make_float2(exp2_(z.x), exp2_(z.y));
        } else {
            e1 = et;
#pragma unroll
            for (int i = 0; i < SQ; ++i) e1 = __fmul2_rn(e1, e1);
        }
    }
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

// ---- a warp per row: small vocabularies, where the row comes out of L1 in the later passes.  Its time grows with the vocabulary, a CTA's with its rows (444 CTAs are there at once, a row
// takes 3.4 us).  bf16, warp and CTA: 200 rows of 512 6.3 and 6.3 us, of 1000 10.3 and 6.3; 1776 rows of 1000 12.4 and 16.5, of 2000 16.5 and 18.5, of 4000 39 and 21; 8192 rows of 2000 46 and 65.
constexpr int WARP_TOP = 128;
bool warp_per_row(long M, long V, int k) { return k <= WARP_TOP && (V <= 512 || (V <= 2048 && M * 512 >= 444 * V)); }
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
        tm = fmaxf(tm, tp[j] != tp[j] ? INFINITY : tp[j]);       // (a NaN is not taken for an entry left out)
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
    if (!HARD && !taught) {                         // neither term: zeros, whatever the logits are (0 times a sum of NaN would be NaN)
        for (int v = lane; v < V; v += 32) st(g + v, 0.f);
        return;
    }
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
__device__ __forceinline__ void unpack(const uint4& r, float2 (&x)[2]) {
    x[0] = make_float2(__uint_as_float(r.x), __uint_as_float(r.y)); x[1] = make_float2(__uint_as_float(r.z), __uint_as_float(r.w));
}
__device__ __forceinline__ void unpack(const uint4& r, float2 (&x)[4]) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ unsigned pair(float2 a) { const __nv_bfloat162 v = __float22bfloat162_rn(a); return *(const unsigned*)&v; }
__device__ __forceinline__ void put(float* p, const float2 (&x)[2]) { *(float4*)p = make_float4(x[0].x, x[0].y, x[1].x, x[1].y); }
__device__ __forceinline__ void put(bf16* p, const float2 (&x)[2]) { *(uint2*)p = make_uint2(pair(x[0]), pair(x[1])); }
__device__ __forceinline__ void put(bf16* p, const float2 (&x)[4]) { *(uint4*)p = make_uint4(pair(x[0]), pair(x[1]), pair(x[2]), pair(x[3])); }
// the largest values so far: of a chunk's words, and both halves' in the end (a NaN comes back by way of the sums)
struct Top {
    float m = -INFINITY;
    __nv_bfloat162 m2 = __float2bfloat162_rn(-INFINITY);
    __device__ __forceinline__ void add(const uint4& r, float) {
        m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(r.x), __uint_as_float(r.y))), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
    }
    __device__ __forceinline__ void add(const uint4& r, bf16) {
        const __nv_bfloat162* const v = (const __nv_bfloat162*)&r;
        m2 = __hmax2(__hmax2(m2, __hmax2(v[0], v[1])), __hmax2(v[2], v[3]));
    }
    __device__ __forceinline__ float value() const { return fmaxf(m, fmaxf(__low2float(m2), __high2float(m2))); }
};
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void copy16(void* smem, const void* g) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(smem)), "l"(g) : "memory");
}
template <int LEFT> __device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

__device__ __forceinline__ void copy4(void* smem, const void* g) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((unsigned)__cvta_generic_to_shared(smem)), "l"(g) : "memory");
}

// A row is cut into chunks of 16 aligned bytes, the first and the last one partly outside the row (there: -infinity).  A thread copies, and in every pass
// handles, the chunks threadIdx.x, + THREADS, ... of its CTA's share, so that it can have the next row's chunk copied to where it has just read this one's for the last
// time: a CTA (or cluster) goes through the rows row0, + step, ... with the next row on its way while the gradient of this one is written.
template <typename TI, typename TO, int SQ, bool HARD, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 3) distill_row_k(DistillArgs a, int ranks, int share) {
    constexpr int E = Chunk<TI>::E;
    extern __shared__ __align__(16) char dyn[];
    uint4* const chunks = (uint4*)dyn;
    TI* const xs = (TI*)dyn;                        // the element of the row at chunk * E + i
    const int k = a.weight > 0.f ? a.k : 0;
    float* const tp = (float*)(chunks + share);     // p of the entries, 0 where an entry is left out
    float* const ts = tp + k;                       // the student's logits there
    int* const tid = (int*)(ts + k);                // their places in the CTA's chunks, -1: left out, or not this CTA's
    int* const raw_ids = tid + k;                   // the entries as they arrive, for this row and the next
    float* const raw_t = (float*)(raw_ids + 2 * k);
    unsigned* const seen = (unsigned*)(raw_t + 2 * k);       // a bit per place
    __shared__ float sh[3][3][WARPS];               // of the warps, for every join
    __shared__ float joined[2][3][MAX_CLUSTER];     // of the CTAs
    __shared__ float lost[MAX_CLUSTER];
    const int R = CLUSTER ? ranks : 1, rank = CLUSTER ? (int)(blockIdx.x % R) : 0, V = (int)a.V;
    const long step = gridDim.x / R;
    if (CLUSTER) cluster_arrive();                  // waited for before anyone writes to another CTA's shared memory
    bool started = !CLUSTER;
    const int first = rank * share;                 // this CTA's chunks of every row

    // of a row: its logits, the place of its first element in its first chunk, how many of the chunks are this CTA's, and which of these lie in the row altogether
    struct Row { const TI* x; int phase, n, lo, whole; };
    auto row_of = [&](long r) {
        Row q;
        q.x = (const TI*)a.logits + r * a.logits_stride;
        q.phase = (int)((uintptr_t)q.x / sizeof(TI) % E);
        q.n = max(0, min(share, (V + q.phase + E - 1) / E - first));
        q.lo = first == 0 && q.phase ? 1 : 0;
        q.whole = max(0, min(q.n, (V + q.phase) / E - first) - q.lo);
        return q;
    };
    const auto inside = [&](const Row& q, int c) { return (unsigned)(c - q.lo) < (unsigned)q.whole; };
    auto chunk_of = [&](const Row& q, int c) { return (const char*)(q.x + ((long)first * E - q.phase)) + (long)c * 16; };
    auto fetch = [&](const Row& q, int c, const char* from) {
        if (inside(q, c)) copy16(chunks + c, from);
        else {
            const int v = (first + c) * E - q.phase;
            for (int i = 0; i < E; ++i) {
                if (v + i >= 0 && v + i < V) xs[c * E + i] = q.x[v + i];
                else st(xs + c * E + i, -INFINITY);
            }
        }
    };
    auto fetch_entries = [&](long r, int buf) {
        for (int j = threadIdx.x; j < k; j += THREADS) { copy4(raw_ids + buf * k + j, a.ids + r * k + j); copy4(raw_t + buf * k + j, a.teacher + r * k + j); }
    };
    // NV values each over the CTA, the same in every thread
    auto join_cta = [&](auto& v, auto f, int slot) {
        constexpr int NV = sizeof(v) / sizeof(float);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            v[i] = reduce_warp(v[i], f);
            if ((threadIdx.x & 31) == 0) sh[slot][i][threadIdx.x >> 5] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            v[i] = sh[slot][i][threadIdx.x % WARPS];
#pragma unroll
            for (int d = WARPS / 2; d; d >>= 1) v[i] = f(v[i], __shfl_xor_sync(~0u, v[i], d));
        }
    };
    // and over the cluster
    auto join = [&](auto& v, auto f, int slot) {
        constexpr int NV = sizeof(v) / sizeof(float);
        join_cta(v, f, slot);
        if (!CLUSTER) return;
        cg::cluster_group cl = cg::this_cluster();
        if (!started) { cluster_wait(); started = true; }
        if (threadIdx.x < R)
#pragma unroll
            for (int i = 0; i < NV; ++i) *cl.map_shared_rank(&joined[slot][i][rank], threadIdx.x) = v[i];
        cluster_arrive();
        cluster_wait();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            v[i] = joined[slot][i][0];
            for (int r = 1; r < R; ++r) v[i] = f(v[i], joined[slot][i][r]);
        }
    };
    const float itau = 1.f / a.tau;
    const Exps<SQ, HARD> exps{itau * LOG2E};
    long row = blockIdx.x / R;
    Row q = row_of(row);
    for (int c = threadIdx.x; c < q.n; c += THREADS) fetch(q, c, chunk_of(q, c));
    fetch_entries(row, 0);
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (k) for (int i = threadIdx.x; i < (share * E + 31) / 32; i += THREADS) seen[i] = 0;       // (a barrier follows before it is used)
    int label = a.labels ? a.labels[row] : 0;
    for (int buf = 0; row < a.M; row += step, buf ^= 1) {
        const bool more = row + step < a.M;
        const Row next = more ? row_of(row + step) : Row{nullptr, 0, 0};
        const int next_label = more && a.labels ? a.labels[row + step] : 0;
        const bool counts = label >= 0 && label < V;
        TO* const g = a.grad ? (TO*)a.grad + row * a.grad_stride : nullptr;
        const int n = q.n;
        Terms t{-INFINITY, 0.f, HARD ? 1.f - a.weight : 0.f, 0.f, 0.f, a.scale};
        bool taught = false;
        float loss = 0.f;
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        const int hit = HARD && counts ? label + q.phase - first * E : -1;       // the label's place
        const bool own = hit >= 0 && hit < n * E;
        float hit_s = 0.f;
        if (counts) {
            // the row's maximum, the teacher's
            float most[2] = {-INFINITY, -INFINITY};
            for (int j = threadIdx.x; j < k; j += THREADS) {
                const int id = raw_ids[buf * k + j], at = id + q.phase - first * E;
                const bool in = id >= 0 && id < V;
                tid[j] = in && at >= 0 && at < n * E ? at : -1;
                tp[j] = in ? raw_t[buf * k + j] : -INFINITY;
                most[1] = fmaxf(most[1], tp[j] != tp[j] ? INFINITY : tp[j]);     // (a NaN is not taken for an entry left out)
            }
            Top top;
#pragma unroll 4
            for (int c = threadIdx.x; c < n; c += THREADS) top.add(chunks[c], TI());
            most[0] = top.value();
            join(most, Max(), 0);                   // (its barrier: the whole row is there for everyone)
            t.m = most[0];
            const float tm = most[1];
            taught = tm != -INFINITY;               // without an entry that has any weight the term is nothing
            const float2 minus = make_float2(-t.m, -t.m);
            // sums: at the student's temperatures, of the teacher's (every CTA those entries that are its own)
            float total[3] = {0.f, 0.f, 0.f};
            if (taught) for (int j = threadIdx.x; j < k; j += THREADS) if (tid[j] >= 0) total[2] += expf((tp[j] - tm) * itau);
            float2 sum_t = make_float2(0.f, 0.f), sum_1 = sum_t;
#pragma unroll 2
            for (int c = threadIdx.x; c < n; c += THREADS) {
                float2 v[E / 2], st_ = make_float2(0.f, 0.f), s1 = st_;
                unpack(chunks[c], v);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) { float2 et, e1; exps(__fadd2_rn(v[i], minus), et, e1); st_ = __fadd2_rn(st_, et); s1 = __fadd2_rn(s1, e1); }
                sum_t = __fadd2_rn(sum_t, st_); if (HARD) sum_1 = __fadd2_rn(sum_1, s1);
            }
            total[0] = sum_t.x + sum_t.y; total[1] = sum_1.x + sum_1.y;
            join(total, Add(), 1);
            const float zt = total[0], z1 = total[1], tz = total[2];
            if (taught) {
                const float logz = logf(zt), logtz = logf(tz), inv = 1.f / tz;
                for (int j = threadIdx.x; j < k; j += THREADS) {
                    const float d = (tp[j] - tm) * itau, p = expf(d) * inv;
                    tp[j] = p;
                    if (tid[j] < 0) continue;
                    ts[j] = ld(xs + tid[j]);
                    if (p != 0.f) loss += p * ((d - logtz) - ((ts[j] - t.m) * itau - logz));
                }
                loss *= a.weight * a.tau * a.tau;
            }
            if (own) hit_s = ld(xs + hit);
            if (HARD && own && threadIdx.x == 0) loss += t.c1 * (logf(z1) - (hit_s - t.m));
            float part[1] = {loss};
            join_cta(part, Add(), 2);               // (its barrier: what is needed of the row beside its chunks has been read)
            loss = part[0];
            if (CLUSTER) {                          // waited for at the row's end
                if (threadIdx.x == 0) *cg::this_cluster().map_shared_rank(&lost[rank], 0) = loss;
                cluster_arrive();
            }
            t.ct = taught ? a.weight * a.tau : 0.f; t.it = 1.f / zt; t.i1 = HARD ? 1.f / z1 : 0.f;
        }
        if (!CLUSTER && threadIdx.x == 0) a.loss[row] = loss;
        // the gradient without label and entries; the next row takes the place of this one
        const char* from = more ? chunk_of(next, threadIdx.x) : nullptr;
        const bool any = counts && (HARD || taught);         // a row with neither term has zeros, whatever its logits are (0 times a sum of NaN would be NaN)
        if (g && any) {
            const float A = t.scale * t.ct * t.it, B = t.scale * t.c1 * t.i1;
            const float2 minus = make_float2(-t.m, -t.m), A2 = make_float2(A, A), B2 = make_float2(B, B);
            const bool vec = (uintptr_t)(g - q.phase) % (E * sizeof(TO)) == 0;   // the chunks of g start where those of x do
            TO* to = g + ((long)first * E - q.phase) + (long)threadIdx.x * E;
#pragma unroll 2
            for (int c = threadIdx.x; c < max(n, next.n); c += THREADS, from += THREADS * 16, to += THREADS * E) {
                uint4 r{};
                if (c < n) r = chunks[c];
                if (c < next.n) fetch(next, c, from);
                if (c >= n) continue;
                float2 v[E / 2];
                unpack(r, v);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    float2 et, e1;
                    exps(__fadd2_rn(v[i], minus), et, e1);
                    v[i] = HARD ? __ffma2_rn(A2, et, __fmul2_rn(B2, e1)) : __fmul2_rn(A2, et);
                }
                if (vec && inside(q, c)) put(to, v);
                else {
                    const int at = (first + c) * E - q.phase;
#pragma unroll
                    for (int i = 0; i < E; ++i) if (at + i >= 0 && at + i < V) st(to + i, i & 1 ? v[i / 2].y : v[i / 2].x);
                }
            }
        } else {
            for (int c = threadIdx.x; c < next.n; c += THREADS, from += THREADS * 16) fetch(next, c, from);
            if (g)
                for (int v = max(0, first * E - q.phase) + threadIdx.x; v < min(V, (first + n) * E - q.phase); v += THREADS) st(g + v, 0.f);
        }
        if (more) fetch_entries(row + step, buf ^ 1);
        asm volatile("cp.async.commit_group;" ::: "memory");
        // those, over it
        if (g && any) {
            const long base = (long)first * E - q.phase;
            auto fix = [&](int at, float s, float p) { float et, e1; exps(s - t.m, et, e1); st(g + base + at, t.at(et, e1, p, HARD && at == hit)); };
            __syncthreads();
            if (own && threadIdx.x == 0) fix(hit, hit_s, 0.f);
            if (taught) {
                int twice = 0;                      // does an id occur twice?
                for (int j = threadIdx.x; j < k; j += THREADS)
                    if (tid[j] >= 0) { const unsigned bit = 1u << (tid[j] & 31); twice |= (atomicOr(seen + (tid[j] >> 5), bit) & bit) != 0; }
                if (!__syncthreads_or(twice)) {
                    for (int j = threadIdx.x; j < k; j += THREADS) if (tid[j] >= 0) fix(tid[j], ts[j], tp[j]);
                } else {
                    for (int j = threadIdx.x; j < k; j += THREADS) {
                        if (tid[j] < 0) continue;
                        float p = 0.f;              // an id that occurs more than once is its first entry's
                        bool one = true;
                        for (int i = 0; i < k; ++i) if (tid[i] == tid[j]) { if (i < j) one = false; p += tp[i]; }
                        if (one) fix(tid[j], ts[j], p);
                    }
                    __syncthreads();                // nobody reads the others' entries any more
                }
                for (int j = threadIdx.x; j < k; j += THREADS) if (tid[j] >= 0) seen[tid[j] >> 5] = 0;
            }
        }
        if (CLUSTER) {
            if (counts) cluster_wait();
            if (rank == 0 && threadIdx.x == 0) {
                if (counts) for (int r = 1; r < R; ++r) loss += lost[r];
                a.loss[row] = loss;
            }
        }
        q = next;
        label = next_label;
    }
    if (CLUSTER && !started) cluster_wait();
}

// How many clusters of R CTAs the device holds at once (asked for once per size: clusters need their SMs in one part of the device, so it is not SMs x CTAs / R).
struct Resident {
    std::atomic<uint64_t> last{0};                  // device, size and R of the last question, and its answer
    int ask(const void* kernel, int R, int smem) {
        int dev = 0;
        cudaGetDevice(&dev);
        const uint64_t key = (uint64_t)(dev + 1) << 52 | (uint64_t)R << 44 | (uint64_t)smem << 16, known = last.load(std::memory_order_relaxed);
        if ((known & ~0xffffull) == key) return (int)(known & 0xffff);
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = R; at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.gridDim = R * 148; cfg.blockDim = THREADS; cfg.dynamicSmemBytes = smem; cfg.attrs = at; cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
        n = n < 1 ? 1 : n > 0xffff ? 0xffff : n;
        last.store(key | (uint64_t)n, std::memory_order_relaxed);
        return n;
    }
};

template <typename TI, typename TO, int SQ, bool HARD>
cudaError_t launch(const DistillArgs& a, cudaStream_t s) {
    if (warp_per_row(a.M, a.V, a.k))
        return klaunch(distill_warp_k<TI, TO, SQ, HARD>, (unsigned)((a.M + WARPS - 1) / WARPS), THREADS, 0, s, a);
    // A CTA's share of a row: up to 100 KB, so that two fit on an SM (three up to 64 KB) and one copies while others compute; smaller where there are too few rows for
    // the SMs, down to 16 KB (8 rows of 32000 bf16 8.3 us, 10.4 in one share each).  1500 rows of 100003 fp32 logits: 271 us in four shares, 327 in eight (more time in the cluster's barriers), 295 in four with 512 threads
    // a CTA (more time in the joins).  With eight CTAs a row at most, shares grow beyond that from 204800 fp32 logits on, to 131 KB and the entries at 262144: one CTA to an SM, and nothing
    // copies while it computes (600 rows of 262144 fp32 455 us for 192 of bytes, 700 of 204800 302 for 175).
    constexpr int E = Chunk<TI>::E;
    const long chunks = (a.V + E - 1) / E + 1;      // with one more for a row that starts inside a chunk
    int R = 1;
    while (R < MAX_CLUSTER && chunks > 6400l * R) R *= 2;
    while (R < MAX_CLUSTER && a.M * R < 148 && chunks > 1024l * R) R *= 2;
    const int share = (int)((chunks + R - 1) / R);
    auto bytes = [](int share, int k) { return share * 16 + k * 28 + (share * E + 31) / 32 * 4; };
    const int smem = bytes(share, a.weight > 0.f ? a.k : 0), most = bytes(std::max(6400, (int)((DISTILL_MAX_VOCAB / E + 1 + MAX_CLUSTER - 1) / MAX_CLUSTER)), DISTILL_MAX_TOP);
    if (R > 1) {
        static OncePerDevice once;
        static Resident resident;
        const auto kernel = distill_row_k<TI, TO, SQ, HARD, true>;
        const cudaError_t e = allow_smem(once, (const void*)kernel, most);
        if (e != cudaSuccess) return e;
        const long rows = std::min<long>(a.M, resident.ask((const void*)kernel, R, smem));       // at once
        return klaunch_cluster(kernel, (unsigned)(rows * R), THREADS, (size_t)smem, s, R, a, R, share);
    }
    // Three CTAs an SM, whatever fits: shares over 64 KB, of which two do, leave the third's rows to a short wave of their own (bf16, bytes' time and time: 4096 rows of 32000 80 and 111 us,
    // 3200 of 40000 78 and 150, 2600 of 50257 80 and 136; fp32 3200 of 20000 78 and 121).
    static OncePerDevice once;
    const auto kernel = distill_row_k<TI, TO, SQ, HARD, false>;
    const cudaError_t e = allow_smem(once, (const void*)kernel, most);
    return e != cudaSuccess ? e : klaunch(kernel, (unsigned)std::min<long>(a.M, 148 * 3), THREADS, (size_t)smem, s, a, 1, share);
}
template <typename TI, typename TO>
cudaError_t pick(const DistillArgs& a, cudaStream_t s) {
    if (!(a.weight < 1.f)) return launch<TI, TO, -1, false>(a, s);
    return a.tau == 1.f ? launch<TI, TO, 0, true>(a, s) : a.tau == 2.f ? launch<TI, TO, 1, true>(a, s) : a.tau == 4.f ? launch<TI, TO, 2, true>(a, s)
           : launch<TI, TO, -1, true>(a, s);
}

}  // namespace

cudaError_t distill(int dti, int dtg, const DistillArgs& a, cudaStream_t s) {
    if (a.M == 0) return cudaSuccess;
    Scope sc(KC_DISTILL, 10.0 * a.M * a.V, (double)a.M * a.V * ((dti ? 2 : 4) + (a.grad ? (dtg ? 2 : 4) : 0)), s);
    if (dti) return pick<bf16, bf16>(a, s);
    return dtg ? pick<float, bf16>(a, s) : pick<float, float>(a, s);
}

}  // namespace fdg
