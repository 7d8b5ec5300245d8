// Gated linear recurrence, per sequence and channel:  a = sigmoid(z),  h_t = a_t h_{t-1} + (1 - a_t) v_t,  y_t = h_t.
// Backward, with d_t = dy_t + a_{t+1} d_{t+1}:  dv_t = (1 - a_t) d_t,  dz_t = a_t (1 - a_t) d_t (h_{t-1} - v_t),  dh_0 = a_1 d_1.
//
// A step is the affine map h -> a h + u, u = (1 - a) v; maps compose: (A, H) then (A', H') is (A' A, A' H + H').  So a sequence is cut into pieces whose
// maps are found side by side and joined: a thread composes STEPS = 4 steps of four channels, a warp its threads by shuffles, the CTA its warps and, where
// a launch would otherwise be too small, a cluster its CTAs through distributed shared memory; then every thread runs its steps again from the state in front of
// them.  The joins are a fixed tree, so equal inputs give equal bits.  Backwards the same with g_t = a_t d_t, the map g -> a (g + dy).
//
// Bound: HBM (forward 3 values a step and channel, backward 5).  A CTA walks along its sequence with a ring of tiles that cp.async fills ahead; a thread
// reads only what it copied itself, so the ring needs no barrier.
// States are held in 32 bits.  The backward pass computes h again from the states that the forward pass leaves in front of every tile: y rounded to bf16 would
// put 2^-9 of h into dz, and the states are 2 / (tile's steps) of the bytes of y.
#include "seqops.h"
#include "launch.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cstdlib>

namespace fdg {
namespace {

namespace cg = cooperative_groups;
using bf16 = __nv_bfloat16;

constexpr int THREADS = 256;
constexpr int STEPS = 4;                // of a thread in a tile
constexpr int N = 4;                    // channels of a thread
constexpr int MAX_CLUSTER = 8;      // of slices up to 64 channels; wider ones have no clusters

// CX threads lie along the channels, the others along the steps.
template <int CX> struct Geo {
    static constexpr int TG = THREADS / CX, CH = CX * N, TILE = TG * STEPS;
    static constexpr int TEAM = CX < 32 ? 32 : CX, TEAMS = THREADS / TEAM;      // a team joins its threads by shuffles (or is one step group)
    static constexpr int RANKS = CX > 16 ? 1 : MAX_CLUSTER;
};

// Values go in pairs through the packed fp32 instructions: the kernels issue too much, not too little, to keep up with HBM.
struct Four { float2 p[2]; };
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }

// a = sigmoid(z) and q = 1 - a, each to a few units of its own last place: e = 2^min(-z log2 e, 100), a = 1 / (1 + e), q = e a.  Behind the bound a is 2^-100
// instead of less and q is 1; NaN stays.
__device__ __forceinline__ void gate(float2 z, float2& a, float2& q) {
    const float2 t = mul(z, both(-1.4426950408889634f));
    float2 e;
    asm("min.NaN.f32 %0, %1, 0f42C80000;" : "=f"(e.x) : "f"(t.x));
    asm("min.NaN.f32 %0, %1, 0f42C80000;" : "=f"(e.y) : "f"(t.y));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    const float2 d = __fadd2_rn(e, both(1.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.x) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.y) : "f"(d.y));
    q = mul(e, a);
}

template <typename T> struct Raw;                    // N values as they are stored
template <> struct Raw<float> { using V = float4; };
template <> struct Raw<bf16> { using V = uint2; };
__device__ __forceinline__ Four unpack(const float4& r) { return {make_float2(r.x, r.y), make_float2(r.z, r.w)}; }
__device__ __forceinline__ Four unpack(const uint2& r) {
    return {make_float2(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u)), make_float2(__uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u))};
}
__device__ __forceinline__ void pack(const Four& x, float4& r) { r = make_float4(x.p[0].x, x.p[0].y, x.p[1].x, x.p[1].y); }
__device__ __forceinline__ void pack(const Four& x, uint2& r) {
    const __nv_bfloat162 lo = __float22bfloat162_rn(x.p[0]), hi = __float22bfloat162_rn(x.p[1]);
    r = make_uint2(*(const unsigned*)&lo, *(const unsigned*)&hi);
}
// a step that changes nothing: gate open (+infinity), value and dy zero
__device__ __forceinline__ void idle(float4* z, float4* x) { *z = make_float4(INFINITY, INFINITY, INFINITY, INFINITY); *x = make_float4(0.f, 0.f, 0.f, 0.f); }
__device__ __forceinline__ void idle(uint2* z, uint2* x) { *z = make_uint2(0x7f807f80u, 0x7f807f80u); *x = make_uint2(0u, 0u); }
__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

template <int BYTES> __device__ __forceinline__ void copy_async(void* smem, const void* g) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((unsigned)__cvta_generic_to_shared(smem)), "l"(g), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// ACC: elements that a copy moves at once, as the addresses allow: 4, 2 (bf16), 1.  A single bf16 is too little for cp.async.
template <typename T, int ACC> __device__ __forceinline__ void fetch(void* slot, const T* g, int left) {
    if constexpr (ACC * sizeof(T) >= 4) {
#pragma unroll
        for (int j = 0; j < N; j += ACC) if (ACC == N || j < left) copy_async<ACC * sizeof(T)>((T*)slot + j, g + j);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) if (j < left) ((T*)slot)[j] = g[j];
    }
}
template <typename T, int ACC> __device__ __forceinline__ void put(T* g, Four x, int left, bool accum) {
    if (accum) {
        if (0 < left) x.p[0].x += ld(g);
        if (1 < left) x.p[0].y += ld(g + 1);
        if (2 < left) x.p[1].x += ld(g + 2);
        if (3 < left) x.p[1].y += ld(g + 3);
    }
    if constexpr (ACC == N) {
        typename Raw<T>::V r;
        pack(x, r);
        *(typename Raw<T>::V*)g = r;
    } else if constexpr (ACC == 2) {
        *(__nv_bfloat162*)g = __float22bfloat162_rn(x.p[0]);
        if (left > 2) *(__nv_bfloat162*)(g + 2) = __float22bfloat162_rn(x.p[1]);
    } else {
        st(g, x.p[0].x);
        if (1 < left) st(g + 1, x.p[0].y);
        if (2 < left) st(g + 2, x.p[1].x);
        if (3 < left) st(g + 3, x.p[1].y);
    }
}
// steps of t0 .. t0 + STEPS - 1 that lie in front of `end`
__device__ __forceinline__ int steps_before(long end, long t0) {
    const long n = end - t0;
    return n <= 0 ? 0 : n < STEPS ? (int)n : STEPS;
}

template <typename T, int TENSORS> struct Ring {
    using V = typename Raw<T>::V;
    static constexpr int STAGES = sizeof(T) == 2 ? 3 : 2;
    static constexpr int STAGE = STEPS * TENSORS * THREADS;
    static constexpr int BYTES = STAGES * STAGE * (int)sizeof(V);
    V* mine;                                                     // this thread's first slot
    __device__ V* slot(int stage, int i, int tensor) const { return mine + stage * STAGE + (i * TENSORS + tensor) * THREADS; }
};

// the map (a1, h1), then (a, h), in place of (a, h)
__device__ __forceinline__ void after(float2 a1, float2 h1, float2& a, float2& h) { h = fma(a, h1, h); a = mul(a, a1); }
__device__ __forceinline__ float2 shfl_up(float2 v, int d) { return make_float2(__shfl_up_sync(~0u, v.x, d), __shfl_up_sync(~0u, v.y, d)); }
__device__ __forceinline__ float2 shfl_down(float2 v, int d) { return make_float2(__shfl_down_sync(~0u, v.x, d), __shfl_down_sync(~0u, v.y, d)); }
// Over the step groups of a warp: (A, H) becomes the map of the groups up to and with this one, (Ax, Hx) that of those before it; UP: in the order of
// the lanes, else against it.
template <int CX, bool UP> __device__ __forceinline__ void join(Four& A, Four& H, Four& Ax, Four& Hx) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < 2; ++j) { Ax.p[j] = both(1.f); Hx.p[j] = both(0.f); }
#pragma unroll
    for (int d = CX; d < 32; d *= 2)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float2 a = UP ? shfl_up(A.p[j], d) : shfl_down(A.p[j], d), h = UP ? shfl_up(H.p[j], d) : shfl_down(H.p[j], d);
            if (UP ? lane >= d : lane < 32 - d) {
                after(a, h, A.p[j], H.p[j]);
                if (d == CX) { Ax.p[j] = a; Hx.p[j] = h; } else after(a, h, Ax.p[j], Hx.p[j]);
            }
        }
}
// Maps of the teams, one {A, H} per channel.
__device__ __forceinline__ void store(float2* p, const Four& A, const Four& H) {
    *(float4*)p = make_float4(A.p[0].x, H.p[0].x, A.p[0].y, H.p[0].y);
    *(float4*)(p + 2) = make_float4(A.p[1].x, H.p[1].x, A.p[1].y, H.p[1].y);
}
// The value that stands in front of a warp, for the channels of its lanes, from values and maps per channel.  Up to 32 channels a lane takes one channel
// through the maps and the lanes exchange them; above, every lane takes its own four.
template <int CX> struct Lanes {
    static constexpr bool ONE = CX * N <= 32;
    static constexpr int M = ONE ? 1 : N;
    float v[M];
    static __device__ __forceinline__ int first() { return ONE ? (threadIdx.x & 31) % (CX * N) : threadIdx.x % CX * N; }
    __device__ __forceinline__ void set(const float* p) {
        if constexpr (ONE) v[0] = *p;
        else { const float4 r = *(const float4*)p; v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
    }
    __device__ __forceinline__ void through(const float2* p) {
        if constexpr (ONE) { const float2 m = *p; v[0] = fmaf(m.x, v[0], m.y); }
        else {
            const float4 m = *(const float4*)p, k = *(const float4*)(p + 2);
            v[0] = fmaf(m.x, v[0], m.y); v[1] = fmaf(m.z, v[1], m.w); v[2] = fmaf(k.x, v[2], k.y); v[3] = fmaf(k.z, v[3], k.w);
        }
    }
    __device__ __forceinline__ Four four() const {
        if constexpr (ONE) {
            const int l = threadIdx.x % CX * N;
            return {make_float2(__shfl_sync(~0u, v[0], l), __shfl_sync(~0u, v[0], l + 1)), make_float2(__shfl_sync(~0u, v[0], l + 2), __shfl_sync(~0u, v[0], l + 3))};
        } else return {make_float2(v[0], v[1]), make_float2(v[2], v[3])};
    }
};
// values of channels first .. of a row of C, zero behind its end
template <int CX> __device__ __forceinline__ void read(Lanes<CX>& l, const float* row, long first, long C) {
#pragma unroll
    for (int j = 0; j < Lanes<CX>::M; ++j) l.v[j] = row && first + j < C ? row[first + j] : 0.f;
}

// One barrier a tile: behind it a warp goes through the maps of the teams in front of it by itself, and the last steps' threads leave the state for the
// next tile, which the next tile's barrier orders.  What stands there is kept twice, by the round's parity.
template <typename T, int ACC, int CX>
__global__ void __launch_bounds__(THREADS, 3) recur_fwd_k(RecurArgs p, int R, int slices) {
    using G = Geo<CX>;
    using Rg = Ring<T, 2>;
    extern __shared__ __align__(16) char dyn[];
    const Rg ring{(typename Rg::V*)dyn + threadIdx.x};
    __shared__ __align__(16) float2 tot[2][G::TEAMS][G::CH];
    __shared__ __align__(16) float carried[2][G::CH];
    __shared__ __align__(16) float2 joined[2][G::RANKS][G::CH];
    const int rank = R > 1 ? (int)(blockIdx.x % R) : 0;
    const long group = blockIdx.x / R, b = group / slices;
    const long c0 = (group - b * slices) * G::CH;
    const int cx = threadIdx.x % CX, tg = threadIdx.x / CX, team = threadIdx.x / G::TEAM, lane = threadIdx.x & 31;
    const long c = c0 + cx * N;
    const int left = (int)min((long)N, p.C - c);                 // channels of this thread that exist
    const long len = p.lengths ? min((long)max(p.lengths[b], 0), p.T) : p.T;
    const long tiles = (p.T + G::TILE - 1) / G::TILE, rounds = (tiles + R - 1) / R, stride = (long)R * G::TILE;
    long t0 = (long)rank * G::TILE + tg * STEPS, tf = t0;        // this thread's first step: of the round, of the next tile to fetch
    const T* zf = (const T*)p.z + b * p.z_b + c + t0 * p.z_t;
    const T* vf = (const T*)p.v + b * p.v_b + c + t0 * p.v_t;
    T* y = (T*)p.y + b * p.y_b + c + t0 * p.y_t;
    auto fetch_tile = [&](int stage) {
        const int n = left > 0 ? steps_before(len, tf) : 0;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < n) {
                fetch<T, ACC>(ring.slot(stage, i, 0), zf + i * p.z_t, left);
                fetch<T, ACC>(ring.slot(stage, i, 1), vf + i * p.v_t, left);
            } else idle(ring.slot(stage, i, 0), ring.slot(stage, i, 1));
        copies_issued();
        tf += stride; zf += stride * p.z_t; vf += stride * p.v_t;
    };
    for (int s = 0; s < Rg::STAGES - 1; ++s) fetch_tile(s);
    if (R > 1) cg::this_cluster().sync();                        // every CTA is there before anyone writes to its shared memory
    const int first = Lanes<CX>::first();
    Lanes<CX> carry;                                             // R > 1: the state in front of the round, in every warp
    read<CX>(carry, p.state ? p.state + b * p.C : nullptr, c0 + first, p.C);
    if (threadIdx.x < G::CH) carried[0][threadIdx.x] = p.state && c0 + threadIdx.x < p.C ? p.state[b * p.C + c0 + threadIdx.x] : 0.f;
    int stage = 0;
    for (long round = 0; round < rounds; ++round) {
        const int now = (int)(round & 1);
        fetch_tile(stage == 0 ? Rg::STAGES - 1 : stage - 1);
        copies_arrived<Rg::STAGES - 1>();
        // the map of this thread's steps
        Four a[STEPS], u[STEPS], A, H, Ax, Hx;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const Four z = unpack(*ring.slot(stage, i, 0)), v = unpack(*ring.slot(stage, i, 1));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float2 q;
                gate(z.p[j], a[i].p[j], q);
                u[i].p[j] = mul(q, v.p[j]);
                if (i == 0) { A.p[j] = a[0].p[j]; H.p[j] = u[0].p[j]; }
                else { H.p[j] = fma(a[i].p[j], H.p[j], u[i].p[j]); A.p[j] = mul(A.p[j], a[i].p[j]); }
            }
        }
        join<CX, true>(A, H, Ax, Hx);                            // of the threads in front of it in its team, and the team's
        if (CX >= 32 || lane >= 32 - CX) store(&tot[now][team][cx * N], A, H);
        __syncthreads();
        Lanes<CX> in;
        if (R > 1) {                                             // the CTA's map goes to every CTA of the cluster
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < G::CH) {
                float ta = 1.f, th = 0.f;
#pragma unroll
                for (int w = 0; w < G::TEAMS; ++w) { const float2 m = tot[now][w][threadIdx.x]; th = fmaf(m.x, th, m.y); ta *= m.x; }
                for (int r = 0; r < R; ++r) *cl.map_shared_rank(&joined[now][rank][threadIdx.x], r) = make_float2(ta, th);
            }
            cl.sync();
            for (int r = 0; r < R; ++r) {
                if (r == rank) in = carry;
                carry.through(&joined[now][r][first]);
            }
        } else in.set(&carried[now][first]);
        if (p.saved && threadIdx.x < G::TEAM && (!Lanes<CX>::ONE || lane < G::CH) && (Lanes<CX>::ONE || CX >= 32 || lane < CX)) {
            const long tile = round * R + rank;
#pragma unroll
            for (int j = 0; j < Lanes<CX>::M; ++j) if (tile < tiles && c0 + first + j < p.C) p.saved[(b * tiles + tile) * p.C + c0 + first + j] = in.v[j];
        }
        for (int w = 0; w < team; ++w) in.through(&tot[now][w][first]);
        Four h = in.four();
#pragma unroll
        for (int j = 0; j < 2; ++j) h.p[j] = fma(Ax.p[j], h.p[j], Hx.p[j]);
        const int n = left > 0 ? steps_before(len, t0) : 0;
        if (n == STEPS) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) h.p[j] = fma(a[i].p[j], h.p[j], u[i].p[j]);
                put<T, ACC>(y + i * p.y_t, h, left, false);
            }
        } else {
            const int out = left > 0 ? steps_before(p.T, t0) : 0;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) h.p[j] = fma(a[i].p[j], h.p[j], u[i].p[j]);
                if (i < out) put<T, ACC>(y + i * p.y_t, i < n ? h : Four{}, left, false);
            }
        }
        if (R == 1 && tg == G::TG - 1) *(float4*)&carried[now ^ 1][cx * N] = make_float4(h.p[0].x, h.p[0].y, h.p[1].x, h.p[1].y);
        t0 += stride; y += stride * p.y_t;
        stage = stage + 1 == Rg::STAGES ? 0 : stage + 1;
    }
    if (R > 1) cg::this_cluster().sync();                        // nobody leaves while others may write to its shared memory
    else { __syncthreads(); carry.set(&carried[rounds & 1][first]); }
    if (p.state_out && rank == 0 && threadIdx.x < G::TEAM) {
#pragma unroll
        for (int j = 0; j < Lanes<CX>::M; ++j) if (c0 + first + j < p.C) p.state_out[b * p.C + c0 + first + j] = carry.v[j];
    }
}

template <typename T, int ACC, int CX>
__global__ void __launch_bounds__(THREADS, 2) recur_bwd_k(RecurArgs p, int R, int slices) {
    using G = Geo<CX>;
    using Rg = Ring<T, 3>;
    extern __shared__ __align__(16) char dyn[];
    const Rg ring{(typename Rg::V*)dyn + threadIdx.x};
    __shared__ __align__(16) float2 tot_h[2][G::TEAMS][G::CH], tot_g[2][G::TEAMS][G::CH];
    __shared__ __align__(16) float carried[2][G::CH];
    __shared__ __align__(16) float2 joined[2][G::RANKS][G::CH];
    const int rank = R > 1 ? (int)(blockIdx.x % R) : 0;
    const long group = blockIdx.x / R, b = group / slices;
    const long c0 = (group - b * slices) * G::CH;
    const int cx = threadIdx.x % CX, tg = threadIdx.x / CX, team = threadIdx.x / G::TEAM, lane = threadIdx.x & 31;
    const long c = c0 + cx * N;
    const int left = (int)min((long)N, p.C - c);
    const long len = p.lengths ? min((long)max(p.lengths[b], 0), p.T) : p.T;
    const long tiles = (p.T + G::TILE - 1) / G::TILE, rounds = (tiles + R - 1) / R, stride = (long)R * G::TILE;
    // rounds go from the end of the sequence to its beginning
    long tile = (rounds - 1) * R + rank;
    long t0 = tile * G::TILE + tg * STEPS, tf = t0;
    const T* zf = (const T*)p.z + b * p.z_b + c + t0 * p.z_t;
    const T* vf = (const T*)p.v + b * p.v_b + c + t0 * p.v_t;
    const T* df = (const T*)p.dy + b * p.dy_b + c + t0 * p.dy_t;
    T* dz = (T*)p.dz + b * p.dz_b + c + t0 * p.dz_t;
    T* dv = (T*)p.dv + b * p.dv_b + c + t0 * p.dv_t;
    auto fetch_tile = [&](int stage) {
        const int n = left > 0 && tf >= 0 ? steps_before(len, tf) : 0;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < n) {
                fetch<T, ACC>(ring.slot(stage, i, 0), zf + i * p.z_t, left);
                fetch<T, ACC>(ring.slot(stage, i, 1), vf + i * p.v_t, left);
                fetch<T, ACC>(ring.slot(stage, i, 2), df + i * p.dy_t, left);
            } else {
                idle(ring.slot(stage, i, 0), ring.slot(stage, i, 1));
                *ring.slot(stage, i, 2) = *ring.slot(stage, i, 1);
            }
        copies_issued();
        tf -= stride; zf -= stride * p.z_t; vf -= stride * p.v_t; df -= stride * p.dy_t;
    };
    for (int s = 0; s < Rg::STAGES - 1; ++s) fetch_tile(s);
    if (R > 1) cg::this_cluster().sync();                        // every CTA is there before anyone writes to its shared memory
    const int first = Lanes<CX>::first();
    Lanes<CX> carry;
    read<CX>(carry, p.dstate_out ? p.dstate_out + b * p.C : nullptr, c0 + first, p.C);
    if (threadIdx.x < G::CH) carried[0][threadIdx.x] = p.dstate_out && c0 + threadIdx.x < p.C ? p.dstate_out[b * p.C + c0 + threadIdx.x] : 0.f;
    int stage = 0;
    for (long round = 0; round < rounds; ++round) {
        const int now = (int)(round & 1);
        fetch_tile(stage == 0 ? Rg::STAGES - 1 : stage - 1);
        Lanes<CX> in_h, in_g;
        read<CX>(in_h, tile < tiles ? p.saved + (b * tiles + tile) * p.C : nullptr, c0 + first, p.C);
        copies_arrived<Rg::STAGES - 1>();
        Four a[STEPS], q[STEPS], A, B, H, Q, Ax, Hx, Ay, Qy;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const Four z = unpack(*ring.slot(stage, i, 0)), v = unpack(*ring.slot(stage, i, 1)), d = unpack(*ring.slot(stage, i, 2));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                gate(z.p[j], a[i].p[j], q[i].p[j]);
                const float2 u = mul(q[i].p[j], v.p[j]);
                if (i == 0) { A.p[j] = a[0].p[j]; H.p[j] = u; Q.p[j] = mul(A.p[j], d.p[j]); }
                else {
                    H.p[j] = fma(a[i].p[j], H.p[j], u);
                    A.p[j] = mul(A.p[j], a[i].p[j]);
                    Q.p[j] = fma(A.p[j], d.p[j], Q.p[j]);        // what dy of this step is in front of the thread's first one
                }
            }
        }
        B = A;
        join<CX, true>(A, H, Ax, Hx);                            // of the threads in front (forward map)
        join<CX, false>(B, Q, Ay, Qy);                           // and behind (backward map)
        if (CX >= 32 || lane >= 32 - CX) store(&tot_h[now][team][cx * N], A, H);
        if (CX >= 32 || lane < CX) store(&tot_g[now][team][cx * N], B, Q);
        __syncthreads();
        if (R > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < G::CH) {
                float ta = 1.f, tq = 0.f;
#pragma unroll
                for (int w = G::TEAMS - 1; w >= 0; --w) { const float2 m = tot_g[now][w][threadIdx.x]; tq = fmaf(m.x, tq, m.y); ta *= m.x; }
                for (int r = 0; r < R; ++r) *cl.map_shared_rank(&joined[now][rank][threadIdx.x], r) = make_float2(ta, tq);
            }
            cl.sync();
            for (int r = R - 1; r >= 0; --r) {
                if (r == rank) in_g = carry;
                carry.through(&joined[now][r][first]);
            }
        } else in_g.set(&carried[now][first]);
        for (int w = 0; w < team; ++w) in_h.through(&tot_h[now][w][first]);
        for (int w = G::TEAMS - 1; w > team; --w) in_g.through(&tot_g[now][w][first]);
        Four g = in_g.four(), before[STEPS];
        before[0] = in_h.four();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            before[0].p[j] = fma(Ax.p[j], before[0].p[j], Hx.p[j]);
            g.p[j] = fma(Ay.p[j], g.p[j], Qy.p[j]);
        }
#pragma unroll
        for (int i = 0; i + 1 < STEPS; ++i) {
            const Four v = unpack(*ring.slot(stage, i, 1));
#pragma unroll
            for (int j = 0; j < 2; ++j) before[i + 1].p[j] = fma(a[i].p[j], before[i].p[j], mul(q[i].p[j], v.p[j]));
        }
        // one step back: its gradients, and g in front of it
        auto back = [&](int i, Four& oz, Four& ov) {
            const Four v = unpack(*ring.slot(stage, i, 1)), e = unpack(*ring.slot(stage, i, 2));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 d = __fadd2_rn(e.p[j], g.p[j]);
                ov.p[j] = mul(q[i].p[j], d);
                g.p[j] = mul(a[i].p[j], d);
                oz.p[j] = mul(mul(a[i].p[j], ov.p[j]), fma(v.p[j], both(-1.f), before[i].p[j]));
            }
        };
        const int n = left > 0 ? steps_before(len, t0) : 0;
        if (n == STEPS) {
#pragma unroll
            for (int i = STEPS - 1; i >= 0; --i) {
                Four oz, ov;
                back(i, oz, ov);
                put<T, ACC>(dz + i * p.dz_t, oz, left, p.accum);
                put<T, ACC>(dv + i * p.dv_t, ov, left, p.accum);
            }
        } else {
            const int out = left > 0 ? steps_before(p.T, t0) : 0;
#pragma unroll
            for (int i = STEPS - 1; i >= 0; --i) {
                Four oz, ov;
                back(i, oz, ov);
                if (i < out) {
                    put<T, ACC>(dz + i * p.dz_t, i < n ? oz : Four{}, left, p.accum);
                    put<T, ACC>(dv + i * p.dv_t, i < n ? ov : Four{}, left, p.accum);
                }
            }
        }
        if (R == 1 && tg == 0) *(float4*)&carried[now ^ 1][cx * N] = make_float4(g.p[0].x, g.p[0].y, g.p[1].x, g.p[1].y);
        t0 -= stride; tile -= R; dz -= stride * p.dz_t; dv -= stride * p.dv_t;
        stage = stage + 1 == Rg::STAGES ? 0 : stage + 1;
    }
    if (R > 1) cg::this_cluster().sync();
    else { __syncthreads(); carry.set(&carried[rounds & 1][first]); }
    if (p.dstate && rank == 0 && threadIdx.x < G::TEAM) {
#pragma unroll
        for (int j = 0; j < Lanes<CX>::M; ++j) if (c0 + first + j < p.C) p.dstate[b * p.C + c0 + first + j] = carry.v[j];
    }
}

// How a launch is cut: CX threads along the channels, clusters of R CTAs along the steps.
struct Cut { int cx, r; };
int sms() {
    static int n[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); return 148; }
    if (!n[dev]) { int v = 0; cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev); n[dev] = v > 0 ? v : 148; }
    return n[dev];
}
Cut cut(long B, long T, long C) {
    auto tile = [](int cx) { return THREADS / cx * STEPS; };
    Cut k{64, 1};
    const char* e = getenv("RCX");      // probe
    if (e) { k.cx = atoi(e); k.r = atoi(getenv("RR")); return k; }
    while (k.cx > 4 && T > tile(k.cx) && B * ((C + 4 * k.cx - 1) / (4 * k.cx)) < 3 * 148) k.cx /= 4;
    const long ctas = B * ((C + 4 * k.cx - 1) / (4 * k.cx)), tiles = (T + tile(k.cx) - 1) / tile(k.cx);
    while (k.r < MAX_CLUSTER && ctas * k.r < 2 * 148 && tiles > k.r) k.r *= 2;
    return k;
}

template <typename T, int ACC, int CX, bool BACK>
cudaError_t launch(const RecurArgs& a, int R, cudaStream_t s) {
    constexpr int bytes = BACK ? Ring<T, 3>::BYTES : Ring<T, 2>::BYTES;
    static OncePerDevice once;
    const auto k = BACK ? recur_bwd_k<T, ACC, CX> : recur_fwd_k<T, ACC, CX>;
    const cudaError_t e = allow_smem(once, (const void*)k, bytes);
    if (e != cudaSuccess) return e;
    const int slices = (int)((a.C + Geo<CX>::CH - 1) / Geo<CX>::CH);
    return klaunch_cluster(k, (unsigned)(a.B * slices * R), THREADS, bytes, s, R > 1 ? R : 0, a, R, slices);
}
template <typename T, int ACC, bool BACK>
cudaError_t pick(const RecurArgs& a, cudaStream_t s) {
    const Cut k = cut(a.B, a.T, a.C);
    switch (k.cx) {
        case 4: return launch<T, ACC, 4, BACK>(a, k.r, s);
        case 8: return launch<T, ACC, 8, BACK>(a, k.r, s);
        case 16: return launch<T, ACC, 16, BACK>(a, k.r, s);
        case 32: return launch<T, ACC, 32, BACK>(a, k.r, s);
        default: return launch<T, ACC, 64, BACK>(a, k.r, s);
    }
}
// elements (4, 2, 1) that may be moved at once: every row of every tensor starts on that many
template <bool BACK>
cudaError_t run(int dt, const RecurArgs& a, cudaStream_t s) {
    const size_t z = dt ? 2 : 4;
    uint64_t m = (uint64_t)a.C * z | (uintptr_t)a.z | (uintptr_t)a.v | (uint64_t)(a.z_b | a.z_t | a.v_b | a.v_t) * z;
    if (BACK) m |= (uintptr_t)a.dy | (uintptr_t)a.dz | (uintptr_t)a.dv | (uint64_t)(a.dy_b | a.dy_t | a.dz_b | a.dz_t | a.dv_b | a.dv_t) * z;
    else m |= (uintptr_t)a.y | (uint64_t)(a.y_b | a.y_t) * z;
    if (dt) return m % 8 == 0 ? pick<bf16, 4, BACK>(a, s) : m % 4 == 0 ? pick<bf16, 2, BACK>(a, s) : pick<bf16, 1, BACK>(a, s);
    return m % 16 == 0 ? pick<float, 4, BACK>(a, s) : pick<float, 1, BACK>(a, s);
}

}  // namespace

size_t recur_saved_bytes(int, long B, long T, long C) {
    const int tile = THREADS / cut(B, T, C).cx * STEPS;
    return (size_t)B * ((T + tile - 1) / tile) * C * sizeof(float);
}

cudaError_t recur_forward(int dt, const RecurArgs& a, cudaStream_t s) {
    if (a.B * a.C == 0) return cudaSuccess;
    Scope sc(KC_RECUR_FWD, 8.0 * a.B * a.T * a.C, 3.0 * a.B * a.T * a.C * (dt ? 2 : 4), s);
    return run<false>(dt, a, s);
}

cudaError_t recur_backward(int dt, const RecurArgs& a, cudaStream_t s) {
    if (a.B * a.C == 0) return cudaSuccess;
    Scope sc(KC_RECUR_BWD, 16.0 * a.B * a.T * a.C, 5.0 * a.B * a.T * a.C * (dt ? 2 : 4), s);
    return run<true>(dt, a, s);
}

}  // namespace fdg
