// Gated linear recurrence, per sequence and channel:  a = sigmoid(z),  h_t = a_t h_{t-1} + (1 - a_t) v_t,  y_t = h_t.
// Backward, with d_t = dy_t + a_{t+1} d_{t+1}:  dv_t = (1 - a_t) d_t,  dz_t = a_t (1 - a_t) d_t (h_{t-1} - v_t),  dh_0 = a_1 d_1.
//
// A step is the affine map h -> a h + u, u = (1 - a) v; maps compose: (A, H) then (A', H') is (A' A, A' H + H').  So a sequence is cut into pieces whose
// maps are found side by side and joined: a thread composes STEPS = 4 steps of four channels, a warp its threads by shuffles, the CTA its warps and, where
// a launch would otherwise be too small, a cluster its CTAs through distributed shared memory; then every thread runs its steps again from the state in front of
// them.  The joins are a fixed tree, so equal inputs give equal bits.  Backwards the same with g_t = a_t d_t, the map g -> a (g + dy).
// The gate is computed twice (once to find the maps, once to apply them): the exponential and the reciprocal cost less than the registers that would hold it.
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

// a = sigmoid(z) and b = 1 - a = sigmoid(-z), each to a few units of its own last place; 0 and 1 at the infinities
__device__ __forceinline__ void gate(float z, float& a, float& b) {
    const float e = __expf(-fabsf(z));
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    const float q = e * r;
    a = z >= 0.f ? r : q;
    b = z >= 0.f ? q : r;
}

template <typename T> struct Raw;                    // N values as they are stored
template <> struct Raw<float> { using V = float4; };
template <> struct Raw<bf16> { using V = uint2; };
__device__ __forceinline__ void unpack(const float4& r, float* x) { x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w; }
__device__ __forceinline__ void unpack(const uint2& r, float* x) {
    x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xffff0000u);
    x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xffff0000u);
}
__device__ __forceinline__ void pack(const float* x, float4& r) { r = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void pack(const float* x, uint2& r) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(x[0], x[1]), hi = __floats2bfloat162_rn(x[2], x[3]);
    r = make_uint2(*(const unsigned*)&lo, *(const unsigned*)&hi);
}
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
        for (int j = 0; j < N; j += ACC) if (j < left) copy_async<ACC * sizeof(T)>((T*)slot + j, g + j);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) if (j < left) ((T*)slot)[j] = g[j];
    }
}
template <typename T, int ACC> __device__ __forceinline__ void put(T* g, float* x, int left, bool accum) {
    if (accum) for (int j = 0; j < N; ++j) if (j < left) x[j] += ld(g + j);
    if constexpr (ACC == N) {
        if (left > 0) { typename Raw<T>::V r; pack(x, r); *(typename Raw<T>::V*)g = r; }
    } else if constexpr (ACC == 2) {
        if (left > 0) *(__nv_bfloat162*)g = __floats2bfloat162_rn(x[0], x[1]);
        if (left > 2) *(__nv_bfloat162*)(g + 2) = __floats2bfloat162_rn(x[2], x[3]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) if (j < left) st(g + j, x[j]);
    }
}

template <typename T, int TENSORS> struct Ring {
    using V = typename Raw<T>::V;
    static constexpr int STAGES = sizeof(T) == 2 ? (TENSORS == 2 ? 4 : 3) : 2;
    static constexpr int BYTES = STAGES * STEPS * TENSORS * THREADS * (int)sizeof(V);
    V* base;
    __device__ V* slot(int stage, int i, int tensor) const { return base + ((stage * STEPS + i) * TENSORS + tensor) * THREADS + threadIdx.x; }
};

// (a1, h1), then (a2, h2)
__device__ __forceinline__ void then(float a1, float h1, float a2, float h2, float& a, float& h) { h = fmaf(a2, h1, h2); a = a2 * a1; }

template <typename T, int ACC, int CX>
__global__ void __launch_bounds__(THREADS) recur_fwd_k(RecurArgs p, int R, int slices) {
    using G = Geo<CX>;
    extern __shared__ __align__(16) char dyn[];
    const Ring<T, 2> ring{(typename Raw<T>::V*)dyn};
    constexpr int STAGES = Ring<T, 2>::STAGES;
    __shared__ __align__(16) float tot_a[G::TEAMS][G::CH], tot_h[G::TEAMS][G::CH], in_h[G::TEAMS][G::CH];
    __shared__ float2 joined[2][G::RANKS][G::CH];
    const int rank = R > 1 ? (int)(blockIdx.x % R) : 0;
    const long group = blockIdx.x / R, b = group / slices;
    const long c0 = (group - b * slices) * G::CH;
    const int cx = threadIdx.x % CX, tg = threadIdx.x / CX, team = threadIdx.x / G::TEAM;
    const long c = c0 + cx * N;
    const int left = (int)min((long)N, p.C - c);                 // channels of this thread that exist
    const T* const z = (const T*)p.z + b * p.z_b + c;
    const T* const v = (const T*)p.v + b * p.v_b + c;
    T* const y = (T*)p.y + b * p.y_b + c;
    const long len = p.lengths ? min((long)max(p.lengths[b], 0), p.T) : p.T;
    const long tiles = (p.T + G::TILE - 1) / G::TILE, rounds = (tiles + R - 1) / R;
    auto fetch_tile = [&](long round) {
        if (round < rounds) {
            const long t0 = (round * R + rank) * G::TILE + tg * STEPS;
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
                if (t0 + i < len) {
                    fetch<T, ACC>(ring.slot((int)(round % STAGES), i, 0), z + (t0 + i) * p.z_t, left);
                    fetch<T, ACC>(ring.slot((int)(round % STAGES), i, 1), v + (t0 + i) * p.v_t, left);
                }
        }
        copies_issued();
    };
    for (int s = 0; s < STAGES - 1; ++s) fetch_tile(s);
    const bool keeper = threadIdx.x < G::CH;                     // one thread per channel joins the teams
    const long kc = c0 + threadIdx.x;
    float carry = keeper && kc < p.C && p.state ? p.state[b * p.C + kc] : 0.f;
    for (long round = 0; round < rounds; ++round) {
        fetch_tile(round + STAGES - 1);
        copies_arrived<STAGES - 1>();
        const int stage = (int)(round % STAGES);
        const long tile = round * R + rank, t0 = tile * G::TILE + tg * STEPS;
        // the map of this thread's steps
        float A[N] = {1.f, 1.f, 1.f, 1.f}, H[N] = {};
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (t0 + i < len) {
                float zz[N], vv[N];
                unpack(*ring.slot(stage, i, 0), zz); unpack(*ring.slot(stage, i, 1), vv);
#pragma unroll
                for (int j = 0; j < N; ++j) { float a, q; gate(zz[j], a, q); H[j] = fmaf(a, H[j], q * vv[j]); A[j] *= a; }
            }
        // of the threads in front of it in its team, and the team's
        float Ax[N], Hx[N];
        if constexpr (CX < 32) {
#pragma unroll
            for (int d = CX; d < 32; d *= 2)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float a = __shfl_up_sync(~0u, A[j], d), h = __shfl_up_sync(~0u, H[j], d);
                    if ((int)(threadIdx.x & 31) >= d) then(a, h, A[j], H[j], A[j], H[j]);
                }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                Ax[j] = __shfl_up_sync(~0u, A[j], CX); Hx[j] = __shfl_up_sync(~0u, H[j], CX);
                if ((int)(threadIdx.x & 31) < CX) { Ax[j] = 1.f; Hx[j] = 0.f; }
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) { Ax[j] = 1.f; Hx[j] = 0.f; }
        }
        if (CX >= 32 || (int)(threadIdx.x & 31) >= 32 - CX) {
            *(float4*)&tot_a[team][cx * N] = make_float4(A[0], A[1], A[2], A[3]);
            *(float4*)&tot_h[team][cx * N] = make_float4(H[0], H[1], H[2], H[3]);
        }
        __syncthreads();
        if (R > 1) {                                             // the CTA's map goes to every CTA of the cluster
            cg::cluster_group cl = cg::this_cluster();
            if (keeper) {
                float a = 1.f, h = 0.f;
                for (int w = 0; w < G::TEAMS; ++w) then(a, h, tot_a[w][threadIdx.x], tot_h[w][threadIdx.x], a, h);
                for (int r = 0; r < R; ++r) *cl.map_shared_rank(&joined[round & 1][rank][threadIdx.x], r) = make_float2(a, h);
            }
            cl.sync();
        }
        if (keeper) {
            float h = carry;
            if (R > 1)
                for (int r = 0; r < R; ++r) {
                    const float2 m = joined[round & 1][r][threadIdx.x];
                    if (r == rank) h = carry;
                    carry = fmaf(m.x, carry, m.y);
                }
            if (p.saved && kc < p.C && tile < tiles) p.saved[(b * tiles + tile) * p.C + kc] = h;
            for (int w = 0; w < G::TEAMS; ++w) { in_h[w][threadIdx.x] = h; h = fmaf(tot_a[w][threadIdx.x], h, tot_h[w][threadIdx.x]); }
            if (R == 1) carry = h;
        }
        __syncthreads();
        float h[N];
        {
            const float4 q = *(const float4*)&in_h[team][cx * N];
            h[0] = fmaf(Ax[0], q.x, Hx[0]); h[1] = fmaf(Ax[1], q.y, Hx[1]); h[2] = fmaf(Ax[2], q.z, Hx[2]); h[3] = fmaf(Ax[3], q.w, Hx[3]);
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if (t0 + i >= p.T) break;
            float o[N] = {};
            if (t0 + i < len) {
                float zz[N], vv[N];
                unpack(*ring.slot(stage, i, 0), zz); unpack(*ring.slot(stage, i, 1), vv);
#pragma unroll
                for (int j = 0; j < N; ++j) { float a, q; gate(zz[j], a, q); o[j] = h[j] = fmaf(a, h[j], q * vv[j]); }
            }
            put<T, ACC>(y + (t0 + i) * p.y_t, o, left, false);
        }
    }
    if (p.state_out && keeper && rank == 0 && kc < p.C) p.state_out[b * p.C + kc] = carry;
    if (R > 1) cg::this_cluster().sync();                        // nobody leaves while others may write to its shared memory
}

template <typename T, int ACC, int CX>
__global__ void __launch_bounds__(THREADS) recur_bwd_k(RecurArgs p, int R, int slices) {
    using G = Geo<CX>;
    extern __shared__ __align__(16) char dyn[];
    const Ring<T, 3> ring{(typename Raw<T>::V*)dyn};
    constexpr int STAGES = Ring<T, 3>::STAGES;
    __shared__ __align__(16) float tot_a[G::TEAMS][G::CH], tot_h[G::TEAMS][G::CH], tot_g[G::TEAMS][G::CH], in_h[G::TEAMS][G::CH], in_g[G::TEAMS][G::CH];
    __shared__ float2 joined[2][G::RANKS][G::CH];
    const int rank = R > 1 ? (int)(blockIdx.x % R) : 0;
    const long group = blockIdx.x / R, b = group / slices;
    const long c0 = (group - b * slices) * G::CH;
    const int cx = threadIdx.x % CX, tg = threadIdx.x / CX, team = threadIdx.x / G::TEAM, lane = threadIdx.x & 31;
    const long c = c0 + cx * N;
    const int left = (int)min((long)N, p.C - c);
    const T* const z = (const T*)p.z + b * p.z_b + c;
    const T* const v = (const T*)p.v + b * p.v_b + c;
    const T* const dy = (const T*)p.dy + b * p.dy_b + c;
    T* const dz = (T*)p.dz + b * p.dz_b + c;
    T* const dv = (T*)p.dv + b * p.dv_b + c;
    const long len = p.lengths ? min((long)max(p.lengths[b], 0), p.T) : p.T;
    const long tiles = (p.T + G::TILE - 1) / G::TILE, rounds = (tiles + R - 1) / R;
    // rounds are counted from the end of the sequence
    auto fetch_tile = [&](long round) {
        if (round < rounds) {
            const long t0 = ((rounds - 1 - round) * R + rank) * G::TILE + tg * STEPS;
            const int stage = (int)(round % STAGES);
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
                if (t0 + i < len) {
                    fetch<T, ACC>(ring.slot(stage, i, 0), z + (t0 + i) * p.z_t, left);
                    fetch<T, ACC>(ring.slot(stage, i, 1), v + (t0 + i) * p.v_t, left);
                    fetch<T, ACC>(ring.slot(stage, i, 2), dy + (t0 + i) * p.dy_t, left);
                }
        }
        copies_issued();
    };
    for (int s = 0; s < STAGES - 1; ++s) fetch_tile(s);
    const bool keeper = threadIdx.x < G::CH;
    const long kc = c0 + threadIdx.x;
    float carry = keeper && kc < p.C && p.dstate_out ? p.dstate_out[b * p.C + kc] : 0.f;
    for (long round = 0; round < rounds; ++round) {
        fetch_tile(round + STAGES - 1);
        const long tile = (rounds - 1 - round) * R + rank, t0 = tile * G::TILE + tg * STEPS;
        const float start = keeper && kc < p.C && tile < tiles ? p.saved[(b * tiles + tile) * p.C + kc] : 0.f;
        copies_arrived<STAGES - 1>();
        const int stage = (int)(round % STAGES);
        float A[N] = {1.f, 1.f, 1.f, 1.f}, H[N] = {}, Q[N] = {};
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (t0 + i < len) {
                float zz[N], vv[N], dd[N];
                unpack(*ring.slot(stage, i, 0), zz); unpack(*ring.slot(stage, i, 1), vv); unpack(*ring.slot(stage, i, 2), dd);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float a, q;
                    gate(zz[j], a, q);
                    H[j] = fmaf(a, H[j], q * vv[j]);
                    A[j] *= a;
                    Q[j] = fmaf(A[j], dd[j], Q[j]);             // what dy of this step is in front of the thread's first one
                }
            }
        float Ax[N], Hx[N], Ay[N], Qy[N];                        // of the threads in front (forward map) and behind (backward map)
        if constexpr (CX < 32) {
            float B[N];
#pragma unroll
            for (int j = 0; j < N; ++j) B[j] = A[j];
#pragma unroll
            for (int d = CX; d < 32; d *= 2)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float a = __shfl_up_sync(~0u, A[j], d), h = __shfl_up_sync(~0u, H[j], d);
                    if (lane >= d) then(a, h, A[j], H[j], A[j], H[j]);
                    const float e = __shfl_down_sync(~0u, B[j], d), q = __shfl_down_sync(~0u, Q[j], d);
                    if (lane < 32 - d) then(e, q, B[j], Q[j], B[j], Q[j]);
                }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                Ax[j] = __shfl_up_sync(~0u, A[j], CX); Hx[j] = __shfl_up_sync(~0u, H[j], CX);
                Ay[j] = __shfl_down_sync(~0u, B[j], CX); Qy[j] = __shfl_down_sync(~0u, Q[j], CX);
                if (lane < CX) { Ax[j] = 1.f; Hx[j] = 0.f; }
                if (lane >= 32 - CX) { Ay[j] = 1.f; Qy[j] = 0.f; }
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) { Ax[j] = Ay[j] = 1.f; Hx[j] = Qy[j] = 0.f; }
        }
        if (CX >= 32 || lane >= 32 - CX) {
            *(float4*)&tot_a[team][cx * N] = make_float4(A[0], A[1], A[2], A[3]);
            *(float4*)&tot_h[team][cx * N] = make_float4(H[0], H[1], H[2], H[3]);
        }
        if (CX >= 32 || lane < CX) *(float4*)&tot_g[team][cx * N] = make_float4(Q[0], Q[1], Q[2], Q[3]);
        __syncthreads();
        if (R > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (keeper) {
                float a = 1.f, g = 0.f;
                for (int w = G::TEAMS - 1; w >= 0; --w) then(a, g, tot_a[w][threadIdx.x], tot_g[w][threadIdx.x], a, g);
                for (int r = 0; r < R; ++r) *cl.map_shared_rank(&joined[round & 1][rank][threadIdx.x], r) = make_float2(a, g);
            }
            cl.sync();
        }
        if (keeper) {
            float h = start, g = carry;
            if (R > 1)
                for (int r = R - 1; r >= 0; --r) {
                    const float2 m = joined[round & 1][r][threadIdx.x];
                    if (r == rank) g = carry;
                    carry = fmaf(m.x, carry, m.y);
                }
            for (int w = 0; w < G::TEAMS; ++w) {
                const int u = G::TEAMS - 1 - w;
                in_h[w][threadIdx.x] = h; h = fmaf(tot_a[w][threadIdx.x], h, tot_h[w][threadIdx.x]);
                in_g[u][threadIdx.x] = g; g = fmaf(tot_a[u][threadIdx.x], g, tot_g[u][threadIdx.x]);
            }
            if (R == 1) carry = g;
        }
        __syncthreads();
        float g[N], a[STEPS][N], q[STEPS][N], before[STEPS][N];
        {
            const float4 x = *(const float4*)&in_h[team][cx * N], w = *(const float4*)&in_g[team][cx * N];
            before[0][0] = fmaf(Ax[0], x.x, Hx[0]); before[0][1] = fmaf(Ax[1], x.y, Hx[1]); before[0][2] = fmaf(Ax[2], x.z, Hx[2]); before[0][3] = fmaf(Ax[3], x.w, Hx[3]);
            g[0] = fmaf(Ay[0], w.x, Qy[0]); g[1] = fmaf(Ay[1], w.y, Qy[1]); g[2] = fmaf(Ay[2], w.z, Qy[2]); g[3] = fmaf(Ay[3], w.w, Qy[3]);
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            float zz[N], vv[N];
            unpack(*ring.slot(stage, i, 0), zz); unpack(*ring.slot(stage, i, 1), vv);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                gate(zz[j], a[i][j], q[i][j]);
                if (i + 1 < STEPS) before[i + 1][j] = fmaf(a[i][j], before[i][j], q[i][j] * vv[j]);
            }
        }
#pragma unroll
        for (int i = STEPS - 1; i >= 0; --i) {
            if (t0 + i >= p.T) continue;
            float oz[N] = {}, ov[N] = {};
            if (t0 + i < len) {
                float vv[N], dd[N];
                unpack(*ring.slot(stage, i, 1), vv); unpack(*ring.slot(stage, i, 2), dd);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float d = dd[j] + g[j];
                    ov[j] = q[i][j] * d;
                    oz[j] = a[i][j] * ov[j] * (before[i][j] - vv[j]);
                    g[j] = a[i][j] * d;
                }
            }
            put<T, ACC>(dz + (t0 + i) * p.dz_t, oz, left, p.accum);
            put<T, ACC>(dv + (t0 + i) * p.dv_t, ov, left, p.accum);
        }
    }
    if (p.dstate && keeper && rank == 0 && kc < p.C) p.dstate[b * p.C + kc] = carry;
    if (R > 1) cg::this_cluster().sync();
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
