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

namespace fdg {
namespace {

namespace cg = cooperative_groups;
using bf16 = __nv_bfloat16;

constexpr int THREADS = 256;
constexpr int STEPS = 4;                // of a thread in a tile
constexpr int N = 4;                    // channels of a thread
constexpr int MAX_CLUSTER = 8;      // of slices up to 32 channels; wider ones have no clusters

// CX threads lie along the channels, the others along the steps.
template <int CX> struct Geo {
    static constexpr int TG = THREADS / CX, CH = CX * N, TILE = TG * STEPS;
    static constexpr int TEAM = CX < 32 ? 32 : CX, TEAMS = THREADS / TEAM;      // a team joins its threads by shuffles (or is one step group)
    static constexpr int RANKS = CX > 8 ? 1 : MAX_CLUSTER;
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
__device__ __forceinline__ int steps_before(int end, int t0) { return min(max(end - t0, 0), STEPS); }

template <typename T, int TENSORS> struct Ring {
    using V = typename Raw<T>::V;
    static constexpr int STAGES = sizeof(T) == 2 ? 3 : 2;
    static constexpr int STAGE = STEPS * TENSORS * THREADS;
    static constexpr int BYTES = STAGES * STAGE * (int)sizeof(V);
    V* mine;                                                     // this thread's first slot
    __device__ V* slot(int stage, int i, int tensor) const { return mine + stage * STAGE + (i * TENSORS + tensor) * THREADS; }
};

__device__ __forceinline__ void store(float* p, const Four& x) { *(float4*)p = make_float4(x.p[0].x, x.p[0].y, x.p[1].x, x.p[1].y); }
__device__ __forceinline__ Four load(const float* p) { const float4 r = *(const float4*)p; return {make_float2(r.x, r.y), make_float2(r.z, r.w)}; }

// Joining the maps of a tile.  Up to 32 channels (CX <= 8) a warp holds several step groups: its threads leave their maps in shared memory, and a lane takes one channel
// and LINKS = 4 of the groups from there; above (a team is one step group) a lane has its own four channels.
template <int CX> struct Lane {
    static constexpr bool ONE = CX <= 8;
    static constexpr int M = ONE ? 1 : N, CH = CX * N, LINKS = 4, SUBS = ONE ? 32 / CX / LINKS : 1;
    static __device__ __forceinline__ int first() { return ONE ? (threadIdx.x & 31) % CH : threadIdx.x % CX * N; }      // channel of the slice
    static __device__ __forceinline__ int sub() { return ONE ? (threadIdx.x & 31) / CH : 0; }
    static __device__ __forceinline__ bool writes() { return ONE ? (threadIdx.x & 31) < CH : true; }
    float v[M];
    __device__ __forceinline__ void set(const float* p) {
        if constexpr (ONE) v[0] = *p;
        else { const float4 r = *(const float4*)p; v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
    }
    // through the map at p: {A, H} of each channel
    __device__ __forceinline__ void through(const float2* p) {
        if constexpr (ONE) { const float2 m = *p; v[0] = fmaf(m.x, v[0], m.y); }
        else {
            const float4 m = *(const float4*)p, k = *(const float4*)(p + 2);
            v[0] = fmaf(m.x, v[0], m.y); v[1] = fmaf(m.z, v[1], m.w); v[2] = fmaf(k.x, v[2], k.y); v[3] = fmaf(k.z, v[3], k.w);
        }
    }
    // values of a row of C channels, c0: the slice's first
    __device__ __forceinline__ void read(const float* row, long c0, long C) {
#pragma unroll
        for (int j = 0; j < M; ++j) v[j] = row && c0 + first() + j < C ? row[c0 + first() + j] : 0.f;
    }
    __device__ __forceinline__ void write(float* row, long c0, long C) const {
#pragma unroll
        for (int j = 0; j < M; ++j) if (c0 + first() + j < C) row[c0 + first() + j] = v[j];
    }
};
// The maps of a warp's step groups, in order (UP) or against it.
template <int CX, bool UP> struct Chain {
    using L = Lane<CX>;
    float a[L::LINKS], h[L::LINKS], ta, th;         // of the lane's groups; of all the warp's
    float fa, fh;                                   // of the groups of the lanes before this one's
    static __device__ __forceinline__ int at(int k) { return (L::sub() * L::LINKS + (UP ? k : L::LINKS - 1 - k)) * L::CH + L::first(); }
    // wa, wh: [step group][channel] of this warp
    __device__ __forceinline__ void read(const float* wa, const float* wh) {
#pragma unroll
        for (int k = 0; k < L::LINKS; ++k) { a[k] = wa[at(k)]; h[k] = wh[at(k)]; }
        ta = a[0]; th = h[0];
#pragma unroll
        for (int k = 1; k < L::LINKS; ++k) { th = fmaf(a[k], th, h[k]); ta *= a[k]; }
        fa = 1.f; fh = 0.f;
        if constexpr (L::SUBS == 2) {
            const float oa = __shfl_xor_sync(~0u, ta, L::CH), oh = __shfl_xor_sync(~0u, th, L::CH);
            const bool later = (L::sub() == 1) == UP;
            if (later) { fa = oa; fh = oh; th = fmaf(ta, oh, th); } else th = fmaf(oa, th, oh);
            ta *= oa;
        }
    }
    // from the value in front of the warp: the values in front of its groups, to w (may be wh)
    __device__ __forceinline__ void apply(float v, float* w) const {
        v = fmaf(fa, v, fh);
#pragma unroll
        for (int k = 0; k < L::LINKS; ++k) { w[at(k)] = v; v = fmaf(a[k], v, h[k]); }
    }
};
__device__ __forceinline__ void store(float2* p, const Four& A, const Four& H) {
    *(float4*)p = make_float4(A.p[0].x, H.p[0].x, A.p[0].y, H.p[0].y);
    *(float4*)(p + 2) = make_float4(A.p[1].x, H.p[1].x, A.p[1].y, H.p[1].y);
}

// One barrier a tile: behind it a warp goes through the maps of the teams in front of it by itself, and the last steps' threads leave the state for the
// next tile, which the next tile's barrier orders.  What stands there is kept twice, by the round's parity.
template <typename T, int ACC, int CX, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 3) recur_fwd_k(RecurArgs p, int ranks, int slices) {
    const int R = CLUSTER ? ranks : 1;
    using G = Geo<CX>;
    using Rg = Ring<T, 2>;
    extern __shared__ __align__(16) char dyn[];
    const Rg ring{(typename Rg::V*)dyn + threadIdx.x};
    __shared__ __align__(16) float2 tot[2][G::TEAMS][G::CH];
    __shared__ __align__(16) float own[2][Lane<CX>::ONE ? THREADS * N : 1];      // a warp's maps, later the states in front of its step groups
    __shared__ __align__(16) float carried[2][G::CH];
    __shared__ __align__(16) float2 joined[2][G::RANKS][G::CH];
    const int rank = CLUSTER ? (int)(blockIdx.x % R) : 0;
    const long group = blockIdx.x / R, b = group / slices;
    const long c0 = (group - b * slices) * G::CH;
    const int cx = threadIdx.x % CX, tg = threadIdx.x / CX, team = threadIdx.x / G::TEAM;
    const long c = c0 + cx * N;
    const int left = (int)min((long)N, p.C - c);                 // channels of this thread that exist
    const int T_ = (int)p.T, len = p.lengths ? min(max(p.lengths[b], 0), T_) : T_;
    const int tiles = (T_ + G::TILE - 1) / G::TILE, rounds = (tiles + R - 1) / R, stride = R * G::TILE;
    int t0 = rank * G::TILE + tg * STEPS, tf = t0;        // this thread's first step: of the round, of the next tile to fetch
    const T* zf = (const T*)p.z + b * p.z_b + c + t0 * p.z_t;
    const T* vf = (const T*)p.v + b * p.v_b + c + t0 * p.v_t;
    T* y = (T*)p.y + b * p.y_b + c + t0 * p.y_t;
    const long z_round = stride * p.z_t, v_round = stride * p.v_t, y_round = stride * p.y_t;
    auto fetch_tile = [&](int stage) {
        const int n = left > 0 ? steps_before(len, tf) : 0;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < n) {
                fetch<T, ACC>(ring.slot(stage, i, 0), zf + i * p.z_t, left);
                fetch<T, ACC>(ring.slot(stage, i, 1), vf + i * p.v_t, left);
            } else idle(ring.slot(stage, i, 0), ring.slot(stage, i, 1));
        copies_issued();
        tf += stride; zf += z_round; vf += v_round;
    };
    for (int s = 0; s < Rg::STAGES - 1; ++s) fetch_tile(s);
    if (CLUSTER) cg::this_cluster().sync();                        // every CTA is there before anyone writes to its shared memory
    const int first = Lane<CX>::first(), mine = (threadIdx.x & ~31) * N;
    Lane<CX> carry;                                              // CLUSTER: the state in front of the round, in every warp
    carry.read(p.state ? p.state + b * p.C : nullptr, c0, p.C);
    if (threadIdx.x < G::CH) carried[0][threadIdx.x] = p.state && c0 + threadIdx.x < p.C ? p.state[b * p.C + c0 + threadIdx.x] : 0.f;
    int stage = 0;
    for (int round = 0; round < rounds; ++round) {
        const int now = round & 1;
        fetch_tile(stage == 0 ? Rg::STAGES - 1 : stage - 1);
        copies_arrived<Rg::STAGES - 1>();
        // the map of this thread's steps
        Four a[STEPS], u[STEPS], A, H;
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
        Chain<CX, true> chain;
        if constexpr (Lane<CX>::ONE) {
            __syncwarp();
            store(&own[0][threadIdx.x * N], A); store(&own[1][threadIdx.x * N], H);
            __syncwarp();
            chain.read(&own[0][mine], &own[1][mine]);
            if (Lane<CX>::writes()) tot[now][team][first] = make_float2(chain.ta, chain.th);
        } else store(&tot[now][team][first], A, H);
        __syncthreads();
        Lane<CX> in;
        if (CLUSTER) {                                             // the CTA's map goes to every CTA of the cluster
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
        if (p.saved && threadIdx.x < G::TEAM && Lane<CX>::writes() && round * R + rank < tiles) in.write(p.saved + ((long)b * tiles + round * R + rank) * p.C, c0, p.C);
        for (int w = 0; w < team; ++w) in.through(&tot[now][w][first]);
        Four h;
        if constexpr (Lane<CX>::ONE) {
            chain.apply(in.v[0], &own[1][mine]);
            __syncwarp();
            h = load(&own[1][threadIdx.x * N]);
        } else h = {make_float2(in.v[0], in.v[1]), make_float2(in.v[2], in.v[3])};
        const int n = left > 0 ? steps_before(len, t0) : 0;
        if (n == STEPS) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) h.p[j] = fma(a[i].p[j], h.p[j], u[i].p[j]);
                put<T, ACC>(y + i * p.y_t, h, left, false);
            }
        } else {
            const int out = left > 0 ? steps_before(T_, t0) : 0;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) h.p[j] = fma(a[i].p[j], h.p[j], u[i].p[j]);
                if (i < out) put<T, ACC>(y + i * p.y_t, i < n ? h : Four{}, left, false);
            }
        }
        if (!CLUSTER && tg == G::TG - 1) *(float4*)&carried[now ^ 1][cx * N] = make_float4(h.p[0].x, h.p[0].y, h.p[1].x, h.p[1].y);
        t0 += stride; y += y_round;
        stage = stage + 1 == Rg::STAGES ? 0 : stage + 1;
    }
    if (CLUSTER) cg::this_cluster().sync();                        // nobody leaves while others may write to its shared memory
    else { __syncthreads(); carry.set(&carried[rounds & 1][first]); }
    if (p.state_out && rank == 0 && threadIdx.x < G::TEAM && Lane<CX>::writes()) carry.write(p.state_out + b * p.C, c0, p.C);
}

template <typename T, int ACC, int CX, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 2) recur_bwd_k(RecurArgs p, int ranks, int slices) {
    const int R = CLUSTER ? ranks : 1;
    using G = Geo<CX>;
    using Rg = Ring<T, 3>;
    extern __shared__ __align__(16) char dyn[];
    const Rg ring{(typename Rg::V*)dyn + threadIdx.x};
    __shared__ __align__(16) float2 tot_h[2][G::TEAMS][G::CH], tot_g[2][G::TEAMS][G::CH];
    __shared__ __align__(16) float own[3][Lane<CX>::ONE ? THREADS * N : 1];
    __shared__ __align__(16) float carried[2][G::CH];
    __shared__ __align__(16) float2 joined[2][G::RANKS][G::CH];
    const int rank = CLUSTER ? (int)(blockIdx.x % R) : 0;
    const long group = blockIdx.x / R, b = group / slices;
    const long c0 = (group - b * slices) * G::CH;
    const int cx = threadIdx.x % CX, tg = threadIdx.x / CX, team = threadIdx.x / G::TEAM;
    const long c = c0 + cx * N;
    const int left = (int)min((long)N, p.C - c);
    const int T_ = (int)p.T, len = p.lengths ? min(max(p.lengths[b], 0), T_) : T_;
    const int tiles = (T_ + G::TILE - 1) / G::TILE, rounds = (tiles + R - 1) / R, stride = R * G::TILE;
    // rounds go from the end of the sequence to its beginning
    int tile = (rounds - 1) * R + rank, t0 = tile * G::TILE + tg * STEPS, tf = t0;
    const T* zf = (const T*)p.z + b * p.z_b + c + t0 * p.z_t;
    const T* vf = (const T*)p.v + b * p.v_b + c + t0 * p.v_t;
    const T* df = (const T*)p.dy + b * p.dy_b + c + t0 * p.dy_t;
    T* dz = (T*)p.dz + b * p.dz_b + c + t0 * p.dz_t;
    T* dv = (T*)p.dv + b * p.dv_b + c + t0 * p.dv_t;
    const long z_round = stride * p.z_t, v_round = stride * p.v_t, d_round = stride * p.dy_t, dz_round = stride * p.dz_t, dv_round = stride * p.dv_t;
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
        tf -= stride; zf -= z_round; vf -= v_round; df -= d_round;
    };
    for (int s = 0; s < Rg::STAGES - 1; ++s) fetch_tile(s);
    if (CLUSTER) cg::this_cluster().sync();                        // every CTA is there before anyone writes to its shared memory
    const int first = Lane<CX>::first(), mine = (threadIdx.x & ~31) * N;
    Lane<CX> carry;
    carry.read(p.dstate_out ? p.dstate_out + b * p.C : nullptr, c0, p.C);
    if (threadIdx.x < G::CH) carried[0][threadIdx.x] = p.dstate_out && c0 + threadIdx.x < p.C ? p.dstate_out[b * p.C + c0 + threadIdx.x] : 0.f;
    int stage = 0;
    for (int round = 0; round < rounds; ++round) {
        const int now = round & 1;
        fetch_tile(stage == 0 ? Rg::STAGES - 1 : stage - 1);
        Lane<CX> in_h, in_g;
        in_h.read(tile < tiles ? p.saved + ((long)b * tiles + tile) * p.C : nullptr, c0, p.C);
        copies_arrived<Rg::STAGES - 1>();
        Four a[STEPS], q[STEPS], A, H, Q;
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
        Chain<CX, true> front;                                   // the forward map
        Chain<CX, false> behind;                                 // the backward map
        if constexpr (Lane<CX>::ONE) {
            __syncwarp();
            store(&own[0][threadIdx.x * N], A); store(&own[1][threadIdx.x * N], H); store(&own[2][threadIdx.x * N], Q);
            __syncwarp();
            front.read(&own[0][mine], &own[1][mine]);
            behind.read(&own[0][mine], &own[2][mine]);
            if (Lane<CX>::writes()) {
                tot_h[now][team][first] = make_float2(front.ta, front.th);
                tot_g[now][team][first] = make_float2(behind.ta, behind.th);
            }
        } else { store(&tot_h[now][team][first], A, H); store(&tot_g[now][team][first], A, Q); }
        __syncthreads();
        if (CLUSTER) {
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
        Four g, before[STEPS];
        if constexpr (Lane<CX>::ONE) {
            front.apply(in_h.v[0], &own[1][mine]);
            behind.apply(in_g.v[0], &own[2][mine]);
            __syncwarp();
            before[0] = load(&own[1][threadIdx.x * N]);
            g = load(&own[2][threadIdx.x * N]);
        } else {
            before[0] = {make_float2(in_h.v[0], in_h.v[1]), make_float2(in_h.v[2], in_h.v[3])};
            g = {make_float2(in_g.v[0], in_g.v[1]), make_float2(in_g.v[2], in_g.v[3])};
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
            const int out = left > 0 ? steps_before(T_, t0) : 0;
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
        if (!CLUSTER && tg == 0) *(float4*)&carried[now ^ 1][cx * N] = make_float4(g.p[0].x, g.p[0].y, g.p[1].x, g.p[1].y);
        t0 -= stride; tile -= R; dz -= dz_round; dv -= dv_round;
        stage = stage + 1 == Rg::STAGES ? 0 : stage + 1;
    }
    if (CLUSTER) cg::this_cluster().sync();
    else { __syncthreads(); carry.set(&carried[rounds & 1][first]); }
    if (p.dstate && rank == 0 && threadIdx.x < G::TEAM && Lane<CX>::writes()) carry.write(p.dstate + b * p.C, c0, p.C);
}

// How a launch is cut: cx threads along the channels, clusters of r CTAs along the steps.  Both directions use the same cut (the states in front of the tiles
// pass between them), and it depends on the sizes alone.
struct Cut { int cx, r; };
Cut cut(long B, long T, long C) {
    if (T <= 16) return {64, 1};
    if (T <= 32) return {32, 1};
    auto tiles = [&](int cx) { return (T + THREADS / cx * STEPS - 1) / (THREADS / cx * STEPS); };
    auto ctas = [&](int cx) { return B * ((C + N * cx - 1) / (N * cx)); };
    Cut k{8, 1};
    if (ctas(8) * MAX_CLUSTER < 2 * 148) k.cx = 4;
    while (k.r < MAX_CLUSTER && ctas(k.cx) * k.r * 2 <= 2 * 148 && tiles(k.cx) >= 16 * k.r) k.r *= 2;
    return k;
}

template <typename T, int ACC, int CX, bool BACK, bool CLUSTER>
cudaError_t launch(const RecurArgs& a, int R, cudaStream_t s) {
    constexpr int bytes = BACK ? Ring<T, 3>::BYTES : Ring<T, 2>::BYTES;
    static OncePerDevice once;
    const auto k = BACK ? recur_bwd_k<T, ACC, CX, CLUSTER> : recur_fwd_k<T, ACC, CX, CLUSTER>;
    const cudaError_t e = allow_smem(once, (const void*)k, bytes);
    if (e != cudaSuccess) return e;
    const int slices = (int)((a.C + Geo<CX>::CH - 1) / Geo<CX>::CH);
    return klaunch_cluster(k, (unsigned)(a.B * slices * R), THREADS, bytes, s, CLUSTER ? R : 0, a, R, slices);
}
template <typename T, int ACC, bool BACK>
cudaError_t pick(const RecurArgs& a, cudaStream_t s) {
    const Cut k = cut(a.B, a.T, a.C);
    switch (k.cx) {
        case 4: return k.r > 1 ? launch<T, ACC, 4, BACK, true>(a, k.r, s) : launch<T, ACC, 4, BACK, false>(a, 1, s);
        case 8: return k.r > 1 ? launch<T, ACC, 8, BACK, true>(a, k.r, s) : launch<T, ACC, 8, BACK, false>(a, 1, s);
        case 32: return launch<T, ACC, 32, BACK, false>(a, 1, s);
        default: return launch<T, ACC, 64, BACK, false>(a, 1, s);
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
