// Gated linear recurrence, per sequence and channel:  a = sigmoid(z),  h_t = a_t h_{t-1} + (1 - a_t) v_t,  y_t = h_t.
// Backward, with d_t = dy_t + a_{t+1} d_{t+1}:  dv_t = (1 - a_t) d_t,  dz_t = a_t (1 - a_t) d_t (h_{t-1} - v_t),  dh_0 = a_1 d_1.
//
// A step is the affine map h -> a h + u, u = (1 - a) v; maps compose: (A, H) then (A', H') is (A' A, A' H + H').  So a sequence is cut into pieces whose
// maps are found side by side and joined: a thread composes 4 or 8 steps of four channels, a warp its threads through shared memory, the CTA its warps and, where
// a launch would otherwise be too small, a cluster its CTAs through distributed shared memory; then every thread runs its steps again from the state in front of
// them.  The joins are a fixed tree, so equal inputs give equal bits.  Backwards the same with g_t = a_t d_t, the map g -> a (g + dy).
//
// Bound: HBM (forward 3 values a step and channel, backward 5).  A CTA walks along its sequence with a ring of tiles that tensor copies fill ahead.
// States are held in 32 bits.  The backward pass computes h again from the states that the forward pass leaves in front of every tile: y rounded to bf16 would
// put 2^-9 of h into dz, and the states are 2 / (tile's steps) of the bytes of y.
#include "seqops.h"
#include "launch.h"
#include "tc_gemm.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <type_traits>

namespace fdg {
namespace {

namespace cg = cooperative_groups;
using bf16 = __nv_bfloat16;

constexpr int THREADS = 256;
constexpr int STEPS = 4;                // of a thread in a tile, backwards (eight, whose gates would have to be computed twice for want of registers: 52 us instead of 39, 8 x 2048 x 1024)
// Forward, where there are registers for eight, and with fp32 no shared memory: 1 x 16384 x 2048 bf16 47 us, with four 54; 1 x 60001 x 512: 55 and 62.
template <typename T> constexpr int STEPS_FWD = sizeof(T) == 2 ? 8 : 4;
constexpr int N = 4;                    // channels of a thread
constexpr int MAX_CLUSTER = 8;          // of slices up to 32 channels; wider ones have no clusters

// CX threads lie along the channels, the others along the steps.
template <int CX, int S> struct Geo {
    static constexpr int TG = THREADS / CX, CH = CX * N, TILE = TG * S;
    static constexpr int TEAM = CX < 32 ? 32 : CX, TEAMS = THREADS / TEAM;      // a team joins its threads by shuffles (or is one step group)
};

// Values go in pairs through the packed fp32 instructions: the kernels issue too much, not too little, to keep up with HBM.
struct Four { float2 p[2]; };
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }

// a = sigmoid(z) and q = 1 - a: e = 2^min(-z log2 e, 126), a = 1 / (1 + e), q = e a.  Each is off by 4 units of its own last place and, for want of bits in the
// argument of the power, by |z| more (evaluated with everything else exact: 4 units up to |z| = 5, 15 at 20, 60 at 69).  Behind the bound, where sigmoid(z) is below the least
// normal number, a is that number, 2^-126, and q is 1; NaN stays.
__device__ __forceinline__ void gate(float2 z, float2& a, float2& q) {
    const float2 t = mul(z, both(-1.4426950408889634f));
    float2 e;
    asm("min.NaN.f32 %0, %1, 0f42FC0000;" : "=f"(e.x) : "f"(t.x));
    asm("min.NaN.f32 %0, %1, 0f42FC0000;" : "=f"(e.y) : "f"(t.y));
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
__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// a step that changes nothing: gate open (+infinity), value and dy zero
__device__ __forceinline__ void idle(Four& z, Four& x) { z = {both(INFINITY), both(INFINITY)}; x = {both(0.f), both(0.f)}; }

// ---- tiles on their way through shared memory
template <int BYTES> __device__ __forceinline__ void copy_async(void* smem, const void* g) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((unsigned)__cvta_generic_to_shared(smem)), "l"(g), "n"(BYTES) : "memory");
}
template <int LEFT> __device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ unsigned smem_u32(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool try_wait(const uint64_t* bar, unsigned parity) {
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok;
}
constexpr long long WAIT_CYCLES = 4000000000ll;      // about 2 s
constexpr long long STAY_CYCLES = 4000000ll;         // about 2 ms
constexpr int TIMEOUT_CODE = 30;                     // in the caller's error word
// How long waits last, in cycles; the caller's error word.  (Not in RecurArgs: with 24 bytes more of arguments a launch takes the host 0.7 us longer, a fifth of a single step's call.)
struct Waits { long long copies, peers; int* err; };
// The maps of gate, value and dy; used by the kernels whose rows lie on 16 bytes.
struct Maps { tc::TensorMap t[3]; };

// ACC: elements that can be moved at once, as the addresses allow.  16 bytes: tensor copies (TMA), one thread for the CTA; their arrival is signalled on a barrier per
// stage.  4 bytes: cp.async, less: plain loads; there every thread copies what it reads itself, and waits for its own copies.
template <typename T, int ACC, int CX, int S, int TENSORS> struct Ring {
    using V = typename Raw<T>::V;
    using G = Geo<CX, S>;
    static constexpr bool TMA = ACC * sizeof(T) == 16;
    static constexpr int STAGES = sizeof(T) == 2 ? 3 : 2, ROW = G::CH * (int)sizeof(T), TENSOR = G::TILE * ROW, STAGE = TENSORS * TENSOR, BYTES = STAGES * STAGE;
    static constexpr int BOX = G::TILE < 256 ? G::TILE : 256;      // rows of a tensor copy
    char* base;                                      // on 128 bytes
    uint64_t* full;                                  // [STAGES]
    int lost = -1;                                   // >= 0: a wait of this thread gave up, when that many tiles had been asked for.  It asks for no more (a barrier takes
                                                     // no arrival before its last phase is over), waits for nothing, and NaN takes the place of what it did not see.
    __device__ __forceinline__ char* mine(int stage, int tensor, int i) const {
        return base + stage * STAGE + tensor * TENSOR + (threadIdx.x / CX * S + i) * ROW + threadIdx.x % CX * (int)sizeof(V);
    }
    __device__ __forceinline__ Four get(int stage, int tensor, int i) const { return unpack(*(const V*)mine(stage, tensor, i)); }
    __device__ __forceinline__ void begin() const {
        if constexpr (TMA) {
            if (threadIdx.x == 0) {
                for (int i = 0; i < STAGES; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(full + i)) : "memory");
                asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            }
            __syncthreads();
        }
    }
    // rows t .. t + TILE - 1 of sequence b, channels c0 ..; g: this thread's first row and channel of every tensor, `left` of its channels exist, n of its rows count
    __device__ __forceinline__ void fetch(int stage, const Maps& maps, long c0, int t, long b, const T* const (&g)[TENSORS], const long (&step)[TENSORS], int left, int n) const {
        if constexpr (TMA) {
            if (threadIdx.x != 0 || lost >= 0) return;
            const unsigned bar = smem_u32(full + stage);
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((unsigned)STAGE) : "memory");
#pragma unroll
            for (int q = 0; q < TENSORS; ++q)
#pragma unroll
                for (int r = 0; r < G::TILE; r += BOX)
                    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
                                     smem_u32(base + stage * STAGE + q * TENSOR + r * ROW)), "l"(&maps.t[q]), "r"(bar), "r"((int)c0), "r"(t + r), "r"((int)b) : "memory");
        } else {
#pragma unroll
            for (int q = 0; q < TENSORS; ++q)
#pragma unroll
                for (int i = 0; i < S; ++i)
                    if (i < n)
#pragma unroll
                        for (int j = 0; j < N; j += ACC)
                            if (j < left) {
                                if constexpr (ACC * sizeof(T) >= 4) copy_async<ACC * sizeof(T)>((T*)mine(stage, q, i) + j, g[q] + i * step[q] + j);
                                else ((T*)mine(stage, q, i))[j] = g[q][i * step[q] + j];
                            }
        }
    }
    __device__ __forceinline__ void issued() const { if constexpr (!TMA) asm volatile("cp.async.commit_group;" ::: "memory"); }
    // the round's tile; LEFT: copies issued later that may be under way.  Bounded by `limit` cycles (0: given up without a look).
    template <int LEFT> __device__ __forceinline__ void arrived(int stage, int round, long long limit) {
        if constexpr (TMA) {
            const unsigned parity = (unsigned)(round / STAGES & 1);
            if (lost >= 0 || (limit > 0 && try_wait(full + stage, parity))) return;
            const long long t0 = clock64();
            do {
                if (clock64() - t0 >= limit) { lost = round + LEFT + 1; return; }
            } while (!try_wait(full + stage, parity));
        } else copies_arrived<LEFT>();
    }
    // in front of the end: what a wait that gave up left under way (bounded as well), and word of it
    __device__ __forceinline__ void drain(int rounds, int* err) const {
        if (lost < 0) return;
        if (err) atomicCAS(err, 0, TIMEOUT_CODE);
        if constexpr (TMA) {
            if (threadIdx.x != 0) return;
            const int n = min(rounds, lost);
            const long long t0 = clock64();
            for (int r = max(0, n - STAGES); r < n; ++r) while (!try_wait(full + r % STAGES, (unsigned)(r / STAGES & 1))) if (clock64() - t0 > WAIT_CYCLES) return;
        }
    }
};
template <typename T, int ACC> __device__ __forceinline__ void put(T* g, Four x, int left, bool accum) {
    if (accum) {
        if (0 < left) x.p[0].x += ld(g);
        if (1 < left) x.p[0].y += ld(g + 1);
        if (2 < left) x.p[1].x += ld(g + 2);
        if (3 < left) x.p[1].y += ld(g + 3);
    }
    if constexpr (ACC >= N) {
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
// steps of t0 .. t0 + S - 1 that lie in front of `end`
template <int S> __device__ __forceinline__ int steps_before(int end, int t0) { return min(max(end - t0, 0), S); }

__device__ __forceinline__ void store(float* p, const Four& x) { *(float4*)p = make_float4(x.p[0].x, x.p[0].y, x.p[1].x, x.p[1].y); }
__device__ __forceinline__ Four load(const float* p) { const float4 r = *(const float4*)p; return {make_float2(r.x, r.y), make_float2(r.z, r.w)}; }

// Maps of the CTAs of a cluster, {A, H} per channel, sent into the shared memory of all of them; a barrier counts their bytes.  (A cluster-wide barrier would wait for the
// outputs under way too, a microsecond a round.)  Two places by the round's parity suffice: whoever has the maps of round k + 1 knows that all have read those of round k.
template <int CH> struct Joined { float2 at[2][MAX_CLUSTER][CH]; uint64_t bar[2]; };
template <int CH> struct Peers {
    Joined<CH>* j;
    __device__ __forceinline__ void begin() const {
        if (threadIdx.x == 0) {
            for (int i = 0; i < 2; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(j->bar + i)) : "memory");
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        cg::this_cluster().sync();                               // every CTA is there, and its barriers
    }
    // the map of this CTA and thread's channel (threads 0 .. CH - 1)
    __device__ __forceinline__ void send(int round, int rank, int R, float a, float h) const {
        if (threadIdx.x == 0)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(j->bar + (round & 1))), "r"((unsigned)(R * CH * sizeof(float2))) : "memory");
        const unsigned to = smem_u32(&j->at[round & 1][rank][threadIdx.x]), bar = smem_u32(j->bar + (round & 1));
        for (int r = 0; r < R; ++r) {
            unsigned t, b;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(t) : "r"(to), "r"(r));
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(bar), "r"(r));
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(t), "f"(a), "f"(h), "r"(b) : "memory");
        }
    }
    // false: not within `limit` cycles (0: without a look)
    __device__ __forceinline__ bool arrived(int round, long long limit) const {
        const unsigned bar = smem_u32(j->bar + (round & 1)), parity = (unsigned)(round >> 1 & 1);
        const long long t0 = clock64();
        while (limit > 0) {
            unsigned ok;
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
            if (ok) return true;
            if (clock64() - t0 >= limit) break;
        }
        return false;
    }
    // in front of the end.  Nobody leaves while others may write to its shared memory; a thread that gave up does not know of all the maps sent to its CTA, which take
    // a microsecond or so, and stays a good while longer.
    __device__ __forceinline__ void leave(bool gave_up) const {
        cg::this_cluster().sync();
        if (!gave_up) return;
        const long long t0 = clock64();
        while (clock64() - t0 < STAY_CYCLES) {}
    }
};

// Joining the maps of a tile.  Up to 32 channels (CX <= 8) a warp holds several step groups: its threads leave their maps in shared memory, and a lane takes one channel
// and LINKS = 4 of the groups from there; above (a team is one step group) a lane has its own four channels.
template <int CX> struct Lane {
    static constexpr bool ONE = CX <= 8;
    static constexpr int M = ONE ? 1 : N, CH = CX * N, LINKS = 4, SUBS = ONE ? 32 / CX / LINKS : 1;
    static __device__ __forceinline__ int first() { return ONE ? (threadIdx.x & 31) % CH : threadIdx.x % CX * N; }      // channel of the slice
    static __device__ __forceinline__ int sub() { return ONE ? (threadIdx.x & 31) / CH : 0; }
    static __device__ __forceinline__ bool writes() { return ONE ? (threadIdx.x & 31) < CH : true; }
    float v[M];
    __device__ __forceinline__ void fill(float x) {
#pragma unroll
        for (int j = 0; j < M; ++j) v[j] = x;
    }
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
__global__ void __launch_bounds__(THREADS, 2) recur_fwd_k(RecurArgs p, const __grid_constant__ Maps maps, Waits waits, int ranks, int slices) {
    const int R = CLUSTER ? ranks : 1;
    constexpr int S = STEPS_FWD<T>, PARTS = S / STEPS;         // tiles of the backward pass in one of this
    using G = Geo<CX, S>;
    using Rg = Ring<T, ACC, CX, S, 2>;
    extern __shared__ __align__(128) char dyn[];
    __shared__ uint64_t full[Rg::STAGES];
    Rg ring{dyn, full};
    __shared__ __align__(16) float2 tot[2][G::TEAMS][G::CH];
    __shared__ __align__(16) float own[2][Lane<CX>::ONE ? THREADS * N : 1];      // a warp's maps, later the states in front of its step groups
    __shared__ __align__(16) float carried[2][G::CH];
    __shared__ __align__(16) Joined<CLUSTER ? G::CH : 2> joined;
    const Peers<CLUSTER ? G::CH : 2> peers{&joined};
    const int rank = CLUSTER ? (int)(blockIdx.x % R) : 0;
    const long group = blockIdx.x / R, b = group / slices;
    const long c0 = (group - b * slices) * G::CH;
    const int cx = threadIdx.x % CX, tg = threadIdx.x / CX, team = threadIdx.x / G::TEAM;
    const long c = c0 + cx * N;
    const int left = (int)min((long)N, p.C - c);                 // channels of this thread that exist
    const int T_ = (int)p.T, len = p.lengths ? min(max(p.lengths[b], 0), T_) : T_;
    const int tiles = (T_ + G::TILE - 1) / G::TILE, rounds = (tiles + R - 1) / R, stride = R * G::TILE;
    const int saves = (T_ + Geo<CX, STEPS>::TILE - 1) / Geo<CX, STEPS>::TILE;
    int t0 = rank * G::TILE + tg * S, tf = t0;        // this thread's first step: of the round, of the next tile to fetch
    const T* gf[2] = {(const T*)p.z + b * p.z_b + c + t0 * p.z_t, (const T*)p.v + b * p.v_b + c + t0 * p.v_t};
    const long step[2] = {p.z_t, p.v_t}, round_step[2] = {stride * p.z_t, stride * p.v_t};
    T* y = (T*)p.y + b * p.y_b + c + t0 * p.y_t;
    const long y_round = stride * p.y_t;
    const int behind = rounds * stride;                          // the first step that no round looks at
    auto fetch_tile = [&](int stage) {
        if (tf < behind) ring.fetch(stage, maps, c0, tf - tg * S, b, gf, step, left, steps_before<S>(len, tf));
        ring.issued();
        tf += stride; gf[0] += round_step[0]; gf[1] += round_step[1];
    };
    ring.begin();
    for (int s = 0; s < Rg::STAGES - 1; ++s) fetch_tile(s);
    if (CLUSTER) peers.begin();
    const int first = Lane<CX>::first(), mine = (threadIdx.x & ~31) * N;
    Lane<CX> carry;                                              // CLUSTER: the state in front of the round, in every warp
    carry.read(p.state ? p.state + b * p.C : nullptr, c0, p.C);
    if (threadIdx.x < G::CH) carried[0][threadIdx.x] = p.state && c0 + threadIdx.x < p.C ? p.state[b * p.C + c0 + threadIdx.x] : 0.f;
    int stage = 0;
    for (int round = 0; round < rounds; ++round) {
        const int now = round & 1;
        fetch_tile(stage == 0 ? Rg::STAGES - 1 : stage - 1);     // where the tile before was: it has been read
        ring.template arrived<Rg::STAGES - 1>(stage, round, waits.copies);
        // the map of this thread's steps
        const int n = steps_before<S>(len, t0);
        Four a[S], u[S], A, H;
        auto look = [&](auto all) {
#pragma unroll
            for (int i = 0; i < S; ++i) {
                Four z = ring.get(stage, 0, i), v = ring.get(stage, 1, i);
                if (!all.value && i >= n) idle(z, v);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float2 q;
                    gate(z.p[j], a[i].p[j], q);
                    u[i].p[j] = mul(q, v.p[j]);
                    if (i == 0) { A.p[j] = a[0].p[j]; H.p[j] = u[0].p[j]; }
                    else { H.p[j] = fma(a[i].p[j], H.p[j], u[i].p[j]); A.p[j] = mul(A.p[j], a[i].p[j]); }
                }
            }
        };
        if (n == S) look(std::true_type()); else look(std::false_type());
        if (ring.lost >= 0) u[0] = H = {both(NAN), both(NAN)};
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
            if (threadIdx.x < G::CH && ring.lost < 0) {
                float ta = 1.f, th = 0.f;
#pragma unroll
                for (int w = 0; w < G::TEAMS; ++w) { const float2 m = tot[now][w][threadIdx.x]; th = fmaf(m.x, th, m.y); ta *= m.x; }
                peers.send(round, rank, R, ta, th);
            }
            if (ring.lost < 0 && !peers.arrived(round, waits.peers)) ring.lost = round + Rg::STAGES;
            for (int r = 0; r < R; ++r) {
                if (r == rank) in = carry;
                carry.through(&joined.at[now][r][first]);
            }
            if (ring.lost >= 0) { in.fill(NAN); carry.fill(NAN); }        // what stands there is nobody's, or an earlier round's
        } else in.set(&carried[now][first]);
        for (int w = 0; w < team; ++w) in.through(&tot[now][w][first]);
        if (p.saved && team % (G::TEAMS / PARTS) == 0 && Lane<CX>::writes()) {
            const int at = (round * R + rank) * PARTS + team / (G::TEAMS / PARTS);
            if (at < saves) in.write(p.saved + ((long)b * saves + at) * p.C, c0, p.C);
        }
        Four h;
        if constexpr (Lane<CX>::ONE) {
            chain.apply(in.v[0], &own[1][mine]);
            __syncwarp();
            h = load(&own[1][threadIdx.x * N]);
        } else h = {make_float2(in.v[0], in.v[1]), make_float2(in.v[2], in.v[3])};
        if (n == S && left > 0) {
#pragma unroll
            for (int i = 0; i < S; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) h.p[j] = fma(a[i].p[j], h.p[j], u[i].p[j]);
                put<T, ACC>(y + i * p.y_t, h, left, false);
            }
        } else {
            const int out = left > 0 ? steps_before<S>(T_, t0) : 0;
#pragma unroll
            for (int i = 0; i < S; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) h.p[j] = fma(a[i].p[j], h.p[j], u[i].p[j]);
                if (i < out) put<T, ACC>(y + i * p.y_t, i < n ? h : Four{}, left, false);
            }
        }
        if (!CLUSTER && tg == G::TG - 1) *(float4*)&carried[now ^ 1][cx * N] = make_float4(h.p[0].x, h.p[0].y, h.p[1].x, h.p[1].y);
        t0 += stride; y += y_round;
        stage = stage + 1 == Rg::STAGES ? 0 : stage + 1;
    }
    ring.drain(rounds, waits.err);
    if (CLUSTER) peers.leave(ring.lost >= 0);
    else { __syncthreads(); carry.set(&carried[rounds & 1][first]); }
    if (p.state_out && rank == 0 && threadIdx.x < G::TEAM && Lane<CX>::writes()) carry.write(p.state_out + b * p.C, c0, p.C);
}

template <typename T, int ACC, int CX, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 2) recur_bwd_k(RecurArgs p, const __grid_constant__ Maps maps, Waits waits, int ranks, int slices) {
    const int R = CLUSTER ? ranks : 1;
    using G = Geo<CX, STEPS>;
    using Rg = Ring<T, ACC, CX, STEPS, 3>;
    extern __shared__ __align__(128) char dyn[];
    __shared__ uint64_t full[Rg::STAGES];
    Rg ring{dyn, full};
    __shared__ __align__(16) float2 tot_h[2][G::TEAMS][G::CH], tot_g[2][G::TEAMS][G::CH];
    // A warp's maps.  fp32: where its gates were in the tile, which nobody needs any more (a room of their own would leave one CTA to an SM: 8 x 2048 x 1024 78 us instead of 57)
    constexpr bool IN_TILE = Lane<CX>::ONE && sizeof(T) == 4;
    static_assert(!IN_TILE || 3 * sizeof(float) <= STEPS * sizeof(T), "three maps' values a thread and channel lie in its gates' place");
    __shared__ __align__(16) float room[3][Lane<CX>::ONE && !IN_TILE ? THREADS * N : 1];
    __shared__ __align__(16) float carried[2][G::CH];
    __shared__ __align__(16) Joined<CLUSTER ? G::CH : 2> joined;
    const Peers<CLUSTER ? G::CH : 2> peers{&joined};
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
    const T* gf[3] = {(const T*)p.z + b * p.z_b + c + t0 * p.z_t, (const T*)p.v + b * p.v_b + c + t0 * p.v_t, (const T*)p.dy + b * p.dy_b + c + t0 * p.dy_t};
    const long step[3] = {p.z_t, p.v_t, p.dy_t}, round_step[3] = {stride * p.z_t, stride * p.v_t, stride * p.dy_t};
    T* dz = (T*)p.dz + b * p.dz_b + c + t0 * p.dz_t;
    T* dv = (T*)p.dv + b * p.dv_b + c + t0 * p.dv_t;
    const long dz_round = stride * p.dz_t, dv_round = stride * p.dv_t;
    auto fetch_tile = [&](int stage) {
        if (tf >= 0) ring.fetch(stage, maps, c0, tf - tg * STEPS, b, gf, step, left, steps_before<STEPS>(len, tf));
        ring.issued();
        tf -= stride;
#pragma unroll
        for (int q = 0; q < 3; ++q) gf[q] -= round_step[q];
    };
    ring.begin();
    for (int s = 0; s < Rg::STAGES - 1; ++s) fetch_tile(s);
    if (CLUSTER) peers.begin();
    const int first = Lane<CX>::first(), at = (threadIdx.x & 31) * N;
    Lane<CX> carry;
    carry.read(p.dstate_out ? p.dstate_out + b * p.C : nullptr, c0, p.C);
    if (threadIdx.x < G::CH) carried[0][threadIdx.x] = p.dstate_out && c0 + threadIdx.x < p.C ? p.dstate_out[b * p.C + c0 + threadIdx.x] : 0.f;
    int stage = 0;
    for (int round = 0; round < rounds; ++round) {
        const int now = round & 1;
        Lane<CX> in_h, in_g;
        in_h.read(tile < tiles ? p.saved + ((long)b * tiles + tile) * p.C : nullptr, c0, p.C);
        ring.template arrived<Rg::STAGES - 2>(stage, round, waits.copies);
        const int n = steps_before<STEPS>(len, t0);
        Four a[STEPS], q[STEPS], A, H, Q;
        auto look = [&](auto all) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                Four z = ring.get(stage, 0, i), v = ring.get(stage, 1, i), d = ring.get(stage, 2, i);
                if (!all.value && i >= n) { idle(z, v); d = v; }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    gate(z.p[j], a[i].p[j], q[i].p[j]);
                    const float2 u = mul(q[i].p[j], v.p[j]);
                    if (i == 0) { A.p[j] = a[0].p[j]; H.p[j] = u; Q.p[j] = mul(A.p[j], d.p[j]); }
                    else {
                        H.p[j] = fma(a[i].p[j], H.p[j], u);
                        A.p[j] = mul(A.p[j], a[i].p[j]);
                        Q.p[j] = fma(A.p[j], d.p[j], Q.p[j]);    // what dy of this step is in front of the thread's first one
                    }
                }
            }
        };
        if (n == STEPS) look(std::true_type()); else look(std::false_type());
        if (ring.lost >= 0) H = Q = {both(NAN), both(NAN)};
        float* own[3];
#pragma unroll
        for (int k = 0; k < 3; ++k)
            own[k] = IN_TILE ? (float*)(dyn + stage * Rg::STAGE + (threadIdx.x >> 5) * (32 * N * STEPS * (int)sizeof(T))) + k * 32 * N : &room[k][(threadIdx.x & ~31) * N];
        Chain<CX, true> front;                                   // the forward map
        Chain<CX, false> behind;                                 // the backward map
        if constexpr (Lane<CX>::ONE) {
            __syncwarp();
            store(own[0] + at, A); store(own[1] + at, H); store(own[2] + at, Q);
            __syncwarp();
            front.read(own[0], own[1]);
            behind.read(own[0], own[2]);
            if (Lane<CX>::writes()) {
                tot_h[now][team][first] = make_float2(front.ta, front.th);
                tot_g[now][team][first] = make_float2(behind.ta, behind.th);
            }
        } else { store(&tot_h[now][team][first], A, H); store(&tot_g[now][team][first], A, Q); }
        if (IN_TILE && Rg::TMA) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the tile before was written to; a tensor copy is about to
        __syncthreads();
        fetch_tile(stage == 0 ? Rg::STAGES - 1 : stage - 1);     // where the tile before was: it has been read
        if (CLUSTER) {
            if (threadIdx.x < G::CH && ring.lost < 0) {
                float ta = 1.f, tq = 0.f;
#pragma unroll
                for (int w = G::TEAMS - 1; w >= 0; --w) { const float2 m = tot_g[now][w][threadIdx.x]; tq = fmaf(m.x, tq, m.y); ta *= m.x; }
                peers.send(round, rank, R, ta, tq);
            }
            if (ring.lost < 0 && !peers.arrived(round, waits.peers)) ring.lost = round + Rg::STAGES;
            for (int r = R - 1; r >= 0; --r) {
                if (r == rank) in_g = carry;
                carry.through(&joined.at[now][r][first]);
            }
            if (ring.lost >= 0) { in_g.fill(NAN); carry.fill(NAN); }
        } else in_g.set(&carried[now][first]);
        for (int w = 0; w < team; ++w) in_h.through(&tot_h[now][w][first]);
        for (int w = G::TEAMS - 1; w > team; --w) in_g.through(&tot_g[now][w][first]);
        Four g, before[STEPS];
        if constexpr (Lane<CX>::ONE) {
            front.apply(in_h.v[0], own[1]);
            behind.apply(in_g.v[0], own[2]);
            __syncwarp();
            before[0] = load(own[1] + at);
            g = load(own[2] + at);
        } else {
            before[0] = {make_float2(in_h.v[0], in_h.v[1]), make_float2(in_h.v[2], in_h.v[3])};
            g = {make_float2(in_g.v[0], in_g.v[1]), make_float2(in_g.v[2], in_g.v[3])};
        }
        if (ring.lost >= 0) before[0] = g = {both(NAN), both(NAN)};       // the maps say it to the others, this to the thread's own steps
#pragma unroll
        for (int i = 0; i + 1 < STEPS; ++i) {
            const Four v = ring.get(stage, 1, i);
#pragma unroll
            for (int j = 0; j < 2; ++j) before[i + 1].p[j] = fma(a[i].p[j], before[i].p[j], mul(q[i].p[j], v.p[j]));
        }
        // one step back: its gradients, and g in front of it
        auto back = [&](int i, Four& oz, Four& ov) {
            const Four v = ring.get(stage, 1, i), e = ring.get(stage, 2, i);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 d = __fadd2_rn(e.p[j], g.p[j]);
                ov.p[j] = mul(q[i].p[j], d);
                g.p[j] = mul(a[i].p[j], d);
                oz.p[j] = mul(mul(a[i].p[j], ov.p[j]), fma(v.p[j], both(-1.f), before[i].p[j]));
            }
        };
        if (n == STEPS && left > 0) {
#pragma unroll
            for (int i = STEPS - 1; i >= 0; --i) {
                Four oz, ov;
                back(i, oz, ov);
                put<T, ACC>(dz + i * p.dz_t, oz, left, p.accum);
                put<T, ACC>(dv + i * p.dv_t, ov, left, p.accum);
            }
        } else {
            const int out = left > 0 ? steps_before<STEPS>(T_, t0) : 0;
#pragma unroll
            for (int i = STEPS - 1; i >= 0; --i) {
                Four oz{}, ov{};
                if (i < n) back(i, oz, ov);
                if (i < out) {
                    put<T, ACC>(dz + i * p.dz_t, oz, left, p.accum);
                    put<T, ACC>(dv + i * p.dv_t, ov, left, p.accum);
                }
            }
        }
        if (!CLUSTER && tg == 0) *(float4*)&carried[now ^ 1][cx * N] = make_float4(g.p[0].x, g.p[0].y, g.p[1].x, g.p[1].y);
        t0 -= stride; tile -= R; dz -= dz_round; dv -= dv_round;
        stage = stage + 1 == Rg::STAGES ? 0 : stage + 1;
    }
    ring.drain(rounds, waits.err);
    if (CLUSTER) peers.leave(ring.lost >= 0);
    else { __syncthreads(); carry.set(&carried[rounds & 1][first]); }
    if (p.dstate && rank == 0 && threadIdx.x < G::TEAM && Lane<CX>::writes()) carry.write(p.dstate + b * p.C, c0, p.C);
}

// One step from a state to a state, without what a backward pass needs: a thread per channel.  A call for 64 sequences of 1024 channels, in a graph: 3.9 us, 6.3 through the tiles.
template <typename T>
__global__ void __launch_bounds__(128) recur_step_k(RecurArgs p) {
    const long id = (long)blockIdx.x * 128 + threadIdx.x;
    if (id >= p.B * p.C) return;
    const long b = id / p.C, c = id - b * p.C;
    const bool live = !p.lengths || p.lengths[b] > 0;
    float h = p.state ? p.state[id] : 0.f;
    if (live) {
        float2 a, q;
        gate(both(ld((const T*)p.z + b * p.z_b + c)), a, q);
        h = fmaf(a.x, h, q.x * ld((const T*)p.v + b * p.v_b + c));
    }
    st((T*)p.y + b * p.y_b + c, live ? h : 0.f);
    if (p.state_out) p.state_out[id] = h;
}

// How a launch is cut: cx threads along the channels, clusters of r CTAs along the steps.  Both directions use the same cut (the states in front of the tiles
// pass between them), and it depends on the sizes alone.  The least of a model's times, in us, fitted to 60 measured backward passes (1 to 64 sequences of 48 to 60001
// steps, 64 to 2048 channels): a round of a CTA takes 1.5 with an SM to itself and 2.4 beside another, 0.6 more in a cluster and a fifth more with a step group
// per team; a launch 3, with clusters 5; more than two CTAs to an SM come in waves.  Measured, 8 x 2048 x 1024: 39 for (8, 1), 53 for (8, 2) and (4, 1), 109 for (32, 1);
// 1 x 60001 x 512: 109 for (4, 8), 152 for (8, 8), 412 for (4, 1).  (Clusters of 16 do not all fit on the device at once: 146 for (8, 16).)
struct Cut { int cx, r; };
Cut cut(long B, long T, long C) {
    Cut best{64, 1};
    double least = 1e300;
    for (int cx : {64, 32, 8, 4}) {
        const long tiles = (T + THREADS / cx * STEPS - 1) / (THREADS / cx * STEPS), groups = B * ((C + N * cx - 1) / (N * cx));
        for (int r = 1; r <= (cx > 8 ? 1 : MAX_CLUSTER) && (r == 1 || r <= tiles); r *= 2) {
            const double rounds = (double)((tiles + r - 1) / r), w = (double)groups * r / 148;
            double round = 1.5 + 0.9 * std::min(1.0, std::max(0.0, w - 1.0));
            if (cx > 8) round *= 1.2;
            if (r > 1) round += 0.6;
            const double us = (r > 1 ? 5 : 3) + (w <= 2 ? rounds * round : std::ceil(w / 2) * (rounds * round + 1));
            if (us < least - 1e-9) { least = us; best = {cx, r}; }
        }
    }
    return best;
}

// The limits of the waits: two seconds or so, or the environment's FDG_WAIT_CYCLES, "copies" or "copies,peers".
Waits limits(int* err) {
    static const Waits known = [] {
        Waits w{WAIT_CYCLES, WAIT_CYCLES, nullptr};
        if (const char* s = getenv("FDG_WAIT_CYCLES")) {
            char* end;
            const long long a = strtoll(s, &end, 10);
            if (end != s && a >= 0) {
                w.copies = w.peers = a;
                if (*end == ',') { const long long b = strtoll(end + 1, nullptr, 10); if (b >= 0) w.peers = b; }
            }
        }
        return w;
    }();
    return {known.copies, known.peers, err};
}

// false: the tensors cannot be described (they are too far apart)
template <typename T, int CX, int S>
bool make_maps(const RecurArgs& a, bool back, Maps& m) {
    using Rg = Ring<T, 16 / (int)sizeof(T), CX, S, 2>;
    const int dt = sizeof(T) == 2, box = Rg::BOX;
    return tc::make_map_rows(&m.t[0], dt, a.z, a.C, a.T, a.B, a.z_t, a.z_b, Geo<CX, S>::CH, box) && tc::make_map_rows(&m.t[1], dt, a.v, a.C, a.T, a.B, a.v_t, a.v_b, Geo<CX, S>::CH, box) &&
           (!back || tc::make_map_rows(&m.t[2], dt, a.dy, a.C, a.T, a.B, a.dy_t, a.dy_b, Geo<CX, S>::CH, box));
}
template <typename T, int ACC, int CX, bool BACK, bool CLUSTER>
cudaError_t launch(const RecurArgs& a, int R, int* err, cudaStream_t s) {
    constexpr int S = BACK ? STEPS : STEPS_FWD<T>;
    using Rg = Ring<T, ACC, CX, S, BACK ? 3 : 2>;
    Maps maps{};
    if constexpr (Rg::TMA) if (!make_maps<T, CX, S>(a, BACK, maps)) return launch<T, (sizeof(T) == 2 ? 2 : 1), CX, BACK, CLUSTER>(a, R, err, s);
    static OncePerDevice once;
    const auto k = BACK ? recur_bwd_k<T, ACC, CX, CLUSTER> : recur_fwd_k<T, ACC, CX, CLUSTER>;
    const cudaError_t e = allow_smem(once, (const void*)k, Rg::BYTES);
    if (e != cudaSuccess) return e;
    const int slices = (int)((a.C + Geo<CX, S>::CH - 1) / Geo<CX, S>::CH);
    return klaunch_cluster(k, (unsigned)(a.B * slices * R), THREADS, Rg::BYTES, s, CLUSTER ? R : 0, a, maps, limits(err), R, slices);
}
template <typename T, int ACC, bool BACK>
cudaError_t pick(const RecurArgs& a, int* err, cudaStream_t s) {
    const Cut k = cut(a.B, a.T, a.C);
    switch (k.cx) {
        case 4: return k.r > 1 ? launch<T, ACC, 4, BACK, true>(a, k.r, err, s) : launch<T, ACC, 4, BACK, false>(a, 1, err, s);
        case 8: return k.r > 1 ? launch<T, ACC, 8, BACK, true>(a, k.r, err, s) : launch<T, ACC, 8, BACK, false>(a, 1, err, s);
        case 32: return launch<T, ACC, 32, BACK, false>(a, 1, err, s);
        default: return launch<T, ACC, 64, BACK, false>(a, 1, err, s);
    }
}
// elements that may be moved at once: every row of every tensor starts on that many, and holds a multiple of them
template <bool BACK>
cudaError_t run(int dt, const RecurArgs& a, int* err, cudaStream_t s) {
    const size_t z = dt ? 2 : 4;
    uint64_t m = (uint64_t)a.C * z | (uintptr_t)a.z | (uintptr_t)a.v | (uint64_t)(a.z_b | a.z_t | a.v_b | a.v_t) * z;
    if (BACK) m |= (uintptr_t)a.dy | (uintptr_t)a.dz | (uintptr_t)a.dv | (uint64_t)(a.dy_b | a.dy_t | a.dz_b | a.dz_t | a.dv_b | a.dv_t) * z;
    else m |= (uintptr_t)a.y | (uint64_t)(a.y_b | a.y_t) * z;
    if (dt) return m % 16 == 0 ? pick<bf16, 8, BACK>(a, err, s) : m % 4 == 0 ? pick<bf16, 2, BACK>(a, err, s) : pick<bf16, 1, BACK>(a, err, s);
    return m % 16 == 0 ? pick<float, 4, BACK>(a, err, s) : pick<float, 1, BACK>(a, err, s);
}

}  // namespace

size_t recur_saved_bytes(int, long B, long T, long C) {
    const int tile = THREADS / cut(B, T, C).cx * STEPS;
    return (size_t)B * ((T + tile - 1) / tile) * C * sizeof(float);
}

cudaError_t recur_forward(int dt, const RecurArgs& a, int* err, cudaStream_t s) {
    if (a.B * a.C == 0) return cudaSuccess;
    Scope sc(KC_RECUR_FWD, 8.0 * a.B * a.T * a.C, 3.0 * a.B * a.T * a.C * (dt ? 2 : 4), s);
    if (a.T == 1 && !a.saved) {
        const unsigned blocks = (unsigned)((a.B * a.C + 127) / 128);
        return dt ? klaunch(recur_step_k<bf16>, blocks, 128, 0, s, a) : klaunch(recur_step_k<float>, blocks, 128, 0, s, a);
    }
    return run<false>(dt, a, err, s);
}

cudaError_t recur_backward(int dt, const RecurArgs& a, int* err, cudaStream_t s) {
    if (a.B * a.C == 0) return cudaSuccess;
    Scope sc(KC_RECUR_BWD, 16.0 * a.B * a.T * a.C, 5.0 * a.B * a.T * a.C * (dt ? 2 : 4), s);
    return run<true>(dt, a, err, s);
}

}  // namespace fdg
