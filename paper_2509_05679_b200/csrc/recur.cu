// Gated linear recurrence, per sequence and channel:  a = sigmoid(z),  h_t = a_t h_{t-1} + (1 - a_t) v_t,  y_t = h_t.
// Backward, with d_t = dy_t + a_{t+1} d_{t+1}:  dv_t = (1 - a_t) d_t,  dz_t = a_t (1 - a_t) d_t (h_{t-1} - v_t),  dh_0 = a_1 d_1.
// States are held in 32 bits.  The backward pass computes h again, in 32 bits, from the states that the forward pass leaves at every TILE-th step: y
// rounded to bf16 would put 2^-9 of h into dz, and the states are 1 / TILE of the bytes.
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

constexpr int TILE = 32;

// a = sigmoid(z) and b = 1 - a = sigmoid(-z), each to a few units of its own last place
__device__ __forceinline__ void gate(float z, float& a, float& b) {
    const float e = expf(-fabsf(z)), r = 1.f / (1.f + e);
    a = z >= 0.f ? r : e * r;
    b = z >= 0.f ? e * r : r;
}

template <typename T>
__global__ void recur_fwd_k(RecurArgs p) {
    const long id = (long)blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= p.B * p.C) return;
    const long b = id / p.C, c = id - b * p.C;
    const T* z = (const T*)p.z + b * p.z_b + c;
    const T* v = (const T*)p.v + b * p.v_b + c;
    T* y = (T*)p.y + b * p.y_b + c;
    const long len = p.lengths ? min((long)max(p.lengths[b], 0), p.T) : p.T, tiles = (p.T + TILE - 1) / TILE;
    float h = p.state ? p.state[id] : 0.f;
    for (long t = 0; t < p.T; ++t) {
        if (p.saved && t % TILE == 0) p.saved[(b * tiles + t / TILE) * p.C + c] = h;
        if (t >= len) { st(y + t * p.y_t, 0.f); continue; }
        float a, g;
        gate(ld(z + t * p.z_t), a, g);
        h = a * h + g * ld(v + t * p.v_t);
        st(y + t * p.y_t, h);
    }
    if (p.state_out) p.state_out[id] = h;
}

template <typename T>
__global__ void recur_bwd_k(RecurArgs p) {
    const long id = (long)blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= p.B * p.C) return;
    const long b = id / p.C, c = id - b * p.C;
    const T* z = (const T*)p.z + b * p.z_b + c;
    const T* v = (const T*)p.v + b * p.v_b + c;
    const T* dy = (const T*)p.dy + b * p.dy_b + c;
    T* dz = (T*)p.dz + b * p.dz_b + c;
    T* dv = (T*)p.dv + b * p.dv_b + c;
    const long len = p.lengths ? min((long)max(p.lengths[b], 0), p.T) : p.T, tiles = (p.T + TILE - 1) / TILE;
    float g = p.dstate_out ? p.dstate_out[id] : 0.f, before[TILE];       // a_t d_t of the step behind
    for (long tile = tiles - 1; tile >= 0; --tile) {
        float h = p.saved[(b * tiles + tile) * p.C + c];
        for (int i = 0; i < TILE; ++i) {
            const long t = tile * TILE + i;
            before[i] = h;
            if (t >= len) continue;
            float a, q;
            gate(ld(z + t * p.z_t), a, q);
            h = a * h + q * ld(v + t * p.v_t);
        }
        for (int i = TILE - 1; i >= 0; --i) {
            const long t = tile * TILE + i;
            if (t >= p.T) continue;
            float rz = 0.f, rv = 0.f;
            if (t < len) {
                float a, q;
                gate(ld(z + t * p.z_t), a, q);
                const float d = ld(dy + t * p.dy_t) + g;
                rv = q * d;
                rz = a * rv * (before[i] - ld(v + t * p.v_t));
                g = a * d;
            }
            if (p.accum) { rz += ld(dz + t * p.dz_t); rv += ld(dv + t * p.dv_t); }
            st(dz + t * p.dz_t, rz);
            st(dv + t * p.dv_t, rv);
        }
    }
    if (p.dstate) p.dstate[id] = g;
}

}  // namespace

size_t recur_saved_bytes(int, long B, long T, long C) { return (size_t)B * ((T + TILE - 1) / TILE) * C * sizeof(float); }

cudaError_t recur_forward(int dt, const RecurArgs& a, cudaStream_t s) {
    if (a.B * a.C == 0) return cudaSuccess;
    Scope sc(KC_RECUR_FWD, 8.0 * a.B * a.T * a.C, 3.0 * a.B * a.T * a.C * (dt ? 2 : 4), s);
    const unsigned blocks = (unsigned)((a.B * a.C + 127) / 128);
    return dt ? klaunch(recur_fwd_k<bf16>, blocks, 128, 0, s, a) : klaunch(recur_fwd_k<float>, blocks, 128, 0, s, a);
}

cudaError_t recur_backward(int dt, const RecurArgs& a, cudaStream_t s) {
    if (a.B * a.C == 0) return cudaSuccess;
    Scope sc(KC_RECUR_BWD, 16.0 * a.B * a.T * a.C, 5.0 * a.B * a.T * a.C * (dt ? 2 : 4), s);
    const unsigned blocks = (unsigned)((a.B * a.C + 127) / 128);
    return dt ? klaunch(recur_bwd_k<bf16>, blocks, 128, 0, s, a) : klaunch(recur_bwd_k<float>, blocks, 128, 0, s, a);
}

}  // namespace fdg
