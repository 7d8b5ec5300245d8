// Embedding lookup with scaling, y[i] = scale * table[tokens[i]], and the gradient of its table, dtable[v] = scale * sum of the dy rows whose token is v.
// Both move rows of C values and do next to nothing with them: the bound is HBM (lookup: rows read and written; gradient: dy read, the table's
// gradient written, zeros included).
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

template <typename T>
__global__ void embed_fwd_k(const int32_t* __restrict__ tokens, long n, const T* __restrict__ table, long vocab, long C, float scale, T* __restrict__ y, long ys) {
    const long total = n * C;
    for (long e = (long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += (long)gridDim.x * blockDim.x) {
        const long i = e / C, c = e - i * C;
        const long tok = tokens[i];
        st(y + i * ys + c, tok >= 0 && tok < vocab ? ld(table + tok * C + c) * scale : 0.f);
    }
}

__global__ void embed_zero_k(float* __restrict__ dtable, long total) {
    for (long e = (long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += (long)gridDim.x * blockDim.x) dtable[e] = 0.f;
}

// A CTA per position and 256 channels: the first position of a token adds up all positions of it, in order.
template <typename T>
__global__ void embed_grad_scan_k(const int32_t* __restrict__ tokens, long n, const T* __restrict__ dy, long dys, long vocab, long C, float scale, int accum,
                                  float* __restrict__ dtable) {
    const long i = blockIdx.x, c = (long)blockIdx.y * 256 + threadIdx.x;
    const int tok = tokens[i];
    if (tok < 0 || tok >= vocab) return;
    int seen = 0;
    for (long j0 = 0; j0 < i; j0 += 256) {
        const long j = j0 + threadIdx.x;
        if (__syncthreads_or(j < i && tokens[j] == tok)) { seen = 1; break; }
    }
    if (seen) return;
    __shared__ int hits[256], counts[8];
    float sum = 0.f;
    for (long j0 = i; j0 < n; j0 += 256) {
        const long j = j0 + threadIdx.x;
        const bool hit = j < n && tokens[j] == tok;
        const unsigned mask = __ballot_sync(~0u, hit);
        const int w = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0) counts[w] = __popc(mask);
        __syncthreads();
        int at = __popc(mask & ((1u << (threadIdx.x & 31)) - 1)), total = 0;
        for (int q = 0; q < 8; ++q) { if (q < w) at += counts[q]; total += counts[q]; }
        if (hit) hits[at] = (int)(j - j0);
        __syncthreads();
        if (c < C) for (int q = 0; q < total; ++q) sum += ld(dy + (j0 + hits[q]) * dys + c);
        __syncthreads();
    }
    if (c < C) { float* const d = dtable + (long)tok * C + c; *d = accum ? *d + sum * scale : sum * scale; }
}

template <typename T>
cudaError_t forward_t(const int32_t* tokens, long n, const void* table, long vocab, long C, float scale, void* y, long ys, cudaStream_t s) {
    const long blocks = (n * C + 255) / 256;
    return klaunch(embed_fwd_k<T>, (unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s, tokens, n, (const T*)table, vocab, C, scale, (T*)y, ys);
}

template <typename T>
cudaError_t backward_t(const int32_t* tokens, long n, const void* dy, long dys, long vocab, long C, float scale, bool accum, float* dtable, cudaStream_t s) {
    if (!accum) {
        const long blocks = (vocab * C + 255) / 256;
        const cudaError_t e = klaunch(embed_zero_k, (unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s, dtable, vocab * C);
        if (e != cudaSuccess || n == 0) return e;
    }
    return klaunch(embed_grad_scan_k<T>, dim3((unsigned)n, (unsigned)((C + 255) / 256)), 256, 0, s, tokens, n, (const T*)dy, dys, vocab, C, scale, (int)accum, dtable);
}

}  // namespace

cudaError_t embed_forward(int dt, const int32_t* tokens, long n, const void* table, long vocab, long C, float scale, void* y, long y_stride, cudaStream_t s) {
    if (n == 0) return cudaSuccess;
    Scope sc(KC_EMBED_FWD, (double)n * C, (double)n * (4 + 2.0 * C * (dt ? 2 : 4)), s);
    return dt ? forward_t<bf16>(tokens, n, table, vocab, C, scale, y, y_stride, s) : forward_t<float>(tokens, n, table, vocab, C, scale, y, y_stride, s);
}

size_t embed_workspace_bytes(long, long, long) { return 0; }

cudaError_t embed_backward(int dt, const int32_t* tokens, long n, const void* dy, long dy_stride, long vocab, long C, float scale, bool accum, float* dtable, void*,
                           cudaStream_t s) {
    if (n == 0 && accum) return cudaSuccess;
    Scope sc(KC_EMBED_GRAD, 2.0 * n * C, (double)n * (4 + C * (dt ? 2.0 : 4.0)) + (accum ? 0.0 : 4.0 * vocab * C), s);
    return dt ? backward_t<bf16>(tokens, n, dy, dy_stride, vocab, C, scale, accum, dtable, s) : backward_t<float>(tokens, n, dy, dy_stride, vocab, C, scale, accum, dtable, s);
}

}  // namespace fdg
