// Operators on token sequences: embedding lookup, gated linear recurrence, distillation loss.  Launch interface shared by the C entry points on a
// caller's tensors (op_api.cu) and the step executor (fdg_api.cu).  Device pointers, `dt` 0: fp32, 1: bf16; sizes are checked by the callers.
// Every function returns the first error of its launches; the runtime keeps it too, which is where the step executor asks.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace fdg {

// ---- embedding (embed.cu): y[i] = scale * table[tokens[i]], rows of zeros for ids outside 0..vocab-1
cudaError_t embed_forward(int dt, const int32_t* tokens, long n, const void* table, long vocab, long C, float scale, void* y, long y_stride, cudaStream_t s);
// dtable[v] (+)= scale * sum over i with tokens[i] = v of dy[i]; not accum: every row is written.  The order of a sum depends on the sizes alone.
size_t embed_workspace_bytes(long n, long vocab, long C);
cudaError_t embed_backward(int dt, const int32_t* tokens, long n, const void* dy, long dy_stride, long vocab, long C, float scale, bool accum, float* dtable, void* ws,
                           cudaStream_t s);

// ---- gated linear recurrence (recur.cu): a = sigmoid(z), h_t = a h_{t-1} + (1 - a) v_t, y_t = h_t
struct RecurArgs {
    long B, T, C;
    const void *z, *v;                       // element strides between sequences and between steps; channels are contiguous
    long z_b, z_t, v_b, v_t;
    const int32_t* lengths;                  // steps of every sequence that count, or nullptr: all
    const float* state;                      // h_0 [B][C], or nullptr: zeros
    // forward
    void* y; long y_b, y_t;
    float* state_out;                        // h after the last step that counts, or nullptr
    float* saved;                            // recur_saved_bytes for the backward pass, or nullptr
    // backward (saved is read)
    const void* dy; long dy_b, dy_t;
    const float* dstate_out;                 // gradient of state_out, or nullptr: zeros
    void *dz, *dv; long dz_b, dz_t, dv_b, dv_t;
    float* dstate;                           // gradient of h_0, or nullptr: not needed
    int accum;                               // dz, dv are added to
};
size_t recur_saved_bytes(int dt, long B, long T, long C);
// err: device word that a kernel sets (from 0) when a wait of its gave up, or nullptr
cudaError_t recur_forward(int dt, const RecurArgs& a, int* err, cudaStream_t s);
cudaError_t recur_backward(int dt, const RecurArgs& a, int* err, cudaStream_t s);

// ---- distillation loss (distill.cu): see fdg_distill_loss
struct DistillArgs {
    long M, V; int k;
    const void* logits; long logits_stride;
    const int32_t* labels;                   // or nullptr: every row counts, weight must be 1
    const int32_t* ids; const float* teacher;
    float tau, weight, scale;
    float* loss;                             // [M]
    void* grad; long grad_stride;            // or nullptr: the loss alone
};
constexpr int DISTILL_MAX_TOP = 1024;
constexpr long DISTILL_MAX_VOCAB = 1l << 18;
cudaError_t distill(int dt_logits, int dt_grad, const DistillArgs& a, cudaStream_t s);

}  // namespace fdg
