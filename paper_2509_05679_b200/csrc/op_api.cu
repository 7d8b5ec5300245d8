// C entry points of the operators on a caller's tensors (include/fdg.h): arguments are checked here, on the host, so that no kernel meets an address or a
// size it cannot take; the kernels are those of embed.cu, recur.cu and distill.cu, which the step executor launches too.
#include "../../include/fdg.h"
#include "launch.h"
#include "seqops.h"

#include <cstdarg>
#include <cstdio>
#include <string>

using namespace fdg;

namespace {

thread_local char t_error[256];

fdg_status fail(fdg_status st, const char* fmt, ...) {
    va_list ap; va_start(ap, fmt); vsnprintf(t_error, sizeof t_error, fmt, ap); va_end(ap);
    return st;
}

constexpr int64_t MOST = INT64_C(1) << 31;           // of every extent: their products then stay inside 64 bits with room for strides

// The current device, which has to be an sm_100 one.  Its architecture is looked up once.
fdg_status device(const char* fn, int* dev) {
    static OncePerDevice known;
    if (cudaGetDevice(dev) != cudaSuccess) { cudaGetLastError(); return fail(FDG_ERR_ARCH, "%s: no CUDA device", fn); }
    if (known.done(*dev)) return FDG_OK;
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev) != cudaSuccess) { cudaGetLastError(); return fail(FDG_ERR_ARCH, "%s: no CUDA device", fn); }
    if (major != 10) return fail(FDG_ERR_ARCH, "%s: this library is built for sm_100a only", fn);
    known.set(*dev);
    return FDG_OK;
}

// Whether kernels on device `dev` can use p: memory of that device (or managed), on a multiple of `align` bytes.
fdg_status usable(const char* fn, const char* name, const void* p, size_t align, int dev) {
    if (!p) return fail(FDG_ERR_INVALID_ARG, "%s: %s is NULL", fn, name);
    if ((uintptr_t)p % align) return fail(FDG_ERR_INVALID_ARG, "%s: %s is not aligned to %zu bytes", fn, name, align);
    cudaPointerAttributes a{};
    const cudaError_t e = cudaPointerGetAttributes(&a, p);
    if (e != cudaSuccess) cudaGetLastError();
    if (e != cudaSuccess || !(a.type == cudaMemoryTypeManaged || (a.type == cudaMemoryTypeDevice && a.device == dev)))
        return fail(FDG_ERR_INVALID_ARG, "%s: %s is not memory of the current device", fn, name);
    return FDG_OK;
}

#define CHECK(call) do { const fdg_status s_ = (call); if (s_ != FDG_OK) return s_; } while (0)

fdg_status enqueued(const char* fn, cudaError_t e) {
    if (e == cudaSuccess) return FDG_OK;
    cudaGetLastError();
    return fail(FDG_ERR_CUDA, "%s: %s", fn, cudaGetErrorString(e));
}

size_t esize(int32_t dtype) { return dtype ? 2 : 4; }
bool bad_dtype(int32_t d) { return d != 0 && d != 1; }
bool bad_extent(int64_t v) { return v < 0 || v >= MOST; }

fdg_status embedding_sizes(const char* fn, int64_t n, int64_t vocab, int64_t channels) {
    if (n < 0 || n > (1 << 30) || vocab < 1 || vocab >= MOST - 1 || channels < 1 || channels > (1 << 20)) return fail(FDG_ERR_INVALID_ARG, "%s: n must be 0..2^30, vocab 1..2^31-2, channels 1..2^20", fn);
    return FDG_OK;
}

fdg_status recurrence_sizes(const char* fn, const fdg_recurrence* s) {
    if (!s) return fail(FDG_ERR_INVALID_ARG, "%s: shape is NULL", fn);
    if (bad_dtype(s->dtype)) return fail(FDG_ERR_INVALID_ARG, "%s: dtype must be 0 (fp32) or 1 (bf16)", fn);
    if (bad_extent(s->batch) || s->steps < 0 || s->steps > (1 << 30) || s->channels < 1 || s->channels > (1 << 20)) return fail(FDG_ERR_INVALID_ARG, "%s: batch must be 0..2^31-1, steps 0..2^30, channels 1..2^20", fn);
    if ((__int128)s->batch * s->steps * s->channels >= (__int128)1 << 46) return fail(FDG_ERR_INVALID_ARG, "%s: the tensors are too large", fn);
    return FDG_OK;
}
// strides that keep the rows of a tensor inside 64 bits; an output's rows must not meet
fdg_status strides(const char* fn, const char* name, const fdg_recurrence* s, int64_t b, int64_t t, bool output) {
    if (b < 0 || t < 0 || b >= INT64_C(1) << 46 || t >= INT64_C(1) << 46 || (__int128)b * s->batch + (__int128)t * s->steps >= (__int128)1 << 48)
        return fail(FDG_ERR_INVALID_ARG, "%s: strides of %s out of range", fn, name);
    if (!output) return FDG_OK;
    const bool many_b = s->batch > 1, many_t = s->steps > 1;
    const bool nested = (!many_t || (t >= s->channels && (!many_b || (__int128)b >= (__int128)t * (s->steps - 1) + s->channels))) && (!many_b || b >= s->channels);
    const bool time_major = (!many_b || (b >= s->channels && (!many_t || (__int128)t >= (__int128)b * (s->batch - 1) + s->channels))) && (!many_t || t >= s->channels);
    if (!nested && !time_major) return fail(FDG_ERR_INVALID_ARG, "%s: rows of %s overlap", fn, name);
    return FDG_OK;
}

}  // namespace

extern "C" {

const char* fdg_op_last_error(void) { return t_error; }

fdg_status fdg_embedding_forward(const int32_t* tokens, int64_t n, const void* table, int32_t dtype, int64_t vocab, int64_t channels, float scale, void* out,
                                 int64_t out_stride, void* stream) {
    const char* const fn = "fdg_embedding_forward";
    CHECK(embedding_sizes(fn, n, vocab, channels));
    if (bad_dtype(dtype)) return fail(FDG_ERR_INVALID_ARG, "%s: dtype must be 0 (fp32) or 1 (bf16)", fn);
    if (out_stride < channels || out_stride >= MOST) return fail(FDG_ERR_INVALID_ARG, "%s: out_stride must be at least channels", fn);
    int dev;
    CHECK(device(fn, &dev));
    if (n == 0) return FDG_OK;
    CHECK(usable(fn, "tokens", tokens, 4, dev));
    CHECK(usable(fn, "table", table, esize(dtype), dev));
    CHECK(usable(fn, "out", out, esize(dtype), dev));
    return enqueued(fn, embed_forward(dtype, tokens, n, table, vocab, channels, scale, out, out_stride, (cudaStream_t)stream));
}

fdg_status fdg_embedding_workspace(int64_t n, int64_t vocab, int64_t channels, size_t* bytes) {
    const char* const fn = "fdg_embedding_workspace";
    CHECK(embedding_sizes(fn, n, vocab, channels));
    if (!bytes) return fail(FDG_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    *bytes = embed_workspace_bytes(n, vocab, channels);
    return FDG_OK;
}

fdg_status fdg_embedding_backward(const int32_t* tokens, int64_t n, const void* dy, int32_t dtype, int64_t dy_stride, int64_t vocab, int64_t channels, float scale,
                                  int32_t accumulate, float* dtable, void* workspace, size_t workspace_bytes, void* stream) {
    const char* const fn = "fdg_embedding_backward";
    CHECK(embedding_sizes(fn, n, vocab, channels));
    if (bad_dtype(dtype)) return fail(FDG_ERR_INVALID_ARG, "%s: dtype must be 0 (fp32) or 1 (bf16)", fn);
    if (dy_stride < 0 || dy_stride >= MOST) return fail(FDG_ERR_INVALID_ARG, "%s: dy_stride out of range", fn);
    const size_t need = embed_workspace_bytes(n, vocab, channels);
    if (workspace_bytes < need) return fail(FDG_ERR_INVALID_ARG, "%s: a workspace of %zu bytes is needed, %zu were given", fn, need, workspace_bytes);
    int dev;
    CHECK(device(fn, &dev));
    if (n > 0) {
        CHECK(usable(fn, "tokens", tokens, 4, dev));
        CHECK(usable(fn, "dy", dy, esize(dtype), dev));
    }
    CHECK(usable(fn, "dtable", dtable, 4, dev));
    if (need) CHECK(usable(fn, "workspace", workspace, 256, dev));
    return enqueued(fn, embed_backward(dtype, tokens, n, dy, dy_stride, vocab, channels, scale, accumulate != 0, dtable, workspace, (cudaStream_t)stream));
}

fdg_status fdg_recurrence_saved(const fdg_recurrence* s, size_t* bytes) {
    const char* const fn = "fdg_recurrence_saved";
    CHECK(recurrence_sizes(fn, s));
    if (!bytes) return fail(FDG_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    *bytes = recur_saved_bytes(s->dtype, s->batch, s->steps, s->channels);
    return FDG_OK;
}

fdg_status fdg_recurrence_forward(const fdg_recurrence* s, const void* gate, const void* value, const int32_t* lengths, const float* state_in, void* y, float* state_out,
                                  void* saved, void* stream) {
    const char* const fn = "fdg_recurrence_forward";
    CHECK(recurrence_sizes(fn, s));
    CHECK(strides(fn, "gate", s, s->gate_batch, s->gate_step, false));
    CHECK(strides(fn, "value", s, s->value_batch, s->value_step, false));
    CHECK(strides(fn, "y", s, s->y_batch, s->y_step, true));
    int dev;
    CHECK(device(fn, &dev));
    if (s->batch == 0) return FDG_OK;
    if (s->steps > 0) {
        CHECK(usable(fn, "gate", gate, esize(s->dtype), dev));
        CHECK(usable(fn, "value", value, esize(s->dtype), dev));
        CHECK(usable(fn, "y", y, esize(s->dtype), dev));
        if (saved) CHECK(usable(fn, "saved", saved, 16, dev));
    }
    if (lengths) CHECK(usable(fn, "lengths", lengths, 4, dev));
    if (state_in) CHECK(usable(fn, "state_in", state_in, 4, dev));
    if (state_out) CHECK(usable(fn, "state_out", state_out, 4, dev));
    RecurArgs a{};
    a.B = s->batch; a.T = s->steps; a.C = s->channels;
    a.z = gate; a.v = value; a.z_b = s->gate_batch; a.z_t = s->gate_step; a.v_b = s->value_batch; a.v_t = s->value_step;
    a.lengths = lengths; a.state = state_in; a.y = y; a.y_b = s->y_batch; a.y_t = s->y_step; a.state_out = state_out; a.saved = (float*)saved;
    return enqueued(fn, recur_forward(s->dtype, a, nullptr, (cudaStream_t)stream));
}

fdg_status fdg_recurrence_backward(const fdg_recurrence* s, const void* gate, const void* value, const int32_t* lengths, const void* saved, const void* dy,
                                   const float* dstate_out, void* dgate, void* dvalue, float* dstate_in, void* stream) {
    const char* const fn = "fdg_recurrence_backward";
    CHECK(recurrence_sizes(fn, s));
    CHECK(strides(fn, "gate", s, s->gate_batch, s->gate_step, false));
    CHECK(strides(fn, "value", s, s->value_batch, s->value_step, false));
    CHECK(strides(fn, "dy", s, s->dy_batch, s->dy_step, false));
    CHECK(strides(fn, "dgate", s, s->dgate_batch, s->dgate_step, true));
    CHECK(strides(fn, "dvalue", s, s->dvalue_batch, s->dvalue_step, true));
    int dev;
    CHECK(device(fn, &dev));
    if (s->batch == 0) return FDG_OK;
    if (s->steps > 0) {
        CHECK(usable(fn, "gate", gate, esize(s->dtype), dev));
        CHECK(usable(fn, "value", value, esize(s->dtype), dev));
        CHECK(usable(fn, "saved", saved, 16, dev));
        CHECK(usable(fn, "dy", dy, esize(s->dtype), dev));
        CHECK(usable(fn, "dgate", dgate, esize(s->dtype), dev));
        CHECK(usable(fn, "dvalue", dvalue, esize(s->dtype), dev));
    }
    if (lengths) CHECK(usable(fn, "lengths", lengths, 4, dev));
    if (dstate_out) CHECK(usable(fn, "dstate_out", dstate_out, 4, dev));
    if (dstate_in) CHECK(usable(fn, "dstate_in", dstate_in, 4, dev));
    RecurArgs a{};
    a.B = s->batch; a.T = s->steps; a.C = s->channels;
    a.z = gate; a.v = value; a.z_b = s->gate_batch; a.z_t = s->gate_step; a.v_b = s->value_batch; a.v_t = s->value_step;
    a.lengths = lengths; a.saved = (float*)saved;
    a.dy = dy; a.dy_b = s->dy_batch; a.dy_t = s->dy_step; a.dstate_out = dstate_out;
    a.dz = dgate; a.dz_b = s->dgate_batch; a.dz_t = s->dgate_step; a.dv = dvalue; a.dv_b = s->dvalue_batch; a.dv_t = s->dvalue_step; a.dstate = dstate_in;
    return enqueued(fn, recur_backward(s->dtype, a, nullptr, (cudaStream_t)stream));
}

fdg_status fdg_distill_loss(const fdg_distill* d, const void* logits, const int32_t* labels, const int32_t* ids, const float* teacher, float* loss, void* dlogits,
                            void* stream) {
    const char* const fn = "fdg_distill_loss";
    if (!d) return fail(FDG_ERR_INVALID_ARG, "%s: d is NULL", fn);
    if (bad_dtype(d->logits_dtype) || (dlogits && bad_dtype(d->dlogits_dtype))) return fail(FDG_ERR_INVALID_ARG, "%s: dtypes must be 0 (fp32) or 1 (bf16)", fn);
    if (dlogits && d->logits_dtype == 1 && d->dlogits_dtype == 0) return fail(FDG_ERR_UNSUPPORTED, "%s: bf16 logits with fp32 dlogits", fn);
    if (bad_extent(d->rows)) return fail(FDG_ERR_INVALID_ARG, "%s: rows must be 0..2^31-1", fn);
    if (d->vocab < 1 || d->vocab > DISTILL_MAX_VOCAB) return fail(FDG_ERR_UNSUPPORTED, "%s: vocab must be 1..%ld", fn, DISTILL_MAX_VOCAB);
    if (d->top < 0 || d->top > DISTILL_MAX_TOP) return fail(FDG_ERR_UNSUPPORTED, "%s: top must be 0..%d", fn, DISTILL_MAX_TOP);
    if (d->logits_stride < 0 || d->logits_stride >= MOST || (dlogits && (d->dlogits_stride < d->vocab || d->dlogits_stride >= MOST)))
        return fail(FDG_ERR_INVALID_ARG, "%s: dlogits_stride must be at least vocab, strides below 2^31", fn);
    if (!(d->temperature > 0.f) || !(d->temperature <= 1e6f) || !(d->temperature >= 1e-6f)) return fail(FDG_ERR_INVALID_ARG, "%s: temperature must be 1e-6..1e6", fn);
    if (!(d->weight >= 0.f && d->weight <= 1.f)) return fail(FDG_ERR_INVALID_ARG, "%s: weight must be 0..1", fn);
    if (!labels && d->weight < 1.f) return fail(FDG_ERR_INVALID_ARG, "%s: labels may be NULL only with weight 1", fn);
    if (dlogits && dlogits == logits && (d->dlogits_dtype != d->logits_dtype || d->dlogits_stride != d->logits_stride))
        return fail(FDG_ERR_INVALID_ARG, "%s: dlogits may be logits only with the same type and stride", fn);
    int dev;
    CHECK(device(fn, &dev));
    if (d->rows == 0) return FDG_OK;
    CHECK(usable(fn, "logits", logits, esize(d->logits_dtype), dev));
    if (labels) CHECK(usable(fn, "labels", labels, 4, dev));
    if (d->weight > 0.f && d->top > 0) {
        CHECK(usable(fn, "ids", ids, 4, dev));
        CHECK(usable(fn, "teacher", teacher, 4, dev));
    }
    CHECK(usable(fn, "loss", loss, 4, dev));
    if (dlogits) CHECK(usable(fn, "dlogits", dlogits, esize(d->dlogits_dtype), dev));
    DistillArgs a{};
    a.M = d->rows; a.V = d->vocab; a.k = d->top;
    a.logits = logits; a.logits_stride = d->logits_stride; a.labels = labels; a.ids = ids; a.teacher = teacher;
    a.tau = d->temperature; a.weight = d->weight; a.scale = d->scale; a.loss = loss; a.grad = dlogits; a.grad_stride = d->dlogits_stride;
    return enqueued(fn, distill(d->logits_dtype, dlogits ? d->dlogits_dtype : d->logits_dtype, a, (cudaStream_t)stream));
}

}  // extern "C"
