// Handle of the operators beside the cached table.
#include "dense_device.h"

#include <algorithm>
#include <new>

namespace fc {

int dense_capturing(fc_dense* d, bool* now) {
    *now = false;
    if (!d->stream) return FC_OK;                // the default stream cannot be
    hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
    FC_HIP(hipStreamIsCapturing(d->stream, &s));
    *now = s != hipStreamCaptureStatusNone;
    d->captured |= *now;
    return FC_OK;
}

// A buffer that a larger one replaces: given back (the device is idle), or kept.
static int dense_replace(fc_dense* d, void* p) {
    if (!p) return FC_OK;
    if (!d->captured) { FC_HIP(hipFree(p)); return FC_OK; }
    auto* k = new (std::nothrow) fc_dense::Kept{p, d->kept};
    if (!k) return FC_ERR_OOM_PINNED;            // host memory
    d->kept = k;
    return FC_OK;
}

// Growth is rare and waits for the whole device: kernels of earlier calls may still use what is given back.
int dense_work(fc_dense* d, size_t bytes) {
    bool now;
    FC_TRY(dense_capturing(d, &now));
    if (bytes <= d->work_cap) return FC_OK;
    if (now) return FC_ERR_HIP;                  // nothing can be allocated: dense_reserve was to be called before
    FC_HIP(hipDeviceSynchronize());
    FC_TRY(dense_replace(d, d->work));
    d->work = nullptr; d->work_cap = 0;
    const size_t cap = (bytes + bytes / 4 + 4095) & ~(size_t)4095;
    FC_HIP(hipMalloc((void**)&d->work, cap));
    d->work_cap = cap;
    return FC_OK;
}

int dense_sort(fc_dense* d, int64_t n) {
    bool now;
    FC_TRY(dense_capturing(d, &now));
    SortBufs& s = d->sort;
    if (n <= s.cap && cdiv(n, RS_TILE) << RS_MAX_BITS <= s.ghist_cap && s.stot[1]) return FC_OK;
    if (now) return FC_ERR_HIP;
    if (d->captured) {
        FC_HIP(hipDeviceSynchronize());
        for (int32_t** p : {&s.keysA, &s.valsA, &s.keysB, &s.valsB, &s.ghist}) { FC_TRY(dense_replace(d, *p)); *p = nullptr; }
        s.cap = s.ghist_cap = 0;
    }
    return ensure_sort(s, n);
}

static void dense_free(fc_dense* d) {
    if (!d) return;
    (void)hipSetDevice(d->device);
    for (fc_dense::Kept* k = d->kept; k;) {
        fc_dense::Kept* const next = k->next;
        (void)hipFree(k->p);
        delete k;
        k = next;
    }
    SortBufs& s = d->sort;
    for (int32_t* p : {s.keysA, s.valsA, s.keysB, s.valsB, s.ghist, s.dtot, s.stot[0], s.stot[1]}) if (p) (void)hipFree(p);
    if (d->work) (void)hipFree(d->work);
    if (d->flags) (void)hipFree(d->flags);
    delete d;
}

static int dense_init(fc_dense* d, void* stream) {
    FC_HIP(hipGetDevice(&d->device));
    d->stream = (hipStream_t)stream;
    FC_HIP(hipMalloc((void**)&d->flags, 4));
    FC_HIP(hipMemset(d->flags, 0, 4));
    FC_HIP(hipStreamSynchronize(nullptr));       // nothing orders the handle's stream behind the null stream
    return FC_OK;
}

__global__ void k_clear_word(uint32_t* p) { *p = 0; }

}  // namespace fc

using namespace fc;

extern "C" {

int dense_create(void* hip_stream, fc_dense** out) {
    if (!out) return FC_ERR_INVALID_ARG;
    *out = nullptr;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || ndev <= 0) { (void)hipGetLastError(); return FC_ERR_HIP; }
    fc_dense* d = new (std::nothrow) fc_dense();
    if (!d) return FC_ERR_OOM_PINNED;                    // host memory
    const int rc = dense_init(d, hip_stream);
    if (rc != FC_OK) { dense_free(d); return rc; }
    *out = d;
    return FC_OK;
}

int dense_reserve(fc_dense* d, int64_t max_tokens, int64_t max_rows, int32_t max_dim, int32_t max_tensors) {
    if (!d || max_tokens < 0 || max_tokens >= DENSE_LIMIT || max_rows < 0 || max_rows >= DENSE_LIMIT || max_dim < 0 || max_dim > DENSE_MAX_DIM ||
        max_tensors < 0)
        return FC_ERR_INVALID_ARG;
    FC_HIP(hipSetDevice(d->device));
    if (max_tokens > 0) FC_TRY(dense_sort(d, max_tokens));
    size_t most = clip_work_bytes(max_tensors);
    if (max_dim > 0) most = std::max({most, token_work_bytes(max_tokens, max_rows, max_dim), norm_work_bytes(DENSE_LIMIT, max_dim)});
    return dense_work(d, most);
}

int dense_check(fc_dense* d) {
    if (!d) return FC_ERR_INVALID_ARG;
    FC_HIP(hipSetDevice(d->device));
    uint32_t flags = 0;
    FC_HIP(hipMemcpyAsync(&flags, d->flags, 4, hipMemcpyDeviceToHost, d->stream));
    FC_HIP(hipStreamSynchronize(d->stream));
    if (!flags) return FC_OK;
    k_clear_word<<<1, 1, 0, d->stream>>>(d->flags);
    FC_HIP(hipGetLastError());
    FC_HIP(hipStreamSynchronize(d->stream));
    return FC_ERR_ID_OUT_OF_RANGE;
}

int dense_destroy(fc_dense* d) {
    if (!d) return FC_ERR_INVALID_ARG;
    (void)hipSetDevice(d->device);
    (void)hipStreamSynchronize(d->stream);
    dense_free(d);
    return FC_OK;
}

}  // extern "C"
