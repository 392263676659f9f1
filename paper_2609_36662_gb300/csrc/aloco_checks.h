// What the entry points check of their arguments (host code).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "aloco_internal.h"

namespace aloco {

inline int fail(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return report_error(code, buf);
}

inline int cuda_fail(cudaError_t e, const char *what) {
    return fail(ALOCO_ERR_CUDA, "%s: %s (%s)", what, cudaGetErrorString(e),
                cudaGetErrorName(e));
}

inline int done() { return report_error(ALOCO_OK, ""); }

// The current device and its SMs.
inline int current_device(int *device, int *sm_count) {
    static PerDevice sms;
    cudaError_t e = cudaGetDevice(device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    const int slot = *device < kMaxDevices ? *device : -1;
    *sm_count = sms.get(slot);
    if (*sm_count == 0) {
        e = cudaDeviceGetAttribute(sm_count, cudaDevAttrMultiProcessorCount, *device);
        if (e != cudaSuccess) return cuda_fail(e, "cudaDeviceGetAttribute");
        sms.set(slot, *sm_count);
    }
    return ALOCO_OK;
}

// An allocation on the current device that a buffer of this call lies in.
struct Range {
    uintptr_t begin = 0, end = 0;
    bool holds(const void *p, size_t bytes) const {
        return (uintptr_t)p >= begin && (uintptr_t)p < end && bytes <= end - (uintptr_t)p;
    }
};

// Device memory of `device`, and its allocation's extent; false where the
// driver says otherwise or cannot say.
inline bool device_range(const void *p, int device, Range *r) {
    typedef CUresult (*Fn)(unsigned, CUpointer_attribute *, void **, CUdeviceptr);
    static const Fn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuPointerGetAttributes", &f, 12000,
                                             cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return (Fn)f;
    }();
    if (!fn) return false;
    unsigned type = 0;
    int ordinal = -1;
    CUdeviceptr start = 0;
    size_t size = 0;
    CUpointer_attribute what[] = {CU_POINTER_ATTRIBUTE_MEMORY_TYPE,
                                  CU_POINTER_ATTRIBUTE_DEVICE_ORDINAL,
                                  CU_POINTER_ATTRIBUTE_RANGE_START_ADDR,
                                  CU_POINTER_ATTRIBUTE_RANGE_SIZE};
    void *out[] = {&type, &ordinal, &start, &size};
    if (fn(4, what, out, (CUdeviceptr)p) != CUDA_SUCCESS || type != CU_MEMORYTYPE_DEVICE ||
        ordinal != device || size == 0)
        return false;
    r->begin = (uintptr_t)start;
    r->end = (uintptr_t)start + size;
    return true;
}

// check_buffer for the buffers of one call.  Small ones mostly share an
// allocation (a framework's pool): one question to the driver serves all that
// lie in the same; what it does not settle goes to check_buffer.
struct RangeCheck {
    static constexpr int kKept = 4;
    Range seen[kKept];
    int n = 0;
    int operator()(const void *p, size_t bytes, int device, const char *name, int index = -1) {
        for (int i = 0; i < n; ++i)
            if (seen[i].holds(p, bytes)) return ALOCO_OK;
        Range r;
        if (device_range(p, device, &r) && r.holds(p, bytes)) {
            seen[n < kKept ? n++ : kKept - 1] = r;
            return ALOCO_OK;
        }
        return check_buffer(p, bytes, device, name, index);
    }
};

// A buffer of a call: [p, p + bytes), written or read.
struct Buffer {
    const char *name;
    const void *p;
    size_t bytes, align;
    bool written;
};

// Most buffers of one call: logits, targets, advantages, old, ref, weights,
// terms, logp, grad, scratch, cu_seqlens.
struct Buffers {
    Buffer b[12];
    int n = 0;
    void add(const char *name, const void *p, size_t bytes, size_t align, bool written) {
        if (bytes) b[n++] = {name, p, bytes, align, written};
    }
};

inline int check_buffers(const Buffers &s, bool grad_over_logits, int *sm_count) {
    for (int i = 0; i < s.n; ++i) {
        const Buffer &x = s.b[i];
        if (!x.p) return fail(ALOCO_ERR_ARG, "NULL %s", x.name);
        if ((uintptr_t)x.p & (x.align - 1))
            return fail(ALOCO_ERR_ARG, "%s: not aligned to %zu bytes", x.name, x.align);
    }
    for (int i = 0; i < s.n; ++i)
        for (int j = i + 1; j < s.n; ++j) {
            const Buffer &x = s.b[i], &y = s.b[j];
            if (!x.written && !y.written) continue;
            if ((uintptr_t)x.p >= (uintptr_t)y.p + y.bytes ||
                (uintptr_t)y.p >= (uintptr_t)x.p + x.bytes)
                continue;
            if (grad_over_logits && !std::strcmp(x.name, "logits") && !std::strcmp(y.name, "grad"))
                continue;
            return fail(ALOCO_ERR_ALIAS, "%s and %s overlap", x.name, y.name);
        }
    int device, rc = current_device(&device, sm_count);
    RangeCheck check;
    for (int i = 0; i < s.n && rc == ALOCO_OK; ++i)
        rc = check(s.b[i].p, s.b[i].bytes, device, s.b[i].name);
    return rc;
}

inline cudaStream_t stream_of(const aloco_opts_t *o) {
    return o ? (cudaStream_t)o->stream : (cudaStream_t) nullptr;
}

}  // namespace aloco
