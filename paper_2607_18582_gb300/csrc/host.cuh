// Host-side plumbing of the C entry points: failures as exceptions that no entry point lets
// through, the last-error text, and device memory through the context's allocator.
#pragma once

#include <cstdarg>
#include <cstdio>
#include <new>
#include <stdexcept>

#include "common.cuh"

namespace mure {

struct Fail {
    mure_status st;
};

inline void set_err(mure_ctx *c, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
inline void set_err(mure_ctx *c, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    if (c) c->err = buf;
}

#define FAILIF(cond, ctx, status, ...)        \
    do {                                      \
        if (cond) {                           \
            set_err(ctx, __VA_ARGS__);        \
            throw Fail{status};               \
        }                                     \
    } while (0)

#define CK(ctx, call)                                                                              \
    do {                                                                                           \
        cudaError_t e_ = (call);                                                                   \
        FAILIF(e_ != cudaSuccess, ctx, MURE_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_));    \
    } while (0)

inline void *dalloc(mure_ctx *c, size_t bytes)
{
    if (bytes == 0) bytes = 16;
    void *p = nullptr;
    if (c->has_alloc) {
        p = c->alloc.alloc(bytes, (void *)c->stream, c->alloc.user);
    } else {
        if (cudaMallocAsync(&p, bytes, c->stream) != cudaSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
    }
    FAILIF(!p, c, MURE_ERR_OOM, "device allocation of %zu bytes failed", bytes);
    return p;
}

inline void dfree(mure_ctx *c, const void *cp)
{
    void *p = const_cast<void *>(cp);
    if (!p) return;
    if (c->has_alloc) c->alloc.free(p, (void *)c->stream, c->alloc.user);
    else cudaFreeAsync(p, c->stream);
}

template <class F>
mure_status run(mure_ctx *c, F &&fn)
{
    if (c) c->err.clear();
    try {
        fn();
    } catch (const Fail &f) {
        return f.st;
    } catch (const std::bad_alloc &) {
        set_err(c, "host allocation failed");
        return MURE_ERR_OOM;
    } catch (const std::length_error &) {   // a host array of more elements than a vector holds
        set_err(c, "host allocation failed");
        return MURE_ERR_OOM;
    }
    return MURE_OK;
}

inline void check_launch(mure_ctx *c)
{
    cudaError_t e = cudaGetLastError();
    FAILIF(e != cudaSuccess, c, MURE_ERR_CUDA, "kernel launch: %s", cudaGetErrorString(e));
}

}  // namespace mure
