// What the host sides of the serving operators have in common: alignment and
// cache checks, the device's size.  Included by serve.hip and batch.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>

#include "../../include/tetra.h"
#include "kv_cache.h"

namespace tetra_host {

constexpr long long kMaxGrid = 0x7FFFFFFFll;
constexpr long long kMaxGroups = 0xFFFFFFFFll / 256;     // of 256 threads: a launch holds less than 2^32
constexpr int kMaxVocab = 1 << 22;     // so that a row's sum of weights, 2^62 at most, fits 64 bits

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int launch_status() { return hipGetLastError() == hipSuccess ? TETRA_OK : TETRA_EDEVICE; }

constexpr int kMaxTokens = 1 << 30;    // of a sequence, so that token numbers have room above them in an int

// a cache's sizes and pointers, as the kernels take them
inline int cache_of(const tetra_kv_cache* c, tetra_dev::KvCache* out) {
    if (!c || !c->k || !c->v || !c->scales || !c->pages || !c->lens) return TETRA_EINVAL;
    if (c->num_pages < 1 || c->kv_heads < 1 || c->seqs < 1 || c->max_pages < 1) return TETRA_EINVAL;
    int shift = 4;
    while (shift < 7 && 1 << shift != c->page_tokens) ++shift;
    if (1 << shift != c->page_tokens) return TETRA_EINVAL;
    if (c->max_pages > kMaxTokens >> shift) return TETRA_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128) return c->head_dim < 1 ? TETRA_EINVAL : TETRA_EUNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->scales, 8) || !aligned(c->pages, 4) ||
        !aligned(c->lens, 4))
        return TETRA_EALIGN;
    *out = {c->k, c->v, c->scales, c->pages, c->lens, c->num_pages, c->page_tokens, shift, c->kv_heads, c->seqs,
            c->max_pages};
    return TETRA_OK;
}

// compute units of the current device, asked for once per device
inline int device_cus(int* cus) {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return TETRA_EDEVICE;
    n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return TETRA_EDEVICE;
        known[dev].store(n, std::memory_order_relaxed);
    }
    *cus = n;
    return TETRA_OK;
}

}  // namespace tetra_host
