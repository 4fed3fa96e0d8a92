// Shared by the operators on caches kept in pages: the view of the pages, a division by the page size, conversions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "common.cuh"

namespace mtad {

// ---- host helpers of the operators that need no context (ops.cu)
void mtad_ops_count(unsigned int kernels);          // kernels enqueued, for mtad_kernel_launches
int ops_status(cudaError_t e);                      // MTAD_OK or MTAD_E_CUDA, the code kept for mtad_ops_cuda_error

// Raises a kernel's limit of dynamic shared memory, once per device.
template <auto* Kernel>
inline cudaError_t ops_smem(int bytes) {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// n / d for 0 <= n < 2^31 and a d fixed at launch: a multiplication and a shift (page sizes need not be powers of two)
struct FastDiv {
    uint32_t d, m, s;
};
inline FastDiv fast_div(uint32_t d) {
    FastDiv f{d, 0, 0};
    while (f.s < 32 && (1ull << f.s) < d) ++f.s;
    f.m = (uint32_t)((((1ull << f.s) - d) << 32) / d + 1);
    return f;
}
__host__ __device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) {
#ifdef __CUDA_ARCH__
    return (__umulhi(n, f.m) + n) >> f.s;
#else
    return (uint32_t)((((uint64_t)n * f.m >> 32) + n) >> f.s);
#endif
}

// Pages of one layer as the kernels see them. Elements are 16 bits wide; offsets are 64-bit (a pool passes 2^31 elements).
struct PagedView {
    uint16_t *k, *v;
    const int32_t* table;
    long long page_stride, head_stride, slot_stride;
    long long table_stride;
    int n_pages, hd, Hkv;
    FastDiv page;
};

// Element offset of (slot, head 0) of a sequence whose table row is `row`; -1 where the table names no page of the pool.
__device__ __forceinline__ long long slot_offset(const PagedView& kv, const int32_t* row, int slot) {
    const uint32_t p = div_by((uint32_t)slot, kv.page);
    const int id = __ldg(row + p);
    if ((unsigned)id >= (unsigned)kv.n_pages) return -1;
    return (long long)id * kv.page_stride + (long long)(slot - (int)(p * kv.page.d)) * kv.slot_stride;
}

template <typename T> struct Num;
template <> struct Num<__nv_bfloat16> {
    static __device__ __forceinline__ float to(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static constexpr uint32_t kExp = 0x7f80u;      // exponent bits: all set means infinity or NaN
};
template <> struct Num<__half> {
    static __device__ __forceinline__ float to(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half from(float x) { return __float2half_rn(x); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 p = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static constexpr uint32_t kExp = 0x7c00u;
};

// Host side: whether the elements of an array that a call writes all lie apart, rows of `inner` of them along the given dimensions (strides >= 0;
// one that is not longer than what it strides over would have two threads write the same place).
struct Dim {
    int64_t count, stride;
};
template <int N>
inline bool lie_apart(int64_t inner, Dim (&&d)[N]) {
    for (int i = 1; i < N; ++i)                          // by stride
        for (int k = i; k > 0 && d[k].stride < d[k - 1].stride; --k) {
            const Dim x = d[k];
            d[k] = d[k - 1];
            d[k - 1] = x;
        }
    for (const Dim& x : d)
        if (x.count < 1) return true;                     // (nothing there)
    __int128 extent = inner;
    for (const Dim& x : d) {
        if (x.count == 1) continue;
        if (x.stride < extent) return false;
        extent += (__int128)x.stride * (x.count - 1);
    }
    return true;
}
// ... of the pages, for calls that write them
inline bool pages_lie_apart(const mtad_paged_kv* kv) {
    return kv->k_pages != kv->v_pages &&
           lie_apart(kv->head_dim, {{kv->n_pages, kv->page_stride}, {kv->n_kv_heads, kv->head_stride}, {kv->page_size, kv->slot_stride}});
}

// Host side: checks of a mtad_paged_kv that every operator makes, and the kernels' view of it.
inline int paged_view(const mtad_paged_kv* kv, PagedView* out) {
    if (!kv || !kv->k_pages || !kv->v_pages || !kv->table) return MTAD_E_INVALID;
    if (kv->dtype != MTAD_BF16 && kv->dtype != MTAD_F16) return MTAD_E_INVALID;
    if (kv->n_pages < 1 || kv->page_size < 1 || kv->n_kv_heads < 1 || kv->max_pages < 1 || kv->table_stride < kv->max_pages)
        return MTAD_E_INVALID;
    if (kv->head_dim < 8 || kv->head_dim > MTAD_PAGED_MAX_HEAD_DIM || kv->head_dim % 8) return MTAD_E_INVALID;
    if (kv->n_kv_heads > MTAD_PAGED_MAX_HEADS) return MTAD_E_CAPACITY;
    if ((long long)kv->max_pages * kv->page_size > MTAD_PAGED_MAX_LEN) return MTAD_E_CAPACITY;
    // rows are read and written in 16-byte pieces
    if ((reinterpret_cast<uintptr_t>(kv->k_pages) | reinterpret_cast<uintptr_t>(kv->v_pages)) & 15) return MTAD_E_INVALID;
    if (kv->page_stride % 8 || kv->head_stride % 8 || kv->slot_stride % 8) return MTAD_E_INVALID;
    if (kv->page_stride < 0 || kv->head_stride < 0 || kv->slot_stride < kv->head_dim) return MTAD_E_INVALID;
    out->k = static_cast<uint16_t*>(kv->k_pages);
    out->v = static_cast<uint16_t*>(kv->v_pages);
    out->table = kv->table;
    out->page_stride = kv->page_stride;
    out->head_stride = kv->head_stride;
    out->slot_stride = kv->slot_stride;
    out->table_stride = kv->table_stride;
    out->n_pages = kv->n_pages;
    out->hd = kv->head_dim;
    out->Hkv = kv->n_kv_heads;
    out->page = fast_div((uint32_t)kv->page_size);
    return MTAD_OK;
}

}  // namespace mtad
