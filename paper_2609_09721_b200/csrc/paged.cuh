// Shared by the operators around a paged cache (rotary.cu, paged_attention.cu): checks of its description, element types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "efq_common.cuh"

namespace efq {

constexpr int kPagedD = 128;

template <typename T> struct Pack2;
template <> struct Pack2<__nv_bfloat16> {
    static __device__ __forceinline__ float2 widen(uint32_t u) { return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t round(float lo, float hi)
    {
        uint32_t d;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
        return d;
    }
};
template <> struct Pack2<__half> {
    static __device__ __forceinline__ float2 widen(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
    static __device__ __forceinline__ uint32_t round(float lo, float hi)
    {
        uint32_t d;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
        return d;
    }
};

inline bool aligned_rows(const void* p, int64_t a, int64_t b, int64_t c) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ((a | b | c) & 7) == 0; }
inline bool aligned_ints(const int32_t* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The cache's own fields; the tables' contents are looked at by the kernels.
inline efq_status_t check_paged(const efq_paged_t& c, int d, int dtype)
{
    if (!c.k || !c.v || (c.n_seqs > 0 && (!c.page_table || !c.cu_seqlens || !c.seq_lens))) return EFQ_ERR_INVALID_ARG;
    if (c.n_pages <= 0 || c.n_heads <= 0 || c.max_pages <= 0 || c.n_seqs < 0 || c.table_stride < 0) return EFQ_ERR_INVALID_ARG;
    if (dtype != EFQ_BF16 && dtype != EFQ_FP16) return EFQ_ERR_UNSUPPORTED;
    if (d != kPagedD || c.page_size < 16 || c.page_size > 4096 || (c.page_size & (c.page_size - 1)) != 0) return EFQ_ERR_UNSUPPORTED;
    // 32-bit indices of a sequence's tokens, up to the end of a tile of 128 of them that the last one lies in
    if (static_cast<int64_t>(c.max_pages) * c.page_size > (1ll << 31) - 256) return EFQ_ERR_UNSUPPORTED;
    if (!aligned_ints(c.page_table) || !aligned_ints(c.cu_seqlens) || !aligned_ints(c.seq_lens)) return EFQ_ERR_ALIGNMENT;
    if (c.k_page < 0 || c.k_head < 0 || c.k_token < 0 || c.v_page < 0 || c.v_head < 0 || c.v_token < 0) return EFQ_ERR_INVALID_ARG;
    if (!aligned_rows(c.k, c.k_page, c.k_head, c.k_token) || !aligned_rows(c.v, c.v_page, c.v_head, c.v_token)) return EFQ_ERR_ALIGNMENT;
    return EFQ_OK;
}

inline bool device_is_sm100()
{
    int dev = 0, major = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) == cudaSuccess && major == 10;
}

}  // namespace efq
