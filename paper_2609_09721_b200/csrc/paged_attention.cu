// efq_paged_attention_fwd: softmax attention of a step's new tokens over a paged cache.  paged_few.cuh holds the kernel for few query rows,
// paged_chunk.cuh that for many, paged_units.h and paged_walk.cuh how the work is shared; here are the kernel that joins parts and the entry points.
#include <cuda.h>

#include <atomic>

#include "efq_internal.cuh"
#include "paged_chunk.cuh"
#include "paged_few.cuh"

namespace efq {
namespace {

constexpr int kMaxCtas = 256;            // of the first kernel; the workspace has room for the parts of as many

// Joins the parts of the query tiles that span CTAs.  blockIdx.x: the CTA that ended the tile.  kWarps warps take a row, every kWarps-th
// part each, a lane four channels.  Few rows may have a part from every CTA (one long context), many rows have two or three as a rule.
// half_rows: rows of the first of the two halves of a tile of many rows (whole tokens); parts keep kRows / 2 for each half.
template <typename T, int kRows, int kWarps>
__global__ void __launch_bounds__(128) paged_join_kernel(const __grid_constant__ PagedArgs A, int half_rows)
{
    constexpr int kAtOnce = 4 / kWarps;         // rows of a block
    ptx::grid_wait();
    const int c = blockIdx.x, lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) % kWarps, which = (threadIdx.x >> 5) / kWarps;
    const PagedRecord rec = {__ldcg(&A.records[c].first), __ldcg(&A.records[c].token0), __ldcg(&A.records[c].tokens), __ldcg(&A.records[c].head)};
    if (rec.first < 0) return;
    __shared__ float4 xs[4][32];
    __shared__ float ls[4];
    for (int r = blockIdx.y * kAtOnce + which; r < rec.tokens * A.G; r += gridDim.y * kAtOnce) {
        const int at = r < half_rows ? r : kRows / 2 + r - half_rows;
        auto slot = [&](int i) { return (2 * i + (i == rec.first ? 1 : 0)) * kRows + at; };
        float top = -INFINITY;
        for (int i = rec.first + lane; i <= c; i += 32) top = fmaxf(top, __ldcg(&A.part_ml[slot(i)].x));
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        const float base = top == -INFINITY ? 0.0f : top;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float l = 0.0f;
#pragma unroll 4
        for (int i = rec.first + warp; i <= c; i += kWarps) {
            const float2 ml = __ldcg(&A.part_ml[slot(i)]);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(A.part_o + static_cast<int64_t>(slot(i)) * kPagedD) + lane);
            const float f = paged_exp2(ml.x - base);
            l = fmaf(ml.y, f, l);
            x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
        }
        if (kWarps > 1) {
            xs[warp][lane] = x;
            if (lane == 0) ls[warp] = l;
            __syncthreads();
#pragma unroll
            for (int w = 1; w < kWarps; ++w) {
                const float4 y = xs[w][lane];
                x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                l += ls[w];
            }
            __syncthreads();
        }
        if (warp != 0) continue;
        const int token = rec.token0 + r / A.G, head = rec.head * A.G + r % A.G;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        *reinterpret_cast<uint2*>(A.o + token * A.o_token + head * A.o_head + 8 * lane) =
            make_uint2(Pack2<T>::round(x.x * inv, x.y * inv), Pack2<T>::round(x.z * inv, x.w * inv));
        if (A.lse != nullptr && lane == 0) A.lse[static_cast<int64_t>(token) * (A.Hkv * A.G) + head] = top * kLn2 + logf(l);
    }
}

// The driver's encoder: asked for once; the library is not linked against the driver, so that it loads where there is none.
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static std::atomic<void*> known{nullptr};
    void* p = known.load(std::memory_order_acquire);
    cudaDriverEntryPointQueryResult found;
    if (p == nullptr && cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) == cudaSuccess && found == cudaDriverEntryPointSuccess)
        known.store(p, std::memory_order_release);
    return reinterpret_cast<EncodeTiled>(p);
}

// Box of 64 channels x `box` rows of dimension 1; strides in elements, as the dimensions 1, 2, 3 have them.
bool encode_rows(CUtensorMap* map, int dtype, const void* base, int rank, const uint64_t* dims, const int64_t* strides, const uint32_t* box)
{
    cuuint64_t bytes[3];
    cuuint32_t ones[4] = {1, 1, 1, 1};
    for (int i = 0; i + 1 < rank; ++i) bytes[i] = dims[i + 1] > 1 ? static_cast<cuuint64_t>(strides[i]) * 2 : 256;      // a dimension of one is never stepped along
    const EncodeTiled encode = encode_tiled();
    return encode != nullptr && encode(map, dtype == EFQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, static_cast<cuuint32_t>(rank),
                                  const_cast<void*>(base), dims, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct PagedPlan {
    int rows;                            // of a part
    size_t ml, records, total;
};
PagedPlan plan_paged(int64_t group_rows)
{
    PagedPlan p;
    p.rows = group_rows <= 16 ? 16 : group_rows <= 32 ? 32 : 2 * kChunkRows;
    p.ml = static_cast<size_t>(2 * kMaxCtas) * p.rows * kPagedD * 4;
    p.records = p.ml + static_cast<size_t>(2 * kMaxCtas) * p.rows * sizeof(float2);
    p.total = p.records + kMaxCtas * sizeof(PagedRecord);
    return p;
}

template <typename Kernel>
cudaError_t allow_smem(Kernel kernel, int bytes, std::atomic<uint64_t>& done, int dev)
{
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if ((done.load(std::memory_order_relaxed) >> dev & 1u) != 0u) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

template <typename T, int kM>
cudaError_t launch_few_rows(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const PagedArgs& A, int ctas, int max_rows, int dev, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    constexpr int smem = static_cast<int>(sizeof(FewSmem<kM>)) + 1024;
    cudaError_t e = allow_smem(paged_few_kernel<T, kM>, smem, done, dev);
    if (e == cudaSuccess) e = launch_overlapped(paged_few_kernel<T, kM>, dim3(static_cast<unsigned>(ctas)), kFewThreads, smem, st, mq, mk, mv, A);
    if (e == cudaSuccess) e = launch_overlapped(paged_join_kernel<T, 16 * kM, 4>, dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(max_rows)), 128, 0, st, A, 16 * kM);
    return e;
}

template <typename T>
cudaError_t launch_chunk(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const PagedArgs& A, int ctas, int dev, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    constexpr int smem = static_cast<int>(sizeof(ChunkSmem)) + 1024;
    cudaError_t e = allow_smem(paged_chunk_kernel<T>, smem, done, dev);
    if (e == cudaSuccess) e = launch_overlapped(paged_chunk_kernel<T>, dim3(static_cast<unsigned>(ctas)), kChunkThreads, smem, st, mq, mk, mv, A);
    if (e == cudaSuccess) e = launch_overlapped(paged_join_kernel<T, 2 * kChunkRows, 1>, dim3(static_cast<unsigned>(ctas), 16), 128, 0, st, A, A.step / 2 * A.G);
    return e;
}

efq_status_t paged_attention(const efq_rows_t* q, float* lse, int64_t total, int max_seqlen_q, const efq_paged_t* cache, int d, int dtype, int causal,
                             float softmax_scale, void* workspace, size_t workspace_bytes, void* stream, bool inject_skip_loads)
{
    if (!q || !cache || !q->src || !q->dst || total < 0 || max_seqlen_q < 0 || q->heads <= 0) return EFQ_ERR_INVALID_ARG;
    if (!(softmax_scale == softmax_scale) || softmax_scale > 3.0e38f) return EFQ_ERR_INVALID_ARG;
    const efq_status_t st = check_paged(*cache, d, dtype);
    if (st != EFQ_OK) return st;
    if (q->heads % cache->n_heads != 0) return EFQ_ERR_INVALID_ARG;
    const int G = q->heads / cache->n_heads;
    if (G > kChunkRows || total >= (1ll << 31) - 256) return EFQ_ERR_UNSUPPORTED;
    if (q->src_head < 0 || q->src_token < 0 || q->dst_head < 0 || q->dst_token < 0) return EFQ_ERR_INVALID_ARG;
    if (!aligned_rows(q->src, q->src_head, q->src_token, 0) || !aligned_rows(q->dst, q->dst_head, q->dst_token, 0)) return EFQ_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return EFQ_ERR_ALIGNMENT;
    if (total == 0 || cache->n_seqs == 0) return EFQ_OK;
    const int64_t group_rows = static_cast<int64_t>(G) * (max_seqlen_q > 0 ? max_seqlen_q : 1);
    const PagedPlan plan = plan_paged(group_rows);
    if (!workspace || workspace_bytes < plan.total) return EFQ_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return EFQ_ERR_ALIGNMENT;
    if (!device_is_sm100()) return EFQ_ERR_ARCH;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return EFQ_ERR_CUDA;
    int ctas = sm_count(dev);
    if (ctas <= 0) return EFQ_ERR_CUDA;
    if (ctas > kMaxCtas) ctas = kMaxCtas;

    PagedArgs A{};
    A.page_table = cache->page_table;
    A.cu_seqlens = cache->cu_seqlens;
    A.seq_lens = cache->seq_lens;
    A.table_stride = cache->table_stride;
    A.n_seqs = cache->n_seqs;
    A.n_pages = cache->n_pages;
    A.max_pages = cache->max_pages;
    A.page_shift = __builtin_ctz(static_cast<unsigned>(cache->page_size));
    A.Hkv = cache->n_heads;
    A.G = G;
    A.causal = causal ? 1 : 0;
    A.total = static_cast<int32_t>(total);
    const double scale = softmax_scale > 0.0f ? static_cast<double>(softmax_scale) : 0.08838834764831844055;
    A.scale_log2 = static_cast<float>(scale * 1.44269504088896340736);
    A.o = static_cast<char*>(q->dst);
    A.o_token = 2 * q->dst_token;
    A.o_head = 2 * q->dst_head;
    A.lse = lse;
    char* const ws = static_cast<char*>(workspace);
    A.part_o = reinterpret_cast<float*>(ws);
    A.part_ml = reinterpret_cast<float2*>(ws + plan.ml);
    A.records = reinterpret_cast<PagedRecord*>(ws + plan.records);
    A.inject_skip_loads = inject_skip_loads ? 1 : 0;
    const bool many = plan.rows > 32;
    A.step = many ? kChunkRows / G * 2 : plan.rows / G;

    CUtensorMap mq, mk, mv;
    const uint64_t q_dims[3] = {kPagedD, static_cast<uint64_t>(q->heads), static_cast<uint64_t>(total)};
    const int64_t q_strides[2] = {q->src_head, q->src_token};
    const uint32_t q_box[3] = {64, static_cast<uint32_t>(G), static_cast<uint32_t>(many ? A.step / 2 : A.step)};
    const uint64_t dims[4] = {kPagedD, static_cast<uint64_t>(cache->page_size), static_cast<uint64_t>(cache->n_heads), static_cast<uint64_t>(cache->n_pages)};
    const int64_t k_strides[3] = {cache->k_token, cache->k_head, cache->k_page}, v_strides[3] = {cache->v_token, cache->v_head, cache->v_page};
    const int keys = many ? kChunkKeys : kFewKeys;
    const uint32_t box[4] = {64, static_cast<uint32_t>(cache->page_size < keys ? cache->page_size : keys), 1, 1};
    if (!encode_rows(&mq, dtype, q->src, 3, q_dims, q_strides, q_box) || !encode_rows(&mk, dtype, cache->k, 4, dims, k_strides, box) ||
        !encode_rows(&mv, dtype, cache->v, 4, dims, v_strides, box))
        return EFQ_ERR_CUDA;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int max_rows = A.step * G;
    using Bf = __nv_bfloat16;
    const bool bf = dtype == EFQ_BF16;
    const cudaError_t e = many ? (bf ? launch_chunk<Bf>(mq, mk, mv, A, ctas, dev, s) : launch_chunk<__half>(mq, mk, mv, A, ctas, dev, s))
                          : plan.rows == 16
                              ? (bf ? launch_few_rows<Bf, 1>(mq, mk, mv, A, ctas, max_rows, dev, s) : launch_few_rows<__half, 1>(mq, mk, mv, A, ctas, max_rows, dev, s))
                              : (bf ? launch_few_rows<Bf, 2>(mq, mk, mv, A, ctas, max_rows, dev, s) : launch_few_rows<__half, 2>(mq, mk, mv, A, ctas, max_rows, dev, s));
    return e == cudaSuccess ? EFQ_OK : EFQ_ERR_CUDA;
}

}  // namespace
}  // namespace efq

extern "C" size_t efq_paged_attention_workspace_bytes(int Hq, int Hkv, int max_seqlen_q, int d)
{
    if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || Hq / Hkv > 128 || max_seqlen_q < 0 || d != efq::kPagedD) return 0;
    return efq::plan_paged(static_cast<int64_t>(Hq / Hkv) * (max_seqlen_q > 0 ? max_seqlen_q : 1)).total;
}

extern "C" efq_status_t efq_paged_attention_fwd(const efq_rows_t* q, float* lse, int64_t total, int max_seqlen_q, const efq_paged_t* cache, int d,
                                                int dtype, int causal, float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    return efq::paged_attention(q, lse, total, max_seqlen_q, cache, d, dtype, causal, softmax_scale, workspace, workspace_bytes, stream, false);
}

extern "C" efq_status_t efq_paged_attention_fwd_inject_timeout(const efq_rows_t* q, float* lse, int64_t total, int max_seqlen_q, const efq_paged_t* cache,
                                                               int d, int dtype, int causal, float softmax_scale, void* workspace,
                                                               size_t workspace_bytes, void* stream)
{
    return efq::paged_attention(q, lse, total, max_seqlen_q, cache, d, dtype, causal, softmax_scale, workspace, workspace_bytes, stream, true);
}
