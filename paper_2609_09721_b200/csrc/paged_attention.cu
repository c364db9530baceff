// efq_paged_attention_fwd: softmax attention of a step's new tokens over a paged cache.  paged_few.cuh holds the kernel for few query rows,
// paged_chunk.cuh that for many, paged_units.h and paged_walk.cuh how the work is shared; here are the kernel that joins parts and the entry points.
#include <cuda.h>

#include <atomic>

#include "efq_internal.cuh"
#include "paged_chunk.cuh"
#include "paged_few.cuh"

namespace efq {
namespace {

// Joins the parts of the query tiles that span CTAs.  blockIdx.x: the CTA that ended the tile, blockIdx.y: a row of it (and further ones where
// a tile has more).  Eight warps take every eighth part each, two of them at a time, a lane four channels: bound by latency, so maxima, sums and
// outputs of as many parts are asked for at once.  One long context may leave a part in every CTA: one head of 60000 keys 15.0 us with eight
// warps, 19.7 with four (of four parts at a time) and 13.7 with sixteen, which cost short steps 0.9 to 2.7.
template <typename T, int kRows>
__global__ void __launch_bounds__(256) paged_join_kernel(const __grid_constant__ PagedArgs A)
{
    constexpr int kWarps = 8, kAhead = 2;
    ptx::grid_wait();
    const int c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int4 found = __ldcg(reinterpret_cast<const int4*>(A.records + c));
    const PagedRecord rec = {found.x, found.y, found.z, found.w};
    if (rec.first < 0) return;
    for (int r = blockIdx.y; r < rec.tokens * A.G; r += gridDim.y) {
        float top = -INFINITY, l = 0.0f;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int first = rec.first + warp; first <= c; first += kAhead * kWarps) {
            float2 ml[kAhead];
            float4 y[kAhead];
            float upto = top;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = first + u * kWarps;
                const int64_t slot = (2 * i + (i == rec.first ? 1 : 0)) * kRows + r;
                ml[u] = make_float2(-INFINITY, 0.0f);
                y[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (i <= c) {
                    ml[u] = __ldcg(A.part_ml + slot);
                    y[u] = __ldcg(reinterpret_cast<const float4*>(A.part_o + slot * kPagedD) + lane);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) upto = fmaxf(upto, ml[u].x);
            const float base = upto == -INFINITY ? 0.0f : upto, before = paged_exp2(top - base);
            top = upto;
            l *= before;
            x.x *= before; x.y *= before; x.z *= before; x.w *= before;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float f = paged_exp2(ml[u].x - base);
                l = fmaf(ml[u].y, f, l);
                x.x = fmaf(y[u].x, f, x.x); x.y = fmaf(y[u].y, f, x.y); x.z = fmaf(y[u].z, f, x.z); x.w = fmaf(y[u].w, f, x.w);
            }
        }
        __shared__ float4 xs[kWarps][32];
        __shared__ float2 mls[kWarps];
        xs[warp][lane] = x;
        if (lane == 0) mls[warp] = make_float2(top, l);
        __syncthreads();
        top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, mls[w].x);
        const float base = top == -INFINITY ? 0.0f : top;
        x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float4 y = xs[w][lane];
            const float f = paged_exp2(mls[w].x - base);
            l = fmaf(mls[w].y, f, l);
            x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
        }
        __syncthreads();
        if (warp != 0) continue;
        const int token = rec.token0 + r / A.G, head = rec.head * A.G + r % A.G;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        *reinterpret_cast<uint2*>(A.o + token * A.o_token + head * A.o_head + 8 * lane) =
            make_uint2(Pack2<T>::round(x.x * inv, x.y * inv), Pack2<T>::round(x.z * inv, x.w * inv));
        if (A.lse != nullptr && lane == 0) A.lse[static_cast<int64_t>(token) * (A.Hkv * A.G) + head] = top * kLn2 + logf(l);
    }
}

// The same for the parts of the kernel for many rows: [half][group of four channels][row].  blockIdx.y: 32 rows of a half; a lane takes a row
// and a warp every fourth group of channels, so that loads are whole lines, and the rows leave by way of shared memory as whole lines too.
template <typename T>
__global__ void __launch_bounds__(128) paged_join_chunk_kernel(const __grid_constant__ PagedArgs A)
{
    constexpr int kGroups = kPagedD / 4 / 4;        // of a warp
    __shared__ uint2 rows[32][kPagedD / 4 + 1];
    ptx::grid_wait();
    const int c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = blockIdx.y >> 2, r = (blockIdx.y & 3) * 32 + lane;
    const int4 found = __ldcg(reinterpret_cast<const int4*>(A.records + c));
    const PagedRecord rec = {found.x, found.y, found.z, found.w};
    const int per = A.step >> 1, tokens = max(0, min(per, rec.tokens - half * per)), first_row = (blockIdx.y & 3) * 32;
    if (rec.first < 0 || first_row >= tokens * A.G) return;
    float top = -INFINITY, l = 0.0f;
    float4 x[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) x[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    // two parts at a time: what a step costs is the wait for its loads
    for (int i0 = rec.first; i0 <= c; i0 += 2) {
        float2 ml[2];
        float4 y[2][kGroups];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = i0 + k;
            ml[k] = make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int u = 0; u < kGroups; ++u) y[k][u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (i <= c) {
                const int64_t at = (2 * i + (i == rec.first ? 1 : 0)) * 2 + half;
                ml[k] = __ldcg(A.part_ml + at * kChunkRows + r);
                const float4* const part = reinterpret_cast<const float4*>(A.part_o + at * kChunkRows * kPagedD) + r;
#pragma unroll
                for (int u = 0; u < kGroups; ++u) y[k][u] = __ldcg(part + (4 * u + warp) * kChunkRows);
            }
        }
        const float upto = fmaxf(top, fmaxf(ml[0].x, ml[1].x)), base = upto == -INFINITY ? 0.0f : upto, before = paged_exp2(top - base);
        const float f0 = paged_exp2(ml[0].x - base), f1 = paged_exp2(ml[1].x - base);
        top = upto;
        l = l * before + ml[0].y * f0 + ml[1].y * f1;
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
            x[u] = make_float4(x[u].x * before + y[0][u].x * f0 + y[1][u].x * f1, x[u].y * before + y[0][u].y * f0 + y[1][u].y * f1,
                               x[u].z * before + y[0][u].z * f0 + y[1][u].z * f1, x[u].w * before + y[0][u].w * f0 + y[1][u].w * f1);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int u = 0; u < kGroups; ++u)
        rows[lane][4 * u + warp] = make_uint2(Pack2<T>::round(x[u].x * inv, x[u].y * inv), Pack2<T>::round(x[u].z * inv, x[u].w * inv));
    if (A.lse != nullptr && warp == 0 && r < tokens * A.G)
        A.lse[static_cast<int64_t>(rec.token0 + half * per + r / A.G) * (A.Hkv * A.G) + rec.head * A.G + r % A.G] = top * kLn2 + logf(l);
    __syncthreads();
    for (int i = warp; i < 32 && first_row + i < tokens * A.G; i += 4) {
        const int row = first_row + i, token = rec.token0 + half * per + row / A.G, head = rec.head * A.G + row % A.G;
        *reinterpret_cast<uint2*>(A.o + token * A.o_token + head * A.o_head + 8 * lane) = rows[i][lane];
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

bool encode(CUtensorMap* map, int dtype, const void* base, int rank, const uint64_t* dims, const uint64_t* strides, const uint32_t* box)
{
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    const EncodeTiled f = encode_tiled();
    return f != nullptr && f(map, dtype == EFQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, static_cast<cuuint32_t>(rank),
                             const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Queries: 64 channels x the heads of a KV group x `tokens`.  Strides in elements.
bool encode_queries(CUtensorMap* map, int dtype, const efq_rows_t& q, int64_t total, int G, int tokens)
{
    const uint64_t dims[3] = {kPagedD, static_cast<uint64_t>(q.heads), static_cast<uint64_t>(total)};
    const uint64_t strides[2] = {q.heads > 1 ? static_cast<uint64_t>(q.src_head) * 2 : 256, total > 1 ? static_cast<uint64_t>(q.src_token) * 2 : 256};
    const uint32_t box[3] = {64, static_cast<uint32_t>(G), static_cast<uint32_t>(tokens)};
    return encode(map, dtype, q.src, 3, dims, strides, box);
}

// One of the cache's two tensors: 64 channels, 8 tokens, halves of the channels, groups of 8 tokens, place; `rows` tokens a copy.  The place is
// page * page_step + head * head_step in units of the greatest common divisor of their strides.
efq_status_t encode_cache(CUtensorMap* map, int dtype, const void* base, int64_t page, int64_t head, int64_t token, const efq_paged_t& c, int rows,
                          int32_t* page_step, int32_t* head_step)
{
    if (c.n_heads == 1) head = 0;
    if (c.n_pages == 1) page = 0;
    int64_t unit = page, rest = head;
    while (rest != 0) {
        const int64_t x = unit % rest;
        unit = rest;
        rest = x;
    }
    if (unit == 0) unit = 8;
    const int64_t places = (c.n_pages - 1) * (page / unit) + (c.n_heads - 1) * (head / unit) + 1;
    if (places >= (1ll << 31)) return EFQ_ERR_UNSUPPORTED;
    *page_step = static_cast<int32_t>(page / unit);
    *head_step = static_cast<int32_t>(head / unit);
    const uint64_t dims[5] = {64, 8, 2, static_cast<uint64_t>(c.page_size / 8), static_cast<uint64_t>(places)};
    const uint64_t strides[4] = {static_cast<uint64_t>(token) * 2, 128, static_cast<uint64_t>(token) * 16, static_cast<uint64_t>(unit) * 2};
    const uint32_t box[5] = {64, 8, 2, static_cast<uint32_t>((c.page_size < rows ? c.page_size : rows) / 8), 1};
    return encode(map, dtype, base, 5, dims, strides, box) ? EFQ_OK : EFQ_ERR_CUDA;
}

// Which kernel: by the rows that the query heads of a KV group and the announced tokens make.  Up to 16, and up to 32: the kernel for few rows with one or
// two groups of them, else that for many.  The lines, both sides measured (32 / 8 heads, us): 16 rows by two groups 16 sequences of 4 tokens on 5000 keys
// 63.9 and 67.0, one of 4 on 8000 14.6 and 14.8, 60 of 4 on 700 43.7 and 46.3, 64 of 1 on 5000 223 and 229; 32 rows by the kernel for many 16 of 8 on
// 5000 74.2 and 74.5, one of 8 on 8000 17.5 and 22.9, 60 of 8 on 700 53.5 and 49.9, 60 of 5 on 700 48.7 and 50.4.
struct PagedPlan {
    int rows;                            // of a query tile
    size_t parts, ml, records, total;    // behind the words of the status
};
PagedPlan plan_paged(int64_t group_rows)
{
    PagedPlan p;
    p.rows = group_rows <= kFewRows ? kFewRows : group_rows <= 2 * kFewRows ? 2 * kFewRows : 2 * kChunkRows;
    const int room = p.rows > kFewRows ? 2 * kChunkRows : kFewRows;         // one size for all that is not a decode step
    p.parts = kPagedExpired + kPagedMaxCtas * sizeof(uint32_t);
    p.ml = p.parts + static_cast<size_t>(2 * kPagedMaxCtas) * room * kPagedD * 4;
    p.records = p.ml + static_cast<size_t>(2 * kPagedMaxCtas) * room * sizeof(float2);
    p.total = p.records + kPagedMaxCtas * sizeof(PagedRecord);       // records on 16 bytes: 2 * kPagedMaxCtas * rows is a multiple of 8
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

template <typename T, int kRows>
cudaError_t launch_few_rows(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const PagedArgs& A, int ctas, int max_rows, int dev, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    constexpr int smem = static_cast<int>(sizeof(FewSmem<kRows>)) + 1024;
    cudaError_t e = allow_smem(paged_few_kernel<T, kRows>, smem, done, dev);
    if (e == cudaSuccess) e = launch_overlapped(paged_few_kernel<T, kRows>, dim3(static_cast<unsigned>(ctas)), kFewThreads, smem, st, mq, mk, mv, A);
    if (e == cudaSuccess) e = launch_overlapped(paged_join_kernel<T, kRows>, dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(max_rows)), 256, 0, st, A);
    return e;
}

template <typename T>
cudaError_t launch_chunk(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const PagedArgs& A, int ctas, int dev, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    constexpr int smem = static_cast<int>(sizeof(ChunkSmem)) + 1024;
    cudaError_t e = allow_smem(paged_chunk_kernel<T>, smem, done, dev);
    if (e == cudaSuccess) e = launch_overlapped(paged_chunk_kernel<T>, dim3(static_cast<unsigned>(ctas)), kChunkThreads, smem, st, mq, mk, mv, A);
    if (e == cudaSuccess) e = launch_overlapped(paged_join_chunk_kernel<T>, dim3(static_cast<unsigned>(ctas), 2 * kChunkRows / 32), 128, 0, st, A);
    return e;
}

efq_status_t paged_attention(const efq_rows_t* q, float* lse, int64_t total, int max_seqlen_q, const efq_paged_t* cache, int d, int dtype, int causal,
                             float softmax_scale, void* workspace, size_t workspace_bytes, void* stream, bool inject_skip_loads)
{
    if (!q || !cache || total < 0 || max_seqlen_q < 0 || q->heads <= 0) return EFQ_ERR_INVALID_ARG;
    if (total > 0 && (!q->src || !q->dst)) return EFQ_ERR_INVALID_ARG;
    const double scale = softmax_scale > 0.0f ? static_cast<double>(softmax_scale) : 0.08838834764831844055;
    const float scale_log2 = static_cast<float>(scale * 1.44269504088896340736);
    if (!(softmax_scale == softmax_scale) || scale_log2 > 3.4028234e38f) return EFQ_ERR_INVALID_ARG;      // infinite in units of log2
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
    const bool many = plan.rows > 2 * kFewRows;
    const int step = many ? kChunkRows / G * 2 : plan.rows / G;         // new tokens of a query tile
    if (paged_too_many_units(total, cache->n_seqs, static_cast<int64_t>(cache->max_pages) * cache->page_size, cache->n_heads, step, many ? kChunkShift : kFewShift,
                             many ? kChunkItem : kFewItem))
        return EFQ_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < plan.total) return EFQ_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return EFQ_ERR_ALIGNMENT;
    if (!device_is_sm100()) return EFQ_ERR_ARCH;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return EFQ_ERR_CUDA;
    int ctas = sm_count(dev);
    if (ctas <= 0) return EFQ_ERR_CUDA;
    if (ctas > kPagedMaxCtas) ctas = kPagedMaxCtas;

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
    A.scale_log2 = scale_log2;
    A.o = static_cast<char*>(q->dst);
    A.o_token = 2 * q->dst_token;
    A.o_head = 2 * q->dst_head;
    A.o_wide = ((reinterpret_cast<uintptr_t>(A.o) | static_cast<uintptr_t>(A.o_token) | static_cast<uintptr_t>(A.o_head)) & 31u) == 0 ? 1 : 0;
    A.lse = lse;
    char* const ws = static_cast<char*>(workspace);
    A.header = reinterpret_cast<uint32_t*>(ws);
    A.expired = reinterpret_cast<uint32_t*>(ws + kPagedExpired);
    A.part_o = reinterpret_cast<float*>(ws + plan.parts);
    A.part_ml = reinterpret_cast<float2*>(ws + plan.ml);
    A.records = reinterpret_cast<PagedRecord*>(ws + plan.records);
    A.inject_skip_loads = inject_skip_loads ? 1 : 0;
    A.step = step;

    CUtensorMap mq, mk, mv;
    const int keys = many ? kChunkKeys : kFewKeys;
    if (!encode_queries(&mq, dtype, *q, total, G, many ? A.step / 2 : A.step)) return EFQ_ERR_CUDA;
    efq_status_t map_status = encode_cache(&mk, dtype, cache->k, cache->k_page, cache->k_head, cache->k_token, *cache, keys, &A.k_page_step, &A.k_head_step);
    if (map_status == EFQ_OK)
        map_status = encode_cache(&mv, dtype, cache->v, cache->v_page, cache->v_head, cache->v_token, *cache, keys, &A.v_page_step, &A.v_head_step);
    if (map_status != EFQ_OK) return map_status;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int max_rows = group_rows < A.step * G ? static_cast<int>(group_rows) : A.step * G;       // the join's blocks; with more rows they go round
    using Bf = __nv_bfloat16;
    const bool bf = dtype == EFQ_BF16;
    const auto few = plan.rows == kFewRows ? (bf ? launch_few_rows<Bf, kFewRows> : launch_few_rows<__half, kFewRows>)
                                           : (bf ? launch_few_rows<Bf, 2 * kFewRows> : launch_few_rows<__half, 2 * kFewRows>);
    const cudaError_t e = !many ? few(mq, mk, mv, A, ctas, max_rows, dev, s)
                        : bf ? launch_chunk<Bf>(mq, mk, mv, A, ctas, dev, s) : launch_chunk<__half>(mq, mk, mv, A, ctas, dev, s);
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
