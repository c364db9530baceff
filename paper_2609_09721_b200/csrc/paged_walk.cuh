// How the kernels of the paged attention share a step's work (paged_units.h), on the device.
#pragma once

#include "paged.cuh"
#include "paged_units.h"
#include "sm100_ptx.cuh"

namespace efq {

// What the kernels get; the tables are device memory.
struct PagedArgs {
    const int32_t *page_table, *cu_seqlens, *seq_lens;
    int64_t table_stride;
    int32_t n_seqs, n_pages, max_pages, page_shift;
    int32_t Hkv, G, causal, total;
    int32_t step;                       // new tokens of a query tile
    float scale_log2;                   // softmax scale / ln 2
    char* o;
    int64_t o_token, o_head;            // bytes
    float* lse;                         // [total, Hkv * G]
    float* part_o;
    float2* part_ml;                    // maximum (of the scores times scale_log2) and sum
    struct PagedRecord* records;
    int32_t inject_skip_loads;
};

// Of a CTA that ends a query tile which an earlier one began: where its parts and its rows are.
struct PagedRecord {
    int32_t first;                      // CTA that began it; -1: nothing to join
    int32_t token0, tokens, head;
};

// Sequence s of the step as a kernel with tiles of kKeys keys sees it.
template <int kKeys>
struct PagedReader {
    const PagedArgs& A;
    __device__ __forceinline__ SeqWork operator()(int s, int& begin) const
    {
        SeqWork w;
        begin = __ldcg(A.cu_seqlens + s);
        w.lq = __ldcg(A.cu_seqlens + s + 1) - begin;
        w.len = max(0, __ldcg(A.seq_lens + s));
        if (begin < 0 || w.lq < 0 || begin > A.total - w.lq) w.lq = 0;      // not tokens of this step: nothing is read or written for it
        if (w.len > A.max_pages << A.page_shift) {
            w.none = 1;
            w.len = 0;
        }
        w.step = A.step;
        w.keys = kKeys;
        w.causal = A.causal;
        return w;
    }
};

// Called by all kThreads threads of a CTA; `scratch` holds a number for each of its warps, in shared memory.
template <int kThreads, int kKeys>
__device__ __forceinline__ void paged_find_run(const PagedArgs& A, int64_t* scratch, PagedRun* run)
{
    const PagedReader<kKeys> read{A};
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = kThreads / 32;
    const int per = (A.n_seqs + kThreads - 1) / kThreads, s0 = min(tid * per, A.n_seqs), s1 = min(s0 + per, A.n_seqs);
    int64_t mine = 0;
    int begin;
    for (int s = s0; s < s1; ++s) mine += read(s, begin).units_per_head() * A.Hkv;
    int64_t upto = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, upto, off);
        if (lane >= off) upto += x;
    }
    if (lane == 31) scratch[warp] = upto;
    if (tid == 0) run->left = 0;
    __syncthreads();
    int64_t before = upto - mine, total = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        if (i < warp) before += scratch[i];
        total += scratch[i];
    }
    const int64_t ctas = min(static_cast<int64_t>(gridDim.x), total), c = blockIdx.x;
    if (c < ctas) {
        int64_t off = paged_first_unit(total, ctas, c) - before;
        if (off >= 0 && off < mine) {
            for (int s = s0; s < s1; ++s) {
                const SeqWork w = read(s, begin);
                const int64_t units = w.units_per_head() * A.Hkv;
                if (off < units) {
                    paged_begin_run(w, s, off, total, ctas, c, run);
                    break;
                }
                off -= units;
            }
        }
    }
    __syncthreads();
}

// Keys that token i of the segment's tile sees
__device__ __forceinline__ int paged_limit(const PagedSegment& g, int i)
{
    return g.w.causal ? max(0, min(g.w.len, g.base + i + 1)) : g.w.len;
}

__device__ __forceinline__ float paged_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float kLn2 = 0.69314718055994530942f;

}  // namespace efq
