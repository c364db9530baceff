// How the kernels of the paged attention share a step's work (paged_units.h), on the device.
#pragma once

#include "efq_internal.cuh"
#include "paged.cuh"
#include "paged_units.h"
#include "sm100_ptx.cuh"

namespace efq {

// Of a CTA that ends a query tile which an earlier one began: where its parts and its rows are.
struct __align__(16) PagedRecord {
    int32_t first;                      // CTA that began it; -1: nothing to join
    int32_t token0, tokens, head;
};

// What the kernels get; the tables are device memory.
struct PagedArgs {
    const int32_t *page_table, *cu_seqlens, *seq_lens;
    int64_t table_stride;
    int32_t n_seqs, n_pages, max_pages, page_shift;
    int32_t k_page_step, k_head_step, v_page_step, v_head_step;      // of the copies' last coordinate
    int32_t Hkv, G, causal, total;
    int32_t step;                       // new tokens of a query tile
    float scale_log2;                   // softmax scale / ln 2
    char* o;
    int64_t o_token, o_head;            // bytes
    int32_t o_wide;                     // rows of o lie on 32 bytes
    float* lse;                         // [total, Hkv * G]
    float* part_o;
    float2* part_ml;                    // maximum (of the scores times scale_log2) and sum
    PagedRecord* records;
    uint32_t* header;                   // of the workspace: kPagedStatus, the number of CTAs
    uint32_t* expired;                  // of every CTA: a bounded wait has run out there
    int32_t inject_skip_loads;
};

// Sequence s of the step.
template <int kShift, int kItem>
struct PagedReader {
    const PagedArgs& A;
    __device__ __forceinline__ void operator()(int s, SeqWork<kShift, kItem>& w, int& begin) const
    {
        begin = __ldcg(A.cu_seqlens + s);
        int lq = __ldcg(A.cu_seqlens + s + 1) - begin, len = max(0, __ldcg(A.seq_lens + s));
        if (begin < 0 || lq < 0 || begin > A.total - lq) lq = 0;      // not tokens of this step: nothing is read or written for it
        const bool none = len > A.max_pages << A.page_shift;
        w.set(lq, none ? 0 : len, A.step, A.causal, none ? 1 : 0);
    }
};

// Called by all kThreads threads of a CTA; `scratch` holds a number for each of its warps, in shared memory.  A thread takes a sequence, or several
// where there are more of them than threads.  Up to 32 sequences every warp adds them up for itself, which saves a barrier; a sequence
// of one query tile has its tile at hand.  Some 3400 clocks, of which 2000 are the first loads after the launch.
template <int kThreads, int kShift, int kItem>
__device__ __noinline__ void paged_find_run(const PagedArgs& A, uint32_t* scratch, PagedRun<kShift, kItem>* run)
{
    const PagedReader<kShift, kItem> read{A};
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = kThreads / 32;
    const bool by_warp = A.n_seqs <= 32;
    const int rank = by_warp ? lane : tid, per = A.n_seqs <= kThreads ? 1 : (A.n_seqs + kThreads - 1) / kThreads;
    const int s0 = min(rank * per, A.n_seqs), s1 = min(s0 + per, A.n_seqs);
    uint32_t mine = 0, per_head = 0;
    int begin = 0;
    SeqWork<kShift, kItem> w;
    for (int s = s0; s < s1; ++s) {
        read(s, w, begin);
        per_head = static_cast<uint32_t>(w.units_per_head());
        mine += per_head * static_cast<uint32_t>(A.Hkv);
    }
    uint32_t upto = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, off);
        if (lane >= off) upto += x;
    }
    uint32_t before = upto - mine, total = 0;
    if (by_warp) {
        total = __shfl_sync(0xffffffffu, upto, 31);
    } else {
        if (lane == 31) scratch[warp] = upto;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            if (i < warp) before += scratch[i];
            total += scratch[i];
        }
    }
    const uint32_t ctas = min(gridDim.x, total), c = blockIdx.x;
    if (c >= ctas) {                          // the whole block
        if (tid == 0) run->left = 0;
        __syncthreads();
        return;
    }
    const PagedShares shares(total, ctas);
    uint32_t off = shares.first(c) - before;          // wraps to a large number where the run begins before
    if (off < mine && (warp == 0 || !by_warp)) {
        int s = s0;
        for (; per > 1 && s < s1; ++s) {      // with one sequence a thread it is at hand
            read(s, w, begin);
            per_head = static_cast<uint32_t>(w.units_per_head());
            const uint32_t units = per_head * static_cast<uint32_t>(A.Hkv);
            if (off < units) break;
            off -= units;
        }
        paged_begin_run(w, s, begin, per_head, off, shares, c, run);
        if (w.tiles == 1) paged_begin_tile(0, shares, c, run);
    }
    __syncthreads();
    const int tiles = run->w.tiles;
    if (tiles == 1) return;
    for (int i = tid; i < tiles; i += kThreads)
        if (paged_begin_tile(i, shares, c, run)) break;
    __syncthreads();
}

// What a CTA leaves before its waits: called by one thread, and a barrier of the block has to follow.
__device__ __forceinline__ void paged_begin_status(const PagedArgs& A)
{
    A.expired[blockIdx.x] = 0u;
    A.records[blockIdx.x].first = -1;
    if (blockIdx.x == 0) *reinterpret_cast<uint2*>(A.header) = make_uint2(kPagedStatus, gridDim.x);
}

// Keys that token i of the segment's tile sees
template <int kShift, int kItem>
__device__ __forceinline__ int paged_limit(const PagedSegment<kShift, kItem>& g, int i)
{
    return g.w.causal ? max(0, min(g.w.len, g.base + i + 1)) : g.w.len;
}

__device__ __forceinline__ float paged_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The exponent of a row's probabilities for the product with V is raised by 2^raise over what it is under the row's maximum: fp16 is exact to half a
// step of 2^-11 from 2^-14 on only, to 2^-25 below, and ends at 65504.  What the maximum is kept as is lower by as much, so sums, parts and lse need to
// know nothing of it.  Rounded up, so that a probability is at most 2^raise wherever the maximum lies.
template <typename T> constexpr bool kNarrowExponent = sizeof(T) == 2 && __is_same(T, __half);
__device__ __forceinline__ float paged_reference(float top, float raise) { return raise == 0.0f ? top : __fadd_ru(top, -raise); }

constexpr float kLn2 = 0.69314718055994530942f;

}  // namespace efq
