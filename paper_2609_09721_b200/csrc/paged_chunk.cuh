// Attention over a paged cache for many query rows: 128 or 256 rows of a KV group against tiles of 128 keys, on the tensor cores.
//
// A query tile is two halves of up to 128 rows (tokens of the chunk times the query heads of the KV group, whole tokens only), each with
// its scores (128 columns of tensor memory, whose first 64 take the probabilities afterwards) and its output (128 columns).  Ten warps: four
// for the softmax of each half, one that issues the MMAs, one that loads (and two that fill their group of four).  While the softmax warps of one half are busy, the tensor core
// has the other half's products: per half and tile Q K^T (both operands in shared memory), then P V (P from tensor memory).
//   - A thread has a row, so maxima and sums need no other thread.  The output is rescaled in tensor memory by the same threads,
//     only when a row's maximum has grown by more than 2^8 (kSlack); the sum refers to the same maximum, so the result is exact.  When
//     the scores of a tile are there, the product of the tile before has ended (the tensor core works in order), so nobody waits for it.
//   - K and V come through one ring of 32 KB slots, pages by TMA; 64 KB hold Q.
// Bound by the exponentials and the MMAs, which take the same time: a tile of 256 x 128 scores is 32768 exponentials at 16 a clock and
// 4 x 128 x 128 x 128 products at 4096 a clock, 2048 clocks each.
#pragma once

#include "paged_few.cuh"

namespace efq {

constexpr int kChunkKeys = 128, kChunkRows = 128;              // keys of a tile, rows of a half
constexpr int kChunkThreads = 384;
constexpr int kChunkSlots = 5;
constexpr int kChunkPart = kChunkKeys * 128;                   // bytes of 64 channels of 128 rows
constexpr uint32_t kChunkColS = 0, kChunkColO = 256;           // + 128 for the second half
constexpr float kSlack = 8.0f;                                 // log2: probabilities stay below 2^8, sums below 2^8 times the keys

struct __align__(1024) ChunkSmem {
    uint8_t q[2][2][kChunkPart];                               // half, channels 0-63 and 64-127; 128-byte swizzle
    uint8_t kv[kChunkSlots][2][kChunkPart];
    uint64_t full[kChunkSlots], empty[kChunkSlots], q_full, q_empty, s_full[2], p_ready[2], o_full[2], drained;
    int64_t scratch[kChunkThreads / 32];
    PagedRun run;
    uint32_t tmem_base;
    volatile uint32_t failed;
};

// Registers of a softmax thread, which holds a row of scores, and of the others: together what the block is launched with, 384 x 168.
constexpr int kChunkRegsMore = 216, kChunkRegsLess = 72;
static_assert(256 * kChunkRegsMore + 128 * kChunkRegsLess <= 384 * 168, "setmaxnreg draws on what the block was launched with");

template <typename T>
__device__ constexpr uint32_t chunk_idesc(bool b_n_major)
{
    return __is_same(T, __nv_bfloat16) ? ptx::bf16_idesc(128, b_n_major) : ptx::bf16_idesc(128, b_n_major) & ~((1u << 7) | (1u << 10));
}

// Of a segment: tokens of a half, and the key tiles of the run that it needs: [j0, end).
struct ChunkHalf {
    int tokens, end;
};
__device__ __forceinline__ ChunkHalf chunk_half(const PagedSegment& g, int half, int step)
{
    const int per = step >> 1;
    ChunkHalf h;
    h.tokens = max(0, min(per, g.tokens - half * per));
    const int seen = h.tokens > 0 ? paged_limit(g, half * per + h.tokens - 1) : 0;
    h.end = max(g.j0, min(g.j1, (seen + kChunkKeys - 1) / kChunkKeys));
    return h;
}

template <typename T>
__global__ void __launch_bounds__(kChunkThreads, 1)
paged_chunk_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                   const __grid_constant__ PagedArgs A)
{
    extern __shared__ uint8_t smem_raw[];
    ChunkSmem* const sm = reinterpret_cast<ChunkSmem*>(smem_raw + ptx::smem_round_up(smem_raw, 1024u));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        sm->failed = 0u;
        for (int i = 0; i < kChunkSlots; ++i) {
            ptx::mbar_init(&sm->full[i], 1);
            ptx::mbar_init(&sm->empty[i], 1);
        }
        ptx::mbar_init(&sm->q_full, 1);
        ptx::mbar_init(&sm->q_empty, 1);
        ptx::mbar_init(&sm->drained, 1);
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&sm->s_full[i], 1);
            ptx::mbar_init(&sm->p_ready[i], 4);
            ptx::mbar_init(&sm->o_full[i], 1);
        }
        ptx::mbar_init_fence();
        ptx::prefetch_tensormap(&mq);
        ptx::prefetch_tensormap(&mk);
        ptx::prefetch_tensormap(&mv);
    }
    if (warp == 8) ptx::tmem_alloc(&sm->tmem_base, 512);
    ptx::tc_fence_before_sync();
    ptx::grid_wait();
    ptx::grid_launch_next();
    paged_find_run<kChunkThreads, kChunkKeys>(A, sm->scratch, &sm->run);      // two barriers of the block
    ptx::tc_fence_after_sync();
    const uint32_t tmem = sm->tmem_base;
    PagedWalk<PagedReader<kChunkKeys>> walk(PagedReader<kChunkKeys>{A}, A.n_seqs, A.Hkv, sm->run);
    PagedSegment g;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kChunkRegsLess));
        if (warp == 9) {
            // ------------------------------------------------------------ loads
            const int P = 1 << A.page_shift, box = min(P, kChunkKeys), row = lane * box;
            uint32_t slot = 0, q_loads = 0;          // loads so far
            bool ok = true;
            while (ok && walk.next(g)) {
                const int end = max(chunk_half(g, 0, A.step).end, chunk_half(g, 1, A.step).end);
                const int32_t* table = A.page_table + g.seq * A.table_stride;
                auto entry_of = [&](int j) {
                    const int key = j * kChunkKeys + row, at = key >> A.page_shift;
                    int e = -1;
                    if (row < kChunkKeys && key < g.w.len && at < A.max_pages) e = __ldcg(table + at);
                    return e < A.n_pages ? e : -1;
                };
                // One operand of a tile: lane i takes its i-th page.  Where an entry is no page, the rows of K are NaN, which makes rows of
                // NaN of the queries that see them, and the rows of V are 0.
                auto load = [&](const CUtensorMap& map, int j, int entry, uint32_t fill) {
                    const uint32_t s = slot % kChunkSlots;
                    if (slot >= kChunkSlots) ok = paged_wait_warp(&sm->empty[s], (slot / kChunkSlots - 1) & 1u, sm);
                    if (!ok) return;
                    const int key = j * kChunkKeys + row;
                    const bool mine = row < kChunkKeys && key < g.w.len, page = mine && entry >= 0 && !A.inject_skip_loads;
                    if (mine && entry < 0) {
                        for (int i = 0; i < box * 8; ++i) {
                            reinterpret_cast<uint4*>(sm->kv[s][0] + row * 128)[i] = make_uint4(fill, fill, fill, fill);
                            reinterpret_cast<uint4*>(sm->kv[s][1] + row * 128)[i] = make_uint4(fill, fill, fill, fill);
                        }
                        ptx::fence_proxy_async_smem();
                    }
                    const uint32_t pages = __popc(__ballot_sync(0xffffffffu, page));
                    if (lane == 0) ptx::mbar_arrive_expect_tx(&sm->full[s], (A.inject_skip_loads ? 1u : pages) * static_cast<uint32_t>(box) * 256u);
                    __syncwarp();
                    if (page) {
                        tma_load_4d(sm->kv[s][0] + row * 128, &map, 0, key & (P - 1), g.head, entry, &sm->full[s]);
                        tma_load_4d(sm->kv[s][1] + row * 128, &map, 64, key & (P - 1), g.head, entry, &sm->full[s]);
                    }
                    ++slot;
                };
                int entry = end > g.j0 ? entry_of(g.j0) : -1;
                for (int j = g.j0; ok && j < end; ++j) {
                    const int ahead = j + 1 < end ? entry_of(j + 1) : -1;
                    load(mk, j, entry, 0x7fff7fffu);
                    if (ok && j == g.j0) {
                        if (q_loads > 0) ok = paged_wait_warp(&sm->q_empty, (q_loads - 1) & 1u, sm);
                        if (!ok) break;
                        if (ptx::elect_one()) {
                            const int per = A.step >> 1;
                            ptx::mbar_arrive_expect_tx(&sm->q_full, static_cast<uint32_t>(A.step * A.G) * 256u);
                            for (int i = 0; i < 4; ++i)
                                tma_load_3d(sm->q[i >> 1][i & 1], &mq, (i & 1) * 64, g.head * A.G, g.token0 + (i >> 1) * per, &sm->q_full);
                        }
                        __syncwarp();
                        ++q_loads;
                    }
                    if (ok) load(mv, j, entry, 0u);
                    entry = ahead;
                }
            }
            if (lane == 0) {        // its copies in flight end before the block does, whatever the others do
                for (uint32_t i = 0; i < kChunkSlots && i < slot && !A.inject_skip_loads; ++i) {
                    const uint32_t last = slot - 1 - i;
                    for (int n = 0; n < 20000 && !ptx::mbar_try_wait_suspend(&sm->full[last % kChunkSlots], (last / kChunkSlots) & 1u, 50000u); ++n) {}
                }
                for (int n = 0; n < 20000 && q_loads > 0 && !ptx::mbar_try_wait_suspend(&sm->q_full, (q_loads - 1) & 1u, 50000u); ++n) {}
            }
        } else if (warp == 8) {
            // ------------------------------------------------------------ MMAs
            uint32_t slot = 0, q_loads = 0, p_count[2] = {0, 0};
            bool ok = true;
            auto wait_slot = [&](uint32_t s) { return paged_wait_warp(&sm->full[s % kChunkSlots], (s / kChunkSlots) & 1u, sm); };
            auto scores = [&](int w, uint32_t s) {
                const uint64_t da = ptx::smem_desc(ptx::smem_u32(sm->q[w][0]), 16, 1024, ptx::kLayoutSw128);
                const uint64_t db = ptx::smem_desc(ptx::smem_u32(sm->kv[s % kChunkSlots][0]), 16, 1024, ptx::kLayoutSw128);
                if (ptx::elect_one()) {
    #pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint64_t off = static_cast<uint64_t>(((i >> 2) * kChunkPart + (i & 3) * 32) >> 4);
                        ptx::mma_bf16(tmem + kChunkColS + 128 * w, da + off, db + off, chunk_idesc<T>(false), i > 0 ? 1u : 0u);
                    }
                    ptx::mma_commit(&sm->s_full[w]);
                }
                __syncwarp();
            };
            while (ok && walk.next(g)) {
                const int e0 = chunk_half(g, 0, A.step).end, e1 = chunk_half(g, 1, A.step).end, end = max(e0, e1);
                if (end == g.j0) continue;
                ok = wait_slot(slot) && paged_wait_warp(&sm->q_full, q_loads & 1u, sm);
                if (!ok) break;
                ++q_loads;
                ptx::tc_fence_after_sync();
                if (g.j0 < e0) scores(0, slot);
                if (g.j0 < e1) scores(1, slot);
                if (ptx::elect_one()) {
                    ptx::mma_commit(&sm->empty[slot % kChunkSlots]);
                    if (g.j0 + 1 == end) ptx::mma_commit(&sm->q_empty);
                }
                __syncwarp();
                ++slot;
                for (int j = g.j0; ok && j < end; ++j) {
                    const uint32_t v_slot = slot, k_slot = slot + 1;
                    const bool more = j + 1 < end;
                    ok = wait_slot(v_slot) && (!more || wait_slot(k_slot));
                    if (!ok) break;
                    slot += more ? 2 : 1;
                    const int inside = g.w.len - j * kChunkKeys;
                    if (inside < kChunkKeys) {      // rows of V past the sequence hold whatever the page held: 0 times that has to be 0
                        uint8_t* const v = sm->kv[v_slot % kChunkSlots][0];
                        for (int i = inside * 8 + lane; i < kChunkKeys * 8; i += 32) {
                            reinterpret_cast<uint4*>(v)[i] = make_uint4(0u, 0u, 0u, 0u);
                            reinterpret_cast<uint4*>(v + kChunkPart)[i] = make_uint4(0u, 0u, 0u, 0u);
                        }
                        ptx::fence_proxy_async_smem();
                        __syncwarp();
                    }
                    const uint64_t dv = ptx::smem_desc(ptx::smem_u32(sm->kv[v_slot % kChunkSlots][0]), kChunkPart, 1024, ptx::kLayoutSw128);
    #pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int e = w == 0 ? e0 : e1;
                        if (!ok || j >= e) continue;
                        ok = paged_wait_warp(&sm->p_ready[w], p_count[w] & 1u, sm);
                        if (!ok) continue;
                        ++p_count[w];
                        ptx::tc_fence_after_sync();
                        if (ptx::elect_one()) {
    #pragma unroll
                            for (int i = 0; i < 8; ++i)
                                ptx::mma_bf16_ts(tmem + kChunkColO + 128 * w, tmem + kChunkColS + 128 * w + 8 * i, dv + static_cast<uint64_t>(i * 2048 >> 4),
                                                 chunk_idesc<T>(true), i > 0 || j > g.j0 ? 1u : 0u);
                            if (j + 1 == e) ptx::mma_commit(&sm->o_full[w]);
                        }
                        __syncwarp();
                        if (j + 1 < e) scores(w, k_slot);
                    }
                    if (!ok) break;
                    if (ptx::elect_one()) {
                        ptx::mma_commit(&sm->empty[v_slot % kChunkSlots]);
                        if (more) ptx::mma_commit(&sm->empty[k_slot % kChunkSlots]);
                        if (j + 2 == end) ptx::mma_commit(&sm->q_empty);
                    }
                    __syncwarp();
                }
            }
            if (!ok) {              // the MMAs that were issued end before tensor memory is given back
                if (ptx::elect_one()) ptx::mma_commit(&sm->drained);
                __syncwarp();
                for (int n = 0; n < 20000 && !ptx::mbar_try_wait_suspend(&sm->drained, 0u, 50000u); ++n) {}
                __syncwarp();
            }
        }
    } else {
        // ------------------------------------------------------------ softmax of a half's rows, output
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kChunkRegsMore));
        const int w = warp >> 2, r = (warp & 3) * 32 + lane, per = A.step >> 1;
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_col = tmem + lane_base + kChunkColS + 128 * w, o_col = tmem + lane_base + kChunkColO + 128 * w;
        const int i = w * per + r / A.G;         // token of the tile
        uint32_t s_count = 0, o_count = 0;
        if (tid == 0) A.records[blockIdx.x].first = -1;
        while (walk.next(g)) {
            const ChunkHalf h = chunk_half(g, w, A.step);
            const bool mine = r < h.tokens * A.G;
            const int limit = paged_limit(g, i);
            const int fewest = h.tokens > 0 ? paged_limit(g, w * per) : 0;      // keys that every row of the half sees
            bool nan = g.w.none != 0;
            float m = -INFINITY, l = 0.0f;
            for (int j = g.j0; j < h.end; ++j) {
                if (!paged_wait_warp(&sm->s_full[w], s_count & 1u, sm)) { nan = true; break; }
                ++s_count;
                ptx::tc_fence_after_sync();
                float s[128];
                ptx::tmem_ld32f<0>(s_col, s);
                ptx::tmem_ld32f<32>(s_col + 32, s);
                ptx::tmem_ld32f<64>(s_col + 64, s);
                ptx::tmem_ld32f<96>(s_col + 96, s);
                ptx::tmem_wait_ld();
                if ((j + 1) * kChunkKeys > fewest) {
                    const int seen = limit - j * kChunkKeys;
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c < seen ? s[c] : -INFINITY;
                }
                float top[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) top[c] = s[c];
#pragma unroll
                for (int c = 4; c < 128; ++c) top[c & 3] = fmaxf(top[c & 3], s[c]);
                const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * A.scale_log2;
                const bool grew = mx > m + kSlack || (m == -INFINITY && mx > m);
                if (__any_sync(0xffffffffu, grew)) {
                    const float alpha = grew ? (m == -INFINITY ? 0.0f : paged_exp2(m - mx)) : 1.0f;
                    if (grew) m = mx;
                    l *= alpha;
                    if (j > g.j0) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float o[32];
                            uint32_t u[32];
                            ptx::tmem_ld32f<0>(o_col + 32 * q, o);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 32; ++c) u[c] = __float_as_uint(o[c] * alpha);
                            ptx::tmem_st32<0>(o_col + 32 * q, u);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.0f : m;        // nothing visible yet: every exponential is 2^-inf = 0
                float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t p[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        const float p0 = paged_exp2(fmaf(s[64 * q + 2 * c], A.scale_log2, -base)), p1 = paged_exp2(fmaf(s[64 * q + 2 * c + 1], A.scale_log2, -base));
                        sum[(2 * c) & 3] += p0;
                        sum[(2 * c + 1) & 3] += p1;
                        // rounded once, to the elements' type (half a step of 2^-8 or 2^-11 of each); the sum is kept unrounded
                        p[c] = Pack2<T>::round(p0, p1);
                    }
                    ptx::tmem_st32<0>(s_col + 32 * q, p);
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                ptx::tmem_wait_st();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sm->p_ready[w]);
            }

            const bool some = h.end > g.j0, all = g.j0 == 0 && g.j1 == g.n;
            if (some && !nan) {
                nan = !paged_wait_warp(&sm->o_full[w], o_count & 1u, sm);
                ++o_count;
                ptx::tc_fence_after_sync();
            }
            if (nan) l = __uint_as_float(0x7fc00000u);
            const int token = g.token0 + i, head = g.head * A.G + r % A.G, slot = 2 * blockIdx.x + (g.j0 == 0 ? 1 : 0);
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            char* const dst = A.o + token * A.o_token + head * A.o_head;
            float4* const part = reinterpret_cast<float4*>(A.part_o + (static_cast<int64_t>(slot) * 2 * kChunkRows + w * kChunkRows + r) * kPagedD);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float o[32];
                if (some && !nan) {
                    ptx::tmem_ld32f<0>(o_col + 32 * q, o);
                    ptx::tmem_wait_ld();
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) o[c] = 0.0f;
                }
                if (mine && all) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        reinterpret_cast<uint4*>(dst)[4 * q + c] = make_uint4(Pack2<T>::round(o[8 * c] * inv, o[8 * c + 1] * inv), Pack2<T>::round(o[8 * c + 2] * inv, o[8 * c + 3] * inv),
                                                                             Pack2<T>::round(o[8 * c + 4] * inv, o[8 * c + 5] * inv), Pack2<T>::round(o[8 * c + 6] * inv, o[8 * c + 7] * inv));
                } else if (mine) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) part[8 * q + c] = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
                }
            }
            ptx::tc_fence_before_sync();
            if (mine && all && A.lse != nullptr) A.lse[static_cast<int64_t>(token) * (A.Hkv * A.G) + head] = m * kLn2 + logf(l);
            if (mine && !all) A.part_ml[slot * 2 * kChunkRows + w * kChunkRows + r] = make_float2(m, l);
            if (tid == 0 && g.j0 > 0 && g.j1 == g.n) A.records[blockIdx.x] = {sm->run.begins, g.token0, g.tokens, g.head};
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 8) ptx::tmem_dealloc(tmem, 512);
}

}  // namespace efq
