// Attention over a paged cache for few query rows: the query heads of a KV group times the new tokens are at most 16 * kM rows, kM = 1, 2.
//
// Bound by the bytes of K and V, which are read once.  One CTA an SM: a warp that loads and eight that compute.  Key tiles of 64
// come through a ring of TMA stages; four warps take a tile, 16 keys each, the other four the next one.  Scores are m16n8k16 products
// of the query rows (padded to 16) with K as it lies in shared memory, and their layout is the operand layout of the product with V, so
// probabilities stay in registers.  Every warp keeps a running maximum, sum and output of its own over the keys that it sees, and the
// eight are joined once, at the end of a query tile: no step of the loop waits for another warp.
// The warp-level MMA is the right one here: a tcgen05 tile has 128 rows, of which 4 to 32 would be used, and every tile of keys would
// pass tensor memory twice.
#pragma once

#include "paged_walk.cuh"

namespace efq {

constexpr int kFewItem = 1;                     // what a query tile costs beside its key tiles, in key tiles
constexpr int kFewShift = 6, kFewKeys = 1 << kFewShift;       // of a stage
constexpr int kFewWarps = 8;                    // that compute
constexpr int kFewThreads = (kFewWarps + 1) * 32;
constexpr int kFewHalf = kFewKeys * 128;        // bytes of 64 channels of a tile
constexpr int kFewRowPad = 136;                 // floats of a row in the join: rows start 8 banks apart

template <int kM>
struct __align__(1024) FewSmem {
    // Even, so that a stage's tiles all belong to one group of four warps: a group that skipped every other phase of a barrier could take the
    // phase before last for the last one, since loads may land in another order than they were issued in.
    static constexpr int kStages = 4;
    static_assert(kStages % 2 == 0, "a stage belongs to one group of warps");
    uint8_t k[kStages][2][kFewHalf], v[kStages][2][kFewHalf];       // [channels 0-63, 64-127], 128-byte swizzle
    uint8_t q[2][2][16 * kM * 128];
    float join_o[kFewWarps / 2][16 * kM][kFewRowPad];
    float2 join_ml[kFewWarps][16 * kM];
    float2 row_ml[16 * kM];
    uint64_t full[kStages], empty[kStages], q_full[2], q_empty[2];
    int64_t scratch[64];
    PagedRun<kFewShift, kFewItem> run;
    uint32_t bad[kStages];                      // the tile lies on an entry that is no page
    volatile uint32_t failed;
};

// Bounded waits.
__device__ __forceinline__ bool paged_poll(uint64_t* bar, uint32_t parity, volatile uint32_t* failed)
{
#pragma unroll 1
    for (int i = 0; i < 20000; ++i) {           // a second at most
        if (*failed != 0u) return false;
        if (ptx::mbar_try_wait_suspend(bar, parity, 50000u)) return true;
    }
    *failed = 1u;
    return false;
}
template <typename Smem>
__device__ __forceinline__ bool paged_wait(uint64_t* bar, uint32_t parity, Smem* sm)
{
    return ptx::mbar_try_wait(bar, parity) || paged_poll(bar, parity, &sm->failed);
}

// The same for a warp, whose lanes leave the wait together: what follows needs all of them (ldmatrix, mma, ballots).
template <typename Smem>
__device__ __forceinline__ bool paged_wait_warp(uint64_t* bar, uint32_t parity, Smem* sm)
{
    return __all_sync(0xffffffffu, paged_wait(bar, parity, sm)) != 0;
}

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(ptx::smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(ptx::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(ptx::smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(ptx::smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (sizeof(T) == 2 && __is_same(T, __nv_bfloat16))
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void few_bar() { asm volatile("bar.sync 1, 256;" ::: "memory"); }       // the warps that compute

// Loads of one tile: lane i takes the i-th page of it.  `entry`: that page's entry in the table (below zero where it is none).
template <int kStages, typename Smem>
__device__ __forceinline__ void few_load_tile(Smem* sm, int stage, const CUtensorMap& mk, const CUtensorMap& mv, const PagedArgs& A, const PagedSegment<kFewShift, kFewItem>& g,
                                              int j, int entry, int lane)
{
    const int P = 1 << A.page_shift, box = min(P, kFewKeys), key = j * kFewKeys + lane * box;
    const bool load = lane * box < kFewKeys && key < g.w.len && !A.inject_skip_loads;
    const bool none = load && entry < 0;
    const uint32_t loads = __popc(__ballot_sync(0xffffffffu, load)), bad = __ballot_sync(0xffffffffu, none);
    if (lane == 0) {
        sm->bad[stage] = bad;
        ptx::mbar_arrive_expect_tx(&sm->full[stage], (A.inject_skip_loads ? 1u : loads) * static_cast<uint32_t>(box) * 512u);
    }
    __syncwarp();
    if (load) {
        const int row = lane * box * 128, token = key & (P - 1), page = max(entry, 0);      // a bad entry marks the tile; page 0 is there
        tma_load_4d(sm->k[stage][0] + row, &mk, 0, token, g.head, page, &sm->full[stage]);
        tma_load_4d(sm->k[stage][1] + row, &mk, 64, token, g.head, page, &sm->full[stage]);
        tma_load_4d(sm->v[stage][0] + row, &mv, 0, token, g.head, page, &sm->full[stage]);
        tma_load_4d(sm->v[stage][1] + row, &mv, 64, token, g.head, page, &sm->full[stage]);
    }
}

template <typename T, int kM>
__global__ void __launch_bounds__(kFewThreads, 1)
paged_few_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                 const __grid_constant__ PagedArgs A)
{
    using Smem = FewSmem<kM>;
    constexpr int kStages = Smem::kStages, kRows = 16 * kM;
    extern __shared__ uint8_t smem_raw[];
    Smem* const sm = reinterpret_cast<Smem*>(smem_raw + ptx::smem_round_up(smem_raw, 1024u));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        sm->failed = 0u;
        for (int i = 0; i < kStages; ++i) {
            ptx::mbar_init(&sm->full[i], 1);
            ptx::mbar_init(&sm->empty[i], kFewWarps / 2);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&sm->q_full[i], 1);
            ptx::mbar_init(&sm->q_empty[i], kFewWarps);
        }
        ptx::mbar_init_fence();
        ptx::prefetch_tensormap(&mq);
        ptx::prefetch_tensormap(&mk);
        ptx::prefetch_tensormap(&mv);
    }
    ptx::grid_wait();
    ptx::grid_launch_next();
    paged_find_run<kFewThreads, kFewShift, kFewItem>(A, sm->scratch, &sm->run);      // barriers of the block
    PagedWalk<kFewShift, kFewItem, PagedReader<kFewShift, kFewItem>> walk(PagedReader<kFewShift, kFewItem>{A}, A.n_seqs, A.Hkv, sm->run);
    PagedSegment<kFewShift, kFewItem> g;

    if (warp == kFewWarps) {
        // ------------------------------------------------------------ loads
        const int P = 1 << A.page_shift, box = min(P, kFewKeys);
        uint32_t tile = 0, seg = 0;
        bool ok = true;
        while (ok && walk.next(g)) {
            const uint32_t qb = seg & 1u;
            if (seg >= 2) ok = paged_wait_warp(&sm->q_empty[qb], ((seg >> 1) - 1) & 1u, sm);
            if (!ok) break;
            if (ptx::elect_one()) {
                ptx::mbar_arrive_expect_tx(&sm->q_full[qb], static_cast<uint32_t>(A.step * A.G) * 256u);
                tma_load_3d(sm->q[qb][0], &mq, 0, g.head * A.G, g.token0, &sm->q_full[qb]);
                tma_load_3d(sm->q[qb][1], &mq, 64, g.head * A.G, g.token0, &sm->q_full[qb]);
            }
            __syncwarp();
            ++seg;
            const int32_t* row = A.page_table + g.seq * A.table_stride;
            auto entry_of = [&](int j) {
                const int key = j * kFewKeys + lane * box, at = key >> A.page_shift;
                int e = -1;
                if (lane * box < kFewKeys && key < g.w.len && at < A.max_pages) e = __ldcg(row + at);
                return e < A.n_pages ? e : -1;
            };
            int entry = entry_of(g.j0);
            for (int j = g.j0; j < g.j1; ++j, ++tile) {
                const int ahead = j + 1 < g.j1 ? entry_of(j + 1) : -1;
                const uint32_t stage = tile % kStages;
                if (tile >= kStages) ok = paged_wait_warp(&sm->empty[stage], (tile / kStages - 1) & 1u, sm);
                if (!ok) break;
                few_load_tile<kStages>(sm, stage, mk, mv, A, g, j, entry, lane);
                entry = ahead;
            }
        }
        if (lane == 0) {        // its copies in flight end before the block does, whatever the others do
            for (uint32_t i = 0; i < kStages && i < tile && !A.inject_skip_loads; ++i) {
                const uint32_t last = tile - 1 - i;
                for (int n = 0; n < 20000 && !ptx::mbar_try_wait_suspend(&sm->full[last % kStages], (last / kStages) & 1u, 50000u); ++n) {}
            }
            for (uint32_t i = 0; i < 2 && i < seg; ++i) {
                const uint32_t last = seg - 1 - i;
                for (int n = 0; n < 20000 && !ptx::mbar_try_wait_suspend(&sm->q_full[last & 1u], (last >> 1) & 1u, 50000u); ++n) {}
            }
        }
        return;
    }

    // ---------------------------------------------------------------- scores, probabilities, output
    const int sub = (warp & 3) * 16;                    // first of the warp's keys in a tile
    const uint32_t group = warp >> 2;
    const uint32_t k_row = sub + (lane & 7) + ((lane >> 4) << 3), v_row = sub + (lane & 15);
    uint32_t tile = 0, seg = 0;
    if (tid == 0) A.records[blockIdx.x].first = -1;
    while (walk.next(g)) {
        const uint32_t qb = seg & 1u;
        uint32_t qa[8][4];                              // kM = 1: the queries stay in registers; 2: they are read again for every tile
        float o[kM][16][4], m[kM][2], l[kM][2];
        bool nan = !paged_wait_warp(&sm->q_full[qb], (seg >> 1) & 1u, sm) || g.w.none != 0;
        auto load_q = [&](uint32_t (&a)[4], int mt, int ks) {
            const uint32_t r = 16 * mt + (lane & 15), c = 2 * ks + (lane >> 4);
            ldmatrix4(a, ptx::smem_u32(sm->q[qb][c >> 3]) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
        };
        if (kM == 1) {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) load_q(qa[ks], 0, ks);
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sm->q_empty[qb]);
        }
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
#pragma unroll
            for (int n = 0; n < 16; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[mt][n][i] = 0.0f;
            m[mt][0] = m[mt][1] = -INFINITY;
            l[mt][0] = l[mt][1] = 0.0f;
        }
        ++seg;
        int limit[kM][2];
        int fewest = g.w.len;                            // keys that every row sees
#pragma unroll
        for (int mt = 0; mt < kM; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i) limit[mt][i] = paged_limit(g, (16 * mt + 8 * i + (lane >> 2)) / A.G);
        if (g.w.causal) fewest = max(0, min(fewest, g.base + 1));

        for (int j = g.j0; j < g.j1; ++j, ++tile) {
            if ((tile & 1u) != group) continue;
            const uint32_t stage = tile % kStages;
            if (!paged_wait_warp(&sm->full[stage], (tile / kStages) & 1u, sm)) { nan = true; continue; }
            nan = nan || sm->bad[stage] != 0u;
            const int key0 = j * kFewKeys + sub;
            float s[kM][2][4];
#pragma unroll
            for (int mt = 0; mt < kM; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[mt][0][i] = s[mt][1][i] = 0.0f;
            const uint32_t kb = ptx::smem_u32(sm->k[stage][0]) + k_row * 128;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                const uint32_t c = 2 * ks + ((lane >> 3) & 1);
                uint32_t b[4];
                ldmatrix4(b, kb + (c >> 3) * kFewHalf + (((c & 7) ^ (k_row & 7)) << 4));
#pragma unroll
                for (int mt = 0; mt < kM; ++mt) {
                    if (kM > 1) load_q(qa[mt], mt, ks);
                    mma16816<T>(s[mt][0], qa[kM > 1 ? mt : ks], b[0], b[1]);
                    mma16816<T>(s[mt][1], qa[kM > 1 ? mt : ks], b[2], b[3]);
                }
            }
            const bool whole = key0 + 16 <= fewest;
            uint32_t p[kM][4];
#pragma unroll
            for (int mt = 0; mt < kM; ++mt) {
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = s[mt][n][i] * A.scale_log2;
                        if (!whole && key0 + 8 * n + 2 * (lane & 3) + (i & 1) >= limit[mt][i >> 1]) x = -INFINITY;
                        s[mt][n][i] = x;
                        top[i >> 1] = fmaxf(top[i >> 1], x);
                    }
                float base[2];
                bool grew = false;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                    top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
                    top[i] = fmaxf(top[i], m[mt][i]);
                    base[i] = top[i] == -INFINITY ? 0.0f : top[i];        // nothing visible yet: every exponential is 2^-inf = 0
                    grew = grew || top[i] > m[mt][i];
                }
                if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float alpha = paged_exp2(m[mt][i] - base[i]);       // m = -inf: 0
                        m[mt][i] = top[i];
                        l[mt][i] *= alpha;
#pragma unroll
                        for (int n = 0; n < 16; ++n) {
                            o[mt][n][2 * i] *= alpha;
                            o[mt][n][2 * i + 1] *= alpha;
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s[mt][n][i] = paged_exp2(s[mt][n][i] - base[i >> 1]);
                        l[mt][i >> 1] += s[mt][n][i];
                    }
                // the scores' layout is that of the left operand: probabilities are rounded once, to the elements' type (half a step of
                // 2^-8 or 2^-11 of each, its sum is kept unrounded)
                p[mt][0] = Pack2<T>::round(s[mt][0][0], s[mt][0][1]);
                p[mt][1] = Pack2<T>::round(s[mt][0][2], s[mt][0][3]);
                p[mt][2] = Pack2<T>::round(s[mt][1][0], s[mt][1][1]);
                p[mt][3] = Pack2<T>::round(s[mt][1][2], s[mt][1][3]);
            }
            // rows of V past the sequence hold whatever the page held, or what an earlier tile left: 0 times that has to be 0
            const int valid = g.w.len - key0 - 2 * (lane & 3);
            const uint32_t keep0 = valid >= 2 ? 0xffffffffu : valid == 1 ? 0xffffu : 0u, keep1 = valid >= 10 ? 0xffffffffu : valid == 9 ? 0xffffu : 0u;
            const bool inside = key0 + 16 <= g.w.len;
            const uint32_t vb = ptx::smem_u32(sm->v[stage][0]) + v_row * 128;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const uint32_t c = 2 * n + (lane >> 4);
                uint32_t b[4];
                ldmatrix4_trans(b, vb + (c >> 3) * kFewHalf + (((c & 7) ^ (v_row & 7)) << 4));
                if (!inside) {
                    b[0] &= keep0; b[1] &= keep1; b[2] &= keep0; b[3] &= keep1;
                }
#pragma unroll
                for (int mt = 0; mt < kM; ++mt) {
                    mma16816<T>(o[mt][2 * n], p[mt], b[0], b[1]);
                    mma16816<T>(o[mt][2 * n + 1], p[mt], b[2], b[3]);
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sm->empty[stage]);
        }

        if (kM > 1) {
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sm->q_empty[qb]);
        }

        // -------------------------------------------------------- the eight warps' parts of the segment
#pragma unroll
        for (int mt = 0; mt < kM; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float& x = l[mt][i];
                x += __shfl_xor_sync(0xffffffffu, x, 1);
                x += __shfl_xor_sync(0xffffffffu, x, 2);
                if (nan) x = __uint_as_float(0x7fc00000u);
                if ((lane & 3) == 0) sm->join_ml[warp][16 * mt + 8 * i + (lane >> 2)] = make_float2(m[mt][i], x);
            }
        few_bar();
#pragma unroll
        for (int mt = 0; mt < kM; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 16 * mt + 8 * i + (lane >> 2);
                float top = -INFINITY, sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kFewWarps; ++w) top = fmaxf(top, sm->join_ml[w][r].x);
                const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
                for (int w = 0; w < kFewWarps; ++w) sum += sm->join_ml[w][r].y * paged_exp2(sm->join_ml[w][r].x - base);
                const float f = paged_exp2(m[mt][i] - base);
#pragma unroll
                for (int n = 0; n < 16; ++n) {
                    o[mt][n][2 * i] *= f;
                    o[mt][n][2 * i + 1] *= f;
                    if (warp >= kFewWarps / 2)
                        *reinterpret_cast<float2*>(&sm->join_o[warp - kFewWarps / 2][r][8 * n + 2 * (lane & 3)]) = make_float2(o[mt][n][2 * i], o[mt][n][2 * i + 1]);
                }
                if (warp == 0 && (lane & 3) == 0) sm->row_ml[r] = make_float2(top, sum);
            }
        few_bar();
        if (warp < kFewWarps / 2) {
#pragma unroll
            for (int mt = 0; mt < kM; ++mt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int n = 0; n < 16; ++n) {
                        float2& x = *reinterpret_cast<float2*>(&sm->join_o[warp][16 * mt + 8 * i + (lane >> 2)][8 * n + 2 * (lane & 3)]);
                        x = make_float2(x.x + o[mt][n][2 * i], x.y + o[mt][n][2 * i + 1]);
                    }
        }
        few_bar();
        const bool all = g.j0 == 0 && g.j1 == g.n;
        const int slot = 2 * blockIdx.x + (g.j0 == 0 ? 1 : 0), rows = g.tokens * A.G;
        for (int i = tid; i < rows * 32; i += kFewWarps * 32) {
            const int r = i >> 5, c = 4 * (i & 31);
            float4 x = *reinterpret_cast<const float4*>(&sm->join_o[0][r][c]);
#pragma unroll
            for (int w = 1; w < kFewWarps / 2; ++w) {
                const float4 y = *reinterpret_cast<const float4*>(&sm->join_o[w][r][c]);
                x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
            }
            const float2 ml = sm->row_ml[r];
            if (all) {
                const int token = g.token0 + r / A.G, head = g.head * A.G + r % A.G;
                const float inv = ml.y == 0.0f ? 0.0f : 1.0f / ml.y;
                *reinterpret_cast<uint2*>(A.o + token * A.o_token + head * A.o_head + 2 * c) =
                    make_uint2(Pack2<T>::round(x.x * inv, x.y * inv), Pack2<T>::round(x.z * inv, x.w * inv));
                if (A.lse != nullptr && c == 0) A.lse[static_cast<int64_t>(token) * (A.Hkv * A.G) + head] = ml.x * kLn2 + logf(ml.y);
            } else {
                *reinterpret_cast<float4*>(A.part_o + (static_cast<int64_t>(slot) * kRows + r) * kPagedD + c) = x;
                if (c == 0) A.part_ml[slot * kRows + r] = ml;
            }
        }
        if (tid == 0 && g.j0 > 0 && g.j1 == g.n)
            A.records[blockIdx.x] = {sm->run.begins, g.token0, g.tokens, g.head};
    }
}

}  // namespace efq
