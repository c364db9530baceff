// Attention over a paged cache for few query rows: the query heads of a KV group times the new tokens are at most 32 rows.
//
// Bound by the bytes of K and V, which are read once: 64 sequences of one token on 4096 to 8192 keys (32 / 8 heads) 244 us, 98 % of the measured copy rate.
// One CTA an SM: a warp that loads and eight that compute.  Key tiles of 64 come through a ring of TMA stages; four warps take a tile, the other
// four the next one.  With up to 16 rows each has 16 of the keys; with up to 32 two have the first 16 rows and two the others, 32 keys each
// (16 keys and all eight warps at one tile: 16 sequences of five tokens 75.3 us and 70.1, half as many reductions, twice as many products at a time).
// Scores are m16n8k16 products of the query rows (padded to 16) with K as it lies in shared memory, and their layout is the operand layout of the
// product with V, so probabilities stay in registers.  Every warp keeps a running maximum, sum and output of its own over the keys that it sees, and
// they are joined once, at the end of a query tile: no step of the loop waits for another warp.
// The warp-level MMA is the right one here: a tcgen05 tile has 128 rows, of which 1 to 32 would be used, and every tile of keys would
// pass tensor memory twice; a quarter of the issue slots and a fifth of the tensor cycles are taken at the rate above.
// Short contexts are bound by the end of a query tile (two tiles and their join in some 5000 clocks): 512 tokens on 100 keys each 72 us of 32.
#pragma once

#include "paged_walk.cuh"

namespace efq {

constexpr int kFewKeys = 1 << kFewShift;        // of a stage
constexpr int kFewWarps = 8;                    // that compute
constexpr int kFewThreads = (kFewWarps + 1) * 32;
constexpr int kFewRows = 16;                     // of a product; a query tile has 16 or 32 rows
constexpr int kFewRowPad = 136;                 // floats of a row in the join: rows start 8 banks apart
constexpr int kNoKey = 0x7fffffff;
// log2 of the largest probability.  fp16: those down to 2^-29 of the row's maximum keep all their bits, smaller ones are off by up to 2^-40 of it.
template <typename T> constexpr float kFewRaise = kNarrowExponent<T> ? 15.0f : 0.0f;

template <int kRows>
struct __align__(1024) FewSmem {
    static constexpr bool kExpired = true;      // an expired wait is told at once (at the end of the block: 512 tokens on 100 keys each 1 us more)
    // Even, so that a stage's tiles all belong to one group of four warps: a group that skipped every other phase of a barrier could take the
    // phase before last for the last one, since loads may land in another order than they were issued in.
    static constexpr int kStages = 4;
    static_assert(kStages % 2 == 0, "a stage belongs to one group of warps");
    static constexpr int kPeers = kFewWarps * kFewRows / kRows;         // warps that share a row's keys
    uint8_t k[kStages][kFewKeys * 256], v[kStages][kFewKeys * 256];     // [8 tokens][channels 0-63, 64-127][token], 128-byte swizzle
    uint8_t q[2][2][kRows * 128];                                       // [channels 0-63, 64-127][row]
    float join_o[kPeers / 2][kRows][kFewRowPad];
    float2 join_ml[kPeers][kRows];
    float2 row_ml[kRows];
    uint64_t full[kStages], empty[kStages], q_full[2], q_empty[2];
    uint32_t scratch[kFewThreads / 32];
    PagedRun<kFewShift, kFewItem> run;
    int32_t bad[kStages];                       // the tile's first key that lies on an entry that is no page; kNoKey: all its entries are pages
    volatile uint32_t failed;
    uint32_t* expired;                          // where the call's status has this block
};

// Bounded waits.
__device__ __forceinline__ bool paged_poll(uint64_t* bar, uint32_t parity, volatile uint32_t* failed, uint32_t* expired)
{
#pragma unroll 1
    for (int i = 0; i < 20000; ++i) {           // a second at most
        if (*failed != 0u) return false;
        if (ptx::mbar_try_wait_suspend(bar, parity, 50000u)) return true;
    }
    *failed = 1u;
    if (expired != nullptr) *expired = 1u;
    return false;
}
template <typename Smem>
__device__ __forceinline__ bool paged_wait(uint64_t* bar, uint32_t parity, Smem* sm)
{
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if constexpr (Smem::kExpired) return paged_poll(bar, parity, &sm->failed, sm->expired);
    else return paged_poll(bar, parity, &sm->failed, nullptr);
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
// A page, or a part of one, of one head: box of 64 channels x 8 tokens x 2 halves of the channels x groups of 8 tokens, so that a page is one copy
// and not one for each half of its channels: a copy of 2 KB costs the copy engine 90 to 120 clocks, one of 4 KB 125 (pages of 16 tokens, 32 KB in
// 1440 to 1880 clocks with two copies a page and 1000 to 1170 with one; at 6.5 TB/s every SM gets 32 KB in 1400).
__device__ __forceinline__ void tma_load_page(void* dst, const CUtensorMap* map, int group, int place, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %3, %4}], [%5];"
                 ::"r"(ptx::smem_u32(dst)), "l"(map), "r"(0), "r"(group), "r"(place), "r"(ptx::smem_u32(bar)) : "memory");
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

// Loads of one tile: of its pages' lanes the first half take K and the others V.  `entry`: that page's entry in the table (below zero where it is none).
template <typename Smem>
__device__ __forceinline__ void few_load_tile(Smem* sm, int stage, const CUtensorMap& mk, const CUtensorMap& mv, const PagedArgs& A, const PagedSegment<kFewShift, kFewItem>& g,
                                              int j, int entry, int lane)
{
    const int P = 1 << A.page_shift, box = min(P, kFewKeys), pages = kFewKeys / box, row = (lane & (pages - 1)) * box, key = j * kFewKeys + row;
    const bool load = lane < 2 * pages && key < g.w.len && !A.inject_skip_loads, is_v = lane >= pages;
    const uint32_t loads = __popc(__ballot_sync(0xffffffffu, load));
    const int bad = __reduce_min_sync(0xffffffffu, load && entry < 0 ? key : kNoKey);       // (lane 0 alone, from a ballot: one token on 8191 13.7 us, 13.4)
    if (lane == 0) {
        sm->bad[stage] = bad;
        ptx::mbar_arrive_expect_tx(&sm->full[stage], (A.inject_skip_loads ? 1u : loads) * static_cast<uint32_t>(box) * 256u);
    }
    __syncwarp();
    if (load)       // in the place of a bad entry comes page 0, which is there
        tma_load_page((is_v ? sm->v[stage] : sm->k[stage]) + row * 256, is_v ? &mv : &mk, (key & (P - 1)) >> 3,
                      max(entry, 0) * (is_v ? A.v_page_step : A.k_page_step) + g.head * (is_v ? A.v_head_step : A.k_head_step), &sm->full[stage]);
}

template <typename T, int kRows>
__global__ void __launch_bounds__(kFewThreads, 1)
paged_few_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                 const __grid_constant__ PagedArgs A)
{
    static_assert(kRows == kFewRows || kRows == 2 * kFewRows, "the two groups of four warps");
    using Smem = FewSmem<kRows>;
    constexpr int kStages = Smem::kStages, kPeers = Smem::kPeers;
    extern __shared__ uint8_t smem_raw[];
    Smem* const sm = reinterpret_cast<Smem*>(smem_raw + ptx::smem_round_up(smem_raw, 1024u));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        sm->failed = 0u;
        sm->expired = A.expired + blockIdx.x;
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
    if (tid == kFewWarps * 32) paged_begin_status(A);
    paged_find_run<kFewThreads, kFewShift, kFewItem>(A, sm->scratch, &sm->run);      // barriers of the block
    PagedWalk<kFewShift, kFewItem, PagedReader<kFewShift, kFewItem>> walk(PagedReader<kFewShift, kFewItem>{A}, A.n_seqs, A.Hkv, sm->run);
    PagedSegment<kFewShift, kFewItem> g;

    if (warp == kFewWarps) {
        // ------------------------------------------------------------ loads
        const int P = 1 << A.page_shift, box = min(P, kFewKeys), pages = kFewKeys / box, row = (lane & (pages - 1)) * box;
        uint32_t tile = 0, seg = 0;
        bool ok = true;
        while (ok && walk.next(g)) {
            const uint32_t qb = seg & 1u;
            const int32_t* table = A.page_table + g.seq * A.table_stride;
            // as it stands in the table: it is looked at when the tile after the next is loaded, so that nobody waits for it here
            auto entry_of = [&](int j) {
                const int key = j * kFewKeys + row;
                int e = -1;
                if (lane < 2 * pages && j < g.j1 && key < g.w.len) e = __ldcg(table + (key >> A.page_shift));
                return e;
            };
            int entry = entry_of(g.j0), next = entry_of(g.j0 + 1);
            if (seg >= 2) ok = paged_wait_warp(&sm->q_empty[qb], ((seg >> 1) - 1) & 1u, sm);
            if (!ok) break;
            if (ptx::elect_one()) {
                ptx::mbar_arrive_expect_tx(&sm->q_full[qb], static_cast<uint32_t>(A.step * A.G) * 256u);
                tma_load_3d(sm->q[qb][0], &mq, 0, g.head * A.G, g.token0, &sm->q_full[qb]);
                tma_load_3d(sm->q[qb][1], &mq, 64, g.head * A.G, g.token0, &sm->q_full[qb]);
            }
            __syncwarp();
            ++seg;
            for (int j = g.j0; j < g.j1; ++j, ++tile) {
                const int ahead = entry_of(j + 2);
                const uint32_t stage = tile % kStages;
                if (tile >= kStages) ok = paged_wait_warp(&sm->empty[stage], (tile / kStages - 1) & 1u, sm);
                if (!ok) break;
                few_load_tile(sm, stage, mk, mv, A, g, j, entry < A.n_pages ? entry : -1, lane);
                entry = next;
                next = ahead;
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
    // Of the four warps of a tile each has 16 rows, and 16 of the tile's keys, or 32 where there are 32 rows.
    constexpr int kWide = kRows / kFewRows, kKeys = 16 * kWide, kSplit = 4 / kWide;
    const uint32_t group = warp >> 2;
    const int sub = (warp % kSplit) * kKeys;            // first of the warp's keys in a tile
    const int row0 = (warp & 3) / kSplit * 16, peer = static_cast<int>(group) * kSplit + warp % kSplit;      // its rows; its place among those that share them
    // the lane's row of a matrix of K (8 keys x 16 bytes) and of V; both have the swizzle of lane & 7
    const uint32_t k_at = ((sub >> 3) + (lane >> 4)) * 2048 + (lane & 7) * 128, v_at = ((sub >> 3) + ((lane >> 3) & 1)) * 2048 + (lane & 7) * 128;
    uint32_t tile = 0, seg = 0;
    while (walk.next(g)) {
        const uint32_t qb = seg & 1u;
        uint32_t qa[8][4];
        float o[16][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
        bool nan = !paged_wait_warp(&sm->q_full[qb], (seg >> 1) & 1u, sm) || g.w.none != 0;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            const uint32_t r = row0 + (lane & 15), c = 2 * ks + (lane >> 4);
            ldmatrix4(qa[ks], ptx::smem_u32(sm->q[qb][c >> 3]) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sm->q_empty[qb]);
#pragma unroll
        for (int n = 0; n < 16; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
        ++seg;
        const int limit[2] = {paged_limit(g, (row0 + (lane >> 2)) / A.G), paged_limit(g, (row0 + 8 + (lane >> 2)) / A.G)};
        const int fewest = paged_limit(g, 0);            // keys that every row sees
        const bool idle = row0 >= g.tokens * A.G;        // no rows of the tile for this warp
        int bad = kNoKey;                                // the first key of those so far that lies on no page: rows that see it are NaN, and no others

        for (int j = g.j0; j < g.j1; ++j, ++tile) {
            if ((tile & 1u) != group) continue;
            const uint32_t stage = tile % kStages;
            if (!paged_wait_warp(&sm->full[stage], (tile / kStages) & 1u, sm)) { nan = true; continue; }
            if (idle) {
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sm->empty[stage]);
                continue;
            }
            bad = min(bad, sm->bad[stage]);
            const int key0 = j * kFewKeys + sub;
            const int values = min(g.w.len, bad);        // keys whose values there are
            float s[2 * kWide][4];
#pragma unroll
            for (int n = 0; n < 2 * kWide; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][i] = 0.0f;
            const uint32_t kb = ptx::smem_u32(sm->k[stage]) + k_at;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                const uint32_t c = 2 * ks + ((lane >> 3) & 1);
#pragma unroll
                for (int h = 0; h < kWide; ++h) {
                    uint32_t b[4];
                    ldmatrix4(b, kb + h * 4096 + (c >> 3) * 1024 + (((c & 7) ^ (lane & 7)) << 4));
                    mma16816<T>(s[2 * h], qa[ks], b[0], b[1]);
                    mma16816<T>(s[2 * h + 1], qa[ks], b[2], b[3]);
                }
            }
            const bool whole = key0 + kKeys <= fewest;
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int n = 0; n < 2 * kWide; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = s[n][i] * A.scale_log2;
                    if (!whole && key0 + 8 * n + 2 * (lane & 3) + (i & 1) >= limit[i >> 1]) x = -INFINITY;
                    s[n][i] = x;
                    top[i >> 1] = fmaxf(top[i >> 1], x);
                }
            float base[2];
            bool grew = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
                top[i] = fmaxf(paged_reference(top[i], kFewRaise<T>), m[i]);
                base[i] = top[i] == -INFINITY ? 0.0f : top[i];        // nothing visible yet: every exponential is 2^-inf = 0
                grew = grew || top[i] > m[i];
            }
            if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float alpha = paged_exp2(m[i] - base[i]);       // m = -inf: 0
                    m[i] = top[i];
                    l[i] *= alpha;
#pragma unroll
                    for (int n = 0; n < 16; ++n) {
                        o[n][2 * i] *= alpha;
                        o[n][2 * i + 1] *= alpha;
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < 2 * kWide; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[n][i] = paged_exp2(s[n][i] - base[i >> 1]);
                    l[i >> 1] += s[n][i];
                }
            const uint32_t vb = ptx::smem_u32(sm->v[stage]) + v_at;
#pragma unroll
            for (int h = 0; h < kWide; ++h) {
                // the scores' layout is that of the left operand: probabilities are rounded once, to the elements' type (off by up to 2^-8 or
                // 2^-11 of each, and kFewRaise; their sum is kept unrounded)
                const uint32_t p[4] = {Pack2<T>::round(s[2 * h][0], s[2 * h][1]), Pack2<T>::round(s[2 * h][2], s[2 * h][3]),
                                       Pack2<T>::round(s[2 * h + 1][0], s[2 * h + 1][1]), Pack2<T>::round(s[2 * h + 1][2], s[2 * h + 1][3])};
                // rows of V past the sequence, or on no page, hold whatever some page held, or what an earlier tile left: 0 times that has to be 0
                const int key = key0 + 16 * h, valid = values - key - 2 * (lane & 3);
                const uint32_t keep0 = valid >= 2 ? 0xffffffffu : valid == 1 ? 0xffffu : 0u, keep1 = valid >= 10 ? 0xffffffffu : valid == 9 ? 0xffffu : 0u;
                const bool inside = key + 16 <= values;
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const uint32_t c = 2 * n + (lane >> 4);
                    uint32_t b[4];
                    ldmatrix4_trans(b, vb + h * 4096 + (c >> 3) * 1024 + (((c & 7) ^ (lane & 7)) << 4));
                    if (!inside) {
                        b[0] &= keep0; b[1] &= keep1; b[2] &= keep0; b[3] &= keep1;
                    }
                    mma16816<T>(o[2 * n], p, b[0], b[1]);
                    mma16816<T>(o[2 * n + 1], p, b[2], b[3]);
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sm->empty[stage]);
        }

        // -------------------------------------------------------- the parts of the segment of the warps that share its rows
        nan = nan || sm->failed != 0u;          // once a wait has expired the parities of the later ones mean nothing
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float& x = l[i];
            x += __shfl_xor_sync(0xffffffffu, x, 1);
            x += __shfl_xor_sync(0xffffffffu, x, 2);
            if (nan || limit[i] > bad) x = __uint_as_float(0x7fc00000u);
            if ((lane & 3) == 0) sm->join_ml[peer][row0 + 8 * i + (lane >> 2)] = make_float2(m[i], x);
        }
        few_bar();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (row0 + 8 * i >= g.tokens * A.G) continue;      // rows that no query has (512 tokens on 100 keys each 79.3 us without this, 72.0 with)
            const int r = row0 + 8 * i + (lane >> 2);
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kPeers; ++w) top = fmaxf(top, sm->join_ml[w][r].x);
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < kPeers; ++w) sum += sm->join_ml[w][r].y * paged_exp2(sm->join_ml[w][r].x - base);
            const float f = paged_exp2(m[i] - base);
#pragma unroll
            for (int n = 0; n < 16; ++n) {
                o[n][2 * i] *= f;
                o[n][2 * i + 1] *= f;
                if (peer >= kPeers / 2)
                    *reinterpret_cast<float2*>(&sm->join_o[peer - kPeers / 2][r][8 * n + 2 * (lane & 3)]) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
            }
            if (peer == 0 && (lane & 3) == 0) sm->row_ml[r] = make_float2(top, sum);
        }
        few_bar();
        if (peer < kPeers / 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (row0 + 8 * i >= g.tokens * A.G) continue;
#pragma unroll
                for (int n = 0; n < 16; ++n) {
                    float2& x = *reinterpret_cast<float2*>(&sm->join_o[peer][row0 + 8 * i + (lane >> 2)][8 * n + 2 * (lane & 3)]);
                    x = make_float2(x.x + o[n][2 * i], x.y + o[n][2 * i + 1]);
                }
            }
        }
        few_bar();
        const bool all = g.j0 == 0 && g.j1 == g.n;
        const int slot = 2 * blockIdx.x + (g.j0 == 0 ? 1 : 0), rows = g.tokens * A.G;
        for (int i = tid; i < rows * 32; i += kFewWarps * 32) {
            const int r = i >> 5, c = 4 * (i & 31);
            float4 x = *reinterpret_cast<const float4*>(&sm->join_o[0][r][c]);
#pragma unroll
            for (int w = 1; w < kPeers / 2; ++w) {
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
