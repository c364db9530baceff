// Attention over a paged cache for many query rows: 128 or 256 rows of a KV group against tiles of 128 keys, on the tensor cores.
//
// A query tile is two halves of up to 128 rows (tokens of the chunk times the query heads of the KV group, whole tokens only), each with
// its scores (128 columns of tensor memory, whose first 64 take the probabilities afterwards) and its output (128 columns).  Twelve warps: four
// for the softmax of each half, one for each half that issues its MMAs, one that loads and tells the others what comes next, one that clears rows
// of V past a sequence.  While the softmax warps of one half are busy, the tensor core has the other half's products: per half and tile Q K^T (both
// operands in shared memory), then P V (P from tensor memory).
//   - A thread has a row, so maxima and sums need no other thread.  The output is rescaled in tensor memory by the same threads,
//     only when a row's maximum has grown by more than 2^14 (2^9 in fp16, kSlack); the sum refers to the same maximum, so the result is exact.  When
//     the scores of a tile are there, the product of the tile before has ended (the tensor core works in order), so nobody waits for it.
//   - K and V come through one ring of 32 KB slots, pages by TMA; 64 KB hold Q.
//   - The CTAs of a head read the same tiles at about the same time, so that L2 has them once and not every CTA's own part of a long context.
// 2048 tokens on 32768 keys (32 / 8 heads): 890 us, 1.20 PFLOP/s of the 1.65 of the library's product.  A tile of 256 x 128 scores takes 2064 clocks of the
// tensor core and some 2800 in all: a half's scores (512), softmax (1600, of which 768 exponentials at 16 a clock an SM) and what is left of its products
// follow one another, and there is no room in tensor memory for its next scores meanwhile.  Calls in a row run at the board's power limit, 1.46 GHz
// instead of 1.97 (one alone takes 780 us), so what saves instructions and traffic counts as much as what shortens the chain.  Between two
// query tiles some 5000 clocks are lost.
#pragma once

#include "paged_few.cuh"

namespace efq {

constexpr int kChunkKeys = 1 << kChunkShift, kChunkRows = 128;      // keys of a tile, rows of a half
constexpr int kChunkThreads = 384;
constexpr int kChunkSlots = 5;
constexpr int kChunkPart = kChunkKeys * 128;                   // bytes of 64 channels of 128 rows
constexpr uint32_t kChunkColS = 0, kChunkColO = 256;           // + 128 for the second half
// log2: how far a row's maximum may grow before the output is rescaled; with kChunkRaise, what the probabilities stay below (fp16 ends at 2^16), sums below
// that times the keys.  Scores that spread as under outlier channels: 2048 tokens on 32768 884 us with 8, 874 with 14, a mixed batch 274 and 271.
// fp16 shares the 15 powers that it has above 1 between the two: probabilities down to 2^-20 of the row's maximum keep all their bits, smaller ones are
// off by up to 2^-31 of it, so that a million of them are less than a rounding.  fp16, raised by 0 with a slack of 14, by 6 with 9, 8 with 7 and 10 with 5:
// 2048 tokens on 32768 901, 927, 949 and 980 us, 300 on 9000 56.9, 58.8, 61.3 and 65.6, 64 chunks of 300 on 600 234, 240, 245 and 255.
template <typename T> constexpr float kChunkRaise = kNarrowExponent<T> ? 6.0f : 0.0f;
template <typename T> constexpr float kSlack = kNarrowExponent<T> ? 9.0f : 14.0f;
// A maximum is a rounded product, a probability's argument a fused one: the two differ by up to half a step of the maximum.  That is a factor which all
// of a row's probabilities have in common, up to 2^(1/2) here; beyond, where it would overflow or leave nothing, the scores are rounded too.
constexpr float kFar = 8388608.0f;                             // 2^23

// A segment of the run, as the warps that load tell it to the others: found out once, since the code of the walk is run rarely and not at hand when it is
// (each of the others walking for itself: 3300 clocks between two segments).  Of [2] one for each half.
struct __align__(16) ChunkSegment {
    int32_t j0;                                                // first key tile; -1: the run has ended
    int32_t end[2];                                            // key tiles [j0, end) are seen by the half
    int32_t fewest[2];                                         // keys that every row of the half sees
    int32_t tokens[2];
    int32_t token0, head, len, base;                           // as in PagedSegment
    int32_t none, all, record;                                 // rows of NaN; the whole query tile; its end, begun by another CTA
};
constexpr int kChunkSegments = 4;

struct __align__(1024) ChunkSmem {
    static constexpr bool kExpired = false;                    // an expired wait is told at the end of the block
    uint8_t q[2][2][kChunkPart];                               // half, channels 0-63 and 64-127; 128-byte swizzle
    uint8_t kv[kChunkSlots][2 * kChunkPart];                   // [8 tokens][channels 0-63, 64-127][token]
    uint64_t full[kChunkSlots], empty[kChunkSlots], q_full, q_empty, s_full[2], p_ready[2], p_rest[2], o_full[2], v_tail, v_clean, drained[2];
    uint64_t seg_full[kChunkSegments], seg_empty[kChunkSegments];
    ChunkSegment seg[kChunkSegments];
    uint32_t scratch[kChunkThreads / 32];
    PagedRun<kChunkShift, kChunkItem> run;
    uint32_t tmem_base;
    volatile uint32_t failed;
};

// Registers of a softmax thread, which holds a row of scores, and of the others: together what the block is launched with, 384 x 168.  208 and 88: 2048
// tokens on 32768 943 us and 889, 224 and 56: 942 and 904.
constexpr int kChunkRegsMore = 216, kChunkRegsLess = 72;
static_assert(256 * kChunkRegsMore + 128 * kChunkRegsLess <= 384 * 168, "setmaxnreg draws on what the block was launched with");

template <typename T>
__device__ constexpr uint32_t chunk_idesc(bool b_n_major)
{
    return __is_same(T, __nv_bfloat16) ? ptx::bf16_idesc(128, b_n_major) : ptx::bf16_idesc(128, b_n_major) & ~((1u << 7) | (1u << 10));
}

// Two FP32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// NaN if one of them is
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 2^x for x <= 15 on the FMA pipe: x = n + f with n the nearest integer, 1 + f q(f) with q of degree 3 fitted to the smallest relative error on
// [-1/2, 1/2] (least squares, reweighted until the error is level: 2.9e-6, a 1300th of what rounding the probability may cost in bf16, a 160th in fp16), n added
// to the exponent.  Below -127 the result is 0, exactly: f = 0 there and the exponent field is empty.  NaN is not kept.
__device__ __forceinline__ float2 poly_exp2(float2 x)
{
    constexpr float kMagic = 12582912.0f;           // 1.5 * 2^23: adding it leaves the integer in the low bits
    x = make_float2(fmaxf(x.x, -127.0f), fmaxf(x.y, -127.0f));
    const float2 t = add2(x, make_float2(kMagic, kMagic)), n = add2(t, make_float2(-kMagic, -kMagic));
    const float2 f = fma2(n, make_float2(-1.0f, -1.0f), x);
    float2 y = fma2(f, make_float2(9.582852944731712e-3f, 9.582852944731712e-3f), make_float2(5.5906426161527634e-2f, 5.5906426161527634e-2f));
    y = fma2(f, y, make_float2(0.24024099111557007f, 0.24024099111557007f));
    y = fma2(f, y, make_float2(0.6931241750717163f, 0.6931241750717163f));
    y = fma2(f, y, make_float2(1.0f, 1.0f));
    return make_float2(__uint_as_float(__float_as_uint(y.x) + (__float_as_uint(t.x) << 23)), __uint_as_float(__float_as_uint(y.y) + (__float_as_uint(t.y) << 23)));
}
// 16 registers into 16 columns of tensor memory
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}

// 16 columns of tensor memory
__device__ __forceinline__ void tmem_ld16f(uint32_t taddr, float (&r)[16])
{
    uint32_t u[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]),
                 "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]) : "r"(taddr) : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __uint_as_float(u[i]);
}
// 32 bytes, a whole sector; p on 32 bytes
__device__ __forceinline__ void store8(void* p, const uint32_t (&u)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]) : "memory");
}

// Tells the compiler that a value is the same in all lanes.
template <typename V>
__device__ __forceinline__ V uniform(V x) { return __shfl_sync(0xffffffffu, x, 0); }

__device__ __forceinline__ ChunkSegment chunk_segment(const PagedSegment<kChunkShift, kChunkItem>& g, int step)
{
    const int per = step >> 1;
    ChunkSegment d;
    d.j0 = g.j0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        d.tokens[w] = max(0, min(per, g.tokens - w * per));
        const int seen = d.tokens[w] > 0 ? paged_limit(g, w * per + d.tokens[w] - 1) : 0;
        d.end[w] = max(g.j0, min(g.j1, (seen + kChunkKeys - 1) >> kChunkShift));
        d.fewest[w] = d.tokens[w] > 0 ? paged_limit(g, w * per) : 0;
    }
    d.token0 = g.token0;
    d.head = g.head;
    d.len = g.w.len;
    d.base = g.base;
    d.none = g.w.none;
    d.all = g.j0 == 0 && g.j1 == g.n ? 1 : 0;
    d.record = g.j0 > 0 && g.j1 == g.n ? 1 : 0;
    return d;
}
// The wait for a segment, or for the room of one.  It goes on when another wait has expired, since the rows of the segments that are left become
// NaN then: their warps let go of them without one, so two seconds are more than any of these waits can take.
__device__ __forceinline__ bool chunk_segment_wait(uint64_t* bar, uint32_t parity, ChunkSmem* sm)
{
    bool there = ptx::mbar_try_wait(bar, parity);
#pragma unroll 1
    for (int i = 0; !there && i < 40000; ++i) there = ptx::mbar_try_wait_suspend(bar, parity, 50000u);
    if (!there) sm->failed = 1u;
    return __all_sync(0xffffffffu, there) != 0;
}

template <typename T>
__global__ void __launch_bounds__(kChunkThreads, 1)
paged_chunk_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                   const __grid_constant__ PagedArgs A)
{
    extern __shared__ uint8_t smem_raw[];
    ChunkSmem* const sm = reinterpret_cast<ChunkSmem*>(smem_raw + ptx::smem_round_up(smem_raw, 1024u));
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    if (tid == 0) {
        sm->failed = 0u;
        for (int i = 0; i < kChunkSlots; ++i) {
            ptx::mbar_init(&sm->full[i], 1);
            ptx::mbar_init(&sm->empty[i], 2);
        }
        ptx::mbar_init(&sm->q_full, 1);
        ptx::mbar_init(&sm->q_empty, 2);
        ptx::mbar_init(&sm->v_tail, 1);
        ptx::mbar_init(&sm->v_clean, 1);
        for (int i = 0; i < kChunkSegments; ++i) {
            ptx::mbar_init(&sm->seg_full[i], 1);
            ptx::mbar_init(&sm->seg_empty[i], 11);             // the warps but the one that loads
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&sm->s_full[i], 1);
            ptx::mbar_init(&sm->p_ready[i], 5);
            ptx::mbar_init(&sm->p_rest[i], 4);
            ptx::mbar_init(&sm->o_full[i], 1);
            ptx::mbar_init(&sm->drained[i], 1);
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
    if (tid == kChunkThreads - 1) paged_begin_status(A);
    paged_find_run<kChunkThreads, kChunkShift, kChunkItem>(A, sm->scratch, &sm->run);      // barriers of the block
    ptx::tc_fence_after_sync();
    const uint32_t tmem = sm->tmem_base;
    uint32_t seg = 0;           // segments so far
    // the next one; false at the end of the run
    auto next = [&](ChunkSegment& d) {
        const uint32_t at = seg % kChunkSegments;
        if (!chunk_segment_wait(&sm->seg_full[at], (seg / kChunkSegments) & 1u, sm)) return false;
        d = sm->seg[at];
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sm->seg_empty[at]);
        ++seg;
        return d.j0 >= 0;
    };
    ChunkSegment d;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kChunkRegsLess));
        if (warp == 9) {
            // ------------------------------------------------------------ loads
            const int P = 1 << A.page_shift, box = min(P, kChunkKeys), row = lane * box;
            PagedWalk<kChunkShift, kChunkItem, PagedReader<kChunkShift, kChunkItem>> walk(PagedReader<kChunkShift, kChunkItem>{A}, A.n_seqs, A.Hkv, sm->run);
            PagedSegment<kChunkShift, kChunkItem> g;
            uint32_t slot = 0, q_loads = 0;          // loads so far
            bool ok = true;
            for (bool more = true; more; ++seg) {
                more = walk.next(g);
                if (more) d = chunk_segment(g, A.step);
                else d.j0 = -1;
                const uint32_t at = seg % kChunkSegments;
                if (seg >= kChunkSegments && !chunk_segment_wait(&sm->seg_empty[at], (seg / kChunkSegments - 1) & 1u, sm)) break;
                if (lane == 0) {
                    sm->seg[at] = d;
                    ptx::mbar_arrive(&sm->seg_full[at]);
                }
                __syncwarp();
                if (!more || !ok) continue;          // after a wait that has expired the segments are told all the same
                const int end = max(d.end[0], d.end[1]);
                const int32_t* table = A.page_table + g.seq * A.table_stride;
                // The tiles that every row sees may come in any order.  The CTAs of a head begin at other places of its keys; so that they read the
                // same tiles at about the same time, tile t of a run is tile t of the sequence (round and round) wherever the segment has it.
                const int body = max(0, min(end, paged_limit(g, 0) >> kChunkShift) - g.j0), around = max(g.w.len >> kChunkShift, 1);
                const int want = static_cast<int>((slot >> 1) % static_cast<uint32_t>(around)), until = want <= g.j0 ? g.j0 - want : g.j0 + around - want;
                const int shift = want >= g.j0 && want < g.j0 + body ? want - g.j0 : until < body ? body - until : 0;
                auto place_of = [&](int j) {
                    const int x = j + shift;
                    return j >= g.j0 + body ? j : x >= g.j0 + body ? x - body : x;
                };
                // as it stands in the table: it is looked at when the tile after the next is loaded, so that nobody waits for it here
                auto entry_of = [&](int j) {
                    const int key = place_of(j) * kChunkKeys + row, at = key >> A.page_shift;
                    int e = -1;
                    if (row < kChunkKeys && j < end && key < g.w.len) e = __ldcg(table + at);
                    return e;
                };
                // One operand of a tile: lane i takes its i-th page.  Where an entry is no page, the rows of K are NaN, which makes rows of
                // NaN of the queries that see them, and the rows of V are 0.
                auto load = [&](const CUtensorMap& map, int page_step, int head_step, int j, int at, uint32_t fill) {
                    const int entry = at < A.n_pages ? at : -1;
                    const uint32_t s = slot % kChunkSlots;
                    if (slot >= kChunkSlots) ok = paged_wait_warp(&sm->empty[s], (slot / kChunkSlots - 1) & 1u, sm);
                    if (!ok) return;
                    const int key = place_of(j) * kChunkKeys + row;
                    const bool mine = row < kChunkKeys && key < g.w.len, page = mine && entry >= 0 && !A.inject_skip_loads;
                    if (mine && entry < 0) {
#pragma unroll 1
                        for (int i = 0; i < box * 16; ++i) reinterpret_cast<uint4*>(sm->kv[s] + row * 256)[i] = make_uint4(fill, fill, fill, fill);
                        ptx::fence_proxy_async_smem();
                    }
                    __syncwarp();           // what the lanes have filled stands before lane 0's arrival
                    const uint32_t pages = __popc(__ballot_sync(0xffffffffu, page));
                    if (lane == 0) ptx::mbar_arrive_expect_tx(&sm->full[s], (A.inject_skip_loads ? 1u : pages) * static_cast<uint32_t>(box) * 256u);
                    __syncwarp();
                    if (page) tma_load_page(sm->kv[s] + row * 256, &map, (key & (P - 1)) >> 3, entry * page_step + g.head * head_step, &sm->full[s]);
                    ++slot;
                };
                int entry = entry_of(g.j0), entry_next = entry_of(g.j0 + 1);
                for (int j = g.j0; ok && j < end; ++j) {
                    const int ahead = entry_of(j + 2);
                    load(mk, A.k_page_step, A.k_head_step, j, entry, 0x7fff7fffu);
                    if (ok && j == g.j0) {
                        if (q_loads > 0) ok = paged_wait_warp(&sm->q_empty, (q_loads - 1) & 1u, sm);
                        if (!ok) break;             // of this segment's loads
                        if (ptx::elect_one()) {
                            const int per = A.step >> 1;
                            ptx::mbar_arrive_expect_tx(&sm->q_full, static_cast<uint32_t>(A.step * A.G) * 256u);
                            for (int i = 0; i < 4; ++i)
                                tma_load_3d(sm->q[i >> 1][i & 1], &mq, (i & 1) * 64, g.head * A.G, g.token0 + (i >> 1) * per, &sm->q_full);
                        }
                        __syncwarp();
                        ++q_loads;
                    }
                    if (ok) load(mv, A.v_page_step, A.v_head_step, j, entry, 0u);
                    entry = entry_next;
                    entry_next = ahead;
                }
            }
            if (lane == 0) {        // its copies in flight end before the block does, whatever the others do
                for (uint32_t i = 0; i < kChunkSlots && i < slot && !A.inject_skip_loads; ++i) {
                    const uint32_t last = slot - 1 - i;
                    for (int n = 0; n < 20000 && !ptx::mbar_try_wait_suspend(&sm->full[last % kChunkSlots], (last / kChunkSlots) & 1u, 50000u); ++n) {}
                }
                for (int n = 0; n < 20000 && q_loads > 0 && !ptx::mbar_try_wait_suspend(&sm->q_full, (q_loads - 1) & 1u, 50000u); ++n) {}
            }
        } else if (warp != 10) {
            // ------------------------------------------------------------ MMAs: warp 8 the first half's, warp 11 the second's
            // The tensor core's queue holds four of these products, 64 clocks each: what a warp does between two of them must not take
            // longer.  So the whole warp walks, on values that the compiler knows to be the same in all lanes (uniform registers, no moves for
            // each operand; a single thread's loop took 1170 to 1530 clocks for 16 products beside busy warps, this one 1030 to 1040), and
            // what one half waits for does not hold up the other.  Every tile of the run is walked by both, so that a slot is free when
            // both have let it go.
            const int w = uniform(warp == 11 ? 1 : 0);
            const uint32_t tm = uniform(tmem), s_tmem = tm + kChunkColS + 128 * w, o_tmem = tm + kChunkColO + 128 * w;
            const uint64_t dq = ptx::smem_desc(ptx::smem_u32(sm->q[0][0]) + w * 2 * kChunkPart, 16, 1024, ptx::kLayoutSw128);
            const uint64_t dk = ptx::smem_desc(ptx::smem_u32(sm->kv[0]), 16, 2048, ptx::kLayoutSw128);
            const uint64_t dv = ptx::smem_desc(ptx::smem_u32(sm->kv[0]), 1024, 2048, ptx::kLayoutSw128);
            constexpr uint32_t kSlotStep = 2 * kChunkPart >> 4;
            uint64_t *const s_full = &sm->s_full[w], *const p_ready = &sm->p_ready[w], *const p_rest = &sm->p_rest[w], *const o_full = &sm->o_full[w];
            uint64_t* const p_ready_other = &sm->p_ready[w ^ 1];
            uint32_t slot = 0, round = 0, q_round = 0, p_round = 0, clean_round = 0;        // parities of the next waits
            uint32_t turns = 0;                  // given to the other half
            bool ok = true;
            auto advance = [&]() {
                if (++slot == kChunkSlots) {
                    slot = 0;
                    round ^= 1u;
                }
            };
            // The halves take turns, the first one first: while one has its products the other has its softmax.  Left to themselves they fall
            // into step, both at the exponentials and then both at the tensor core.  A half's turn for a tile is an arrival of the other
            // half's warp on the barrier of its probabilities, so that there is one wait for both.  Half 0 gives half 1 the turn for the same
            // tile, half 1 half 0 that for the next.
            // The barrier takes one turn a phase: a warp that does not wait for its own half's probabilities waits until the last one has been taken.
            auto turn_taken = [&]() { return turns == 0u || paged_wait_warp(p_ready_other, (turns & 1u) ^ 1u, sm); };
            // one thread's; hands over before the last products, which the queue holds until the other warp is there
            auto scores = [&](bool hand_over) {
                const uint64_t k = dk + slot * kSlotStep;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t off = ((i >> 2) * kChunkPart + (i & 3) * 32) >> 4, k_off = ((i >> 2) * 1024 + (i & 3) * 32) >> 4;
                    ptx::mma_bf16(s_tmem, dq + off, k + k_off, chunk_idesc<T>(false), i > 0 ? 1u : 0u);
                    if (i == 4 && hand_over) ptx::mbar_arrive(p_ready_other);
                }
                ptx::mma_commit(s_full);
                ptx::mma_commit(&sm->empty[slot]);
            };
            while (next(d)) {
                const int j0 = uniform(d.j0), mine = uniform(w ? d.end[1] : d.end[0]), other = uniform(w ? d.end[0] : d.end[1]), end = max(mine, other);
                const int clean = uniform(d.len < end * kChunkKeys ? 1 : 0);
                if (!ok || end == j0) continue;
                ok = paged_wait_warp(&sm->q_full, q_round, sm) && paged_wait_warp(&sm->full[slot], round, sm);
                q_round ^= 1u;
                // the first scores; half 1 gives half 0 the turn for the first tile
                const bool opens = w == 1 && j0 < other;
                if (opens) ok = ok && turn_taken();
                if (!ok) continue;
                if (ptx::elect_one()) {
                    if (j0 < mine) {
                        scores(opens);
                    } else {
                        if (opens) ptx::mbar_arrive(p_ready_other);
                        ptx::mbar_arrive(&sm->empty[slot]);
                    }
                    if (j0 + 1 == end) ptx::mma_commit(&sm->q_empty);
                }
                __syncwarp();
                turns += opens ? 1u : 0u;
                advance();
                for (int j = j0; j < end; ++j) {
                    const uint32_t v_slot = slot;
                    ok = paged_wait_warp(&sm->full[slot], round, sm);
                    advance();
                    if (clean && j + 1 == end) {
                        if (w == 0 && ptx::elect_one()) ptx::mbar_arrive(&sm->v_tail);
                        __syncwarp();
                        ok = ok && paged_wait_warp(&sm->v_clean, clean_round, sm);
                        clean_round ^= 1u;
                    }
                    const bool more = j + 1 < end, hand_over = j + w < other;          // w = 0: tile j of the other half, w = 1: tile j + 1
                    if (more) ok = ok && paged_wait_warp(&sm->full[slot], round, sm);
                    if (j < mine) {
                        const uint64_t v = dv + v_slot * kSlotStep;
                        ok = ok && paged_wait_warp(p_ready, p_round, sm);
                        if (!ok) break;
                        ptx::tc_fence_after_sync();
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int i = 0; i < 6; ++i)
                                ptx::mma_bf16_ts(o_tmem, s_tmem + 8 * i, v + (i * 4096u >> 4), chunk_idesc<T>(true), i > 0 || j > j0 ? 1u : 0u);
                        }
                        __syncwarp();
                        ok = paged_wait_warp(p_rest, p_round, sm);
                        p_round ^= 1u;
                        if (!ok) break;
                        ptx::tc_fence_after_sync();
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int i = 6; i < 8; ++i) ptx::mma_bf16_ts(o_tmem, s_tmem + 8 * i, v + (i * 4096u >> 4), chunk_idesc<T>(true), 1u);
                            if (j + 1 < mine) {
                                scores(hand_over);
                            } else {
                                ptx::mma_commit(o_full);
                                if (hand_over) ptx::mbar_arrive(p_ready_other);
                                if (more) ptx::mbar_arrive(&sm->empty[slot]);
                            }
                            ptx::mma_commit(&sm->empty[v_slot]);
                            if (j + 2 == end) ptx::mma_commit(&sm->q_empty);
                        }
                        __syncwarp();
                    } else {
                        if (hand_over) ok = ok && turn_taken();
                        if (!ok) break;
                        if (ptx::elect_one()) {
                            if (hand_over) ptx::mbar_arrive(p_ready_other);
                            ptx::mbar_arrive(&sm->empty[v_slot]);
                            if (more) ptx::mbar_arrive(&sm->empty[slot]);
                            if (j + 2 == end) ptx::mma_commit(&sm->q_empty);
                        }
                        __syncwarp();
                    }
                    turns += hand_over ? 1u : 0u;
                    if (more) advance();
                }
            }
            if (!ok) {              // the MMAs that were issued end before tensor memory is given back
                if (ptx::elect_one()) ptx::mma_commit(&sm->drained[w]);
                __syncwarp();
                for (int n = 0; n < 20000 && !ptx::mbar_try_wait_suspend(&sm->drained[w], 0u, 50000u); ++n) {}
                __syncwarp();
            }
        } else if (warp == 10) {
            // ------------------------------------------------------------ rows of V past a sequence
            // They hold whatever the page held, and 0 times that has to be 0.
            uint32_t slot = 0, round = 0;           // loads so far; parity of the next wait
            bool ok = true;
            while (next(d)) {
                const int end = max(d.end[0], d.end[1]), inside = d.len - (end - 1) * kChunkKeys;
                if (end == d.j0) continue;
                slot += 2 * (end - d.j0);
                if (!ok || inside >= kChunkKeys) continue;
                ok = paged_wait_warp(&sm->v_tail, round, sm);
                if (!ok) continue;
                round ^= 1u;
                uint8_t* const v = sm->kv[(slot - 1) % kChunkSlots];
#pragma unroll 1
                for (int i = inside * 16 + lane; i < kChunkKeys * 16; i += 32) {       // 16 bytes: row i / 16, channels from 8 (i % 16) on
                    const int r = i >> 4;
                    *reinterpret_cast<uint4*>(v + (r >> 3) * 2048 + ((i >> 3) & 1) * 1024 + (r & 7) * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sm->v_clean);
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
        while (next(d)) {
            // what decides the loop's course is the same in all lanes (2048 tokens on 32768 930 us without the compiler knowing it, 904 with)
            const int j0 = uniform(d.j0), end = uniform(w ? d.end[1] : d.end[0]), fewest = uniform(w ? d.fewest[1] : d.fewest[0]);
            const bool mine = r < uniform((w ? d.tokens[1] : d.tokens[0]) * A.G);
            const int limit = A.causal ? max(0, min(d.len, d.base + i + 1)) : d.len;
            bool nan = d.none != 0;
            float m = -INFINITY, l = 0.0f;
            for (int j = j0; j < end; ++j) {
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
                float top[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) top[c] = s[c];
#pragma unroll
                for (int c = 8; c < 120; c += 16)
#pragma unroll
                    for (int q = 0; q < 8; ++q) top[q] = max3(top[q], s[c + q], s[c + 8 + q]);
#pragma unroll
                for (int q = 0; q < 8; ++q) top[q] = max3(top[q], s[120 + q], top[q]);
                float mx = max3(max3(top[0], top[1], top[2]), max3(top[3], top[4], top[5]), max3(top[6], top[7], top[7])) * A.scale_log2;
                mx = mine ? mx : -INFINITY;          // rows that no query has hold anything, and their output is not stored: nothing is done for what they hold
                const float reference = paged_reference(mx, kChunkRaise<T>);
                const bool grew = !(reference <= __fadd_rd(m, kSlack<T>));        // also a NaN; a step of m may be more than the slack
                const bool far = fabsf(mx) > kFar && fabsf(mx) < INFINITY;
                float scale = A.scale_log2;
                if (__any_sync(0xffffffffu, grew || far)) {
                    if (__any_sync(0xffffffffu, far)) {
#pragma unroll
                        for (int c = 0; c < 128; ++c) s[c] *= scale;
                        scale = 1.0f;
                    }
                    const float alpha = grew ? (m == -INFINITY ? 0.0f : paged_exp2(m - reference)) : 1.0f;
                    if (grew) m = reference < INFINITY ? reference : __uint_as_float(0x7fc00000u);      // an infinite score makes a row of NaN, as inf - inf does
                    l *= alpha;
                    if (j > j0) {
#pragma unroll 1
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
                const float2 scale2 = make_float2(scale, scale), minus2 = make_float2(-base, -base);
                float2 sum2[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t p[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        if (q == 3 && c == 8) {          // the product with V begins while the last quarter is made
                            ptx::tmem_wait_st();
                            ptx::tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(&sm->p_ready[w]);
                        }
                        float2 y = fma2(make_float2(s[32 * q + 2 * c], s[32 * q + 2 * c + 1]), scale2, minus2);
                        // a quarter of the exponentials by polynomial (an eighth: 946 us and 889, three eighths: 903)
                        y = c % 4 == 3 ? poly_exp2(y) : make_float2(paged_exp2(y.x), paged_exp2(y.y));
                        sum2[c & 1] = add2(sum2[c & 1], y);
                        // rounded once, to the elements' type (off by up to 2^-8 or 2^-11 of each, and kChunkRaise); the sum is kept unrounded
                        p[c] = Pack2<T>::round(y.x, y.y);
                    }
                    tmem_st16(s_col + 16 * q, p);        // over scores that have been read
                }
                ptx::tmem_wait_st();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sm->p_rest[w]);
                sum2[0] = add2(sum2[0], sum2[1]);
                l += sum2[0].x + sum2[0].y;
            }

            const bool some = end > j0, all = d.all != 0;
            if (some && !nan) {
                nan = !paged_wait_warp(&sm->o_full[w], o_count & 1u, sm);
                ++o_count;
                ptx::tc_fence_after_sync();
            }
            nan = nan || sm->failed != 0u;          // once a wait has expired the parities of the later ones mean nothing
            if (nan) l = __uint_as_float(0x7fc00000u);
            const int token = d.token0 + i, head = d.head * A.G + r % A.G, slot = 2 * blockIdx.x + (j0 == 0 ? 1 : 0);
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            char* const dst = A.o + token * A.o_token + head * A.o_head;
            // of four channels the 128 rows side by side, so that a warp's stores are whole lines
            float4* const part = reinterpret_cast<float4*>(A.part_o + (static_cast<int64_t>(slot) * 2 + w) * kChunkRows * kPagedD) + r;
            // short code: it is run rarely and not at hand when it is (32 columns a round: 64 chunks of 300 tokens on 600 242 us, 16 231)
#pragma unroll 1
            for (int q = 0; q < 8; ++q) {
                float o[16];
                tmem_ld16f(o_col + 16 * q, o);
                ptx::tmem_wait_ld();
                if (!some || nan) {
#pragma unroll
                    for (int c = 0; c < 16; ++c) o[c] = 0.0f;
                }
                if (mine && all) {
                    uint32_t u[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] = Pack2<T>::round(o[2 * i] * inv, o[2 * i + 1] * inv);
                    char* const at = dst + 32 * q;
                    if (A.o_wide) {
                        store8(at, u);
                    } else {
                        reinterpret_cast<uint4*>(at)[0] = make_uint4(u[0], u[1], u[2], u[3]);
                        reinterpret_cast<uint4*>(at)[1] = make_uint4(u[4], u[5], u[6], u[7]);
                    }
                } else if (mine) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) part[(4 * q + c) * kChunkRows] = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
                }
            }
            ptx::tc_fence_before_sync();
            if (mine && all && A.lse != nullptr) A.lse[static_cast<int64_t>(token) * (A.Hkv * A.G) + head] = m * kLn2 + logf(l);
            if (mine && !all) A.part_ml[slot * 2 * kChunkRows + w * kChunkRows + r] = make_float2(m, l);
            if (tid == 0 && d.record) A.records[blockIdx.x] = {sm->run.begins, d.token0, d.tokens[0] + d.tokens[1], d.head};
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (tid == 0 && sm->failed != 0u) A.expired[blockIdx.x] = 1u;
    if (warp == 8) ptx::tmem_dealloc(tmem, 512);
}

}  // namespace efq
