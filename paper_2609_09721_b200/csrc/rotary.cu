// Rotary positions with several axes:
//   efq_rotary        q and k of a dense problem, forward or turned back (its gradient), with any strides on both sides
//   efq_paged_append  new keys (turned) and values into the pages of a cache, the queries turned beside them
//
// One pass over the data; bound by the bytes.  A warp takes a token and a run of its heads, so that the token's angles are
// made once for all of them: every lane makes two pairs' sine and cosine and gets the eight that it needs from its neighbours, and
// keeps them in registers while it goes through the heads.  Eight lanes share a row of 128 channels: a lane loads the two
// 16-byte pieces that hold both channels of its eight pairs and writes them back, so rows may be turned in place.
// The angle is formed in double: at position 900000 an FP32 product is off by up to 0.03 radians.  Reduced to a turn there, its
// sine and cosine are FP32 functions of an argument in [-1, 1].
#include "paged.cuh"
#include "efq_internal.cuh"
#include "sm100_ptx.cuh"

namespace efq {
namespace {

constexpr int kWarps = 4;               // of a block
// Rows a lane has in flight.  Two leave 32 warps to an SM, four 20: 24 + 24 heads of 32760 tokens 132.2 us and 129.9, of 4097 tokens, which
// the 32 warps take in one go, 20.6 and 22.6, a chunk of 8192 tokens into the cache 37.7 and 37.1.  Asking for the first rows before the angles
// are made costs time (32760 tokens 135 and 151 us), as do angles shared by a block instead of a warp (142).
constexpr int kRowsAhead = 2;

struct RotaryRows {
    const char* src;
    char* dst;
    int64_t src_batch, src_head, src_token, dst_batch, dst_head, dst_token;      // bytes
    int32_t heads, turned;
};

struct RotaryArgs {
    RotaryRows rows[3];                 // efq_rotary: q, k; efq_paged_append: q, k, v
    const double* inv_freq;
    const int32_t* positions;           // null: the token's index in its sequence
    int64_t position_axis, position_batch;
    int64_t tokens, S;                  // tokens of all batch entries, of one
    int32_t axis_end[4];                // pairs of an axis and those before it
    int32_t n_pairs, heads, groups, heads_per_group, inverse;
    // paged
    const int32_t *page_table, *cu_seqlens, *seq_lens;
    int64_t table_stride;
    int32_t n_seqs, n_pages, max_pages, page_shift;
};

// The sequence that holds token t: the largest s with cu[s] <= t and cu[s + 1] > t, -1 behind the last.  The 32 lanes cut the range
// into as many parts at a time.
__device__ __forceinline__ int find_sequence(const int32_t* cu, int n_seqs, int64_t t, int lane)
{
    int lo = 0, n = n_seqs;             // the last entry <= t of cu[lo .. lo + n]
    while (n > 0) {
        const int step = (n + 31) / 32, at = lo + (lane + 1) * step;
        const bool before = (lane + 1) * step <= n && __ldcg(cu + at) <= t;
        const int below = __popc(__ballot_sync(0xffffffffu, before));       // entries do not decrease: the lanes that hold stand in front
        lo += below * step;
        n = min(step - 1, n - below * step);
    }
    return lo < n_seqs ? lo : -1;
}

template <typename T, bool kInterleaved, bool kPaged>
__global__ void __launch_bounds__(kWarps * 32, 8) rotary_kernel(const __grid_constant__ RotaryArgs A)
{
    ptx::grid_wait();
    const int lane = threadIdx.x & 31;
    const int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int64_t bt = task / A.groups;
    if (bt >= A.tokens) return;
    const int group = static_cast<int>(task - bt * A.groups);
    const int64_t b = kPaged ? 0 : bt / A.S, t = kPaged ? bt : bt - b * A.S;

    int index = 0;
    int64_t page = -1;
    if (kPaged) {
        const int s = find_sequence(A.cu_seqlens, A.n_seqs, t, lane);
        if (s < 0) return;
        index = __ldcg(A.seq_lens + s) - __ldcg(A.cu_seqlens + s + 1) + static_cast<int>(t);
        const int entry = index >> A.page_shift;
        if (index >= 0 && entry < A.max_pages) {
            page = __ldcg(A.page_table + s * A.table_stride + entry);
            if (page >= A.n_pages) page = -1;
        }
    }
    const int64_t slot = index & ((1 << A.page_shift) - 1);

    // sine and cosine of pairs 2 lane and 2 lane + 1
    float c[2], s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = 2 * lane + i;
        c[i] = 1.0f;
        s[i] = 0.0f;
        if (p < A.n_pairs) {
            const int axis = p < A.axis_end[0] ? 0 : p < A.axis_end[1] ? 1 : p < A.axis_end[2] ? 2 : 3;
            const int position = kPaged && A.positions == nullptr ? index : __ldcg(A.positions + axis * A.position_axis + b * A.position_batch + t);
            const double turns = static_cast<double>(position) * __ldcg(A.inv_freq + p) * 0.15915494309189533577;      // 1 / (2 pi)
            sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s[i], &c[i]);
            if (A.inverse) s[i] = -s[i];
        }
    }
    const int j = lane & 7;                     // pairs 8j to 8j + 7, made by lanes 4j to 4j + 3
    float co[8], si[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        co[i] = __shfl_sync(0xffffffffu, c[i & 1], 4 * j + (i >> 1));
        si[i] = __shfl_sync(0xffffffffu, s[i & 1], 4 * j + (i >> 1));
    }
    // the two 16-byte pieces of a row that this lane takes
    const int turned = A.n_pairs >> 3;          // of the eight lanes of a row; the others copy what lies behind the turned channels
    const int first = j >= turned || kInterleaved ? 2 * j : j, second = j >= turned || kInterleaved ? 2 * j + 1 : j + turned;

    const int end = min(A.heads, (group + 1) * A.heads_per_group);
    for (int h0 = group * A.heads_per_group + (lane >> 3); h0 < end; h0 += 4 * kRowsAhead) {
        uint4 x[kRowsAhead], y[kRowsAhead];
        char* dst[kRowsAhead];
        bool turn[kRowsAhead];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const int h = h0 + 4 * u;
            dst[u] = nullptr;
            turn[u] = false;
            if (h < end) {
                const bool is_q = h < A.rows[0].heads, is_k = h < A.rows[0].heads + A.rows[1].heads;
                const RotaryRows& r = is_q ? A.rows[0] : is_k ? A.rows[1] : A.rows[2];
                const int64_t head = h - (is_q ? 0 : is_k ? A.rows[0].heads : A.rows[0].heads + A.rows[1].heads);
                const char* src = r.src + b * r.src_batch + head * r.src_head + t * r.src_token;
                if (!kPaged || is_q)
                    dst[u] = r.dst + b * r.dst_batch + head * r.dst_head + t * r.dst_token;
                else if (page >= 0)
                    dst[u] = r.dst + page * r.dst_batch + head * r.dst_head + slot * r.dst_token;
                turn[u] = r.turned && j < turned;
                if (dst[u] != nullptr) {
                    x[u] = __ldcs(reinterpret_cast<const uint4*>(src) + first);
                    y[u] = __ldcs(reinterpret_cast<const uint4*>(src) + second);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            if (dst[u] == nullptr) continue;
            if (turn[u]) {
                uint32_t* a = reinterpret_cast<uint32_t*>(&x[u]);
                uint32_t* z = reinterpret_cast<uint32_t*>(&y[u]);
                if (kInterleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t& w = i < 4 ? a[i] : z[i - 4];
                        const float2 f = Pack2<T>::widen(w);
                        w = Pack2<T>::round(f.x * co[i] - f.y * si[i], f.x * si[i] + f.y * co[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = Pack2<T>::widen(a[i]), g = Pack2<T>::widen(z[i]);
                        a[i] = Pack2<T>::round(f.x * co[2 * i] - g.x * si[2 * i], f.y * co[2 * i + 1] - g.y * si[2 * i + 1]);
                        z[i] = Pack2<T>::round(f.x * si[2 * i] + g.x * co[2 * i], f.y * si[2 * i + 1] + g.y * co[2 * i + 1]);
                    }
                }
            }
            reinterpret_cast<uint4*>(dst[u])[first] = x[u];
            reinterpret_cast<uint4*>(dst[u])[second] = y[u];
        }
    }
}

efq_status_t set_rotation(RotaryArgs& A, const efq_rotary_t* rotary)
{
    A.n_pairs = 0;
    if (rotary == nullptr) return EFQ_OK;
    if (rotary->n_axes < 1 || rotary->n_axes > 4 || !rotary->inv_freq) return EFQ_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(rotary->inv_freq) & 7u) return EFQ_ERR_ALIGNMENT;
    A.inv_freq = rotary->inv_freq;
    for (int a = 0; a < 4; ++a) {
        if (a < rotary->n_axes) {
            if (rotary->pairs[a] < 0) return EFQ_ERR_INVALID_ARG;
            if (rotary->pairs[a] > kPagedD / 2) return EFQ_ERR_UNSUPPORTED;
            A.n_pairs += rotary->pairs[a];
        }
        A.axis_end[a] = A.n_pairs;
    }
    return A.n_pairs > kPagedD / 2 || (A.n_pairs & 7) != 0 ? EFQ_ERR_UNSUPPORTED : EFQ_OK;
}

efq_status_t set_rows(RotaryRows& r, const efq_rows_t& g, bool with_dst, bool turned)
{
    if (!g.src || (with_dst && !g.dst) || g.heads <= 0) return EFQ_ERR_INVALID_ARG;
    if (!aligned_rows(g.src, g.src_batch, g.src_head, g.src_token) || (with_dst && !aligned_rows(g.dst, g.dst_batch, g.dst_head, g.dst_token)))
        return EFQ_ERR_ALIGNMENT;
    r = {static_cast<const char*>(g.src), static_cast<char*>(g.dst), 2 * g.src_batch, 2 * g.src_head, 2 * g.src_token,
         2 * g.dst_batch, 2 * g.dst_head, 2 * g.dst_token, g.heads, turned ? 1 : 0};
    return EFQ_OK;
}

template <bool kPaged>
efq_status_t launch(RotaryArgs& A, int dtype, bool interleaved, void* stream)
{
    if (!aligned_ints(A.positions)) return EFQ_ERR_ALIGNMENT;
    const int64_t all_heads = static_cast<int64_t>(A.rows[0].heads) + A.rows[1].heads + A.rows[2].heads;
    if (all_heads >= (1ll << 31) - 256) return EFQ_ERR_UNSUPPORTED;
    A.heads = static_cast<int32_t>(all_heads);
    if (!device_is_sm100()) return EFQ_ERR_ARCH;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return EFQ_ERR_CUDA;
    // A token's heads go to as many warps as it takes to give every SM 16 of them, down to one row a lane.
    const int64_t want = 16ll * sm_count(dev), most = (A.heads + 3) / 4;
    int64_t groups = (want + A.tokens - 1) / A.tokens;
    groups = groups < 1 ? 1 : groups > most ? most : groups;
    A.heads_per_group = static_cast<int32_t>(((A.heads + groups - 1) / groups + 3) / 4 * 4);
    A.groups = (A.heads + A.heads_per_group - 1) / A.heads_per_group;
    const int64_t blocks = (A.tokens * A.groups + kWarps - 1) / kWarps;
    if (blocks >= (1ll << 31)) return EFQ_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(blocks));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    using Bf = __nv_bfloat16;
    const cudaError_t e = dtype == EFQ_BF16 ? (interleaved ? launch_overlapped(rotary_kernel<Bf, true, kPaged>, grid, kWarps * 32, 0, st, A)
                                                           : launch_overlapped(rotary_kernel<Bf, false, kPaged>, grid, kWarps * 32, 0, st, A))
                                            : (interleaved ? launch_overlapped(rotary_kernel<__half, true, kPaged>, grid, kWarps * 32, 0, st, A)
                                                           : launch_overlapped(rotary_kernel<__half, false, kPaged>, grid, kWarps * 32, 0, st, A));
    return e == cudaSuccess ? EFQ_OK : EFQ_ERR_CUDA;
}

}  // namespace
}  // namespace efq

extern "C" efq_status_t efq_rotary(const efq_rows_t* q, const efq_rows_t* k, const int32_t* positions, int64_t position_axis,
                                   int64_t position_batch, int B, int64_t S, int d, int dtype, const efq_rotary_t* rotary, int inverse, void* stream)
{
    if (B < 0 || S < 0) return EFQ_ERR_INVALID_ARG;
    if ((!q && !k) || !rotary) return EFQ_ERR_INVALID_ARG;
    if (d != efq::kPagedD || (dtype != EFQ_BF16 && dtype != EFQ_FP16)) return EFQ_ERR_UNSUPPORTED;
    efq::RotaryArgs A{};
    efq_status_t st = efq::set_rotation(A, rotary);
    if (st != EFQ_OK) return st;
    if (B == 0 || S == 0) return EFQ_OK;
    if (!positions) return EFQ_ERR_INVALID_ARG;
    if (q && (st = efq::set_rows(A.rows[0], *q, true, true)) != EFQ_OK) return st;
    if (k && (st = efq::set_rows(A.rows[1], *k, true, true)) != EFQ_OK) return st;
    if (S > (1ll << 40) / B) return EFQ_ERR_UNSUPPORTED;
    A.positions = positions;
    A.position_axis = position_axis;
    A.position_batch = position_batch;
    A.tokens = B * S;
    A.S = S;
    A.inverse = inverse ? 1 : 0;
    return efq::launch<false>(A, dtype, rotary->interleaved != 0, stream);
}

extern "C" efq_status_t efq_paged_append(const efq_rows_t* k, const efq_rows_t* v, const efq_rows_t* q, int64_t total, const int32_t* positions,
                                         int64_t position_axis, const efq_paged_t* cache, int d, int dtype, const efq_rotary_t* rotary, void* stream)
{
    if (!k || !v || !cache || total < 0) return EFQ_ERR_INVALID_ARG;
    efq_status_t st = efq::check_paged(*cache, d, dtype);
    if (st != EFQ_OK) return st;
    efq::RotaryArgs A{};
    if ((st = efq::set_rotation(A, rotary)) != EFQ_OK) return st;
    if (total == 0 || cache->n_seqs == 0) return EFQ_OK;
    if (total >= (1ll << 31)) return EFQ_ERR_UNSUPPORTED;        // cu_seqlens is 32 bits wide
    if (k->heads != cache->n_heads || v->heads != cache->n_heads) return EFQ_ERR_INVALID_ARG;
    efq_rows_t kc = *k, vc = *v;
    kc.src_batch = vc.src_batch = 0;
    kc.dst = cache->k;
    kc.dst_batch = cache->k_page; kc.dst_head = cache->k_head; kc.dst_token = cache->k_token;
    vc.dst = cache->v;
    vc.dst_batch = cache->v_page; vc.dst_head = cache->v_head; vc.dst_token = cache->v_token;
    if ((st = efq::set_rows(A.rows[1], kc, true, true)) != EFQ_OK || (st = efq::set_rows(A.rows[2], vc, true, false)) != EFQ_OK) return st;
    if (q) {
        efq_rows_t qc = *q;
        qc.src_batch = qc.dst_batch = 0;
        if ((st = efq::set_rows(A.rows[0], qc, true, true)) != EFQ_OK) return st;
    }
    A.positions = positions;
    A.position_axis = position_axis;
    A.tokens = A.S = total;
    A.page_table = cache->page_table;
    A.table_stride = cache->table_stride;
    A.cu_seqlens = cache->cu_seqlens;
    A.seq_lens = cache->seq_lens;
    A.n_seqs = cache->n_seqs;
    A.n_pages = cache->n_pages;
    A.max_pages = cache->max_pages;
    A.page_shift = __builtin_ctz(static_cast<unsigned>(cache->page_size));
    return efq::launch<true>(A, dtype, rotary != nullptr && rotary->interleaved != 0, stream);
}
