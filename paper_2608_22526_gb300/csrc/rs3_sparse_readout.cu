// rs3_sparse_readout.cu -- attention of each kept query over the blocks listed for it, scattered
// back to the grid (Sec. 3.1's readout, Eq. 6 and Eq. 7, over chosen blocks of the bank).
//
// Two paths (by_blocks() holds the rule):
//   by query   a CTA per (query, head) reads the blocks of its list: few queries, narrow heads
//   by block   a block that many queries chose is read once for all of them: the lists are turned
//              into lists of queries per block (k_block_lists), a block and up to 64 of its queries make
//              an item, whose attention is computed on the tensor cores (k_attend_blocks; fp32 on the CUDA
//              cores, k_attend_blocks_fp32), and the partial results of a query's blocks are joined by
//              their log-sum-exp (k_join_blocks)
#include "rs3_sparse.cuh"

#include "rs3_blocks_tma.cuh"
#include "rs3_cluster.cuh"

#include <cmath>

namespace {

struct AttendArgs {
    SparseArgs s;
    const uint8_t *k_store, *v_store;
    const int32_t *sel;
    const void *residual;
    void *out;
    float scale_log2;
};

// out = residual (or zeros) on every cell; the kept ones are written after it
__global__ void __launch_bounds__(256) k_pass_through(const uint4 *__restrict__ res, uint4 *__restrict__ out, int64_t nvec)
{
    pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < nvec; i += (int64_t)gridDim.x * 256)
        out[i] = res ? __ldcs(res + i) : make_uint4(0, 0, 0, 0);
}

template <typename T>
struct Row;                                // 16 bytes of a row as fp32
template <>
struct Row<uint16_t> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void widen(uint4 v, float *f)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ uint4 narrow(const float *f)
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Row<float> {
    static constexpr int N = 4;
    __device__ static __forceinline__ void widen(uint4 v, float *f)
    {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    __device__ static __forceinline__ uint4 narrow(const float *f)
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

// The larger of two scores, NaN where either is: a maximum that passed over a NaN would drop rows whose scores are all NaN.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

constexpr int GATHER_WARPS = 16;           // at most

// A CTA per (query, head): its warps take the listed blocks in turn.  L lanes hold a row (ITEMS
// pieces of 16 bytes each), so a warp reads 32 / L rows at once; scores are summed over the L lanes,
// the softmax runs online per warp in the log2 domain, and the warps' results are joined at the end.
template <typename T, int ITEMS, int L>
__global__ void __launch_bounds__(32 * GATHER_WARPS) k_attend_gather(AttendArgs a)
{
    constexpr int N = Row<T>::N, GATHER_FLIGHT = 8 / ITEMS;    // rows in flight per lane group
    pdl_wait();
    __shared__ float s_o[GATHER_WARPS][256];
    __shared__ float s_m[GATHER_WARPS], s_l[GATHER_WARPS];
    const int n_warps = (int)blockDim.x >> 5;
    const SparseArgs &s = a.s;
    const int j = blockIdx.x, h = blockIdx.y, u = blockIdx.z;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int cnt, g;
    LiveRows rows;
    if (!sparse_unit(s, u, threadIdx.x == 0 && j == 0, cnt, g, rows) || j >= cnt) return;
    const int cell = s.idx[(int64_t)u * s.k_max + j];
    if (cell < 0 || cell >= s.mn) {
        if (threadIdx.x == 0) latch_status(s.status, RS3_EINVAL);
        return;
    }
    const int D = s.H * s.d, sub = lane & (L - 1), group = lane / L;
    constexpr int groups = 32 / L;
    // this lane's pieces of the query, rotated, times scale * log2 e
    float q[ITEMS][N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (sub + L * i) * N;
        Row<T>::widen(__ldg(reinterpret_cast<const uint4 *>(static_cast<const T *>(s.q) + ((int64_t)g * s.mn + cell) * D + h * s.d + c)), q[i]);
        if (s.rope) {
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const float4 f = __ldg(reinterpret_cast<const float4 *>(s.rope + (int64_t)cell * s.d + c + e));
                const float x0 = q[i][e], x1 = q[i][e + 1], x2 = q[i][e + 2], x3 = q[i][e + 3];
                q[i][e] = x0 * f.x - x1 * f.y;
                q[i][e + 1] = x0 * f.y + x1 * f.x;
                q[i][e + 2] = x2 * f.z - x3 * f.w;
                q[i][e + 3] = x2 * f.w + x3 * f.z;
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) q[i][e] *= a.scale_log2;
    }
    const int32_t *sel = a.sel + (((int64_t)u * s.H + h) * s.k_max + j) * s.n_top;
    const T *K = reinterpret_cast<const T *>(a.k_store) + (int64_t)u * s.bank.rows_per_unit * D + h * s.d;
    const T *V = reinterpret_cast<const T *>(a.v_store) + (int64_t)u * s.bank.rows_per_unit * D + h * s.d;
    float m = -INFINITY, l = 0.f, o[ITEMS][N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) o[i][e] = 0.f;
    for (int t = warp; t < s.n_top; t += n_warps) {
        const int b = sel[t];
        if (b < 0) continue;
        if (b >= s.nb) {
            if (lane == 0) latch_status(s.status, RS3_EINVAL);
            continue;
        }
        const int64_t row0 = (int64_t)b * s.bs;
        const uint64_t on[2] = {rows.mask64(row0) & (s.bs == 32 ? 0xffffffffull : ~0ull), s.bs > 64 ? rows.mask64(row0 + 64) : 0ull};
        for (int r0 = 0; r0 < s.bs; r0 += groups * GATHER_FLIGHT) {
            bool live[GATHER_FLIGHT];
            float x[GATHER_FLIGHT], top = -INFINITY;
            uint4 kv[GATHER_FLIGHT][ITEMS], vv[GATHER_FLIGHT][ITEMS];
#pragma unroll
            for (int f = 0; f < GATHER_FLIGHT; ++f) {
                const int r = r0 + f * groups + group;
                const int64_t row = row0 + r;
                live[f] = r < s.bs && ((r < 64 ? on[0] : on[1]) >> (r & 63) & 1ull);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    const int64_t at = row * D + (sub + L * i) * N;
                    kv[f][i] = live[f] ? __ldg(reinterpret_cast<const uint4 *>(K + at)) : make_uint4(0, 0, 0, 0);
                    vv[f][i] = live[f] ? __ldg(reinterpret_cast<const uint4 *>(V + at)) : make_uint4(0, 0, 0, 0);
                }
            }
#pragma unroll
            for (int f = 0; f < GATHER_FLIGHT; ++f) {
                float w[N];
                x[f] = 0.f;
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    Row<T>::widen(kv[f][i], w);
#pragma unroll
                    for (int e = 0; e < N; ++e) x[f] = fmaf(q[i][e], w[e], x[f]);
                }
            }
#pragma unroll
            for (int k = L >> 1; k > 0; k >>= 1)
#pragma unroll
                for (int f = 0; f < GATHER_FLIGHT; ++f) x[f] += __shfl_xor_sync(0xffffffffu, x[f], k);
#pragma unroll
            for (int f = 0; f < GATHER_FLIGHT; ++f) {
                if (!live[f]) x[f] = -INFINITY;
                top = max_nan(top, x[f]);
            }
#pragma unroll
            for (int k = L; k < 32; k <<= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, k));
            if (top == -INFINITY) continue;                  // no row that weighs anything (uniform)
            const float m1 = max_nan(m, top), keep = exp2f(m - m1);
            m = m1;
            l *= keep;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) o[i][e] *= keep;
#pragma unroll
            for (int f = 0; f < GATHER_FLIGHT; ++f) {
                const float p = exp2f(x[f] - m);
                l += p;
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    float w[N];
                    Row<T>::widen(vv[f][i], w);
#pragma unroll
                    for (int e = 0; e < N; ++e) o[i][e] = fmaf(p, w[e], o[i][e]);
                }
            }
        }
    }
#pragma unroll
    for (int k = L; k < 32; k <<= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, k);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) o[i][e] += __shfl_xor_sync(0xffffffffu, o[i][e], k);
    }
    if (group == 0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) s_o[warp][(sub + L * i) * N + e] = o[i][e];
    }
    if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
    __syncthreads();
    if (threadIdx.x >= s.d / N) return;
    float top = -INFINITY, total = 0.f, y[N];
    for (int w = 0; w < n_warps; ++w) top = max_nan(top, s_m[w]);
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = 0.f;
    if (top != -INFINITY) {
        for (int w = 0; w < n_warps; ++w) {
            const float f = exp2f(s_m[w] - top);
            total = fmaf(f, s_l[w], total);
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = fmaf(f, s_o[w][threadIdx.x * N + e], y[e]);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] /= total;
    }
    const int64_t at = ((int64_t)u * s.mn + cell) * D + h * s.d + threadIdx.x * N;
    if (a.residual) {
        float r[N];
        Row<T>::widen(*reinterpret_cast<const uint4 *>(static_cast<const T *>(a.residual) + at), r);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] += r[e];
    }
    *reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + at) = Row<T>::narrow(y);
}

using GatherKernel = void (*)(AttendArgs);

template <typename T>
GatherKernel gather_kernel(int pieces)         // a power of two: of 2 (bf16) or 4 (fp32) to 32
{
    switch (pieces) {
    case 2: return k_attend_gather<T, 1, 2>;
    case 4: return k_attend_gather<T, 1, 4>;
    case 8: return k_attend_gather<T, 1, 8>;
    case 16: return k_attend_gather<T, 1, 16>;
    default: return k_attend_gather<T, 1, 32>;
    }
}

// ---------------------------------------------------------------------------
// by block
// ---------------------------------------------------------------------------
constexpr int TILE = 64, TILE_FP32 = 32;   // queries of an item: four tiles of 16, or eight warps' four each
constexpr int LIST_THREADS = 512;
constexpr int LIST_HELD = 8;               // list entries that a thread holds
constexpr int LIST_BINS = 8192;            // blocks that are counted at a time
constexpr int LIST_CTAS = 8;               // largest cluster of a (unit, head)
constexpr int MAX_HEADS = 1024;            // (unit, head) pairs whose item counts a CTA of the attention holds at a time
constexpr int CHUNK_ITEMS = 64;            // items whose records it holds

// Part of a block (part_rows() of its rows) and up to TILE (TILE_FP32) of the queries that chose it.
struct BlockItem {
    int32_t uh, part, first, n;            // unit * H + head, its rows in parts, first list entry, entries
    uint32_t live[2];                      // its live rows
    int64_t q;                             // element of its unit's and head's first query row (k_attend_blocks)
};

struct BlockWork {                         // in the workspace
    int32_t *n_items;                      // [U * H]
    BlockItem *items;                      // [U * H][max_items]
    int2 *list;                            // [U * H][k_max * n_top]: (query * n_top + entry, row of the query)
    uint4 *q;                              // [U][k_max][H * d]: the kept queries, rotated (calls with angles)
    float2 *ml;                            // [U * H][k_max][n_top][parts]: (max in the log2 domain, sum)
    float *o;                              // [U * H][k_max][n_top][parts][d]
    int32_t cluster, bins, parts, parts_log2, tile, tile_log2, list_ctas, pass_ctas;
    int64_t max_items;
    uint64_t wait_ns;                      // limit of each wait
    uint32_t per_top, per_top_shift;       // x / n_top = x * per_top >> per_top_shift for x < 2^28
};

// 16 bytes of a query, rotated.
template <typename T>
__device__ __forceinline__ uint4 rotate_piece(uint4 v, const float *f)
{
    if (sizeof(T) == 2) return rotate_q_piece(v, f);
    const float4 c = __ldg(reinterpret_cast<const float4 *>(f));
    float x[4], y[4];
    Row<float>::widen(v, x);
    y[0] = x[0] * c.x - x[1] * c.y;
    y[1] = x[0] * c.y + x[1] * c.x;
    y[2] = x[2] * c.z - x[3] * c.w;
    y[3] = x[2] * c.w + x[3] * c.z;
    return Row<float>::narrow(y);
}

// The queries of every block, a counting sort: the CTAs of a cluster share the list entries of one (unit, head).
// Each counts its entries per block in shared memory; then each owns some of the blocks, adds up their counts
// through distributed shared memory, gives every block a run of the sorted list and its items, and
// tells every CTA where its entries of the block go.  Entries of one block come in any order; each
// is computed by itself, so the result does not depend on it.  Out of place the launch's other CTAs
// write out = residual (or zeros) on every cell, and with angles a further few rotate the kept queries once for all
// of their blocks (in fp32; bf16 queries rounded to bf16 for the tensor cores).  Bound by latency: three cluster barriers and some
// six dependent loads, 13 us for one head's 24 200 entries over 4 700 blocks and 16 for 32 heads' 372 000 over 990 with
// 17 MB passed through; with every CTA going through all of a head's entries for its share of the blocks 18 and 22.
template <typename T>
__global__ void __launch_bounds__(LIST_THREADS, 2) k_block_lists(AttendArgs a, BlockWork w, int64_t nvec)
{
    pdl_wait();
    if ((int)blockIdx.x >= w.list_ctas) {
        const uint4 *res = static_cast<const uint4 *>(a.residual);
        uint4 *out = static_cast<uint4 *>(a.out);
        const int64_t first = (int64_t)((int)blockIdx.x - w.list_ctas) * LIST_THREADS + threadIdx.x;
        const int64_t pass = (int64_t)w.pass_ctas * LIST_THREADS;
        if (first < pass) {
            for (int64_t i = first; i < nvec; i += 4 * pass) {
                uint4 v[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) v[f] = res && i + f * pass < nvec ? __ldcs(res + i + f * pass) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int f = 0; f < 4; ++f)
                    if (i + f * pass < nvec) out[i + f * pass] = v[f];
            }
            return;
        }
        const SparseArgs &s = a.s;
        if (!s.rope) return;                           // (the grid is whole clusters)
        constexpr int N = Row<T>::N;
        const int width = s.H * s.d / N;               // 16-byte pieces of a query row
        const int64_t i = first - pass;
        const int u = (int)(i / ((int64_t)s.k_max * width)), r = (int)(i - (int64_t)u * s.k_max * width), j = r / width, c = r - j * width;
        if (u >= s.U) return;
        const int cnt = s.count[u], g = s.unit_group[u];
        if (cnt > s.k_max || j >= cnt || g < 0 || g >= s.G) return;
        const int cell = s.idx[(int64_t)u * s.k_max + j];
        if (cell < 0 || cell >= s.mn) return;
        const uint4 x = __ldg(static_cast<const uint4 *>(s.q) + ((int64_t)g * s.mn + cell) * width + c);
        w.q[i] = rotate_piece<T>(x, s.rope + (int64_t)cell * s.d + (c * N & (s.d - 1)));
        return;
    }
    extern __shared__ int32_t s_bin[];                 // [bins] counts, then next places
    __shared__ int32_t s_part[2][LIST_THREADS / 32], s_total[LIST_CTAS][2];
    const SparseArgs &s = a.s;
    const int C = w.cluster, rank = (int)cluster_rank(), uh = (int)blockIdx.x / C, u = uh / s.H;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t base = (int64_t)uh * s.k_max * s.n_top;
    const int32_t *sel = a.sel + base, *idx = s.idx + (int64_t)u * s.k_max;
    const int first = rank * LIST_THREADS + (int)threadIdx.x, step = C * LIST_THREADS, most = s.k_max * s.n_top;
    const auto query_of = [&](int e) { return (int)((uint64_t)(uint32_t)e * w.per_top >> w.per_top_shift); };     // e / n_top
    // the first entries and their queries' cells are on their way while the unit's counters are read
    int held[LIST_HELD], row[LIST_HELD];               // blocks; rows of their queries, -1 for none
#pragma unroll
    for (int i = 0; i < LIST_HELD; ++i) {
        const int e = first + i * step;
        held[i] = e < most ? __ldg(sel + e) : -1;
        row[i] = e < most ? __ldg(idx + query_of(e)) : 0;
    }
    int cnt, g;
    LiveRows rows;
    // (the same for the whole cluster)
    if (!sparse_unit(s, u, threadIdx.x == 0 && rank == 0 && uh == u * s.H, cnt, g, rows)) {
        if (threadIdx.x == 0 && rank == 0) w.n_items[uh] = 0;
        return;
    }
    const int pairs = cnt * s.n_top;
    bool bad = false;                                  // a query off the grid (it is in no list), a block past the last
    const auto row_of = [&](int e, int b, int cell) {
        if (e >= pairs) return -1;
        const bool off = (uint32_t)cell >= (uint32_t)s.mn;
        bad |= off || b >= s.nb;
        return off || b >= s.nb ? -1 : s.rope ? query_of(e) : cell;
    };
#pragma unroll
    for (int i = 0; i < LIST_HELD; ++i) row[i] = row_of(first + i * step, held[i], row[i]);
    const int pr = s.bs / w.parts;                     // rows of a part
    int entry0 = 0, item0 = 0;                         // of this window of blocks
    for (int lo = 0; lo < s.nb; lo += w.bins) {
        const int n_bins = min(w.bins, s.nb - lo);
        for (int i = threadIdx.x; i < n_bins; i += LIST_THREADS) s_bin[i] = 0;
        __syncthreads();
        const auto each = [&](auto f) {                // f(entry, block of the window, row of its query)
#pragma unroll
            for (int i = 0; i < LIST_HELD; ++i)
                if (row[i] >= 0 && (uint32_t)(held[i] - lo) < (uint32_t)n_bins) f(first + i * step, held[i] - lo, row[i]);
            for (int e = first + LIST_HELD * step; e < pairs; e += step) {
                const int b = __ldg(sel + e), r = row_of(e, b, __ldg(idx + query_of(e)));
                if (r >= 0 && (uint32_t)(b - lo) < (uint32_t)n_bins) f(e, b - lo, r);
            }
        };
        each([&](int, int b, int) { atomicAdd(&s_bin[b], 1); });
        cluster_barrier();
        // a run of blocks for each thread
        const int own = (n_bins + C - 1) / C, per = (own + LIST_THREADS - 1) / LIST_THREADS;
        const int end = min(n_bins, (rank + 1) * own);
        const int b0 = min(end, rank * own + (int)threadIdx.x * per), b1 = min(end, b0 + per);
        int entries = 0, items = 0, c[LIST_CTAS];      // the CTAs' entries of one block
        const auto counts = [&](int b) {
            int n = 0;
#pragma unroll
            for (int r = 0; r < LIST_CTAS; ++r) c[r] = r < C ? (int)dsmem_ld_u32(dsmem_addr(s_bin + b, r)) : 0;
#pragma unroll
            for (int r = 0; r < LIST_CTAS; ++r) n += c[r];
            return n;
        };
        for (int b = b0; b < b1; ++b) {
            const int n = counts(b);
            entries += n;
            items += (n + w.tile - 1) >> w.tile_log2;
        }
        int e_sum = entries, i_sum = items;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, e_sum, o), y = __shfl_up_sync(0xffffffffu, i_sum, o);
            if (lane >= o) { e_sum += x; i_sum += y; }
        }
        if (lane == 31) { s_part[0][warp] = e_sum; s_part[1][warp] = i_sum; }
        __syncthreads();
        int e_all = 0, i_all = 0;
#pragma unroll
        for (int i = 0; i < LIST_THREADS / 32; ++i) {
            if (i == warp) { e_sum += e_all; i_sum += i_all; }
            e_all += s_part[0][i];
            i_all += s_part[1][i];
        }
        if ((int)threadIdx.x < C) {
            dsmem_st_u32(dsmem_addr(&s_total[rank][0], threadIdx.x), (uint32_t)e_all);
            dsmem_st_u32(dsmem_addr(&s_total[rank][1], threadIdx.x), (uint32_t)i_all);
        }
        cluster_barrier();
        int next = entry0 + e_sum - entries, item = item0 + i_sum - items;
        for (int r = 0; r < C; ++r) {
            if (r < rank) { next += s_total[r][0]; item += s_total[r][1]; }
            entry0 += s_total[r][0];
            item0 += s_total[r][1];
        }
        BlockItem *out = w.items + uh * w.max_items + (int64_t)item * w.parts;
        for (int b = b0; b < b1; ++b) {
            const int from = next;
            if (per > 1) counts(b);                    // (else they are at hand)
#pragma unroll
            for (int r = 0; r < LIST_CTAS; ++r)
                if (r < C) {
                    dsmem_st_u32(dsmem_addr(s_bin + b, r), (uint32_t)next);
                    next += c[r];
                }
            for (int p = 0; next > from && p < w.parts; ++p) {
                BlockItem it = {};
                it.uh = uh;
                it.part = (lo + b) * w.parts + p;
                const uint64_t live = rows.mask64((int64_t)it.part * pr);
                it.live[0] = (uint32_t)live;
                it.live[1] = pr > 32 ? (uint32_t)(live >> 32) : 0u;
                for (int e = from; e < next; e += w.tile) {
                    it.first = e;
                    it.n = min(w.tile, next - e);
                    *out++ = it;
                }
            }
        }
        cluster_barrier();                             // (the last use of another CTA's shared memory)
        int2 *list = w.list + base;
        each([&](int e, int b, int r) { list[atomicAdd(&s_bin[b], 1)] = make_int2(e, r); });
        __syncthreads();
    }
    if (threadIdx.x == 0 && rank == 0) w.n_items[uh] = item0 * w.parts;
    if (bad) latch_status(s.status, RS3_EINVAL);
}

__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void ld_matrix4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// c (16 x 8, fp32) += a (16 x 16, bf16) b (16 x 8, bf16)
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int D, int TR>
struct BlockTile {
    static constexpr int CONSUMERS = 7, THREADS = 32 * (CONSUMERS + 1);
    static constexpr int CTAS = D == 256 ? 1 : 2;      // per SM
    static constexpr int HALF = TR * D * 2, STAGE = 2 * HALF;      // bytes of a part's keys; keys and values
    static constexpr int FIT = (D == 256 ? 196608 : 98304) / STAGE, STAGES = FIT > 8 ? 8 : FIT;
    static constexpr int SMEM = STAGES * STAGE + 1024;             // stages begin at a multiple of 1 KB
    // the next tile's queries are loaded while a tile goes on, where the registers have room (heads of 128: 98.6 us
    // without it, 102.9 with, 4 100 queries of 16 blocks; heads of 64 took 121 us for 129)
    static constexpr bool EARLY = D != 128;
};

// Persistent CTAs walk the items.  A producer thread brings the parts' keys and values by TMA (128-byte
// swizzle) into a ring of stages; every consumer warp takes tiles of 16 queries by itself, item after item:
// S = Q K^T from query fragments that it loads straight from the grid (the columns of a 64-column box
// are taken in the order in which adjacent lanes can load 16 bytes of a row), the softmax of its rows in
// registers, O = P V from those, and (m, l, O) stored for k_join_blocks.  No warp waits for another.
// mma.sync: a block of a long bank has some 20 queries, so the call is bound by the bytes of K and V, and
// tiles of 128 rows would be four fifths empty.  23 264 queries of 16 blocks in 32 heads of 64 (18 538 blocks, 304 MB read
// and 97 MB of results): 75 us, 5.3 TB/s; the loads alone take 60.  757 queries of 32 blocks, one head of 256 (1 278 blocks, 84 MB): 28 us,
// 21 of them the loads with their start and end.  The weights are rounded to bf16 for the second product, as the dense
// readout's are; their sum and every partial result stay fp32.  A weight is off by 2^-8 of itself at most, either way, and a
// result by less: 7.1e-4 and 7.0e-4 from 64 bits in the two calls above, by its own rounding; fp32 weights give the same.  Seven warps
// and the producer leave 128 registers (255 at D = 256)
// where eight and it left 96.
template <int D, int TR>
__global__ void __launch_bounds__(BlockTile<D, TR>::THREADS, BlockTile<D, TR>::CTAS)
k_attend_blocks(AttendArgs a, BlockWork w, const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv)
{
    using X = BlockTile<D, TR>;
    using namespace tc;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_bars[2 * X::STAGES];
    __shared__ int32_t s_first[MAX_HEADS + 1];
    __shared__ BlockItem s_item[CHUNK_ITEMS];
    __shared__ int s_abort;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    const uint32_t full = smem_u32(s_bars), empty = full + 8u * X::STAGES;
    volatile int *abort_flag = &s_abort;
    const SparseArgs &s = a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < X::STAGES; ++i) {
            mbar_init(full + 8u * i, 1);
            mbar_init(empty + 8u * i, X::CONSUMERS);
        }
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmk)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmv)) : "memory");
    }
    pdl_wait();
    const int heads = s.U * s.H;
    const int64_t row_elems = (int64_t)s.H * D;
    uint32_t cnt = 0, issued = 0;                      // parts gone through: stage cnt % STAGES, phase cnt / STAGES; the producer's
    int next = blockIdx.x, turn = 0;                   // this CTA's next item; the warp that takes the next tile
    for (int g0 = 0; g0 < heads; g0 += MAX_HEADS) {
        const int n = min(MAX_HEADS, heads - g0);
        const auto before_each = [&]() {               // items before each (unit, head)
            int run = 0;
            for (int c0 = 0; c0 < n; c0 += 32) {
                int v = c0 + lane < n ? w.n_items[g0 + c0 + lane] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int t = __shfl_up_sync(0xffffffffu, v, o);
                    if (lane >= o) v += t;
                }
                if (c0 + lane < n) s_first[c0 + lane + 1] = run + v;
                run += __shfl_sync(0xffffffffu, v, 31);
            }
            if (lane == 0) s_first[0] = 0;
        };
        if (heads <= 32) {                             // every warp for itself, the same values: no barrier
            before_each();
            __syncwarp();
        } else {
            __syncthreads();
            if (warp == 0) before_each();
            __syncthreads();
        }
        const int total = s_first[n];
        while (next < total) {
            // the records of this CTA's next items
            const int chunk = min(CHUNK_ITEMS, (total - next + (int)gridDim.x - 1) / (int)gridDim.x);
            if ((int)threadIdx.x < chunk) {
                const int at = next + threadIdx.x * gridDim.x;
                int x = 0, y = n;                      // the last one whose items begin at or before `at`
                while (y - x > 1) {
                    const int mid = (x + y) >> 1;
                    if (s_first[mid] <= at) x = mid; else y = mid;
                }
                BlockItem it = w.items[(g0 + x) * w.max_items + (at - s_first[x])];
                const int u = it.uh / s.H;
                it.q = ((s.rope ? (int64_t)u * s.k_max : (int64_t)__ldg(s.unit_group + u) * s.mn) * s.H + (it.uh - u * s.H)) * D;
                s_item[threadIdx.x] = it;
            }
            __syncthreads();
            if (warp == X::CONSUMERS) {
                if (lane == 0) {
                    const uint64_t once = l2_once();   // L2 keeps the results for k_join_blocks (21 -> 18.5 us there)
                    uint32_t k = cnt;
                    for (int i = 0; i < chunk; ++i, ++k) {
                        const uint32_t st = k % X::STAGES;
                        if (!mbar_wait(empty + 8u * st, (k / X::STAGES & 1u) ^ 1u, abort_flag, w.wait_ns)) break;
                        const int u = s_item[i].uh / s.H, h = s_item[i].uh - u * s.H;
                        const int y = (int)(u * s.bank.rows_per_unit + (int64_t)s_item[i].part * TR);
                        const uint32_t dst = base + st * X::STAGE, bar = full + 8u * st;
                        mbar_expect_tx(bar, X::STAGE);
#pragma unroll
                        for (int c = 0; c < D / 64; ++c) tma_load_2d_once(dst + c * (TR * 128), &tmk, bar, h * D + c * 64, y, once);
#pragma unroll
                        for (int c = 0; c < D / 64; ++c) tma_load_2d_once(dst + X::HALF + c * (TR * 128), &tmv, bar, h * D + c * 64, y, once);
                    }
                    issued = k;
                }
                __syncwarp();
            } else {
                bool ok = true;
                const int r = lane >> 2, t = lane & 3;
                // the warps take the items' tiles in turn (an item has four at most)
                const auto next_turn = [](int turn, int n) {
                    turn += (n + 15) >> 4;
                    return turn >= X::CONSUMERS ? turn - X::CONSUMERS : turn;
                };
                // list entries of this warp's next tile, at or behind item i (rows lane / 4 and + 8), and its queries:
                // of 64 columns this lane holds the pieces 2 (lane % 4) and + 1
                int2 ahead[2];
                int64_t ahead_q = 0;
                const auto look_ahead = [&](int i, int turn) {
                    ahead[0] = ahead[1] = make_int2(-1, -1);
                    for (; i < chunk; turn = next_turn(turn, s_item[i].n), ++i) {
                        const int tile = warp - turn + (warp < turn ? X::CONSUMERS : 0), m = s_item[i].n - tile * 16;
                        if (m <= 0) continue;
                        const int2 *list = w.list + (int64_t)s_item[i].uh * s.k_max * s.n_top + s_item[i].first + tile * 16;
#pragma unroll
                        for (int x = 0; x < 2; ++x)
                            if (r + 8 * x < m) ahead[x] = __ldg(list + r + 8 * x);
                        ahead_q = s_item[i].q;
                        break;
                    }
                };
                const uint16_t *rotated = reinterpret_cast<const uint16_t *>(w.q);
                const uint16_t *Q = s.rope ? rotated : static_cast<const uint16_t *>(s.q);
                uint4 q[2][D / 32];
                const auto load_q = [&]() {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            q[x][c] = make_uint4(0, 0, 0, 0);
                            if (ahead[x].y >= 0)
                                q[x][c] = __ldg(reinterpret_cast<const uint4 *>(Q + ahead_q + ahead[x].y * row_elems) + (c >> 1) * 8 + 2 * t + (c & 1));
                        }
                };
                look_ahead(0, turn);
                if (X::EARLY) load_q();
                for (int i = 0; i < chunk && ok; ++i) {
                    const uint32_t k = cnt + i, st = k % X::STAGES;
                    const int tile = warp - turn + (warp < turn ? X::CONSUMERS : 0);
                    const int m = s_item[i].n - tile * 16;     // queries of this warp's tile
                    turn = next_turn(turn, s_item[i].n);
                    if (m <= 0) {                      // the others'
                        ok = mbar_wait_warp(full + 8u * st, k / X::STAGES & 1u, abort_flag, w.wait_ns);
                        if (ok && lane == 0) mbar_arrive(empty + 8u * st);
                        continue;
                    }
                    const int64_t pair0 = (int64_t)s_item[i].uh * s.k_max * s.n_top;
                    const int entry[2] = {ahead[0].x, ahead[1].x};
                    if (!X::EARLY) load_q();
                    look_ahead(i + 1, turn);
                    ok = mbar_wait_warp(full + 8u * st, k / X::STAGES & 1u, abort_flag, w.wait_ns);
                    if (!ok) break;
                    const uint32_t sk = base + st * X::STAGE, sv = sk + X::HALF;
                    const uint32_t live[2] = {s_item[i].live[0], s_item[i].live[1]};
                    const bool whole = live[0] == 0xffffffffu && (TR == 32 || live[1] == 0xffffffffu);
                    float c[TR / 8][4];
#pragma unroll
                    for (int x = 0; x < TR / 8; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) c[x][y] = 0.f;
#pragma unroll
                    for (int b = 0; b < D / 32; ++b) {
                        const uint32_t col = sk + (b >> 1) * (TR * 128) + (((2 * t + (b & 1)) ^ r) << 4);
#pragma unroll
                        for (int x = 0; x < TR / 8; ++x) {
                            const uint4 y = lds128(col + (x * 8 + r) * 128);
                            mma_16x8x16(c[x], q[0][b].x, q[1][b].x, q[0][b].y, q[1][b].y, y.x, y.y);
                            mma_16x8x16(c[x], q[0][b].z, q[1][b].z, q[0][b].w, q[1][b].w, y.z, y.w);
                        }
                    }
                    if (X::EARLY) load_q();            // the next tile's, while this one goes on
                    // this lane holds keys 8 x + 2 t, + 1 of its two rows
                    if (!whole) {
#pragma unroll
                        for (int x = 0; x < TR / 8; ++x)
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                if (!(live[x >> 2] >> ((x & 3) * 8 + 2 * t + (y & 1)) & 1u)) c[x][y] = -INFINITY;
                    }
                    float mx[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f}, ref[2];
#pragma unroll
                    for (int x = 0; x < TR / 8; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) mx[y >> 1] = fmaxf(mx[y >> 1], c[x][y]);
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], 1));
                        mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], 2)) * a.scale_log2;
                        ref[y] = mx[y] == -INFINITY ? 0.f : -mx[y];
                    }
                    uint32_t p[TR / 8][2];
#pragma unroll
                    for (int x = 0; x < TR / 8; ++x)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const float p0 = ex2_approx(fmaf(c[x][2 * y], a.scale_log2, ref[y]));
                            const float p1 = ex2_approx(fmaf(c[x][2 * y + 1], a.scale_log2, ref[y]));
                            sum[y] += p0 + p1;
                            p[x][y] = pack_bf16x2(p0, p1);
                        }
                    if (!whole) {                      // dead rows may hold anything: as values they are zeros
                        for (int row = 0; row < TR; ++row)
                            if (!(live[row >> 5] >> (row & 31) & 1u) && lane < D / 8)
                                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};"
                                             ::"r"(sv + (lane >> 3) * (TR * 128) + row * 128 + (lane & 7) * 16), "r"(0) : "memory");
                        fence_proxy_async();
                        __syncwarp();
                    }
                    float o[D / 8][4];
#pragma unroll
                    for (int x = 0; x < D / 8; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
#pragma unroll
                    for (int b = 0; b < TR / 16; ++b) {
                        const uint32_t row = sv + (b * 16 + (lane & 15)) * 128;
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            uint32_t v[4];
                            ld_matrix4_t(v, row + (x >> 2) * (TR * 128) + ((((x & 3) * 2 + (lane >> 4)) ^ (lane & 7)) << 4));
                            mma_16x8x16(o[2 * x], p[2 * b][0], p[2 * b][1], p[2 * b + 1][0], p[2 * b + 1][1], v[0], v[1]);
                            mma_16x8x16(o[2 * x + 1], p[2 * b][0], p[2 * b][1], p[2 * b + 1][0], p[2 * b + 1][1], v[2], v[3]);
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(empty + 8u * st);
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 1);
                        sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 2);
                        if (entry[y] < 0) continue;
                        const int64_t slot = (pair0 + entry[y]) * w.parts + s_item[i].part % w.parts;
                        if (t == 0) w.ml[slot] = make_float2(sum[y] == sum[y] ? mx[y] : sum[y], sum[y]);   // (NaN for the join)
                        float *dst = w.o + slot * D + 2 * t;
#pragma unroll
                        for (int x = 0; x < D / 8; ++x)
                            *reinterpret_cast<float2 *>(dst + 8 * x) = make_float2(o[x][2 * y], o[x][2 * y + 1]);
                    }
                    __syncwarp();
                }
            }
            __syncthreads();                           // the records are read
            if (*abort_flag) {                         // the same for all threads: it is set before the barrier
                if (threadIdx.x == 0) latch_status(s.status, RS3_ETIMEOUT);
                // copies in flight land before the CTA ends (only the producer's thread has issued any)
                for (uint32_t d = issued > X::STAGES ? issued - X::STAGES : 0; d < issued; ++d)
                    mbar_drain(full + 8u * (d % X::STAGES), d / X::STAGES & 1u);
                return;
            }
            cnt += chunk;
            next += chunk * (int)gridDim.x;
            __syncthreads();
        }
        next -= total;
    }
}

// The same in fp32 on the CUDA cores.  A CTA brings a part's rows into shared memory and its warps take its queries, four
// each: a lane holds the scores of a row (of two, where a part has 64), so that a key read once serves four queries, then
// the columns that it adds up, a value read once for the four.  Four CTAs per SM (heads of 64) load while others compute.
// Bound by the latency of an item (its load, its scores, its sums) and next by shared-memory reads.  9 500 queries of 16
// blocks in 16 heads of 64: the call takes 206 us, by query 617; four warps with up to sixteen queries each 260, eight queries
// to a warp 237.
template <int D, int PR>
struct Fp32Tile {
    static constexpr int WARPS = 8, THREADS = 32 * WARPS, QUERIES = 4, PITCH = D + 4;     // floats of a key row: lanes meet different banks
    static constexpr int KEYS = PR * PITCH, VALUES = PR * D, Q = QUERIES * D, P = PR * QUERIES;
    static constexpr int SMEM = (KEYS + VALUES + WARPS * (Q + P)) * 4;
};

template <int D, int PR>
__global__ void __launch_bounds__(Fp32Tile<D, PR>::THREADS) k_attend_blocks_fp32(AttendArgs a, BlockWork w)
{
    using X = Fp32Tile<D, PR>;
    constexpr int M = X::QUERIES, S = PR / 32, V4 = D < 128 ? 1 : D / 128;      // score rows, column groups of a lane
    extern __shared__ __align__(16) float s_mem[];
    __shared__ int32_t s_first[MAX_HEADS + 1];
    pdl_wait();
    const SparseArgs &s = a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *s_k = s_mem, *s_v = s_k + X::KEYS, *s_q = s_v + X::VALUES + warp * (X::Q + X::P), *s_p = s_q + X::Q;
    const float *Q = s.rope ? reinterpret_cast<const float *>(w.q) : static_cast<const float *>(s.q);
    const int heads = s.U * s.H;
    const int64_t row_elems = (int64_t)s.H * D;
    int next = blockIdx.x;
    for (int g0 = 0; g0 < heads; g0 += MAX_HEADS) {
        const int n = min(MAX_HEADS, heads - g0);
        __syncthreads();
        if (warp == 0) {                               // items before each (unit, head)
            int run = 0;
            for (int c0 = 0; c0 < n; c0 += 32) {
                int v = c0 + lane < n ? w.n_items[g0 + c0 + lane] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int t = __shfl_up_sync(0xffffffffu, v, o);
                    if (lane >= o) v += t;
                }
                if (c0 + lane < n) s_first[c0 + lane + 1] = run + v;
                run += __shfl_sync(0xffffffffu, v, 31);
            }
            if (lane == 0) s_first[0] = 0;
        }
        __syncthreads();
        const int total = s_first[n];
        for (; next < total; next += gridDim.x) {
            int x = 0, y = n;                          // the last one whose items begin at or before `next`
            while (y - x > 1) {
                const int mid = (x + y) >> 1;
                if (s_first[mid] <= next) x = mid; else y = mid;
            }
            const BlockItem it = w.items[(g0 + x) * w.max_items + (next - s_first[x])];
            const int u = it.uh / s.H, h = it.uh - u * s.H;
            const float *K = reinterpret_cast<const float *>(a.k_store) + (u * s.bank.rows_per_unit) * row_elems + h * D;
            const float *V = reinterpret_cast<const float *>(a.v_store) + (u * s.bank.rows_per_unit) * row_elems + h * D;
            const uint64_t live = (uint64_t)it.live[1] << 32 | it.live[0];
            // dead rows may hold anything, or lie past the storage: they are zeros, and nothing is read
            for (int i = threadIdx.x; i < PR * (D / 4); i += X::THREADS) {
                const int r = i / (D / 4), c = 4 * (i % (D / 4)), bytes = (live >> r & 1u) ? 16 : 0;
                const int64_t at = bytes ? ((int64_t)it.part * PR + r) * row_elems + c : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                             ::"r"((uint32_t)__cvta_generic_to_shared(s_k + r * X::PITCH + c)), "l"(K + at), "r"(bytes) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                             ::"r"((uint32_t)__cvta_generic_to_shared(s_v + r * D + c)), "l"(V + at), "r"(bytes) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            const float *q_rows = Q + ((s.rope ? (int64_t)u * s.k_max : (int64_t)__ldg(s.unit_group + u) * s.mn) * s.H + h) * D;
            const int2 *list = w.list + (int64_t)it.uh * s.k_max * s.n_top + it.first;
            int2 entry = make_int2(-1, -1);            // of the warp's four queries: lane i's the i-th
            const auto load_q = [&](int q0) {
                entry = make_int2(-1, -1);
                if (lane < M && q0 + lane < it.n) entry = __ldg(list + q0 + lane);
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    const int row = __shfl_sync(0xffffffffu, entry.y, i);
#pragma unroll
                    for (int c = 4 * lane; c < D; c += 128)
                        *reinterpret_cast<float4 *>(s_q + i * D + c) =
                            row >= 0 ? __ldg(reinterpret_cast<const float4 *>(q_rows + row * row_elems + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
                __syncwarp();
            };
            if (M * warp < it.n) load_q(M * warp);
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();
            for (int q0 = M * warp; q0 < it.n; q0 += M * X::WARPS) {
                if (q0 != M * warp) load_q(q0);
                float c[S][M];
#pragma unroll
                for (int i = 0; i < S; ++i)
#pragma unroll
                    for (int q = 0; q < M; ++q) c[i][q] = 0.f;
#pragma unroll 4
                for (int e = 0; e < D; e += 4) {
                    float4 k[S];
#pragma unroll
                    for (int i = 0; i < S; ++i) k[i] = *reinterpret_cast<const float4 *>(s_k + (32 * i + lane) * X::PITCH + e);
#pragma unroll
                    for (int q = 0; q < M; ++q) {
                        const float4 z = *reinterpret_cast<const float4 *>(s_q + q * D + e);
#pragma unroll
                        for (int i = 0; i < S; ++i)
                            c[i][q] = fmaf(z.w, k[i].w, fmaf(z.z, k[i].z, fmaf(z.y, k[i].y, fmaf(z.x, k[i].x, c[i][q]))));
                    }
                }
                float mx[M], sum[M];
#pragma unroll
                for (int q = 0; q < M; ++q) {
                    mx[q] = -INFINITY;
#pragma unroll
                    for (int i = 0; i < S; ++i) {
                        if (!(live >> (32 * i + lane) & 1u)) c[i][q] = -INFINITY;
                        mx[q] = fmaxf(mx[q], c[i][q]);
                    }
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                    for (int q = 0; q < M; ++q) mx[q] = fmaxf(mx[q], __shfl_xor_sync(0xffffffffu, mx[q], o));
#pragma unroll
                for (int q = 0; q < M; ++q) {
                    mx[q] *= a.scale_log2;
                    const float ref = mx[q] == -INFINITY ? 0.f : -mx[q];
                    sum[q] = 0.f;
#pragma unroll
                    for (int i = 0; i < S; ++i) {
                        c[i][q] = exp2f(fmaf(c[i][q], a.scale_log2, ref));
                        sum[q] += c[i][q];
                    }
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                    for (int q = 0; q < M; ++q) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], o);
#pragma unroll
                for (int i = 0; i < S; ++i)
#pragma unroll
                    for (int q = 0; q < M; q += 4)
                        *reinterpret_cast<float4 *>(s_p + (32 * i + lane) * M + q) = make_float4(c[i][q], c[i][q + 1], c[i][q + 2], c[i][q + 3]);
                __syncwarp();
                // columns 4 lane, 128 + 4 lane, ... (heads of 64: 2 lane)
                constexpr int COLS = D < 128 ? 2 : 4;
                float o[M][V4][COLS];
#pragma unroll
                for (int q = 0; q < M; ++q)
#pragma unroll
                    for (int v = 0; v < V4; ++v)
#pragma unroll
                        for (int e = 0; e < COLS; ++e) o[q][v][e] = 0.f;
#pragma unroll 4
                for (int r = 0; r < PR; ++r) {
                    float pq[M];
#pragma unroll
                    for (int q = 0; q < M; q += 4) {
                        const float4 p = *reinterpret_cast<const float4 *>(s_p + r * M + q);
                        pq[q] = p.x; pq[q + 1] = p.y; pq[q + 2] = p.z; pq[q + 3] = p.w;
                    }
#pragma unroll
                    for (int v = 0; v < V4; ++v) {
                        const float *at = s_v + r * D + 128 * v + COLS * lane;
                        float4 f;
                        if (COLS == 4) f = *reinterpret_cast<const float4 *>(at);
                        else f = make_float4(at[0], at[1], 0.f, 0.f);
                        const float y[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                        for (int q = 0; q < M; ++q)
#pragma unroll
                            for (int e = 0; e < COLS; ++e) o[q][v][e] = fmaf(pq[q], y[e], o[q][v][e]);
                    }
                }
#pragma unroll
                for (int q = 0; q < M; ++q) {
                    const int e = __shfl_sync(0xffffffffu, entry.x, q);
                    if (e < 0) continue;               // (the same for the warp)
                    const int64_t slot = ((int64_t)it.uh * s.k_max * s.n_top + e) * w.parts + it.part % w.parts;
                    if (lane == 0) w.ml[slot] = make_float2(sum[q] == sum[q] ? mx[q] : sum[q], sum[q]);     // (NaN for the join)
#pragma unroll
                    for (int v = 0; v < V4; ++v) {
                        float *dst = w.o + slot * D + 128 * v + COLS * lane;
                        if (COLS == 2) *reinterpret_cast<float2 *>(dst) = make_float2(o[q][v][0], o[q][v][1]);
                        else *reinterpret_cast<float4 *>(dst) = make_float4(o[q][v][0], o[q][v][1], o[q][v][COLS - 2], o[q][v][COLS - 1]);
                    }
                }
                __syncwarp();                          // (the queries and weights are read)
            }
            __syncthreads();                           // the rows are read
        }
        next -= total;
    }
}

// Groups of D / 4 lanes, G = D / 64 to a (unit, head, query): each joins its share of the blocks' results by
// their running maximum, eight loads at a time, then the groups are joined:
//   out = residual + sum_t 2^(m_t - M) O_t / sum_t 2^(m_t - M) l_t
// Wide heads have few queries and much to load for each; for heads of 64 four groups a query took 33 us where
// one took 21 (23 264 queries of 16 blocks; 18.5 since the attention leaves its results in L2).
constexpr int JOIN_THREADS = 256;

template <typename T, int D>
__global__ void __launch_bounds__(JOIN_THREADS) k_join_blocks(AttendArgs a, BlockWork w)
{
    constexpr int L = D / 4, G = D / 64, PER = JOIN_THREADS / (G * L);
    pdl_wait();
    __shared__ float4 s_y[JOIN_THREADS];
    __shared__ float2 s_ml[JOIN_THREADS / L];
    const SparseArgs &s = a.s;
    const int u = blockIdx.y, sub = threadIdx.x % L, part = threadIdx.x / L;
    const int64_t jh = (int64_t)blockIdx.x * PER + part / G;
    const int j = (int)(jh / s.H), h = (int)(jh - (int64_t)j * s.H);
    const int cnt = s.count[u], g = s.unit_group[u];
    if (cnt < 0 || cnt > s.k_max || g < 0 || g >= s.G || (int64_t)blockIdx.x * PER >= (int64_t)cnt * s.H) return;
    const int cell = j < cnt ? s.idx[(int64_t)u * s.k_max + j] : -1;
    const bool here = cell >= 0 && cell < s.mn;
    const int64_t base = (((int64_t)u * s.H + h) * s.k_max + j) * s.n_top;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    // all of a query's loads go out together: what an entry without a block left in its place is not used
    // (a unit whose counters are unsound has no items: nothing was computed for it)
    const int n = j < cnt && w.n_items[u * s.H + h] > 0 ? s.n_top * w.parts : 0;
    constexpr int F = 8;                               // results in flight
    for (int t0 = part % G; t0 < n; t0 += G * F) {
        float2 ml[F];
        float4 v[F];
        int b[F];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int t = min(t0 + G * f, n - 1);
            b[f] = __ldg(a.sel + base + (t >> w.parts_log2));
            ml[f] = __ldg(w.ml + base * w.parts + t);
            v[f] = __ldcs(reinterpret_cast<const float4 *>(w.o + (base * w.parts + t) * D) + sub);
        }
#pragma unroll
        for (int f = 0; f < F; ++f)
            if (!here || t0 + G * f >= n || b[f] < 0 || b[f] >= s.nb) {
                ml[f] = make_float2(-INFINITY, 0.f);
                v[f] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
        float top = m;
#pragma unroll
        for (int f = 0; f < F; ++f) top = max_nan(top, ml[f].x);
        if (top == -INFINITY) continue;
        const float keep = exp2f(m - top);
        m = top;
        l *= keep;
        y = make_float4(y.x * keep, y.y * keep, y.z * keep, y.w * keep);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const float e = exp2f(ml[f].x - top);
            l = fmaf(e, ml[f].y, l);
            y = make_float4(fmaf(e, v[f].x, y.x), fmaf(e, v[f].y, y.y), fmaf(e, v[f].z, y.z), fmaf(e, v[f].w, y.w));
        }
    }
    if (G > 1) {
        s_y[threadIdx.x] = y;
        if (sub == 0) s_ml[part] = make_float2(m, l);
        __syncthreads();
        if (part % G != 0) return;
#pragma unroll
        for (int x = 1; x < G; ++x) m = max_nan(m, s_ml[part + x].x);
        y = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
        if (m != -INFINITY)
#pragma unroll
            for (int x = 0; x < G; ++x) {
                const float e = exp2f(s_ml[part + x].x - m);
                const float4 v = s_y[threadIdx.x + x * L];
                l = fmaf(e, s_ml[part + x].y, l);
                y = make_float4(fmaf(e, v.x, y.x), fmaf(e, v.y, y.y), fmaf(e, v.z, y.z), fmaf(e, v.w, y.w));
            }
    }
    if (!here) return;
    if (m != -INFINITY) {
        const float inv = 1.f / l;
        y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
    }
    const int64_t at = ((int64_t)u * s.mn + cell) * ((int64_t)s.H * D) + h * D + sub * 4;
    if (a.residual) {
        const float4 r = load4(static_cast<const T *>(a.residual) + at);
        y = make_float4(y.x + r.x, y.y + r.y, y.z + r.z, y.w + r.w);
    }
    if (sizeof(T) == 4) *reinterpret_cast<float4 *>(static_cast<T *>(a.out) + at) = y;
    else *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + at) = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
}

// Where the parts of a by-block call lie in its workspace.
struct WorkLayout {
    int64_t max_items;
    size_t n_items, items, list, q, ml, o, total;
};

// Rows of a block that an item takes: what the shared memory of the kernels holds several of.
int part_rows(bool fp32, int64_t d, int64_t bs) { return bs == 32 || (fp32 && d > 64) ? 32 : 64; }
int most_parts(bool fp32, int64_t d) { return 128 / part_rows(fp32, d, 128); }

WorkLayout work_layout(bool fp32, int64_t U, int64_t H, int64_t d, int64_t k_max, int64_t n_top, int64_t nb, int64_t parts)
{
    WorkLayout l = {};
    const int64_t uh = U * H, pairs = k_max * n_top;
    l.max_items = ((nb < pairs ? nb : pairs) + pairs / (fp32 ? TILE_FP32 : TILE) + 1) * parts;
    size_t at = 0;
    const auto part = [&](size_t bytes) {
        const size_t x = at;
        at = align_up(at + bytes, 256);
        return x;
    };
    l.n_items = part((size_t)uh * 4);
    l.items = part((size_t)(uh * l.max_items) * sizeof(BlockItem));
    l.list = part((size_t)(uh * pairs) * 8);
    l.q = part((size_t)(uh * k_max * d) * (fp32 ? 4 : 2));
    l.ml = part((size_t)(uh * pairs * parts) * 8);
    l.o = part((size_t)(uh * pairs * parts) * (size_t)d * 4);
    l.total = at;
    return l;
}

// Whether a call's path may be by block, for which its workspace is sized: the kernels by block are built for heads of 64, 128 and
// 256, and narrower heads are always by query.  Three launches against one, and every row
// read once against once per query.  bf16, of one bank of 200 frames, blocks of 64 (by block / by query): 4 heads of 64,
// 64 queries of 4 blocks 14.9 / 9.3 us, 128 of 4 15.5 / 15.4, 64 of 16 16.9 / 16.5, 128 of 16 18.5 / 30, 787 of 16
// 29 / 129; one head of 256, 16 queries of 4 blocks 16.0 / 21, 64 of 4 17.0 / 22, 787 of 16 33 / 162.
bool sized_by_blocks(rs3_dtype dtype, int64_t U, int64_t H, int64_t d, int64_t k_max, int64_t n_top)
{
    const double pairs = (double)U * H * k_max * n_top;
    return d >= 64 && (dtype == RS3_BF16 ? pairs * d * d * d >= 0x1p30 : pairs >= 4096);
}

// fp32 by the rows too, 6 000 lists' entries of 64: 4 heads of 64 of a bank of 100 frames, 64 queries of 16 blocks
// 22.9 / 20.6 us, 128 of 16 31 / 34, 300 of 4 28 / 22, 700 of 4 34 / 48, 700 of 16 68 / 163; one head of 256,
// 300 of 16 44 / 38, 700 of 16 74 / 111.  Beyond the sizes that the lists' and the tensor maps' 32-bit numbers
// hold it is by query.
bool by_blocks(const SparseArgs &s, rs3_dtype dtype)
{
    const bool fp32 = dtype == RS3_F32;
    return sized_by_blocks(dtype, s.U, s.H, s.d, s.k_max, s.n_top) && (int64_t)s.k_max * s.n_top < (1ll << 28) &&
           (!fp32 || (double)s.U * s.H * s.k_max * s.n_top * s.bs >= 0x1.8p18) &&
           (int64_t)s.U * s.H * work_layout(fp32, s.U, s.H, s.d, s.k_max, s.n_top, s.nb, most_parts(fp32, s.d)).max_items < (1ll << 30) &&
           s.U * s.bank.rows_per_unit < (1ll << 31) - 128;
}

template <int D, int TR>
rs3_status launch_attend(const AttendArgs &a, const BlockWork &w, cudaStream_t st)
{
    using X = BlockTile<D, TR>;
    const rs3_status r = rs3_kernel_smem((const void *)k_attend_blocks<D, TR>, X::SMEM);
    if (r != RS3_OK) return r;
    CUtensorMap mk, mv;
    const int64_t rows = a.s.U * a.s.bank.rows_per_unit, width = (int64_t)a.s.H * D;
    // a head of 64 is 128 bytes of a row: no more is fetched of its neighbour, whose turn comes later (78 -> 74 us)
    const CUtensorMapL2promotion grain = D == 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B;
    if (!tc::make_rows_map(&mk, a.k_store, 2, width, rows, 64, TR, true, grain) ||
        !tc::make_rows_map(&mv, a.v_store, 2, width, rows, 64, TR, true, grain))
        return RS3_ECUDA;
    launch_pdl(k_attend_blocks<D, TR>, dim3((unsigned)(rs3_sm_count() * X::CTAS)), dim3(X::THREADS), X::SMEM, st, a, w, mk, mv);
    return RS3_OK;
}

template <int D, int PR>
rs3_status launch_attend_fp32(const AttendArgs &a, const BlockWork &w, cudaStream_t st)
{
    using X = Fp32Tile<D, PR>;
    const rs3_status r = rs3_kernel_smem((const void *)k_attend_blocks_fp32<D, PR>, X::SMEM + 8 * 1024);   // (its static arrays count too)
    if (r != RS3_OK) return r;
    constexpr int CTAS = 220 * 1024 / (X::SMEM + 6 * 1024);
    launch_pdl(k_attend_blocks_fp32<D, PR>, dim3((unsigned)(rs3_sm_count() * CTAS)), dim3(X::THREADS), X::SMEM, st, a, w);
    return RS3_OK;
}

rs3_status launch_by_blocks(const AttendArgs &a, bool fp32, void *workspace, cudaStream_t st)
{
    const SparseArgs &s = a.s;
    const int parts = s.bs / part_rows(fp32, s.d, s.bs);
    const WorkLayout l = work_layout(fp32, s.U, s.H, s.d, s.k_max, s.n_top, s.nb, parts);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    BlockWork w = {};
    w.n_items = reinterpret_cast<int32_t *>(ws + l.n_items);
    w.items = reinterpret_cast<BlockItem *>(ws + l.items);
    w.list = reinterpret_cast<int2 *>(ws + l.list);
    w.q = reinterpret_cast<uint4 *>(ws + l.q);
    w.ml = reinterpret_cast<float2 *>(ws + l.ml);
    w.o = reinterpret_cast<float *>(ws + l.o);
    w.bins = s.nb < LIST_BINS ? s.nb : LIST_BINS;
    // with 2^t >= n_top and M = ceil(2^(28 + t) / n_top): x M / 2^(28 + t) is above x / n_top by less than 2^-t <= 1 / n_top
    uint32_t t = 0;
    while ((1 << t) < s.n_top) ++t;
    w.per_top_shift = 28 + t;
    w.per_top = (uint32_t)(((1ull << w.per_top_shift) + s.n_top - 1) / s.n_top);
    // the largest cluster whose CTAs are on the SMs at once
    w.cluster = LIST_CTAS;
    while (w.cluster > 1 && (int64_t)s.U * s.H * w.cluster > rs3_sm_count()) w.cluster /= 2;
    w.parts = parts;
    w.parts_log2 = parts == 4 ? 2 : parts - 1;
    w.tile = fp32 ? TILE_FP32 : TILE;
    w.tile_log2 = fp32 ? 5 : 6;
    static_assert(TILE_FP32 == 1 << 5 && TILE == 1 << 6, "their logarithms");
    w.list_ctas = s.U * s.H * w.cluster;
    w.max_items = l.max_items;
    w.wait_ns = rs3_get_wait_limit_ns();
    int64_t nvec = 0, pass = 0;
    if (a.out != a.residual) {
        nvec = (int64_t)s.U * s.mn * s.H * s.d / (fp32 ? 4 : 8);
        pass = (nvec + 4 * LIST_THREADS - 1) / (4 * LIST_THREADS);
        if (pass > 2 * rs3_sm_count()) pass = 2 * rs3_sm_count();
    }
    w.pass_ctas = (int32_t)pass;
    const int64_t turn = s.rope ? ((int64_t)s.U * s.k_max * s.H * s.d / (fp32 ? 4 : 8) + LIST_THREADS - 1) / LIST_THREADS : 0;
    const int64_t ctas = (w.list_ctas + pass + turn + w.cluster - 1) / w.cluster * w.cluster;     // whole clusters
    launch_pdl_cluster(fp32 ? k_block_lists<float> : k_block_lists<uint16_t>, w.cluster, dim3((unsigned)ctas), dim3(LIST_THREADS), (size_t)w.bins * 4, st, a, w, nvec);
    rs3_status r = RS3_EINTERNAL;
    const bool half = s.bs == 32;
    if (fp32) {
        if (s.d == 64) r = half ? launch_attend_fp32<64, 32>(a, w, st) : launch_attend_fp32<64, 64>(a, w, st);
        if (s.d == 128) r = launch_attend_fp32<128, 32>(a, w, st);
        if (s.d == 256) r = launch_attend_fp32<256, 32>(a, w, st);
    } else {
        if (s.d == 64) r = half ? launch_attend<64, 32>(a, w, st) : launch_attend<64, 64>(a, w, st);
        if (s.d == 128) r = half ? launch_attend<128, 32>(a, w, st) : launch_attend<128, 64>(a, w, st);
        if (s.d == 256) r = half ? launch_attend<256, 32>(a, w, st) : launch_attend<256, 64>(a, w, st);
    }
    if (r != RS3_OK) return r;
    void (*join)(AttendArgs, BlockWork) = s.d == 64 ? k_join_blocks<uint16_t, 64> : s.d == 128 ? k_join_blocks<uint16_t, 128> : k_join_blocks<uint16_t, 256>;
    if (fp32) join = s.d == 64 ? k_join_blocks<float, 64> : s.d == 128 ? k_join_blocks<float, 128> : k_join_blocks<float, 256>;
    const int per = JOIN_THREADS * 256 / (s.d * s.d);      // queries of a CTA: G * L lanes each
    launch_pdl(join, dim3((unsigned)(((int64_t)s.k_max * s.H + per - 1) / per), (unsigned)s.U), dim3(JOIN_THREADS), 0, st, a, w);
    return RS3_OK;
}

}  // namespace

static size_t readout_bytes(int U, int H, int d, int k_max, int n_top, int n_blocks, rs3_dtype dtype, int block)
{
    if (U < 1 || H < 1 || d < 1 || k_max < 0 || n_top < 1 || n_blocks < 0) return 0;
    if (dtype != RS3_F32 && dtype != RS3_BF16) return 0;
    const bool fp32 = dtype == RS3_F32;
    return 16 + (sized_by_blocks(dtype, U, H, d, k_max, n_top) ? work_layout(fp32, U, H, d, k_max, n_top, n_blocks, block / part_rows(fp32, d, block)).total : 0);
}

extern "C" size_t rs3_sparse_readout_workspace_bytes(int U, int H, int d, int k_max, int n_top, int n_blocks, rs3_dtype dtype)
{
    return readout_bytes(U, H, d, k_max, n_top, n_blocks, dtype, 128);
}

extern "C" size_t rs3_sparse_readout_block_workspace_bytes(int U, int H, int d, int k_max, int n_top, int n_blocks, rs3_dtype dtype,
                                                           int block)
{
    if (block != 32 && block != 64 && block != 128) return 0;
    return readout_bytes(U, H, d, k_max, n_top, n_blocks, dtype, block);
}

extern "C" rs3_status rs3_sparse_readout(const void *q, rs3_dtype dtype, int G, int mn, int H, int d,
                                         const int32_t *unit_group, const int32_t *idx, const int32_t *count, int k_max,
                                         const rs3_bank *bank, int block, const int32_t *sel, int n_top, const float *rope,
                                         const void *residual, void *out, float scale, void *workspace,
                                         size_t workspace_bytes, int32_t *status, rs3_stream_t stream)
{
    AttendArgs a = {};
    const rs3_status r = sparse_args(a.s, q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, block, rope, n_top, status);
    if (r != RS3_OK) return r;
    if (!sel || !out || !workspace || !(scale >= 0.f) || std::isinf(scale)) return RS3_EINVAL;
    if (!rs3_aligned16(out) || !rs3_aligned16(workspace) || (residual && !rs3_aligned16(residual))) return RS3_EINVAL;
    if (workspace_bytes < readout_bytes(a.s.U, H, d, k_max, n_top, a.s.nb, dtype, block)) return RS3_ECAPACITY;
    const bool blocks = a.s.nb > 0 && by_blocks(a.s, dtype);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    a.k_store = static_cast<const uint8_t *>(bank->k_store);
    a.v_store = static_cast<const uint8_t *>(bank->v_store);
    a.sel = sel;
    a.residual = residual;
    a.out = out;
    a.scale_log2 = (scale == 0.f ? 1.f / std::sqrt((float)d) : scale) * 1.4426950408889634f;
    if (out != residual && !blocks) {
        const int64_t nvec = (int64_t)a.s.U * mn * H * d * (int64_t)elem_bytes(dtype) / 16;
        const int64_t ctas = (nvec + 1023) / 1024, most = 8ll * rs3_sm_count();
        launch_pdl(k_pass_through, dim3((unsigned)(ctas < most ? ctas : most)), dim3(256), 0, st,
                   static_cast<const uint4 *>(residual), static_cast<uint4 *>(out), nvec);
    }
    if (blocks) {
        const rs3_status e = launch_by_blocks(a, dtype == RS3_F32, workspace, st);
        if (e != RS3_OK) return e;
    } else if (k_max > 0) {
        const int pieces = d * (int)elem_bytes(dtype) / 16;
        const dim3 grid((unsigned)k_max, (unsigned)H, (unsigned)a.s.U);
        // the fewer the queries, the more warps share a query's blocks, a block to a warp at least.  Of heads of 64 in fp32,
        // 16 blocks of 32 rows (16 / 8 / 4 warps): 128 CTAs 9.8 / 11.3 / 15.4 us, 600 CTAs 30 / 24 / 21; of 256, 300 CTAs
        // 27 / 23 / 28; 600 CTAs of 4 blocks 22 / 12.9 / 8.8
        const int64_t ctas = (int64_t)k_max * H * a.s.U;
        int warps = ctas <= rs3_sm_count() ? GATHER_WARPS : ctas <= 3ll * rs3_sm_count() ? GATHER_WARPS / 2 : GATHER_WARPS / 4;
        while (warps > GATHER_WARPS / 4 && warps >= 2 * n_top) warps /= 2;
        GatherKernel kern = k_attend_gather<float, 2, 32>;
        if (pieces <= 32) kern = dtype == RS3_BF16 ? gather_kernel<uint16_t>(pieces) : gather_kernel<float>(pieces);
        launch_pdl(kern, grid, dim3(32 * warps), 0, st, a);
    }
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
