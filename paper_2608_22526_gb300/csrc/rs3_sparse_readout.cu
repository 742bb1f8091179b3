// rs3_sparse_readout.cu -- attention of each kept query over the blocks listed for it, scattered
// back to the grid (Sec. 3.1's readout, Eq. 6 and Eq. 7, over chosen blocks of the bank).
//
// Two paths (by_blocks() holds the rule):
//   by query   a CTA per (query, head) reads the blocks of its list: few queries, fp32, narrow heads
//   by block   a block that many queries chose is read once for all of them: the lists are turned
//              into lists of queries per block (k_block_lists), a CTA per (block, up to 64 queries)
//              computes their attention over the block on the tensor cores (k_attend_blocks), and the
//              partial results of a query's blocks are joined by their log-sum-exp (k_join_blocks)
#include "rs3_sparse.cuh"

#include "rs3_readout_common.cuh"

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

constexpr int GATHER_WARPS = 4;
constexpr int GATHER_FLIGHT = 4;           // rows in flight per lane group

// A CTA per (query, head): its warps take the listed blocks in turn.  L lanes hold a row (ITEMS
// pieces of 16 bytes each), so a warp reads 32 / L rows at once; scores are summed over the L lanes,
// the softmax runs online per warp in the log2 domain, and the warps' results are joined at the end.
template <typename T, int ITEMS>
__global__ void __launch_bounds__(32 * GATHER_WARPS) k_attend_gather(AttendArgs a, int L)
{
    constexpr int N = Row<T>::N;
    pdl_wait();
    __shared__ float s_o[GATHER_WARPS][256];
    __shared__ float s_m[GATHER_WARPS], s_l[GATHER_WARPS];
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
    const int D = s.H * s.d, sub = lane & (L - 1), group = lane / L, groups = 32 / L;
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
    for (int t = warp; t < s.n_top; t += GATHER_WARPS) {
        const int b = sel[t];
        if (b < 0) continue;
        if (b >= s.nb) {
            if (lane == 0) latch_status(s.status, RS3_EINVAL);
            continue;
        }
        for (int r0 = 0; r0 < s.bs; r0 += groups * GATHER_FLIGHT) {
            bool live[GATHER_FLIGHT];
            float x[GATHER_FLIGHT], top = -INFINITY;
            uint4 kv[GATHER_FLIGHT][ITEMS], vv[GATHER_FLIGHT][ITEMS];
#pragma unroll
            for (int f = 0; f < GATHER_FLIGHT; ++f) {
                const int r = r0 + f * groups + group;
                const int64_t row = (int64_t)b * s.bs + r;
                live[f] = r < s.bs && rows.holds(row);
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
                for (int k = L >> 1; k > 0; k >>= 1) x[f] += __shfl_xor_sync(0xffffffffu, x[f], k);
                if (!live[f]) x[f] = -INFINITY;
                top = fmaxf(top, x[f]);
            }
            for (int k = L; k < 32; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
            if (top == -INFINITY) continue;                  // no live row (uniform)
            const float m1 = fmaxf(m, top), keep = exp2f(m - m1);
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
#pragma unroll
    for (int w = 0; w < GATHER_WARPS; ++w) top = fmaxf(top, s_m[w]);
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = 0.f;
    if (top > -INFINITY) {
#pragma unroll
        for (int w = 0; w < GATHER_WARPS; ++w) {
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

// ---------------------------------------------------------------------------
// by block
// ---------------------------------------------------------------------------
constexpr int TILE = 64;                   // queries of an item
constexpr int LIST_THREADS = 512;
constexpr int LIST_BINS = 8192;            // blocks that a CTA counts
constexpr int MAX_SEGMENTS = 1024;         // (unit, head, segment) triples that a CTA of the attention holds at a time

// A block and up to TILE of the queries that chose it.
struct BlockItem {
    int32_t uh, b, first, n;               // unit * H + head, block, first list entry, entries
    uint32_t live[4];                      // its live rows
};

struct BlockWork {                         // in the workspace
    int32_t *n_items, *first_item;         // [U * H][segments]
    BlockItem *items;                      // [U * H][max_items]
    int2 *list;                            // [U * H][k_max * n_top]: (query * n_top + entry, cell)
    float2 *ml;                            // [U * H][k_max][n_top]: (max in the log2 domain, sum)
    float *o;                              // [U * H][k_max][n_top][d]
    int32_t segments, bins;
    int64_t max_items;
};

// The queries of every block: CTA (segment, unit * H + head) counts the lists' entries for its
// blocks, gives every block a run of list entries and its items, and fills them in.  Entries of one block
// come in any order; each is computed by itself, so the result does not depend on it.
__global__ void __launch_bounds__(LIST_THREADS) k_block_lists(AttendArgs a, BlockWork w)
{
    pdl_wait();
    extern __shared__ int32_t s_bin[];                 // [bins + 1] counts, then first entries
    __shared__ int32_t s_part[LIST_THREADS / 32], s_items[LIST_THREADS / 32], s_before;
    const SparseArgs &s = a.s;
    const int uh = blockIdx.y, u = uh / s.H, seg = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int lo = seg * w.bins, hi = min(s.nb, lo + w.bins), n_bins = hi - lo;
    int cnt, g;
    LiveRows rows;
    const bool work = sparse_unit(s, u, threadIdx.x == 0 && seg == 0 && uh == u * s.H, cnt, g, rows) && n_bins > 0;
    if (!work) {
        if (threadIdx.x == 0) w.n_items[uh * w.segments + seg] = 0;
        return;
    }
    for (int i = threadIdx.x; i <= n_bins; i += LIST_THREADS) s_bin[i] = 0;
    __syncthreads();
    const int64_t base = (int64_t)uh * s.k_max * s.n_top;
    const int32_t *sel = a.sel + base, *idx = s.idx + (int64_t)u * s.k_max;
    const int pairs = cnt * s.n_top;
    int before = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < pairs; i += LIST_THREADS) {
        const int b = __ldg(sel + i);
        const int cell = __ldg(idx + i / s.n_top);
        if (b >= s.nb || cell < 0 || cell >= s.mn) {   // such an entry is in no list
            if (seg == 0) latch_status(s.status, RS3_EINVAL);
            continue;
        }
        if (b >= lo && b < hi) atomicAdd(&s_bin[b - lo], 1);
        before += b >= 0 && b < lo;
    }
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0) s_part[warp] = before;
    __syncthreads();
    if (threadIdx.x == 0) {
        int t = 0;
        for (int i = 0; i < LIST_THREADS / 32; ++i) t += s_part[i];
        s_before = t;
    }
    __syncthreads();
    before = s_before;
    // entries and items before each bin: a run of bins per thread
    const int per = (n_bins + LIST_THREADS - 1) / LIST_THREADS;
    const int b0 = min(n_bins, (int)threadIdx.x * per), b1 = min(n_bins, b0 + per);
    int entries = 0, items = 0;
    for (int b = b0; b < b1; ++b) {
        entries += s_bin[b];
        items += (s_bin[b] + TILE - 1) / TILE;
    }
    int e_sum = entries, i_sum = items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, e_sum, o), y = __shfl_up_sync(0xffffffffu, i_sum, o);
        if (lane >= o) { e_sum += x; i_sum += y; }
    }
    if (lane == 31) { s_part[warp] = e_sum; s_items[warp] = i_sum; }
    __syncthreads();
    int n_items = 0;
#pragma unroll
    for (int i = 0; i < LIST_THREADS / 32; ++i) {
        e_sum += i < warp ? s_part[i] : 0;
        i_sum += i < warp ? s_items[i] : 0;
        n_items += s_items[i];
    }
    // the segments before this one have at most an item per block or entry, and one more per TILE entries
    const int item0 = min(lo, before) + before / TILE;
    if (threadIdx.x == 0) {
        w.n_items[uh * w.segments + seg] = n_items;
        w.first_item[uh * w.segments + seg] = item0;
    }
    int first = before + e_sum - entries;
    BlockItem *out = w.items + uh * w.max_items + item0 + i_sum - items;
    for (int b = b0; b < b1; ++b) {
        const int n = s_bin[b];
        s_bin[b] = first;
        if (n > 0) {
            const int64_t r0 = (int64_t)(lo + b) * s.bs;
            BlockItem it;
            it.uh = uh;
            it.b = lo + b;
#pragma unroll
            for (int i = 0; i < 4; ++i) it.live[i] = i * 32 < s.bs ? 0xffffffffu : 0u;
            if (rows.count(r0, r0 + s.bs) < s.bs)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t m = 0;
                    for (int r = 0; r < 32 && i * 32 < s.bs; ++r) m |= (uint32_t)rows.holds(r0 + i * 32 + r) << r;
                    it.live[i] = m;
                }
            for (int e = 0; e < n; e += TILE) {
                it.first = first + e;
                it.n = min(TILE, n - e);
                *out++ = it;
            }
        }
        first += n;
    }
    __syncthreads();
    int2 *list = w.list + base;
#pragma unroll 4
    for (int i = threadIdx.x; i < pairs; i += LIST_THREADS) {
        const int b = __ldg(sel + i);
        const int cell = __ldg(idx + i / s.n_top);
        if (b >= lo && b < hi && cell >= 0 && cell < s.mn) list[atomicAdd(&s_bin[b - lo], 1)] = make_int2(i, cell);
    }
}

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool some)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(some ? 16 : 0) : "memory");
}

__device__ __forceinline__ void ld_matrix4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void ld_matrix2(uint32_t (&r)[2], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void ld_matrix4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// c (16 x 8, fp32) += a (16 x 16, bf16) b (16 x 8, bf16)
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D, int BS>
struct BlockTile {
    static constexpr int NW = D == 64 ? 4 : 8;         // warps
    static constexpr int ROW = 2 * D + 16;             // bytes of a K, V or Q row: 8 rows at 16-byte steps hit all banks
    static constexpr int PROW = 2 * BS + 16;
    static constexpr int KEYS = BS / NW < 8 ? 8 : BS / NW;     // keys of a warp's scores
    static constexpr int SW = BS / KEYS;               // warps with scores
    static constexpr int COLS = D / NW;                // columns of a warp's values
    static constexpr int M = 32;                       // queries of a pass
    static constexpr int K0 = 0, V0 = BS * ROW, Q0 = 2 * BS * ROW, P0 = Q0 + M * ROW, MAX0 = P0 + M * PROW, SUM0 = MAX0 + 4 * M * NW,
                         LIST0 = SUM0 + 4 * M * NW, BYTES = LIST0 + 8 * TILE;
};

// Persistent CTAs walk the items.  Per item the block's K and V rows come by cp.async (dead rows as
// zeros), and up to 64 queries pass in tiles of 32: S = Q K^T with the keys shared out to the warps, the
// rows' maxima and sums exchanged through shared memory, P as bf16, O = P V with the columns shared
// out, and (m, l, O) stored for k_join_blocks.  mma.sync: a block of a long bank has some 20 queries, so the
// call is bound by the bytes of K and V and tiles of 128 rows would be four fifths empty.
template <int D, int BS>
__global__ void __launch_bounds__(32 * BlockTile<D, BS>::NW) k_attend_blocks(AttendArgs a, BlockWork w)
{
    using X = BlockTile<D, BS>;
    constexpr int THREADS = 32 * X::NW, PIECES = D / 8;
    pdl_wait();
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int32_t s_first[MAX_SEGMENTS + 1];
    const SparseArgs &s = a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *s_max = reinterpret_cast<float *>(smem + X::MAX0), *s_sum = reinterpret_cast<float *>(smem + X::SUM0);
    int2 *s_list = reinterpret_cast<int2 *>(smem + X::LIST0);
    const uint32_t sk = smem_addr(smem + X::K0), sv = smem_addr(smem + X::V0), sq = smem_addr(smem + X::Q0), sp = smem_addr(smem + X::P0);
    const int n_seg = s.U * s.H * w.segments;
    const int64_t row_elems = (int64_t)s.H * D;
    int next = blockIdx.x;
    for (int g0 = 0; g0 < n_seg; g0 += MAX_SEGMENTS) {
        const int n = min(MAX_SEGMENTS, n_seg - g0);
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += THREADS) s_first[i + 1] = w.n_items[g0 + i];
        __syncthreads();
        if (warp == 0) {                               // items before each segment
            int run = 0;
            for (int c0 = 0; c0 < n; c0 += 32) {
                int v = c0 + lane < n ? s_first[c0 + lane + 1] : 0;
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
            int x = 0, y = n;                          // the last segment whose items begin at or before `next`
            while (y - x > 1) {
                const int mid = (x + y) >> 1;
                if (s_first[mid] <= next) x = mid; else y = mid;
            }
            const int uh0 = (g0 + x) / w.segments;
            const BlockItem *ip = w.items + uh0 * w.max_items + w.first_item[g0 + x] + (next - s_first[x]);
            const int4 head = __ldg(reinterpret_cast<const int4 *>(ip));
            const uint4 live4 = __ldg(reinterpret_cast<const uint4 *>(ip) + 1);
            const uint32_t live[4] = {live4.x, live4.y, live4.z, live4.w};
            const int u = head.x / s.H, h = head.x - u * s.H, nq = head.w;
            // the block's rows
            const int64_t off = ((int64_t)u * s.bank.rows_per_unit + (int64_t)head.y * BS) * row_elems + h * D;
            const uint16_t *K = reinterpret_cast<const uint16_t *>(a.k_store) + off;
            const uint16_t *V = reinterpret_cast<const uint16_t *>(a.v_store) + off;
            for (int v = 0; v < 2; ++v) {
                const uint16_t *src = v ? V : K;
                const uint32_t dst = v ? sv : sk;
#pragma unroll 4
                for (int i = threadIdx.x; i < BS * PIECES; i += THREADS) {
                    const int r = i / PIECES, p = i - r * PIECES;
                    const bool on = (live[BS > 32 ? r >> 5 : 0] >> (r & 31)) & 1u;
                    copy16(dst + r * X::ROW + p * 16, on ? src + r * row_elems + p * 8 : K, on);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
            const int64_t base = (int64_t)head.x * s.k_max * s.n_top;
            for (int i = threadIdx.x; i < nq; i += THREADS) s_list[i] = w.list[base + head.z + i];
            __syncthreads();
            const uint16_t *Q = static_cast<const uint16_t *>(s.q) + (int64_t)s.unit_group[u] * s.mn * row_elems + h * D;
            for (int q0 = 0; q0 < nq; q0 += X::M) {
                const int m = min(X::M, nq - q0), tiles = m > 16 ? 2 : 1;
                // query rows, rotated and rounded as the memory readout's; rows past the last are zeros
                for (int i = threadIdx.x; i < tiles * 16 * PIECES; i += THREADS) {
                    const int r = i / PIECES, p = i - r * PIECES;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (r < m) {
                        const int cell = s_list[q0 + r].y;
                        v = __ldg(reinterpret_cast<const uint4 *>(Q + cell * row_elems) + p);
                        if (s.rope) v = rotate_q_piece(v, s.rope + (int64_t)cell * D + p * 8);
                    }
                    *reinterpret_cast<uint4 *>(smem + X::Q0 + r * X::ROW + p * 16) = v;
                }
                if (q0 == 0) asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncthreads();
                float c[2][X::KEYS / 8][4];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < X::KEYS / 8; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) c[t][i][e] = 0.f;
                float top[2][2];
                if (warp < X::SW) {
#pragma unroll 4
                    for (int k = 0; k < D / 16; ++k) {
                        uint32_t qa[2][4];
                        ld_matrix4(qa[0], sq + (lane & 15) * X::ROW + k * 32 + (lane >> 4) * 16);
                        if (tiles == 2) ld_matrix4(qa[1], sq + (16 + (lane & 15)) * X::ROW + k * 32 + (lane >> 4) * 16);
                        if (X::KEYS == 8) {
                            uint32_t kb[2];
                            ld_matrix2(kb, sk + (warp * 8 + (lane & 7)) * X::ROW + k * 32 + ((lane >> 3) & 1) * 16);
                            mma_16x8x16(c[0][0], qa[0], kb[0], kb[1]);
                            if (tiles == 2) mma_16x8x16(c[1][0], qa[1], kb[0], kb[1]);
                        } else {
#pragma unroll
                            for (int i = 0; i < X::KEYS / 16; ++i) {
                                uint32_t kb[4];
                                ld_matrix4(kb, sk + (warp * X::KEYS + i * 16 + (lane & 7) + ((lane >> 4) << 3)) * X::ROW + k * 32 +
                                                   ((lane >> 3) & 1) * 16);
#pragma unroll
                                for (int t = 0; t < 2; ++t) {
                                    if (t == 1 && tiles == 1) break;
                                    mma_16x8x16(c[t][(2 * i) % (X::KEYS / 8)], qa[t], kb[0], kb[1]);
                                    mma_16x8x16(c[t][(2 * i + 1) % (X::KEYS / 8)], qa[t], kb[2], kb[3]);
                                }
                            }
                        }
                    }
                    // this lane holds columns 2 (lane % 4), + 1 of rows lane / 4 and + 8
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            float mx = -INFINITY;
#pragma unroll
                            for (int i = 0; i < X::KEYS / 8; ++i)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int key = warp * X::KEYS + i * 8 + (lane & 3) * 2 + e;
                                    const bool on = (live[BS > 32 ? key >> 5 : 0] >> (key & 31)) & 1u;
                                    float &v = c[t][i][2 * r + e];
                                    v = on ? v * a.scale_log2 : -INFINITY;
                                    mx = fmaxf(mx, v);
                                }
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                            if ((lane & 3) == 0) s_max[warp * X::M + t * 16 + r * 8 + (lane >> 2)] = mx;
                        }
                }
                __syncthreads();
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float mx = -INFINITY;
#pragma unroll
                        for (int i = 0; i < X::SW; ++i) mx = fmaxf(mx, s_max[i * X::M + t * 16 + r * 8 + (lane >> 2)]);
                        top[t][r] = mx;
                    }
                if (warp < X::SW) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (t == 1 && tiles == 1) break;
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float ref = top[t][r] == -INFINITY ? 0.f : top[t][r];
                            const int row = t * 16 + r * 8 + (lane >> 2);
                            float sum = 0.f;
#pragma unroll
                            for (int i = 0; i < X::KEYS / 8; ++i) {
                                const float p0 = exp2f(c[t][i][2 * r] - ref), p1 = exp2f(c[t][i][2 * r + 1] - ref);
                                sum += p0 + p1;
                                *reinterpret_cast<uint32_t *>(smem + X::P0 + row * X::PROW + (warp * X::KEYS + i * 8 + (lane & 3) * 2) * 2) =
                                    pack_bf16x2(p0, p1);
                            }
                            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                            if ((lane & 3) == 0) s_sum[warp * X::M + row] = sum;
                        }
                    }
                }
                if (q0 == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
                __syncthreads();
                float o[2][X::COLS / 8][4];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < X::COLS / 8; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
#pragma unroll
                for (int k = 0; k < BS / 16; ++k) {
                    uint32_t pa[2][4];
                    ld_matrix4(pa[0], sp + (lane & 15) * X::PROW + k * 32 + (lane >> 4) * 16);
                    if (tiles == 2) ld_matrix4(pa[1], sp + (16 + (lane & 15)) * X::PROW + k * 32 + (lane >> 4) * 16);
#pragma unroll
                    for (int i = 0; i < X::COLS / 16; ++i) {
                        uint32_t vb[4];
                        ld_matrix4_t(vb, sv + (k * 16 + (lane & 15)) * X::ROW + (warp * X::COLS + i * 16 + (lane >> 4) * 8) * 2);
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if (t == 1 && tiles == 1) break;
                            mma_16x8x16(o[t][2 * i], pa[t], vb[0], vb[1]);
                            mma_16x8x16(o[t][2 * i + 1], pa[t], vb[2], vb[3]);
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int row = t * 16 + r * 8 + (lane >> 2);
                        if (row >= m) continue;
                        const int64_t slot = base + s_list[q0 + row].x;
                        if (warp == 0 && (lane & 3) == 0) {
                            float l = 0.f;
#pragma unroll
                            for (int i = 0; i < X::SW; ++i) l += s_sum[i * X::M + row];
                            w.ml[slot] = make_float2(top[t][r], l);
                        }
                        float *dst = w.o + slot * D + warp * X::COLS + (lane & 3) * 2;
#pragma unroll
                        for (int i = 0; i < X::COLS / 8; ++i)
                            *reinterpret_cast<float2 *>(dst + i * 8) = make_float2(o[t][i][2 * r], o[t][i][2 * r + 1]);
                    }
                __syncthreads();                       // P, Q and the sums are free; after the last pass K, V and the list too
            }
        }
        next -= total;
    }
}

// Lanes of D / 4 (at most 32) take a (unit, head, query): out = residual + sum_t 2^(m_t - M) O_t / sum_t 2^(m_t - M) l_t
template <int D>
__global__ void __launch_bounds__(256) k_join_blocks(AttendArgs a, BlockWork w)
{
    constexpr int L = D / 4 < 32 ? D / 4 : 32, ITEMS = D / 4 / L;
    pdl_wait();
    const SparseArgs &s = a.s;
    const int u = blockIdx.y, sub = threadIdx.x % L;
    const int64_t jh = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int j = (int)(jh / s.H), h = (int)(jh - (int64_t)j * s.H);
    const int cnt = s.count[u], g = s.unit_group[u];
    if (cnt < 0 || cnt > s.k_max || g < 0 || g >= s.G || j >= cnt) return;
    const int cell = s.idx[(int64_t)u * s.k_max + j];
    if (cell < 0 || cell >= s.mn) return;
    const int64_t base = (((int64_t)u * s.H + h) * s.k_max + j) * s.n_top;
    float top = -INFINITY;
    for (int t = sub; t < s.n_top; t += L) {
        const int b = a.sel[base + t];
        if (b >= 0 && b < s.nb) top = fmaxf(top, w.ml[base + t].x);
    }
    const uint32_t group = L == 32 ? 0xffffffffu : ((1u << L) - 1u) << ((threadIdx.x & 31) / L * L);
#pragma unroll
    for (int o = L >> 1; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(group, top, o));
    float4 y[ITEMS];
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (top > -INFINITY) {
#pragma unroll 4
        for (int t = 0; t < s.n_top; ++t) {
            const int b = __ldg(a.sel + base + t);
            if (b < 0 || b >= s.nb) continue;
            const float2 ml = w.ml[base + t];
            const float f = exp2f(ml.x - top);
            l = fmaf(f, ml.y, l);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const float4 v = __ldcs(reinterpret_cast<const float4 *>(w.o + (base + t) * D) + sub + L * i);
                y[i].x = fmaf(f, v.x, y[i].x);
                y[i].y = fmaf(f, v.y, y[i].y);
                y[i].z = fmaf(f, v.z, y[i].z);
                y[i].w = fmaf(f, v.w, y[i].w);
            }
        }
        const float inv = 1.f / l;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) y[i] = make_float4(y[i].x * inv, y[i].y * inv, y[i].z * inv, y[i].w * inv);
    }
    const int64_t at = ((int64_t)u * s.mn + cell) * ((int64_t)s.H * D) + h * D;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t x = at + (sub + L * i) * 4;
        if (a.residual) {
            const float4 r = load4(static_cast<const uint16_t *>(a.residual) + x);
            y[i] = make_float4(y[i].x + r.x, y[i].y + r.y, y[i].z + r.z, y[i].w + r.w);
        }
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + x) = make_uint2(pack_bf16x2(y[i].x, y[i].y), pack_bf16x2(y[i].z, y[i].w));
    }
}

// Where the parts of a by-block call lie in its workspace.
struct WorkLayout {
    int64_t segments, bins, max_items;
    size_t n_items, first_item, items, list, ml, o, total;
};

WorkLayout work_layout(int64_t U, int64_t H, int64_t d, int64_t k_max, int64_t n_top, int64_t nb)
{
    WorkLayout l = {};
    const int64_t uh = U * H, pairs = k_max * n_top;
    const int64_t least = nb > LIST_BINS ? (nb + LIST_BINS - 1) / LIST_BINS : 1;
    // lists are made by about two CTAs per SM, of no fewer than 64 blocks each
    l.segments = least;
    while (uh * l.segments < 256 && nb / (2 * l.segments) >= 64) l.segments *= 2;
    l.bins = (nb + l.segments - 1) / l.segments;
    l.max_items = (nb < pairs ? nb : pairs) + pairs / TILE + 1;
    size_t at = 0;
    const auto part = [&](size_t bytes) {
        const size_t x = at;
        at = align_up(at + bytes, 256);
        return x;
    };
    l.n_items = part((size_t)(uh * least + 512) * 4);      // at least uh * segments, and never falling
    l.first_item = part((size_t)(uh * least + 512) * 4);
    l.items = part((size_t)(uh * l.max_items) * sizeof(BlockItem));
    l.list = part((size_t)(uh * pairs) * 8);
    l.ml = part((size_t)(uh * pairs) * 8);
    l.o = part((size_t)(uh * pairs) * (size_t)d * 4);
    l.total = at;
    return l;
}

// Whether a call's path may be by block, for which its workspace is sized.
bool sized_by_blocks(rs3_dtype dtype, int64_t U, int64_t H, int64_t d, int64_t k_max, int64_t n_top)
{
    return dtype == RS3_BF16 && d >= 64 && U * H * k_max * n_top >= 4096;
}

bool by_blocks(rs3_dtype dtype, int64_t U, int64_t H, int64_t d, int64_t k_max, int64_t n_top)
{
    return sized_by_blocks(dtype, U, H, d, k_max, n_top) && k_max * n_top < (1ll << 30) && U * H < 65536;
}

template <int D, int BS>
rs3_status launch_attend(const AttendArgs &a, const BlockWork &w, cudaStream_t st)
{
    using X = BlockTile<D, BS>;
    const rs3_status r = rs3_kernel_smem((const void *)k_attend_blocks<D, BS>, X::BYTES);
    if (r != RS3_OK) return r;
    const int per_sm = 225 * 1024 / (X::BYTES + 6 * 1024);
    launch_pdl(k_attend_blocks<D, BS>, dim3((unsigned)(rs3_sm_count() * (per_sm > 8 ? 8 : per_sm))), dim3(32 * X::NW), X::BYTES, st, a, w);
    return RS3_OK;
}

rs3_status launch_by_blocks(const AttendArgs &a, void *workspace, cudaStream_t st)
{
    const SparseArgs &s = a.s;
    const WorkLayout l = work_layout(s.U, s.H, s.d, s.k_max, s.n_top, s.nb);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    BlockWork w = {};
    w.n_items = reinterpret_cast<int32_t *>(ws + l.n_items);
    w.first_item = reinterpret_cast<int32_t *>(ws + l.first_item);
    w.items = reinterpret_cast<BlockItem *>(ws + l.items);
    w.list = reinterpret_cast<int2 *>(ws + l.list);
    w.ml = reinterpret_cast<float2 *>(ws + l.ml);
    w.o = reinterpret_cast<float *>(ws + l.o);
    w.segments = (int32_t)l.segments;
    w.bins = (int32_t)l.bins;
    w.max_items = l.max_items;
    launch_pdl(k_block_lists, dim3((unsigned)l.segments, (unsigned)(s.U * s.H)), dim3(LIST_THREADS), (size_t)(l.bins + 1) * 4, st, a, w);
    rs3_status r = RS3_EINTERNAL;
    if (s.d == 64) r = s.bs == 32 ? launch_attend<64, 32>(a, w, st) : s.bs == 64 ? launch_attend<64, 64>(a, w, st) : launch_attend<64, 128>(a, w, st);
    if (s.d == 128) r = s.bs == 32 ? launch_attend<128, 32>(a, w, st) : s.bs == 64 ? launch_attend<128, 64>(a, w, st) : launch_attend<128, 128>(a, w, st);
    if (s.d == 256) r = s.bs == 32 ? launch_attend<256, 32>(a, w, st) : s.bs == 64 ? launch_attend<256, 64>(a, w, st) : launch_attend<256, 128>(a, w, st);
    if (r != RS3_OK) return r;
    void (*join)(AttendArgs, BlockWork) = s.d == 64 ? k_join_blocks<64> : s.d == 128 ? k_join_blocks<128> : k_join_blocks<256>;
    const int per = 256 / (s.d / 4 < 32 ? s.d / 4 : 32);
    launch_pdl(join, dim3((unsigned)(((int64_t)s.k_max * s.H + per - 1) / per), (unsigned)s.U), dim3(256), 0, st, a, w);
    return RS3_OK;
}

}  // namespace

extern "C" size_t rs3_sparse_readout_workspace_bytes(int U, int H, int d, int k_max, int n_top, int n_blocks, rs3_dtype dtype)
{
    if (U < 1 || H < 1 || d < 1 || k_max < 0 || n_top < 1 || n_blocks < 0) return 0;
    if (dtype != RS3_F32 && dtype != RS3_BF16) return 0;
    return 16 + (sized_by_blocks(dtype, U, H, d, k_max, n_top) ? work_layout(U, H, d, k_max, n_top, n_blocks).total : 0);
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
    if (workspace_bytes < rs3_sparse_readout_workspace_bytes(a.s.U, H, d, k_max, n_top, a.s.nb, dtype)) return RS3_ECAPACITY;
    const bool blocks = a.s.nb > 0 && by_blocks(dtype, a.s.U, H, d, k_max, n_top);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    a.k_store = static_cast<const uint8_t *>(bank->k_store);
    a.v_store = static_cast<const uint8_t *>(bank->v_store);
    a.sel = sel;
    a.residual = residual;
    a.out = out;
    a.scale_log2 = (scale == 0.f ? 1.f / std::sqrt((float)d) : scale) * 1.4426950408889634f;
    if (out != residual) {
        const int64_t nvec = (int64_t)a.s.U * mn * H * d * (int64_t)elem_bytes(dtype) / 16;
        const int64_t ctas = (nvec + 1023) / 1024, most = 8ll * rs3_sm_count();
        launch_pdl(k_pass_through, dim3((unsigned)(ctas < most ? ctas : most)), dim3(256), 0, st,
                   static_cast<const uint4 *>(residual), static_cast<uint4 *>(out), nvec);
    }
    if (blocks) {
        const rs3_status e = launch_by_blocks(a, workspace, st);
        if (e != RS3_OK) return e;
    } else if (k_max > 0) {
        const int pieces = d * (int)elem_bytes(dtype) / 16;
        const dim3 grid((unsigned)k_max, (unsigned)H, (unsigned)a.s.U);
        void (*kern)(AttendArgs, int) = dtype == RS3_BF16 ? k_attend_gather<uint16_t, 1>
                                        : pieces > 32     ? k_attend_gather<float, 2> : k_attend_gather<float, 1>;
        launch_pdl(kern, grid, dim3(32 * GATHER_WARPS), 0, st, a, pieces > 32 ? 32 : pieces);
    }
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
