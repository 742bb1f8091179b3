// rs3_shared_readout.cu -- readout of units that share the rows of a bank (hypotheses of a track
// and what they were forked from):
//
//   A = softmax(q~ [K_prefix; K_own]^T scale) [V_prefix; V_own]
//
// The softmax over both parts is the merge of the two parts' own: with (m, l, O) = (max, sum of
// 2^(s - m), sum of 2^(s - m) v) of each, M = max m, A = sum 2^(m - M) O / sum 2^(m - M) l.  A
// query's part over the prefix depends on its grid and cell alone, not on the unit, so the units
// of one group and prefix form a class whose queries are the union of their kept cells, each
// attended to once.  Launches:
//   k_classes     a CTA per unit: the class's first unit takes the union of the kept cells as
//                 a bit per cell, with the counts before each word (a cell's place among them)
//   k_plan_two    the readout's stream-K plans of the classes over the prefix bank and of the
//                 units over their own, every result in partial slots
//   k_readout_*   the readout's kernels over either plan, on the bank each reads
//   k_merge_prefix  between the two, the classes' pieces: one for each row and head
//   k_merge_two   log-sum-exp merge of a row's pieces over both banks, and the scatter
// Eight hypotheses of some 750 queries behind 300 000 rows of 256, six frames of their own: 255 us, of
// which the attention over the prefix 187 (what it would take for each hypothesis), over the own rows 33.
#include "rs3_readout_common.cuh"

#include <algorithm>

namespace {

struct ShareArgs {
    const int32_t *unit_group, *idx, *count, *prefix_unit;
    int32_t *status;
    int32_t *own_count;                    // [U] kept queries; 0 for a unit that is skipped
    int32_t *leader;                       // [U] first unit of its class, -1 without a prefix
    int32_t *class_group, *class_bank, *class_count;   // [U] at the class's first unit; counts 0 elsewhere
    int32_t *class_idx;                    // [U][class_stride]
    uint32_t *bits;                        // [U][words] kept cells of the class
    int32_t *before;                       // [U][words] kept cells before each word
    int U, G, mn, k_max, words, class_stride, prefix_U;
};

constexpr int SHARE_THREADS = 512;
constexpr int SHARE_WORDS = RS3_MAX_MN / 32;

// The unit's prefix, -1 for none, -2 when its arguments are not sound.
__device__ __forceinline__ int prefix_of(const ShareArgs &a, int u, int &g, int &n)
{
    const int p = a.prefix_unit[u];
    n = a.count[u];
    g = a.unit_group[u];
    return g < 0 || g >= a.G || n < 0 || n > a.k_max || p < -1 || p >= a.prefix_U ? -2 : p;
}

__global__ void __launch_bounds__(SHARE_THREADS) k_classes(const __grid_constant__ ShareArgs a)
{
    pdl_wait();
    __shared__ uint32_t s_bits[SHARE_WORDS];
    __shared__ int s_unit[SHARE_THREADS], s_kept[SHARE_THREADS], s_n, s_first, s_sum[SHARE_THREADS / 32];
    const int u = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    int g, gv, n, nv;
    const int p = prefix_of(a, u, g, n);
    if (t == 0) s_first = u;
    for (int w = t; w < a.words; w += SHARE_THREADS) s_bits[w] = 0u;
    // the class's units, some at a time, and their kept cells; a unit with one before it leaves that to it
    for (int v0 = 0; p >= 0 && v0 < a.U; v0 += SHARE_THREADS) {
        if (t == 0) s_n = 0;
        __syncthreads();
        const int v = v0 + t;
        if (v < a.U && prefix_of(a, v, gv, nv) == p && gv == g) {
            if (v < u) atomicMin(&s_first, v);
            const int at = atomicAdd(&s_n, 1);
            s_unit[at] = v;
            s_kept[at] = nv;
        }
        __syncthreads();
        if (s_first < u) break;
        const int64_t all = (int64_t)s_n * a.k_max;
        for (int64_t i = t; i < all; i += 4 * SHARE_THREADS) {
            int cell[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int64_t at = i + x * SHARE_THREADS;
                const int m = at < all ? (int)(at / a.k_max) : 0, j = (int)(at - (int64_t)m * a.k_max);
                cell[x] = at < all && j < s_kept[m] ? __ldg(a.idx + (int64_t)s_unit[m] * a.k_max + j) : INT32_MIN;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (cell[x] >= 0 && cell[x] < a.mn) atomicOr(&s_bits[cell[x] >> 5], 1u << (cell[x] & 31));
                else if (cell[x] != INT32_MIN) latch_status(a.status, RS3_EINVAL);
            }
        }
        __syncthreads();                                   // the list is read, the bits are set
    }
    const bool leads = p >= 0 && s_first == u;
    if (t == 0) {
        if (p == -2) latch_status(a.status, RS3_EINVAL);
        a.own_count[u] = p == -2 ? 0 : n;
        a.leader[u] = p >= 0 ? s_first : -1;
        a.class_group[u] = leads ? g : 0;
        a.class_bank[u] = leads ? p : -1;
        if (!leads) a.class_count[u] = 0;
    }
    if (!leads) return;
    // their places: a thread takes a word (512 at most)
    uint32_t b = t < a.words ? s_bits[t] : 0u;
    const int mine = __popc(b);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
    int at = upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < SHARE_THREADS / 32; ++w) {
        if (w < warp) at += s_sum[w];
        total += s_sum[w];
    }
    if (t == 0) a.class_count[u] = total;
    int32_t *out = a.class_idx + (int64_t)u * a.class_stride;
    if (t >= a.words) return;
    a.bits[(int64_t)u * a.words + t] = b;
    a.before[(int64_t)u * a.words + t] = at;
    for (; b; b &= b - 1u) out[at++] = t * 32 + __ffs(b) - 1;
}
static_assert(SHARE_THREADS >= SHARE_WORDS, "a word each");

// A row's pieces over one bank.
struct Pieces {
    const float2 *ml;
    const float *o;
    int64_t step;                          // rows of a slot
    int n, slot0, slice;
    __device__ __forceinline__ int64_t slot(int s) const { return s == 0 ? slot0 : 2 * (int64_t)(slice + s); }
};

__device__ __forceinline__ GroupParts load_parts(const GroupParts *g)
{
    const int4 *p = reinterpret_cast<const int4 *>(g);
    const int4 a = __ldg(p), b = __ldg(p + 1);
    return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

constexpr int PREFIX_PIECES = 4;           // more pieces of a class's row than these are merged ahead

// Of row r of a group; `merged`: many pieces have become one, in the first's slot.
__device__ __forceinline__ Pieces pieces_of(const ReadoutMore &a, const GroupParts &g, int r, int BM, bool merged)
{
    Pieces p;
    p.ml = reinterpret_cast<const float2 *>(a.part_ml) + r;
    p.o = a.part_o + (int64_t)r * a.d;
    p.step = BM;
    p.n = merged && g.n > PREFIX_PIECES ? 1 : g.n;
    p.slot0 = g.slot0;
    p.slice = g.slice;
    return p;
}

// Merges a row's pieces of two lists (the second may be empty).  L lanes take four columns each
// (twice, for heads of 256); with SPLIT a whole warp takes one row, each L lanes every (32 / L)-th
// piece, else each L lanes a row of their own (n 0: none).  The pieces' (m, l) are shared out among the
// row's lanes, and their weights come from the lane that holds their m.  Returns with the columns' sums,
// not divided by l.  Every lane of the warp calls it.
template <int L, int CB, bool SPLIT>
__device__ __forceinline__ void merge_row(const Pieces &p, const Pieces &q, int d, float4 (&acc)[CB], float &M, float &l)
{
    constexpr int W = SPLIT ? 32 : L;                      // lanes of a row
    constexpr int S = W / L, F = 4;                        // sub-groups of a row's lanes; pieces of each in flight
    const int lane = threadIdx.x % W, sub = lane / L, col = 4 * (lane % L), n = p.n + q.n;
    const int most = SPLIT ? n : __reduce_max_sync(0xffffffffu, n);
    const auto ml = [&](int i) { return i < p.n ? __ldcg(p.ml + p.slot(i) * p.step) : __ldcg(q.ml + q.slot(i - p.n) * q.step); };
    float4 o[F][CB];
    const auto load = [&](int i0) {                        // pieces i0 + sub, i0 + S + sub, ... of the row
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int i = i0 + S * f + sub;
            const bool in = i < n, first = i < p.n;
            const int64_t row = first ? p.slot(i) * p.step : q.slot(i - p.n) * q.step;
            const float *src = (first ? p.o : q.o) + (in ? row * d : 0) + col;
#pragma unroll
            for (int c = 0; c < CB; ++c)
                o[f][c] = in ? __ldcg(reinterpret_cast<const float4 *>(src + 128 * c)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    float2 mine = lane < n ? ml(lane) : make_float2(-INFINITY, 0.f);
    load(0);                                               // (under way while the weights are found)
    M = mine.x;
    for (int i = lane + W; i < n; i += W) M = fmaxf(M, ml(i).x);
#pragma unroll
    for (int x = W / 2; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, x));
    const float ref = M == -INFINITY ? 0.f : M;
    l = 0.f;
#pragma unroll
    for (int c = 0; c < CB; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    static_assert(W % (S * F) == 0, "whole batches");
    for (int i0 = 0; i0 < most; i0 += W) {
        if (i0 > 0) mine = i0 + lane < n ? ml(i0 + lane) : make_float2(-INFINITY, 0.f);
        const float w = exp2f(mine.x - ref);
        l = fmaf(w, mine.y, l);
        for (int k0 = 0; k0 < W && i0 + k0 < most; k0 += S * F) {      // (uniform: the shuffles name all lanes)
            if (i0 + k0 > 0) load(i0 + k0);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int k = k0 + S * f + sub;
                float wt = __shfl_sync(0xffffffffu, w, k, W);
                if (i0 + k >= n) wt = 0.f;
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    acc[c].x = fmaf(wt, o[f][c].x, acc[c].x);
                    acc[c].y = fmaf(wt, o[f][c].y, acc[c].y);
                    acc[c].z = fmaf(wt, o[f][c].z, acc[c].z);
                    acc[c].w = fmaf(wt, o[f][c].w, acc[c].w);
                }
            }
        }
    }
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if constexpr (S > 1) {
#pragma unroll
        for (int o = 16; o >= L; o >>= 1)
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                acc[c].x += __shfl_xor_sync(0xffffffffu, acc[c].x, o);
                acc[c].y += __shfl_xor_sync(0xffffffffu, acc[c].y, o);
                acc[c].z += __shfl_xor_sync(0xffffffffu, acc[c].z, o);
                acc[c].w += __shfl_xor_sync(0xffffffffu, acc[c].w, o);
            }
    }
}

constexpr int MERGE_THREADS = 256;

// The pieces of the classes' rows become one each, in the first's slot, where there are many: a long
// prefix is read in a score of pieces, by every unit of the class (eight hypotheses of 750 queries
// behind 300 000 keys: 19 pieces, the merges 40 us without this, 26 with it).  A warp takes a row of a head.
template <int L, int CB>
__global__ void __launch_bounds__(MERGE_THREADS) k_merge_prefix(const __grid_constant__ ReadoutMore pre)
{
    pdl_wait();
    const int lane = threadIdx.x & 31, BM = pre.header->bm;
    const int64_t rows = (int64_t)pre.header->n_groups * BM;
    for (int64_t i = (int64_t)blockIdx.x * (MERGE_THREADS / 32) + (threadIdx.x >> 5); i < rows; i += (int64_t)gridDim.x * (MERGE_THREADS / 32)) {
        const GroupParts g = load_parts(pre.parts + i / BM);
        const int r = (int)(i % BM);
        if (g.n <= PREFIX_PIECES || g.qt * BM + r >= g.cnt) continue;
        const Pieces p = pieces_of(pre, g, r, BM, false);
        Pieces none = p;
        none.n = 0;
        float4 acc[CB];
        float M, l;
        merge_row<L, CB, true>(p, none, pre.d, acc, M, l);
        __syncwarp();                                      // the pieces are read before the first's place is written
        const int64_t row = p.slot0 * p.step;
        if (lane < L)
#pragma unroll
            for (int k = 0; k < CB; ++k)
                __stcg(reinterpret_cast<float4 *>(const_cast<float *>(p.o) + row * pre.d + 4 * lane + 128 * k), acc[k]);
        if (lane == 0) __stcg(const_cast<float2 *>(p.ml) + row, make_float2(M, l));
    }
}

// A row's pieces over its unit's bank and its one over the prefix, and the scatter.
template <typename T, int L, int CB>
__global__ void __launch_bounds__(MERGE_THREADS) k_merge_two(const __grid_constant__ ReadoutMore own, const __grid_constant__ ReadoutMore pre,
                                                             const __grid_constant__ ShareArgs s)
{
    pdl_wait();
    const int lane = threadIdx.x % L, BM = own.header->bm, BMP = pre.header->bm;
    const int64_t rows = (int64_t)own.header->n_groups * BM;
    constexpr int PER = MERGE_THREADS / L;                 // rows of a CTA
    for (int64_t i0 = (int64_t)blockIdx.x * PER; i0 < rows; i0 += (int64_t)gridDim.x * PER) {
        const int64_t i = i0 + threadIdx.x / L;            // (BM is a multiple of the rows of a warp: all of one group)
        const GroupParts g = load_parts(own.parts + min(i, rows - 1) / BM);
        const int r = (int)(i % BM), j = g.qt * BM + r;
        bool here = i < rows && j < g.cnt;
        Pieces p = pieces_of(own, g, r, BM, false), q = p;
        q.n = 0;
        int cell = 0;
        if (here) {
            cell = __ldg(s.idx + (int64_t)g.u * own.k_max + j);
            if (cell < 0 || cell >= own.mn) {
                if (lane == 0) latch_status(own.status, RS3_EINVAL);
                here = false;
            }
        }
        const int c = s.leader[g.u];
        if (here && c >= 0) {
            const int64_t w = (int64_t)c * s.words + (cell >> 5);
            const int place = s.before[w] + __popc(s.bits[w] & ((1u << (cell & 31)) - 1u));
            const RangeSet *rs = pre.ranges + c;
            here = place < rs->cnt;                        // (else its prefix is unsound)
            if (here) q = pieces_of(pre, load_parts(pre.parts + rs->first_group + place / BMP * pre.H + g.h), place % BMP, BMP, true);
        }
        if (!here) p.n = q.n = 0;
        float4 acc[CB];
        float M, l;
        merge_row<L, CB, false>(p, q, own.d, acc, M, l);
        const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l;
        if (here)
#pragma unroll
            for (int k = 0; k < CB; ++k) {
                const float o4[4] = {acc[k].x * inv, acc[k].y * inv, acc[k].z * inv, acc[k].w * inv};
                store_out4<T>(own, g.u, cell, g.h * own.d + 4 * lane + 128 * k, o4);
            }
    }
}

template <int L, int CB>
void launch_merges(const ReadoutMore &own, const ReadoutMore &pre, const ShareArgs &s, rs3_dtype dtype, cudaStream_t st, bool prefix)
{
    const int64_t rows = (int64_t)own.U * (own.k_max > 0 ? own.k_max : 1) * own.H, per = MERGE_THREADS / (prefix ? 32 : L);
    const unsigned ctas = (unsigned)std::min<int64_t>((rows + per - 1) / per, 8ll * rs3_sm_count());
    if (prefix) launch_pdl(k_merge_prefix<L, CB>, dim3(ctas), dim3(MERGE_THREADS), 0, st, pre);
    else if (dtype == RS3_BF16) launch_pdl(k_merge_two<uint16_t, L, CB>, dim3(ctas), dim3(MERGE_THREADS), 0, st, own, pre, s);
    else launch_pdl(k_merge_two<float, L, CB>, dim3(ctas), dim3(MERGE_THREADS), 0, st, own, pre, s);
}

rs3_status launch_merge(const ReadoutMore &own, const ReadoutMore &pre, const ShareArgs &s, rs3_dtype dtype, cudaStream_t st, bool prefix)
{
    switch (own.d) {
    case 16: launch_merges<4, 1>(own, pre, s, dtype, st, prefix); break;
    case 32: launch_merges<8, 1>(own, pre, s, dtype, st, prefix); break;
    case 64: launch_merges<16, 1>(own, pre, s, dtype, st, prefix); break;
    case 128: launch_merges<32, 1>(own, pre, s, dtype, st, prefix); break;
    default: launch_merges<32, 2>(own, pre, s, dtype, st, prefix); break;
    }
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}

// Byte offsets in the workspace.
struct ShareLayout {
    ReadoutPath own, pre;
    ReadoutLayout own_l, pre_l;
    size_t words, idx, own_ws, pre_ws, total;
    int n_words, class_stride;
};

// Queries of a class: no more than cells, nor than its units keep.
int class_stride(int U, int mn, int k_max) { return (int)std::min<int64_t>(mn, (int64_t)U * k_max); }

// `few`: of the paths with fewer query rows to a CTA, where there are such (1: yes, 0: no, -1: as the calls have them)
ShareLayout share_layout(const rs3_bank *bank, const rs3_bank *prefix, int k_max, int few)
{
    const rs3_dtype dtype = (rs3_dtype)bank->dtype;
    const int U = bank->U, H = bank->H, d = bank->d;
    ShareLayout L;
    L.own = choose_readout_path(dtype, d, U, H, k_max, bank->rows_per_unit, SIZE_MAX);
    L.pre = choose_readout_path(dtype, d, U, H, k_max, prefix->rows_per_unit, SIZE_MAX);
    if (L.own.kind == 0) {
        if (few < 0 ? rs3_has_few_rows(L.own, U, H, d, k_max, bank->rows_per_unit) : few) L.own = rs3_few_rows(L.own, d);
        if (few < 0 ? rs3_has_few_rows(L.pre, U, H, d, k_max, prefix->rows_per_unit) : few) L.pre = rs3_few_rows(L.pre, d);
    }
    // the classes' tiles together are no more than their units' (a sum's ceiling is no more than the sum of ceilings)
    L.own_l = rs3_readout_layout(U, H, d, k_max, L.own, true);
    L.pre_l = rs3_readout_layout(U, H, d, k_max, L.pre, true);
    L.n_words = (bank->mn + 31) / 32;
    L.class_stride = class_stride(U, bank->mn, k_max);
    size_t off = align_up((size_t)U * 5 * 4, 256);
    L.words = off;
    off = align_up(off + (size_t)U * L.n_words * 8, 256);
    L.idx = off;
    off = align_up(off + (size_t)U * L.class_stride * 4, 256);
    L.own_ws = off;
    off = align_up(off + L.own_l.total, 256);
    L.pre_ws = off;
    L.total = off + L.pre_l.total;
    return L;
}

bool bank_known(const rs3_bank *b) { return b && b->magic == RS3_BANK_MAGIC; }

}  // namespace

extern "C" size_t rs3_shared_readout_workspace_bytes(const rs3_bank *bank, const rs3_bank *prefix, int k_max)
{
    if (!bank_known(bank) || !bank_known(prefix) || k_max < 0) return 0;
    // (each part's is the larger of both paths': a call of fewer queries may take the other one)
    const ShareLayout a = share_layout(bank, prefix, k_max, rs3_always_few_rows(bank->d)), b = share_layout(bank, prefix, k_max, 1);
    return a.own_ws + align_up(std::max(a.own_l.total, b.own_l.total), 256) + std::max(a.pre_l.total, b.pre_l.total);
}

extern "C" rs3_status rs3_shared_readout(const void *q, rs3_dtype dtype, int G, int mn, int H, int d, const int32_t *unit_group,
                                         const int32_t *idx, const int32_t *count, int k_max, const rs3_bank *bank,
                                         const rs3_bank *prefix, const int32_t *prefix_unit, const float *rope,
                                         const void *residual, void *out, float scale, void *workspace, size_t workspace_bytes,
                                         int32_t *status, rs3_stream_t stream)
{
    rs3_status s = rs3_readout_check(q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, residual, out, workspace, status);
    if (s != RS3_OK) return s;
    if (!bank_known(prefix) || !prefix->meta || !prefix->k_store || !prefix->v_store || !prefix_unit) return RS3_EINVAL;
    if (prefix->dtype != bank->dtype || prefix->H != H || prefix->d != d || bank->mn != mn || prefix->mn != mn || k_max > mn) return RS3_EINVAL;
    if (prefix->U > RS3_MAX_UNITS) return RS3_EUNSUPPORTED;
    const ShareLayout L = share_layout(bank, prefix, k_max, -1);
    if (!rs3_readout_fits(bank->U, H, k_max, L.own) || !rs3_readout_fits(bank->U, H, k_max, L.pre)) return RS3_EUNSUPPORTED;
    if (workspace_bytes < rs3_shared_readout_workspace_bytes(bank, prefix, k_max)) return RS3_ECAPACITY;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int U = bank->U;
    int32_t *w = reinterpret_cast<int32_t *>(ws);
    ShareArgs sh = {};
    sh.unit_group = unit_group;
    sh.idx = idx;
    sh.count = count;
    sh.prefix_unit = prefix_unit;
    sh.status = status;
    sh.own_count = w;
    sh.leader = w + U;
    sh.class_group = w + 2 * U;
    sh.class_bank = w + 3 * U;
    sh.class_count = w + 4 * U;
    sh.bits = reinterpret_cast<uint32_t *>(ws + L.words);
    sh.before = reinterpret_cast<int32_t *>(ws + L.words) + (size_t)U * L.n_words;
    sh.class_idx = reinterpret_cast<int32_t *>(ws + L.idx);
    sh.U = U;
    sh.G = G;
    sh.mn = mn;
    sh.k_max = k_max;
    sh.words = L.n_words;
    sh.class_stride = L.class_stride;
    sh.prefix_U = prefix->U;
    ReadoutMore own = {}, pre = {};
    rs3_readout_fill(&own, L.own, L.own_l, ws + L.own_ws, q, G, mn, H, d, unit_group, idx, sh.own_count, k_max, U, bank, rope, residual,
                     out, scale, status);
    own.parts = reinterpret_cast<GroupParts *>(ws + L.own_ws + L.own_l.parts);
    rs3_readout_fill(&pre, L.pre, L.pre_l, ws + L.pre_ws, q, G, mn, H, d, sh.class_group, sh.class_idx, sh.class_count, L.class_stride, U,
                     prefix, rope, nullptr, nullptr, scale, status);
    pre.parts = reinterpret_cast<GroupParts *>(ws + L.pre_ws + L.pre_l.parts);
    pre.bank_unit = sh.class_bank;
    launch_pdl(k_classes, dim3((unsigned)U), dim3(SHARE_THREADS), 0, st, sh);
    if (cudaGetLastError() != cudaSuccess) return RS3_ECUDA;
    if ((s = rs3_readout_plan_two(pre, own, dtype, st)) != RS3_OK) return s;
    if ((s = rs3_readout_run_launch(pre, L.pre, dtype, st)) != RS3_OK) return s;
    if ((s = launch_merge(own, pre, sh, dtype, st, true)) != RS3_OK) return s;
    if ((s = rs3_readout_run_launch(own, L.own, dtype, st)) != RS3_OK) return s;
    return launch_merge(own, pre, sh, dtype, st, false);
}
