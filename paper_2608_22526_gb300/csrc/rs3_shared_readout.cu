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
//   k_merge_two   log-sum-exp merge of a row's pieces over both banks, and the scatter
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

constexpr int SHARE_THREADS = 256;
constexpr int SHARE_WORDS = RS3_MAX_MN / 32;

// The unit's prefix, -1 for none, -2 when its arguments are not sound.
__device__ __forceinline__ int prefix_of(const ShareArgs &a, int u, int &g)
{
    const int p = a.prefix_unit[u], n = a.count[u];
    g = a.unit_group[u];
    return g < 0 || g >= a.G || n < 0 || n > a.k_max || p < -1 || p >= a.prefix_U ? -2 : p;
}

__global__ void __launch_bounds__(SHARE_THREADS) k_classes(const __grid_constant__ ShareArgs a)
{
    pdl_wait();
    __shared__ uint32_t s_bits[SHARE_WORDS];
    __shared__ int s_list[SHARE_THREADS], s_n, s_first, s_sum[SHARE_THREADS / 32];
    const int u = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    int g, gv;
    const int p = prefix_of(a, u, g);
    if (t == 0) s_first = u;
    for (int w = t; w < a.words; w += SHARE_THREADS) s_bits[w] = 0u;
    __syncthreads();
    if (p >= 0)
        for (int v = t; v < u; v += SHARE_THREADS)
            if (prefix_of(a, v, gv) == p && gv == g) atomicMin(&s_first, v);
    __syncthreads();
    const bool leads = p >= 0 && s_first == u;
    if (t == 0) {
        if (p == -2) latch_status(a.status, RS3_EINVAL);
        a.own_count[u] = p == -2 ? 0 : a.count[u];
        a.leader[u] = p >= 0 ? s_first : -1;
        a.class_group[u] = leads ? g : 0;
        a.class_bank[u] = leads ? p : -1;
        if (!leads) a.class_count[u] = 0;
    }
    if (!leads) return;
    // the kept cells of the class's units
    for (int v0 = u; v0 < a.U; v0 += SHARE_THREADS) {
        if (t == 0) s_n = 0;
        __syncthreads();
        const int v = v0 + t;
        if (v < a.U && prefix_of(a, v, gv) == p && gv == g) s_list[atomicAdd(&s_n, 1)] = v;
        __syncthreads();
        const int n = s_n;
        for (int i = 0; i < n; ++i) {
            const int w = s_list[i], kept = a.count[w];
            const int32_t *row = a.idx + (int64_t)w * a.k_max;
            for (int j = t; j < kept; j += SHARE_THREADS) {
                const int cell = row[j];
                if (cell >= 0 && cell < a.mn) atomicOr(&s_bits[cell >> 5], 1u << (cell & 31));
                else latch_status(a.status, RS3_EINVAL);
            }
        }
        __syncthreads();
    }
    // their places: a thread takes two words (512 at most)
    const int w0 = 2 * t;
    const uint32_t b0 = w0 < a.words ? s_bits[w0] : 0u, b1 = w0 + 1 < a.words ? s_bits[w0 + 1] : 0u;
    const int mine = __popc(b0) + __popc(b1);
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
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (w0 + i >= a.words) break;
        uint32_t b = i ? b1 : b0;
        a.bits[(int64_t)u * a.words + w0 + i] = b;
        a.before[(int64_t)u * a.words + w0 + i] = at;
        for (; b; b &= b - 1u) out[at++] = (w0 + i) * 32 + __ffs(b) - 1;
    }
}
static_assert(2 * SHARE_THREADS >= SHARE_WORDS, "words of a thread");

// A row's pieces over one bank.
struct Pieces {
    const float2 *ml;
    const float *o;
    int64_t step;                          // rows of a slot
    int n, slot0, slice;
    __device__ __forceinline__ int64_t slot(int s) const { return s == 0 ? slot0 : 2 * (int64_t)(slice + s); }
    __device__ __forceinline__ float2 at(int s) const { return __ldg(ml + slot(s) * step); }
};

__device__ __forceinline__ Pieces pieces_of(const ReadoutArgs &a, int u, int j, int h)
{
    const int BM = a.header->bm;
    const GroupParts g = a.parts[a.ranges[u].slot_base + j / BM * a.H + h];
    Pieces p;
    p.ml = reinterpret_cast<const float2 *>(a.part_ml) + j % BM;
    p.o = a.part_o + (int64_t)(j % BM) * a.d;
    p.step = BM;
    p.n = g.n;
    p.slot0 = g.slot0;
    p.slice = g.slice;
    return p;
}

// L lanes take a row of one head, four columns each at a time.
template <typename T, int L>
__global__ void __launch_bounds__(256) k_merge_two(const __grid_constant__ ReadoutArgs own, const __grid_constant__ ReadoutArgs pre,
                                                   const __grid_constant__ ShareArgs s)
{
    pdl_wait();
    const int lane = threadIdx.x % L;
    const int64_t rows = (int64_t)own.U * own.k_max * own.H;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L; i < rows; i += (int64_t)gridDim.x * (256 / L)) {
        const int h = (int)(i % own.H);
        const int64_t r = i / own.H;
        const int u = (int)(r / own.k_max), j = (int)(r - (int64_t)u * own.k_max);
        if (j >= own.ranges[u].cnt) continue;              // (0 for a unit that is skipped)
        const int cell = __ldg(s.idx + r);
        if (cell < 0 || cell >= own.mn) {
            if (lane == 0) latch_status(own.status, RS3_EINVAL);
            continue;
        }
        const int c = s.leader[u];
        Pieces p[2];
        p[0] = pieces_of(own, u, j, h);
        p[1].n = 0;
        if (c >= 0) {
            const int64_t w = (int64_t)c * s.words + (cell >> 5);
            const int place = s.before[w] + __popc(s.bits[w] & ((1u << (cell & 31)) - 1u));
            if (place >= pre.ranges[c].cnt) continue;      // (its prefix is unsound)
            p[1] = pieces_of(pre, c, place, h);
        }
        float M = -INFINITY, l = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
            for (int x = 0; x < p[b].n; ++x) M = fmaxf(M, p[b].at(x).x);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int b = 0; b < 2; ++b)
            for (int x = 0; x < p[b].n; ++x) {
                const float2 v = p[b].at(x);
                l = fmaf(exp2f(v.x - ref), v.y, l);
            }
        const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l;
        for (int col = 4 * lane; col < own.d; col += 4 * L) {
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll 4
                for (int x = 0; x < p[b].n; ++x) {
                    const float wt = exp2f(p[b].at(x).x - ref);
                    const float4 o = __ldg(reinterpret_cast<const float4 *>(p[b].o + p[b].slot(x) * p[b].step * own.d + col));
                    acc.x = fmaf(wt, o.x, acc.x);
                    acc.y = fmaf(wt, o.y, acc.y);
                    acc.z = fmaf(wt, o.z, acc.z);
                    acc.w = fmaf(wt, o.w, acc.w);
                }
            const float o4[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
            store_out4<T>(own, u, cell, h * own.d + col, o4);
        }
    }
}

template <typename T>
void launch_merge(const ReadoutArgs &own, const ReadoutArgs &pre, const ShareArgs &s, cudaStream_t st)
{
    using Kern = void (*)(ReadoutArgs, ReadoutArgs, ShareArgs);
    const int L = own.d >= 128 ? 32 : own.d / 4;
    const Kern kern = L == 32 ? k_merge_two<T, 32> : L == 16 ? k_merge_two<T, 16> : L == 8 ? k_merge_two<T, 8> : k_merge_two<T, 4>;
    int64_t ctas = ((int64_t)own.U * own.k_max * own.H * L + 255) / 256;
    if (ctas > 16ll * rs3_sm_count()) ctas = 16ll * rs3_sm_count();
    if (ctas < 1) ctas = 1;
    launch_pdl(kern, dim3((unsigned)ctas), dim3(256), 0, st, own, pre, s);
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

ShareLayout share_layout(const rs3_bank *bank, const rs3_bank *prefix, int k_max)
{
    const rs3_dtype dtype = (rs3_dtype)bank->dtype;
    const int U = bank->U, H = bank->H, d = bank->d;
    ShareLayout L;
    L.own = choose_readout_path(dtype, d, U, H, k_max, bank->rows_per_unit, SIZE_MAX);
    L.pre = choose_readout_path(dtype, d, U, H, k_max, prefix->rows_per_unit, SIZE_MAX);
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
    return share_layout(bank, prefix, k_max).total;
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
    const ShareLayout L = share_layout(bank, prefix, k_max);
    if (!rs3_readout_fits(bank->U, H, k_max, L.own) || !rs3_readout_fits(bank->U, H, k_max, L.pre)) return RS3_EUNSUPPORTED;
    if (workspace_bytes < L.total) return RS3_ECAPACITY;
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
    ReadoutArgs own, pre;
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
    if ((s = rs3_readout_run_launch(own, L.own, dtype, st)) != RS3_OK) return s;
    if (dtype == RS3_BF16) launch_merge<uint16_t>(own, pre, sh, st);
    else launch_merge<float>(own, pre, sh, st);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
