// rs3_sparse_readout.cu -- attention of each kept query over the blocks listed for it, scattered
// back to the grid (Sec. 3.1's readout, Eq. 6 and Eq. 7, over chosen blocks of the bank).
#include "rs3_sparse.cuh"

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

}  // namespace

extern "C" size_t rs3_sparse_readout_workspace_bytes(int U, int H, int d, int k_max, int n_top, int n_blocks, rs3_dtype dtype)
{
    if (U < 1 || H < 1 || d < 1 || k_max < 0 || n_top < 1 || n_blocks < 0) return 0;
    if (dtype != RS3_F32 && dtype != RS3_BF16) return 0;
    return 16;
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
    if (k_max > 0) {
        const int pieces = d * (int)elem_bytes(dtype) / 16;
        const dim3 grid((unsigned)k_max, (unsigned)H, (unsigned)a.s.U);
        void (*kern)(AttendArgs, int) = dtype == RS3_BF16 ? k_attend_gather<uint16_t, 1>
                                        : pieces > 32     ? k_attend_gather<float, 2> : k_attend_gather<float, 1>;
        launch_pdl(kern, grid, dim3(32 * GATHER_WARPS), 0, st, a, pieces > 32 ? 32 : pieces);
    }
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
