// rs3_block_norm.cu -- the norms around a block with its gate and residual scale in one pass:
//
//   x' = alpha x + gate * post(y),   h = pre(x')
//   post, pre:  n(v) * weight + bias;  n(v) = v, v / sqrt(mean(v^2) + eps), or
//               (v - mean) / sqrt(mean((v - mean)^2) + eps)
//
// over the kept cells of every unit or all of them, in fp32, x' and h rounded once (h is taken
// from x' before its rounding).  A row of x and y is read once into the registers of a group of
// lanes, the variance is summed around the mean that is already known, and gate * weight and
// gate * bias are formed once per CTA; the next row is fetched while one is normed.  The call is bound by the
// bytes of y, x, x' and h: 147 456 rows of 256 in bf16 (302 MB) 58 us, 5.2 TB/s, where a plain copy of as
// many bytes takes 52; next by issuing (54% of the slots).  8 192 rows of 1 024 in fp32, a CTA to a row and
// three sums over it each: 29 us (32 without the fetch ahead).
#include "rs3_rows.cuh"

namespace {

struct BlockNorm {
    const uint8_t *y, *x;              // [U][mn][C]; y may be NULL (a zero block)
    uint8_t *xo, *ho;                  // each may be NULL
    const int32_t *idx, *count;        // NULL: every cell
    int32_t *status;
    const float *vec[5];               // post weight, post bias, gate, pre weight, pre bias; NULL: 1, 0, 1, 1, 0
    int64_t stride[5];                 // elements between units
    int32_t post, pre;                 // rs3_norm_kind
    float post_eps, pre_eps, alpha;
    int32_t mn, C, k_max, pieces, per_cta;
};

constexpr int BN_THREADS = 256;

template <int N>
__device__ __forceinline__ void load_vec(float *v, const float *p, float without)
{
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        const float4 w = p ? __ldg(reinterpret_cast<const float4 *>(p + e)) : make_float4(without, without, without, without);
        v[e] = w.x; v[e + 1] = w.y; v[e + 2] = w.z; v[e + 3] = w.w;
    }
}

// Sum over the L lanes of a row, or over the CTA's threads (L = BN_THREADS).
template <int L>
__device__ __forceinline__ float row_sum(float v)
{
#pragma unroll
    for (int o = (L < 32 ? L : 32) >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (L > 32) {
        __shared__ float part[BN_THREADS / 32];
        __syncthreads();                                   // the sums before have been read
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < BN_THREADS / 32; ++w) v += part[w];
    }
    return v;
}

// v[ITEMS][N] of a row of C values normed in place; lanes without a piece hold zeros.
template <int L, int ITEMS, int N>
__device__ __forceinline__ void norm_row(float (&v)[ITEMS][N], int kind, float eps, float inv_c, const bool (&in)[ITEMS])
{
    if (kind == RS3_NORM_NONE) return;
    float s = 0.f;
    if (kind == RS3_NORM_LAYER) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) s += v[i][e];
        const float mean = row_sum<L>(s) * inv_c;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) v[i][e] = in[i] ? v[i][e] - mean : 0.f;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) s = fmaf(v[i][e], v[i][e], s);
    const float r = rsqrtf(fmaf(row_sum<L>(s), inv_c, eps));
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) v[i][e] *= r;
}

// Rows [blockIdx.x per_cta, + per_cta) of unit blockIdx.y; a group of L lanes takes every
// (BN_THREADS / L)-th of them, lane l the pieces l, l + L, ... (ITEMS of them at most).
template <typename T, int L, int ITEMS>
__global__ void __launch_bounds__(BN_THREADS, ITEMS == 1 ? 3 : 2) k_block_norm(const __grid_constant__ BlockNorm a)
{
    constexpr int N = Piece<T>::N, GROUPS = BN_THREADS / L;
    pdl_wait();
    const int u = blockIdx.y, lane = threadIdx.x % L;
    int rows = a.mn;
    if (a.idx) {
        rows = a.count[u];
        if (rows < 0 || rows > a.k_max) {
            if (threadIdx.x == 0 && blockIdx.x == 0) latch_status(a.status, RS3_EINVAL);
            return;
        }
    }
    const int first = blockIdx.x * a.per_cta, last = min(rows, first + a.per_cta);
    if (first >= last) return;
    const float inv_c = 1.f / (float)a.C;
    bool in[ITEMS];
    int at[ITEMS];                                         // first channel of a piece
    float ga[ITEMS][N], gb[ITEMS][N], w[ITEMS][N], b[ITEMS][N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        in[i] = lane + i * L < a.pieces;
        at[i] = in[i] ? (lane + i * L) * N : 0;
        const float *p[5];
#pragma unroll
        for (int k = 0; k < 5; ++k) p[k] = a.vec[k] ? a.vec[k] + u * a.stride[k] + at[i] : nullptr;
        float g[N];
        load_vec<N>(g, p[2], 1.f);
        load_vec<N>(ga[i], p[0], 1.f);
        load_vec<N>(gb[i], p[1], 0.f);
        load_vec<N>(w[i], p[3], 1.f);
        load_vec<N>(b[i], p[4], 0.f);
#pragma unroll
        for (int e = 0; e < N; ++e) { ga[i][e] *= g[e]; gb[i][e] *= g[e]; }
    }
    const int64_t row_bytes = (int64_t)a.C * sizeof(T), unit = (int64_t)u * a.mn;
    // (a warp's groups go round together: their shuffles name all lanes)
    const int turns = (last - first + GROUPS - 1) / GROUPS;
    uint4 yn[ITEMS], xn[ITEMS];                            // the next row's, under way while this one is normed
    int64_t next = -1;                                     // its first byte, or -1
    const auto fetch = [&](int t) {
        const int j = first + t * GROUPS + threadIdx.x / L;
        int cell = t < turns && j < last ? (a.idx ? __ldg(a.idx + (int64_t)u * a.k_max + j) : j) : -1;
        if (t < turns && j < last && (cell < 0 || cell >= a.mn)) {
            if (lane == 0) latch_status(a.status, RS3_EINVAL);
            cell = -1;
        }
        next = cell < 0 ? -1 : (unit + cell) * row_bytes;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const bool take = in[i] && next >= 0;
            yn[i] = take && a.y ? __ldcs(reinterpret_cast<const uint4 *>(a.y + next) + lane + i * L) : make_uint4(0, 0, 0, 0);
            xn[i] = take ? __ldcs(reinterpret_cast<const uint4 *>(a.x + next) + lane + i * L) : make_uint4(0, 0, 0, 0);
        }
    };
    fetch(0);
    for (int t = 0; t < turns; ++t) {
        const int64_t off = next;
        uint4 yr[ITEMS], xr[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) { yr[i] = yn[i]; xr[i] = xn[i]; }
        fetch(t + 1);
        float v[ITEMS][N], x[ITEMS][N];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            Piece<T>::widen(yr[i], v[i]);
            Piece<T>::widen(xr[i], x[i]);
        }
        if (a.y) {
            norm_row<L>(v, a.post, a.post_eps, inv_c, in);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) x[i][e] = in[i] ? fmaf(a.alpha, x[i][e], fmaf(v[i][e], ga[i][e], gb[i][e])) : 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) x[i][e] *= a.alpha;
        }
        if (a.xo) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (in[i] && off >= 0) reinterpret_cast<uint4 *>(a.xo + off)[lane + i * L] = Piece<T>::narrow(x[i]);
        }
        if (a.ho) {
            norm_row<L>(x, a.pre, a.pre_eps, inv_c, in);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
                for (int e = 0; e < N; ++e) x[i][e] = fmaf(x[i][e], w[i][e], b[i][e]);
                if (in[i] && off >= 0) reinterpret_cast<uint4 *>(a.ho + off)[lane + i * L] = Piece<T>::narrow(x[i]);
            }
        }
    }
}

using BlockKernel = void (*)(BlockNorm);

// The lanes and pieces per lane of a row.
template <typename T>
BlockKernel block_kernel(int pieces, int &lanes)
{
    if (pieces <= 32) {
        lanes = 1;
        while (lanes < pieces) lanes <<= 1;
        switch (lanes) {
        case 1: return k_block_norm<T, 1, 1>;
        case 2: return k_block_norm<T, 2, 1>;
        case 4: return k_block_norm<T, 4, 1>;
        case 8: return k_block_norm<T, 8, 1>;
        case 16: return k_block_norm<T, 16, 1>;
        default: return k_block_norm<T, 32, 1>;
        }
    }
    lanes = 32;
    if (pieces <= 64) return k_block_norm<T, 32, 2>;
    lanes = BN_THREADS;
    if (pieces <= 256) return k_block_norm<T, BN_THREADS, 1>;
    if constexpr (sizeof(T) == 4)
        if (pieces > 512) return k_block_norm<T, BN_THREADS, 4>;
    return k_block_norm<T, BN_THREADS, 2>;                 // bf16: 512 pieces at most
}

bool norm_ok(const rs3_norm *n, const float **vec, int64_t *stride, int at_weight, int at_bias, int C)
{
    if (!n) return true;
    if (n->kind < RS3_NORM_NONE || n->kind > RS3_NORM_LAYER || !(n->eps >= 0.f)) return false;
    const float *p[2] = {n->weight, n->bias};
    const int64_t s[2] = {n->weight_stride, n->bias_stride};
    const int at[2] = {at_weight, at_bias};
    for (int i = 0; i < 2; ++i) {
        if (p[i] && (!rs3_aligned16(p[i]) || (s[i] != 0 && (s[i] < C || s[i] % 4 != 0)))) return false;
        vec[at[i]] = p[i];
        stride[at[i]] = s[i];
    }
    return true;
}

// Two operands of `bytes` bytes are the same or share none.
bool same_or_apart(const void *a, const void *b, uint64_t bytes)
{
    if (!a || !b || a == b) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x + bytes <= y || y + bytes <= x;
}

}  // namespace

extern "C" rs3_status rs3_norm_residual(const void *y, const void *x, rs3_dtype dtype, int U, int mn, int C, const int32_t *idx,
                                        const int32_t *count, int k_max, const rs3_norm *post, const float *gate,
                                        int64_t gate_stride, float alpha, const rs3_norm *pre, void *x_out, void *h_out,
                                        int32_t *status, rs3_stream_t stream)
{
    if (dtype != RS3_F32 && dtype != RS3_BF16) return RS3_EINVAL;
    const int esz = dtype == RS3_BF16 ? 2 : 4;
    if (!x || (!x_out && !h_out) || U < 1 || mn < 1 || C < 1 || C * (int64_t)esz % 16 != 0) return RS3_EINVAL;
    if (!rs3_aligned16(x) || !rs3_aligned16(y) || !rs3_aligned16(x_out) || !rs3_aligned16(h_out)) return RS3_EINVAL;
    if (!!idx != !!count || (idx && (k_max < 0 || k_max > mn || !status))) return RS3_EINVAL;
    if (!(alpha == alpha) || alpha - alpha != 0.f) return RS3_EINVAL;
    BlockNorm a = {};
    if (!norm_ok(post, a.vec, a.stride, 0, 1, C) || !norm_ok(pre, a.vec, a.stride, 3, 4, C)) return RS3_EINVAL;
    if (gate && (!rs3_aligned16(gate) || (gate_stride != 0 && (gate_stride < C || gate_stride % 4 != 0)))) return RS3_EINVAL;
    if (C > 4096 || mn > RS3_MAX_MN || U > 65535) return RS3_EUNSUPPORTED;
    const uint64_t bytes = (uint64_t)U * mn * C * esz;
    // the two results may each be an operand, in place; they share no byte with each other
    if (x_out && h_out && (x_out == h_out || !same_or_apart(x_out, h_out, bytes))) return RS3_EINVAL;
    if (!same_or_apart(x_out, x, bytes) || !same_or_apart(x_out, y, bytes) || !same_or_apart(h_out, x, bytes) ||
        !same_or_apart(h_out, y, bytes))
        return RS3_EINVAL;
    a.y = static_cast<const uint8_t *>(y);
    a.x = static_cast<const uint8_t *>(x);
    a.xo = static_cast<uint8_t *>(x_out);
    a.ho = static_cast<uint8_t *>(h_out);
    a.idx = idx;
    a.count = count;
    a.status = status;
    a.vec[2] = gate;
    a.stride[2] = gate_stride;
    a.post = post ? post->kind : RS3_NORM_NONE;
    a.pre = pre ? pre->kind : RS3_NORM_NONE;
    a.post_eps = post ? post->eps : 0.f;
    a.pre_eps = pre ? pre->eps : 0.f;
    a.alpha = alpha;
    a.mn = mn;
    a.C = C;
    a.k_max = idx ? k_max : mn;
    a.pieces = C * esz / 16;
    const int rows = a.k_max;
    if (rows == 0) return RS3_OK;
    int lanes;
    const BlockKernel kern = dtype == RS3_BF16 ? block_kernel<uint16_t>(a.pieces, lanes) : block_kernel<float>(a.pieces, lanes);
    const int groups = BN_THREADS / lanes;
    // rows of a CTA: the channels' vectors are read once for them; fewer where SMs would be idle
    int per = 16;
    while (per > 1 && (int64_t)U * ((rows + per * groups - 1) / (per * groups)) < 4ll * rs3_sm_count()) per >>= 1;
    a.per_cta = per * groups;
    const int blocks = (rows + a.per_cta - 1) / a.per_cta;
    launch_pdl(kern, dim3((unsigned)blocks, (unsigned)U), dim3(BN_THREADS), 0, reinterpret_cast<cudaStream_t>(stream), a);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
