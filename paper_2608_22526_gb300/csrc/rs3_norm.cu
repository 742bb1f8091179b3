// rs3_norm.cu -- RMS norm of every query and key head with the position rotation
// (Sec. 3.1, Eq. 7) in the same pass.
//
//   y = x / sqrt(mean(x^2) + eps) * w,  then each pair (y0, y1) of the row's cell becomes
//   (y0 cos - y1 sin, y0 sin + y1 cos)
//
// in fp32, rounded once to the stored type.  A head is read once into the registers of a
// group of lanes (16 bytes each), so the sum of squares, the scaling and the rotation cost no
// second read: the call is bound by the bytes of x and y, and next by issuing instructions.  Queries of
// 16 streams and two fifths of the rows of 48 objects' keys, 96 x 96 cells of 4 heads of 64 in bf16
// (335 MB): 65 us, 5.2 TB/s.  Lanes of a head fixed at compile time, so that the reductions of the rows in flight
// run side by side, and products in pairs took that from 86 us; two rows in flight 66, four (they spill) 68.
#include "rs3_rows.cuh"

namespace {

// One of the call's two tensors (queries or keys).
struct NormSide {
    const uint8_t *x;
    uint8_t *y;
    const float *weight;       // [d] or NULL
    const uint8_t *keep;       // [rows] or NULL
    int64_t rows, x_stride, y_stride;      // strides in bytes
    int32_t H, turns;          // heads; rows of one cell: ceil(rows / mn)
    int32_t per_cta;           // turns that one CTA takes
    int32_t ctas;              // CTAs of this side: cell blocks x turn blocks
    int32_t cell_blocks;
};

constexpr int NORM_THREADS = 256;
constexpr int NORM_FLIGHT = 3;             // rows in flight per lane group
constexpr int NORM_TURNS = 16;             // rows of a cell that a CTA takes

// Two fp32 values in a register pair; a product of pairs is one instruction.
__device__ __forceinline__ uint64_t pair2(float x, float y)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
    return v;
}
__device__ __forceinline__ uint64_t square2(uint64_t x, uint64_t sum)
{
    asm("fma.rn.f32x2 %0, %1, %1, %0;" : "+l"(sum) : "l"(x));
    return sum;
}
__device__ __forceinline__ float2 scale2(uint64_t x, uint64_t r)
{
    float2 v;
    asm("{\n\t.reg .b64 t;\n\tmul.rn.f32x2 t, %2, %3;\n\tmov.b64 {%0, %1}, t;\n\t}" : "=f"(v.x), "=f"(v.y) : "l"(x), "l"(r));
    return v;
}

// A group of L lanes holds one head, ITEMS pieces each; it takes the rows of
// one (cell, head) through the grids that share the cell, so the cell's angles are loaded once.
template <typename T, int ITEMS, int L>
__global__ void __launch_bounds__(NORM_THREADS, ITEMS == 1 ? 4 : 2)
k_norm_rope(NormSide q, NormSide k, int mn, int d, float eps, const float *__restrict__ rope)
{
    constexpr int N = Piece<T>::N, GROUPS = NORM_THREADS / L;
    pdl_wait();
    const bool is_q = (int)blockIdx.x < q.ctas;
    const NormSide &s = is_q ? q : k;
    const int b = is_q ? (int)blockIdx.x : (int)blockIdx.x - q.ctas;
    const int cb = b % s.cell_blocks, tb = b / s.cell_blocks;
    const int lane = threadIdx.x & (L - 1);
    const int64_t g = (int64_t)cb * GROUPS + threadIdx.x / L;      // (cell, head)
    const int pieces = d / N;
    const bool here = g < (int64_t)mn * s.H;
    const int cell = here ? (int)(g / s.H) : 0, head = here ? (int)(g % s.H) : 0;
    // what the cell's rows share, the weights times the angles: a pair becomes
    // (x0 wc0 - x1 ws1, x0 ws0 + x1 wc1) / norm, (wc, ws) = (w cos, w sin)
    float co[ITEMS][N], si[ITEMS][N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int p = lane + i * L;
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            float4 w = make_float4(1.f, 1.f, 1.f, 1.f), c = make_float4(1.f, 0.f, 1.f, 0.f);
            if (p < pieces && s.weight) w = __ldg(reinterpret_cast<const float4 *>(s.weight + p * N + e));
            if (p < pieces && rope) c = __ldg(reinterpret_cast<const float4 *>(rope + (int64_t)cell * d + p * N + e));
            co[i][e] = w.x * c.x; si[i][e] = w.x * c.y;
            co[i][e + 1] = w.y * c.x; si[i][e + 1] = w.y * c.y;
            co[i][e + 2] = w.z * c.z; si[i][e + 2] = w.z * c.w;
            co[i][e + 3] = w.w * c.z; si[i][e + 3] = w.w * c.w;
        }
    }
    const float inv_d = 1.f / (float)d;
    const int t0 = tb * s.per_cta, t1 = min(s.turns, t0 + s.per_cta);
    const int64_t row0 = (int64_t)t0 * mn + cell;
    const uint8_t *src = s.x + row0 * s.x_stride + (head * pieces + lane) * 16;
    uint8_t *dst = s.y + row0 * s.y_stride + (head * pieces + lane) * 16;
    const int64_t x_turn = s.x_stride * mn, y_turn = s.y_stride * mn;
    // the rows that are kept, a bit for each of this CTA's turns (NORM_TURNS at most): a group's lanes look them up
    uint32_t kept = 0;
#pragma unroll
    for (int f = lane; f < NORM_TURNS; f += L) {
        const int64_t row = row0 + (int64_t)f * mn;
        kept |= (uint32_t)(here && t0 + f < t1 && row < s.rows && (!s.keep || s.keep[row] != 0)) << f;
    }
#pragma unroll
    for (int o = L >> 1; o > 0; o >>= 1) kept |= __shfl_xor_sync(0xffffffffu, kept, o);
    // a warp goes from one turn to the next that any of its lanes keeps
    uint32_t todo = __reduce_or_sync(0xffffffffu, kept);
    while (todo != 0u) {
        uint4 v[NORM_FLIGHT][ITEMS];
        int turn[NORM_FLIGHT];
        float sum[NORM_FLIGHT];
#pragma unroll
        for (int f = 0; f < NORM_FLIGHT; ++f) {
            turn[f] = todo != 0u ? __ffs(todo) - 1 : -1;
            todo &= todo - 1u;
            const bool take = turn[f] >= 0 && (kept >> turn[f] & 1u);
            const uint4 *x = reinterpret_cast<const uint4 *>(src + turn[f] * x_turn);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) v[f][i] = take && lane + i * L < pieces ? __ldcs(x + i * L) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int f = 0; f < NORM_FLIGHT; ++f) {
            uint64_t two = 0;                          // (0.f, 0.f)
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                float x[N];
                Piece<T>::widen(v[f][i], x);
#pragma unroll
                for (int e = 0; e < N; e += 2) two = square2(pair2(x[e], x[e + 1]), two);
            }
            sum[f] = __uint_as_float((uint32_t)two) + __uint_as_float((uint32_t)(two >> 32));
        }
#pragma unroll
        for (int o = L >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int f = 0; f < NORM_FLIGHT; ++f) sum[f] += __shfl_xor_sync(0xffffffffu, sum[f], o);
#pragma unroll
        for (int f = 0; f < NORM_FLIGHT; ++f) {
            if (turn[f] < 0) break;
            const float r = rsqrtf(fmaf(sum[f], inv_d, eps));
            uint4 *y = reinterpret_cast<uint4 *>(dst + turn[f] * y_turn);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                float x[N], z[N];
                Piece<T>::widen(v[f][i], x);
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const float2 n = scale2(pair2(x[e], x[e + 1]), pair2(r, r));
                    z[e] = fmaf(n.x, co[i][e], -(n.y * si[i][e + 1]));
                    z[e + 1] = fmaf(n.x, si[i][e], n.y * co[i][e + 1]);
                }
                if ((kept >> turn[f] & 1u) && lane + i * L < pieces) y[i * L] = Piece<T>::narrow(z);
            }
        }
    }
}

using NormKernel = void (*)(NormSide, NormSide, int, int, float, const float *);

template <typename T>
NormKernel norm_kernel(int L)
{
    switch (L) {
    case 1: return k_norm_rope<T, 1, 1>;
    case 2: return k_norm_rope<T, 1, 2>;
    case 4: return k_norm_rope<T, 1, 4>;
    case 8: return k_norm_rope<T, 1, 8>;
    case 16: return k_norm_rope<T, 1, 16>;
    default: return k_norm_rope<T, 1, 32>;
    }
}

// Fills one side; false when its arguments are not what the header asks for.
bool norm_side(NormSide &s, const void *x, int64_t rows, int64_t stride, int H, const float *weight, const uint8_t *keep,
               void *y, int64_t y_stride, int esz, int d)
{
    s = {};
    s.cell_blocks = 1;
    if (rows == 0 && !x && !y) return true;
    if (!x || !y || rows < 0 || H < 1) return false;
    if (!rs3_aligned16(x) || !rs3_aligned16(y) || (weight && !rs3_aligned16(weight))) return false;
    const int64_t width = (int64_t)H * d;
    if (stride < width || y_stride < width || stride * esz % 16 != 0 || y_stride * esz % 16 != 0) return false;
    if (x == y && stride != y_stride) return false;          // in place: every row over itself
    s.x = static_cast<const uint8_t *>(x);
    s.y = static_cast<uint8_t *>(y);
    s.weight = weight;
    s.keep = keep;
    s.rows = rows;
    s.x_stride = stride * esz;
    s.y_stride = y_stride * esz;
    s.H = H;
    return true;
}

// No result lies over an operand or the other result, but for its own operand in place.
bool norm_apart(const NormSide &s, const NormSide &t, int64_t s_width, int64_t t_width)
{
    return (s.x == s.y || rows_apart(s.y, s.rows, s.y_stride, s_width, s.x, s.rows, s.x_stride, s_width)) &&
           rows_apart(s.y, s.rows, s.y_stride, s_width, t.x, t.rows, t.x_stride, t_width) &&
           rows_apart(s.y, s.rows, s.y_stride, s_width, t.y, t.rows, t.y_stride, t_width);
}

}  // namespace

extern "C" rs3_status rs3_qk_norm_rope(const void *q, int64_t q_rows, int64_t q_stride, int Hq, const float *q_weight,
                                       const uint8_t *q_keep, void *q_out, int64_t q_out_stride, const void *k,
                                       int64_t k_rows, int64_t k_stride, int Hk, const float *k_weight,
                                       const uint8_t *k_keep, void *k_out, int64_t k_out_stride, rs3_dtype dtype, int mn,
                                       int d, float eps, const float *rope, rs3_stream_t stream)
{
    if (dtype != RS3_F32 && dtype != RS3_BF16) return RS3_EINVAL;
    if (mn < 1 || d < 1 || !(eps >= 0.f) || (rope && !rs3_aligned16(rope))) return RS3_EINVAL;
    const int esz = dtype == RS3_BF16 ? 2 : 4;
    if (d * esz % 16 != 0) return RS3_EINVAL;
    if (d > 256 || mn > RS3_MAX_MN) return RS3_EUNSUPPORTED;
    NormSide s[2];
    if (!norm_side(s[0], q, q_rows, q_stride, Hq, q_weight, q_keep, q_out, q_out_stride, esz, d) ||
        !norm_side(s[1], k, k_rows, k_stride, Hk, k_weight, k_keep, k_out, k_out_stride, esz, d))
        return RS3_EINVAL;
    const int64_t width[2] = {(int64_t)s[0].H * d * esz, (int64_t)s[1].H * d * esz};
    if (!norm_apart(s[0], s[1], width[0], width[1]) || !norm_apart(s[1], s[0], width[1], width[0])) return RS3_EINVAL;
    const int pieces = d * esz / 16, items = pieces > 32 ? 2 : 1;
    int L = 1;
    while (L * items < pieces) L <<= 1;
    const int groups = NORM_THREADS / L;
    int64_t total = 0;
    for (NormSide &t : s) {
        if (t.rows == 0) continue;
        const int64_t turns = (t.rows + mn - 1) / mn, cells = t.rows < mn ? t.rows : mn;
        const int64_t cb = (cells * t.H + groups - 1) / groups;
        // fewer rows to a CTA where SMs would be idle
        int64_t per = NORM_TURNS;
        while (per > 1 && cb * ((turns + per - 1) / per) < 4ll * rs3_sm_count()) per >>= 1;
        const int64_t ctas = cb * ((turns + per - 1) / per);
        if (turns > INT32_MAX || ctas > INT32_MAX) return RS3_EUNSUPPORTED;
        t.turns = (int32_t)turns;
        t.per_cta = (int32_t)per;
        t.cell_blocks = (int32_t)cb;
        t.ctas = (int32_t)ctas;
        total += ctas;
    }
    if (total == 0) return RS3_OK;
    if (total > INT32_MAX) return RS3_EUNSUPPORTED;
    NormKernel kern = k_norm_rope<float, 2, 32>;
    if (items == 1) kern = dtype == RS3_BF16 ? norm_kernel<uint16_t>(L) : norm_kernel<float>(L);
    launch_pdl(kern, dim3((unsigned)total), dim3(NORM_THREADS), 0, reinterpret_cast<cudaStream_t>(stream), s[0], s[1], mn, d,
               eps, rope);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
