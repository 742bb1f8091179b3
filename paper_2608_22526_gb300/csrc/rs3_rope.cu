// rs3_rope.cu -- rotary positions (Sec. 3.1, Eq. 7) from the coordinates of a row: tables of
// (cos, sin), and rows turned in place or out of place.
//
// Pair p of an axis with n pairs turns by pos * f_p, f_p = base^(-p/n), stretched for positions
// beyond those trained on.  An angle of a far position loses its fraction in fp32, and fp64 is slow
// here, so positions are counted in turns in whole numbers: F_p = f_p / (2 pi) as a fraction of
// 2^64, pos * F_p mod 2^64 is the angle's fraction of a turn without rounding (F_p's own error of
// 2^-53 relative, times pos, is all there is).  Its nearest quarter turn is taken off in whole
// numbers too, and what is left, |t| <= pi / 4, goes through the Taylor series of sine and cosine:
// up to t^11 and t^10, whose next terms are below 1e-11 and 2e-10 there.
//
// A warp takes rows one after another: a row's angles are computed once, a pair per lane, and go
// through shared memory to the pieces of all of its heads; the loads of the next rows are in flight
// meanwhile.  The call is bound by the bytes of x and y.
#include "rs3_rows.cuh"

#include <cmath>

namespace {

constexpr int ROPE_PAIRS = 128;            // of a head of 256
constexpr int ROPE_WARPS = 8;
constexpr int ROPE_FLIGHT = 4;             // rows of a warp in flight

// The pairs' frequencies in turns per position, of 2^64.
struct RopeTurns {
    uint64_t f[ROPE_PAIRS];
    uint8_t axis[ROPE_PAIRS];
    int32_t half, axes;
    float magnitude, sign;                 // of the turned elements; -1 turns back
};

// (cos, sin) of `turn` / 2^64 turns.
__device__ __forceinline__ float2 cos_sin(uint64_t turn)
{
    const uint32_t quarter = (uint32_t)((turn + (1ull << 61)) >> 62);
    const int64_t rest = (int64_t)(turn - ((uint64_t)quarter << 62));      // within an eighth of a turn of 0
    const float t = (float)(int32_t)(rest >> 30) * (6.283185307179586f / 17179869184.f);   // 2^34 to a turn
    const float z = t * t;
    float s = fmaf(z, -1.f / 39916800.f, 1.f / 362880.f);
    s = fmaf(s, z, -1.f / 5040.f);
    s = fmaf(s, z, 1.f / 120.f);
    s = fmaf(s, z, -1.f / 6.f);
    s = fmaf(s * z, t, t);
    float c = fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
    c = fmaf(c, z, -1.f / 720.f);
    c = fmaf(c, z, 1.f / 24.f);
    c = fmaf(c, z, -0.5f);
    c = fmaf(c, z, 1.f);
    const float a = quarter & 1u ? s : c, b = quarter & 1u ? c : s;
    return make_float2((quarter + 1u) & 2u ? -a : a, quarter & 2u ? -b : b);
}

__device__ __forceinline__ float2 row_angle(const int32_t *pos, uint64_t f, int axis, float sign, float magnitude)
{
    const float2 v = cos_sin((uint64_t)(int64_t)__ldg(pos + axis) * f);
    return make_float2(v.x * magnitude, v.y * sign * magnitude);
}

// One of the call's two tensors (queries or keys).
struct RopeSide {
    const uint8_t *x;
    uint8_t *y;
    const int32_t *pos;                    // [rows][axes]
    const uint8_t *keep;                   // [rows] or NULL
    int64_t rows, x_stride, y_stride;      // strides in bytes
    int32_t H, chunk;                      // heads; rows of a warp
    int32_t ctas;
};

__device__ __forceinline__ void load_turns(const RopeTurns &t, uint64_t *f, uint8_t *axis)
{
    for (int p = threadIdx.x; p < t.half; p += blockDim.x) {
        f[p] = t.f[p];
        axis[p] = t.axis[p];
    }
    __syncthreads();
}

// x[N] of a piece that begins at element e of a head, each with its partner and its pair's angle.
// pairs: (2p, 2p + 1); halves: (p, p + half), whose partners lie in a second piece.
template <int N>
__device__ __forceinline__ void turn_pairs(float *x, const float2 *cs)
{
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        const float2 a = cs[e / 2];
        const float x0 = x[e], x1 = x[e + 1];
        x[e] = fmaf(x0, a.x, -(x1 * a.y));
        x[e + 1] = fmaf(x0, a.y, x1 * a.x);
    }
}

// WIDE: halves whose two pieces begin on 16-byte boundaries; a lane holds both.  Otherwise a lane
// holds one piece, and with halves reads its partners from the row's copy in shared memory.
template <typename T, bool HALVES, bool WIDE>
__global__ void __launch_bounds__(ROPE_WARPS * 32, 3)
k_rope_rows(const __grid_constant__ RopeSide q, const __grid_constant__ RopeSide k, const __grid_constant__ RopeTurns turns, int d)
{
    constexpr int N = Piece<T>::N;
    pdl_wait();
    extern __shared__ __align__(16) uint8_t s_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int half = turns.half, rot = 2 * half;
    // [half] turns, [half] axes; per warp [FLIGHT][half] (cos, sin) and, for halves of odd places, a row
    uint64_t *s_f = reinterpret_cast<uint64_t *>(s_raw);
    uint8_t *s_axis = s_raw + 8 * ROPE_PAIRS;
    const bool is_q = (int)blockIdx.x < q.ctas;
    const RopeSide &s = is_q ? q : k;
    const int pieces = d / N;
    float2 *s_cs = reinterpret_cast<float2 *>(s_raw + 9 * ROPE_PAIRS) + warp * ROPE_FLIGHT * half;
    T *s_row = reinterpret_cast<T *>(s_raw + 9 * ROPE_PAIRS + ROPE_WARPS * ROPE_FLIGHT * half * 8) +
               (size_t)warp * ROPE_FLIGHT * d;
    load_turns(turns, s_f, s_axis);
    // a head's items: WIDE: half / N pairs of pieces, then the pieces past the turned ones
    const int both = WIDE ? half / N : 0;
    const int items = WIDE ? both + pieces - 2 * both : pieces;
    const int64_t warp_id = (int64_t)((int)blockIdx.x - (is_q ? 0 : q.ctas)) * ROPE_WARPS + warp;
    const int64_t row0 = warp_id * s.chunk;
    if (row0 >= s.rows) return;
    const int n = (int)min((int64_t)s.chunk, s.rows - row0);
    uint32_t todo = __ballot_sync(0xffffffffu, lane < n && (!s.keep || s.keep[row0 + (lane < n ? lane : 0)] != 0));
    while (todo) {
        int row[ROPE_FLIGHT], m = 0;
#pragma unroll
        for (int r = 0; r < ROPE_FLIGHT; ++r) {
            row[r] = todo ? __ffs(todo) - 1 : -1;
            m += todo != 0;
            todo &= todo - 1u;
        }
        // the rows' angles
        for (int p = lane; p < half; p += 32) {
            const uint64_t f = s_f[p];
            const int axis = s_axis[p];
#pragma unroll
            for (int r = 0; r < ROPE_FLIGHT; ++r)
                if (row[r] >= 0) s_cs[r * half + p] = row_angle(s.pos + (row0 + row[r]) * turns.axes, f, axis, turns.sign, turns.magnitude);
        }
        __syncwarp();
        if constexpr (HALVES && !WIDE) {
            // head by head: the rows' copies, then every piece with its partners
            for (int h = 0; h < s.H; ++h) {
                for (int i = lane; i < m * pieces; i += 32) {
                    const int r = i / pieces, p = i - r * pieces;
                    const int rr = r == 0 ? row[0] : r == 1 ? row[1] : r == 2 ? row[2] : row[3];
                    reinterpret_cast<uint4 *>(s_row + r * d)[p] =
                        *(reinterpret_cast<const uint4 *>(s.x + (row0 + rr) * s.x_stride) + h * pieces + p);
                }
                __syncwarp();
                for (int i = lane; i < m * pieces; i += 32) {
                    const int r = i / pieces, p = i - r * pieces;
                    const int rr = r == 0 ? row[0] : r == 1 ? row[1] : r == 2 ? row[2] : row[3];
                    float x[N];
                    Piece<T>::widen(reinterpret_cast<const uint4 *>(s_row + r * d)[p], x);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const int at = p * N + e;
                        if (at >= rot) break;
                        const bool low = at < half;
                        const float2 a = s_cs[r * half + (low ? at : at - half)];
                        const T other = s_row[r * d + (low ? at + half : at - half)];
                        float o;
                        if constexpr (sizeof(T) == 2) o = bf16_bits_to_float(other);
                        else o = other;
                        x[e] = low ? fmaf(x[e], a.x, -(o * a.y)) : fmaf(o, a.y, x[e] * a.x);
                    }
                    *(reinterpret_cast<uint4 *>(s.y + (row0 + rr) * s.y_stride) + h * pieces + p) = Piece<T>::narrow(x);
                }
                __syncwarp();
            }
        } else {
            for (int i = lane; i < s.H * items; i += 32) {
                const int h = i / items, it = i - h * items;
                const bool two = WIDE && it < both;
                const int p = WIDE && !two ? 2 * both + it - both : it;
                uint4 v[ROPE_FLIGHT], o[ROPE_FLIGHT];
#pragma unroll
                for (int r = 0; r < ROPE_FLIGHT; ++r) {
                    if (row[r] < 0) continue;
                    const uint4 *x = reinterpret_cast<const uint4 *>(s.x + (row0 + row[r]) * s.x_stride) + h * pieces;
                    v[r] = __ldcs(x + p);
                    if (two) o[r] = __ldcs(x + p + both);
                }
#pragma unroll
                for (int r = 0; r < ROPE_FLIGHT; ++r) {
                    if (row[r] < 0) continue;
                    uint4 *y = reinterpret_cast<uint4 *>(s.y + (row0 + row[r]) * s.y_stride) + h * pieces;
                    float x[N];
                    Piece<T>::widen(v[r], x);
                    if constexpr (WIDE) {
                        if (two) {
                            float z[N];
                            Piece<T>::widen(o[r], z);
                            const float2 *cs = s_cs + r * half + p * N;
#pragma unroll
                            for (int e = 0; e < N; ++e) {
                                const float2 a = cs[e];
                                const float x0 = x[e], x1 = z[e];
                                x[e] = fmaf(x0, a.x, -(x1 * a.y));
                                z[e] = fmaf(x0, a.y, x1 * a.x);
                            }
                            y[p + both] = Piece<T>::narrow(z);
                        }
                    } else {
                        const int first = p * N;           // pairs end on an even element: inside a piece the turned ones come first
                        if (first + N <= rot) {
                            turn_pairs<N>(x, s_cs + r * half + first / 2);
                        } else {
#pragma unroll
                            for (int e = 0; e < N; e += 2)
                                if (first + e < rot) turn_pairs<2>(x + e, s_cs + r * half + (first + e) / 2);
                        }
                    }
                    y[p] = Piece<T>::narrow(x);
                }
            }
        }
        __syncwarp();                                      // the angles are read before the next rows'
    }
}

__global__ void __launch_bounds__(256) k_rope_table(const int32_t *pos, int64_t rows, const __grid_constant__ RopeTurns turns, float2 *out)
{
    __shared__ uint64_t s_f[ROPE_PAIRS];
    __shared__ uint8_t s_axis[ROPE_PAIRS];
    pdl_wait();
    load_turns(turns, s_f, s_axis);
    const int64_t total = rows * turns.half;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = i / turns.half;
        const int p = (int)(i - r * turns.half);
        out[i] = row_angle(pos + r * turns.axes, s_f[p], s_axis[p], turns.sign, turns.magnitude);
    }
}

// The pairs' turns; false when the description is not what the header asks for.
bool rope_turns(const rs3_rope_spec *s, RopeTurns &t)
{
    if (!s || s->rot < 2 || s->rot % 2 != 0 || s->axes < 1 || s->axes > 3) return false;
    if (s->layout != RS3_ROPE_PAIRS && s->layout != RS3_ROPE_HALVES) return false;
    if (!(s->base >= 1.0 && s->base <= 1e12) || !(s->factor >= 1.0 && s->factor <= 1e9) || !(s->context >= 0.0 && s->context <= 1e12)) return false;
    if (s->context > 0.0 && !(s->beta_slow >= 0.0 && s->beta_fast > s->beta_slow && s->beta_fast <= 1e12)) return false;
    if (!(s->magnitude > -1e30f && s->magnitude < 1e30f)) return false;
    int sum = 0;
    for (int a = 0; a < s->axes; ++a) {
        if (s->pairs[a] < 0 || s->pairs[a] > s->rot / 2) return false;
        sum += s->pairs[a];
    }
    if (sum != s->rot / 2) return false;
    if (s->rot > 2 * ROPE_PAIRS) return true;              // (the caller tells that it is not supported)
    const double two_pi = 6.283185307179586476925;
    int p = 0;
    for (int a = 0; a < s->axes; ++a)
        for (int i = 0; i < s->pairs[a]; ++i, ++p) {
            double f = std::pow(s->base, -(double)i / (double)s->pairs[a]);
            double share = 0.0;                            // of the frequency as trained
            if (s->context > 0.0) {
                share = (s->context * f / two_pi - s->beta_slow) / (s->beta_fast - s->beta_slow);
                share = share < 0.0 ? 0.0 : share > 1.0 ? 1.0 : share;
            }
            f *= share + (1.0 - share) / s->factor;
            t.f[p] = (uint64_t)std::ldexp(f / two_pi, 64);
            t.axis[p] = (uint8_t)a;
        }
    t.half = s->rot / 2;
    t.axes = s->axes;
    t.magnitude = s->magnitude;
    t.sign = s->inverse ? -1.f : 1.f;
    return true;
}

// Fills one side; false when its arguments are not what the header asks for.
bool rope_side(RopeSide &s, const void *x, int64_t rows, int64_t stride, int H, const int32_t *pos, const uint8_t *keep, void *y,
               int64_t y_stride, int esz, int d)
{
    s = {};
    if (rows == 0 && !x && !y) return true;
    if (!x || !y || rows < 0 || H < 1 || (rows > 0 && !pos)) return false;
    if (!rs3_aligned16(x) || !rs3_aligned16(y) || (reinterpret_cast<uintptr_t>(pos) & 3u)) return false;
    const int64_t width = (int64_t)H * d;
    if (stride < width || y_stride < width || stride * esz % 16 != 0 || y_stride * esz % 16 != 0) return false;
    if (x == y && stride != y_stride) return false;        // in place: every row over itself
    s.x = static_cast<const uint8_t *>(x);
    s.y = static_cast<uint8_t *>(y);
    s.pos = pos;
    s.keep = keep;
    s.rows = rows;
    s.x_stride = stride * esz;
    s.y_stride = y_stride * esz;
    s.H = H;
    return true;
}

// No result lies over an operand or the other result, but for its own operand in place.
bool rope_apart(const RopeSide &s, const RopeSide &t, int64_t s_width, int64_t t_width)
{
    return (s.x == s.y || rows_apart(s.y, s.rows, s.y_stride, s_width, s.x, s.rows, s.x_stride, s_width)) &&
           rows_apart(s.y, s.rows, s.y_stride, s_width, t.x, t.rows, t.x_stride, t_width) &&
           rows_apart(s.y, s.rows, s.y_stride, s_width, t.y, t.rows, t.y_stride, t_width);
}

}  // namespace

extern "C" void rs3_default_rope_spec(rs3_rope_spec *s)
{
    *s = {};
    s->layout = RS3_ROPE_PAIRS;
    s->axes = 1;
    s->base = 10000.0;
    s->factor = 1.0;
    s->beta_fast = 32.0;
    s->beta_slow = 1.0;
    s->magnitude = 1.f;
}

extern "C" rs3_status rs3_rope_table(const int32_t *pos, int64_t rows, const rs3_rope_spec *spec, float *cos_sin, rs3_stream_t stream)
{
    RopeTurns t = {};
    if (rows < 0 || !rope_turns(spec, t)) return RS3_EINVAL;
    if (rows == 0) return RS3_OK;
    if (!pos || !cos_sin || (reinterpret_cast<uintptr_t>(pos) & 3u) || !rs3_aligned16(cos_sin)) return RS3_EINVAL;
    if (spec->rot > 2 * ROPE_PAIRS || rows > INT64_MAX / 1024) return RS3_EUNSUPPORTED;
    int64_t ctas = (rows * t.half + 255) / 256;
    if (ctas > 16ll * rs3_sm_count()) ctas = 16ll * rs3_sm_count();
    launch_pdl(k_rope_table, dim3((unsigned)ctas), dim3(256), 0, reinterpret_cast<cudaStream_t>(stream), pos, rows, t,
               reinterpret_cast<float2 *>(cos_sin));
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}

extern "C" rs3_status rs3_rope_rows(const void *q, int64_t q_rows, int64_t q_stride, int Hq, const int32_t *q_pos,
                                    const uint8_t *q_keep, void *q_out, int64_t q_out_stride, const void *k, int64_t k_rows,
                                    int64_t k_stride, int Hk, const int32_t *k_pos, const uint8_t *k_keep, void *k_out,
                                    int64_t k_out_stride, rs3_dtype dtype, int d, const rs3_rope_spec *spec, rs3_stream_t stream)
{
    if (dtype != RS3_F32 && dtype != RS3_BF16) return RS3_EINVAL;
    RopeTurns t = {};
    if (d < 1 || !rope_turns(spec, t) || spec->rot > d) return RS3_EINVAL;
    const int esz = dtype == RS3_BF16 ? 2 : 4, n = 16 / esz;
    if (d % n != 0) return RS3_EINVAL;
    if (d > 2 * ROPE_PAIRS) return RS3_EUNSUPPORTED;
    RopeSide s[2];
    if (!rope_side(s[0], q, q_rows, q_stride, Hq, q_pos, q_keep, q_out, q_out_stride, esz, d) ||
        !rope_side(s[1], k, k_rows, k_stride, Hk, k_pos, k_keep, k_out, k_out_stride, esz, d))
        return RS3_EINVAL;
    const int64_t width[2] = {(int64_t)s[0].H * d * esz, (int64_t)s[1].H * d * esz};
    if (!rope_apart(s[0], s[1], width[0], width[1]) || !rope_apart(s[1], s[0], width[1], width[0])) return RS3_EINVAL;
    int64_t total = 0;
    for (RopeSide &r : s) {
        if (r.rows == 0) continue;
        // fewer rows to a warp where SMs would be idle
        int chunk = 32;
        while (chunk > 1 && (r.rows + chunk - 1) / chunk < 16ll * rs3_sm_count()) chunk >>= 1;
        const int64_t warps = (r.rows + chunk - 1) / chunk, ctas = (warps + ROPE_WARPS - 1) / ROPE_WARPS;
        if (ctas > INT32_MAX) return RS3_EUNSUPPORTED;
        r.chunk = chunk;
        r.ctas = (int32_t)ctas;
        total += ctas;
    }
    if (total == 0) return RS3_OK;
    if (total > INT32_MAX) return RS3_EUNSUPPORTED;
    const bool halves = spec->layout == RS3_ROPE_HALVES, wide = halves && t.half % n == 0;
    size_t smem = 9 * ROPE_PAIRS + (size_t)ROPE_WARPS * ROPE_FLIGHT * t.half * 8;
    if (halves && !wide) smem += (size_t)ROPE_WARPS * ROPE_FLIGHT * d * esz;
    using Kern = void (*)(RopeSide, RopeSide, RopeTurns, int);
    Kern kern;
    if (dtype == RS3_BF16)
        kern = wide ? k_rope_rows<uint16_t, true, true> : halves ? k_rope_rows<uint16_t, true, false> : k_rope_rows<uint16_t, false, false>;
    else
        kern = wide ? k_rope_rows<float, true, true> : halves ? k_rope_rows<float, true, false> : k_rope_rows<float, false, false>;
    if (rs3_kernel_smem((const void *)kern, smem) != RS3_OK) return RS3_ECUDA;
    launch_pdl(kern, dim3((unsigned)total), dim3(ROPE_WARPS * 32), smem, reinterpret_cast<cudaStream_t>(stream), s[0], s[1], t, d);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
