// rs3_rope.cu -- rotary positions (Sec. 3.1, Eq. 7) from the coordinates of a row: tables of
// (cos, sin), and rows turned in place or out of place.
//
// Pair p of an axis with n pairs turns by pos * f_p, f_p = base^(-p/n), stretched for positions
// beyond those trained on.  An angle of a far position loses its fraction in fp32, and fp64 is slow
// here, so angles are counted in turns in whole numbers: with F_p = f_p / (2 pi) as a fraction of 2^64,
// pos * F_p mod 2^64 is the angle's fraction of a turn, of which the upper 32 bits are found.  The host has f_p in pairs of
// doubles (100 bits; in one, the ramp of a stretch alone can cost a dozen of the 53), so F_p is off by its rounding, 2^-65,
// the lower bit that turn_of drops and what it cuts off are 2^-64 and 2^-31: |pos| (2^-65 + 2^-64) + 2^-31 is
// below 2^-30 of a turn.  Its nearest quarter turn is
// taken off in whole numbers too (what is left are the low 30 bits, with their sign), and that, |t| <= pi
// / 4, goes through the Taylor series of sine and cosine: up to t^11 and t^10, whose next terms are below
// 1e-11 and 2e-10 there.
//
// A lane keeps one piece of the heads and its pairs' frequencies; its angles of a row are found once, two
// by two on packed pairs, and serve all heads of the row, whose pieces are under way meanwhile.  With
// halves a piece's partners come from the lane that holds them.  Queries of 16 streams and two fifths of
// the rows of 48 objects' keys, 96 x 96 cells of 4 heads of 64 in bf16, 48 elements of a head turned (337
// MB): 89 us, 3.8 TB/s; bound by issuing instructions (per row and lane about 23 for an angle and 40
// for a piece) and by the loads' latency beside few warps (a lane's frequencies, angles and pieces
// under way take 128 registers; 24 warps of 80 registers with four pieces spill: 98 us).  Angles through
// shared memory, so that a row finds each once: 96 to 155 us, as every piece then reads eight of them again.
#include "rs3_rows.cuh"

#include <cmath>

namespace {

constexpr int ROPE_PAIRS = 128;            // of a head of 256
constexpr int ROPE_WARPS = 8;
constexpr int ROPE_CTAS = 2;               // resident per SM
constexpr int ROPE_ROWS = 32;              // rows of a warp
constexpr int ROPE_COPIES = 4;             // of which copies are held at a time, where partners come from copies
constexpr int ROPE_FLIGHT = 4;             // pieces of a lane under way

// The pairs' frequencies in turns per position, of 2^64 (turned back: negative ones).
struct RopeTurns {
    uint64_t f[ROPE_PAIRS];
    uint8_t axis[ROPE_PAIRS];
    int32_t half, axes;
    float magnitude;                       // of the turned elements
};

__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t pair_of(float a, float b)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void split_pair(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }

// The upper 32 bits of pos * f mod 2^64, but for the last (f's lower half loses one).
__device__ __forceinline__ uint32_t turn_of(int32_t pos, uint64_t f)
{
    return (uint32_t)pos * (uint32_t)(f >> 32) + ((uint32_t)__mulhi(pos, (int32_t)((uint32_t)f >> 1)) << 1);
}

// (cos, sin) * magnitude of two angles in 2^-32 turns, the second sine's and cosine's operations on packed
// pairs; the sines with `flip` (0 or the sign bit) changed.
__device__ __forceinline__ void cos_sin_two(uint32_t t0, uint32_t t1, float magnitude, uint32_t flip, float *c, float *s)
{
    const auto both = [](float x) { return pair_of(x, x); };
    const int32_t r0 = (int32_t)(t0 << 2) >> 2, r1 = (int32_t)(t1 << 2) >> 2;
    const uint64_t t = mul_pair(pair_of((float)r0, (float)r1), both(6.283185307179586f / 4294967296.f));
    const uint64_t z = mul_pair(t, t);
    uint64_t a = fma_pair(z, both(-1.f / 39916800.f), both(1.f / 362880.f));
    a = fma_pair(a, z, both(-1.f / 5040.f));
    a = fma_pair(a, z, both(1.f / 120.f));
    a = fma_pair(a, z, both(-1.f / 6.f));
    a = mul_pair(fma_pair(mul_pair(a, z), t, t), both(magnitude));
    uint64_t b = fma_pair(z, both(-1.f / 3628800.f), both(1.f / 40320.f));
    b = fma_pair(b, z, both(-1.f / 720.f));
    b = fma_pair(b, z, both(1.f / 24.f));
    b = fma_pair(b, z, both(-0.5f));
    b = mul_pair(fma_pair(b, z, both(1.f)), both(magnitude));
    float sn[2], cs[2];
    split_pair(a, sn[0], sn[1]);
    split_pair(b, cs[0], cs[1]);
    const uint32_t w[2] = {t0 + (1u << 29), t1 + (1u << 29)};          // the quarter in the two upper bits
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool odd = w[i] & (1u << 30);
        const float x = odd ? sn[i] : cs[i], y = odd ? cs[i] : sn[i];
        c[i] = __uint_as_float(__float_as_uint(x) ^ ((w[i] + (1u << 30)) & 0x80000000u));
        s[i] = __uint_as_float(__float_as_uint(y) ^ ((w[i] ^ flip) & 0x80000000u));
    }
}

// One of the call's two tensors (queries or keys).
struct RopeSide {
    const uint8_t *x;
    uint8_t *y;
    const int32_t *pos;                    // [rows][axes]
    const uint8_t *keep;                   // [rows] or NULL
    int64_t rows, x_stride, y_stride;      // strides in bytes
    int32_t H, chunk;                      // heads; rows that a warp takes before it turns to others
    int64_t chunks;
};

// Into shared memory; pairs behind the last do not turn.
__device__ __forceinline__ void load_turns(const RopeTurns &t, uint64_t *f, uint8_t *axis)
{
    for (int p = threadIdx.x; p < ROPE_PAIRS; p += blockDim.x) {
        f[p] = t.f[p];
        axis[p] = t.axis[p];
    }
    __syncthreads();
}

// LANES: pairs lie within a piece, or a piece's partners are another's of the same head, which a lane
// of the same turn holds.  COPY: halves otherwise, partners come from the rows' copies in shared memory.
enum RopeMode { PAIR_LANES, HALF_LANES, HALF_COPY };

// A piece whose elements from `first` (an even one) on keep the bits that they had.
template <int N>
__device__ __forceinline__ uint4 keep_tail(uint4 turned, uint4 own, int first)
{
    constexpr int W = N / 4;                               // elements of a word
    return make_uint4(first > 0 ? turned.x : own.x, first > W ? turned.y : own.y, first > 2 * W ? turned.z : own.z,
                      first > 3 * W ? turned.w : own.w);
}

// Lanes take the pieces of one head of some rows side by side; heads of more than 32 pieces part by part.
template <typename T, RopeMode MODE>
__global__ void __launch_bounds__(ROPE_WARPS * 32, ROPE_CTAS)
k_rope_rows(const __grid_constant__ RopeSide q, const __grid_constant__ RopeSide k, const __grid_constant__ RopeTurns turns, int d)
{
    constexpr int N = Piece<T>::N;
    constexpr int NP = MODE == PAIR_LANES ? N / 2 : N;     // angles of a piece
    pdl_wait();
    extern __shared__ __align__(16) uint8_t s_raw[];       // copies: [ROPE_COPIES][d] and their (cos, sin) [][half] of each warp
    __shared__ uint64_t s_f[ROPE_PAIRS];
    __shared__ uint8_t s_axis[ROPE_PAIRS];
    __shared__ int s_rows[ROPE_WARPS][ROPE_ROWS], s_pos[ROPE_WARPS][ROPE_ROWS][3];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int half = turns.half, rot = 2 * half, pieces = d / N;
    const int64_t chunk = (int64_t)blockIdx.x * ROPE_WARPS + warp;
    const bool is_q = chunk < q.chunks;
    const uint8_t *x0 = is_q ? q.x : k.x, *keep = is_q ? q.keep : k.keep;
    uint8_t *y0 = is_q ? q.y : k.y;
    const int32_t *pos_in = is_q ? q.pos : k.pos;
    const int64_t x_stride = is_q ? q.x_stride : k.x_stride, y_stride = is_q ? q.y_stride : k.y_stride, n_rows = is_q ? q.rows : k.rows;
    const int H = is_q ? q.H : k.H, per_warp = is_q ? q.chunk : k.chunk;
    const int64_t row0 = (is_q ? chunk : chunk - q.chunks) * per_warp;
    // the rows that are kept, one after another, and their positions
    const bool in = lane < per_warp && row0 + lane < n_rows, on = in && (!keep || keep[row0 + lane] != 0);
    int32_t pos[3];
#pragma unroll
    for (int a = 0; a < 3; ++a) pos[a] = in && a < turns.axes ? __ldg(pos_in + (row0 + lane) * turns.axes + a) : 0;
    load_turns(turns, s_f, s_axis);
    const uint32_t kept = __ballot_sync(0xffffffffu, on);
    if (on) {
        const int at = __popc(kept & ((1u << lane) - 1u));
        s_rows[warp][at] = lane;
#pragma unroll
        for (int a = 0; a < 3; ++a) s_pos[warp][at][a] = pos[a];
    }
    __syncwarp();
    const int n_kept = __popc(kept);
    if (n_kept == 0) return;
    x0 += row0 * x_stride;
    y0 += row0 * y_stride;
    if constexpr (MODE == HALF_COPY) {
        const int copy_bytes = (ROPE_COPIES * d * (int)sizeof(T) + 15) / 16 * 16;
        uint8_t *mine = s_raw + (size_t)warp * (copy_bytes + (ROPE_COPIES * half * 8 + 15) / 16 * 16);
        T *s_row = reinterpret_cast<T *>(mine);
        float2 *s_cs = reinterpret_cast<float2 *>(mine + copy_bytes);
        for (int k0 = 0; k0 < n_kept; k0 += ROPE_COPIES) {
            const int m = min(ROPE_COPIES, n_kept - k0);
            const int *rows = s_rows[warp] + k0;
            for (int i = lane; i < m * half; i += 32) {
                const int r = i / half, p = i - r * half;
                const uint32_t t = turn_of(s_pos[warp][k0 + r][s_axis[p]], s_f[p]);
                float c[2], g[2];
                cos_sin_two(t, t, turns.magnitude, 0u, c, g);
                s_cs[i] = make_float2(c[0], g[0]);
            }
            __syncwarp();
            // head by head: the rows' copies, then every piece with its partners
            for (int h = 0; h < H; ++h) {
                for (int i = lane; i < m * pieces; i += 32) {
                    const int r = i / pieces, p = i - r * pieces;
                    reinterpret_cast<uint4 *>(s_row + r * d)[p] = *(reinterpret_cast<const uint4 *>(x0 + rows[r] * x_stride) + h * pieces + p);
                }
                __syncwarp();
                for (int i = lane; i < m * pieces; i += 32) {
                    const int r = i / pieces, p = i - r * pieces;
                    const uint4 own = reinterpret_cast<const uint4 *>(s_row + r * d)[p];
                    float x[N];
                    Piece<T>::widen(own, x);
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
                        x[e] = fmaf(x[e], a.x, o * (low ? -a.y : a.y));
                    }
                    *(reinterpret_cast<uint4 *>(y0 + rows[r] * y_stride) + h * pieces + p) = keep_tail<N>(Piece<T>::narrow(x), own, rot - p * N);
                }
                __syncwarp();
            }
        }
    } else {
        const int lanes = min(pieces, 32), side = lane / lanes, beside = 32 / lanes;       // of a head; the lane's row of `beside`
        const int both = MODE == HALF_LANES ? half / N : 0, head_bytes = pieces * 16;
        for (int part = 0; part < pieces; part += 32) {
            const int piece = part + lane - side * lanes;
            const bool mine = side < beside && piece < pieces;
            const bool low = piece < both;
            // what this lane's pairs turn by per position (pairs behind the last: nothing), and whose
            uint64_t f[NP];
            int axis[NP];
            const int first = MODE == HALF_LANES ? (low ? piece : piece - both) * N : piece * NP;
#pragma unroll
            for (int e = 0; e < NP; ++e) {
                const int p = first + e < half ? first + e : ROPE_PAIRS - 1;
                f[e] = first + e < half ? s_f[p] : 0ull;
                axis[e] = s_axis[p];
            }
            const uint32_t flip = low ? 0x80000000u : 0u;
            const int from = MODE == HALF_LANES ? (low ? lane + both : lane - both) : 0, tail = rot - piece * N;
            // this lane's row of some rows side by side (a lane without one: the last, whose results it keeps to itself)
            int r = min(side, n_kept - 1);
            bool here = mine && side < n_kept;
            const uint8_t *x = x0 + s_rows[warp][r] * x_stride + (mine ? piece * 16 : 0);
            uint4 v[ROPE_FLIGHT];
#pragma unroll
            for (int i = 0; i < ROPE_FLIGHT; ++i)
                if (i < H) v[i] = __ldcs(reinterpret_cast<const uint4 *>(x + i * head_bytes));
            for (int r0 = 0; r0 < n_kept; r0 += beside) {
                uint8_t *y = y0 + s_rows[warp][r] * y_stride + (mine ? piece * 16 : 0);
                float c[NP], g[NP];
                const int32_t *at = s_pos[warp][r];
#pragma unroll
                for (int e = 0; e < NP; e += 2)
                    cos_sin_two(turn_of(at[axis[e]], f[e]), turn_of(at[axis[e + 1]], f[e + 1]), turns.magnitude, flip, c + e, g + e);
                // the next rows'
                const bool store = here;
                const int rn = r0 + beside + side;
                r = min(rn, n_kept - 1);
                here = mine && rn < n_kept;
                const uint8_t *xn = x0 + s_rows[warp][r] * x_stride + (mine ? piece * 16 : 0);
                const bool more = r0 + beside < n_kept;
                for (int h0 = 0; h0 < H; h0 += ROPE_FLIGHT) {
#pragma unroll
                    for (int i = 0; i < ROPE_FLIGHT; ++i) {
                        const int h = h0 + i;
                        if (h >= H) break;                 // (uniform: the exchange names all lanes)
                        const uint4 own = v[i];
                        // the place's next piece: of a later head, or of the next rows
                        if (h + ROPE_FLIGHT < H) v[i] = __ldcs(reinterpret_cast<const uint4 *>(x + (h + ROPE_FLIGHT) * (int64_t)head_bytes));
                        else if (more) v[i] = __ldcs(reinterpret_cast<const uint4 *>(xn + i * (int64_t)head_bytes));
                        float a[N];
                        Piece<T>::widen(own, a);
                        if constexpr (MODE == HALF_LANES) {
                            const uint4 w = make_uint4(__shfl_sync(0xffffffffu, own.x, from), __shfl_sync(0xffffffffu, own.y, from),
                                                       __shfl_sync(0xffffffffu, own.z, from), __shfl_sync(0xffffffffu, own.w, from));
                            float z[N];
                            Piece<T>::widen(w, z);
#pragma unroll
                            for (int e = 0; e < N; e += 2)
                                split_pair(fma_pair(pair_of(a[e], a[e + 1]), pair_of(c[e], c[e + 1]), mul_pair(pair_of(z[e], z[e + 1]), pair_of(g[e], g[e + 1]))),
                                           a[e], a[e + 1]);
                        } else {
#pragma unroll
                            for (int e = 0; e < N; e += 2) {
                                const float a0 = a[e], a1 = a[e + 1];
                                a[e] = fmaf(a0, c[e / 2], -(a1 * g[e / 2]));
                                a[e + 1] = fmaf(a0, g[e / 2], a1 * c[e / 2]);
                            }
                        }
                        if (store) *reinterpret_cast<uint4 *>(y + h * (int64_t)head_bytes) = keep_tail<N>(Piece<T>::narrow(a), own, tail);
                    }
                }
                x = xn;
            }
        }
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
        const uint32_t t = turn_of(__ldg(pos + r * turns.axes + s_axis[p]), s_f[p]);
        float c[2], g[2];
        cos_sin_two(t, t, turns.magnitude, 0u, c, g);
        out[i] = make_float2(c[0], g[0]);
    }
}

// A number as the sum of two doubles, the second at most half a last place of the first: some 100 bits.  Sums and products by
// the error-free transformations of Knuth and Dekker (the product's with a fused multiply-add).
struct Two {
    double hi, lo;
};

Two two_sum(double a, double b)
{
    const double s = a + b, v = s - a;
    return {s, (a - (s - v)) + (b - v)};
}

Two operator+(Two a, Two b)
{
    const Two s = two_sum(a.hi, b.hi);
    return two_sum(s.hi, s.lo + (a.lo + b.lo));
}

Two operator-(Two a, Two b) { return a + Two{-b.hi, -b.lo}; }

Two operator*(Two a, Two b)
{
    const double p = a.hi * b.hi, e = std::fma(a.hi, b.hi, -p);
    return two_sum(p, e + (a.hi * b.lo + a.lo * b.hi));
}

Two operator/(Two a, Two b)
{
    const double q = a.hi / b.hi;
    const Two r = a - b * Two{q, 0.0};
    const double c = r.hi / b.hi;
    return two_sum(q, c) + Two{(r - b * Two{c, 0.0}).hi / b.hi, 0.0};
}

Two power(Two x, int n)
{
    Two y = {1.0, 0.0};
    for (; n > 0; n >>= 1, x = x * x)
        if (n & 1) y = y * x;
    return y;
}

// base^(-1/n): a step of Newton's iteration from the value in one double, whose error of 2^-52 or so it squares.
Two root_of(double base, int n)
{
    const double r = std::pow(base, -1.0 / n);
    const Two off = power({r, 0.0}, n) * Two{base, 0.0} - Two{1.0, 0.0};
    return two_sum(r, -r * off.hi / n);
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
    const Two per_turn = {0x1.45f306dc9c883p-3, -0x1.6b01ec5417056p-57};       // 1 / (2 pi)
    const Two one = {1.0, 0.0}, slow = {s->beta_slow, 0.0}, part = one / Two{s->factor, 0.0};
    const Two ramp = two_sum(s->beta_fast, -s->beta_slow), slope = s->context > 0.0 ? one / ramp : one;
    int p = 0;
    for (int a = 0; a < s->axes; ++a) {
        const Two step = s->pairs[a] > 1 ? root_of(s->base, s->pairs[a]) : one;
        Two f = per_turn;                                  // pair i: base^(-i/n) / (2 pi)
        for (int i = 0; i < s->pairs[a]; ++i, ++p, f = f * step) {
            Two turn = f * part;
            if (s->context > 0.0) {
                const Two up = f * Two{s->context, 0.0} - slow, share = up * slope;       // of the frequency as trained
                if (up.hi >= ramp.hi) turn = f;            // (a ramp may be too short for its slope)
                else if (up.hi > 0.0) turn = f * share + turn * (one - share);
            }
            // (below 2^62, and what lies behind its whole number within some hundreds)
            const double hi = turn.hi * 0x1p64;
            const int64_t whole = (int64_t)hi;
            const double rest = turn.lo * 0x1p64 + (hi - (double)whole);
            t.f[p] = (uint64_t)(whole + (int64_t)(rest < 0.0 ? rest - 0.5 : rest + 0.5));
            if (s->inverse) t.f[p] = 0 - t.f[p];
            t.axis[p] = (uint8_t)a;
        }
    }
    t.half = s->rot / 2;
    t.axes = s->axes;
    t.magnitude = s->magnitude;
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
        r.chunk = chunk;
        r.chunks = (r.rows + chunk - 1) / chunk;
        total += r.chunks;
    }
    if (total == 0) return RS3_OK;
    const int64_t ctas = (total + ROPE_WARPS - 1) / ROPE_WARPS;
    if (ctas > INT32_MAX) return RS3_EUNSUPPORTED;
    const int pieces = d / n;
    const RopeMode mode = spec->layout == RS3_ROPE_PAIRS ? PAIR_LANES : t.half % n == 0 && pieces <= 32 ? HALF_LANES : HALF_COPY;
    size_t smem = 0;
    if (mode == HALF_COPY) smem = ROPE_WARPS * (align_up((size_t)ROPE_COPIES * d * esz, 16) + align_up((size_t)ROPE_COPIES * t.half * 8, 16));
    using Kern = void (*)(RopeSide, RopeSide, RopeTurns, int);
    Kern kern;
    if (dtype == RS3_BF16)
        kern = mode == PAIR_LANES ? k_rope_rows<uint16_t, PAIR_LANES> : mode == HALF_LANES ? k_rope_rows<uint16_t, HALF_LANES> : k_rope_rows<uint16_t, HALF_COPY>;
    else
        kern = mode == PAIR_LANES ? k_rope_rows<float, PAIR_LANES> : mode == HALF_LANES ? k_rope_rows<float, HALF_LANES> : k_rope_rows<float, HALF_COPY>;
    // (beside up to 8 KB that the kernel has anyhow)
    if (rs3_kernel_smem((const void *)kern, smem + 8192) != RS3_OK) return RS3_ECUDA;
    launch_pdl(kern, dim3((unsigned)ctas), dim3(ROPE_WARPS * 32), smem, reinterpret_cast<cudaStream_t>(stream), s[0], s[1], t, d);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
