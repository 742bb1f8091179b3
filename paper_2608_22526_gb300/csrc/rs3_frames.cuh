// rs3_frames.cuh -- the frames of a scored readout (rs3_scored_readout.cu): key tiles of those that are
// read, each row's frame, and a bit for each kept cell.
#pragma once

#include "rs3_readout_common.cuh"
#include "rs3_bank.cuh"

namespace frames {

struct Stretch { int64_t x, y; };

struct FramesArgs {
    BankDev bank;
    const uint8_t *keep;        // [U][F + 2] or NULL
    int32_t *tile_n;            // [tables][U]; -1: counters or frames that are unsound
    Stretch *stretch;           // [tables][U][F] first and end ring position of frames that are read and follow one another
    int4 *runs;                 // [tables][U][F + 4] storage rows of those and of the other regions: (first row, rows, first tile)
    int2 *tiles;                // [tables][U][tile_stride]
    int32_t *row_frame;         // [U][rows_per_unit], or NULL without biases
    int tile_stride, U, tables, row_ctas, rest_ctas;   // CTAs of a unit that write rows' frames; those that make no tables
    int BN[2];                  // rows of a tile, of either table
    const int32_t *idx, *count; // kept queries [U][k_max]
    uint32_t *kept;             // [U][words] a bit for each of their cells, or NULL
    int k_max, mn, words;
};

constexpr int FRAMES_THREADS = 256;
constexpr int COND_PIECES = 16;            // parts that the pinned rows are written in

// Exclusive sums of two numbers over the CTA's threads, and their totals.
__device__ __forceinline__ void scan_two(int &a, int &b, int &all_a, int &all_b)
{
    __shared__ int s_a[FRAMES_THREADS / 32], s_b[FRAMES_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, a0 = a, b0 = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) { a += x; b += y; }
    }
    __syncthreads();                                       // the sums before have been read
    if (lane == 31) { s_a[warp] = a; s_b[warp] = b; }
    __syncthreads();
    a -= a0;
    b -= b0;
    all_a = all_b = 0;
#pragma unroll
    for (int w = 0; w < FRAMES_THREADS / 32; ++w) {
        if (w < warp) { a += s_a[w]; b += s_b[w]; }
        all_a += s_a[w];
        all_b += s_b[w];
    }
}

// A unit's frames: their ring positions, whether they are read.
struct UnitFrames {
    const int64_t *off, *len;
    const uint8_t *keep;
    int64_t head, tail, cond, ptr;
    int n, oldest, F;
    __device__ __forceinline__ bool load(const BankDev &b, const uint8_t *keep_all, int64_t u)
    {
        const int64_t *mu = b.meta + u * b.stride_words;
        head = mu[BM_HEAD];
        tail = mu[BM_TAIL];
        cond = mu[BM_COND_LEN];
        ptr = mu[BM_PTRLEN];
        const int64_t frames = mu[BM_NFRAMES], first = mu[BM_OLDEST];
        F = b.max_frames;
        off = mu + BM_HEADER_WORDS;
        len = off + F;
        keep = keep_all ? keep_all + u * (F + 2) : nullptr;
        if (!(head >= 0 && tail >= head && tail - head <= b.ring_cap && cond >= 0 && cond <= b.pinned_cap && ptr >= 0 && ptr <= b.n_ptr &&
              frames >= 0 && frames <= F && (frames == 0 || (first >= 0 && first < F))))
            return false;
        n = (int)frames;
        oldest = (int)first;
        return true;
    }
    // The frames in their order fill [head, tail) without gap or overlap: of the i-th oldest, it begins where
    // the one before it ends (the first at the head), and the last ends at the tail.
    __device__ __forceinline__ bool follows(int i) const
    {
        const int s = oldest + i < F ? oldest + i : oldest + i - F, before = s > 0 ? s - 1 : F - 1;
        const int64_t a = off[s], l = len[s], from = i == 0 ? head : off[before] + len[before];
        return a == from && a >= head && a <= tail && l >= 0 && l <= tail - a && (i + 1 < n || l == tail - a);
    }
    // of the i-th oldest frame
    __device__ __forceinline__ bool read(int i) const { return !keep || keep[n - 1 - i] != 0; }
    __device__ __forceinline__ void span(int i, int64_t &a, int64_t &e) const
    {
        const int s = oldest + i < F ? oldest + i : oldest + i - F;
        a = min(max(off[s], head), tail);
        e = min(max(off[s] + len[s], a), tail);
    }
    __device__ __forceinline__ bool cond_read() const { return !keep || keep[F] != 0; }
    __device__ __forceinline__ bool ptr_read() const { return !keep || keep[F + 1] != 0; }
};

static __device__ void unit_tiles(const FramesArgs &f, int u, int table)
{
    const BankDev &b = f.bank;
    const int BN = f.BN[table];
    const int64_t slot = (int64_t)table * f.U + u;
    UnitFrames x;
    if (!x.load(b, f.keep, u)) {                           // (the plan latches it)
        if (threadIdx.x == 0) f.tile_n[slot] = -1;
        return;
    }
    Stretch *stretch = f.stretch + slot * x.F;
    int4 *runs = f.runs + slot * (x.F + 4);
    // stretches of frames that are read: the first frame of one writes where it begins, the last where it ends
    int n_str = 0;
    bool gap = x.n == 0 && x.head != x.tail;
    for (int i0 = 0; i0 < x.n; i0 += FRAMES_THREADS) {
        const int i = i0 + threadIdx.x;
        gap = gap || (i < x.n && !x.follows(i));
        const bool on = i < x.n && x.read(i), begins = on && (i == 0 || !x.read(i - 1)), ends = on && (i == x.n - 1 || !x.read(i + 1));
        int before = begins, none = 0, all, zero;
        scan_two(before, none, all, zero);
        if (on && (begins || ends)) {
            const int k = n_str + before + (begins ? 1 : 0) - 1;
            int64_t a, e;
            x.span(i, a, e);
            if (begins) stretch[k].x = a;
            if (ends) stretch[k].y = e;
        }
        n_str += all;
    }
    // (the tables hold frames that fill the ring's rows, no more, and rows between frames have no bias)
    if (__syncthreads_or(gap)) {
        if (threadIdx.x == 0) f.tile_n[slot] = -1;
        return;
    }
    // runs of storage rows: the pinned ones, the stretches (cut at the ring's end), the pointers
    int n_runs = 0, n_tiles = 0;
    const int sh = 31 - __clz(BN);
    for (int k0 = 0; k0 < n_str + 2; k0 += FRAMES_THREADS) {
        const int k = k0 + threadIdx.x;
        int64_t row[2] = {0, 0}, len[2] = {0, 0};
        if (k == 0) {
            len[0] = x.cond_read() ? x.cond : 0;
        } else if (k == n_str + 1) {
            row[0] = b.pinned_cap + b.ring_cap;
            len[0] = x.ptr_read() ? x.ptr : 0;
        } else if (k < n_str + 1) {
            const Stretch s = stretch[k - 1];
            if (s.y > s.x) {
                const int64_t p0 = s.x % b.ring_cap;       // rows are held, so ring_cap > 0
                row[0] = b.pinned_cap + p0;
                len[0] = min(s.y - s.x, b.ring_cap - p0);
                row[1] = b.pinned_cap;
                len[1] = s.y - s.x - len[0];
            }
        }
        const int t0 = (int)((len[0] + BN - 1) >> sh), t1 = (int)((len[1] + BN - 1) >> sh);
        int r = (t0 > 0) + (t1 > 0), t = t0 + t1, all_r, all_t;
        scan_two(r, t, all_r, all_t);
        r += n_runs;
        t += n_tiles;
        if (t0 > 0) runs[r++] = make_int4((int)row[0], (int)len[0], t, 0);
        if (t1 > 0) runs[r] = make_int4((int)row[1], (int)len[1], t + t0, 0);
        n_runs += all_r;
        n_tiles += all_t;
    }
    if (threadIdx.x == 0) f.tile_n[slot] = n_tiles;
    __syncthreads();
    int2 *tiles = f.tiles + slot * f.tile_stride;
    for (int t = threadIdx.x; t < n_tiles; t += FRAMES_THREADS) {
        int lo = 0, hi = n_runs;                           // the last run that begins at or before tile t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (runs[mid].z <= t) lo = mid; else hi = mid;
        }
        const int4 r = runs[lo];
        const int at = (t - r.z) << sh;
        tiles[t] = make_int2(r.x + at, min(BN, r.y - at));
    }
}

// A warp writes the frames of a ring frame's rows, or of a part of the pinned rows, or of the pointers.
static __device__ void unit_rows(const FramesArgs &f, int u, int warp, int warps)
{
    const BankDev &b = f.bank;
    UnitFrames x;
    if (!x.load(b, f.keep, u)) return;
    const int lane = threadIdx.x & 31;
    int32_t *out = f.row_frame + (int64_t)u * b.rows_per_unit;
    for (int i = warp; i < x.n + COND_PIECES + 1; i += warps) {
        if (i < x.n) {
            int64_t a, e;
            x.span(i, a, e);
            if (e <= a || !x.read(i)) continue;
            int64_t p = b.pinned_cap + a % b.ring_cap;
            const int64_t end = b.pinned_cap + b.ring_cap;
            for (int64_t r = a + lane; r < e; r += 32) {
                const int64_t at = p + (r - a);
                out[at < end ? at : at - b.ring_cap] = x.n - 1 - i;
            }
        } else if (i < x.n + COND_PIECES) {
            const int64_t per = (x.cond + COND_PIECES - 1) / COND_PIECES, a = per * (i - x.n), e = min(a + per, x.cond);
            for (int64_t r = a + lane; r < e; r += 32) out[r] = x.F;
        } else {
            for (int64_t r = lane; r < x.ptr; r += 32) out[b.pinned_cap + b.ring_cap + r] = x.F + 1;
        }
    }
}

static __device__ void unit_kept(const FramesArgs &f, int u)
{
    __shared__ uint32_t s_bits[RS3_MAX_MN / 32];
    for (int w = threadIdx.x; w < f.words; w += FRAMES_THREADS) s_bits[w] = 0u;
    __syncthreads();
    const int n = f.count[u];
    for (int j = threadIdx.x; j < n && n <= f.k_max; j += FRAMES_THREADS) {
        const int cell = __ldg(f.idx + (int64_t)u * f.k_max + j);
        if (cell >= 0 && cell < f.mn) atomicOr(&s_bits[cell >> 5], 1u << (cell & 31));
    }
    __syncthreads();
    for (int w = threadIdx.x; w < f.words; w += FRAMES_THREADS) f.kept[(int64_t)u * f.words + w] = s_bits[w];
}

// What CTA x of a unit does, the first f.tables of them apart (unit_tiles).
__device__ __forceinline__ void unit_rest(const FramesArgs &f, int u, int x)
{
    if (x < f.row_ctas) unit_rows(f, u, x * (FRAMES_THREADS / 32) + ((int)threadIdx.x >> 5), f.row_ctas * (FRAMES_THREADS / 32));
    else unit_kept(f, u);
}

}  // namespace frames
