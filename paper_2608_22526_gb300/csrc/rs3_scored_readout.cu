// rs3_scored_readout.cu -- readout over the rows of chosen frames, with scores that are capped by a
// tanh and biased by their row's frame:
//
//   s = scale q~.k;  s = cap tanh(s / cap);  s = s + bias[u][h][frame(row)];  softmax, V
//
// A frame that is left out costs nothing: its rows lie in no key tile.  Launches:
//   k_frames       a CTA per unit: frames that are read and follow one another make runs of storage
//                  rows (cut at the ring's end), the runs make a table of key tiles; with biases,
//                  other CTAs write each row's frame beside it; out of place, one more a bit per kept cell
//   k_plan, k_readout_*, k_combine   the readout's, over the table
// The kernels are the readout's own with a score's change compiled in.  The key producer's warp looks
// the biases of a tile's rows up ahead (tile, frames, biases, a turn of its loop each) and leaves them beside K.
// Scores that a cap of 55 or less bounds need no running maximum (RS3_BOUNDED): weights are taken against the largest bias
// so far, the same for all rows, and cap and power are one pass.  V rows of a tile that belong to no
// live row are zeroed in shared memory, so that nothing comes of what they hold.  Eight objects of one 64 x 64 grid
// (7 frames, heads of 256, 46 GFLOP), in place: 68 us capped and biased, 65 capped, 66 biased, 59 with neither (the
// plain readout 58); 174 000 of 302 000 rows of a video after a cut: 127 us, 200 over all rows.
#include "rs3_readout_common.cuh"
#include "rs3_bank.cuh"

#include <algorithm>
#include <cmath>

namespace {

struct Stretch { int64_t x, y; };

struct FramesArgs {
    BankDev bank;
    const uint8_t *keep;        // [U][F + 2] or NULL
    int32_t *tile_n;            // [tables][U]; -1: counters or frames that are unsound
    Stretch *stretch;           // [tables][U][F] first and end ring position of frames that are read and follow one another
    int4 *runs;                 // [tables][U][F + 4] storage rows of those and of the other regions: (first row, rows, first tile)
    int2 *tiles;                // [tables][U][tile_stride]
    int32_t *row_frame;         // [U][rows_per_unit], or NULL without biases
    int tile_stride, U, tables, row_ctas;
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

__device__ void unit_tiles(const FramesArgs &f, int u, int table)
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
__device__ void unit_rows(const FramesArgs &f, int u, int warp, int warps)
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

__device__ void unit_kept(const FramesArgs &f, int u)
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

__global__ void __launch_bounds__(FRAMES_THREADS) k_frames(const __grid_constant__ FramesArgs f)
{
    pdl_wait();
    const int u = blockIdx.y;
    const int x = (int)blockIdx.x - f.tables;
    if (x < 0) unit_tiles(f, u, (int)blockIdx.x);
    else if (x < f.row_ctas) unit_rows(f, u, x * (FRAMES_THREADS / 32) + ((int)threadIdx.x >> 5), f.row_ctas * (FRAMES_THREADS / 32));
    else unit_kept(f, u);
}

// Byte offsets in the workspace.
struct ScoredLayout {
    ReadoutPath path;
    ReadoutLayout l;
    size_t stretch, runs, tiles, rows, kept, ws, total;
    int64_t tile_stride;
    int words;                  // of 32 cells
    int tables;                 // of key tiles: where a head's two kernels have tiles of different rows, two
};

ReadoutPath scored_path(const rs3_bank *bank, int k_max)
{
    return choose_readout_path((rs3_dtype)bank->dtype, bank->d, bank->U, bank->H, k_max, bank->rows_per_unit, SIZE_MAX);
}

ScoredLayout scored_layout(const rs3_bank *bank, int k_max, const ReadoutPath &path)
{
    const int U = bank->U, F = bank->max_frames;
    ScoredLayout L;
    L.path = path;
    L.tables = L.path.either && L.path.BN != 128 ? 2 : 1;
    const size_t n = (size_t)U * L.tables;
    L.l = rs3_readout_layout(U, bank->H, bank->d, k_max, L.path, false);
    L.tile_stride = bank->rows_per_unit / L.path.BN + F + 4;       // whole tiles, and a part at each run's end
    size_t off = align_up(n * 4, 256);
    L.stretch = off;
    off = align_up(off + n * F * 16, 256);
    L.runs = off;
    off = align_up(off + n * (F + 4) * 16, 256);
    L.tiles = off;
    off = align_up(off + n * L.tile_stride * 8, 256);
    L.rows = off;
    off = align_up(off + (size_t)U * bank->rows_per_unit * 4, 256);
    L.kept = off;
    L.words = (bank->mn + 31) / 32;
    if (L.path.either) off = align_up(off + (size_t)U * L.words * 4, 256);
    L.ws = off;
    L.total = off + L.l.total;
    return L;
}

}  // namespace

extern "C" size_t rs3_scored_readout_workspace_bytes(const rs3_bank *bank, int k_max)
{
    if (!bank || bank->magic != RS3_BANK_MAGIC || k_max < 0) return 0;
    const ReadoutPath p = scored_path(bank, k_max);        // (a call of fewer queries may take the other one)
    const size_t n = scored_layout(bank, k_max, p).total;
    return p.kind == 0 ? std::max(n, scored_layout(bank, k_max, rs3_few_rows(p, bank->d)).total) : n;
}

extern "C" rs3_status rs3_scored_readout(const void *q, rs3_dtype dtype, int G, int mn, int H, int d, const int32_t *unit_group,
                                         const int32_t *idx, const int32_t *count, int k_max, const rs3_bank *bank, float cap,
                                         const float *frame_bias, int64_t bias_stride, const uint8_t *frame_keep, const float *rope,
                                         const void *residual, void *out, float scale, void *workspace, size_t workspace_bytes,
                                         int32_t *status, rs3_stream_t stream)
{
    rs3_status s = rs3_readout_check(q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, residual, out, workspace, status);
    if (s != RS3_OK) return s;
    if (!(cap == 0.f || (cap >= 0x1p-10f && cap <= 0x1p10f))) return RS3_EINVAL;
    const int F = bank->max_frames;
    if (frame_bias && ((reinterpret_cast<uintptr_t>(frame_bias) & 3u) || (bias_stride != 0 && bias_stride < (int64_t)H * (F + 2)))) return RS3_EINVAL;
    if ((int64_t)bank->U * bank->rows_per_unit >= (int64_t)1 << 31) return RS3_EUNSUPPORTED;
    ReadoutPath path = scored_path(bank, k_max);
    if (!rs3_readout_fits(bank->U, H, k_max, path)) return RS3_EUNSUPPORTED;
    if (workspace_bytes < rs3_scored_readout_workspace_bytes(bank, k_max)) return RS3_ECAPACITY;
    if (rs3_has_few_rows(path, bank->U, H, d, k_max, bank->rows_per_unit)) path = rs3_few_rows(path, d);
    const ScoredLayout L = scored_layout(bank, k_max, path);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    FramesArgs f = {};
    f.bank = bank_dev(bank);
    f.keep = frame_keep;
    f.tile_n = reinterpret_cast<int32_t *>(ws);
    f.stretch = reinterpret_cast<Stretch *>(ws + L.stretch);
    f.runs = reinterpret_cast<int4 *>(ws + L.runs);
    f.tiles = reinterpret_cast<int2 *>(ws + L.tiles);
    f.row_frame = frame_bias ? reinterpret_cast<int32_t *>(ws + L.rows) : nullptr;
    f.tile_stride = (int)L.tile_stride;
    f.U = bank->U;
    f.tables = L.tables;
    f.BN[0] = L.path.BN;
    f.BN[1] = 128;
    ReadoutMore a = {};
    rs3_readout_fill(&a, L.path, L.l, ws + L.ws, q, G, mn, H, d, unit_group, idx, count, k_max, bank->U, bank, rope, residual, out, scale,
                     status);
    a.score.tile_n = f.tile_n;
    a.score.tiles = f.tiles;
    a.score.pair_tile_n = f.tile_n + (L.tables - 1) * (int64_t)bank->U;
    a.score.pair_tiles = f.tiles + (L.tables - 1) * (int64_t)bank->U * L.tile_stride;
    a.score.row_frame = f.row_frame;
    a.score.bias = frame_bias;
    a.score.bias_stride = bias_stride;
    a.score.tile_stride = f.tile_stride;
    a.score.frames = F + 2;
    const float log2e = 1.4426950408889634f;
    a.score.cap = cap * log2e;
    a.score.bounded = cap > 0.f && a.score.cap <= RS3_BOUNDED;
    // tensor cores: of a raw score, for e^2x; CUDA cores: of one in the log2 domain, for tanh itself
    if (cap > 0.f) a.score.cap_step = L.path.kind == 1 ? 2.f * a.scale_log2 / cap : 1.f / a.score.cap;
    if (cap > 0.f) {
        // tanh(x) / x in x^2 with the least largest relative error over 0 < x <= 1/2 (alternation points found in 64
        // bits): 5.4e-7, with its roundings 6.2e-7
        static const double poly[4] = {0.99999945577, -0.33326317936, 0.13190296603, -0.04440222613};
        const double unit = (double)a.scale_log2 / a.score.cap;
        a.score.cap_half = (float)(0.5 / unit);
        double by = unit * a.score.cap;
        for (int i = 0; i < 4; ++i, by *= unit * unit) {
            a.score.cap_poly[i] = (float)(poly[i] * by);
            if (!(std::fabs(a.score.cap_poly[i]) > 1e-30f && std::fabs(a.score.cap_poly[i]) < 1e30f)) a.score.cap_half = -1.f;   // out of range: never
        }
    }
    // Out of place, calls of much work leave the cells that are not kept to a warp that the attention has to spare,
    // and what that has not reached to the merge (48 objects of 96 x 96 cells, 453 MB: 1 137 us, 1 187 where the
    // plan's launch passes them through)
    if (L.path.either && residual != out && mn == bank->mn) {
        f.kept = reinterpret_cast<uint32_t *>(ws + L.kept);
        a.kept = f.kept;
        a.words = L.words;
    }
    f.idx = idx;
    f.count = count;
    f.k_max = k_max;
    f.mn = mn;
    f.words = L.words;
    f.row_ctas = frame_bias ? std::min((F + COND_PIECES + 1 + 7) / 8, 32) : 0;
    launch_pdl(k_frames, dim3((unsigned)(L.tables + f.row_ctas + (f.kept ? 1 : 0)), (unsigned)bank->U), dim3(FRAMES_THREADS), 0, st, f);
    if (cudaGetLastError() != cudaSuccess) return RS3_ECUDA;
    return rs3_scored_launch(a, L.path, L.l.max_combine, dtype, st);
}
