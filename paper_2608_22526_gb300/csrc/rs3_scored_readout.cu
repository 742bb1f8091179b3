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
// One unit's frames are gone through in the plan's launch (k_plan_one, rs3_readout.cu).
// The kernels are the readout's own with a score's change compiled in.  The key producer's warp looks
// the biases of a tile's rows up ahead (tile, frames, biases, a turn of its loop each) and leaves them beside K.
// Scores that a cap of 55 or less bounds need no running maximum (RS3_BOUNDED): weights are taken against the largest bias
// so far, the same for all rows, and cap and power are one pass.  V rows of a tile that belong to no
// live row are zeroed in shared memory, so that nothing comes of what they hold.  Eight objects of one 64 x 64 grid
// (7 frames, heads of 256, 46 GFLOP), in place, the call alone: 68 us capped and biased, 65 capped, 63 to 72 biased (as
// biases move the running maximum), 59 with neither (the plain readout 57); 174 000 of 302 000 rows of a video after a
// cut: 125 us, 194 over all rows.
#include "rs3_frames.cuh"

#include <algorithm>
#include <cmath>

namespace {

using namespace frames;

__global__ void __launch_bounds__(FRAMES_THREADS) k_frames(const __grid_constant__ FramesArgs f)
{
    pdl_wait();
    const int x = (int)blockIdx.x - f.tables;
    if (x < 0) unit_tiles(f, blockIdx.y, (int)blockIdx.x);
    else unit_rest(f, blockIdx.y, x);
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
    const size_t few = p.kind == 0 ? scored_layout(bank, k_max, rs3_few_rows(p, bank->d)).total : 0;
    return few && rs3_always_few_rows(bank->d) ? few : std::max(few, scored_layout(bank, k_max, p).total);
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
    // and what that has not reached to the merge (48 objects of 96 x 96 cells, 453 MB: 45 us less than where the
    // plan's launch passes them through, 1 158 us then)
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
    f.rest_ctas = f.row_ctas + (f.kept ? 1 : 0);
    // (one unit's tiles are the plan's own CTA's first work)
    if (bank->U == 1) return rs3_scored_launch(a, &f, L.path, L.l.max_combine, dtype, st);
    launch_pdl(k_frames, dim3((unsigned)(L.tables + f.rest_ctas), (unsigned)bank->U), dim3(FRAMES_THREADS), 0, st, f);
    if (cudaGetLastError() != cudaSuccess) return RS3_ECUDA;
    return rs3_scored_launch(a, nullptr, L.path, L.l.max_combine, dtype, st);
}
