// rs3_readout_common.cuh -- argument block and helpers shared by the readout
// kernels (CUDA-core and tensor-core paths).
#pragma once

#include "rs3_internal.cuh"

#define RS3_MAX_UNITS 4096  // units per readout call
#define RS3_PAIR_ITEMS (1 << 30)   // above every item index
// Scores in the log2 domain whose weights 2^s can be summed as they are: 2^80, the 2^8 that biases may rise by before the
// reference follows, a million of them and values up to 2^18 stay within fp32's (and bf16's) 2^127, and 2^-80 leaves 2^-46 to values.
#define RS3_BOUNDED 80.f

struct GroupParts {         // a group's n pieces: 0 is in slot0, s >= 1 in slot 2 (slice + s); whose they are
    int32_t slot0, slice, n, u, h, qt;
    int32_t cnt, pad;       // kept queries of the unit
};

// Scores changed by their row's frame (rs3_scored_readout).
struct ScoreArgs {
    const int32_t *tile_n;      // [U] key tiles of rows that are read; NULL: the readout's own tiles
    const int2 *tiles;          // [U][tile_stride] first row (in the unit's storage) and rows of each
    const int32_t *pair_tile_n; // the same for the kernel with two query tiles
    const int2 *pair_tiles;
    const int32_t *row_frame;   // [U][rows_per_unit] entry of the bias table of each live row (where there is a table)
    const float *bias;          // [H][frames], bias_stride elements between units
    int64_t bias_stride;
    int tile_stride, frames;
    int bounded;                // the cap holds scores within 2^+-RS3_BOUNDED: weights need no reference beside the biases'
    float cap;                  // cap * log2(e)
    float cap_step;             // 2 log2(e) scale / cap: tanh(x) = 1 - 2 / (1 + e^2x)
    float cap_half;             // raw scores up to here have |x| <= 1/2, where the polynomial holds
    float cap_poly[4];          // cap * log2(e) * tanh(x) / raw score, by powers of the raw score's square
};

// A frame's bias in the log2 domain; one below any that a score could show beside counts as minus infinity.
__device__ __forceinline__ float log2_bias(float b) { return b < -1e30f ? -INFINITY : b * 1.4426950408889634f; }

// What a readout kernel does to a score: nothing, or a cap and a bias by the row's frame.
struct PlainScores {
    static constexpr bool on = false, cap = false, bias = false;
};
template <bool CAP, bool BIAS>
struct FrameScores {
    static constexpr bool on = true, cap = CAP, bias = BIAS;
};

struct ReadoutArgs {
    const void *q;
    const void *k_store;
    const void *v_store;
    const int64_t *meta;
    int64_t meta_stride_words;
    int64_t pinned_cap, ring_cap, rows_per_unit;
    int64_t n_ptr;
    const int32_t *unit_group;
    const int32_t *idx;
    const int32_t *count;
    const float *rope;
    const void *residual;
    void *out;
    int32_t *status;
    int U, G, mn, H, d, D, k_max;
    int BM, BN, n_sm, min_chunk;
    int plan_ov;            // leading plan slots per group: a piece's start-up cost in tiles
    int either;             // the plan may take the two-tile kernel (the four above are the one-tile kernel's)
    int tensor;             // a tensor-core kernel runs the plan
    int64_t max_slots;
    int grid_ctas;          // CTAs of the readout launch (the plan's slice count bound)
    int32_t *cta_items;     // [grid_ctas][2]: CTA b runs items [cta_items[2b], cta_items[2b+1]); the first
                            // of the two with RS3_PAIR_ITEMS where they are for the two-tile kernel
    float scale_log2;       // softmax scale * log2(e)
    uint64_t wait_ns;       // limit of each device-side wait (global-timer ns)
    ReadoutHeader *header;
    RangeSet *ranges;
    WorkItem *items;
    CombineItem *combine;
    float *part_o;          // [slot][BM][d]
    float *part_ml;         // [slot][BM] (m, l) pairs, m in the log2 domain
    int bank_U;             // units of the bank
};

// The arguments of the calls whose plan or scores are not the plain readout's.
struct ReadoutMore : ReadoutArgs {
    // units that read units of a bank by number, and leave all results in partial slots
    const int32_t *bank_unit;   // [U] the bank's unit that unit u reads (-1: none); NULL: unit u
    GroupParts *parts;          // [group] its pieces (groups numbered as the plan does); NULL: whole groups are written out
    // cells that are not kept are passed through (out = residual, or zeros) beside the attention and behind it, not by
    // the plan's launch: a bit for each kept cell, 32 to a word, [U][words].  NULL: by the plan's launch
    const uint32_t *kept;
    int words;
    // changed scores (counts and cells that are out of range are skipped, not taken for others)
    ScoreArgs score;
};

// What is left of the pass-through of rows of bf16, by one warp, 32 cells of a unit at a time.
__device__ __forceinline__ void pass_cells(const ReadoutMore &a)
{
    constexpr int F = 8;                                    // 16-byte pieces of a lane under way
    const int lane = threadIdx.x & 31, n = a.U * a.words, vecs = a.D / 8;
    const uint4 *res = static_cast<const uint4 *>(a.residual);
    uint4 *out = static_cast<uint4 *>(a.out);
    while (true) {
        int c = n;
        // (mostly nothing is: thousands of warps would wait for one another's sums)
        if (lane == 0 && __ldcg(&a.header->passed) < n) c = atomicAdd(&a.header->passed, 1);
        c = __shfl_sync(0xffffffffu, c, 0);
        if (c >= n || c < 0) return;
        const int u = c / a.words, cell0 = 32 * (c - u * a.words);
        // (a unit that is skipped is passed through as a whole)
        const uint32_t kept = __ldg(&a.ranges[u].cnt) > 0 ? __ldg(a.kept + c) : 0u;
        const int total = min(32, a.mn - cell0) * vecs;
        const int64_t at = ((int64_t)u * a.mn + cell0) * vecs;
        for (int i0 = lane; i0 < total; i0 += 32 * F) {
            uint4 v[F];
            bool in[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int i = i0 + 32 * f;
                in[f] = i < total && !(kept >> (i / vecs) & 1u);
                v[f] = in[f] && res ? __ldcs(res + at + i) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (in[f]) out[at + i0 + 32 * f] = v[f];
        }
    }
}

// What a kernel takes for a kind of scores.
template <class X>
struct ReadoutOf {
    using Args = ReadoutMore;
};
template <>
struct ReadoutOf<PlainScores> {
    using Args = ReadoutArgs;
};

struct ReadoutPath {
    int kind;        // 0 = CUDA-core, 1 = tensor-core (tcgen05)
    bool either;     // ... with one or two query tiles, as the plan finds
    int BM, BN;      // of one query tile
    int part_rows;   // rows of a partial slot
    int grid;   // CTAs of the readout launch
};

// the path of a call over banks of this many rows with this workspace (INT64_MAX and
// SIZE_MAX: the path that any workspace is sized for)
ReadoutPath choose_readout_path(rs3_dtype dtype, int d, int U, int H, int k_max, int64_t bank_rows, size_t workspace_bytes);
// The CUDA-core path `p` with fewer query rows to a CTA, and whether a call has too few of them for `p`; heads whose calls
// always have.
ReadoutPath rs3_few_rows(ReadoutPath p, int d);
bool rs3_has_few_rows(const ReadoutPath &p, int U, int H, int d, int k_max, int64_t bank_rows);
constexpr bool rs3_always_few_rows(int d) { return d == 128; }
bool rs3_tc_supported(int d);
int rs3_tc_block_n(int d);
rs3_status rs3_launch_tc_readout(const ReadoutArgs &a, cudaStream_t st);
rs3_status rs3_launch_either_readout(const ReadoutArgs &a, cudaStream_t st);   // d = 64, 128
// CUDA-core path: rows and keys of a tile and resident CTAs per SM, for a head width
void rs3_simt_tile(int d, bool few, int &bm, int &bn, int &ctas_per_sm);
rs3_status rs3_launch_simt_readout(const ReadoutArgs &a, rs3_dtype dtype, cudaStream_t st);
rs3_status rs3_readout_prepare(const void *q, rs3_dtype dtype, int G, int mn, int H, int d,
                               const int32_t *unit_group, const int32_t *idx, const int32_t *count,
                               int k_max, const rs3_bank *bank, const float *rope,
                               const void *residual, void *out, float scale, void *workspace,
                               size_t workspace_bytes, int32_t *status, ReadoutArgs *a,
                               ReadoutPath *path, int64_t *grid_combine);
// The workspace of a path, from `base` on; with `parts`, slots for every group and their table.
ReadoutLayout rs3_readout_layout(int U, int H, int d, int k_max, const ReadoutPath &p, bool parts);
// Checks of what readouts of a bank have in common, and the arguments of one over the path and layout.
rs3_status rs3_readout_check(const void *q, rs3_dtype dtype, int G, int mn, int H, int d, const int32_t *unit_group,
                             const int32_t *idx, const int32_t *count, int k_max, const rs3_bank *bank, const float *rope,
                             const void *residual, const void *out, const void *workspace, const int32_t *status);
bool rs3_readout_fits(int U, int H, int k_max, const ReadoutPath &p);      // its work list's indices
void rs3_readout_fill(ReadoutArgs *a, const ReadoutPath &p, const ReadoutLayout &L, uint8_t *ws, const void *q, int G, int mn, int H,
                      int d, const int32_t *unit_group, const int32_t *idx, const int32_t *count, int k_max, int U,
                      const rs3_bank *bank, const float *rope, const void *residual, void *out, float scale, int32_t *status);
// The attention kernel over the plan in the workspace.
rs3_status rs3_readout_run_launch(const ReadoutArgs &a, const ReadoutPath &p, rs3_dtype dtype, cudaStream_t st);
rs3_status rs3_launch_scored_either(const ReadoutMore &a, cudaStream_t st);
rs3_status rs3_launch_scored_tc(const ReadoutMore &a, cudaStream_t st);
rs3_status rs3_launch_scored_simt(const ReadoutMore &a, rs3_dtype dtype, cudaStream_t st);
// A readout over changed scores; `one`: of a single unit, whose frames are still to be gone through.
namespace frames { struct FramesArgs; }
rs3_status rs3_scored_launch(const ReadoutMore &a, const frames::FramesArgs *one, const ReadoutPath &p, int64_t max_combine, rs3_dtype dtype, cudaStream_t st);
// Two plans in one launch, with the second's pass-through.
rs3_status rs3_readout_plan_two(const ReadoutMore &first, const ReadoutMore &second, rs3_dtype dtype, cudaStream_t st);
// phases of a readout: the attention over the bank (pass-through, plan,
// readout kernel) and the merge of split-KV partials
enum { RS3_PHASE_PLAN = 1, RS3_PHASE_RUN = 4, RS3_PHASE_ATTEND = 1 | 4, RS3_PHASE_MERGE = 2 };
rs3_status rs3_readout_launch(const ReadoutArgs &a, const ReadoutPath &p,
                              int64_t max_combine, rs3_dtype dtype, cudaStream_t st, int phases);

// Tile t of a unit's bank (tiles of BN rows, never crossing a range end) ->
// first physical row and the number of valid rows.
__device__ __forceinline__ void tile_rows(const RangeSet &rs, int t, int BN, int64_t &row0, int &nvalid)
{
    row0 = 0;
    nvalid = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (t < rs.tiles[r]) {
            row0 = rs.start[r] + (int64_t)t * BN;
            nvalid = min(BN, rs.len[r] - t * BN);
            return;
        }
        t -= rs.tiles[r];
    }
}

// Same, reading the range set in place (global memory) instead of a local copy.
__device__ __forceinline__ void tile_rows(const RangeSet *rs, int t, int BN, int64_t &row0, int &nvalid)
{
    row0 = 0;
    nvalid = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int tiles = __ldg(&rs->tiles[r]);
        if (t < tiles) {
            row0 = __ldg(&rs->start[r]) + (int64_t)t * BN;
            nvalid = min(BN, __ldg(&rs->len[r]) - t * BN);
            return;
        }
        t -= tiles;
    }
}

__device__ __forceinline__ float4 load4(const float *p) { return __ldg(reinterpret_cast<const float4 *>(p)); }
__device__ __forceinline__ float4 load4(const uint16_t *p)
{
    const uint2 w = __ldg(reinterpret_cast<const uint2 *>(p));
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u),
                       __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}

// Two fp32 values to a bf16 pair (round to nearest even), `lo` in the low half;
// one cvt instruction (the per-value conversions cost about three times more).
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// A 16-byte piece of a query row (four pairs) rotated by the (cos, sin) of those
// pairs at f (Eq. 7), rounded once per element.
__device__ __forceinline__ uint4 rotate_q_piece(uint4 v, const float *f)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int p = 0; p < 4; p += 2) {
        const float4 c = __ldg(reinterpret_cast<const float4 *>(f) + p / 2);
        const float x0 = __uint_as_float(w[p] << 16), x1 = __uint_as_float(w[p] & 0xffff0000u);
        const float y0 = __uint_as_float(w[p + 1] << 16), y1 = __uint_as_float(w[p + 1] & 0xffff0000u);
        w[p] = pack_bf16x2(x0 * c.x - x1 * c.y, x0 * c.y + x1 * c.x);
        w[p + 1] = pack_bf16x2(y0 * c.z - y1 * c.w, y0 * c.w + y1 * c.z);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// out[u][cell][c .. c+1] (store_out2) or [c .. c+3] (store_out4) =
// residual[...] + o, rounded once to T
template <typename T>
__device__ __forceinline__ void store_out2(const ReadoutArgs &a, int u, int cell, int c, const float *o);

template <>
__device__ __forceinline__ void store_out2<float>(const ReadoutArgs &a, int u, int cell, int c, const float *o)
{
    const int64_t off = ((int64_t)u * a.mn + cell) * a.D + c;
    float2 r = make_float2(0.f, 0.f);
    if (a.residual) r = *reinterpret_cast<const float2 *>(static_cast<const float *>(a.residual) + off);
    *reinterpret_cast<float2 *>(static_cast<float *>(a.out) + off) = make_float2(r.x + o[0], r.y + o[1]);
}

template <>
__device__ __forceinline__ void store_out2<uint16_t>(const ReadoutArgs &a, int u, int cell, int c, const float *o)
{
    const int64_t off = ((int64_t)u * a.mn + cell) * a.D + c;
    float r0 = 0.f, r1 = 0.f;
    if (a.residual) {
        const uint32_t x = *reinterpret_cast<const uint32_t *>(static_cast<const uint16_t *>(a.residual) + off);
        r0 = __uint_as_float(x << 16);
        r1 = __uint_as_float(x & 0xffff0000u);
    }
    *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(a.out) + off) = pack_bf16x2(r0 + o[0], r1 + o[1]);
}

template <typename T>
__device__ __forceinline__ void store_out4(const ReadoutArgs &a, int u, int cell, int c, const float *o);

template <>
__device__ __forceinline__ void store_out4<float>(const ReadoutArgs &a, int u, int cell, int c, const float *o)
{
    const int64_t off = ((int64_t)u * a.mn + cell) * a.D + c;
    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.residual) r = load4(static_cast<const float *>(a.residual) + off);
    *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + off) =
        make_float4(r.x + o[0], r.y + o[1], r.z + o[2], r.w + o[3]);
}

template <>
__device__ __forceinline__ void store_out4<uint16_t>(const ReadoutArgs &a, int u, int cell, int c, const float *o)
{
    const int64_t off = ((int64_t)u * a.mn + cell) * a.D + c;
    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.residual) r = load4(static_cast<const uint16_t *>(a.residual) + off);
    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + off) =
        make_uint2(pack_bf16x2(r.x + o[0], r.y + o[1]), pack_bf16x2(r.z + o[2], r.w + o[3]));
}
