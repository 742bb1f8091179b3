// rs3_blocks.cu -- digests of a bank's blocks, and the blocks whose digests score highest for
// each kept query and head.
//
// A block is `block` consecutive storage rows of a unit.  Its digest, per head, is the mean of
// its live keys in 8 bits with a power of two (EightBits), so that scores are whole numbers times
// a power of two: exact, hence the same whatever order they are summed in.
#include "rs3_sparse.cuh"

namespace {

// ---------------------------------------------------------------------------
// digests
// ---------------------------------------------------------------------------
constexpr int DIGEST_THREADS = 256;        // 32 pieces x 8 partial sums

struct DigestArgs {
    BankDev bank;
    const uint8_t *k_store;
    int8_t *digest;
    float *step;
    int32_t *status;
    int64_t row_bytes;
    int32_t H, d, bs, nb, refresh;
};

// Blocks that a refresh of the newest frames visits: those of the frames' rows (two runs when
// the ring wraps), then those of the ring's oldest and newest rows and of its two ends.  Frames
// given up or overwritten since leave dead rows beside live ones only there.
__device__ int64_t refresh_block(const DigestArgs &a, const LiveRows &rows, int64_t u, int64_t t)
{
    const int64_t *mu = a.bank.meta + u * a.bank.stride_words;
    const int64_t *fl = mu + BM_HEADER_WORDS + a.bank.max_frames;
    const int64_t nf = mu[BM_NFRAMES], oldest = mu[BM_OLDEST];
    const int64_t live = rows.len[1] + rows.len[2];
    int64_t fresh = 0;
    for (int64_t i = 0; i < a.refresh && i < nf; ++i) fresh += fl[(oldest + nf - 1 - i) % a.bank.max_frames];
    fresh = min(live, max((int64_t)0, fresh));
    const int64_t cap = a.bank.ring_cap, base = a.bank.pinned_cap;
    if (cap == 0) return -1;
    const int64_t tail = live > 0 ? (rows.start[1] - base + live) % cap : 0;      // one past the newest row
    const int64_t from = live > 0 ? (tail - fresh + cap) % cap : 0;
    int64_t runs[2][2] = {{from, min(from + fresh, cap)}, {0, from + fresh - cap}};
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        if (runs[r][1] <= runs[r][0]) continue;
        const int64_t b0 = (base + runs[r][0]) / a.bs, b1 = (base + runs[r][1] - 1) / a.bs;
        if (t <= b1 - b0) return b0 + t;
        t -= b1 - b0 + 1;
    }
    if (t == 0) return base / a.bs;
    if (t == 1) return (base + cap - 1) / a.bs;
    if (live > 0 && t == 2) return rows.start[1] / a.bs;
    if (live > 0 && t == 3) return (base + (tail + cap - 1) % cap) / a.bs;
    return -1;
}

// A CTA digests 32 x ITEMS pieces (16 bytes each: whole heads) of one block: thread (piece, p)
// sums rows p, p + 8, ... of its piece, then the eight partial sums of a channel are joined
// as ((0 + 4) + (2 + 6)) + ((1 + 5) + (3 + 7)).  Dead rows are not read.
template <typename T, int ITEMS>
__global__ void __launch_bounds__(DIGEST_THREADS) k_digest(DigestArgs a)
{
    constexpr int N = 16 / sizeof(T), COLS = 32 * ITEMS * N;
    pdl_wait();
    __shared__ float s_sum[8][COLS];
    __shared__ float s_max[DIGEST_THREADS / 32];
    __shared__ int64_t s_block;
    const int64_t u = blockIdx.z;
    LiveRows rows;
    if (!rows.load(a.bank, u)) {
        if (threadIdx.x == 0) latch_status(a.status, RS3_EINTERNAL);
        return;
    }
    int64_t b = blockIdx.x;
    if (a.refresh >= 0) {
        if (threadIdx.x == 0) s_block = refresh_block(a, rows, u, b);
        __syncthreads();
        b = s_block;
        if (b < 0) return;
    }
    const int64_t r0 = b * a.bs;
    const int64_t n_live = rows.count(r0, r0 + a.bs);
    const int piece = threadIdx.x & 31, p = threadIdx.x >> 5;
    const int nvec = (int)(a.row_bytes / 16), v0 = blockIdx.y * 32 * ITEMS;
    const uint8_t *src = a.k_store + (u * a.bank.rows_per_unit + r0) * a.row_bytes;
    float sum[ITEMS][N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[i][e] = 0.f;
#pragma unroll 4
    for (int r = p; r < a.bs; r += 8) {
        const bool live = rows.holds(r0 + r);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int v = v0 + piece + 32 * i;
            if (!live || v >= nvec) continue;
            const uint4 w = __ldg(reinterpret_cast<const uint4 *>(src + r * a.row_bytes) + v);
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (N == 8) {
                    sum[i][2 * e] += __uint_as_float(x[e] << 16);
                    sum[i][2 * e + 1] += __uint_as_float(x[e] & 0xffff0000u);
                } else {
                    sum[i][e] += __uint_as_float(x[e]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) s_sum[p][(piece + 32 * i) * N + e] = sum[i][e];
    __syncthreads();
    // a channel per thread and round; a head is a run of d threads
    const float n = (float)(n_live > 0 ? n_live : 1);
    for (int c0 = 0; c0 < COLS; c0 += DIGEST_THREADS) {
        const int c = c0 + threadIdx.x;                       // COLS <= 256, or a multiple of it
        const bool in = c < COLS && v0 * N + c < a.H * a.d;
        float x = 0.f;
        if (c < COLS) {
            x = ((s_sum[0][c] + s_sum[4][c]) + (s_sum[2][c] + s_sum[6][c])) +
                ((s_sum[1][c] + s_sum[5][c]) + (s_sum[3][c] + s_sum[7][c]));
            x = __fdiv_rn(x, n);
        }
        float m = fabsf(x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            if (o < a.d) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (a.d > 32) {
            __syncthreads();
            if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
            __syncthreads();
            const int w0 = (threadIdx.x >> 5) / (a.d >> 5) * (a.d >> 5);
            for (int w = 0; w < a.d >> 5; ++w) m = fmaxf(m, s_max[w0 + w]);
        }
        if (!in) continue;                                    // uniform over a head; no barrier follows for these
        const EightBits q(m);
        const int col = v0 * N + c, h = col / a.d, e = col - h * a.d;
        const int64_t at = (u * a.H + h) * a.nb + b;
        a.digest[at * a.d + e] = (int8_t)q(x);
        if (e == 0) a.step[at] = q.step;
    }
}

// ---------------------------------------------------------------------------
// selection
// ---------------------------------------------------------------------------
constexpr int SELECT_THREADS = 256;
constexpr int SELECT_KEYS_BYTES = 96 * 1024;       // scores of a CTA's queries, with few blocks
constexpr int SELECT_MAX_BLOCKS = 48 * 1024;       // one query's scores fill a CTA's shared memory

struct SelectArgs {
    SparseArgs s;
    const int8_t *digest;
    const float *step;
    int32_t *sel;
    int32_t qt;                // queries of a CTA
    int32_t bf16;
};

__device__ __forceinline__ float load_q(const SelectArgs &a, int64_t i)
{
    return a.bf16 ? bf16_bits_to_float(static_cast<const uint16_t *>(a.s.q)[i]) : static_cast<const float *>(a.s.q)[i];
}

// a score as a number that orders as it does; 0 is left for blocks that are not there
__device__ __forceinline__ uint32_t order_bits(float s)
{
    const uint32_t b = __float_as_uint(s + 0.f);             // -0 becomes +0
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(SELECT_THREADS) k_block_select(SelectArgs a)
{
    pdl_wait();
    extern __shared__ uint32_t s_keys[];                     // [qt][nb]
    __shared__ __align__(16) int8_t s_q[8][256];
    const SparseArgs &s = a.s;
    const int u = blockIdx.z, h = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int cnt, g;
    LiveRows rows;
    if (!sparse_unit(s, u, threadIdx.x == 0, cnt, g, rows)) return;
    const int j0 = blockIdx.x * a.qt, nq = min(a.qt, cnt - j0);
    if (nq <= 0) return;
    // the queries in 8 bits, a warp each: rotated by their own cell (each product and sum rounded)
    if (warp < nq) {
        const int cell = s.idx[(int64_t)u * s.k_max + j0 + warp];
        const bool ok = cell >= 0 && cell < s.mn;
        if (!ok && lane == 0) latch_status(s.status, RS3_EINVAL);
        float x[8], m = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = lane + 32 * i;
            float x0 = 0.f, x1 = 0.f;
            if (ok && 2 * p < s.d) {
                const int64_t at = ((int64_t)g * s.mn + cell) * (s.H * s.d) + h * s.d + 2 * p;
                x0 = load_q(a, at);
                x1 = load_q(a, at + 1);
                if (s.rope) {
                    const float2 c = __ldg(reinterpret_cast<const float2 *>(s.rope + (int64_t)cell * s.d) + p);
                    const float y0 = __fsub_rn(__fmul_rn(x0, c.x), __fmul_rn(x1, c.y));
                    x1 = __fadd_rn(__fmul_rn(x0, c.y), __fmul_rn(x1, c.x));
                    x0 = y0;
                }
            }
            x[2 * i] = x0;
            x[2 * i + 1] = x1;
            m = fmaxf(m, fmaxf(fabsf(x0), fabsf(x1)));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const EightBits e(m);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = lane + 32 * i;
            if (2 * p < s.d) {
                s_q[warp][2 * p] = (int8_t)e(x[2 * i]);
                s_q[warp][2 * p + 1] = (int8_t)e(x[2 * i + 1]);
            }
        }
    }
    __syncthreads();
    // scores, a block per thread
    const int64_t dig = ((int64_t)u * s.H + h) * s.nb;
    for (int b = threadIdx.x; b < s.nb; b += SELECT_THREADS) {
        int acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const bool live = rows.count((int64_t)b * s.bs, (int64_t)(b + 1) * s.bs) > 0;
        if (live) {
            const uint4 *t = reinterpret_cast<const uint4 *>(a.digest + (dig + b) * s.d);
            for (int v = 0; v < s.d / 16; ++v) {
                const uint4 w = __ldg(t + v);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    if (q >= nq) break;
                    const int4 y = *reinterpret_cast<const int4 *>(&s_q[q][16 * v]);
                    acc[q] = __dp4a((int)w.x, y.x, acc[q]);
                    acc[q] = __dp4a((int)w.y, y.y, acc[q]);
                    acc[q] = __dp4a((int)w.z, y.z, acc[q]);
                    acc[q] = __dp4a((int)w.w, y.w, acc[q]);
                }
            }
        }
        const float step = live ? __ldg(a.step + dig + b) : 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < nq) s_keys[q * s.nb + b] = live ? order_bits((float)acc[q] * step) : 0u;
    }
    __syncthreads();
    if (warp >= nq) return;
    // the n-th largest key of a query, bit by bit; a warp per query
    const uint32_t *key = s_keys + warp * s.nb;
    int32_t *out = a.sel + (((int64_t)u * s.H + h) * s.k_max + j0 + warp) * s.n_top;
    const auto at_least = [&](uint32_t x) {
        int n = 0;
        for (int b = lane; b < s.nb; b += 32) n += key[b] >= x;
        return (int)__reduce_add_sync(0xffffffffu, n);
    };
    const int want = min(s.n_top, at_least(1u));
    uint32_t cut = 0;
    if (want > 0)
        for (int bit = 31; bit >= 0; --bit)
            if (at_least(cut | 1u << bit) >= want) cut |= 1u << bit;
    // every key above the cut, and the first of those at it
    int above = 0;
    for (int b = lane; b < s.nb; b += 32) above += key[b] > cut;
    int equal = want - (int)__reduce_add_sync(0xffffffffu, above), n = 0;
    for (int b0 = 0; b0 < s.nb && n < want; b0 += 32) {
        const int b = b0 + lane;
        const uint32_t k = b < s.nb ? key[b] : 0u;
        uint32_t lm;
        asm("mov.u32 %0, %%lanemask_lt;" : "=r"(lm));
        const uint32_t same = __ballot_sync(0xffffffffu, k == cut && k > 0);
        const bool take = k > cut || (k == cut && k > 0 && __popc(same & lm) < equal);
        const uint32_t bal = __ballot_sync(0xffffffffu, take);
        if (take) out[n + __popc(bal & lm)] = b;
        n += __popc(bal);
        equal -= min(equal, __popc(same));
    }
    for (int i = want + lane; i < s.n_top; i += 32) out[i] = -1;
}

}  // namespace

extern "C" int64_t rs3_bank_blocks(const rs3_bank *bank, int block)
{
    if (!bank_ok(bank) || block < 1) return -1;
    return (bank->rows_per_unit + block - 1) / block;
}

extern "C" rs3_status rs3_bank_digest(const rs3_bank *bank, int block, int refresh, int8_t *digest, float *step,
                                      int32_t *status, rs3_stream_t stream)
{
    if (!bank_ok(bank) || !digest || !step || !status || refresh < -1) return RS3_EINVAL;
    if (!rs3_aligned16(digest) || !rs3_aligned16(step)) return RS3_EINVAL;
    const int d = bank->d;
    if (block != 32 && block != 64 && block != 128) return RS3_EUNSUPPORTED;
    if (d < 16 || d > 256 || (d & (d - 1)) != 0) return RS3_EUNSUPPORTED;
    const int64_t nb = (bank->rows_per_unit + block - 1) / block;
    if (nb > INT32_MAX) return RS3_EUNSUPPORTED;
    if (nb == 0) return RS3_OK;
    DigestArgs a = {};
    a.bank = bank_dev(bank);
    a.k_store = static_cast<const uint8_t *>(bank->k_store);
    a.digest = digest;
    a.step = step;
    a.status = status;
    a.row_bytes = (int64_t)bank->D * (int64_t)elem_bytes(bank->dtype);
    a.H = bank->H;
    a.d = d;
    a.bs = block;
    a.nb = (int32_t)nb;
    a.refresh = refresh;
    // blocks of the frames' rows in two runs, and the four single ones
    const int64_t most = (int64_t)refresh * bank->mn / block + 8;
    const int64_t x = refresh < 0 || most > nb + 8 ? nb + (refresh < 0 ? 0 : 8) : most;
    const bool wide = bank->dtype == RS3_F32 && d == 256;
    const int pieces = wide ? 64 : 32;
    const int64_t slabs = (a.row_bytes / 16 + pieces - 1) / pieces;
    if (slabs > 65535) return RS3_EUNSUPPORTED;
    const dim3 grid((unsigned)x, (unsigned)slabs, (unsigned)bank->U);
    void (*kern)(DigestArgs) = bank->dtype == RS3_BF16 ? k_digest<uint16_t, 1> : wide ? k_digest<float, 2> : k_digest<float, 1>;
    launch_pdl(kern, grid, dim3(DIGEST_THREADS), 0, reinterpret_cast<cudaStream_t>(stream), a);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}

extern "C" size_t rs3_block_select_workspace_bytes(int U, int H, int k_max, int n_blocks)
{
    if (U < 1 || H < 1 || k_max < 0 || n_blocks < 0) return 0;
    return 16;
}

extern "C" rs3_status rs3_block_select(const void *q, rs3_dtype dtype, int G, int mn, int H, int d,
                                       const int32_t *unit_group, const int32_t *idx, const int32_t *count, int k_max,
                                       const rs3_bank *bank, int block, const int8_t *digest, const float *step,
                                       const float *rope, int n_top, int32_t *sel, void *workspace,
                                       size_t workspace_bytes, int32_t *status, rs3_stream_t stream)
{
    SelectArgs a = {};
    const rs3_status s = sparse_args(a.s, q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, block, rope, n_top, status);
    if (s != RS3_OK) return s;
    if (!digest || !step || !sel || !workspace) return RS3_EINVAL;
    if (!rs3_aligned16(digest) || !rs3_aligned16(workspace)) return RS3_EINVAL;
    if (a.s.nb > SELECT_MAX_BLOCKS) return RS3_EUNSUPPORTED;
    if (workspace_bytes < rs3_block_select_workspace_bytes(a.s.U, H, k_max, a.s.nb)) return RS3_ECAPACITY;
    if (k_max == 0) return RS3_OK;
    a.digest = digest;
    a.step = step;
    a.sel = sel;
    a.bf16 = dtype == RS3_BF16;
    a.qt = 8;
    while (a.qt > 1 && (int64_t)a.qt * a.s.nb * 4 > SELECT_KEYS_BYTES) a.qt >>= 1;
    const size_t smem = (size_t)a.qt * (size_t)a.s.nb * 4;
    const rs3_status r = rs3_kernel_smem((const void *)k_block_select, smem);
    if (r != RS3_OK) return r;
    const dim3 grid((unsigned)((k_max + a.qt - 1) / a.qt), (unsigned)H, (unsigned)a.s.U);
    launch_pdl(k_block_select, grid, dim3(SELECT_THREADS), smem, reinterpret_cast<cudaStream_t>(stream), a);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
