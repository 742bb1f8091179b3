// rs3_blocks.cu -- digests of a bank's blocks, and the blocks whose digests score highest for
// each kept query and head.
//
// A block is `block` consecutive storage rows of a unit.  Its digest, per head, is the mean of
// its live keys in 8 bits with a power of two (EightBits), so that scores are whole numbers times
// a power of two: exact, hence the same whatever order they are summed in.
#include "rs3_sparse.cuh"

#include "rs3_blocks_tma.cuh"

#include <cfloat>

namespace {

// ---------------------------------------------------------------------------
// digests
// ---------------------------------------------------------------------------
struct DigestArgs {
    BankDev bank;
    int8_t *digest;
    float *step;
    int32_t *status;
    int64_t row_bytes, visits; // blocks to visit
    int32_t H, d, bs, nb, refresh;
    uint64_t wait_ns;          // limit of each wait
};

// Rows of the newest `refresh` ring frames, -1 where the counters are inconsistent; by a whole warp.
__device__ int64_t fresh_rows(const DigestArgs &a, int64_t u)
{
    const int64_t *mu = a.bank.meta + u * a.bank.stride_words;
    const int64_t *fl = mu + BM_HEADER_WORDS + a.bank.max_frames;
    const int64_t nf = mu[BM_NFRAMES], oldest = mu[BM_OLDEST];
    if (nf < 0 || nf > a.bank.max_frames || (nf > 0 && (oldest < 0 || oldest >= a.bank.max_frames))) return -1;
    int64_t n = 0;
    for (int64_t i = threadIdx.x & 31; i < a.refresh && i < nf; i += 32) {
        int64_t slot = oldest + nf - 1 - i;
        if (slot >= a.bank.max_frames) slot -= a.bank.max_frames;
        n += fl[slot];
    }
    return warp_sum(n);
}

// Blocks that a refresh of the newest frames visits: those of the frames' `fresh` rows (two runs when
// the ring wraps), then those of the ring's two ends and of its oldest and newest rows.  Frames
// given up or overwritten since leave dead rows beside live ones only there.  -1 behind the last.
__device__ int64_t refresh_block(const DigestArgs &a, const LiveRows &rows, int64_t fresh, int64_t t)
{
    const int64_t live = rows.len[1] + rows.len[2], cap = a.bank.ring_cap, base = a.bank.pinned_cap;
    if (cap == 0) return -1;
    fresh = min(live, max((int64_t)0, fresh));
    // one past the newest row, and the first fresh one
    int64_t tail = live > 0 ? rows.start[1] - base + live : 0;
    tail -= tail >= cap ? cap : 0;
    const int64_t from = tail - fresh + (tail < fresh ? cap : 0);
    const int64_t runs[2][2] = {{from, min(from + fresh, cap)}, {0, from + fresh - cap}};
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
    if (live > 0 && t == 3) return (base + (tail == 0 ? cap : tail) - 1) / a.bs;
    return -1;
}

// A warp digests 32 x ITEMS pieces (16 bytes each: whole heads) of one block after another, by itself: its first
// lane brings the rows by TMA, 16 at a time (8 of 1 KB), into one of the warp's two buffers while the other's are added.  A
// lane adds its pieces' rows up in the eight partial sums, which it then joins as
// ((0 + 4) + (2 + 6)) + ((1 + 5) + (3 + 7)): no barrier among warps.  Which rows live is worked out for 32 blocks at
// a time, one per lane; pieces without a live row are not read.  192 KB in flight per SM: with the rows loaded
// into registers (64 KB) all blocks of eight banks (252 MB) took 64 us, 51 to 59 so.  The blocks of a newest frame take
// 10 us, the latency of the bank's counters, the frames' lengths, a copy and its sums one after another.
constexpr int DIGEST_WARPS = 12;

template <typename T, int ITEMS>
__global__ void __launch_bounds__(32 * DIGEST_WARPS, 1) k_digest(DigestArgs a, const __grid_constant__ CUtensorMap map)
{
    using namespace tc;
    constexpr int N = 16 / sizeof(T), ROWS = 16 / ITEMS, BUFFER = 8192, PER = 64 / ROWS;     // of a piece; pieces of 64 rows
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_bars[DIGEST_WARPS][2];
    __shared__ int s_abort;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t buffer = ((smem_u32(smem_raw) + 127u) & ~127u) + (uint32_t)warp * 2u * BUFFER, bar = smem_u32(s_bars[warp]);
    if (threadIdx.x == 0) s_abort = 0;
    if (lane == 0) {
        mbar_init(bar, 1);
        mbar_init(bar + 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    __syncthreads();
    pdl_wait();
    const int64_t u = blockIdx.z;
    LiveRows rows;
    const bool sane = rows.load(a.bank, u);
    const int64_t fresh = a.refresh > 0 ? fresh_rows(a, u) : 0;
    if (!sane || fresh < 0) {
        if (threadIdx.x == 0) latch_status(a.status, RS3_EINTERNAL);
        return;
    }
    const int nvec = (int)(a.row_bytes / 16), slab0 = blockIdx.y * 32 * ITEMS;
    const uint32_t pitch = (uint32_t)min(nvec, 32 * ITEMS) * 16u;      // bytes of a row in a buffer
    const int64_t warps = (int64_t)gridDim.x * DIGEST_WARPS;
    const int y0 = (int)(u * a.bank.rows_per_unit);
    uint32_t issued = 0, used = 0;                                     // of the warp's pieces
    bool ok = true;
    for (int64_t t0 = (int64_t)blockIdx.x * DIGEST_WARPS + warp; t0 < a.visits && ok; t0 += 32 * warps) {
        // this warp's next 32 blocks, one per lane, and their live rows
        const int64_t t = t0 + lane * warps;
        const int mine = (int)(t >= a.visits ? -1 : a.refresh < 0 ? t : refresh_block(a, rows, fresh, t));
        uint64_t live[2] = {0ull, 0ull};
        if (mine >= 0) {
            live[0] = rows.mask64((int64_t)mine * a.bs) & (a.bs == 32 ? 0xffffffffull : ~0ull);
            if (a.bs > 64) live[1] = rows.mask64((int64_t)mine * a.bs + 64);
        }
        // the pieces with a live row, a bit each
        constexpr uint32_t ALL = (1u << ROWS) - 1u;
        uint32_t some = 0;
#pragma unroll
        for (int j = 0; j < 2 * PER; ++j) some |= (uint32_t)(((uint32_t)(live[j / PER] >> (ROWS * (j % PER))) & ALL) != 0u) << j;
        int ahead = 0;                                                 // the block whose pieces are brought next, and which are left
        uint32_t left = __shfl_sync(0xffffffffu, some, 0);
        const auto bring = [&]() {
            while (left == 0u && ahead < 31) left = __shfl_sync(0xffffffffu, some, ++ahead);
            const int b = __shfl_sync(0xffffffffu, mine, ahead);
            if (left == 0u) return;
            if (lane == 0) {
                const uint32_t st = issued & 1u;
                mbar_expect_tx(bar + 8u * st, ROWS * pitch);
                tma_load_2d(buffer + st * BUFFER, &map, bar + 8u * st, slab0 * N, y0 + b * a.bs + ROWS * (__ffs(left) - 1));
            }
            left &= left - 1u;
            ++issued;
        };
        bring();
        bring();
        for (int i = 0; i < 32 && ok; ++i) {
            const int b = __shfl_sync(0xffffffffu, mine, i);
            if (b < 0) break;
            float sum[ITEMS][8][N];
#pragma unroll
            for (int x = 0; x < ITEMS; ++x)
#pragma unroll
                for (int p = 0; p < 8; ++p)
#pragma unroll
                    for (int e = 0; e < N; ++e) sum[x][p][e] = 0.f;
            int n_live = 0;
            for (int j = 0; ROWS * j < a.bs; ++j) {
                const uint32_t on = (uint32_t)(__shfl_sync(0xffffffffu, j < PER ? live[0] : live[1], i) >> (ROWS * (j % PER))) & ALL;
                if (on == 0u) continue;
                n_live += __popc(on);
                const uint32_t st = used & 1u, src = buffer + st * BUFFER + lane * 16;
                ok = mbar_wait_warp(bar + 8u * st, used >> 1 & 1u, &s_abort, a.wait_ns);
                if (!ok) break;
                ++used;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    if (!(on >> r & 1u)) continue;
#pragma unroll
                    for (int x = 0; x < ITEMS; ++x) {
                        uint32_t y[4];
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3])
                                     : "r"(src + r * pitch + 512u * x) : "memory");
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (N == 8) {
                                sum[x][r & 7][2 * e] += __uint_as_float(y[e] << 16);
                                sum[x][r & 7][2 * e + 1] += __uint_as_float(y[e] & 0xffff0000u);
                            } else {
                                sum[x][r & 7][e] += __uint_as_float(y[e]);
                            }
                        }
                    }
                }
                __syncwarp();
                bring();
            }
            if (!ok) break;
            // dividing by a power of two is exact either way
            const bool pow2 = (n_live & (n_live - 1)) == 0;
            const float n = (float)max(1, n_live), inv = 1.f / n;
#pragma unroll
            for (int x = 0; x < ITEMS; ++x)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const auto &v = sum[x];
                    const float y = ((v[0][e] + v[4][e]) + (v[2][e] + v[6][e])) + ((v[1][e] + v[5][e]) + (v[3][e] + v[7][e]));
                    sum[x][0][e] = pow2 ? y * inv : __fdiv_rn(y, n);
                }
            // a head is a run of d / N lanes (ITEMS = 2: of all 32, both items)
            float m = 0.f;
#pragma unroll
            for (int x = 0; x < ITEMS; ++x)
#pragma unroll
                for (int e = 0; e < N; ++e) m = fmaxf(m, fabsf(sum[x][0][e]));
            for (int o = min(32, a.d / N) >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const EightBits q(m);
#pragma unroll
            for (int x = 0; x < ITEMS; ++x) {
                const int v = slab0 + 32 * x + lane;
                if (v >= nvec) continue;
                const int col = v * N, h = col / a.d, e0 = col - h * a.d;
                const int64_t at = (u * a.H + h) * a.nb + b;
                uint32_t word[N / 4];
#pragma unroll
                for (int e = 0; e < N; e += 4)
                    word[e / 4] = (uint32_t)(q(sum[x][0][e]) & 255) | (uint32_t)(q(sum[x][0][e + 1]) & 255) << 8 |
                                  (uint32_t)(q(sum[x][0][e + 2]) & 255) << 16 | (uint32_t)q(sum[x][0][e + 3]) << 24;
                if (N == 8) *reinterpret_cast<uint2 *>(a.digest + at * a.d + e0) = make_uint2(word[0], word[N / 4 - 1]);
                else *reinterpret_cast<uint32_t *>(a.digest + at * a.d + e0) = word[0];
                if (e0 == 0) a.step[at] = q.step;
            }
        }
    }
    if (!ok) {
        // copies in flight land before the CTA ends
        if (lane == 0) {
            for (; used < issued; ++used) mbar_drain(bar + 8u * (used & 1u), used >> 1 & 1u);
            latch_status(a.status, RS3_ETIMEOUT);
        }
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

// the score of a number of order_bits()
__device__ __forceinline__ float score_of(uint32_t key)
{
    return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
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

// The same on the tensor cores, for what most calls are: up to 992 blocks that hold a live row in one piece, or more
// in pieces of up to 992 whose choices k_merge_blocks joins.
//
// A CTA scores 16 queries against its blocks: whole numbers of at most 127 are exact in fp16, and their
// products' sums stay below 2^22, exact in the fp32 accumulators.  A lane's 16 bytes of a digest are
// spread over four steps of the matrix instruction, and the queries' columns are taken in the same order.
// Then a warp per query holds the scores in registers, 32 blocks to a lane.  Of n wanted, a number that n or few more
// of the maxima of four blocks each reach is a bound that few more than n scores reach: these candidates are ranked
// by counting.  (Where they are many, as among ties, the registers are cut exactly.)
// Bound by instruction issue and, at the start, latency.  Also built: a lane per query that keeps a running threshold;
// as scores grow towards the newest frames, that admits nearly every block and took several times as long.
constexpr int TC_ROWS = 16;                // queries of a CTA
constexpr int TC_THREADS = 256;
constexpr int TC_BLOCKS = 992;             // blocks of a piece: three CTAs per SM
constexpr int TC_TOP = 64;                 // choices of a piece that the workspace has room for
constexpr int TC_HELD = 64;                // candidates of a query that are compacted
constexpr int TC_PAIRS = 3264;             // candidates of a query that are joined in shared memory
constexpr size_t TC_SMS = 256;             // SMs that pieces are cut for, at most

struct PickArgs {
    SelectArgs a;
    int2 *cand;                // [rows][splits][take]: (ordered score, block)
    int32_t *n_cand;           // [rows][splits]
    int32_t *n_pieces;         // [U]: pieces of a unit's queries
    int32_t splits, piece;     // most pieces of a query's blocks, blocks of the largest (a multiple of 32)
    int32_t wanted;            // pieces that keep the SMs busy
    int32_t take;              // room for a piece's choices
};

// The words (32 blocks each) of a unit that hold a live row, as four runs in ascending order; the others
// are never looked at.
struct LiveWords {
    int32_t first[4], n[4], total;
    __device__ __forceinline__ LiveWords(const LiveRows &rows, int bs)
    {
        const int sh = 31 - __clz(32 * bs);
        int end = 0;                                       // one past the last word so far
        total = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i == 1 ? 2 : i == 2 ? 1 : i;     // pinned, the ring's wrapped piece, its other, pointers
            const int lo = max(end, (int)(rows.start[r] >> sh)), hi = (int)((rows.start[r] + rows.len[r] - 1) >> sh) + 1;
            first[i] = lo;
            n[i] = rows.len[r] > 0 ? max(0, hi - lo) : 0;
            if (rows.len[r] > 0) end = max(end, hi);
            total += n[i];
        }
    }
    __device__ __forceinline__ int at(int i) const         // the i-th of them
    {
        int w = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (i >= 0 && i < n[r]) w = first[r] + i;
            i -= n[r];
        }
        return w;
    }
};

// Words of a piece: what the pieces that are wanted leave for each, at most TC_BLOCKS blocks.
__device__ __forceinline__ int piece_words(const PickArgs &p, int total)
{
    const int pieces = max(p.wanted, (total + TC_BLOCKS / 32 - 1) / (TC_BLOCKS / 32));
    return max(1, (total + pieces - 1) / pieces);
}

// The blocks of a word that hold a live row, a bit each.
__device__ __forceinline__ uint32_t live_blocks(const LiveRows &rows, int bs, int word)
{
    const int sh = 31 - __clz(bs);
    uint64_t live = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (rows.len[r] == 0) continue;
        const int lo = max(0, (int)(rows.start[r] >> sh) - 32 * word);
        const int hi = min(31, (int)((rows.start[r] + rows.len[r] - 1) >> sh) - 32 * word);
        if (lo <= hi) live |= (2ull << hi) - (1ull << lo);
    }
    return (uint32_t)live;
}

// Four signed bytes of w as two fp16 pairs: a byte u on top of 0x6400 is 1024 + u exactly, u = x + 128.
__device__ __forceinline__ void bytes_to_fp16(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    w ^= 0x80808080u;
    asm("{\n\t.reg .b32 a;\n\tprmt.b32 a, %1, 0x64646464, 0x4140;\n\tsub.rn.f16x2 %0, a, %2;\n\t}" : "=r"(lo) : "r"(w), "r"(0x64806480u));
    asm("{\n\t.reg .b32 a;\n\tprmt.b32 a, %1, 0x64646464, 0x4342;\n\tsub.rn.f16x2 %0, a, %2;\n\t}" : "=r"(hi) : "r"(w), "r"(0x64806480u));
}

__device__ __forceinline__ void mma_fp16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t lanes_below()
{
    uint32_t m;
    asm("mov.u32 %0, %%lanemask_lt;" : "=r"(m));
    return m;
}

// A number that `want` of a warp's keys reach and no more than want + slack, or the largest that `want` reach where equal
// keys allow none: n_at_least(x) is how many keys are x or more (the same for all lanes), at least `want` are `low` or
// more, and none is `high` or more.  Halving the range ends after some steps where `low` is near.
template <typename F>
__device__ __forceinline__ uint32_t cut_at(int want, int slack, uint32_t low, uint32_t high, F n_at_least)
{
    while (high - low > 1u) {
        const uint32_t mid = low + (high - low) / 2u;
        const int n = n_at_least(mid);
        if (n >= want) low = mid;
        else high = mid;
        if (n >= want && n <= want + slack) break;
    }
    return low;
}

constexpr uint32_t LEAST_KEY = 0x00800000u;                // of -FLT_MAX: every live block's score reaches it

// Where the choices of a query go: the list itself, or a piece's candidates.
struct Choice {
    int32_t *sel;
    int2 *cand;
    __device__ __forceinline__ void put(int at, uint32_t key, int block) const
    {
        if (cand) cand[at] = make_int2((int)key, block);
        else sel[at] = block;
    }
};

// The `want` first of up to 64 (key, block) pairs in ascending block order, by (key desc, block asc): two to a lane,
// counted by ballots.  At least `want` keys are `low` or more, none is above `most`; key 0 is none.
__device__ __forceinline__ void choose_64(const int2 *pair, int n, int want, uint32_t low, uint32_t most, const Choice &out)
{
    const int lane = threadIdx.x & 31;
    const int2 e0 = lane < n ? pair[lane] : make_int2(0, 0), e1 = lane + 32 < n ? pair[lane + 32] : make_int2(0, 0);
    const uint32_t k0 = (uint32_t)e0.x, k1 = (uint32_t)e1.x;
    const auto ballots = [&](bool a, bool b) { return __popc(__ballot_sync(0xffffffffu, a)) + (n > 32 ? __popc(__ballot_sync(0xffffffffu, b)) : 0); };
    const uint32_t cut = n > want ? cut_at(want, 0, low, most + 1u, [&](uint32_t x) { return ballots(k0 >= x, k1 >= x); }) : 0u;
    // of those at the cut, the first
    const int ties = cut > 0u ? want - ballots(k0 > cut, k1 > cut) : 0;
    const uint32_t same0 = __ballot_sync(0xffffffffu, k0 == cut), same1 = __ballot_sync(0xffffffffu, k1 == cut);
    const bool take0 = k0 > cut || (k0 == cut && __popc(same0 & lanes_below()) < ties);
    const bool take1 = k1 > cut || (k1 == cut && __popc(same0) + __popc(same1 & lanes_below()) < ties);
    const uint32_t all0 = __ballot_sync(0xffffffffu, take0), all1 = __ballot_sync(0xffffffffu, take1);
    if (take0) out.put(__popc(all0 & lanes_below()), k0, e0.y);
    if (take1) out.put(__popc(all0) + __popc(all1 & lanes_below()), k1, e1.y);
}

// The `want` first of n (key, block) pairs in ascending block order, by (key desc, block asc); key 0 is none,
// and at least `want` are `low` or more.  The first 32 * HELD keys are held in registers.
template <int HELD, typename Load>
__device__ __forceinline__ void choose(int n, int want, uint32_t low, const Choice &out, Load load)
{
    const int lane = threadIdx.x & 31;
    uint32_t k[HELD], most = 0u;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        k[i] = 32 * i + lane < n ? (uint32_t)load(32 * i + lane).x : 0u;
        most = max(most, k[i]);
    }
    for (int i = 32 * HELD + lane; i < n; i += 32) most = max(most, (uint32_t)load(i).x);
    most = __reduce_max_sync(0xffffffffu, most);
    const auto n_at_least = [&](uint32_t x) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i) c += k[i] >= x;
        for (int i = 32 * HELD + lane; i < n; i += 32) c += (uint32_t)load(i).x >= x;
        return (int)__reduce_add_sync(0xffffffffu, c);
    };
    const uint32_t cut = n > want ? cut_at(want, 0, low, most + 1u, n_at_least) : 0u;
    int equal = n > want ? want - n_at_least(cut + 1u) : n, at = 0;
    for (int i0 = 0; i0 < n && at < want; i0 += 32) {
        const int i = i0 + lane;
        const int2 e = i < n ? load(i) : make_int2(0, 0);
        const uint32_t x = (uint32_t)e.x, same = __ballot_sync(0xffffffffu, x > 0 && x == cut);
        const bool take = x > 0 && (x > cut || (x == cut && __popc(same & lanes_below()) < equal));
        const uint32_t bal = __ballot_sync(0xffffffffu, take);
        if (take) out.put(at + __popc(bal & lanes_below()), x, e.y);
        at += __popc(bal);
        equal -= min(equal, __popc(same));
    }
}

// Where a word's i-th score lies in its query's row: fours of scores in an order of the word's own, so that lanes
// reading the same four of their words meet different banks.
__device__ __forceinline__ int score_at(int word, int i) { return 32 * word + (i ^ (4 * (word & 7))); }

template <typename T>
__global__ void __launch_bounds__(TC_THREADS, 3) k_score_blocks(PickArgs p)
{
    constexpr int N = 16 / sizeof(T);
    pdl_wait();
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ uint32_t s_live[TC_BLOCKS / 32];
    __shared__ int32_t s_word[TC_BLOCKS / 32];
    __shared__ int32_t s_size[2];                                          // words of this piece, whether there are others
    __shared__ int2 s_pair[TC_THREADS / 32][TC_HELD];
    __shared__ __align__(8) float s_step[TC_BLOCKS];                       // of the piece's blocks; NaN: no live row, it scores NaN
    const SparseArgs &s = p.a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tiles = (s.k_max + TC_ROWS - 1) / TC_ROWS;
    const int tile = blockIdx.x % tiles, split = blockIdx.x / tiles, h = blockIdx.y, u = blockIdx.z;
    // the first loads go out together: the unit's counts, the counters for the last warp, a cell for the others' lanes
    const int cnt = s.count[u], g = s.unit_group[u], j0 = tile * TC_ROWS;
    const int parts = s.d / N, L = min(32, parts), sub = lane & (L - 1), at_once = 32 / L, row0 = warp * at_once + lane / L;
    LiveRows rows;
    bool sane = true;
    int first_cell = 0;
    if (warp == TC_THREADS / 32 - 1) sane = rows.load(s.bank, u);
    else if (row0 < TC_ROWS && j0 + row0 < s.k_max) first_cell = __ldg(s.idx + (int64_t)u * s.k_max + j0 + row0);
    if (cnt < 0 || cnt > s.k_max || g < 0 || g >= s.G) {
        if (threadIdx.x == 0) latch_status(s.status, RS3_EINVAL);
        return;
    }
    const int nq = min(TC_ROWS, cnt - j0);
    if (nq <= 0) return;
    const int stride = p.piece + 8;                                        // of a query's scores
    float *s_score = reinterpret_cast<float *>(smem);
    const int width = s.d < 64 ? 64 : s.d, q_row = 2 * width + 16;         // columns, bytes of a query
    uint8_t *s_q = smem + TC_ROWS * stride * 4;
    const int r = lane >> 2, t = lane & 3;
    const int64_t dig = ((int64_t)u * s.H + h) * s.nb;
    if (warp == TC_THREADS / 32 - 1) {
        // the piece's words and the live blocks of each, a word per lane
        if (!sane && lane == 0) latch_status(s.status, RS3_EINTERNAL);
        const LiveWords words(rows, s.bs);
        const int per = piece_words(p, words.total);
        const int n = sane ? max(0, min(per, words.total - split * per)) : -1;
        if (lane < n) {
            const int word = words.at(split * per + lane);
            s_word[lane] = word;
            s_live[lane] = live_blocks(rows, s.bs, word);
        }
        if (lane == 0) {
            s_size[0] = n;
            s_size[1] = words.total > per;
            if (p.splits > 1 && tile == 0 && split == 0 && h == 0) p.n_pieces[u] = sane ? (words.total + per - 1) / per : 0;
        }
    } else {
        // the queries in 8 bits, held as fp16: a group of lanes per query, 16 bytes (up to two) each
        for (int r0 = warp * at_once; r0 < TC_ROWS; r0 += (TC_THREADS / 32 - 1) * at_once) {
            const int row = r0 + lane / L;                                 // rows past the tile: none of the lanes' groups writes
            const int cell = row == row0 ? first_cell : row < nq ? s.idx[(int64_t)u * s.k_max + j0 + row] : 0;
            const bool ok = row < nq && cell >= 0 && cell < s.mn;
            if (row < nq && !ok && sub == 0) latch_status(s.status, RS3_EINVAL);
            float x[2][N], m = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int c = sub + 32 * i;                                // its piece of the row
#pragma unroll
                for (int e = 0; e < N; ++e) x[i][e] = 0.f;
                if (i * 32 >= parts || !ok) continue;
                const uint4 w = __ldg(reinterpret_cast<const uint4 *>(static_cast<const T *>(s.q) + ((int64_t)g * s.mn + cell) * (s.H * s.d) + h * s.d) + c);
                const uint32_t y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (N == 8) {
                        x[i][2 * e] = __uint_as_float(y[e] << 16);
                        x[i][2 * e + 1] = __uint_as_float(y[e] & 0xffff0000u);
                    } else {
                        x[i][e] = __uint_as_float(y[e]);
                    }
                }
                if (s.rope) {                                              // each product and each sum rounded
#pragma unroll
                    for (int e = 0; e < N; e += 4) {
                        const float4 f = __ldg(reinterpret_cast<const float4 *>(s.rope + (int64_t)cell * s.d + c * N + e));
                        const float x0 = x[i][e], x1 = x[i][e + 1], x2 = x[i][e + 2], x3 = x[i][e + 3];
                        x[i][e] = __fsub_rn(__fmul_rn(x0, f.x), __fmul_rn(x1, f.y));
                        x[i][e + 1] = __fadd_rn(__fmul_rn(x0, f.y), __fmul_rn(x1, f.x));
                        x[i][e + 2] = __fsub_rn(__fmul_rn(x2, f.z), __fmul_rn(x3, f.w));
                        x[i][e + 3] = __fadd_rn(__fmul_rn(x2, f.w), __fmul_rn(x3, f.z));
                    }
                }
#pragma unroll
                for (int e = 0; e < N; ++e) m = fmaxf(m, fabsf(x[i][e]));
            }
            for (int o = L >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const EightBits bits(m);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (i * 32 >= parts || row >= TC_ROWS) continue;
                uint32_t w[N / 2];
#pragma unroll
                for (int e = 0; e < N; e += 2)
                    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[e / 2]) : "f"((float)bits(x[i][e + 1])), "f"((float)bits(x[i][e])));
                uint8_t *to = s_q + row * q_row + (sub + 32 * i) * 2 * N;
                if (N == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[N / 2 - 2], w[N / 2 - 1]);
                else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
            }
        }
        // heads of 16 and 32: the columns up to 64 are zeros
        for (int i = threadIdx.x; i < TC_ROWS * (width - s.d) / 8; i += TC_THREADS - 32) {
            const int row = i / ((width - s.d) / 8);
            *reinterpret_cast<uint4 *>(s_q + row * q_row + 2 * s.d + 16 * (i - row * ((width - s.d) / 8))) = make_uint4(0, 0, 0, 0);
        }
    }
    __syncthreads();
    if (s_size[0] < 0) return;
    const int n = 32 * s_size[0];                                          // places: blocks of the words, 32 each
    const bool alone = !s_size[1];
    // this warp's steps: 16 places, then 64 columns after 64; a step's digests are loaded two steps ahead
    int b0 = warp * 16, k0 = 0;
    uint4 w[2], w1[2];
    const uint8_t *digests = reinterpret_cast<const uint8_t *>(p.a.digest) + (dig * s.d + r * s.d + 16 * t);
    const auto load_step = [&](uint4 (&v)[2], int place, int k) {
        const int first = place < n ? s_word[place >> 5] * 32 + (place & 31) : s.nb;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            v[x] = make_uint4(0, 0, 0, 0);
            if (first + 8 * x + r < s.nb && k + 16 * t < s.d) v[x] = __ldg(reinterpret_cast<const uint4 *>(digests + (int64_t)(first + 8 * x) * s.d + k));
        }
    };
    const auto next_step = [&](int &b, int &k) {
        const bool more = k + 64 < width;
        b += more ? 0 : TC_THREADS / 2;
        k = more ? k + 64 : 0;
    };
    load_step(w, b0, k0);
    int b1 = b0, k1 = k0;
    next_step(b1, k1);
    load_step(w1, b1, k1);
    {
        // its places' steps: 16 after 128, four to a lane
        float f[TC_BLOCKS / 256 + 1];
#pragma unroll
        for (int i = 0; i < TC_BLOCKS / 256 + 1; ++i) {
            const int place = b0 + 256 * i + 128 * (lane >> 4) + (lane & 15);
            f[i] = place < n && (s_live[place >> 5] >> (place & 31) & 1u)
                       ? __ldg(p.a.step + dig + 32 * s_word[place >> 5] + (place & 31)) : __int_as_float(0x7fffffff);
        }
#pragma unroll
        for (int i = 0; i < TC_BLOCKS / 256 + 1; ++i) {
            const int place = b0 + 256 * i + 128 * (lane >> 4) + (lane & 15);
            if (place < n) s_step[place] = f[i];
        }
        __syncwarp();
    }
    float c[2][4];
    while (b0 < n) {
        if (k0 == 0) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) c[x][y] = 0.f;
        }
        int b2 = b1, k2 = k1;
        next_step(b2, k2);
        uint4 w2[2];
        load_step(w2, b2, k2);
        const uint8_t *qa = s_q + r * q_row + 2 * (k0 + 16 * t);
        uint4 qv[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) qv[x][y] = *reinterpret_cast<const uint4 *>(qa + 8 * x * q_row + 16 * y);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            uint32_t b[4][2];
            bytes_to_fp16(w[x].x, b[0][0], b[0][1]);
            bytes_to_fp16(w[x].y, b[1][0], b[1][1]);
            bytes_to_fp16(w[x].z, b[2][0], b[2][1]);
            bytes_to_fp16(w[x].w, b[3][0], b[3][1]);
            mma_fp16(c[x], qv[0][0].x, qv[1][0].x, qv[0][0].y, qv[1][0].y, b[0][0], b[0][1]);
            mma_fp16(c[x], qv[0][0].z, qv[1][0].z, qv[0][0].w, qv[1][0].w, b[1][0], b[1][1]);
            mma_fp16(c[x], qv[0][1].x, qv[1][1].x, qv[0][1].y, qv[1][1].y, b[2][0], b[2][1]);
            mma_fp16(c[x], qv[0][1].z, qv[1][1].z, qv[0][1].w, qv[1][1].w, b[3][0], b[3][1]);
        }
        if (k1 == 0) {
            // this lane holds places 8 x + 2 t, + 1 of queries r and r + 8
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float2 f = *reinterpret_cast<const float2 *>(s_step + b0 + 8 * x + 2 * t);
                float *to = s_score + r * stride + score_at(b0 >> 5, (b0 & 31) + 8 * x + 2 * t);
                *reinterpret_cast<float2 *>(to) = make_float2(c[x][0] * f.x, c[x][1] * f.y);
                *reinterpret_cast<float2 *>(to + 8 * stride) = make_float2(c[x][2] * f.x, c[x][3] * f.y);
            }
        }
        b0 = b1;
        k0 = k1;
        b1 = b2;
        k1 = k2;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            w[x] = w1[x];
            w1[x] = w2[x];
        }
    }
    __syncthreads();
    // a warp per query, a lane per word: blocks ascend with the lanes
    const int n_live = __reduce_add_sync(0xffffffffu, lane < s_size[0] ? __popc(s_live[lane]) : 0);
    const int want = min(s.n_top, n_live), word = lane < s_size[0] ? 32 * s_word[lane] : 0;
    for (int q = warp; q < nq; q += TC_THREADS / 32) {
        const int64_t row = ((int64_t)u * s.H + h) * s.k_max + j0 + q;
        const Choice out = {p.a.sel + row * s.n_top, alone ? nullptr : p.cand + (row * p.splits + split) * p.take};
        float *score = s_score + q * stride;
        float k[32];
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const float4 v = lane < s_size[0] ? *reinterpret_cast<const float4 *>(score + score_at(lane, i)) : make_float4(NAN, NAN, NAN, NAN);
            k[i] = v.x; k[i + 1] = v.y; k[i + 2] = v.z; k[i + 3] = v.w;
        }
        // a bound from the maxima of four blocks each (a NaN is passed over); where fewer of those hold a live block than are
        // wanted, all live blocks are candidates
        float g[8], best = -INFINITY;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            g[x] = fmaxf(fmaxf(k[4 * x], k[4 * x + 1]), fmaxf(k[4 * x + 2], k[4 * x + 3]));
            best = fmaxf(best, g[x]);
        }
        const auto groups = [&](uint32_t x) {
            const float f = score_of(x);
            int n = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) n += g[i] >= f;
            return (int)__reduce_add_sync(0xffffffffu, n);
        };
        const uint32_t most = __reduce_max_sync(0xffffffffu, best > -INFINITY ? order_bits(best) : 0u);
        uint32_t low = LEAST_KEY;
        if (want > 0) {
            // the least of the lanes' own maxima, if enough reach it, is a near lower end
            const uint32_t least = __reduce_min_sync(0xffffffffu, best > -INFINITY ? order_bits(best) : 0xffffffffu);
            if (groups(least) >= want) low = cut_at(want, 4, least, most + 1u, groups);
            else if (groups(LEAST_KEY) >= want) low = cut_at(want, 4, LEAST_KEY, least, groups);
        }
        const float bound = score_of(low);
        // the candidates as (key, block) pairs in block order
        uint32_t in = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i)
            asm("{\n\t.reg .pred p;\n\tsetp.ge.f32 p, %1, %2;\n\t@p or.b32 %0, %0, %3;\n\t}" : "+r"(in) : "f"(k[i]), "f"(bound), "r"(1u << i));
        const int mine = __popc(in);
        int end = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, end, o);
            if (lane >= o) end += x;
        }
        const int c = __shfl_sync(0xffffffffu, end, 31);
        if (want > 0 && c <= TC_HELD) {
            int2 *pair = s_pair[warp];
            __syncwarp();
            for (int at = end - mine; in != 0u; ++at, in &= in - 1u) {
                const int i = __ffs(in) - 1;
                pair[at] = make_int2((int)order_bits(score[score_at(lane, i)]), word + i);
            }
            __syncwarp();
            choose_64(pair, c, want, low, most, out);
        } else if (want > 0) {
            // the cut among all of the row's scores
#pragma unroll
            for (int i = 0; i < 32; ++i) k[i] = __uint_as_float(k[i] > -INFINITY ? order_bits(k[i]) : 0u);     // (NaN: 0)
            const auto n_at_least = [&](uint32_t x) {
                int n = 0;
#pragma unroll
                for (int i = 0; i < 32; ++i) n += __float_as_uint(k[i]) >= x;
                return (int)__reduce_add_sync(0xffffffffu, n);
            };
            const uint32_t cut = cut_at(want, 0, low, most + 1u, n_at_least);
            const int equal = want - n_at_least(cut + 1u);
            // per lane: how many lie above the cut and at it, and how many of the latter go to lower lanes
            int above = 0, same = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t x = __float_as_uint(k[i]);
                above += x > cut;
                same += x == cut && x > 0u;
            }
            int same_end = same;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, same_end, o);
                if (lane >= o) same_end += x;
            }
            int left = max(0, min(same, equal - (same_end - same)));       // of those at the cut, this lane's first ones
            int to = above + left;
            const int n = to;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, to, o);
                if (lane >= o) to += x;
            }
            to -= n;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t x = __float_as_uint(k[i]);
                const bool tie = x == cut && x > 0u && left > 0;
                left -= tie;
                if (x > cut || tie) out.put(to++, x, word + i);
            }
        }
        if (!alone) {
            if (lane == 0) p.n_cand[row * p.splits + split] = want;
        } else if (split == 0) {                           // no piece but this one
            for (int i = want + lane; i < s.n_top; i += 32) out.sel[i] = -1;
        }
    }
}

// The choices of a query's pieces joined: a warp per query.  The pieces follow one another, so their
// candidates are in ascending block order.
__global__ void __launch_bounds__(128) k_merge_blocks(PickArgs p, int room)
{
    pdl_wait();
    extern __shared__ int2 s_pairs[];                      // [4][room]
    const SparseArgs &s = p.a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int j = blockIdx.x * 4 + warp, h = blockIdx.y, u = blockIdx.z;
    const int cnt = s.count[u], g = s.unit_group[u];
    if (cnt < 0 || cnt > s.k_max || g < 0 || g >= s.G || j >= cnt) return;
    const int64_t row = ((int64_t)u * s.H + h) * s.k_max + j;
    const int pieces = p.n_pieces[u];
    if (pieces <= 1) return;                               // (its choices are the list; or the unit was refused)
    int2 *pair = s_pairs + warp * room;
    // places without a candidate hold key 0
    const int n = pieces * p.take;
    int some = 0;
#pragma unroll 4
    for (int i = lane; i < n; i += 32) {
        const int x = i / p.take;
        const bool on = i - x * p.take < p.n_cand[row * p.splits + x];
        const int2 e = p.cand[row * p.splits * p.take + i];
        pair[i] = on ? e : make_int2(0, 0);
        some += on;
    }
    some = __reduce_add_sync(0xffffffffu, some);
    __syncwarp();
    const int want = min(s.n_top, some);
    const Choice out = {p.a.sel + row * s.n_top, nullptr};
    if (want > 0 && n <= 64) choose_64(pair, n, want, 1u, 0xfffffffeu, out);
    else if (want > 0) choose<12>(n, want, 1u, out, [&](int i) { return pair[i]; });
    for (int i = want + lane; i < s.n_top; i += 32) out.sel[i] = -1;
}

// ---------------------------------------------------------------------------
// selection for many queries
// ---------------------------------------------------------------------------
constexpr int TILE_ROWS = 128;             // queries of a CTA
constexpr int TILE_THREADS = 256;          // a warp per 32 queries, three for the digests, one that issues
constexpr int TILE_COLS = 64;              // blocks of a tile: two words
constexpr int TILE_TOP = 32;               // most blocks per query
constexpr int TILE_WORDS = 512;            // most words of a unit

struct TileArgs {
    SelectArgs a;
    int32_t cap;               // room for a query's candidates: n_top + 48 at least
    uint64_t wait_ns;          // limit of each wait
};

// The blocks that hold a live row, as four runs.
struct LiveBlocks {
    int32_t first[4], last[4];
    __device__ __forceinline__ LiveBlocks(const LiveRows &rows, int bs)
    {
        const int sh = 31 - __clz(bs);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            first[r] = rows.len[r] > 0 ? (int)(rows.start[r] >> sh) : 0;
            last[r] = rows.len[r] > 0 ? (int)((rows.start[r] + rows.len[r] - 1) >> sh) : -1;
        }
    }
    __device__ __forceinline__ bool holds(int b) const
    {
        bool in = false;
#pragma unroll
        for (int r = 0; r < 4; ++r) in |= b >= first[r] && b <= last[r];
        return in;
    }
};

// A lane's run of floats in shared memory, -infinity behind the last; runs begin an odd number of 16 bytes apart, so
// lanes that read the same four of theirs meet different banks.
struct Column {
    float *v;

    __device__ __forceinline__ void clear(int from, int to) const
    {
        for (; from < to && (from & 3) != 0; ++from) v[from] = -INFINITY;
        for (; from < to; from += 4) *reinterpret_cast<float4 *>(v + from) = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    }

    // how many are x or more, among the first `most` (the same for the warp)
    __device__ __forceinline__ int at_least(float x, int most) const
    {
        int c[4] = {0, 0, 0, 0};
#pragma unroll 4
        for (int i = 0; i < most; i += 4) {
            const float4 y = *reinterpret_cast<const float4 *>(v + i);
            c[0] += y.x >= x;
            c[1] += y.y >= x;
            c[2] += y.z >= x;
            c[3] += y.w >= x;
        }
        return (c[0] + c[1]) + (c[2] + c[3]);
    }
};

// Bitonic networks in registers, without a branch: a full sort of 32, and the merge of a bitonic run, descending.
__device__ __forceinline__ void merge_down_32(float (&x)[32])
{
#pragma unroll
    for (int lj = 4; lj >= 0; --lj)
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            const int i = (n >> lj) << (lj + 1) | (n & ((1 << lj) - 1)), j = i + (1 << lj);
            const float hi = fmaxf(x[i], x[j]), lo = fminf(x[i], x[j]);
            x[i] = hi;
            x[j] = lo;
        }
}

__device__ __forceinline__ void sort_32(float (&x)[32])
{
#pragma unroll
    for (int lk = 1; lk <= 5; ++lk)
#pragma unroll
        for (int lj = lk - 1; lj >= 0; --lj)
#pragma unroll
            for (int n = 0; n < 16; ++n) {
                // the n-th pair 2^lj apart, descending where bit lk of the first is 0
                const int i = (n >> lj) << (lj + 1) | (n & ((1 << lj) - 1)), j = i + (1 << lj);
                const float hi = fmaxf(x[i], x[j]), lo = fminf(x[i], x[j]);
                x[i] = (i >> lk & 1) == 0 ? hi : lo;
                x[j] = (i >> lk & 1) == 0 ? lo : hi;
            }
}

// The want-th largest (from 1, at most 32) of the first `most` of a column: 32 after 32 are sorted and merged into the 32
// largest so far, some 21 instructions for each of 32 queries' entries.  A search by halving, which goes on
// for the slowest lane, took five times as long.
__device__ __forceinline__ float nth_largest(const Column &c, int most, int want)
{
    float top[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) top[i] = -INFINITY;
    for (int i0 = 0; i0 < most; i0 += 32) {
        float x[32];
#pragma unroll
        for (int i = 0; i < 32; i += 4) {                  // (a column ends at a multiple of four)
            const float4 t = i0 + i < most ? *reinterpret_cast<const float4 *>(c.v + i0 + i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            x[i] = t.x; x[i + 1] = t.y; x[i + 2] = t.z; x[i + 3] = t.w;
        }
        sort_32(x);
#pragma unroll
        for (int i = 0; i < 32; ++i) top[i] = fmaxf(top[i], x[31 - i]);
        merge_down_32(top);
    }
    float y = top[0];
#pragma unroll
    for (int i = 1; i < 32; ++i)                           // (chosen like this, the array stays in registers)
        asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %2, %3;\n\t@p mov.f32 %0, %1;\n\t}" : "+f"(y) : "f"(top[i]), "r"(want), "r"(i + 1));
    return y;
}

// Candidates of a lane's query in block order.
struct Candidates {
    Column score;
    uint16_t *block;
    int n;

    // Cuts down the lanes that hold more than `want` to the best by (score desc, block asc); for those the key of the
    // want-th, else `low`.
    __device__ __forceinline__ uint32_t cut(int want, uint32_t low)
    {
        const bool over = n > want;
        const int most = __reduce_max_sync(0xffffffffu, over ? n : 0);
        if (most == 0) return low;
        const uint32_t key = order_bits(nth_largest(score, most, want));
        const float x = score_of(key);
        // of those that equal it, the first stay
        int ties = want - score.at_least(score_of(key + 1u), most);
        // four at a time, predicated: what stays moves down, in order
        const uint32_t first = static_cast<uint32_t>(__cvta_generic_to_shared(score.v));
        uint32_t at = first, at_block = static_cast<uint32_t>(__cvta_generic_to_shared(block));
        for (int i = 0; i < most; i += 4) {
            const float4 t = *reinterpret_cast<const float4 *>(score.v + i);
            const float y[4] = {t.x, t.y, t.z, t.w};
            const uint2 b = *reinterpret_cast<const uint2 *>(block + i);
            const uint16_t id[4] = {(uint16_t)b.x, (uint16_t)(b.x >> 16), (uint16_t)b.y, (uint16_t)(b.y >> 16)};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool tie = y[e] == x, in = over && (y[e] > x || (tie && ties > 0));
                ties -= tie;
                asm volatile("{\n\t.reg .pred p;\n\t"
                             "setp.ne.s32 p, %2, 0;\n\t"
                             "@p st.shared.f32 [%0], %3;\n\t"
                             "@p st.shared.u16 [%1], %4;\n\t"
                             "@p add.u32 %0, %0, 4;\n\t"
                             "@p add.u32 %1, %1, 2;\n\t}"
                             : "+r"(at), "+r"(at_block) : "r"((int)in), "f"(y[e]), "h"(id[e]) : "memory");
            }
        }
        const int to = (int)(at - first) >> 2;
        if (!over) return low;
        score.clear(to, n);
        n = to;
        return key;
    }
};

// A CTA takes 128 queries of a head and its blocks in tiles of 64, twice; tcgen05 gives the scores, a query per lane of
// tensor memory, and a thread goes through its query's scores by itself.
//   first pass   the maxima of groups of blocks (8 or more).  The n_top-th largest of them is a bound that n_top scores or
//                few more reach, whatever the blocks' order.
//   second pass  the scores that reach the bound, in block order, as candidates in shared memory; where they are too
//                many (ties, or fewer groups than choices), they are cut down and the bound rises.
// Then the candidates are cut to n_top.  Three warps spread the digests (fp16, 128-byte swizzle) a tile ahead, one issues
// the products.  Per query this takes a third of k_score_blocks' instructions, but a CTA goes through all of the
// blocks twice, so it is for calls whose queries fill the SMs: 23 264 queries over 990 blocks 65 us against 93, 757 over
// 4 700 the other way round (74 against 46).  A step of 64 blocks takes some 1 600 cycles in the first pass and 2 100 in the
// second, where a score's predicated stores fill the shared memory's pipe; the digests are there in time.  The maxima take
// the whole of the warp's part of shared memory: in groups of 16 blocks where 8 have room, 16 choices took 70 us and
// 32 took 163 instead of 92, as two of a group's blocks are often among the best.
template <typename T>
__global__ void __launch_bounds__(TILE_THREADS, 2) k_score_tiles(TileArgs p)
{
    using namespace tc;
    constexpr int N = 16 / sizeof(T), ISSUER = 7;           // warps 0 to 3: queries, 4 to 6: digests
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_bars[9];
    __shared__ __align__(16) float s_step[2][TILE_COLS];
    __shared__ int32_t s_word[TILE_WORDS + 4];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const SparseArgs &s = p.a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    const int h = blockIdx.y, u = blockIdx.z;
    int cnt, g;
    LiveRows rows;
    if (!sparse_unit(s, u, threadIdx.x == 0, cnt, g, rows)) return;
    const int j0 = blockIdx.x * TILE_ROWS, nq = min(TILE_ROWS, cnt - j0);
    if (nq <= 0) return;
    const LiveWords words(rows, s.bs);
    const int n_words = words.total;
    if (n_words == 0) {                                    // nothing to choose from
        const int64_t row0 = ((int64_t)u * s.H + h) * s.k_max + j0;
        for (int i = threadIdx.x; i < nq * s.n_top; i += TILE_THREADS) p.a.sel[row0 * s.n_top + i] = -1;
        return;
    }
    const int n_tiles = (n_words + 1) / 2;

    // shared memory: queries [128] and two tiles' digests [64], fp16, in 64-column blocks; then the candidates
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw);
    const int width = s.d < 64 ? 64 : s.d, q_bytes = TILE_ROWS * 2 * width, b_bytes = TILE_COLS * 2 * width;
    uint8_t *s_b = smem + q_bytes;
    const int cap = p.cap;
    // a query warp's part: its lanes' candidates, scores then blocks; before those the maxima, in longer runs
    float *s_mine = reinterpret_cast<float *>(s_b + 2 * b_bytes + (warp & 3) * 32 * cap * 6), *s_cand = s_mine + lane * cap;
    uint16_t *s_block = reinterpret_cast<uint16_t *>(s_mine + 32 * cap) + lane * cap;
    const uint32_t bars = smem_u32(s_bars);
    const uint32_t SFULL = bars, SFREE = bars + 16, BFULL = bars + 32, BFREE = bars + 48, DRAIN = bars + 64;
    volatile int *abort_flag = &s_abort;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(SFULL + 8 * i, 2);                   // the commit, and the issuing thread for the steps
            mbar_init(SFREE + 8 * i, 4);
            mbar_init(BFULL + 8 * i, 3);
            mbar_init(BFREE + 8 * i, 1);
        }
        mbar_init(DRAIN, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    if (warp == ISSUER) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(2 * TILE_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // the words; none behind the last
    for (int i = threadIdx.x; i < 2 * n_tiles; i += TILE_THREADS) s_word[i] = i < n_words ? 32 * words.at(i) : -1;
    if (s.d < 64)                                          // the columns up to 64 are zeros
        for (int i = threadIdx.x; i < (TILE_ROWS + 2 * TILE_COLS) * 8; i += TILE_THREADS) *reinterpret_cast<uint4 *>(smem + 16 * i) = make_uint4(0, 0, 0, 0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    {
        // the queries in 8 bits, 16 per warp: a group of lanes per query, 16 bytes each; four groups' rows
        // are loaded together
        const int parts = s.d / N, L = min(32, parts), sub = lane & (L - 1), at_once = 32 / L, first = 16 * warp;
        const int my_cell = (lane < 16 && first + lane < nq) ? s.idx[(int64_t)u * s.k_max + j0 + first + lane] : -1;
        if (lane < 16 && first + lane < nq && (my_cell < 0 || my_cell >= s.mn)) latch_status(s.status, RS3_EINVAL);
        const T *grid = static_cast<const T *>(s.q) + (int64_t)g * s.mn * (s.H * s.d) + h * s.d;
        constexpr int F = 4;
        for (int r0 = 0; r0 < 16; r0 += F * at_once) {
            uint4 v[F];
            float4 f[F][N / 4];
#pragma unroll
            for (int x = 0; x < F; ++x) {
                const int row = r0 + x * at_once + lane / L, cell = __shfl_sync(0xffffffffu, my_cell, row & 15);
                v[x] = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < N / 4; ++e) f[x][e] = make_float4(1.f, 0.f, 1.f, 0.f);
                if (row >= 16 || cell < 0 || cell >= s.mn) continue;
                v[x] = __ldg(reinterpret_cast<const uint4 *>(grid + (int64_t)cell * (s.H * s.d)) + sub);
                if (s.rope)
#pragma unroll
                    for (int e = 0; e < N / 4; ++e) f[x][e] = __ldg(reinterpret_cast<const float4 *>(s.rope + (int64_t)cell * s.d + sub * N) + e);
            }
#pragma unroll
            for (int x = 0; x < F; ++x) {
                const int row = r0 + x * at_once + lane / L;
                const uint32_t y[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
                float z[N], m = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (N == 8) {
                        z[2 * e] = __uint_as_float(y[e] << 16);
                        z[2 * e + 1] = __uint_as_float(y[e] & 0xffff0000u);
                    } else {
                        z[e] = __uint_as_float(y[e]);
                    }
                }
                if (s.rope) {                              // each product and each sum rounded
#pragma unroll
                    for (int e = 0; e < N; e += 4) {
                        const float4 t = f[x][e / 4];
                        const float x0 = z[e], x1 = z[e + 1], x2 = z[e + 2], x3 = z[e + 3];
                        z[e] = __fsub_rn(__fmul_rn(x0, t.x), __fmul_rn(x1, t.y));
                        z[e + 1] = __fadd_rn(__fmul_rn(x0, t.y), __fmul_rn(x1, t.x));
                        z[e + 2] = __fsub_rn(__fmul_rn(x2, t.z), __fmul_rn(x3, t.w));
                        z[e + 3] = __fadd_rn(__fmul_rn(x2, t.w), __fmul_rn(x3, t.z));
                    }
                }
#pragma unroll
                for (int e = 0; e < N; ++e) m = fmaxf(m, fabsf(z[e]));
                for (int o = L >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                const EightBits bits(m);
                if (row >= 16) continue;
                uint32_t w[N / 2];
#pragma unroll
                for (int e = 0; e < N; e += 2)
                    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[e / 2]) : "f"((float)bits(z[e + 1])), "f"((float)bits(z[e])));
                // N fp16 columns: a chunk of 8, or half of one
                uint8_t *to = smem + sw128_offset(TILE_ROWS, first + row, sub * N / 8) + (N == 8 ? 0 : (sub & 1) * 8);
                if (N == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[N / 2 - 2], w[N / 2 - 1]);
                else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
            }
        }
        fence_proxy_async();
    }
    __syncthreads();

    // step k: tile k mod n_tiles, scores and digests in buffer k mod 2
    if (warp >= 4 && warp < ISSUER) {
        // digests: pieces of 16 bytes, a word's 2 d after the other's, loaded a step ahead
        constexpr int CONVERT = 96, MOST = (4 * 128 + CONVERT - 1) / CONVERT;
        const int pt = threadIdx.x - 128, n_pieces = 4 * s.d, sh = 31 - __clz(s.d / 16), n_x = (n_pieces + CONVERT - 1) / CONVERT;
        const uint8_t *digests = reinterpret_cast<const uint8_t *>(p.a.digest) + ((int64_t)u * s.H + h) * s.nb * s.d;
        uint4 v[MOST];
        const auto load_tile = [&](int i) {
            const int word[2] = {s_word[2 * i], s_word[2 * i + 1]};
#pragma unroll
            for (int x = 0; x < MOST; ++x) {
                if (x >= n_x) break;
                const int e = pt + CONVERT * x, second = e >= 2 * s.d;
                const int first = second ? word[1] : word[0], b = first + ((e >> sh) & 31);
                v[x] = make_uint4(0, 0, 0, 0);
                if (e < n_pieces && first >= 0 && b < s.nb)
                    v[x] = __ldg(reinterpret_cast<const uint4 *>(digests + (int64_t)first * s.d + 16 * (e - (second ? 2 * s.d : 0))));
            }
        };
        load_tile(0);
        for (int k = 0, i = 0; k < 2 * n_tiles; ++k) {
            const uint32_t buf = k & 1, ph = k >> 1 & 1;
            if (!mbar_wait_warp(BFREE + 8 * buf, ph ^ 1u, abort_flag, p.wait_ns)) break;
#pragma unroll
            for (int x = 0; x < MOST; ++x) {
                const int e = pt + CONVERT * x;
                if (x >= n_x) break;
                if (e >= n_pieces) continue;
                const int row = e >> sh, ch = 2 * (e & ((1 << sh) - 1));
                uint32_t w[8];
                bytes_to_fp16(v[x].x, w[0], w[1]);
                bytes_to_fp16(v[x].y, w[2], w[3]);
                bytes_to_fp16(v[x].z, w[4], w[5]);
                bytes_to_fp16(v[x].w, w[6], w[7]);
                *reinterpret_cast<uint4 *>(s_b + buf * b_bytes + sw128_offset(TILE_COLS, row, ch)) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4 *>(s_b + buf * b_bytes + sw128_offset(TILE_COLS, row, ch + 1)) = make_uint4(w[4], w[5], w[6], w[7]);
            }
            i = i + 1 == n_tiles ? 0 : i + 1;
            if (k + 1 < 2 * n_tiles) load_tile(i);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(BFULL + 8 * buf);
        }
    } else if (warp == ISSUER) {
        // steps of the tile's blocks (a block without a live row scores NaN: it reaches nothing), and the products
        const LiveBlocks live(rows, s.bs);
        const float *steps = p.a.step + ((int64_t)u * s.H + h) * s.nb;
        const auto step_of = [&](int word) {
            const int b = word + lane;
            return word >= 0 && b < s.nb && live.holds(b) ? __ldg(steps + b) : __int_as_float(0x7fffffff);
        };
        float step[2] = {step_of(s_word[0]), step_of(s_word[1])};
        constexpr uint32_t ID = (1u << 4) | ((uint32_t)(TILE_COLS >> 3) << 17) | ((uint32_t)(TILE_ROWS >> 4) << 24);   // fp16 in, fp32 out
        const uint64_t dq = desc_sw128((uint32_t)uniform((int)base), 16, 1024);
        const uint32_t tm = (uint32_t)uniform((int)tmem);
        for (int k = 0, i = 0; k < 2 * n_tiles; ++k) {
            const uint32_t buf = k & 1, ph = k >> 1 & 1;
            // the buffer's last scores have been read, and with them its steps
            if (!mbar_wait_warp(SFREE + 8 * buf, ph ^ 1u, abort_flag, p.wait_ns)) break;
            s_step[buf][lane] = step[0];
            s_step[buf][lane + 32] = step[1];
            i = i + 1 == n_tiles ? 0 : i + 1;
            if (k + 1 < 2 * n_tiles) {
                step[0] = step_of(s_word[2 * i]);
                step[1] = step_of(s_word[2 * i + 1]);
            }
            __syncwarp();
            if (!mbar_wait_warp(BFULL + 8 * buf, ph, abort_flag, p.wait_ns)) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t db = desc_sw128(base + (uint32_t)q_bytes + buf * (uint32_t)b_bytes, 16, 1024);
#pragma unroll 4
                for (int kk = 0; kk < width / 16; ++kk) {
                    const uint32_t oq = (uint32_t)((kk >> 2) * (TILE_ROWS * 128) + (kk & 3) * 32), ob = (uint32_t)((kk >> 2) * (TILE_COLS * 128) + (kk & 3) * 32);
                    tc_mma(tm + TILE_COLS * buf, dq + (oq >> 4), db + (ob >> 4), ID, kk > 0 ? 1u : 0u);
                }
                tc_commit(SFULL + 8 * buf);
                tc_commit(BFREE + 8 * buf);
                mbar_arrive(SFULL + 8 * buf);
            }
            __syncwarp();
        }
        if (elect_one()) {                                 // every product is done before the tensor memory goes
            tc_commit(DRAIN);
            mbar_drain(DRAIN, 0);
        }
        __syncwarp();
    } else {
        const int q = threadIdx.x;
        const bool mine = q < nq, busy = (q & ~31) < nq;
        const uint32_t tl = tmem + ((uint32_t)(q & ~31) << 16);
        const int places = TILE_COLS * n_tiles;
        const int most_maxima = ((cap * 3 / 2 / 4 - 1) | 1) * 4;      // an odd number of 16 bytes
        int blocks = 8;                                    // blocks of a maximum
        while (places > blocks * most_maxima) blocks *= 2;
        const int n_maxima = (places + blocks - 1) / blocks;
        const Column maxima = {s_mine + lane * most_maxima};
        Candidates c = {{s_cand}, s_block, 0};
        maxima.clear(0, most_maxima);
        // waits for the next scores and loads them, times their blocks' steps
        uint32_t x[TILE_COLS];
        int k = 0;
        const auto next = [&]() {
            const uint32_t buf = k & 1, ph = k >> 1 & 1;
            ++k;
            if (!mbar_wait_warp(SFULL + 8 * buf, ph, abort_flag, p.wait_ns)) return false;
            tc_fence_after();
            if (busy) {
                tmem_ld_cols<TILE_COLS>(tl + TILE_COLS * buf, x);
                tmem_wait_ld();
#pragma unroll
                for (int b = 0; b < TILE_COLS; b += 4) {
                    const float4 f = *reinterpret_cast<const float4 *>(&s_step[buf][b]);
                    x[b] = __float_as_uint(__uint_as_float(x[b]) * f.x);
                    x[b + 1] = __float_as_uint(__uint_as_float(x[b + 1]) * f.y);
                    x[b + 2] = __float_as_uint(__uint_as_float(x[b + 2]) * f.z);
                    x[b + 3] = __float_as_uint(__uint_as_float(x[b + 3]) * f.w);
                }
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(SFREE + 8 * buf);
            return true;
        };
        // first pass: the maxima (fmaxf passes over NaN)
        bool ok = true;
        float top = -INFINITY;
        int at_max = 0;
        for (int i = 0; i < n_tiles && ok; ++i) {
            ok = next();
            if (!ok || !busy) continue;
#pragma unroll
            for (int b = 0; b < TILE_COLS; b += 8) {
                float m[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) m[e] = fmaxf(__uint_as_float(x[b + e]), __uint_as_float(x[b + 4 + e]));
                top = fmaxf(top, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
                if (((TILE_COLS * i + b + 8) & (blocks - 1)) == 0) {
                    maxima.v[at_max++] = top;
                    top = -INFINITY;
                }
            }
        }
        if (busy && (places & (blocks - 1)) != 0) maxima.v[at_max] = top;
        // the bound: the n_top-th largest of the maxima, which n_top scores reach; where fewer maxima hold a live block, every
        // live one's score
        float bound = INFINITY;
        uint32_t low = LEAST_KEY;
        if (ok && busy) {
            const float nth = nth_largest(maxima, n_maxima, s.n_top);
            __syncwarp();                                  // (the lanes' maxima are read: candidates take their place)
            if (nth > -INFINITY) low = order_bits(nth);
            if (mine) bound = score_of(low);
            c.score.clear(0, cap);
        }
        // second pass: the candidates
        uint32_t at = smem_u32(s_cand), at_block = smem_u32(s_block);
        for (int i = 0; i < n_tiles && ok; ++i) {
            ok = next();
            if (!ok || !busy) continue;
#pragma unroll
            for (int word = 0; word < TILE_COLS / 32; ++word) {
                const uint32_t first = (uint32_t)s_word[2 * i + word];
#pragma unroll
                for (int b = 0; b < 32; ++b) {
                    // predicated, as a branch per score would cost more than the stores
                    const uint16_t block = (uint16_t)(first + b);
                    asm volatile("{\n\t.reg .pred p;\n\t"
                                 "setp.ge.f32 p, %2, %3;\n\t"
                                 "@p st.shared.f32 [%0], %2;\n\t"
                                 "@p st.shared.u16 [%1], %4;\n\t"
                                 "@p add.u32 %0, %0, 4;\n\t"
                                 "@p add.u32 %1, %1, 2;\n\t}"
                                 : "+r"(at), "+r"(at_block) : "f"(__uint_as_float(x[32 * word + b])), "f"(bound), "h"(block) : "memory");
                }
                c.n = (int)(at - smem_u32(s_cand)) >> 2;
                if (__any_sync(0xffffffffu, c.n > cap - 32)) {
                    const bool over = c.n > s.n_top;
                    low = c.cut(s.n_top, low);
                    if (over) bound = score_of(low + 1u);  // later blocks have to be better
                    at = smem_u32(s_cand) + 4u * c.n;
                    at_block = smem_u32(s_block) + 2u * c.n;
                }
            }
        }
        if (ok && busy) {
            // the choices: the candidates above the n_top-th largest, and of those that equal it the first
            const int most = __reduce_max_sync(0xffffffffu, c.n);
            float cut = -FLT_MAX;
            int ties = c.n;
            if (most > s.n_top) {
                const uint32_t key = order_bits(nth_largest(c.score, most, s.n_top));
                const int above = c.score.at_least(score_of(key + 1u), most);
                if (c.n > s.n_top) {
                    cut = score_of(key);
                    ties = s.n_top - above;
                }
            }
            if (mine) {
                int32_t *out = p.a.sel + (((int64_t)u * s.H + h) * s.k_max + j0 + q) * s.n_top;
                int to = 0;
#pragma unroll 4
                for (int e = 0; e < c.n; ++e) {
                    const float y = s_cand[e];
                    const bool tie = y == cut, take = y > cut || (tie && ties > 0);
                    ties -= tie;
                    if (take) out[to++] = s_block[e];
                }
                for (; to < s.n_top; ++to) out[to] = -1;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == ISSUER) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * TILE_COLS));
    if (threadIdx.x == 0 && *abort_flag) latch_status(s.status, RS3_ETIMEOUT);
}

// Pieces of a query's blocks: as many as their size needs, more where that leaves SMs idle.
int64_t select_splits(int64_t U, int64_t H, int64_t k_max, int64_t nb, int64_t n_top, int64_t sms, int64_t &wanted)
{
    const int64_t tiles = U * H * ((k_max + TC_ROWS - 1) / TC_ROWS), least = (nb + TC_BLOCKS - 1) / TC_BLOCKS;
    wanted = tiles > 0 ? (4 * sms + tiles - 1) / tiles : 1;
    if (wanted > nb / 512) wanted = nb / 512;
    if (wanted > TC_PAIRS / n_top) wanted = TC_PAIRS / n_top;      // 50 x 64 at the most blocks and choices
    if (wanted < 1) wanted = 1;
    return wanted > least ? wanted : least > 0 ? least : 1;
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
    a.visits = refresh < 0 ? nb : most > nb + 8 ? nb + 8 : most;
    const bool wide = bank->dtype == RS3_F32 && d == 256;
    const int pieces = wide ? 64 : 32;
    const int64_t slabs = (a.row_bytes / 16 + pieces - 1) / pieces;
    if (slabs > 65535) return RS3_EUNSUPPORTED;
    const int64_t rows = bank->U * bank->rows_per_unit;
    if (rows >= (1ll << 31) - 256) return RS3_EUNSUPPORTED;    // tensor maps take 32-bit rows
    a.wait_ns = rs3_get_wait_limit_ns();
    CUtensorMap map;
    const int es = (int)elem_bytes(bank->dtype), cols = (int)(a.row_bytes < pieces * 16 ? a.row_bytes : pieces * 16) / es;
    if (!tc::make_rows_map(&map, bank->k_store, es, bank->D, rows, cols, wide ? 8 : 16)) return RS3_ECUDA;
    // a CTA per SM in all, a block per warp at least
    int64_t x = (rs3_sm_count() + slabs * bank->U - 1) / (slabs * bank->U);
    if (x > (a.visits + DIGEST_WARPS - 1) / DIGEST_WARPS) x = (a.visits + DIGEST_WARPS - 1) / DIGEST_WARPS;
    const dim3 grid((unsigned)x, (unsigned)slabs, (unsigned)bank->U);
    void (*kern)(DigestArgs, CUtensorMap) = bank->dtype == RS3_BF16 ? k_digest<uint16_t, 1> : wide ? k_digest<float, 2> : k_digest<float, 1>;
    const size_t smem = (size_t)DIGEST_WARPS * 2 * 8192 + 128;
    const rs3_status r = rs3_kernel_smem((const void *)kern, smem);
    if (r != RS3_OK) return r;
    launch_pdl(kern, grid, dim3(32 * DIGEST_WARPS), smem, reinterpret_cast<cudaStream_t>(stream), a, map);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}

extern "C" size_t rs3_block_select_workspace_bytes(int U, int H, int k_max, int n_blocks)
{
    if (U < 1 || H < 1 || k_max < 0 || n_blocks < 0) return 0;
    // rows x pieces: beyond what the blocks need, pieces only fill up four CTAs of 16 rows per SM
    const size_t rows = (size_t)U * (size_t)H * (size_t)k_max, least = ((size_t)n_blocks + TC_BLOCKS - 1) / TC_BLOCKS;
    const size_t pieces = 8 * TC_SMS * TC_ROWS + (least > 1 ? rows * (least + 1) : 0);
    return 256 + align_up((pieces + (size_t)U) * 4, 256) + pieces * TC_TOP * sizeof(int2);
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
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    a.digest = digest;
    a.step = step;
    a.sel = sel;
    a.bf16 = dtype == RS3_BF16;
    // 128 queries to a CTA, where those are at least one per SM and their candidates have room; the more choices, the more
    // candidates are cut down again, and the more tiles it takes.  Tiles are counted by k_max, as the counts are on the device.
    // Heads of 64 with all of k_max kept / with three fifths of it kept, L2 flushed, us (128 queries to a CTA : 16):
    //   blocks   choices   48 tiles   80, 96             160, 192            240       320, 384             640 (heads of 32)
    //   990      16        50 : 36    50 : 59, 56 : 37   64 : 101, 62 : 56   64 : 72   101 : 189, 70 : 99   107 : 184
    //   990      24        62 : 39    62 : 63            78 : 109, 79 : 60   83 : 76   130 : 201, 101 : 105 144 : 193
    //   990      32        70 : 44    72 : 70, 100 : 48  109 : 126, 111 : 66 117 : 85  165 : 238, 154 : 119 222 : 213
    //   4 500    16                   183 : 148, 181 : 101  228 : 277, 181 : 185  218 : 263  224 : 353      380 : 690
    //   4 500    24                   197 : 154          273 : 291, 199 : 193  236 : 273  261 : 369          433 : 720
    //   4 500    32                   236 : 163, 228 : 116  363 : 310, 236 : 205  302 : 292  361 : 396      566 : 752
    // Over 325 blocks 160 tiles 31 : 33 (16 choices), 320 tiles 60 : 54 (24).  Heads of 128, 4 choices, 990 blocks: 80 tiles 56 : 42,
    // 160 tiles 58 : 68, 320 tiles 74 : 115; of 16, 160 tiles, 16 choices 56 : 58; fp32 as bf16.
    const int fixed = (TILE_ROWS + 2 * TILE_COLS) * 2 * (d < 64 ? 64 : d) + 1024, each = TILE_ROWS * 6;
    const int cap = (((106 * 1024 - fixed) / each / 4 - 1) | 1) * 4;       // an odd number of 16 bytes
    const int64_t tiles = (int64_t)a.s.U * H * ((k_max + TILE_ROWS - 1) / TILE_ROWS);
    if (4 * tiles >= (int64_t)rs3_sm_count() * (n_top <= 16 ? 4 : n_top <= 24 ? 5 : 10) && n_top <= TILE_TOP && cap >= n_top + 48 &&
        a.s.nb <= 32 * TILE_WORDS) {
        TileArgs p = {a, cap, rs3_get_wait_limit_ns()};
        const size_t smem = (size_t)fixed + (size_t)cap * each;
        void (*kern)(TileArgs) = dtype == RS3_BF16 ? k_score_tiles<uint16_t> : k_score_tiles<float>;
        const rs3_status r = rs3_kernel_smem((const void *)kern, smem);
        if (r != RS3_OK) return r;
        launch_pdl(kern, dim3((unsigned)((k_max + TILE_ROWS - 1) / TILE_ROWS), (unsigned)H, (unsigned)a.s.U), dim3(TILE_THREADS), smem, st, p);
        return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
    }
    const int sms = rs3_sm_count() < (int)TC_SMS ? rs3_sm_count() : (int)TC_SMS;
    int64_t wanted, splits = select_splits(a.s.U, H, k_max, a.s.nb, n_top, sms, wanted);
    if (n_top > TC_TOP && a.s.nb <= TC_BLOCKS) splits = wanted = 1;
    if (splits == 1 || n_top <= TC_TOP) {
        PickArgs p = {};
        p.a = a;
        p.splits = (int32_t)splits;
        p.wanted = (int32_t)wanted;
        // blocks of the largest piece that piece_words() can ask for
        const int64_t words = (a.s.nb + 31) / 32, per = (words + wanted - 1) / wanted;
        p.piece = (int32_t)(32 * (per < 1 ? 1 : per < TC_BLOCKS / 32 ? per : TC_BLOCKS / 32));
        p.take = n_top < p.piece ? n_top : p.piece;
        const int64_t pieces = (int64_t)a.s.U * H * k_max * splits;
        p.n_cand = static_cast<int32_t *>(workspace);
        p.n_pieces = p.n_cand + pieces;
        p.cand = reinterpret_cast<int2 *>(static_cast<uint8_t *>(workspace) + align_up((size_t)(pieces + a.s.U) * 4, 256));
        const size_t smem = (size_t)TC_ROWS * ((size_t)(p.piece + 8) * 4 + 2 * (d < 64 ? 64 : d) + 16);
        void (*kern)(PickArgs) = dtype == RS3_BF16 ? k_score_blocks<uint16_t> : k_score_blocks<float>;
        rs3_status r = rs3_kernel_smem((const void *)kern, smem + 16 * 1024);      // (its own static arrays count too)
        if (r != RS3_OK) return r;
        const dim3 grid((unsigned)((k_max + TC_ROWS - 1) / TC_ROWS * splits), (unsigned)H, (unsigned)a.s.U);
        launch_pdl(kern, grid, dim3(TC_THREADS), smem, st, p);
        if (splits > 1) {
            const int room = p.splits * p.take;
            const size_t bytes = 4 * (size_t)room * sizeof(int2);
            r = rs3_kernel_smem((const void *)k_merge_blocks, bytes);
            if (r != RS3_OK) return r;
            launch_pdl(k_merge_blocks, dim3((unsigned)((k_max + 3) / 4), (unsigned)H, (unsigned)a.s.U), dim3(128), bytes, st, p, room);
        }
        return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
    }
    a.qt = 8;
    while (a.qt > 1 && (int64_t)a.qt * a.s.nb * 4 > SELECT_KEYS_BYTES) a.qt >>= 1;
    const size_t smem = (size_t)a.qt * (size_t)a.s.nb * 4;
    const rs3_status r = rs3_kernel_smem((const void *)k_block_select, smem + 4 * 1024);   // (its own static arrays count too)
    if (r != RS3_OK) return r;
    const dim3 grid((unsigned)((k_max + a.qt - 1) / a.qt), (unsigned)H, (unsigned)a.s.U);
    launch_pdl(k_block_select, grid, dim3(SELECT_THREADS), smem, st, a);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
