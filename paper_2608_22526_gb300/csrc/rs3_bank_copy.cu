// rs3_bank_copy.cu -- units of one bank copied, forked and compacted into another, and
// ring frames given up at either end.
//
// A copy moves the kept rows of a source unit, in logical order, to the first pinned, ring
// and pointer rows of a destination unit.  It is bound by the bytes of those rows, each read
// once per destination and written once.  Chunks of 64 logical rows of all units form one
// axis that the CTAs walk in strides, because only the device knows the banks' lengths.
//
// With a keep mask the rows' places depend on the kept rows before them: k_keep_count turns the
// mask into words of 64 rows and counts the kept rows over all SMs, and the last CTA of a unit to arrive sums the
// counts up; k_bank_copy then moves the rows and publishes the counters.  Without one the places are known and the
// copy is the only launch.
#include "rs3_bank.cuh"

#include <initializer_list>

namespace {

constexpr int COPY_CHUNK = 64;             // logical rows of a chunk: a word of the mask
constexpr int COPY_THREADS = 256;
constexpr int COPY_FLIGHT = 4;             // pieces of K and of V in flight per thread
constexpr int SLOT_CHUNKS = 64;            // chunks that a CTA counts together
constexpr int COPY_UNITS = 1024;           // units whose chunk counts a CTA holds at a time

struct CopyArgs {
    BankDev src, dst;
    const uint8_t *k_src, *v_src;
    uint8_t *k_dst, *v_dst;
    const int32_t *parent;
    const uint8_t *keep;
    int64_t keep_stride;
    int64_t *place;            // [U][chunks + 3]: kept rows of its slot before each chunk; of the pinned rows (-1: they do
                               // not fit), of pinned + ring, of all
    uint64_t *words;           // [U][chunks]: the kept rows of each
    int64_t *before;           // [U][slots]: kept rows before each slot
    int64_t slots;
    int64_t chunks;            // of a mask row
    int64_t row_bytes;
    int32_t U, U_src;
    int32_t same;              // both banks are one
    int32_t *status;
};

// What becomes of destination unit u.
struct CopyUnit {
    int32_t p;                 // its source unit, -1: nothing to do
    LiveRows rows;             // of the source
    int64_t length;
};

// Everything that is wrong is found by every CTA alike and latched by those with `latch`.
__device__ CopyUnit copy_unit(const CopyArgs &a, int u, bool latch)
{
    CopyUnit c;
    c.p = -1;
    c.length = 0;
    const int32_t p = a.parent[u];
    if (p == -1) return c;
    // in one bank a source has to stay as it is while others copy it
    const bool bad = p < -1 || p >= a.U_src ||
                     (a.same && (p == u ? a.keep != nullptr : a.parent[p] != -1 && (a.parent[p] != p || a.keep)));
    if (bad) {
        if (latch) latch_status(a.status, RS3_EINVAL);
        return c;
    }
    if (a.same && p == u) return c;
    const int64_t *mp = a.src.meta + (int64_t)p * a.src.stride_words;
    const int64_t nf = mp[BM_NFRAMES], oldest = mp[BM_OLDEST];
    if (!c.rows.load(a.src, p) || nf < 0 || nf > a.src.max_frames || oldest < 0 || oldest >= a.src.max_frames) {
        if (latch) latch_status(a.status, RS3_EINTERNAL);
        return c;
    }
    c.length = c.rows.len[0] + c.rows.len[1] + c.rows.len[2] + c.rows.len[3];
    // what can be known without the counts; a mask has to cover every row
    const bool fits = nf <= a.dst.max_frames && mp[BM_NCOND] <= a.dst.n_cond &&
                      (a.keep || (c.rows.len[0] <= a.dst.pinned_cap && c.rows.len[1] + c.rows.len[2] <= a.dst.ring_cap &&
                                  c.rows.len[3] <= a.dst.n_ptr));
    if (!fits || (a.keep && c.length > a.keep_stride)) {
        if (latch) latch_status(a.status, fits ? RS3_EINVAL : RS3_ECAPACITY);
        c.length = 0;
        return c;
    }
    c.p = p;
    return c;
}

__device__ __forceinline__ int64_t frame_len(const CopyArgs &a, int p, int i)
{
    const int64_t *mp = a.src.meta + (int64_t)p * a.src.stride_words;
    int64_t slot = mp[BM_OLDEST] + i;
    if (slot >= a.src.max_frames) slot -= a.src.max_frames;
    return mp[BM_HEADER_WORDS + a.src.max_frames + slot];
}

// Inclusive sums of one value per thread over the CTA.
__device__ int64_t cta_sums(int64_t v)
{
    __shared__ int64_t s_part[COPY_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    __syncthreads();
    if (lane == 31) s_part[warp] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < COPY_THREADS / 32; ++w) v += w < warp ? s_part[w] : 0;
    return v;
}

// The destination's counters for a copy of source unit p with `cond`, `ring` and `ptr` kept
// rows.  By the whole CTA; `before(r0, r1)` turns the ring rows r0 and r1 where a frame begins and
// ends into the kept ring rows before them.
template <typename F>
__device__ void publish(const CopyArgs &a, int u, int p, int64_t live, int64_t cond, int64_t ring, int64_t ptr, F before)
{
    const int64_t *mp = a.src.meta + (int64_t)p * a.src.stride_words;
    int64_t *mu = a.dst.meta + (int64_t)u * a.dst.stride_words;
    const int nf = (int)mp[BM_NFRAMES];
    int64_t *fo = mu + BM_HEADER_WORDS, *fl = fo + a.dst.max_frames;
    int64_t base = 0;
    __shared__ int64_t s_base;
    for (int i0 = 0; i0 < nf; i0 += COPY_THREADS) {
        const int i = i0 + threadIdx.x;
        const int64_t n = i < nf ? max((int64_t)0, frame_len(a, p, i)) : 0;
        const int64_t end = base + cta_sums(n);
        int64_t r0 = min(live, end - n), r1 = min(live, end);
        before(r0, r1);
        if (i < nf) {
            fo[i] = r0;
            fl[i] = r1 - r0;
        }
        __syncthreads();
        if (threadIdx.x == COPY_THREADS - 1) s_base = end;
        __syncthreads();
        base = s_base;
    }
    if (threadIdx.x == 0) {
        mu[BM_HEAD] = 0;
        mu[BM_TAIL] = ring;
        mu[BM_COND_LEN] = cond;
        mu[BM_NFRAMES] = nf;
        mu[BM_OLDEST] = 0;
        mu[BM_NCOND] = mp[BM_NCOND];
        mu[BM_PTRLEN] = ptr;
        mu[BM_COPIES] += 1;                       // (what moves with the rows on the host's side goes by this)
    }
}

// Kept rows of unit u before its logical row r, of n in all.
__device__ __forceinline__ int64_t kept_before(const CopyArgs &a, int u, int64_t r, int64_t length)
{
    const int64_t *place = a.place + (int64_t)u * (a.chunks + 3);
    if (r >= length) return __ldcg(place + a.chunks + 2);
    const int64_t ch = r / COPY_CHUNK;
    return __ldcg(a.before + u * a.slots + ch / SLOT_CHUNKS) + __ldcg(place + ch) +
           __popcll(__ldcg(a.words + u * a.chunks + ch) & ((1ull << (r % COPY_CHUNK)) - 1ull));
}

// The mask's words and their counts: a thread takes 16 rows, four threads a chunk, a CTA a slot; the last CTA of a
// unit to arrive sums the slots up and decides whether the rows fit.
__global__ void __launch_bounds__(COPY_THREADS) k_keep_count(CopyArgs a)
{
    static_assert(SLOT_CHUNKS * COPY_CHUNK == 16 * COPY_THREADS, "a CTA's rows are a slot");
    pdl_wait();
    const int u = blockIdx.y;
    const CopyUnit c = copy_unit(a, u, blockIdx.x == 0 && threadIdx.x == 0);
    int64_t *place = a.place + (int64_t)u * (a.chunks + 3);
    if (c.p < 0) {
        if (blockIdx.x == 0 && threadIdx.x == 0) place[a.chunks] = -1;
        return;
    }
    const uint8_t *m = a.keep + (int64_t)u * a.keep_stride;
    const bool wide = (reinterpret_cast<uintptr_t>(m) & 15u) == 0;
    const int64_t n_slots = (c.length + 16 * COPY_THREADS - 1) / (16 * COPY_THREADS);
    for (int64_t slot = blockIdx.x; slot < n_slots; slot += gridDim.x) {
        const int64_t r = slot * (16 * COPY_THREADS) + 16 * threadIdx.x;
        uint32_t bits = 0;
        if (wide && r + 16 <= c.length) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(m + r));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)                    // a bit per byte, then the four side by side
                bits |= (((__vcmpne4(w[i], 0u) & 0x08040201u) * 0x01010101u) >> 24) << (4 * i);
        } else {
            for (int i = 0; i < 16; ++i)
                if (r + i < c.length) bits |= (uint32_t)(m[r + i] != 0) << i;
        }
        uint64_t word = (uint64_t)bits << (16 * (threadIdx.x & 3));
        word |= __shfl_xor_sync(0xffffffffu, word, 1);
        word |= __shfl_xor_sync(0xffffffffu, word, 2);
        const int64_t end = cta_sums(__popc(bits));
        if ((threadIdx.x & 3) == 0 && r < c.length) {
            a.words[u * a.chunks + r / COPY_CHUNK] = word;
            place[r / COPY_CHUNK] = end - __popc(bits);
        }
        if (threadIdx.x == COPY_THREADS - 1) a.before[u * a.slots + slot] = end;
    }
    __shared__ bool s_last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        int64_t *arrive = a.dst.meta + (int64_t)u * a.dst.stride_words + BM_ARRIVE;
        s_last = atomicAdd(reinterpret_cast<unsigned long long *>(arrive), 1ull) == gridDim.x - 1;
        if (s_last) *arrive = 0;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    // exclusive sums over the slots
    __shared__ int64_t s_run;
    int64_t run = 0;
    for (int64_t s0 = 0; s0 < n_slots; s0 += COPY_THREADS) {
        const int64_t slot = s0 + threadIdx.x;
        const int64_t n = slot < n_slots ? __ldcg(a.before + u * a.slots + slot) : 0;
        const int64_t end = run + cta_sums(n);
        if (slot < n_slots) a.before[u * a.slots + slot] = end - n;
        if (threadIdx.x == COPY_THREADS - 1) s_run = end;
        __syncthreads();
        run = s_run;
    }
    if (threadIdx.x == 0) place[a.chunks + 2] = run;
    __syncthreads();
    if (threadIdx.x != 0) return;
    const int64_t cond = kept_before(a, u, c.rows.len[0], c.length);
    const int64_t ring = kept_before(a, u, c.rows.len[0] + c.rows.len[1] + c.rows.len[2], c.length) - cond;
    const bool fits = cond <= a.dst.pinned_cap && ring <= a.dst.ring_cap && run - cond - ring <= a.dst.n_ptr;
    if (!fits) latch_status(a.status, RS3_ECAPACITY);
    place[a.chunks] = fits ? cond : -1;
    place[a.chunks + 1] = cond + ring;
}

template <bool KEEP>
__global__ void __launch_bounds__(COPY_THREADS, 3) k_bank_copy(CopyArgs a)
{
    pdl_wait();
    __shared__ int64_t s_first[COPY_UNITS + 1];       // chunks before each unit of the round
    __shared__ int64_t s_from[COPY_CHUNK], s_to[COPY_CHUNK];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // a thread's piece of 16 bytes and its rows of a chunk: rows t / nvec, + step, ... (rows of more than
    // 256 pieces: every row, pieces t, + 256, ...)
    const int nvec = (int)(a.row_bytes / 16);
    const int step = nvec < COPY_THREADS ? COPY_THREADS / nvec : 1;
    const int row0 = nvec < COPY_THREADS ? (int)threadIdx.x / nvec : 0, piece0 = (int)threadIdx.x - row0 * nvec;
    int64_t next = blockIdx.x;                        // this CTA's next chunk, counted from the round's first
    int last = -1;                                    // the unit that c describes
    CopyUnit c;
    for (int u0 = 0; u0 < a.U; u0 += COPY_UNITS) {
        const int n_units = min(COPY_UNITS, a.U - u0);
        __syncthreads();
        for (int i = threadIdx.x; i < n_units; i += COPY_THREADS) {
            const CopyUnit x = copy_unit(a, u0 + i, !KEEP && blockIdx.x == 0);
            int64_t n = (x.length + COPY_CHUNK - 1) / COPY_CHUNK;
            if (KEEP && n > 0 && a.place[(int64_t)(u0 + i) * (a.chunks + 3) + a.chunks] < 0) n = 0;   // does not fit
            s_first[i + 1] = n;
        }
        __syncthreads();
        if (warp == 0) {                              // inclusive sums
            int64_t run = 0;
            for (int c0 = 0; c0 < n_units; c0 += 32) {
                const int i = c0 + lane;
                int64_t s = i < n_units ? s_first[i + 1] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int64_t t = __shfl_up_sync(0xffffffffu, s, o);
                    if (lane >= o) s += t;
                }
                if (i < n_units) s_first[i + 1] = run + s;
                run += __shfl_sync(0xffffffffu, s, 31);
            }
            if (lane == 0) s_first[0] = 0;
        }
        __syncthreads();
        const int64_t total = s_first[n_units];
        for (; next < total; next += gridDim.x) {
            int lo = 0, hi = n_units;                 // the last unit whose chunks begin at or before `next`
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_first[mid] <= next) lo = mid; else hi = mid;
            }
            const int u = u0 + lo;
            const int64_t ch = next - s_first[lo];
            const int64_t *place = a.place + (int64_t)u * (a.chunks + 3);
            const uint64_t word = KEEP ? a.words[u * a.chunks + ch] : 0;
            const int64_t first = KEEP ? a.before[u * a.slots + ch / SLOT_CHUNKS] + place[ch] : ch * COPY_CHUNK;
            if (u != last) c = copy_unit(a, u, false);
            last = u;
            const int64_t left = c.length - ch * COPY_CHUNK;
            const uint64_t kept = KEEP ? word : left >= COPY_CHUNK ? ~0ull : (1ull << left) - 1ull;
            const int n = __popcll(kept);
            // a row per thread: where it lies and where it goes
            if (threadIdx.x < COPY_CHUNK && (kept >> threadIdx.x & 1ull)) {
                const int at = __popcll(kept & ((1ull << threadIdx.x) - 1ull));
                int64_t from = 0, x = ch * COPY_CHUNK + threadIdx.x;
                int region = 0;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (x >= 0 && x < c.rows.len[g]) { from = c.rows.start[g] + x; region = g; }
                    x -= c.rows.len[g];
                }
                const int64_t n_cond = KEEP ? place[a.chunks] : c.rows.len[0];
                const int64_t n_ring = KEEP ? place[a.chunks + 1] : n_cond + c.rows.len[1] + c.rows.len[2];
                const int64_t rank = first + at;
                s_from[at] = from * a.row_bytes;
                s_to[at] = (region == 0 ? rank : region < 3 ? a.dst.pinned_cap + rank - n_cond
                                                            : a.dst.pinned_cap + a.dst.ring_cap + rank - n_ring) * a.row_bytes;
            }
            __syncthreads();
            const uint8_t *ks = a.k_src + (int64_t)c.p * a.src.rows_per_unit * a.row_bytes;
            const uint8_t *vs = a.v_src + (int64_t)c.p * a.src.rows_per_unit * a.row_bytes;
            uint8_t *kd = a.k_dst + (int64_t)u * a.dst.rows_per_unit * a.row_bytes;
            uint8_t *vd = a.v_dst + (int64_t)u * a.dst.rows_per_unit * a.row_bytes;
            for (int p = row0 < step ? piece0 : nvec; p < nvec; p += COPY_THREADS)
                for (int r0 = row0; r0 < n; r0 += step * COPY_FLIGHT) {
                    uint4 kv[COPY_FLIGHT], vv[COPY_FLIGHT];
#pragma unroll
                    for (int f = 0; f < COPY_FLIGHT; ++f) {
                        const int r = r0 + f * step;
                        if (r < n) {
                            const int64_t at = s_from[r] + 16 * p;
                            kv[f] = __ldcs(reinterpret_cast<const uint4 *>(ks + at));
                            vv[f] = __ldcs(reinterpret_cast<const uint4 *>(vs + at));
                        }
                    }
#pragma unroll
                    for (int f = 0; f < COPY_FLIGHT; ++f) {
                        const int r = r0 + f * step;
                        if (r < n) {
                            const int64_t at = s_to[r] + 16 * p;
                            *reinterpret_cast<uint4 *>(kd + at) = kv[f];
                            *reinterpret_cast<uint4 *>(vd + at) = vv[f];
                        }
                    }
                }
            __syncthreads();
        }
        next -= total;
    }
    // the counters, a unit per CTA, from the last one on, which has no more chunks than the others (a source's counters
    // are never written)
    for (int64_t u = gridDim.x - 1 - blockIdx.x; u < a.U; u += gridDim.x) {
        const CopyUnit x = copy_unit(a, (int)u, false);
        if (x.p < 0) continue;
        const int64_t ring0 = x.rows.len[0], ring1 = ring0 + x.rows.len[1] + x.rows.len[2];
        if (!KEEP) {
            publish(a, (int)u, x.p, ring1 - ring0, ring0, ring1 - ring0, x.rows.len[3], [](int64_t &, int64_t &) {});
        } else {
            const int64_t *place = a.place + u * (a.chunks + 3) + a.chunks;
            const int64_t cond = place[0], both = place[1];
            if (cond < 0) continue;
            publish(a, (int)u, x.p, ring1 - ring0, cond, both - cond, place[2] - both, [&](int64_t &r0, int64_t &r1) {
                r0 = kept_before(a, (int)u, ring0 + r0, x.length) - cond;
                r1 = kept_before(a, (int)u, ring0 + r1, x.length) - cond;
            });
        }
    }
}

// A warp per unit: the frames given up at either end leave the counters.
__global__ void k_drop_frames(BankDev bk, int U, const int32_t *n_oldest, const int32_t *n_newest, int32_t *status)
{
    pdl_wait();
    const int u = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (u >= U) return;
    int64_t *mu = bk.meta + (int64_t)u * bk.stride_words;
    const int64_t nf = mu[BM_NFRAMES], oldest = mu[BM_OLDEST];
    const int64_t a = n_oldest ? n_oldest[u] : 0, b = n_newest ? n_newest[u] : 0;
    const bool sane = nf >= 0 && nf <= bk.max_frames && oldest >= 0 && oldest < bk.max_frames;
    if (!sane || a < 0 || b < 0 || a + b > nf) {
        if (lane == 0) latch_status(status, sane ? RS3_EINVAL : RS3_EINTERNAL);
        return;
    }
    const int64_t *fl = mu + BM_HEADER_WORDS + bk.max_frames;
    int64_t first = 0, last = 0;
    for (int64_t i = lane; i < a; i += 32) first += fl[(oldest + i) % bk.max_frames];
    for (int64_t i = lane; i < b; i += 32) last += fl[(oldest + nf - 1 - i) % bk.max_frames];
    first = warp_sum(first);
    last = warp_sum(last);
    if (lane == 0) {
        mu[BM_HEAD] += first;
        mu[BM_TAIL] -= last;
        mu[BM_NFRAMES] = nf - a - b;
        mu[BM_OLDEST] = (oldest + a) % bk.max_frames;
    }
}

int64_t copy_chunks(int64_t keep_stride) { return (keep_stride + COPY_CHUNK - 1) / COPY_CHUNK; }
int64_t copy_slots(int64_t keep_stride) { return (copy_chunks(keep_stride) + SLOT_CHUNKS - 1) / SLOT_CHUNKS; }

// Storage [a, a + n) and [b, b + m) share a byte.
bool overlap(const void *a, int64_t n, const void *b, int64_t m)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)m && y < x + (uintptr_t)n;
}

}  // namespace

extern "C" size_t rs3_bank_copy_workspace_bytes(int U, int64_t keep_stride)
{
    if (U < 1 || keep_stride < 1) return 0;
    return (size_t)U * (size_t)(2 * copy_chunks(keep_stride) + 3 + copy_slots(keep_stride)) * 8;
}

extern "C" rs3_status rs3_bank_copy(const rs3_bank *dst, const rs3_bank *src, const int32_t *parent, const uint8_t *keep,
                                    int64_t keep_stride, void *workspace, size_t workspace_bytes, int32_t *status,
                                    rs3_stream_t stream)
{
    if (!bank_ok(dst) || !bank_ok(src) || !parent || !status) return RS3_EINVAL;
    if (dst->H != src->H || dst->d != src->d || dst->dtype != src->dtype || dst->mn != src->mn) return RS3_EINVAL;
    if (keep && (keep_stride < 1 || !workspace || !rs3_aligned16(workspace))) return RS3_EINVAL;
    if (keep && workspace_bytes < rs3_bank_copy_workspace_bytes(dst->U, keep_stride)) return RS3_ECAPACITY;
    const int64_t row_bytes = (int64_t)dst->D * (int64_t)elem_bytes(dst->dtype);
    const bool same = dst->k_store == src->k_store && dst->v_store == src->v_store && dst->meta == src->meta;
    if (same && (dst->U != src->U || dst->pinned_cap != src->pinned_cap || dst->ring_cap != src->ring_cap || dst->n_ptr != src->n_ptr ||
                 dst->max_frames != src->max_frames))
        return RS3_EINVAL;                         // one storage in two layouts
    const int64_t sb = src->U * src->rows_per_unit * row_bytes, db = dst->U * dst->rows_per_unit * row_bytes;
    const int64_t sm = src->U * src->meta_stride, dm = dst->U * dst->meta_stride;
    if (!same) {
        for (const void *d : {dst->k_store, dst->v_store})
            if (overlap(d, db, src->k_store, sb) || overlap(d, db, src->v_store, sb) || overlap(d, db, src->meta, sm)) return RS3_EINVAL;
        for (const void *s : {src->k_store, src->v_store})
            if (overlap(dst->meta, dm, s, sb)) return RS3_EINVAL;
        if (overlap(dst->meta, dm, src->meta, sm)) return RS3_EINVAL;
    }
    if (row_bytes > (1 << 20)) return RS3_EUNSUPPORTED;
    CopyArgs a = {};
    a.U = dst->U;
    a.U_src = src->U;
    a.src = bank_dev(src);
    a.dst = bank_dev(dst);
    a.k_src = static_cast<const uint8_t *>(src->k_store);
    a.v_src = static_cast<const uint8_t *>(src->v_store);
    a.k_dst = static_cast<uint8_t *>(dst->k_store);
    a.v_dst = static_cast<uint8_t *>(dst->v_store);
    a.parent = parent;
    a.keep = keep;
    a.keep_stride = keep_stride;
    a.place = static_cast<int64_t *>(workspace);
    a.chunks = keep ? copy_chunks(keep_stride) : 0;
    a.slots = keep ? copy_slots(keep_stride) : 0;
    a.words = reinterpret_cast<uint64_t *>(a.place + a.U * (a.chunks + 3));
    a.before = reinterpret_cast<int64_t *>(a.words + a.U * a.chunks);
    a.row_bytes = row_bytes;
    a.same = same;
    a.status = status;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    // no more CTAs than chunks that full banks would have
    const int64_t most = keep ? a.chunks : (src->rows_per_unit + COPY_CHUNK - 1) / COPY_CHUNK;
    int64_t ctas = 3ll * rs3_sm_count();
    if (most * a.U < ctas) ctas = most * a.U > 0 ? most * a.U : 1;
    if (keep) {
        int64_t per = (2ll * rs3_sm_count() + a.U - 1) / a.U;
        if (per > a.slots) per = a.slots;
        launch_pdl(k_keep_count, dim3((unsigned)per, (unsigned)a.U), dim3(COPY_THREADS), 0, st, a);
        launch_pdl(k_bank_copy<true>, dim3((unsigned)ctas), dim3(COPY_THREADS), 0, st, a);
    } else {
        launch_pdl(k_bank_copy<false>, dim3((unsigned)ctas), dim3(COPY_THREADS), 0, st, a);
    }
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}

extern "C" rs3_status rs3_bank_drop_frames(const rs3_bank *bank, const int32_t *n_oldest, const int32_t *n_newest,
                                           int32_t *status, rs3_stream_t stream)
{
    if (!bank_ok(bank) || !status) return RS3_EINVAL;
    launch_pdl(k_drop_frames, dim3((bank->U + 3) / 4), dim3(128), 0, reinterpret_cast<cudaStream_t>(stream), bank_dev(bank),
               bank->U, n_oldest, n_newest, status);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}
