// rs3_bank.cuh -- what the kernels that touch a bank share: the bank's sizes as
// kernels take them, and a unit's live rows.
#pragma once

#include "rs3_internal.cuh"

struct BankDev {
    int64_t *meta;
    int64_t stride_words;
    int32_t max_frames, window, n_cond, n_ptr;
    int64_t pinned_cap, ring_cap, rows_per_unit;
};

inline BankDev bank_dev(const rs3_bank *b)
{
    BankDev v;
    v.meta = static_cast<int64_t *>(b->meta);
    v.stride_words = b->meta_stride / 8;
    v.max_frames = b->max_frames;
    v.window = b->window;
    v.n_cond = b->n_cond;
    v.n_ptr = b->n_ptr;
    v.pinned_cap = b->pinned_cap;
    v.ring_cap = b->ring_cap;
    v.rows_per_unit = b->rows_per_unit;
    return v;
}

inline bool bank_ok(const rs3_bank *b)
{
    return b && b->magic == RS3_BANK_MAGIC && b->meta && b->k_store && b->v_store && b->U >= 1;
}

inline size_t elem_bytes(int dtype) { return dtype == RS3_BF16 ? 2 : 4; }

// A unit's live rows: four runs of storage rows in logical order (pinned, the ring's
// two pieces, pointers).
struct LiveRows {
    int64_t start[4], len[4];

    // From the unit's counters; false (and no rows) when they are inconsistent.
    __device__ __forceinline__ bool load(const BankDev &b, int64_t u)
    {
        const int64_t *mu = b.meta + u * b.stride_words;
        const int64_t head = mu[BM_HEAD], tail = mu[BM_TAIL], cond = mu[BM_COND_LEN], ptr = mu[BM_PTRLEN];
#pragma unroll
        for (int r = 0; r < 4; ++r) start[r] = len[r] = 0;
        if (!(head >= 0 && tail >= head && tail - head <= b.ring_cap && cond >= 0 && cond <= b.pinned_cap && ptr >= 0 &&
              ptr <= b.n_ptr))
            return false;
        len[0] = cond;
        const int64_t live = tail - head;
        if (live > 0) {
            const int64_t p0 = head % b.ring_cap;          // live <= ring_cap, so ring_cap > 0
            len[1] = min(live, b.ring_cap - p0);
            start[1] = b.pinned_cap + p0;
            start[2] = b.pinned_cap;
            len[2] = live - len[1];
        }
        start[3] = b.pinned_cap + b.ring_cap;
        len[3] = ptr;
        return true;
    }

    // the storage rows [a, a + 64) that live, a bit each
    __device__ __forceinline__ uint64_t mask64(int64_t a) const
    {
        uint64_t m = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int lo = (int)max((int64_t)0, min((int64_t)64, start[r] - a));
            const int hi = (int)max((int64_t)0, min((int64_t)64, start[r] + len[r] - a));
            if (hi > lo) m |= (hi - lo == 64 ? ~0ull : (1ull << (hi - lo)) - 1ull) << lo;
        }
        return m;
    }

    // live rows among the storage rows [a, b)
    __device__ __forceinline__ int64_t count(int64_t a, int64_t b) const
    {
        int64_t n = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) n += max((int64_t)0, min(b, start[r] + len[r]) - max(a, start[r]));
        return n;
    }
};
