// rs3_sparse.cuh -- what the block-sparse read side shares: a call's arguments, its
// units, and the 8-bit form of a vector.
#pragma once

#include "rs3_bank.cuh"

#define RS3_MAX_TOP 1024                   // blocks listed per query and head

struct SparseArgs {
    const void *q;
    const int32_t *unit_group, *idx, *count;
    const float *rope;
    int32_t *status;
    BankDev bank;
    int32_t G, U, mn, H, d, k_max;
    int32_t bs, nb;            // rows of a block, blocks of a unit
    int32_t n_top;
};

// Checks what rs3_block_select and rs3_sparse_readout have in common.
inline rs3_status sparse_args(SparseArgs &a, const void *q, rs3_dtype dtype, int G, int mn, int H, int d,
                              const int32_t *unit_group, const int32_t *idx, const int32_t *count, int k_max,
                              const rs3_bank *bank, int block, const float *rope, int n_top, int32_t *status);

// Kept queries and group of unit u; false when there is nothing to do.  What is wrong is
// latched by the calls with `latch`.
__device__ __forceinline__ bool sparse_unit(const SparseArgs &a, int u, bool latch, int &cnt, int &g, LiveRows &rows)
{
    cnt = a.count[u];
    g = a.unit_group[u];
    const bool sound = rows.load(a.bank, u);               // (before the checks: all loads go out together)
    if (cnt < 0 || cnt > a.k_max || g < 0 || g >= a.G) {
        if (latch) latch_status(a.status, RS3_EINVAL);
        return false;
    }
    if (!sound) {
        if (latch) latch_status(a.status, RS3_EINTERNAL);
        return false;
    }
    return cnt > 0;
}

// The 8-bit form of a vector whose largest element is `amax`: whole numbers t with
// |t| <= 127, standing for t * step, step a power of two: e = min(floor(log2 amax), 110),
// t = rint(x 2^(6 - e)) cut to 127, step = 2^(e - 6).  Scaling by a power of two is exact, so a
// score t . t' * step never rounds: |t . t'| <= 127^2 * 256 < 2^22, whatever the order of its
// sums, and with steps up to 2^104 it is finite: every live block has a rank.  Vectors below 2^-100 are
// zeros with step 0.  A NaN is a 0 (maxima pass over it, and so does the conversion).
struct EightBits {
    float up, step;
    __device__ __forceinline__ explicit EightBits(float amax)
    {
        const int e = min((int)(__float_as_uint(amax) >> 23) - 127, 110);
        const bool some = amax >= 7.888609052210118e-31f;
        up = some ? __uint_as_float((uint32_t)(133 - e) << 23) : 0.f;
        step = some ? __uint_as_float((uint32_t)(121 + e) << 23) : 0.f;
    }
    __device__ __forceinline__ int operator()(float x) const
    {
        return min(127, max(-127, __float2int_rn(x * up)));
    }
};

inline rs3_status sparse_args(SparseArgs &a, const void *q, rs3_dtype dtype, int G, int mn, int H, int d,
                              const int32_t *unit_group, const int32_t *idx, const int32_t *count, int k_max,
                              const rs3_bank *bank, int block, const float *rope, int n_top, int32_t *status)
{
    if (!bank_ok(bank) || !q || !unit_group || !idx || !count || !status) return RS3_EINVAL;
    if (G < 1 || mn < 1 || k_max < 0 || n_top < 1) return RS3_EINVAL;
    if ((int)dtype != bank->dtype || mn != bank->mn || H != bank->H || d != bank->d) return RS3_EINVAL;
    if (!rs3_aligned16(q) || (rope && !rs3_aligned16(rope))) return RS3_EINVAL;
    if (block != 32 && block != 64 && block != 128) return RS3_EUNSUPPORTED;
    if (d < 16 || d > 256 || (d & (d - 1)) != 0 || H > 65535) return RS3_EUNSUPPORTED;
    if (n_top > RS3_MAX_TOP || k_max > mn) return n_top > RS3_MAX_TOP ? RS3_EUNSUPPORTED : RS3_EINVAL;
    const int64_t nb = (bank->rows_per_unit + block - 1) / block;
    if (nb > INT32_MAX) return RS3_EUNSUPPORTED;
    a.q = q;
    a.unit_group = unit_group;
    a.idx = idx;
    a.count = count;
    a.rope = rope;
    a.status = status;
    a.bank = bank_dev(bank);
    a.G = G;
    a.U = bank->U;
    a.mn = mn;
    a.H = H;
    a.d = d;
    a.k_max = k_max;
    a.bs = block;
    a.nb = (int32_t)nb;
    a.n_top = n_top;
    return RS3_OK;
}
