// rs3_scored_tc.cu -- the one-tile tensor-core readout (rs3_readout_tc.cuh) over scores that are
// capped and biased by their row's frame.  A cap costs a score four fp32 operations beside the softmax's two
// within half of it, else a power and a quarter of a reciprocal (change_scores), and the key producer's warp
// looks the rows' biases up.
#include "rs3_readout_tc.cuh"

namespace tc {

template <int DH, class X>
__global__ void __launch_bounds__(Cfg<DH>::NTHREADS, 1)
k_readout_scored(const ReadoutMore a, const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv)
{
    const uint32_t tmem = set_up_tc<DH>(tmk, tmv);
    pdl_wait();                      // the plan
    readout_tc<DH, X>(a, tmk, tmv, tmem, a.cta_items[2 * blockIdx.x], a.cta_items[2 * blockIdx.x + 1]);
}

template <int DH, class X>
rs3_status launch_scored(const ReadoutMore &a, cudaStream_t st)
{
    constexpr int smem = Cfg<DH>::SMEM + BiasRing<X, Cfg<DH>::BN, Cfg<DH>::KSTK, 2>::BYTES;
    static_assert(smem <= 232448, "shared memory budget");
    if (rs3_kernel_smem((const void *)k_readout_scored<DH, X>, smem) != RS3_OK) return RS3_ECUDA;
    const int64_t rows = (int64_t)a.bank_U * a.rows_per_unit;
    if (rows >= (int64_t)1 << 31) return RS3_EUNSUPPORTED;
    CUtensorMap mk, mv;
    if (!make_kv_map(&mk, a.k_store, a.D, rows, Cfg<DH>::BN) || !make_kv_map(&mv, a.v_store, a.D, rows, Cfg<DH>::BN)) return RS3_ECUDA;
    launch_pdl(k_readout_scored<DH, X>, dim3((unsigned)a.grid_ctas), dim3(Cfg<DH>::NTHREADS), smem, st, a, mk, mv);
    return cudaGetLastError() == cudaSuccess ? RS3_OK : RS3_ECUDA;
}

template <int DH>
rs3_status launch_width(const ReadoutMore &a, cudaStream_t st)
{
    const bool cap = a.score.cap > 0.f, bias = a.score.bias != nullptr;
    if (cap) return bias ? launch_scored<DH, FrameScores<true, true>>(a, st) : launch_scored<DH, FrameScores<true, false>>(a, st);
    return bias ? launch_scored<DH, FrameScores<false, true>>(a, st) : launch_scored<DH, FrameScores<false, false>>(a, st);
}

}  // namespace tc

rs3_status rs3_launch_scored_tc(const ReadoutMore &a, cudaStream_t st)
{
    switch (a.d) {
    case 64: return tc::launch_width<64>(a, st);
    case 128: return tc::launch_width<128>(a, st);
    case 256: return tc::launch_width<256>(a, st);
    default: return RS3_EUNSUPPORTED;
    }
}
