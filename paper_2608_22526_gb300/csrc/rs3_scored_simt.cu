// rs3_scored_simt.cu -- the CUDA-core readout (rs3_readout_simt.cuh) over scores that are capped
// and biased by their row's frame: tanhf of each score and a sum, beside d multiply-adds.
#include "rs3_readout_simt.cuh"

namespace {

template <typename T, int D>
rs3_status launch_scored(const ReadoutMore &a, cudaStream_t st)
{
    const bool cap = a.score.cap > 0.f, bias = a.score.bias != nullptr;
    if (cap) return bias ? launch<T, D, FrameScores<true, true>>(a, st) : launch<T, D, FrameScores<true, false>>(a, st);
    return bias ? launch<T, D, FrameScores<false, true>>(a, st) : launch<T, D, FrameScores<false, false>>(a, st);
}

}  // namespace

rs3_status rs3_launch_scored_simt(const ReadoutMore &a, rs3_dtype dtype, cudaStream_t st)
{
    if (dtype == RS3_BF16) {                 // the other widths have a tensor-core tile
        switch (a.d) {
        case 16: return launch_scored<uint16_t, 16>(a, st);
        case 32: return launch_scored<uint16_t, 32>(a, st);
        default: return RS3_EUNSUPPORTED;
        }
    }
    switch (a.d) {
    case 16: return launch_scored<float, 16>(a, st);
    case 32: return launch_scored<float, 32>(a, st);
    case 64: return launch_scored<float, 64>(a, st);
    case 128: return launch_scored<float, 128>(a, st);
    case 256: return launch_scored<float, 256>(a, st);
    default: return RS3_EUNSUPPORTED;
    }
}
