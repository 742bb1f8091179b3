// rs3_scored_pair.cu -- the readout with one or two query tiles (rs3_readout_pair.cuh) over scores
// that are capped and biased by their row's frame.
#include "rs3_readout_pair.cuh"

namespace {

template <int DH>
rs3_status launch_width(const ReadoutMore &a, cudaStream_t st)
{
    using namespace tc::pair;
    const bool cap = a.score.cap > 0.f, bias = a.score.bias != nullptr;
    if (cap) return bias ? launch<DH, FrameScores<true, true>>(a, st) : launch<DH, FrameScores<true, false>>(a, st);
    return bias ? launch<DH, FrameScores<false, true>>(a, st) : launch<DH, FrameScores<false, false>>(a, st);
}

}  // namespace

rs3_status rs3_launch_scored_either(const ReadoutMore &a, cudaStream_t st)
{
    switch (a.d) {
    case 64: return launch_width<64>(a, st);
    case 128: return launch_width<128>(a, st);
    default: return RS3_EUNSUPPORTED;
    }
}
