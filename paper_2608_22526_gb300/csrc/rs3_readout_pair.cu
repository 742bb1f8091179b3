// rs3_readout_pair.cu -- the readout with one or two query tiles (rs3_readout_pair.cuh) over plain scores.
#include "rs3_readout_pair.cuh"

rs3_status rs3_launch_either_readout(const ReadoutArgs &a, cudaStream_t st)
{
    switch (a.d) {
    case 64: return tc::pair::launch<64>(a, st);
    case 128: return tc::pair::launch<128>(a, st);
    default: return RS3_EUNSUPPORTED;
    }
}
