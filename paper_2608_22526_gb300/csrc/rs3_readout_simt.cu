// rs3_readout_simt.cu -- the CUDA-core readout (rs3_readout_simt.cuh) over plain scores.
#include "rs3_readout_simt.cuh"

namespace {

template <int ROWS>
void tile(int d, int &bm, int &ctas_per_sm)
{
    switch (d) {
    case 16: bm = Cfg<16, ROWS>::BM; ctas_per_sm = Cfg<16, ROWS>::CTAS; break;
    case 32: bm = Cfg<32, ROWS>::BM; ctas_per_sm = Cfg<32, ROWS>::CTAS; break;
    case 64: bm = Cfg<64, ROWS>::BM; ctas_per_sm = Cfg<64, ROWS>::CTAS; break;
    case 128: bm = Cfg<128, ROWS>::BM; ctas_per_sm = Cfg<128, ROWS>::CTAS; break;
    default: bm = Cfg<256, ROWS>::BM; ctas_per_sm = Cfg<256, ROWS>::CTAS; break;
    }
}

}  // namespace

void rs3_simt_tile(int d, bool few, int &bm, int &bn, int &ctas_per_sm)
{
    bn = BN;
    if (few) tile<FEW>(d, bm, ctas_per_sm);
    else tile<0>(d, bm, ctas_per_sm);
}

rs3_status rs3_launch_simt_readout(const ReadoutArgs &a, rs3_dtype dtype, cudaStream_t st)
{
    if (dtype == RS3_BF16) {                 // the other widths have a tensor-core tile
        switch (a.d) {
        case 16: return launch<uint16_t, 16, PlainScores>(a, st);
        case 32: return launch<uint16_t, 32, PlainScores>(a, st);
        default: return RS3_EUNSUPPORTED;
        }
    }
    switch (a.d) {
    case 16: return launch<float, 16, PlainScores>(a, st);
    case 32: return launch<float, 32, PlainScores>(a, st);
    case 64: return launch<float, 64, PlainScores>(a, st);
    case 128: return launch<float, 128, PlainScores>(a, st);
    case 256: return launch<float, 256, PlainScores>(a, st);
    default: return RS3_EUNSUPPORTED;
    }
}
