// rs3_readout_simt.cu -- the CUDA-core readout (rs3_readout_simt.cuh) over plain scores.
#include "rs3_readout_simt.cuh"

void rs3_simt_tile(int d, int &bm, int &bn, int &ctas_per_sm)
{
    bn = BN;
    switch (d) {
    case 16: bm = Cfg<16>::BM; ctas_per_sm = Cfg<16>::CTAS; break;
    case 32: bm = Cfg<32>::BM; ctas_per_sm = Cfg<32>::CTAS; break;
    case 64: bm = Cfg<64>::BM; ctas_per_sm = Cfg<64>::CTAS; break;
    case 128: bm = Cfg<128>::BM; ctas_per_sm = Cfg<128>::CTAS; break;
    default: bm = Cfg<256>::BM; ctas_per_sm = Cfg<256>::CTAS; break;
    }
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
