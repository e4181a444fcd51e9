// esb_attention_64.cu -- attention for heads of up to 64 values.
#include "esb_attention.cuh"

namespace esb {

int attention_most_64(int) { return 4; }

cudaError_t attention_run_64(const AttnArgs& a, int nt, int planes, bool lin, void* workspace, cudaStream_t st)
{
    switch (nt * 10 + planes) {
    case 11: return Variant<64, 1, 1>::run(a, lin, workspace, st);
    case 21: return Variant<64, 2, 1>::run(a, lin, workspace, st);
    case 41: return Variant<64, 4, 1>::run(a, lin, workspace, st);
    case 12: return Variant<64, 1, 2>::run(a, lin, workspace, st);
    case 22: return Variant<64, 2, 2>::run(a, lin, workspace, st);
    default: return Variant<64, 4, 2>::run(a, lin, workspace, st);
    }
}

size_t attention_bytes_64(int nt, int planes)
{
    switch (nt * 10 + planes) {
    case 11: return Variant<64, 1, 1>::bytes();
    case 21: return Variant<64, 2, 1>::bytes();
    case 41: return Variant<64, 4, 1>::bytes();
    case 12: return Variant<64, 1, 2>::bytes();
    case 22: return Variant<64, 2, 2>::bytes();
    default: return Variant<64, 4, 2>::bytes();
    }
}

}  // namespace esb
