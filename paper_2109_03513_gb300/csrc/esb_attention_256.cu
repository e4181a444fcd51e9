// esb_attention_256.cu -- attention for heads of up to 256 values.
#include "esb_attention.cuh"

namespace esb {

int attention_most_256(int planes) { return planes == 1 ? 2 : 1; }

cudaError_t attention_run_256(const AttnArgs& a, int nt, int planes, bool lin, void* workspace, cudaStream_t st)
{
    switch (nt * 10 + planes) {
    case 11: return Variant<256, 1, 1>::run(a, lin, workspace, st);
    case 21: return Variant<256, 2, 1>::run(a, lin, workspace, st);
    default: return Variant<256, 1, 2>::run(a, lin, workspace, st);
    }
}

size_t attention_bytes_256(int nt, int planes)
{
    switch (nt * 10 + planes) {
    case 11: return Variant<256, 1, 1>::bytes();
    case 21: return Variant<256, 2, 1>::bytes();
    default: return Variant<256, 1, 2>::bytes();
    }
}

}  // namespace esb
