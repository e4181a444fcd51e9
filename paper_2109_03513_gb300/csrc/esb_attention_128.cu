// esb_attention_128.cu -- attention for heads of up to 128 values.
#include "esb_attention.cuh"

namespace esb {

int attention_most_128(int planes) { return planes == 1 ? 4 : 2; }

cudaError_t attention_run_128(const AttnArgs& a, int nt, int planes, bool lin, void* workspace, cudaStream_t st)
{
    switch (nt * 10 + planes) {
    case 11: return Variant<128, 1, 1>::run(a, lin, workspace, st);
    case 21: return Variant<128, 2, 1>::run(a, lin, workspace, st);
    case 41: return Variant<128, 4, 1>::run(a, lin, workspace, st);
    case 12: return Variant<128, 1, 2>::run(a, lin, workspace, st);
    default: return Variant<128, 2, 2>::run(a, lin, workspace, st);
    }
}

size_t attention_bytes_128(int nt, int planes)
{
    switch (nt * 10 + planes) {
    case 11: return Variant<128, 1, 1>::bytes();
    case 21: return Variant<128, 2, 1>::bytes();
    case 41: return Variant<128, 4, 1>::bytes();
    case 12: return Variant<128, 1, 2>::bytes();
    default: return Variant<128, 2, 2>::bytes();
    }
}

}  // namespace esb
