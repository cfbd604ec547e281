// 16-bit products with B or both operands across K: gradients of a layer's inputs and weights in 16 bits.
#include "dsq_product16.cuh"

namespace dsq {

cudaError_t product16_gradient(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiBlocks<1>& epi, cudaStream_t st) {
  return a.across ? product16<kAcross, kAcross>(plan, a, b, s, epi, st) : product16<kAlong, kAcross>(plan, a, b, s, epi, st);
}

}  // namespace dsq
