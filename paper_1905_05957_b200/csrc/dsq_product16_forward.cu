// 16-bit products, both operands along K: a layer's forward product.
#include "dsq_product16.cuh"

namespace dsq {

cudaError_t product16_forward(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiBlocks<1>& epi, cudaStream_t st) {
  return product16<kAlong, kAlong>(plan, a, b, s, epi, st);
}

}  // namespace dsq
