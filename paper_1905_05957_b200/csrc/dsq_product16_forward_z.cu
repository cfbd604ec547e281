// 16-bit products, both operands along K, with the values before the activation as a second result: the forward product in training.
#include "dsq_product16.cuh"

namespace dsq {

cudaError_t product16_forward_z(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiBlocks<2>& epi, cudaStream_t st) {
  return product16<kAlong, kAlong>(plan, a, b, s, epi, st);
}

}  // namespace dsq
