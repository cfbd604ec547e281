// 16-bit products whose results are floats: gradients that go into a row of a step, or on in 32 bits.
#include "dsq_product16.cuh"

namespace dsq {

cudaError_t product16_floats(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiFloats& epi, cudaStream_t st) {
  if (!b.across) return product16<kAlong, kAlong>(plan, a, b, s, epi, st);
  return a.across ? product16<kAcross, kAcross>(plan, a, b, s, epi, st) : product16<kAlong, kAcross>(plan, a, b, s, epi, st);
}

}  // namespace dsq
