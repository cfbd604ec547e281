// 16-bit products with the operands' places exchanged: few rows of out, or outputs on no boundary.
#include "dsq_product16.cuh"

namespace dsq {

cudaError_t product16_turned(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiTurned& epi, cudaStream_t st) {
  if (a.across) return b.across ? product16<kAcross, kAcross>(plan, a, b, s, epi, st) : product16<kAcross, kAlong>(plan, a, b, s, epi, st);
  if (plan.bn != 32) return product16<kAlong, kAlong>(plan, a, b, s, epi, st);
  CUtensorMap ma, mb;
  cudaError_t e = operand_map(&ma, a, s.k, kMmaRows);
  if (e == cudaSuccess) e = operand_map(&mb, b, s.k, 32);
  if (e != cudaSuccess) return e;
  return plan.parts > 1 ? launch_mma_split<kMmaHalf, 32, kAlong, kAlong>(plan.parts, ma, mb, mb, s, epi, st)
                        : launch_mma_bn<kMmaHalf, 32, kAlong, kAlong>(ma, mb, mb, s, epi, st);
}

}  // namespace dsq
