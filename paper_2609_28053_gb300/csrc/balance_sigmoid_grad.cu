// balance_sigmoid_grad.cu -- instances of the balance loss's pass over z.
#include "balance.cuh"

namespace eqb {

int launch_balance_sigmoid_grad(const BalanceArgs& a, BalanceRun* run, cudaStream_t s) {
  return launch_bal_type<true, true>(a, run, s);
}

}  // namespace eqb
