// balance_sigmoid_value.cu -- instances of the balance loss's pass over z.
#include "balance.cuh"

namespace eqb {

int launch_balance_sigmoid_value(const BalanceArgs& a, BalanceRun* run, cudaStream_t s) {
  return launch_bal_type<true, false>(a, run, s);
}

}  // namespace eqb
