// balance_sigmoid_grad.cu -- instances of the balance loss's pass over z.
#include "balance.cuh"

namespace eqb {

int launch_balance_sigmoid_grad(const BalanceArgs& a, int64_t tpc, cudaStream_t s) { return launch_bal_type<true, true>(a, tpc, s); }

}  // namespace eqb
