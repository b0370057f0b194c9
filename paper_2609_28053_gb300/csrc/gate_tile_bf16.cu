// The gate of many tokens from bf16 logits (gate_tile.cuh).
#include "gate_tile.cuh"

namespace eqb {

int launch_gate_tile_bf16(const GateArgs& a, cudaStream_t s) { return launch_tile_groups<false>(a, s); }

}  // namespace eqb
