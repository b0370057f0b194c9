// The gate of many tokens from fp32 logits (gate_tile.cuh).
#include "gate_tile.cuh"

namespace eqb {

int launch_gate_tile_fp32(const GateArgs& a, cudaStream_t s) { return launch_tile_groups<true>(a, s); }

}  // namespace eqb
