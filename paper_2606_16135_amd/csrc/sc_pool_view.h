// Device-side addressing of a pool's blocks (rope.hip, decode_attn.hip).
#pragma once

#include "sc_internal.h"

namespace sc {

// t / block_size for 0 <= t < 2^31.
__device__ __forceinline__ int block_of(const PoolView &p, int t) {
  return (int)(((uint64_t)(uint32_t)t * p.block_magic) >> (31 + p.block_shift));
}

// The layer's slice of block `id` (its K half), or nullptr for an id outside
// the pool or beyond the HBM blocks it lends.
__device__ __forceinline__ char *block_layer(const PoolView &p, int32_t id) {
  // Selects between scalar values: indexing p's arrays by a lane's tier
  // would read the kernel arguments back through memory.
  const int64_t host0 = p.first[0], rc0 = p.first[1], lent = p.lent;
  char *const dev = p.tier[0], *const host = p.tier[1], *const rc = p.tier[2];
  const bool in_dev = id < host0, in_rc = id >= rc0;
  const bool ok = id >= 0 && id < p.n_ids && (!in_dev || id < lent);
  char *const base = in_dev ? dev : in_rc ? rc : host;
  const int32_t local = id - (in_dev ? 0 : in_rc ? (int32_t)rc0 : (int32_t)host0);
  char *const at = base + (int64_t)local * p.block_bytes + p.layer_off;
  return ok ? at : nullptr;
}

}  // namespace sc
