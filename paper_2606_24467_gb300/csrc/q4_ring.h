// A warp's ring of shared-memory stages for the attention's tiles: a tile is
// copied into each stage as soon as there is one to copy, the tiles are taken
// in order, and the i-th copy into a stage completes phase i of its barrier.
// Plain C++, so that the host can run it too.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define CKV_RING_FN __host__ __device__ __forceinline__
#else
#define CKV_RING_FN inline
#endif

namespace ckv {

template <int kStages>
struct TileRing {
  int stage = 0;       // of the tile to take next
  uint32_t phase = 0;  // parity that its barrier completes with it

  CKV_RING_FN void advance() {
    if (++stage == kStages) {
      stage = 0;
      phase ^= 1u;
    }
  }
  // With `left` tiles to take, the copies that are under way (or have landed
  // and wait to be taken): of this tile and of the next ones.
  static CKV_RING_FN int in_flight(int left) { return left < kStages ? left : kStages; }
  // Stage and parity of the k-th of them.  Stages before `stage` are a round ahead.
  CKV_RING_FN int stage_of(int k) const { return stage + k < kStages ? stage + k : stage + k - kStages; }
  CKV_RING_FN uint32_t phase_of(int k) const { return stage + k < kStages ? phase : phase ^ 1u; }
};

}  // namespace ckv
