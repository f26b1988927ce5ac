// Packed sequences: the work list that the attention kernels walk.
#pragma once

#include "fox_device.h"

namespace fox {

constexpr int kPackedBlock = 128;  // rows of a work item
// A block of rows of one sequence: rows start + 128 block .. of the packed tensors, the
// sequence being rows start .. start + len - 1.  len = 0: an unused place of the list.
struct PackedItem {
  int start, len, block, seq;
};
// Item i of a list for N rows.  One that does not lie within them (a list made for another
// batch) counts as unused, so that no list leads out of the tensors.
__device__ __forceinline__ PackedItem packed_item(const PackedItem* __restrict__ plan, size_t i,
                                                  int N) {
  PackedItem it = plan[i];
  const bool inside = it.start >= 0 && it.start <= N && it.len <= N - it.start && it.block >= 0 &&
                      it.block < (it.len + kPackedBlock - 1) / kPackedBlock;
  if (!inside) it.len = 0;
  return it;
}

// Head of the i-th workgroup of an item: the key heads take turns, so that workgroups with
// numbers equal modulo 8 (one XCD) read few key heads (Hkv = 4: one of them).
__device__ __forceinline__ int packed_head(int i, int Hkv, int G) { return i % Hkv * G + i / Hkv; }

}  // namespace fox
