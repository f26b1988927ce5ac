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

// Head of the i-th workgroup of an item: the key heads take turns, so that workgroups with
// numbers equal modulo 8 (one XCD) read few key heads (Hkv = 4: one of them).
__device__ __forceinline__ int packed_head(int i, int Hkv, int G) { return i % Hkv * G + i / Hkv; }

}  // namespace fox
