// Dropout from a counter-based generator.
#pragma once
#include "kernels.h"

namespace cephalo {

constexpr int kDropoutBlock = 256;
constexpr int64_t kDropoutMost = (((int64_t)1 << 32) / kDropoutBlock - 1) * kDropoutBlock * 8;      // a thread has 8 elements, a launch fewer than 2^32 threads
struct DropoutArgs {
  int64_t n;
  uint64_t seed, first;              // first: a multiple of 8
  const uint64_t* counter;           // device, added to `first`; may be null
  unsigned drop;                     // of the 65536 values of a word, those that drop an element
  float scale;
};
template <typename T> int launch_dropout_add(const DropoutArgs& d, const T* branch, const float* resid, float* out, hipStream_t s);
template <typename T> int launch_dropout_bwd(const DropoutArgs& d, const float* dy, T* dbranch, hipStream_t s);

}  // namespace cephalo
