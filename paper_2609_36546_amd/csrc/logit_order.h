// The order of a row's entries that sample_logits.hip and drafts.hip cut by.
#pragma once

#include "common.h"

namespace ipdv {
namespace {

// Temperatures below act as this: bins and slopes per unit of logit, 8 / T and
// log2(e) / T, stay finite in fp32.
constexpr float kLeastTemp = 0x1p-124f;

// Logits as unsigned numbers of the same order, and back to one of equal order.
__device__ __forceinline__ unsigned key_of(float l) {
  const unsigned u = __float_as_uint(l == 0.f ? 0.f : l);   // -0 is +0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of_key(unsigned key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}
// Order of entries: logit, then the lower index.
constexpr int kIndexBits = 18;
__device__ __forceinline__ unsigned long long order_of(float l, int v) {
  return ((unsigned long long)key_of(l) << kIndexBits) | (unsigned)(((1 << kIndexBits) - 1) ^ v);
}
__device__ __forceinline__ float logit_of(unsigned long long order) { return logit_of_key((unsigned)(order >> kIndexBits)); }
__device__ __forceinline__ int index_of(unsigned long long order) {
  return (int)(((1 << kIndexBits) - 1) ^ (unsigned)(order & ((1 << kIndexBits) - 1)));
}

}  // namespace
}  // namespace ipdv
