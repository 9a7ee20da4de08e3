// Argument checks that the operators on a caller's tensors share; each sets the
// calling thread's message and returns the status.
#pragma once
#include <cstdint>

#include "capi.h"

namespace axon {

constexpr int64_t MAX_TOKENS = 1 << 30;  // token and column numbers stay 32-bit in the kernels

inline std::string num(int64_t v) { return std::to_string(v); }

inline int check_type(const char* name, int32_t dtype) {
  if (dtype != AXON_BF16 && dtype != AXON_F32)
    return fail(AXON_E_DTYPE, std::string(name) + " must be AXON_BF16 or AXON_F32, got " + num(dtype));
  return AXON_OK;
}

// a required array: not NULL, aligned to its elements
inline int check_array(const char* name, const void* p, size_t elem) {
  if (!p) return fail(AXON_E_INVALID, std::string(name) + " is NULL");
  if ((uintptr_t)p % elem) return fail(AXON_E_INVALID, std::string(name) + " is not aligned to its elements");
  return AXON_OK;
}

inline size_t size_of(int32_t dtype) { return dtype == AXON_BF16 ? 2 : 4; }

inline int check_rows(const char* name, const void* p, int32_t dtype, int64_t ld, int64_t rows, int64_t cols) {
  if (int r = check_type(name, dtype)) return r;
  if (ld < cols)
    return fail(AXON_E_INVALID, std::string("the row stride of ") + name + " is " + num(ld) + ", less than its " +
                                    num(cols) + " columns");
  return rows > 0 ? check_array(name, p, size_of(dtype)) : AXON_OK;
}

inline int check_workspace(const void* ws, int64_t bytes, int64_t need) {
  if (bytes < need) return fail(AXON_E_CAPACITY, "the workspace has " + num(bytes) + " bytes, " + num(need) + " are needed");
  if (need > 0 && !ws) return fail(AXON_E_INVALID, "workspace is NULL");
  if ((uintptr_t)ws % 16) return fail(AXON_E_INVALID, "workspace is not aligned to 16 bytes");
  return AXON_OK;
}

// prefix sums of the sequence lengths on both sides: 0 .. tokens, never falling
inline int check_cu(const int32_t* d_cu, const int32_t* h_cu, int32_t seqs, int64_t tokens) {
  if (int r = check_array("d_cu_seqlens", d_cu, 4)) return r;
  if (int r = check_array("h_cu_seqlens", h_cu, 4)) return r;
  if (h_cu[0] != 0) return fail(AXON_E_INVALID, "cu_seqlens[0] must be 0");
  for (int i = 0; i < seqs; ++i)
    if (h_cu[i + 1] < h_cu[i])
      return fail(AXON_E_INVALID, "sequence " + num(i) + " has length " + num((int64_t)h_cu[i + 1] - h_cu[i]));
  if (h_cu[seqs] != tokens)
    return fail(AXON_E_INVALID, "cu_seqlens end at " + num(h_cu[seqs]) + ", the logits have " + num(tokens) + " rows");
  return AXON_OK;
}

}  // namespace axon
