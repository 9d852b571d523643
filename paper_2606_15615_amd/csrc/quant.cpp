// C ABI of the 8-bit rows and products: argument checks and launches.  Every
// call enqueues on the caller's stream and neither allocates nor waits.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "internal.h"
#include "moeca.h"

namespace {

int fail(int code, const std::string& m) { return moeca::set_error(code, m); }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int64_t kMaxK = 1 << 20;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1024;

int launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return MOECA_OK;
  return fail(MOECA_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// What every call on rows of the activation type checks of them.
const char* bad_rows(const void* p, int dtype, int64_t rows, int64_t K, int64_t ld) {
  if (dtype != MOECA_DTYPE_BF16 && dtype != MOECA_DTYPE_FP32) return "unknown dtype";
  if (rows < 0 || rows > kMaxRows) return "rows out of range";
  if (K < 1 || K > kMaxK) return "K and N must be in [1, 1048576]";
  if (ld < K || ld > (int64_t(1) << 40)) return "the row stride must be at least K";
  if (rows > 0 && p == nullptr) return "the rows are NULL";
  if ((reinterpret_cast<uintptr_t>(p) & (dtype == MOECA_DTYPE_BF16 ? 1u : 3u)) != 0)
    return "the rows are not aligned to their type";
  return nullptr;
}

}  // namespace

extern "C" {

size_t moeca_quant_pitch(int64_t K) {
  return K < 1 ? 0 : static_cast<size_t>((K + 127) / 128 * 128);
}

size_t moeca_quant_scale_pitch(int64_t K) {
  return K < 1 ? 0 : static_cast<size_t>(((K + 127) / 128 + 15) / 16 * 16);
}

int moeca_quant_rows(const void* src, int dtype, int64_t rows, int64_t K, int64_t ld,
                     const int32_t* slot, int64_t slots, void* q, void* scale, float* norm,
                     void* stream) {
  if (const char* m = bad_rows(src, dtype, rows, K, ld)) return fail(MOECA_E_INVAL, m);
  if (slots < 0 || slots > kMaxRows) return fail(MOECA_E_INVAL, "slots out of range");
  if (slot == nullptr && rows > slots)
    return fail(MOECA_E_INVAL, "more rows than slots, and no slot indexes");
  if (rows == 0 || slots == 0) return MOECA_OK;
  if (q == nullptr || scale == nullptr)
    return fail(MOECA_E_INVAL, "the quantised elements and scales are required");
  if (!aligned16(q) || !aligned16(scale))
    return fail(MOECA_E_INVAL, "quantised elements and scales must be 16-byte aligned");
  if (((reinterpret_cast<uintptr_t>(slot) | reinterpret_cast<uintptr_t>(norm)) & 3u) != 0)
    return fail(MOECA_E_INVAL, "slots and norms must be 4-byte aligned");
  return launched(moeca::launch_quant_rows(src, dtype == MOECA_DTYPE_BF16, rows,
                                           static_cast<int>(K), ld, slot, nullptr, slots,
                                           static_cast<uint8_t*>(q), static_cast<uint8_t*>(scale),
                                           norm, static_cast<hipStream_t>(stream)),
                  "quantise rows");
}

int moeca_dequant_rows(const void* q, const void* scale, int64_t slots, int64_t K,
                       const int32_t* slot, int64_t rows, void* dst, int dtype, int64_t ld,
                       void* stream) {
  if (const char* m = bad_rows(dst, dtype, rows, K, ld)) return fail(MOECA_E_INVAL, m);
  if (slots < 0 || slots > kMaxRows) return fail(MOECA_E_INVAL, "slots out of range");
  if (slot == nullptr && rows > slots)
    return fail(MOECA_E_INVAL, "more rows than slots, and no slot indexes");
  if (rows == 0) return MOECA_OK;
  if (slots > 0 && (q == nullptr || scale == nullptr))
    return fail(MOECA_E_INVAL, "the quantised elements and scales are required");
  if (!aligned16(q) || !aligned16(scale))
    return fail(MOECA_E_INVAL, "quantised elements and scales must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(slot) & 3u) != 0)
    return fail(MOECA_E_INVAL, "slots must be 4-byte aligned");
  return launched(moeca::launch_dequant_rows(static_cast<const uint8_t*>(q),
                                             static_cast<const uint8_t*>(scale), slots,
                                             static_cast<int>(K), slot, rows, dst,
                                             dtype == MOECA_DTYPE_BF16, ld,
                                             static_cast<hipStream_t>(stream)),
                  "read quantised rows");
}

int moeca_quant_matrix(const void* W, int dtype, int64_t count, int64_t N, int64_t K, void* q,
                       void* scale, void* stream) {
  if (const char* m = bad_rows(W, dtype, count, K, K)) return fail(MOECA_E_INVAL, m);
  if (count > 65535) return fail(MOECA_E_INVAL, "at most 65535 matrices in a call");
  if (N < 1 || N > kMaxK) return fail(MOECA_E_INVAL, "K and N must be in [1, 1048576]");
  if (count == 0) return MOECA_OK;
  if (q == nullptr || scale == nullptr)
    return fail(MOECA_E_INVAL, "the quantised elements and scales are required");
  if (!aligned16(q) || !aligned16(scale))
    return fail(MOECA_E_INVAL, "quantised elements and scales must be 16-byte aligned");
  return launched(moeca::launch_quant_matrix(W, dtype == MOECA_DTYPE_BF16,
                                             static_cast<int>(count), static_cast<int>(N),
                                             static_cast<int>(K), static_cast<uint8_t*>(q),
                                             static_cast<uint8_t*>(scale),
                                             static_cast<hipStream_t>(stream)),
                  "quantise matrix");
}

size_t moeca_quant_linear_bytes(int64_t M, int64_t K) {
  return M < 1 || K < 1 ? 0 : moeca::q8_bytes(M, K);
}

int moeca_quant_linear(const void* x, int dtype, int64_t M, int64_t K, int64_t ldx, const void* q,
                       const void* scale, int64_t N, const float* bias, void* out, int64_t ldo,
                       void* workspace, size_t bytes, void* stream) {
  if (const char* m = bad_rows(x, dtype, M, K, ldx)) return fail(MOECA_E_INVAL, m);
  if (const char* m = bad_rows(out, dtype, M, N, ldo)) return fail(MOECA_E_INVAL, m);
  if (M == 0) return MOECA_OK;
  if (((M + 127) / 128) * ((N + 127) / 128) >= (int64_t(1) << 31))
    return fail(MOECA_E_INVAL, "M * N too large");
  if (q == nullptr || scale == nullptr)
    return fail(MOECA_E_INVAL, "the weights' elements and scales are required");
  if (!aligned16(q) || !aligned16(scale))
    return fail(MOECA_E_INVAL, "quantised elements and scales must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(bias) & 3u) != 0)
    return fail(MOECA_E_INVAL, "the bias must be 4-byte aligned");
  if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(MOECA_E_INVAL, "a 256-byte aligned workspace is required");
  if (bytes < moeca::q8_bytes(M, K))
    return fail(MOECA_E_INVAL, "workspace too small: need " +
                                   std::to_string(moeca::q8_bytes(M, K)) + " bytes, got " +
                                   std::to_string(bytes));
  const auto st = static_cast<hipStream_t>(stream);
  const bool bf16 = dtype == MOECA_DTYPE_BF16;
  if (M <= moeca::q8_few_rows())
    return launched(moeca::launch_q8_few(x, bf16, M, static_cast<int>(K), ldx, q, scale,
                                         static_cast<int>(N), bias, out, ldo, st),
                    "quantised product");
  const moeca::Q8 v = moeca::q8_view(workspace, M, K);
  const hipError_t e = moeca::launch_quant_rows(x, bf16, M, static_cast<int>(K), ldx, nullptr,
                                                nullptr, M, v.q, v.s, nullptr, st);
  if (e != hipSuccess) return launched(e, "quantise rows");
  return launched(moeca::launch_q8_linear(v, M, static_cast<int>(K), q, scale,
                                          static_cast<int>(N), bias, out, bf16, ldo, st),
                  "quantised product");
}

}  // extern "C"
