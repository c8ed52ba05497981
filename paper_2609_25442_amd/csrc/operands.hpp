// What the operators' C entries check of their operands (ops_api.cpp, train_api.cpp).
#ifndef WB_OPERANDS_HPP
#define WB_OPERANDS_HPP

#include <hip/hip_runtime_api.h>

#include <string>

#include "entry.hpp"
#include "ops.hpp"

namespace wb {

constexpr int64_t kMaxRows = 4194303;            // a row may take a workgroup of 1024 threads: 2^32 in a launch
constexpr int64_t kMaxCols = int64_t(1) << 26;  // 2048 to a workgroup in y of a launch
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxExtent = int64_t(1) << 50;  // rows times row distance: bytes and offsets stay within 63 bits

inline bool is_float(int32_t t) { return t == WB_F32 || t == WB_BF16; }
inline int64_t type_bytes(int32_t t) { return t == WB_F32 ? 4 : t == WB_BF16 ? 2 : 1; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// One call's operands: each is refused for the first thing wrong with it, and
// `rc` keeps the first refusal.
struct Operands {
  KnownRange range;
  int rc = WB_OK;
  bool memory = true;  // look pointers up

  int refuse(const std::string& msg) {
    if (rc == WB_OK) rc = set_error(WB_EINVAL, msg);
    return rc;
  }

  void array(const void* p, int64_t count, int64_t bytes_each, const char* name) {
    if (rc != WB_OK || count == 0 || !memory) return;
    rc = check_extent_as(p, count * bytes_each, [&] { return std::string(name); }, static_cast<int>(bytes_each), &range);
  }

  void matrix(const wb_matrix& m, int64_t rows, int64_t cols, const char* name) {
    if (rc != WB_OK) return;
    if (m.rows != rows || m.cols != cols) {
      refuse(std::string(name) + " is " + std::to_string(m.rows) + " x " + std::to_string(m.cols) + ", not " +
             std::to_string(rows) + " x " + std::to_string(cols));
      return;
    }
    if (rows < 0 || cols < 1 || cols > kMaxCols || m.ld < cols || m.ld > kMaxStride || rows > kMaxExtent / m.ld) {
      refuse(std::string(name) + ": sizes or row distance out of range");
      return;
    }
    if (rows == 0 || !memory) return;
    const int64_t es = type_bytes(m.dtype);
    rc = check_extent_as(m.data, ((rows - 1) * m.ld + cols) * es, [&] { return std::string(name); }, static_cast<int>(es),
                         &range);
  }

  void floats(const wb_matrix& m, const char* name) {
    if (rc == WB_OK && !is_float(m.dtype)) refuse(std::string(name) + " is neither WB_F32 nor WB_BF16");
  }

  void scales(const wb_matrix& m, int64_t rows, int64_t cols, const char* name) {
    if (rc == WB_OK && m.data == nullptr && rows > 0) refuse(std::string(name) + " is null: fp8 values need scales");
    if (rc == WB_OK && m.dtype != WB_F32) refuse(std::string(name) + " is not WB_F32");
    matrix(m, rows, cols, name);
  }

  // a result of any of the three types
  void result(const wb_matrix& out, const wb_matrix* scales_of, int64_t rows, int64_t cols) {
    if (rc == WB_OK && !is_float(out.dtype) && out.dtype != WB_F8E4M3) refuse("out: unknown type");
    matrix(out, rows, cols, "out");
    const bool given = scales_of && scales_of->data;
    if (rc == WB_OK && out.dtype == WB_F8E4M3) {
      if (!scales_of) {
        refuse("fp8 out needs scales");
      } else {
        scales(*scales_of, rows, ceil_div(cols, kScaleBlock), "scales of out");
      }
    } else if (rc == WB_OK && given) {
      refuse("scales are given for an out that is not fp8");
    }
  }
};

inline int too_many_rows(int64_t rows) {
  if (rows < 0) return set_error(WB_EINVAL, "negative number of rows");
  if (rows > kMaxRows) return set_error(WB_EUNSUPPORTED, "more than 4194303 rows");
  return WB_OK;
}

inline int launched(int e, const char* what) { return e == 0 ? WB_OK : hip_fail(static_cast<hipError_t>(e), what); }

}  // namespace wb

#endif
