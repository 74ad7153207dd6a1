// Checks of arguments shared by the entry points that take tensors of rows in fp32 or bf16.
#pragma once
#include "cg_internal.h"

namespace cg {
namespace {

bool type_ok(int type) { return type == CG_TYPE_FP32 || type == CG_TYPE_BF16; }
size_t type_size(int type) { return type == CG_TYPE_FP32 ? 4 : 2; }
bool rows_fit(int64_t rows, int64_t cols) { return rows <= INT32_MAX && cols <= INT32_MAX && rows * cols <= INT32_MAX; }
// a tensor of `rows` rows: there, on an element's boundary, rows that do not overlap
bool tensor_ok(const void *p, int64_t ld, int64_t cols, int type)
{
    return p && (reinterpret_cast<uintptr_t>(p) & (type_size(type) - 1)) == 0 && ld >= cols;
}
bool optional_ok(const void *p, int64_t ld, int64_t cols, int type) { return !p || tensor_ok(p, ld, cols, type); }
bool floats_ok(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

}  // namespace
}  // namespace cg
