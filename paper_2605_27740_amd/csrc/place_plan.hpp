// Places on the stack of free pages. Whole numbers only (no HIP), so that they can be checked without a GPU; the kernels use the same functions.
#pragma once
#include <stdint.h>

namespace unique {

// The place behind `size` pages and `before` others that come back, where a sequence's begin, or, of all of them, the stack's new size. Each of these numbers may be nearly
// 2^31, and what does not fit is lost, so that places at and beyond the capacity need not be told apart.
constexpr int stack_place(int size, int64_t before, int capacity) { return (int)(size + before < capacity ? size + before : capacity); }

// Whether the i-th page from there on fits (a sum could pass 2^31).
constexpr bool stack_has(int place, int i, int capacity) { return i < capacity - place; }

}  // namespace unique
