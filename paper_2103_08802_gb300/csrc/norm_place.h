// Where the norms' asynchronous copies read: at a vector's border always, also those that copy nothing.
#pragma once
#include <stdint.h>

namespace pnn {
namespace norm {

// The address at which a piece of `bytes` is read whose values lie at `at`, in a row that begins at `row`.  A piece
// that is `empty` (behind the width) copies nothing, but its address has to be aligned all the same: the border at or
// before the row's first value.  (Row 0 begins on one, so that this is inside the tensor.)
constexpr uintptr_t piece_address(uintptr_t row, uintptr_t at, bool empty, int bytes) { return empty ? row & ~(uintptr_t)(bytes - 1) : at; }

}  // namespace norm
}  // namespace pnn
