// Which arrivals of the tensor cores k_attend_tc's barriers get.  An arrival comes when the products before it are done,
// in its own time, and must not find the memory of a CTA that has ended: one is asked for only where a warp of the
// CTA waits for it.
#pragma once

namespace pnn {
namespace attend {

constexpr int RING = 5;  // tiles
// A tile's place is given back where a later load of the CTA's `loads` takes it.
constexpr bool place_again(int load, int loads) { return load + RING < loads; }
// So are a quarter's two buffers of K', which every second quarter of 4 a chunk has.
constexpr bool buffer_again(int quarter, int chunks) { return quarter + 2 < 4 * chunks; }

}  // namespace attend
}  // namespace pnn
