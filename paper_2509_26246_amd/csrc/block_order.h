// Which piece of a divided row of work a block takes.
#pragma once

#ifdef __HIPCC__
#define SLIMATTN_HOST_DEVICE __host__ __device__
#else
#define SLIMATTN_HOST_DEVICE
#endif

namespace slimattn {

constexpr int kXcds = 8;   // blocks are handed to the XCDs in turn, by their numbers

// The piece of block `block` when `n` blocks have work (block < n): each XCD gets a run of pieces, since neighbours read the same keys, and all XCDs the same
// number of them, give or take one.  n is what there is to do, not what was launched: the launch only knows an upper bound, and runs cut by that bound would
// put all the work on the first XCDs.
SLIMATTN_HOST_DEVICE constexpr int piece_of_block(int block, int n) {
  const int xcd = block % kXcds, more = n % kXcds;
  return xcd * (n / kXcds) + (xcd < more ? xcd : more) + block / kXcds;
}

}  // namespace slimattn
