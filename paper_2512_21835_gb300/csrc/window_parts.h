// window_parts.h -- how a block of the prompt attention ended, and what that means for
// the rows that its row tile's blocks share.
#pragma once

#ifdef __CUDACC__
#define LOIP_HD __host__ __device__
#else
#define LOIP_HD
#endif

namespace loip {

enum PartEnd : unsigned {
    kPartGood = 0,
    kPartNotFinite = 1,  // met values that are not finite and that only some rows see: the rows are walked one by one
    kPartStopped = 2,    // a wait ran out: what the block holds may be anything, and no row is stored
};
LOIP_HD constexpr unsigned part_end(bool stopped, bool not_finite) {
    return stopped ? kPartStopped : not_finite ? kPartNotFinite : kPartGood;
}
// A row tile ends as the worst of its parts.
LOIP_HD constexpr unsigned worse(unsigned a, unsigned b) { return a > b ? a : b; }

}  // namespace loip
