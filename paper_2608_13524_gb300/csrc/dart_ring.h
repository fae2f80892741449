// The fills of a ring of stages, by number.  Host code too: a test walks it
// through a wait that runs out.
#pragma once

#ifdef __CUDACC__
#define DART_RING_FN __host__ __device__ __forceinline__
#else
#define DART_RING_FN inline
#endif

namespace dart {

// Fill i lies in stage i % kStages; its barrier's phase has the parity (i / kStages) & 1.
// Fills [used, filled) are on their way or not yet read.  Once a wait has run out
// nothing is read or filled any more, and these are what the warp has to wait
// for before it ends: the fill whose wait ran out and all behind it.
template <int kStages>
struct StageRing {
    int filled = 0, used = 0;
    static DART_RING_FN int stage(int i) { return i % kStages; }
    static DART_RING_FN unsigned parity(int i) { return static_cast<unsigned>(i / kStages) & 1u; }
    DART_RING_FN bool room() const { return filled - used < kStages; }
    // The turn of fill `used` has passed: it was read, unless a wait has run out.
    DART_RING_FN void passed(bool failed) { used += !failed; }
};

}  // namespace dart
