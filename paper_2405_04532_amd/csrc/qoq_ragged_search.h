// The search of 64 lanes for a number in 0 .. B, of which a condition tells whether it lies further on (internal to the library;
// host and device).
//
// A round asks 64 candidates at once, spread evenly over what is left, and keeps the part between the last that holds and the next.
// The end is a window of 64 candidates, lo + 1 .. lo + 64, one to a lane, of which the caller counts those that hold.  Counted
// are at most 63, so that lo + count lies in the window, but where the window ends at B: all 64 then mean B, the end of the range.
#pragma once
#include "qoq_layout.h"

namespace qoq {

struct LaneSearch {
    int lo, n;                                               // the number lies in lo .. lo + n

    // with n = 64 in front of B the count could be 64 and the number still be a candidate, which no lane of the window looks at
    QOQ_HD bool near(int B) const { return n < 64 || (n == 64 && lo + n == B); }
    QOQ_HD int candidate(int lane) const { return lo + (lane + 1) * ((n + 63) / 64); }
    QOQ_HD bool asks(int lane) const { return candidate(lane) <= lo + n; }
    // `holds` of the round's candidates, the first ones
    QOQ_HD void narrow(int holds)
    {
        const int step = (n + 63) / 64, left = n - holds * step;
        lo += holds * step;
        n = left < step - 1 ? left : step - 1;
    }
};

}  // namespace qoq
