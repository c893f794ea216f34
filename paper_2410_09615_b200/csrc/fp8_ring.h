// The stages of the 8-bit layer's kernels (fwd_fp8.cu), for the kernels and (as plain C++) for the model of their barriers in the tests.
//
// Group g of a CTA (or pair) uses place g % places of the ring.  A loader waits for the MMAs of group g - places before it asks for group g, so
// behind its last request the arrivals of the last `places` groups are still to come: they are asynchronous (tcgen05.commit), in a pair from the
// other CTA, and nothing else in the kernel waits for them.  A CTA that left before them would have them written into shared memory that
// is another CTA's by then, so a loader waits for them too.
#pragma once
#include "handover.h"

namespace slim {

// The first group whose release its loader has not waited for when it has requested `requested` of them.
SLIM_BOTH int ring_tail(int requested, int places) { return requested > places ? requested - places : 0; }

}  // namespace slim
