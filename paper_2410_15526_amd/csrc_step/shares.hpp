// shares.hpp -- which work item of an attention kernel a block takes.  Plain
// arithmetic, for the host too.
#pragma once

#include <stdint.h>

namespace sdp4 {

// Work items in eight shares, one for each XCD: blocks are dealt to the XCDs in turn, so the blocks of one share, which read the
// same keys and values, meet in one L2.  A grid of more blocks than these (beyond 2^22 it is rounded up) has none for the others:
// they get `items`.
constexpr int64_t share_size(int64_t items) { return (items + 7) / 8; }
constexpr int64_t shared_blocks(int64_t items) { return 8 * share_size(items); }
constexpr int64_t shared_item(int64_t block, int64_t items)
{
    return (block >> 3) < share_size(items) ? (block & 7) * share_size(items) + (block >> 3) : items;
}

} // namespace sdp4
