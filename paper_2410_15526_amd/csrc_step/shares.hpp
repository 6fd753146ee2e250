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

// The place of unit x in its head's `per_head` units, which are sorted by their work: where a head spans several shares, each
// share takes an even sample of them in order, unit j of the `count` of its own as the fraction (j + 1/2) / count of the list.
// Cut into runs, the list would give one XCD the longest walks and another the shortest.
constexpr int dealt_place(int64_t x, int per_head, int64_t units)
{
    const int64_t each = share_size(units), begin = x / per_head * per_head, end = begin + per_head;
    const auto from = [=](int share) { return share * each < begin ? begin : share * each; };
    const auto count = [=](int share) { return (unsigned)(((share + 1) * each < end ? (share + 1) * each : end) - from(share)); };
    const int mine = (int)(x / each);
    if (mine * each <= begin && end <= (mine + 1) * each)
        return (int)(x - begin);
    const int last = (int)((end - 1) / each);
    const unsigned at = 2 * (unsigned)(x - from(mine)) + 1;
    unsigned place = 0;
    for (int share = (int)(begin / each); share <= last; ++share) { // its units at a lower fraction; of the same, lower shares'
        const unsigned m = at * count(share);
        place += ((share < mine ? m : m - 1) / count(mine) + 1) / 2;
    }
    return (int)place;
}

} // namespace sdp4
