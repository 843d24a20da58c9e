// Where a token lies in the pages of its sequence, the exponent of an e4m3 row, and how one decode step over the pages of many
// sequences is dealt to workgroups.  No device code: the host tests run it, too.
#pragma once

#include "key_range.h"

namespace kvp {

// ---- pages: [n_pages][n_kv_heads][page_size][head_dim], page_size = 1 << shift
struct PagePlace {
  int column;       // of the sequence's row of the table
  int offset;       // row within the page
};
KVP_HOST_DEVICE PagePlace place_of(int position, int shift) { return PagePlace{position >> shift, position & ((1 << shift) - 1)}; }
KVP_HOST_DEVICE bool in_table(long long position, int width, int shift) { return position >= 0 && position < (long long)width << shift; }
// row of a (page, head, offset), in rows of head_dim numbers
KVP_HOST_DEVICE unsigned long long page_row(int page, int n_heads, int head, int offset, int shift) {
  return (((unsigned long long)(unsigned)page * (unsigned)n_heads + (unsigned)head) << shift) + (unsigned)offset;
}

// ---- e4m3: the least e >= -126 with most <= 448 * 2^e, as e + 127, for a largest magnitude given as the lower 15 bits of a finite
// bf16.  448 = 1.75 * 2^8, and 0x60 are the bits of 1.75 behind the point.
KVP_HOST_DEVICE int e4m3_exponent(unsigned bf16_magnitude) {
  const int e = (int)(bf16_magnitude >> 7) - 8 + ((bf16_magnitude & 0x7Fu) > 0x60u ? 1 : 0);
  return e < 1 ? 1 : e;
}

// ---- decode.  A sequence's keys are cut into tiles of kPagedTile; a unit is one tile of one KV head, and the units of all sequences lie in
// one row: sequence by sequence, in it KV head by KV head, in it tile by tile.  A workgroup takes `share` units in a row, whatever sequences
// and heads they belong to: every workgroup has the same work, however the lengths are spread, and the host needs to know none of them.  The
// units of one sequence and head in one workgroup are a piece.  A workgroup has one piece at most that another workgroup's goes before (its
// first) and one that another's follows (its last, perhaps the same); every other is whole, and its result final.
constexpr int kPagedTile = 256;

KVP_HOST_DEVICE int paged_tiles(int length) { return (int)(((unsigned)length + kPagedTile - 1) / kPagedTile); }
// units of a workgroup
KVP_HOST_DEVICE unsigned paged_share(unsigned units, unsigned workgroups) { return units == 0 ? 1u : (units - 1) / workgroups + 1; }
// A sequence and head's units are first .. first + tiles - 1.
KVP_HOST_DEVICE bool piece_is_whole(unsigned first, unsigned tiles, unsigned share) { return first / share == (first + tiles - 1) / share; }
// The place of a piece's partial result: two for each workgroup, the second for a piece that is not the first of its workgroup.
KVP_HOST_DEVICE unsigned piece_slot(unsigned first, unsigned workgroup, unsigned share) { return 2 * workgroup + (first > workgroup * share ? 1u : 0u); }

}  // namespace kvp
