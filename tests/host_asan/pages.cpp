// csrc/pages.h: exponents of e4m3 rows against their definition, places in the pages, and the pieces of a decode step followed unit by unit.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <map>
#include <vector>

#include "pages.h"

static int fail(const char* what, long long a, long long b, long long c) {
  std::printf("%s: %lld, %lld, %lld\n", what, a, b, c);
  return 1;
}

int main() {
  for (unsigned m = 0; m < 0x7F80; ++m) {
    const uint32_t bits = m << 16;
    float most;
    std::memcpy(&most, &bits, 4);
    int e = -126;
    while ((double)most > std::ldexp(448.0, e)) ++e;
    if (kvp::e4m3_exponent(m) != e + 127) return fail("exponent", m, kvp::e4m3_exponent(m), e + 127);
  }
  for (int shift = 4; shift <= 8; ++shift)
    for (long long position = -3; position < 5000; ++position) {
      const bool in = kvp::in_table(position, 7, shift);
      if (in != (position >= 0 && position < 7 * (1 << shift))) return fail("in_table", position, shift, in);
      if (!in) continue;
      const kvp::PagePlace at = kvp::place_of((int)position, shift);
      if (at.column * (1 << shift) + at.offset != position || at.offset < 0 || at.offset >= 1 << shift || at.column >= 7)
        return fail("place", position, at.column, at.offset);
    }
  if (kvp::in_table(1ll << 31, 1 << 26, 4) || !kvp::in_table((1ll << 30) - 1, 1 << 26, 4)) return fail("in_table", 1ll << 31, 26, 4);
  // rows of the last page of a pool beyond 32 bits
  if (kvp::page_row(2147483646, 64, 63, 255, 8) != ((2147483646ull * 64 + 63) << 8) + 255) return fail("row", 0, 0, 0);

  for (int length : {0, 1, 127, 128, 129, 255, 256, 257, 1 << 30})
    if (kvp::paged_tiles(length) != (length + kvp::kPagedTile - 1LL) / kvp::kPagedTile) return fail("tiles", length, kvp::paged_tiles(length), 0);
  uint64_t seed = 1;
  auto below = [&](unsigned n) { seed = seed * 6364136223846793005ull + 1442695040888963407ull; return (unsigned)((seed >> 33) % n); };
  for (int trial = 0; trial < 3000; ++trial) {
    const unsigned workgroups = 1 + below(trial % 2 ? 40 : 700), heads = 1 + below(9);
    std::vector<unsigned> tiles(1 + below(30));
    unsigned units = 0;
    for (unsigned& t : tiles) {
      t = below(4) == 0 ? 0 : below(trial % 3 ? 6 : 300);
      units += t * heads;
    }
    const unsigned share = kvp::paged_share(units, workgroups);
    if ((unsigned long long)share * workgroups < units) return fail("share", share, workgroups, units);
    // the workgroups' side: the slot of every piece that is not whole
    std::map<unsigned, unsigned> left;             // slot -> the first unit of its sequence and head
    std::vector<unsigned> first_of(units), tiles_of(units);
    unsigned u = 0;
    for (unsigned t : tiles)
      for (unsigned h = 0; h < heads; ++h) {
        for (unsigned i = 0; i < t; ++i) first_of[u + i] = u, tiles_of[u + i] = t;
        u += t;
      }
    for (unsigned w = 0; w < workgroups; ++w) {
      const unsigned end = units < (w + 1) * share ? units : (w + 1) * share;
      for (unsigned at = w * share; at < end;) {
        const unsigned first = first_of[at], n = tiles_of[at], stop = end < first + n ? end : first + n;
        const bool whole = kvp::piece_is_whole(first, n, share);
        if (whole != (at == first && stop == first + n)) return fail("whole", first, n, share);
        if (!whole && !left.emplace(kvp::piece_slot(first, w, share), first).second) return fail("slot taken twice", first, w, share);
        at = stop;
      }
    }
    for (const auto& l : left)
      if (l.first >= 2 * workgroups) return fail("slot", l.first, workgroups, 0);
    // the side that joins them
    unsigned found = 0;
    for (unsigned at = 0; at < units; at += tiles_of[at]) {
      if (kvp::piece_is_whole(at, tiles_of[at], share)) continue;
      for (unsigned w = at / share; w <= (at + tiles_of[at] - 1) / share; ++w, ++found) {
        const auto l = left.find(kvp::piece_slot(at, w, share));
        if (l == left.end() || l->second != at) return fail("joined", at, w, share);
      }
    }
    if (found != left.size()) return fail("not joined", found, (long long)left.size(), share);
  }
  return 0;
}
