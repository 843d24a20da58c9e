// Rows of K and V into the pages of their sequences and back (kvp_page_write, kvp_page_read), bf16 as they are or e4m3 with a power
// of two per row.
//
// Both move a row of K and the same row of V with D / 8 lanes, 16 bytes of bf16 a lane, four (D = 64: eight) rows a wave.  A wave's rows
// are neighbours, heads fastest, so that what leaves a projection is read in whole lines; in the pages a row is a line of its own.
//
// The scale is a power of two, so dividing by it is exact and a number is rounded once, to e4m3: of a row as it is held, the numbers are
// those nearest to the input whose exponent allows four significant bits.  The way back is exact, too: a bf16 number of which four
// significant bits are left is still one (a multiple of 2^-133, and only what rounds up to 2^128 is none).
//
// Bound by HBM: the bf16 side is read or written once, the pages once (11 sequences of 32 heads, d 64, out of bf16 pages of 16: 147 us, 5.2 TB/s), and by
// latency where there are few (1024 tokens of 4 heads out of e4m3 pages 3.2 us).  bf16 into pages, four rows a wave, is not there yet: the compiler keeps three of the rows of K
// in scratch memory (17976 tokens of 8 heads, d 128, 41 us for 147 MB).
#include <type_traits>

#include "lane_tools.h"
#include "serve.h"

namespace kvp {
namespace {

constexpr int kThreads = 256;

// A wave has kUnits times the rows that its lanes hold at once, for the price of one search for their places: 4, or 1 where all waves
// run at once anyway.  (17976 tokens of 8 heads, d 128, to e4m3 25.4 us with 1 and a search for every row, 20.4 with 4; 48 tokens 3.4 and 4.2 us.)

// Where the first head's row of a token is in the pages: lane i's of token from + i.  The token's sequence is the number of those that begin no
// later, less one; -1 or n_seqs: none.  One load and a vote per token for every 64 sequences.  What is needed of the sequence itself, where it begins and
// its first place, comes out of the same load if there is only one (16640 rows of 8 heads into e4m3 pages 19.1 us with loads of their own behind it, 18.0
// so; 48 rows 2.76 and 2.73), else out of loads behind it (300 sequences 3.3 us, 3.5 with what is needed passed on from group to group).
constexpr long long kNoPlace = -1, kNoSequence = -2;
__device__ __forceinline__ long long place_of_token(const PageRowsArgs& a, int from, int to, int lane) {
  int count = 0, begin = 0, first = 0;
  if (a.n_seqs < 64 && a.first != nullptr && lane < a.n_seqs) first = a.first[lane];
  for (int base = 0; base <= a.n_seqs; base += 64) {
    const bool any = base + lane <= a.n_seqs;
    begin = any ? a.seq_begin[base + lane] : 0;
    for (int t = from; t <= to; ++t) {
      const int n = __popcll(__ballot(any && begin <= t));
      count += t == from + lane ? n : 0;
    }
  }
  const int seq = count - 1, token = from + lane;
  if (a.n_seqs < 64) begin = __shfl(begin, max(seq, 0)), first = __shfl(first, max(seq, 0));
  if (token > to || seq < 0 || seq >= a.n_seqs) return kNoSequence;
  if (a.n_seqs >= 64) begin = a.seq_begin[seq], first = a.first != nullptr ? a.first[seq] : 0;
  const long long position = (long long)token - begin + first;
  if (!in_table(position, a.width, a.pool.shift)) return kNoPlace;
  const PagePlace at = place_of((int)position, a.pool.shift);
  const int page = a.table[(size_t)seq * a.width + at.column];
  if (page < 0 || page >= a.pool.n_pages) return kNoPlace;
  return (long long)page_row(page, a.pool.n_heads, 0, at.offset, a.pool.shift);
}

// The rows of a wave: the token and head of each, 16 bytes of it to a lane.
template <int D, int kUnits>
struct WaveRows {
  static constexpr int kPieces = D / 8, kRows = 64 / kPieces;
  int piece, from, to;                            // tokens from .. to
  int token[kUnits], head[kUnits];
  bool mine[kUnits];                              // (the last wave: rows behind the last one are that one again)
  __device__ __forceinline__ bool begin(const PageRowsArgs& a, int lane) {
    const unsigned row0 = (blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * (unsigned)(kUnits * kRows);
    if (row0 >= (unsigned)a.n_rows) return false;
    piece = lane % kPieces;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const unsigned row = row0 + u * kRows + lane / kPieces;
      mine[u] = row < (unsigned)a.n_rows;
      const unsigned at = mine[u] ? row : a.n_rows - 1;
      token[u] = (int)quotient(at, a.by_heads);
      head[u] = (int)at - token[u] * a.pool.n_heads;
    }
    from = __builtin_amdgcn_readfirstlane(token[0]);
    to = __builtin_amdgcn_readlane(token[kUnits - 1], 63);
    return true;
  }
  __device__ __forceinline__ long long place(long long places, int u) const { return __shfl(places, token[u] - from); }
};

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

template <int kCtrl>
__device__ __forceinline__ u16x2 max_dpp(u16x2 x) {
  const int w = __builtin_bit_cast(int, x);
  return __builtin_elementwise_max(x, __builtin_bit_cast(u16x2, __builtin_amdgcn_update_dpp(0, w, kCtrl, 0xF, 0xF, false)));
}
// the largest magnitude of a row, as the lower 15 bits of a bf16, in all of its lanes
template <int kPieces>
__device__ __forceinline__ unsigned row_magnitude(const uint4 w) {
  auto size = [](unsigned x) { return __builtin_bit_cast(u16x2, x & 0x7FFF7FFFu); };
  u16x2 most = __builtin_elementwise_max(__builtin_elementwise_max(size(w.x), size(w.y)), __builtin_elementwise_max(size(w.z), size(w.w)));
  most = max_dpp<0xB1>(most);                              // as row_sum
  most = max_dpp<0x4E>(most);
  most = max_dpp<0x141>(most);
  if constexpr (kPieces == 16) most = max_dpp<0x140>(most);
  return most.x > most.y ? most.x : most.y;
}
constexpr unsigned kInfinite = 0x7F80;
__device__ __forceinline__ uint4 only_finite(uint4 w, unsigned instead) {          // numbers that are not finite, replaced
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned& x = (&w.x)[i];
    if ((x & 0x7FFFu) >= kInfinite) x = (x & 0xFFFF0000u) | instead;
    if ((x >> 16 & 0x7FFFu) >= kInfinite) x = (x & 0xFFFFu) | instead << 16;
  }
  return w;
}
struct E4m3 {
  uint2 numbers;
  unsigned exp;
};
// Numbers that have been brought to 448 at most do not overflow, and the division by a power of two is part of the conversion.
template <int kPieces>
__device__ __forceinline__ E4m3 to_e4m3(uint4 w) {
  unsigned most = row_magnitude<kPieces>(w);
  if (__any(most >= kInfinite)) {                          // rarely
    most = row_magnitude<kPieces>(only_finite(w, 0u));
    w = only_finite(w, 0x7FC0u);
  }
  const int e = e4m3_exponent(most);
  const float by = __uint_as_float((unsigned)e << 23);
  auto four = [&](unsigned lo, unsigned hi) {
    i16x2 y = {0, 0};
    y = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(y, __builtin_bit_cast(bf16x2, lo), by, false);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(y, __builtin_bit_cast(bf16x2, hi), by, true);
    return __builtin_bit_cast(unsigned, y);
  };
  return E4m3{uint2{four(w.x, w.y), four(w.z, w.w)}, (unsigned)e};
}

template <int D, bool kE4m3, int kUnits>
__global__ void __launch_bounds__(kThreads) page_write_kernel(const PageRowsArgs a) {
  constexpr int kPieces = D / 8;
  const int lane = threadIdx.x & 63;
  WaveRows<D, kUnits> r;
  if (!r.begin(a, lane)) return;
  uint4 k[kUnits], v[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    k[u] = *reinterpret_cast<const uint4*>(a.k + r.token[u] * a.k_token + r.head[u] * a.k_head + 8 * r.piece);
    v[u] = *reinterpret_cast<const uint4*>(a.v + r.token[u] * a.v_token + r.head[u] * a.v_head + 8 * r.piece);
  }
  const long long places = place_of_token(a, r.from, r.to, lane);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const long long place = r.place(places, u);
    const bool write = r.mine[u] && place >= 0;
    const size_t to = place + ((size_t)r.head[u] << a.pool.shift);
    if constexpr (!kE4m3) {
      if (!write) continue;
      reinterpret_cast<uint4*>(a.pool.k)[to * kPieces + r.piece] = k[u];
      reinterpret_cast<uint4*>(a.pool.v)[to * kPieces + r.piece] = v[u];
    } else {
      const E4m3 y = to_e4m3<kPieces>(k[u]), z = to_e4m3<kPieces>(v[u]);
      if (!write) continue;
      reinterpret_cast<uint2*>(a.pool.k)[to * kPieces + r.piece] = y.numbers;
      reinterpret_cast<uint2*>(a.pool.v)[to * kPieces + r.piece] = z.numbers;
      if (r.piece == 0) {
        a.pool.k_exp[to] = (uint8_t)y.exp;
        a.pool.v_exp[to] = (uint8_t)z.exp;
      }
    }
  }
}

__device__ __forceinline__ uint4 from_e4m3(const uint2 y, unsigned exp) {
  const float by = __uint_as_float(exp << 23);
  auto low = [&](unsigned w) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, by, false)); };
  auto high = [&](unsigned w) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, by, true)); };
  return uint4{low(y.x), high(y.x), low(y.y), high(y.y)};
}

template <int D, bool kE4m3, int kUnits>
__global__ void __launch_bounds__(kThreads) page_read_kernel(const PageRowsArgs a) {
  constexpr int kPieces = D / 8;
  typedef typename std::conditional<kE4m3, uint2, uint4>::type Held;
  const int lane = threadIdx.x & 63;
  WaveRows<D, kUnits> r;
  if (!r.begin(a, lane)) return;
  const long long places = place_of_token(a, r.from, r.to, lane);
  Held k[kUnits], v[kUnits];
  unsigned k_exp[kUnits], v_exp[kUnits];
  long long place[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    place[u] = r.place(places, u);
    const size_t from = max(place[u], 0ll) + ((size_t)r.head[u] << a.pool.shift);       // (rows without a place: some row, not used)
    k[u] = reinterpret_cast<const Held*>(a.pool.k)[from * kPieces + r.piece];
    v[u] = reinterpret_cast<const Held*>(a.pool.v)[from * kPieces + r.piece];
    if constexpr (kE4m3) k_exp[u] = a.pool.k_exp[from], v_exp[u] = a.pool.v_exp[from];
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (!r.mine[u] || place[u] == kNoSequence) continue;
    uint4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
    if (place[u] >= 0) {
      if constexpr (kE4m3) x = from_e4m3(k[u], k_exp[u]), y = from_e4m3(v[u], v_exp[u]);
      else x = k[u], y = v[u];
    }
    *reinterpret_cast<uint4*>(a.k + r.token[u] * a.k_token + r.head[u] * a.k_head + 8 * r.piece) = x;
    *reinterpret_cast<uint4*>(a.v + r.token[u] * a.v_token + r.head[u] * a.v_head + 8 * r.piece) = y;
  }
}

constexpr int kMostUnits = 4, kWavesOfChip = 256 * 32;

template <int D, bool kE4m3, bool kWrite, int kUnits>
hipError_t launch_units(const PageRowsArgs& a, hipStream_t s) {
  const unsigned rows = kThreads / 64 * kUnits * (512 / D), grid = ((unsigned)a.n_rows + rows - 1) / rows;
  if constexpr (kWrite) hipLaunchKernelGGL((page_write_kernel<D, kE4m3, kUnits>), dim3(grid), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((page_read_kernel<D, kE4m3, kUnits>), dim3(grid), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <bool kWrite>
hipError_t launch_rows(const PageRowsArgs& a, int head_dim, bool e4m3, hipStream_t s) {
  const bool few = a.n_rows <= kWavesOfChip * (512 / head_dim);
  if (head_dim == 128) {
    if (e4m3) return few ? launch_units<128, true, kWrite, 1>(a, s) : launch_units<128, true, kWrite, kMostUnits>(a, s);
    return few ? launch_units<128, false, kWrite, 1>(a, s) : launch_units<128, false, kWrite, kMostUnits>(a, s);
  }
  if (e4m3) return few ? launch_units<64, true, kWrite, 1>(a, s) : launch_units<64, true, kWrite, kMostUnits>(a, s);
  return few ? launch_units<64, false, kWrite, 1>(a, s) : launch_units<64, false, kWrite, kMostUnits>(a, s);
}

}  // namespace

hipError_t launch_page_write(const PageRowsArgs& a, int head_dim, bool e4m3, hipStream_t s) { return launch_rows<true>(a, head_dim, e4m3, s); }
hipError_t launch_page_read(const PageRowsArgs& a, int head_dim, bool e4m3, hipStream_t s) { return launch_rows<false>(a, head_dim, e4m3, s); }

}  // namespace kvp
