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
// Bound by HBM: the bf16 side is read or written once, the pages once.
#include <type_traits>

#include "lane_tools.h"
#include "serve.h"

namespace kvp {
namespace {

constexpr int kThreads = 256;

// The sequence of a token: the number of sequences that begin no later, less one.  One load and one vote for every 64 sequences.  The
// tokens of a wave are few and in a row; every lane gets that of its own.  -1 or n_seqs: none.
__device__ __forceinline__ int sequence_of(const int32_t* seq_begin, int n_seqs, int token, int lane) {
  const int from = __builtin_amdgcn_readfirstlane(token), to = __builtin_amdgcn_readlane(token, 63);
  int count = 0;
  for (int base = 0; base <= n_seqs; base += 64) {
    const bool any = base + lane <= n_seqs;
    const int begin = any ? seq_begin[base + lane] : 0;
    for (int t = from; t <= to; ++t) {
      const int n = __popcll(__ballot(any && begin <= t));
      count += t == token ? n : 0;
    }
  }
  return count - 1;
}

struct RowPlace {
  bool known;                    // the token has a sequence
  int page;                      // -1: no place in the pages
  int offset;
};
__device__ __forceinline__ RowPlace place_of_token(const PageRowsArgs& a, int token, int lane) {
  const int seq = sequence_of(a.seq_begin, a.n_seqs, token, lane);
  RowPlace p{seq >= 0 && seq < a.n_seqs, -1, 0};
  if (!p.known) return p;
  const long long position = (long long)token - a.seq_begin[seq] + (a.first != nullptr ? a.first[seq] : 0);
  if (!in_table(position, a.width, a.pool.shift)) return p;
  const PagePlace at = place_of((int)position, a.pool.shift);
  const int page = a.table[(size_t)seq * a.width + at.column];
  if (page < 0 || page >= a.pool.n_pages) return p;
  p.page = page;
  p.offset = at.offset;
  return p;
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

template <int kCtrl>
__device__ __forceinline__ int max_dpp(int x) {
  return max(x, __builtin_amdgcn_update_dpp(0, x, kCtrl, 0xF, 0xF, false));
}
// the largest finite magnitude of a row, as the lower 15 bits of a bf16, in all of its lanes
template <int kPieces>
__device__ __forceinline__ int row_magnitude(const uint4 w) {
  int most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned x = (&w.x)[i];
    const int lo = x & 0x7FFF, hi = x >> 16 & 0x7FFF;
    most = max(most, max(lo < 0x7F80 ? lo : 0, hi < 0x7F80 ? hi : 0));
  }
  most = max_dpp<0xB1>(most);                              // as row_sum
  most = max_dpp<0x4E>(most);
  most = max_dpp<0x141>(most);
  if constexpr (kPieces == 16) most = max_dpp<0x140>(most);
  return most;
}
// x / 2^e as e4m3, two at a time; what is not finite as a NaN.  Numbers that have been brought to 448 at most do not overflow.
__device__ __forceinline__ unsigned four_to_e4m3(const float a, const float b, const float c, const float d, float by) {
  auto scaled = [&](float x) { return fabsf(x) < INFINITY ? x * by : __builtin_nanf(""); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(a), scaled(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(c), scaled(d), w, true);
  return (unsigned)w;
}

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kThreads) page_write_kernel(const PageRowsArgs a) {
  constexpr int kPieces = D / 8, kRows = 64 / kPieces;
  const int lane = threadIdx.x & 63, piece = lane % kPieces;
  const unsigned row0 = (blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * kRows;
  if (row0 >= (unsigned)a.n_rows) return;
  const unsigned row = row0 + lane / kPieces;
  const bool mine = row < (unsigned)a.n_rows;                        // (the last wave: its other lanes go with the last row)
  const int at = mine ? (int)row : a.n_rows - 1;
  const int token = (int)quotient((unsigned)at, a.by_heads), head = at - token * a.pool.n_heads;
  const uint4 k = *reinterpret_cast<const uint4*>(a.k + token * a.k_token + head * a.k_head + 8 * piece);
  const uint4 v = *reinterpret_cast<const uint4*>(a.v + token * a.v_token + head * a.v_head + 8 * piece);
  const RowPlace p = place_of_token(a, token, lane);
  const size_t to = page_row(max(p.page, 0), a.pool.n_heads, head, p.offset, a.pool.shift);
  const bool write = mine && p.page >= 0;
  if constexpr (!kE4m3) {
    if (!write) return;
    reinterpret_cast<uint4*>(a.pool.k)[to * kPieces + piece] = k;
    reinterpret_cast<uint4*>(a.pool.v)[to * kPieces + piece] = v;
  } else {
    auto put = [&](const uint4 w, char* rows, uint8_t* exps) __attribute__((always_inline)) {
      const int e = e4m3_exponent((unsigned)row_magnitude<kPieces>(w));
      const float by = __uint_as_float((unsigned)(254 - e) << 23);
      float x[8];
      unpack8(w, x);
      const uint2 y = {four_to_e4m3(x[0], x[1], x[2], x[3], by), four_to_e4m3(x[4], x[5], x[6], x[7], by)};
      if (!write) return;
      reinterpret_cast<uint2*>(rows)[to * kPieces + piece] = y;
      if (piece == 0) exps[to] = (uint8_t)e;
    };
    put(k, a.pool.k, a.pool.k_exp);
    put(v, a.pool.v, a.pool.v_exp);
  }
}

__device__ __forceinline__ uint4 from_e4m3(const uint2 y, unsigned exp) {
  const float by = __uint_as_float(exp << 23);
  auto pair = [&](unsigned w, auto high) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, by, decltype(high)::value)); };
  typedef std::integral_constant<bool, false> Low;
  typedef std::integral_constant<bool, true> High;
  return uint4{pair(y.x, Low{}), pair(y.x, High{}), pair(y.y, Low{}), pair(y.y, High{})};
}

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kThreads) page_read_kernel(const PageRowsArgs a) {
  constexpr int kPieces = D / 8, kRows = 64 / kPieces;
  const int lane = threadIdx.x & 63, piece = lane % kPieces;
  const unsigned row0 = (blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * kRows;
  if (row0 >= (unsigned)a.n_rows) return;
  const unsigned row = row0 + lane / kPieces;
  const bool mine = row < (unsigned)a.n_rows;
  const int at = mine ? (int)row : a.n_rows - 1;
  const int token = (int)quotient((unsigned)at, a.by_heads), head = at - token * a.pool.n_heads;
  const RowPlace p = place_of_token(a, token, lane);
  if (!mine || !p.known) return;
  uint4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (p.page >= 0) {
    const size_t from = page_row(p.page, a.pool.n_heads, head, p.offset, a.pool.shift);
    if constexpr (kE4m3) {
      k = from_e4m3(reinterpret_cast<const uint2*>(a.pool.k)[from * kPieces + piece], a.pool.k_exp[from]);
      v = from_e4m3(reinterpret_cast<const uint2*>(a.pool.v)[from * kPieces + piece], a.pool.v_exp[from]);
    } else {
      k = reinterpret_cast<const uint4*>(a.pool.k)[from * kPieces + piece];
      v = reinterpret_cast<const uint4*>(a.pool.v)[from * kPieces + piece];
    }
  }
  *reinterpret_cast<uint4*>(a.k + token * a.k_token + head * a.k_head + 8 * piece) = k;
  *reinterpret_cast<uint4*>(a.v + token * a.v_token + head * a.v_head + 8 * piece) = v;
}

template <class Kernel>
hipError_t launch_rows(Kernel kernel, const PageRowsArgs& a, int head_dim, hipStream_t s) {
  const int rows = kThreads / (head_dim / 8);
  hipLaunchKernelGGL(kernel, dim3(((unsigned)a.n_rows + rows - 1) / rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_write(const PageRowsArgs& a, int head_dim, bool e4m3, hipStream_t s) {
  if (head_dim == 128) return launch_rows(e4m3 ? page_write_kernel<128, true> : page_write_kernel<128, false>, a, head_dim, s);
  return launch_rows(e4m3 ? page_write_kernel<64, true> : page_write_kernel<64, false>, a, head_dim, s);
}

hipError_t launch_page_read(const PageRowsArgs& a, int head_dim, bool e4m3, hipStream_t s) {
  if (head_dim == 128) return launch_rows(e4m3 ? page_read_kernel<128, true> : page_read_kernel<128, false>, a, head_dim, s);
  return launch_rows(e4m3 ? page_read_kernel<64, true> : page_read_kernel<64, false>, a, head_dim, s);
}

}  // namespace kvp
