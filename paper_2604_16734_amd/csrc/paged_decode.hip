// One decode step of many sequences, each over its own pages (kvp_paged_decode): out = softmax(scale q K^T) V with one query row per
// query head.
//
// Bound by HBM (96 sequences of up to 16640 keys, 12 of them without any, 32/8 heads, d 128, bf16: 314 us, 5.7 TB/s, what a copy reaches): every key and value is read once
// and meets the G query heads of its KV head, 4 G flops for two numbers.  So what counts is
// that every CU has loads on their way all the time, and that none of them has more to do than the others.
//
// Who does what.  The lengths are on the device, and the host plans nothing: pages.h deals the units of all sequences, tiles of 256 keys of
// one KV head, to a fixed number of workgroups, as many as the chip holds at once, in equal shares; a workgroup finds its share by adding up the
// lengths.  A piece that is all of a sequence and head is finished at once; the partial results (maximum, sum, unscaled output) of the others go
// to the workspace, and a second kernel joins them, in the order of the workgroups, so that the same input gives the same bits.
//
// Within a tile each of the eight waves takes 32 keys by itself, through two strips of LDS of its own, one for K and one for V: the next
// tile's K is on its way as soon as this one's has been read, and the same for V; no barrier until a piece is done.  The rows come by
// buffer_load ... lds, 16 at a time (no page is shorter), through descriptors that end with the last row there is: rows behind a
// sequence's end, and of pages that do not exist, come as zeros without being read.
//
// Products.  S^T = K Q^T with 16x16x32 matrix instructions: rows are 16 keys, columns the query heads of the KV head (up to 16; the columns
// beyond repeat the last one and are dropped).  A lane has four neighbouring keys of one query head of each 16, and these eight exponentials are, as they lie, its
// part of the second operand of O^T = V^T P^T, whose first comes out of LDS by transposing reads in the same order of keys.  e4m3 numbers
// become bf16 on the way from LDS to the matrix instruction, exactly; the powers of two of the rows are applied to the keys and to the
// weights (V), exactly, too, but for weights that come out below 2^-126, the least bf16 number of full precision.  Sums and maxima are in fp32; weights are rounded to bf16 for the product only.
#include <type_traits>

#include "mfma_tools.h"
#include "serve.h"

namespace kvp {
namespace {

constexpr int kKeys = 32;                      // keys of a wave's part of a tile: two blocks of 16
constexpr int kHeads = 16;                     // columns of the products
constexpr int kWaves = 8, kThreads = 64 * kWaves;
static_assert(kKeys * kWaves == kPagedTile, "tiles of pages.h");

typedef int i32x2 __attribute__((ext_vector_type(2)));

// Ways to spread the work: in shares, as above; or a workgroup for every sequence and KV head, with nothing to join.
enum Way { kShares, kAlone };

template <int D, bool kE4m3>
struct Shape {
  static constexpr int kRow = kE4m3 ? D : 2 * D;                  // bytes of a row in the pages
  static constexpr int kChunks = kRow / 16;
  static constexpr int kLoads = kRow / 64;                        // of 1 KiB, for 16 rows
  static constexpr int kStrip = kKeys * kRow;
  static constexpr int kExps = kE4m3 ? 256 : 0;
  static constexpr int kWaveBytes = 2 * kStrip + kExps;           // K, V, exponents
  static constexpr int kLds = kWaves * kWaveBytes;
  static constexpr int kPerCu = kLds > 80 * 1024 ? 1 : 2;         // workgroups of a CU
  // what a wave leaves of a piece lies over its strips: the output as it is in the accumulators, then maxima and sums
  static constexpr int kOut = kHeads * D * 4, kStat = kE4m3 ? 2 * kStrip : kOut;
  static_assert(kOut <= 2 * kStrip && kStat + 2 * kHeads * 4 <= kWaveBytes, "room for a piece");
};

// In LDS the 16-byte chunk ch of row r lies at position ch ^ f(r), for reads free of bank conflicts.  K is read in chunks of one
// column, 16 rows at a time; V by transposing reads of 8 bytes, of which half a wave's touch eight rows (bf16: 0 .. 7) or 16 (e4m3: 0 .. 7
// and 16 .. 23).
template <int kRow>
__device__ __forceinline__ int k_swizzle(int row) { return row / (256 / kRow) % (kRow / 16); }
template <int kRow, bool kE4m3>
__device__ __forceinline__ int v_swizzle_of(int row) {
  if constexpr (!kE4m3) return 2 * (row / (256 / kRow) % (kRow / 32));
  else return row / (256 / kRow) % (kRow / 32) + kRow / 32 * (row / 16 % 2);
}

// eight e4m3 numbers times a power of two as bf16, exactly
__device__ __forceinline__ bf16x8 eight_of_e4m3(unsigned lo, unsigned hi, float by) {
  const u32x4 w = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false)),
                   __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true)),
                   __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false)),
                   __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true))};
  return __builtin_bit_cast(bf16x8, w);
}
// the larger one, in one instruction (fmaxf makes NaNs quiet first, with one more for each operand)
__device__ __forceinline__ float max_of(float x, float y) {
  float m;
  asm("v_max_f32 %0, %1, %2" : "=v"(m) : "v"(x), "v"(y));
  return m;
}
__device__ __forceinline__ float max_of(float x, float y, float z) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(x), "v"(y), "v"(z));
  return m;
}
// 2^e of the i-th of four exponents
__device__ __forceinline__ float power_of(unsigned exps, int i) { return __uint_as_float((exps >> (8 * i) & 0xFFu) << 23); }
// two transposing reads: four keys of this lane's channel, and the four that lie `rows` bytes further
__device__ __forceinline__ bf16x8 lds_read_vt16(const unsigned char* p, int rows) {
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((i16x4 __attribute__((address_space(3)))*)(p));
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((i16x4 __attribute__((address_space(3)))*)(p + rows));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Logits that are all minus infinity leave a sum of 0, as no key does.  To tell 0 / 0 from a result of zeros the reference of a part with keys is never
// less than the lowest number, beside which a sum of 0 is as good as beside minus infinity.
constexpr float kLowest = -3.40282347e38f;
__device__ __forceinline__ float inverse_of(float sum, float reference) { return sum == 0.f ? (reference == -INFINITY ? 0.f : NAN) : 1.f / sum; }

// ---- where the units of the sequences begin, in all lanes of a wave
__device__ __forceinline__ int length_of(const PagedDecodeArgs& a, int seq) {
  return seq < a.n_seqs ? min(max(a.lengths[seq], 0), a.width << a.pool.shift) : 0;
}
// Not in shares: workgroup b has all of sequence b / n_heads, KV head b % n_heads, and there is nothing to join.
template <int D, bool kE4m3, Way kWay>
__global__ void __launch_bounds__(kThreads, 4)
paged_decode_kernel(const PagedDecodeArgs a) {
  using S = Shape<D, kE4m3>;
  constexpr bool kDirect = kWay == kAlone;
  constexpr int kRow = S::kRow, kChunks = S::kChunks, kLoads = S::kLoads;
  constexpr int kSteps = D / 32;                 // products with K of a block of 16 keys
  constexpr int kTiles = D / 16;                 // channel tiles of the output
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // ---- this workgroup's share, and the sequence that it begins in
  unsigned at = 0, end = 1, share = 1;
  int seq = -1, n_keys = 0, direct_head = 0;
  // of 64 sequences at a time: lengths, and the units up to each
  int group0 = 0, length = 0;
  unsigned before = 0, tiles = 0, upto = 0;
  auto next_group = [&](int from) __attribute__((always_inline)) {
    before += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
    group0 = from;
    length = length_of(a, group0 + lane);
    tiles = (unsigned)paged_tiles(length) * (unsigned)a.pool.n_heads;
    upto = (unsigned)sum_upto((int)tiles);
  };
  // lane i: the page of block i % 2 of this wave's 32 keys in tile base + i / 2
  int ids = -1;
  auto load_ids = [&](int base, int most) __attribute__((always_inline)) {
    const int at = kPagedTile * (base + lane / 2) + kKeys * wave + 16 * (lane & 1);
    ids = at < most ? a.table[(size_t)seq * a.width + (at >> a.pool.shift)] : -1;
  };
  if constexpr (kDirect) {
    seq = (int)quotient(blockIdx.x, a.by_heads);
    direct_head = (int)blockIdx.x - seq * a.pool.n_heads;
    load_ids(0, a.width << a.pool.shift);            // (beside the length, not after it)
    n_keys = __builtin_amdgcn_readfirstlane(length_of(a, seq));
    if (n_keys == 0) {
      for (int i = threadIdx.x; i < a.group * D / 8; i += kThreads)
        reinterpret_cast<u32x4*>(a.out + ((size_t)seq * a.n_q_heads + direct_head * a.group) * D)[i] = u32x4{0u, 0u, 0u, 0u};
      return;
    }
  } else {
    next_group(0);
    int others = 0;
    for (int s = 64 + lane; s < a.n_seqs; s += 64) others += paged_tiles(length_of(a, s));
    unsigned units = (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
    if (a.n_seqs > 64) units += (unsigned)sum_of_wave(others) * (unsigned)a.pool.n_heads;
    share = (unsigned)__builtin_amdgcn_readfirstlane(paged_share(units, (unsigned)a.workgroups));
    at = blockIdx.x * share;
    if (at >= units) return;
    end = min(units, at + share);
  }

  // ---- LDS: [wave][K strip, V strip, exponents]
  unsigned char* const k_strip = lds + wave * S::kWaveBytes;
  unsigned char* const v_strip = k_strip + S::kStrip;
  unsigned char* const exps = v_strip + S::kStrip;
  const unsigned lds_at =
      __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) void*)lds) + (unsigned)(wave * S::kWaveBytes);

  // ---- global -> LDS.  Load i of 16 rows brings in rows 1024 / kRow * i + ..; its immediate offset moves both of its addresses by 1 KiB.
  // (Inline assembly, and waits of this kernel's own: the compiler would have every read of LDS wait for all loads.  s_nop: a load may read a
  // scalar register five wait states after a vector instruction has written it.)
  unsigned k_lane[kLoads], v_lane[2][kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int sub = lane / kChunks, pos = lane % kChunks, row = 1024 / kRow * i + sub;
    k_lane[i] = (unsigned)(sub * kRow + 16 * (pos ^ k_swizzle<kRow>(row)));
#pragma unroll
    for (int b = 0; b < 2; ++b) v_lane[b][i] = (unsigned)(sub * kRow + 16 * (pos ^ v_swizzle_of<kRow, kE4m3>(16 * b + row)));
  }
  auto load_rows = [&](u32x4 buffer, const unsigned (&of)[kLoads], unsigned to) __attribute__((always_inline)) {
    if constexpr (kLoads == 4)
      asm volatile("s_mov_b32 m0, %5\n\ts_nop 3\n\t"
                   "buffer_load_dwordx4 %0, %4, 0 offen lds\n\t"
                   "buffer_load_dwordx4 %1, %4, 0 offen offset:1024 lds\n\t"
                   "buffer_load_dwordx4 %2, %4, 0 offen offset:2048 lds\n\t"
                   "buffer_load_dwordx4 %3, %4, 0 offen offset:3072 lds" ::"v"(of[0]), "v"(of[1]), "v"(of[2]), "v"(of[3]), "s"(buffer), "s"(to)
                   : "m0", "memory");
    else if constexpr (kLoads == 2)
      asm volatile("s_mov_b32 m0, %3\n\ts_nop 3\n\t"
                   "buffer_load_dwordx4 %0, %2, 0 offen lds\n\t"
                   "buffer_load_dwordx4 %1, %2, 0 offen offset:1024 lds" ::"v"(of[0]), "v"(of[1]), "s"(buffer), "s"(to)
                   : "m0", "memory");
    else
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\t"
                   "buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(of[0]), "s"(buffer), "s"(to)
                   : "m0", "memory");
  };
  auto buffer_at = [&](const char* base, unsigned bytes) __attribute__((always_inline)) -> u32x4 {
    const unsigned long long x = (unsigned long long)base;
    // (through the first lane: the compiler would carry some of it in vector registers)
    return u32x4{(unsigned)__builtin_amdgcn_readfirstlane((int)x), (unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) & 0xFFFFu,
                 (unsigned)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
  };
  auto wait_all_but = [&](auto newest) __attribute__((always_inline)) {
    constexpr int k = decltype(newest)::value;
    static_assert(k < 64);
    __builtin_amdgcn_s_waitcnt(0x0F70 | (k & 15) | (k >> 4 << 14));
    asm volatile("" ::: "memory");
  };
  typedef std::integral_constant<int, 2 * kLoads + (kE4m3 ? 1 : 0)> KLoads;      // of a tile: exponents and K
  typedef std::integral_constant<int, 2 * kLoads> VLoads;
  typedef std::integral_constant<int, 0> None;

  // ---- where the fragments are
  int k_off[kSteps], v_off[kTiles];
  if constexpr (!kE4m3) {
#pragma unroll
    for (int st = 0; st < kSteps; ++st) k_off[st] = l16 * kRow + 16 * ((4 * st + g) ^ k_swizzle<kRow>(l16));
    const int row = 4 * g + l16 / 4;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
      v_off[dt] = row * kRow + 16 * ((2 * dt + l16 % 4 / 2) ^ v_swizzle_of<kRow, kE4m3>(row)) + 8 * (l16 & 1);
  } else {
#pragma unroll
    for (int st = 0; st < kSteps; ++st) k_off[st] = l16 * kRow + 16 * ((4 * (st / 2) + g) ^ k_swizzle<kRow>(l16));      // 16 channels: two steps
    const int key = l16 / 2, row = key < 4 ? 4 * g + key : 16 + 4 * g + key - 4;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) v_off[dt] = row * kRow + 16 * (dt ^ v_swizzle_of<kRow, kE4m3>(row)) + 8 * (l16 & 1);
  }
  const float sl2 = a.scale_log2;

  // ---- pieces
  unsigned seq_first = 0, seq_end = 0;
  while (at < end) {
    if (!kDirect && (seq < 0 || at >= seq_end)) {               // the sequence of unit `at`
      while (before + (unsigned)__builtin_amdgcn_readlane((int)upto, 63) <= at && group0 + 64 < a.n_seqs) next_group(group0 + 64);
      const int i = __builtin_ctzll(__ballot(before + upto > at));
      seq = group0 + i;
      n_keys = __builtin_amdgcn_readlane(length, i);
      seq_end = before + (unsigned)__builtin_amdgcn_readlane((int)upto, i);
      seq_first = seq_end - (unsigned)__builtin_amdgcn_readlane((int)tiles, i);
    }
    const unsigned n_tiles = (unsigned)paged_tiles(n_keys);
    const int head = kDirect ? direct_head : __builtin_amdgcn_readfirstlane((int)((at - seq_first) / n_tiles));
    const unsigned first = seq_first + (unsigned)head * n_tiles;      // the first unit of this sequence and head
    const int t0 = kDirect ? 0 : (int)(at - first), t1 = kDirect ? (int)n_tiles : (int)(min(end, first + n_tiles) - first);

    // Where the two blocks of 16 keys of 32 tiles, from tile base on, begin in the pages, and how many bytes of them there are: one to a lane, as
    // in ids.  (Read out of there, three numbers for a block, they cost a tile a third of what finding them costs.)
    int base = t0;
    unsigned long long block_at = 0;
    unsigned block_bytes = 0;
    auto find_blocks = [&]() __attribute__((always_inline)) {
      const int at = kPagedTile * (base + lane / 2) + kKeys * wave + 16 * (lane & 1);
      const bool there = at < n_keys && ids >= 0 && ids < a.pool.n_pages;
      block_at = there ? page_row(ids, a.pool.n_heads, head, place_of(at, a.pool.shift).offset, a.pool.shift) * kRow : 0ull;
      block_bytes = there ? (unsigned)min(16, n_keys - at) * kRow : 0u;
      asm volatile("" : "+v"(block_at), "+v"(block_bytes));      // here, not where they are used: the wait there would be for all loads, every time
    };
    if (kDirect) find_blocks();
    else load_ids(base, n_keys);

    // Q: second operand, column l16 of the products; channels in the order of K's fragments
    bf16x8 qf[kSteps];
    {
      const u16* const q = a.q + seq * a.q_token + (head * a.group + min(l16, a.group - 1)) * a.q_head;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const int ch = kE4m3 ? 16 * (4 * (st / 2) + g) + 8 * (st % 2) : 32 * st + 8 * g;
        qf[st] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(q + ch));
      }
    }
    if (!kDirect) find_blocks();
    f32x4 o[kTiles];
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    unsigned seen = 0;                             // bytes of keys that take part, or'ed (alone: block_bytes has all of them)

    struct Tile {
      unsigned long long at[2];          // its blocks in the pages
      unsigned bytes[2];                 // of them that take part
    };
    const int my_end = min(t1, (n_keys - kKeys * wave + kPagedTile - 1) / kPagedTile);      // tiles in which this wave has keys
    auto tile_at = [&](int t) __attribute__((always_inline)) -> Tile {
      if (!kDirect && t - base >= 32) {
        load_ids(t, n_keys);
        base = t;
        find_blocks();
      }
      Tile x;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int i = 2 * (t - base) + b;
        const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(block_at >> 32), i), lo = (unsigned)__builtin_amdgcn_readlane((int)block_at, i);
        x.at[b] = (unsigned long long)hi << 32 | lo;
        x.bytes[b] = (unsigned)__builtin_amdgcn_readlane((int)block_bytes, i);
      }
      return x;
    };
    auto issue_k = [&](const Tile& x) __attribute__((always_inline)) {
      const unsigned to = lds_at;
      if constexpr (kE4m3) {                      // four exponents a lane: of block lane / 4 % 2, K's and V's
        const unsigned long long at0 = x.at[0] / kRow, at1 = x.at[1] / kRow, row = lane & 4 ? at1 : at0;
        const uint8_t* const src = (lane & 8 ? a.pool.v_exp : a.pool.k_exp) + row + 4 * (lane & 3);
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dword %0, off" ::"v"(src), "s"(to + 2 * S::kStrip) : "m0", "memory");
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) load_rows(buffer_at(a.pool.k + x.at[b], x.bytes[b]), k_lane, to + b * 16 * kRow);
    };
    auto issue_v = [&](const Tile& x) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) load_rows(buffer_at(a.pool.v + x.at[b], x.bytes[b]), v_lane[b], lds_at + S::kStrip + b * 16 * kRow);
    };

    Tile next{{0ull, 0ull}, {0u, 0u}};
    if (t0 < my_end) {
      next = tile_at(t0);
      issue_k(next);
      issue_v(next);
#pragma unroll
      for (int st = 0; st < kSteps; ++st) asm volatile("" : "+v"(qf[st]));         // here, as block_at
    }
    for (int t = t0; t < my_end; ++t) {
      const Tile now = next;
      const bool more = t + 1 < my_end;
      if constexpr (!kDirect) seen |= now.bytes[0] | now.bytes[1];
      // ---- logits
      wait_all_but(VLoads{});
      f32x4 s[2];
      unsigned v_exp[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        s[b] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (!kE4m3) {
#pragma unroll
          for (int st = 0; st < kSteps; ++st) {
            const bf16x8 kf = *reinterpret_cast<const bf16x8*>(k_strip + b * 16 * kRow + k_off[st]);
            s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[st], s[b], 0, 0, 0);
          }
        } else {
          v_exp[b] = *reinterpret_cast<const unsigned*>(exps + 32 + 16 * b + 4 * g);
          const float by = __uint_as_float((unsigned)exps[16 * b + l16] << 23);       // of the key whose numbers this lane has
#pragma unroll
          for (int st = 0; st < kSteps; st += 2) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(k_strip + b * 16 * kRow + k_off[st]);
#pragma unroll
            for (int half = 0; half < 2; ++half)
              s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_of_e4m3(w[2 * half], w[2 * half + 1], by), qf[st + half], s[b], 0, 0, 0);
          }
        }
      }
      // K has been read; and a vector instruction may read a product 11 wait states after it, which the compiler does not see to in
      // another basic block
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_nop 7\n\ts_nop 3" : "+v"(s[0]), "+v"(s[1])::"memory");
      if (more) {
        next = tile_at(t + 1);
        issue_k(next);
      }
      // ---- weights
      if (now.bytes[0] + now.bytes[1] < kKeys * kRow) {         // no row: no weight, and no exponent
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool there = 4 * g + i % 4 < (int)(now.bytes[i / 4] / kRow);
          s[i / 4][i % 4] = there ? s[i / 4][i % 4] : -INFINITY;
          if constexpr (kE4m3) v_exp[i / 4] = there ? v_exp[i / 4] : v_exp[i / 4] & ~(0xFFu << (8 * (i % 4)));
        }
      }
      float top = max_of(max_of(s[0][0], s[0][1], s[0][2]), max_of(s[0][3], s[1][0], s[1][1]), max_of(s[1][2], s[1][3]));
      {
        float y = top;
        swap_lanes<16>(top, y);
        top = max_of(top, y);
        y = top;
        swap_lanes<32>(top, y);
        top = max_of(top, y);
      }
      if (__any(top > m)) {                       // a larger logit: what has been added up is brought onto it
        const float m_new = fmaxf(m, top);
        const float by = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * sl2);
        m = m_new;
        l *= by;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) o[dt] *= by;
      }
      const float minus = m == -INFINITY ? 0.f : -m * sl2;
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], sl2, minus));
        l += p[i];
        if constexpr (kE4m3) p[i] *= power_of(v_exp[i / 4], i % 4);
      }
      const u32x4 pw = {pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
      const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
      // ---- values
      if (more) wait_all_but(KLoads{});
      else wait_all_but(None{});
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) {
        bf16x8 vf;
        if constexpr (!kE4m3) vf = lds_read_vt16(v_strip + v_off[dt], 16 * kRow);
        else {
          const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3)))*)(v_strip + v_off[dt]));
          vf = eight_of_e4m3((unsigned)w[0], (unsigned)w[1], 1.f);
        }
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[dt], 0, 0, 0);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) issue_v(next);
    }

    // ---- the waves' results of the piece, joined
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(o[dt]));        // (as above)
    {
      float y = l;
      swap_lanes<16>(l, y);
      l += y;
      y = l;
      swap_lanes<32>(l, y);
      l += y;
      if (kDirect ? __any(block_bytes != 0) : seen != 0) m = fmaxf(m, kLowest);
    }
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) reinterpret_cast<f32x4*>(k_strip)[64 * dt + lane] = o[dt];
    if (lane < kHeads) {
      float* const stat = reinterpret_cast<float*>(k_strip + S::kStat);
      stat[lane] = m;
      stat[kHeads + lane] = l;
    }
    __syncthreads();
    const bool whole = kDirect || piece_is_whole(first, n_tiles, share);
    const size_t slot = kDirect ? 0 : (size_t)piece_slot(first, blockIdx.x, share) * a.group;
#pragma unroll
    for (int i = 0; i < (64 * kTiles + kThreads - 1) / kThreads; ++i) {
      const int item = kThreads * i + threadIdx.x, column = item % 16, ch = 16 * (item / 64) + 4 * (item / 16 % 4);
      if (column >= a.group || item >= 64 * kTiles) continue;
      float top = -INFINITY, f[kWaves], total = 0.f;
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, reinterpret_cast<const float*>(lds + w * S::kWaveBytes + S::kStat)[column]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float* const stat = reinterpret_cast<const float*>(lds + w * S::kWaveBytes + S::kStat);
        f[w] = __builtin_amdgcn_exp2f((stat[column] - (top == -INFINITY ? 0.f : top)) * sl2);
        total += f[w] * stat[kHeads + column];
        sum += f[w] * reinterpret_cast<const f32x4*>(lds + w * S::kWaveBytes)[item];
      }
      if (whole) {
        const float inv = inverse_of(total, top);
        const u32x2 y = {pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
        *reinterpret_cast<u32x2*>(a.out + ((size_t)seq * a.n_q_heads + head * a.group + column) * D + ch) = y;
      } else {
        *reinterpret_cast<f32x4*>(a.partial + (slot + column) * D + ch) = sum;
        if (ch == 0) {
          float* const stat = a.partial + (size_t)2 * a.workgroups * a.group * D + 2 * (slot + column);
          stat[0] = top == kLowest ? kLowest : top * sl2;
          stat[1] = total;
        }
      }
    }
    if constexpr (kDirect) return;
    __syncthreads();
    at = first + (unsigned)t1;
  }
}

// ---- the pieces of one sequence and query head, joined; a sequence without keys has zeros.  First their weights, then the weighted sum, whose
// loads do not wait for one another.
constexpr int kJoinWaves = 4, kJoinThreads = 64 * kJoinWaves;
struct Pieces {
  unsigned first, n_tiles, share, w0, n;       // first unit, units; the workgroups that have pieces are w0 .. w0 + n - 1; n = 1: whole
};
__device__ __forceinline__ Pieces pieces_of(const PagedDecodeArgs& a, int seq, int head, int lane) {
  int all = 0, earlier = 0;
  for (int s = lane; s < a.n_seqs; s += 64) {
    const int t = paged_tiles(length_of(a, s));
    all += t;
    earlier += s < seq ? t : 0;
  }
  Pieces p;
  const unsigned units = (unsigned)sum_of_wave(all) * (unsigned)a.pool.n_heads;
  p.n_tiles = (unsigned)paged_tiles(length_of(a, seq));
  p.share = (unsigned)__builtin_amdgcn_readfirstlane((int)paged_share(units, (unsigned)a.workgroups));
  p.first = (unsigned)sum_of_wave(earlier) * (unsigned)a.pool.n_heads + (unsigned)head * p.n_tiles;
  p.w0 = (unsigned)__builtin_amdgcn_readfirstlane((int)(p.first / p.share));
  p.n = p.n_tiles == 0 ? 0u : (unsigned)__builtin_amdgcn_readfirstlane((int)((p.first + p.n_tiles - 1) / p.share)) - p.w0 + 1;
  return p;
}

// Many sequences: a wave for each query head of one.  (96 sequences, 32/8 heads, d 128: 15.8 us with the kernel below, 4.9 this way.)
template <int D>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const PagedDecodeArgs a) {
  constexpr int kLanes = D / 4, kSlots = 64 / kLanes;
  const int lane = threadIdx.x & 63, seq = blockIdx.y, hq = kJoinWaves * blockIdx.x + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (hq >= a.n_q_heads) return;
  const int head = (int)quotient((unsigned)hq, a.by_group), column = hq - head * a.group;
  const Pieces p = pieces_of(a, seq, head, lane);
  u16* const out = a.out + ((size_t)seq * a.n_q_heads + hq) * D;
  if (p.n == 0 && lane < kLanes) reinterpret_cast<u32x2*>(out)[lane] = u32x2{0u, 0u};
  if (p.n <= 1) return;
  const float* const stats = a.partial + (size_t)2 * a.workgroups * a.group * D;
  auto slot_of = [&](unsigned i) __attribute__((always_inline)) { return (size_t)piece_slot(p.first, p.w0 + i, p.share) * a.group + column; };
  const int sub = lane / kLanes, piece = lane % kLanes;
  constexpr int kFirst = 4;
  f32x4 first[kFirst];                         // beside the maxima and sums, not after them
#pragma unroll
  for (int j = 0; j < kFirst; ++j) first[j] = *reinterpret_cast<const f32x4*>(a.partial + slot_of(min((unsigned)(sub + kSlots * j), p.n - 1)) * D + 4 * piece);
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (unsigned base = 0; base < p.n; base += 64) {
    const unsigned here = min(64u, p.n - base);
    const bool mine = (unsigned)lane < here;
    const float* const stat = stats + 2 * slot_of(base + (mine ? lane : 0));
    const float top = mine ? stat[0] : -INFINITY, sum = mine ? stat[1] : 0.f;
    const float most = fmaxf(m, over_wave(top, FloatMax{})), use = most == -INFINITY ? 0.f : most;
    const float by = __builtin_amdgcn_exp2f(m - use), f = __builtin_amdgcn_exp2f(top - use);
    m = most;
    l = l * by + over_wave(f * sum, FloatSum{});
    o *= by;
    auto add = [&](unsigned i, const f32x4& row) __attribute__((always_inline)) {      // (all lanes)
      const float w = __shfl(f, (int)i);
      if (i < here) o += w * row;
    };
    unsigned i = sub;
    if (base == 0) {
#pragma unroll
      for (int j = 0; j < kFirst; ++j) add(sub + kSlots * j, first[j]);
      i += kSlots * kFirst;
    }
#pragma unroll 4
    for (; i < (here + kSlots - 1) / kSlots * kSlots; i += kSlots) add(i, *reinterpret_cast<const f32x4*>(a.partial + slot_of(base + min(i, here - 1)) * D + 4 * piece));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x = o[e], y = x;
    if constexpr (kSlots == 4) {
      swap_lanes<16>(x, y);
      x += y;
      y = x;
    }
    swap_lanes<32>(x, y);
    o[e] = x + y;
  }
  const float inv = inverse_of(l, m);
  if (sub == 0) reinterpret_cast<u32x2*>(out)[piece] = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
}

// Few sequences, each in many pieces: four waves share the pieces of one query head, and a workgroup takes kJoinChannels of its channels.
// (131071 keys of 28/4 heads: 14.8 us with all channels to a workgroup and one loop of dependent loads, 4.8 with weights first, 4.0 this way.)
constexpr int kJoinChannels = 32;

template <int D>
__global__ void __launch_bounds__(kJoinThreads) paged_join_many_kernel(const PagedDecodeArgs a) {
  constexpr int kLanes = kJoinChannels / 4, kSlots = kJoinThreads / kLanes;       // lanes of a slot's channels; slots at a time
  __shared__ f32x4 rows[kSlots][kLanes];
  __shared__ float weights[kPagedMostWorkgroups], tops[kJoinWaves], sums[kJoinWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hq = blockIdx.x, seq = blockIdx.y;
  const int head = (int)quotient((unsigned)hq, a.by_group), column = hq - head * a.group;
  const Pieces p = pieces_of(a, seq, head, lane);
  u16* const out = a.out + ((size_t)seq * a.n_q_heads + hq) * D + kJoinChannels * blockIdx.z;
  if (p.n == 0 && tid < kLanes) reinterpret_cast<u32x2*>(out)[tid] = u32x2{0u, 0u};
  if (p.n <= 1) return;
  const unsigned n = p.n;
  const float* const stats = a.partial + (size_t)2 * a.workgroups * a.group * D;
  auto slot_of = [&](unsigned i) __attribute__((always_inline)) { return (size_t)piece_slot(p.first, p.w0 + i, p.share) * a.group + column; };
  // maxima, sums and the first rows in one trip to memory
  constexpr int kMine = kPagedMostWorkgroups / kJoinThreads, kRows = 8;
  f32x2 stat[kMine];
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const unsigned i = tid + kJoinThreads * j;
    stat[j] = i < n ? *reinterpret_cast<const f32x2*>(stats + 2 * slot_of(i)) : f32x2{-INFINITY, 0.f};
  }
  const int sub = tid / kLanes, piece = tid % kLanes;
  const float* const at = a.partial + kJoinChannels * blockIdx.z + 4 * piece;
  f32x4 first[kRows];
#pragma unroll
  for (int j = 0; j < kRows; ++j) first[j] = *reinterpret_cast<const f32x4*>(at + slot_of(min(sub + kSlots * j, (int)n - 1)) * D);
  float top = stat[0][0];
#pragma unroll
  for (int j = 1; j < kMine; ++j) top = fmaxf(top, stat[j][0]);
  top = over_wave(top, FloatMax{});
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = tops[0];
#pragma unroll
  for (int w = 1; w < kJoinWaves; ++w) top = fmaxf(top, tops[w]);
  const float use = top == -INFINITY ? 0.f : top;
  float total = 0.f;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const float f = __builtin_amdgcn_exp2f(stat[j][0] - use);
    total += f * stat[j][1];
    weights[tid + kJoinThreads * j] = f;                 // 0 where there is no piece
  }
  total = over_wave(total, FloatSum{});
  if (lane == 0) sums[wave] = total;
  __syncthreads();
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kRows; ++j)
    if (sub + kSlots * j < (int)n) o += weights[sub + kSlots * j] * first[j];
#pragma unroll 8
  for (unsigned i = sub + kSlots * kRows; i < n; i += kSlots) o += weights[i] * *reinterpret_cast<const f32x4*>(at + slot_of(i) * D);
  rows[sub][piece] = o;
  __syncthreads();
  if (tid >= kLanes) return;
  total = sums[0];
#pragma unroll
  for (int w = 1; w < kJoinWaves; ++w) total += sums[w];
  const int in_use = min((int)n, kSlots);
  f32x4 sum = rows[0][tid];
  for (int i = 1; i < in_use; ++i) sum += rows[i][tid];
  const float inv = inverse_of(total, top);
  reinterpret_cast<u32x2*>(out)[tid] = u32x2{pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
}

constexpr int kCus = 256;
static_assert(kCus * 2 <= kPagedMostWorkgroups, "room for the weights of pieces");
// A workgroup of its own for every sequence and KV head: where no sequence can have more keys than this, by the width of the table; more
// where there are so many that all CUs have one.  8 KV heads, d 128, e4m3, alone and in shares: one sequence of 512 keys 5.7 and 8.5 us, 1024 7.5
// and 8.7, 1280 8.7 and 8.8, 1536 9.7 and 8.9 (bf16 5.7 and 8.6, 7.7 and 8.8, 8.6 and 8.8, 9.5 and 8.8); 32 sequences of 512 7.1 and 12.2, of 1000 13.3 and
// 17.9, of 2500 27.1 and 31.5, of 4000 43.4 and 46.9; of 2500 once and 300 else 13.6 and 11.8, of 4000 once 19.4 and 12.3.
constexpr long long kAloneKeys = 1280, kAloneKeysOfMany = 2560;

template <int D, bool kE4m3>
hipError_t launch(const PagedDecodeArgs& a, hipStream_t s) {
  using S = Shape<D, kE4m3>;
  const unsigned pairs = (unsigned)a.n_seqs * (unsigned)a.pool.n_heads;
  if (a.most_keys <= (pairs >= kCus ? kAloneKeysOfMany : kAloneKeys)) {
    hipLaunchKernelGGL((paged_decode_kernel<D, kE4m3, kAlone>), dim3(pairs), dim3(kThreads), S::kLds, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((paged_decode_kernel<D, kE4m3, kShares>), dim3(a.workgroups), dim3(kThreads), S::kLds, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // the sequences' query heads fit the chip four waves each, or else a wave each
  if ((long long)a.n_q_heads * a.n_seqs * (D / kJoinChannels) <= 512)
    hipLaunchKernelGGL(paged_join_many_kernel<D>, dim3(a.n_q_heads, a.n_seqs, D / kJoinChannels), dim3(kJoinThreads), 0, s, a);
  else
    hipLaunchKernelGGL(paged_join_kernel<D>, dim3((a.n_q_heads + kJoinWaves - 1) / kJoinWaves, a.n_seqs), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

template <int D, bool kE4m3>
hipError_t prepare() {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(paged_decode_kernel<D, kE4m3, kAlone>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           Shape<D, kE4m3>::kLds);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute(reinterpret_cast<const void*>(paged_decode_kernel<D, kE4m3, kShares>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             Shape<D, kE4m3>::kLds);
}

}  // namespace

// as many as the chip holds at once
int paged_decode_workgroups(int head_dim, bool e4m3) {
  if (head_dim == 128) return kCus * (e4m3 ? Shape<128, true>::kPerCu : Shape<128, false>::kPerCu);
  return kCus * (e4m3 ? Shape<64, true>::kPerCu : Shape<64, false>::kPerCu);
}

hipError_t prepare_paged_decode() {
  hipError_t e;
  if ((e = prepare<128, false>()) != hipSuccess || (e = prepare<128, true>()) != hipSuccess) return e;
  if ((e = prepare<64, false>()) != hipSuccess) return e;
  return prepare<64, true>();
}

hipError_t launch_paged_decode(const PagedDecodeArgs& a, int head_dim, bool e4m3, hipStream_t s) {
  if (head_dim == 128) return e4m3 ? launch<128, true>(a, s) : launch<128, false>(a, s);
  return e4m3 ? launch<64, true>(a, s) : launch<64, false>(a, s);
}

}  // namespace kvp
