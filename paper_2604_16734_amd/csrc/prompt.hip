// Causal attention inside each of many prompts that lie one behind the other (kvp_prompt_attention), for gfx950: bf16 MFMA 32x32x16, K
// and V tiles through LDS.
//
// Bound by the matrix cores for long prompts (16640 rows of 32/8 heads, d 128, 1826 us, 1240 TFLOP/s; a large library product here 1365): 4 d flops for each pair of a row and a key that it sees, against 2 d numbers of K and V that serve
// the 128 rows of a workgroup and come out of the L2 cache of its die.
//
// Formulation.  A wave owns 32 query rows of one head and works on the transposed problem, S^T = K Q^T and O^T = V^T P^T: in the 32x32
// accumulator layout a lane then holds one query row, the softmax reference and sum are a number per lane, and the exponentiated
// accumulators are, register for register, the second operand of the second product.  Accumulator register r of lane (g = lane / 32) holds key
// 8 (r / 4) + 4 g + r % 4 of its 32; V is read out of LDS, transposed, in that order of keys.
//
// Many rows: a workgroup is four waves, 128 neighbouring rows of one head, and two of them share a CU (at d 64 three): what one waits for the other fills.
// Or it is two groups of four waves for the same rows, which take the tiles in turns.  (Few rows, and short prompts: below.)  Tiles of 64 keys come by
// buffer_load ... lds into two K and two V buffers of a group, row by row with the 16-byte chunks of a row swizzled by its number, so that all
// reads are free of bank conflicts.  The descriptors end with the last row that a row of the workgroup sees: what lies behind it comes as zeros and costs
// nothing.  Of tile t the wave takes the blocks of 32 keys X and Y; matrix and vector work overlap in program order:
//   phase 1   MFMA: S_Y(t), O += P_Y(t-1) V     | vector: P_X(t) = exp(S_X(t) - m)
//   barrier
//   phase 2   MFMA: S_X(t+1), O += P_X(t) V     | vector: P_Y(t) = exp(S_Y(t) - m), the loads of K(t+2) and V(t+1)
//
// Softmax reference.  exp(S - m) is exact for any m as long as nothing overflows: a row takes the maximum of the first 32 keys that it
// sees (two groups: each its own, and so is its sum) and O is never rescaled.  A row sum beyond 2^64 says that this did not do, and minus infinity is no reference; a result that is not finite may also
// come from a value that the row does not see, because 0 times infinity is no 0.  In these cases the wave takes its rows again the slow way, with a
// running maximum and values only where they are seen: 60 to 70 times slower where all rows have to (2048 rows of 32/8 heads, d 128: 42 us and 3.0 ms).
#include <type_traits>

#include "mfma_tools.h"
#include "serve.h"

namespace kvp {
namespace {

constexpr int kWaves = 4;              // of a workgroup, or of each half of one
static_assert(kPromptRows == 32 * kWaves, "rows of a workgroup");
constexpr int kTileKeys = 64;

// In LDS the 16-byte chunk ch of a row of K (or of Q, or of the result) lies at position ch ^ k_swizzle(row): sixteen rows, read in the same column, are
// then in all of the 64 banks.  (At d 64 two rows fill them.  With the row's number itself a third of all LDS cycles were conflicts, now 3 %; the time is the same, as LDS is not what it waits for.)
template <int D>
__device__ __forceinline__ int k_swizzle(int row) { return D == 64 ? row / 2 % 8 : row % 16; }

// KS: groups of four waves that share the keys of the same rows, tile by tile in turns
template <int D, int KS>
struct Shape {
  static constexpr int kThreads = 64 * kWaves * KS;
  static constexpr int kChunks = D / 8;                        // 16-byte chunks of a row
  static constexpr int kRowsPerLoad = 64 / kChunks;
  static constexpr int kLoads = kTileKeys / kWaves / kRowsPerLoad;      // of a wave, tensor and tile: 16 rows
  static constexpr int kTile = kTileKeys * D;                  // numbers
  static constexpr int kGroupLds = 5 * kTile * 2;              // two K, two V buffers, half of the query rows
  static constexpr int kLds = KS * kGroupLds;
  static constexpr int kPerSimd = D == 64 && KS == 1 ? 3 : 2;  // waves
  static_assert(kPromptRows * D == 2 * kTile && 2 * kGroupLds <= 160 * 1024, "two groups per CU");
  static_assert(kPromptRows * D * 4 + 2 * kPromptRows * 4 <= kGroupLds, "what a group leaves for the first one");
};

// Tile of kRows rows number `rank` of a list of all sequences' tiles, those that see most keys first, so that the workgroups that come last are the
// short ones: tile t of a sequence comes before all tiles t - 1.  With more than 64 sequences the list goes through the sequences instead, each
// one's last tile first: a look at all of them for every step of the search would take longer than it saves.
struct PromptTile {
  int begin, length, tile;            // the sequence's first row and its rows; length 0: no such tile
};
template <int kRows>
__device__ __forceinline__ PromptTile find_tile(const PromptArgs& a, int rank, int lane) {
  int before = 0;
  for (int base = 0; base < a.n_seqs; base += 64) {
    const int s = min(base + lane, a.n_seqs - 1);
    const int begin = min(max(a.seq_begin[s], 0), a.n_tokens), end = min(max(a.seq_begin[s + 1], begin), a.n_tokens);
    const int tiles = base + lane < a.n_seqs ? (end - begin + kRows - 1) / kRows : 0;
    const int upto = sum_upto(tiles);
    if (a.n_seqs <= 64) {
      if (__builtin_amdgcn_readlane(upto, 63) <= rank) break;
      if (a.n_seqs == 1) {
        const int all = __builtin_amdgcn_readlane(upto, 63);
        return PromptTile{__builtin_amdgcn_readlane(begin, 0), __builtin_amdgcn_readlane(end - begin, 0), all - 1 - rank};
      }
      // the t with  tiles from t + 1 on <= rank < tiles from t on
      int lo = 0, hi = __builtin_amdgcn_readfirstlane((int)over_wave((float)tiles, FloatMax{})), from_hi = 0;      // (below 2^24)
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2, n = sum_of_wave(max(tiles - mid, 0));
        if (n > rank) lo = mid;
        else hi = mid, from_hi = n;
      }
      // of the sequences that have a tile lo, the one before which so many come
      unsigned long long there = __ballot(tiles > lo);
      for (int skip = min(rank - from_hi, 63); skip > 0; --skip) there &= there - 1;        // (below 64 if the bounds do not descend)
      const int i = __builtin_ctzll(there);
      return PromptTile{__builtin_amdgcn_readlane(begin, i), __builtin_amdgcn_readlane(end - begin, i), lo};
    }
    const unsigned long long there = __ballot(before + upto > rank);
    if (there != 0) {
      const int i = __builtin_ctzll(there);
      return PromptTile{__builtin_amdgcn_readlane(begin, i), __builtin_amdgcn_readlane(end - begin, i),
                        before + __builtin_amdgcn_readlane(upto, i) - 1 - rank};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return PromptTile{0, 0, 0};
}

// Dies and KV heads are dealt out to each other: dies_per_set dies share the query heads of as few KV heads as that allows, whose K and V
// their L2 caches then hold, and take turns along the list of (tile, query head).
struct Item {
  int rank, head;
};
// Item number `mine` of this workgroup's die.
__device__ __forceinline__ Item item_of(const PromptArgs& a, unsigned mine) {
  const int xcd = blockIdx.x % kXcds, set = xcd / a.dies_per_set;
  const unsigned item = mine * (unsigned)a.dies_per_set + (unsigned)(xcd - set * a.dies_per_set);
  const int rank = (int)quotient(item, a.by_set_heads);
  return Item{rank, set * a.set_heads + (int)item - rank * a.set_heads};
}

// bytes up to the end of the last of `rows` rows, of `most` at most (no branches)
template <int D>
__device__ __forceinline__ unsigned bytes_of_rows(int rows, int most, unsigned row_bytes) {
  return (unsigned)max(min(max(rows, 0), most) * (int)row_bytes - (int)(row_bytes - 2u * D), 0);
}

// Query rows q0 .. q0 + 31 of a prompt of n the slow way, straight from memory: running maximum, and a value only where it is seen.  `qf`: the
// second operand of the products; the rows come out as the accumulators of O^T have them.
template <int D>
__device__ __forceinline__ void rows_the_slow_way(const bf16x8 (&qf)[D / 16], const u16* k_rows, long long k_token, const u16* v_rows, long long v_token, int q0,
                                                  int n, float sl2, int l32, int g, f32x16 (&o)[D / 32], float& l_row) {
  constexpr int kNK = D / 16, kND = D / 32;
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY;
  l_row = 0.f;
#pragma unroll
  for (int dt = 0; dt < kND; ++dt) o[dt] = zero;
  for (int kb = 0; kb < min(n, q0 + 32); kb += 32) {
    f32x16 s = zero;
    const u16* const kr = k_rows + (long long)min(kb + l32, n - 1) * k_token + 8 * g;
#pragma unroll
    for (int st = 0; st < kNK; ++st)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(kr + 16 * st)), qf[st], s, 0, 0, 0);
    const int lim = q0 + l32 - kb - 4 * g;
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = (8 * (r >> 2) + (r & 3) <= lim) ? s[r] : -INFINITY;
      mx = fmaxf(mx, s[r]);
    }
    const float m_new = fmaxf(m_run, max_with_other_half(mx)), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run - m_use) * sl2), neg = -m_use * sl2;
    m_run = m_new;
    l_row *= alpha;
#pragma unroll
    for (int dt = 0; dt < kND; ++dt) o[dt] *= alpha;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sl2, neg));
      sum += s[r];
    }
    l_row += sum_with_other_half(sum);
    // key by key; key 8 (r / 4) + 4 half + r % 4 is in register r of the lanes of that half
#pragma unroll 1
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = kb + 8 * (r >> 2) + 4 * half + (r & 3);
        const float mine = s[r], others = __shfl_xor(mine, 32), p = g == half ? mine : others;
        const u16* const vr = v_rows + (long long)min(key, n - 1) * v_token + 4 * g;
        const bool seen = key <= q0 + l32;
#pragma unroll
        for (int dt = 0; dt < kND; ++dt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(vr + 32 * dt + 8 * j);
            const float v[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
            for (int e = 0; e < 4; ++e) o[dt][4 * j + e] = seen ? __builtin_fmaf(p, v[e], o[dt][4 * j + e]) : o[dt][4 * j + e];
          }
      }
  }
}

// rows of a wave to memory, through 32 of its rows of LDS so that the stores are whole rows
template <int D>
__device__ __forceinline__ void store_rows(const f32x16 (&o)[D / 32], float inv, u32x4* rows, u16* to, long long to_token, int n_rows, int lane) {
  constexpr int kChunks = D / 8;
  const int l32 = lane & 31, g = lane >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; j += 2) {        // fours j of a channel tile are its channels 8 j + 4 g .. + 3: the halves of the wave exchange one of two
      const f32x16& x = o[dt];
      const auto lo = __builtin_amdgcn_permlane32_swap(pack_bf16(x[4 * j] * inv, x[4 * j + 1] * inv), pack_bf16(x[4 * j + 4] * inv, x[4 * j + 5] * inv), false, false);
      const auto hi = __builtin_amdgcn_permlane32_swap(pack_bf16(x[4 * j + 2] * inv, x[4 * j + 3] * inv), pack_bf16(x[4 * j + 6] * inv, x[4 * j + 7] * inv), false, false);
      rows[l32 * kChunks + ((4 * dt + j + g) ^ k_swizzle<D>(l32))] = u32x4{lo[0], hi[0], lo[1], hi[1]};
    }
#pragma unroll
  for (int it = 0; it < kChunks / 2; ++it) {
    const int r = (64 * it + lane) / kChunks, ch = lane % kChunks;
    const u32x4 val = rows[r * kChunks + (ch ^ k_swizzle<D>(r))];
    if (r < n_rows) *reinterpret_cast<u32x4*>(to + (long long)r * to_token + 8 * ch) = val;
  }
}

template <int D, int KS>
__global__ void __launch_bounds__((Shape<D, KS>::kThreads), (Shape<D, KS>::kPerSimd)) prompt_kernel(const PromptArgs a) {
  using S = Shape<D, KS>;
  constexpr int kNK = D / 16, kNV = (D / 32) * 2, kND = D / 32;       // K and V fragments of a block of 32 keys; channel tiles
  extern __shared__ __align__(16) unsigned char lds_raw[];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int all_waves = __builtin_amdgcn_readfirstlane(tid >> 6), wave = all_waves % kWaves, ks = KS == 1 ? 0 : all_waves / kWaves;
  u16* const lds_k = reinterpret_cast<u16*>(lds_raw + ks * S::kGroupLds);      // [2][kTile]
  u16* const lds_v = lds_k + 2 * S::kTile;                                     // [2][kTile]

  const Item item = item_of(a, blockIdx.x / kXcds);
  const int rank = item.rank, h = item.head;
  const PromptTile pt = find_tile<kPromptRows>(a, rank, lane);
  const int n = pt.length, wg_row = pt.tile * kPromptRows;
  if (wg_row >= n) return;
  const int hk = (int)quotient((unsigned)h, a.by_group);
  const u16* const q_rows = a.q + pt.begin * a.q_token + h * a.q_head;
  const u16* const k_rows = a.k + pt.begin * a.k_token + hk * a.k_head;
  const u16* const v_rows = a.v + pt.begin * a.v_token + hk * a.v_head;
  u16* const out_rows = a.out + pt.begin * a.out_token + h * a.out_head;
  const int q0 = wg_row + 32 * wave;                    // this wave's first row; it may lie past the end
  const int rows_end = min(n, wg_row + kPromptRows);
  // tiles of a group: ks, ks + KS, ..
  auto of_group = [&](int tiles, int which) __attribute__((always_inline)) { return (tiles - which + KS - 1) / KS; };
  const int n_tiles = of_group((rows_end + kTileKeys - 1) / kTileKeys, 0);                 // steps of the workgroup
  const int seen = q0 < n ? (min(n, q0 + 32) + kTileKeys - 1) / kTileKeys : 0;
  const int my_tiles = of_group(seen, ks);                                                // that this wave sees
  const int n_plain = of_group(min(seen, (q0 + 1) / kTileKeys), ks);                      // that all of its rows see whole
  const float sl2 = a.scale_log2;

  // ---- staging.  Wave w brings in rows 16 w .. 16 w + 15 of a tile; load j's immediate offset moves both of its addresses by 1 KiB, and the lane's part
  // takes that back where rows lie further apart.  (Inline assembly, and waits of this kernel's own: the compiler would have every read of
  // LDS wait for all loads.  s_nop: a load may read a scalar register five wait states after a vector instruction has written it.)
  const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) void*)lds_raw) + (unsigned)(ks * S::kGroupLds);
  auto lds_dst = [&](const u16* tile) __attribute__((always_inline)) -> unsigned {
    return lds_at + 2u * (unsigned)((int)(tile - lds_k) + 16 * wave * D);
  };
  const int ld_sub = lane / S::kChunks, ld_pos = lane % S::kChunks;
  unsigned k_lane[S::kLoads], v_lane[S::kLoads];
#pragma unroll
  for (int j = 0; j < S::kLoads; ++j) {
    const int row = 16 * wave + S::kRowsPerLoad * j + ld_sub;
    k_lane[j] = (unsigned)row * a.k_bytes + 16u * (unsigned)(ld_pos ^ k_swizzle<D>(row)) - 1024u * j;
    v_lane[j] = (unsigned)row * a.v_bytes + 16u * (unsigned)(ld_pos ^ v_swizzle<D>(row)) - 1024u * j;
  }
  struct Feed {
    unsigned long long at;
    unsigned bytes, row_bytes;
    int rows;                          // from this tile's first one on
  };
  auto bytes_of = [&](int rows, unsigned row_bytes) __attribute__((always_inline)) -> unsigned { return bytes_of_rows<D>(rows, kTileKeys, row_bytes); };
  auto feed_at = [&](const u16* first, unsigned row_bytes, int rows) __attribute__((always_inline)) -> Feed {
    return Feed{(unsigned long long)first, bytes_of(rows, row_bytes), row_bytes, rows};
  };
  auto load_fed = [&](const Feed& f, const unsigned (&of)[S::kLoads], auto which, unsigned to) __attribute__((always_inline)) {
    constexpr int j = decltype(which)::value;
    const u32x4 buffer = {(unsigned)f.at, (unsigned)(f.at >> 32) & 0xFFFFu, f.bytes, 0x00020000u};
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen offset:%3 lds" ::"v"(of[j]), "s"(buffer), "s"(to), "n"(1024 * j)
                 : "m0", "memory");
  };
  auto move_on = [&](Feed& f) __attribute__((always_inline)) {
    f.at += (unsigned long long)(KS * kTileKeys) * f.row_bytes;
    f.rows -= KS * kTileKeys;
    f.bytes = bytes_of(f.rows, f.row_bytes);
  };
  auto load_tile = [&](const Feed& f, const unsigned (&of)[S::kLoads], unsigned to) __attribute__((always_inline)) {
    load_fed(f, of, std::integral_constant<int, 0>{}, to);
    load_fed(f, of, std::integral_constant<int, 1>{}, to);
    if constexpr (S::kLoads == 4) {
      load_fed(f, of, std::integral_constant<int, 2>{}, to);
      load_fed(f, of, std::integral_constant<int, 3>{}, to);
    }
  };
  auto wait_all_but = [&](auto newest) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70 | decltype(newest)::value);
    asm volatile("" ::: "memory");
  };
  typedef std::integral_constant<int, 0> None;

  // ---- where the fragments are (in numbers)
  int k_off[kNK], v_off[kND];
#pragma unroll
  for (int st = 0; st < kNK; ++st) k_off[st] = l32 * D + 8 * ((2 * st) ^ (g ^ k_swizzle<D>(l32)));
  {
    const int rsub = 4 * g + ((lane & 15) >> 2), z = v_swizzle<D>(rsub);
#pragma unroll
    for (int dt = 0; dt < kND; ++dt) v_off[dt] = rsub * D + 8 * ((4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ z) + 4 * (lane & 1);
  }

  // ---- the wave's query rows, through the V buffer that is filled last and one like it; beside them the first tiles: one trip to memory for all
  u16* const q_strip = lds_v + S::kTile + wave * 32 * D;
  {
    const int rows = min(32, n - q0);
    const u16* const at = q_rows + (long long)q0 * a.q_token;
    const unsigned long long base = (unsigned long long)at;
    const u32x4 buffer = {(unsigned)base, (unsigned)(base >> 32) & 0xFFFFu, rows > 0 ? (unsigned)(rows - 1) * a.q_bytes + 2u * D : 0u, 0x00020000u};
    const unsigned to = lds_at + 2u * (unsigned)(q_strip - lds_k);
#pragma unroll
    for (int j = 0; j < 2 * S::kLoads; ++j) {
      const int row = S::kRowsPerLoad * j + ld_sub;
      const unsigned of = (unsigned)row * a.q_bytes + 16u * (unsigned)(ld_pos ^ k_swizzle<D>(row));
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(of), "s"(buffer), "s"(to + 1024u * j) : "m0", "memory");
    }
  }
  const int key0 = kTileKeys * ks;
  Feed k_feed = feed_at(k_rows + (long long)key0 * a.k_token, a.k_bytes, rows_end - key0);
  Feed v_feed = feed_at(v_rows + (long long)key0 * a.v_token, a.v_bytes, rows_end - key0);
  load_tile(k_feed, k_lane, lds_dst(lds_k));
  load_tile(v_feed, v_lane, lds_dst(lds_v));
  move_on(k_feed);
  move_on(v_feed);
  load_tile(k_feed, k_lane, lds_dst(lds_k + S::kTile));
  move_on(k_feed);

  bf16x8 qf[kNK];                        // second operand: Q[q0 + l32][16 s + 8 g .. + 7]
  f32x16 o[kND], sx, sy;
  unsigned px[8], py[8];
  float m_ref = -INFINITY, l_run = 0.f;
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int dt = 0; dt < kND; ++dt) o[dt] = zero;
#pragma unroll
  for (int r = 0; r < 8; ++r) px[r] = py[r] = 0u;
  wait_all_but(std::integral_constant<int, 2 * S::kLoads>{});          // V(0) and K(1) may still be on their way
#pragma unroll
  for (int st = 0; st < kNK; ++st) qf[st] = lds_read_b128(q_strip + k_off[st]);
#pragma unroll
  for (int st = 0; st < kNK; ++st) asm volatile("" : "+v"(qf[st]));    // read, before the strip is filled again
  __syncthreads();
  sx = zero;
#pragma unroll
  for (int st = 0; st < kNK; ++st) sx = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read_b128(lds_k + k_off[st]), qf[st], sx, 0, 0, 0);
  // (a vector instruction may read a product 12 wait states after it, which the compiler does not see to in another basic block)
  asm volatile("s_nop 7\n\ts_nop 7" : "+v"(sx));

  // Hides keys that a row does not see; the first block's maximum becomes the row's reference.
  auto prepare = [&](f32x16& s, int kb, auto mask, auto reference) __attribute__((always_inline)) {
    if constexpr (decltype(mask)::value) {
      const int lim = q0 + l32 - kb - 4 * g;       // key kb + 8 (r / 4) + 4 g + r % 4
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (8 * (r >> 2) + (r & 3) <= lim) ? s[r] : -INFINITY;
    }
    if constexpr (decltype(reference)::value) {
      float v = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) v = fmaxf(v, s[r]);
      m_ref = max_with_other_half(v);
    }
  };

  // One phase, one basic block: every MFMA is followed by its share of the exponentials of the block computed in the phase before, and LDS
  // reads run kAhead fragments ahead.  Written in the order in which it should issue, with a scheduling fence after every share.  The
  // work on an element is a chain (scale and shift, exponential, sum, pack), which is skewed over the MFMAs so that no instruction needs the result of the one
  // before it.
  //   s_exp -> p_out   P = exp2((S - m) * scale);   s_new = S^T of the next block;   O += P_pend V (kValues)
  constexpr int kAhead = D / 32;
  bf16x8 first[kAhead];                            // the first K fragments of a phase 1, read at the end of the phase before it
  auto phase = [&](const f32x16& s_exp, unsigned (&p_out)[8], f32x16& s_new, const u16* kt, const unsigned (&p_pend)[8], const u16* vt, auto have,
                   auto values, auto next, const u16* next_kt, auto&& after_mfma) __attribute__((always_inline)) {
    constexpr bool kHave = decltype(have)::value, kValues = decltype(values)::value, kNext = decltype(next)::value;
    constexpr int kMfmas = kNK + (kValues ? kNV : 0);
    const float neg = m_ref == -INFINITY ? 0.f : -m_ref * sl2;
    float sum = 0.f;
    bf16x8 kfr[kNK], vfr[kNV];
    auto read_v = [&](int vi) __attribute__((always_inline)) { vfr[vi] = lds_read_vt(vt + v_off[vi / 2] + 16 * (vi % 2) * D, 8 * D); };
    int ei = 0;
    float arg = __builtin_fmaf(s_exp[0], sl2, neg), pe1 = 0.f, pe2 = 0.f;
    // (sums of the packed weights, two to an instruction by v_dot2_f32_bf16: 6 % slower)
    auto finish_element = [&](int e) __attribute__((always_inline)) {
      sum += pe1;
      asm volatile("" : "+v"(sum));          // (left alone the compiler gathers the additions of several phases in one place)
      if (e & 1) p_out[e >> 1] = pack_bf16(pe2, pe1);
    };
    auto share = [&](int i) __attribute__((always_inline)) {
#pragma unroll
      for (; ei < 16 * (i + 1) / kMfmas; ++ei) {
        const float pe = __builtin_amdgcn_exp2f(arg);
        if (ei + 1 < 16) arg = __builtin_fmaf(s_exp[ei + 1], sl2, neg);
        if (ei >= 1) finish_element(ei - 1);
        pe2 = pe1;
        pe1 = pe;
      }
    };
#pragma unroll
    for (int st = 0; st < kAhead; ++st) {
      if constexpr (kHave) kfr[st] = first[st];
      else kfr[st] = lds_read_b128(kt + k_off[st]);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int st = 0; st < kNK; ++st) {
      if (st + kAhead < kNK) kfr[st + kAhead] = lds_read_b128(kt + k_off[st + kAhead]);
      else if constexpr (kValues) read_v(st + kAhead - kNK);
      s_new = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kfr[st], qf[st], st == 0 ? zero : s_new, 0, 0, 0);
      share(st);
      after_mfma(std::integral_constant<int, 0>{}, st);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (kValues) {
#pragma unroll
      for (int vi = 0; vi < kNV; ++vi) {
        if (vi + kAhead < kNV) read_v(vi + kAhead);
        else if constexpr (kNext) first[vi + kAhead - kNV] = lds_read_b128(next_kt + k_off[vi + kAhead - kNV]);
        const int mm = vi % 2;
        const u32x4 pw = {p_pend[4 * mm], p_pend[4 * mm + 1], p_pend[4 * mm + 2], p_pend[4 * mm + 3]};
        o[vi / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vfr[vi], __builtin_bit_cast(bf16x8, pw), o[vi / 2], 0, 0, 0);
        share(kNK + vi);
        after_mfma(std::integral_constant<int, 1>{}, vi);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    finish_element(15);
    l_run += sum;
  };

  typedef std::true_type Yes;
  typedef std::false_type No;
  // kTag: t & 1 where the compiler knows it, else -1.  kStart: tile 0, which has no values to add yet and gives the rows their reference.
  auto body = [&](int t, auto buf_tag, auto start, auto mask) __attribute__((always_inline)) {
    constexpr int kTag = decltype(buf_tag)::value;
    constexpr bool kStart = decltype(start)::value;
    const int buf = kTag >= 0 ? kTag : (t & 1);
    u16* const k_cur = lds_k + buf * S::kTile;
    u16* const k_nxt = lds_k + (buf ^ 1) * S::kTile;
    u16* const v_cur = lds_v + buf * S::kTile;
    u16* const v_prv = lds_v + (buf ^ 1) * S::kTile;
    const int kb = (KS * t + ks) * kTileKeys;
    prepare(sx, kb, mask, start);
    phase(sx, px, sy, k_cur + 32 * D, py, v_prv + 32 * D, std::integral_constant<bool, !kStart>{}, std::integral_constant<bool, !kStart>{}, No{}, nullptr,
          [](auto, int) {});
    // P_X is due here, in the shadow of this phase's products
#pragma unroll
    for (int r = 0; r < 8; ++r) asm volatile("" ::"v"(px[r]));
    __builtin_amdgcn_sched_barrier(0);
    wait_all_but(None{});              // the loads that this wave issued in the last phase 2 have landed
    __syncthreads();
    prepare(sy, kb + 32, mask, No{});
    constexpr int kEvery = kNK / S::kLoads;
    const unsigned k_to = lds_dst(k_cur), v_to = lds_dst(v_prv);
    phase(sy, py, sx, k_nxt, px, v_cur, No{}, Yes{}, Yes{}, k_nxt + 32 * D, [&](auto half, int i) __attribute__((always_inline)) {
      if (i % kEvery != 0) return;
      auto load = [&](auto which) __attribute__((always_inline)) {
        if constexpr (decltype(half)::value == 0) load_fed(k_feed, k_lane, which, k_to);
        else load_fed(v_feed, v_lane, which, v_to);
      };
      switch (i / kEvery) {
        case 0: load(std::integral_constant<int, 0>{}); break;
        case 1: load(std::integral_constant<int, 1>{}); break;
        case 2: if constexpr (S::kLoads == 4) load(std::integral_constant<int, 2>{}); break;
        default: if constexpr (S::kLoads == 4) load(std::integral_constant<int, 3>{}); break;
      }
    });
    move_on(k_feed);
    move_on(v_feed);
  };
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  typedef std::integral_constant<int, -1> Any;
  int t = 0;
  if (my_tiles > 0) {
    if (n_plain > 0) body(0, Even{}, Yes{}, No{});
    else body(0, Even{}, Yes{}, Yes{});
    for (t = 1; t + 1 < n_plain; t += 2) {
      body(t, Odd{}, No{}, No{});
      body(t + 1, Even{}, No{}, No{});
    }
    // the last tile of them all has the diagonal: in its first block, and then nobody sees the second one, or in the second
    const bool half = KS * (my_tiles - 1) + ks == seen - 1 && q0 % kTileKeys == 0 && t < my_tiles;
    for (; t < my_tiles - half; ++t) body(t, Any{}, No{}, Yes{});       // (a mask does nothing to a tile that is seen whole)
    auto add_values = [&](const unsigned (&p)[8], const u16* vt) __attribute__((always_inline)) {
#pragma unroll
      for (int vi = 0; vi < kNV; ++vi) {
        const u32x4 pw = {p[4 * (vi % 2)], p[4 * (vi % 2) + 1], p[4 * (vi % 2) + 2], p[4 * (vi % 2) + 3]};
        o[vi / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read_vt(vt + v_off[vi / 2] + 16 * (vi % 2) * D, 8 * D), __builtin_bit_cast(bf16x8, pw), o[vi / 2], 0, 0, 0);
      }
    };
    // O += P_Y V of the last tile: its V is there since the barrier inside the last body, until the next one
    add_values(py, lds_v + ((t & 1) ^ 1) * S::kTile + 32 * D);
    if (half) {
      prepare(sx, (KS * t + ks) * kTileKeys, Yes{}, No{});
      const float neg = m_ref == -INFINITY ? 0.f : -m_ref * sl2;
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sx[r], sl2, neg)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sx[r + 1], sl2, neg));
        l_run += p0 + p1;
        px[r / 2] = pack_bf16(p0, p1);
      }
      wait_all_but(None{});
      __syncthreads();
      load_tile(k_feed, k_lane, lds_dst(lds_k + (t & 1) * S::kTile));
      load_tile(v_feed, v_lane, lds_dst(lds_v + ((t & 1) ^ 1) * S::kTile));
      move_on(k_feed);
      move_on(v_feed);
      add_values(px, lds_v + (t & 1) * S::kTile);
      ++t;
    }
  }
  // tiles that only later rows of the workgroup see: in step with their waves
  for (; t < n_tiles; ++t) {
    wait_all_but(None{});
    __syncthreads();
    load_tile(k_feed, k_lane, lds_dst(lds_k + (t & 1) * S::kTile));
    load_tile(v_feed, v_lane, lds_dst(lds_v + ((t & 1) ^ 1) * S::kTile));
    move_on(k_feed);
    move_on(v_feed);
  }
  wait_all_but(None{});
  __syncthreads();               // nothing is on its way into LDS, and nobody reads a tile any more
  if constexpr (kND == 4) asm volatile("s_nop 7\n\ts_nop 7" : "+v"(o[0]), "+v"(o[1]), "+v"(o[2]), "+v"(o[3]));       // (as after the first products)
  else asm volatile("s_nop 7\n\ts_nop 7" : "+v"(o[0]), "+v"(o[1]));
  float l_row = sum_with_other_half(l_run);
  if (m_ref == -INFINITY && q0 + l32 >= kTileKeys * ks) l_row = NAN;           // keys, but no reference
  if constexpr (KS == 2) {
    // the second group leaves its rows as they lie in the accumulators, and the first one adds them up
    float* const stat = reinterpret_cast<float*>(lds_raw + S::kGroupLds + kPromptRows * D * 4) + 64 * wave;       // [row, or 32 + row]
    f32x4* const left = reinterpret_cast<f32x4*>(lds_raw + S::kGroupLds) + wave * 32 * D / 4 + lane;
    auto four = [&](int k) __attribute__((always_inline)) -> f32x4 { return f32x4{o[k / 4][4 * (k % 4)], o[k / 4][4 * (k % 4) + 1], o[k / 4][4 * (k % 4) + 2], o[k / 4][4 * (k % 4) + 3]}; };
    if (ks == 1) {
#pragma unroll
      for (int k = 0; k < 4 * kND; ++k) left[64 * k] = four(k);
      if (g == 0) {
        stat[l32] = m_ref;
        stat[32 + l32] = l_row;
      }
    }
    __syncthreads();
    if (ks == 1) return;
    const float m_other = stat[l32], l_other = stat[32 + l32], top = fmaxf(m_ref, m_other), use = top == -INFINITY ? 0.f : top;
    const float f0 = __builtin_amdgcn_exp2f((m_ref - use) * sl2), f1 = __builtin_amdgcn_exp2f((m_other - use) * sl2);
    // (each sum by itself: the factor of a reference far below the other one is 0, which leaves out 2^64 2^-126 at most, not what is above)
    const bool of_use = l_row <= 0x1p64f && l_other <= 0x1p64f;
    l_row = of_use ? l_row * f0 + l_other * f1 : NAN;
#pragma unroll
    for (int k = 0; k < 4 * kND; ++k) {
      const f32x4 x = left[64 * k];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[k / 4][4 * (k % 4) + e] = o[k / 4][4 * (k % 4) + e] * f0 + x[e] * f1;
    }
  }
  if (q0 >= n) return;
  // what is not finite is not 0 when it is multiplied by 0
  float check[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int dt = 0; dt < kND; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) check[r % 8] = __builtin_fmaf(o[dt][r], 0.f, check[r % 8]);
  check[0] += check[1] + check[2] + check[3];
  check[4] += check[5] + check[6] + check[7];
  if (__any(!(l_row <= 0x1p64f) || !(check[0] + check[4] == 0.f))) {
    rows_the_slow_way<D>(qf, k_rows, a.k_token, v_rows, a.v_token, q0, n, sl2, l32, g, o, l_row);
  }

  store_rows<D>(o, 1.f / l_row, reinterpret_cast<u32x4*>(lds_raw) + wave * 32 * S::kChunks, out_rows + (long long)q0 * a.out_token, a.out_token, n - q0, lane);
}

// ---- Few rows: workgroups of 128 would leave most of the chip idle and each have a long way to go.  Here one has 32 rows of one head, and its eight waves
// share the keys, every eighth block of 32 each, as they come through two strips of LDS of the wave's own: no barrier between the query rows and
// the end, where the waves' results are added up.  Bound by latency: the loads, a block or a few, and the sum over the waves.
// Short prompts: the same with each of four waves at 32 rows of its own, for which it goes through all keys by itself.
template <int D, bool kShared>
struct FewShape {
  static constexpr int kWaves = kShared ? 8 : 4, kThreads = 64 * kWaves, kRows = 32;
  static constexpr int kItems = kShared ? 1 : kWaves;          // tiles of a workgroup
  static constexpr int kChunks = D / 8, kRowsPerLoad = 64 / kChunks;
  static constexpr int kLoads = 16 / kRowsPerLoad;             // for 16 rows
  static constexpr int kStrip = 32 * D;                        // numbers: 32 keys
  static constexpr int kWaveBytes = 2 * kStrip * 2;            // K, V; then what the wave leaves of its rows, as it is in the accumulators
  static constexpr int kQ = kWaves * kWaveBytes, kStat = kQ + kRows * D * 2;      // (shared)
  static constexpr int kLds = kShared ? kStat + kWaves * 2 * kRows * 4 : kQ;
  static constexpr unsigned kPerCu = kLds > 80 * 1024 ? 1 : 2;
  static_assert(kRows * D * 4 <= kWaveBytes && kLds <= 160 * 1024, "LDS of a CU");
};

template <int D, bool kShared>
__global__ void __launch_bounds__((FewShape<D, kShared>::kThreads), 2) prompt_few_kernel(const PromptArgs a) {
  using S = FewShape<D, kShared>;
  constexpr int kNK = D / 16, kNV = (D / 32) * 2, kND = D / 32;
  extern __shared__ __align__(16) unsigned char lds_raw[];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Item item = item_of(a, blockIdx.x / kXcds * S::kItems + (kShared ? 0 : wave));
  const PromptTile pt = find_tile<S::kRows>(a, item.rank, lane);
  const int n = pt.length, q0 = pt.tile * S::kRows, h = item.head;
  if (q0 >= n) return;
  const int hk = (int)quotient((unsigned)h, a.by_group);
  const u16* const q_rows = a.q + pt.begin * a.q_token + h * a.q_head;
  const u16* const k_rows = a.k + pt.begin * a.k_token + hk * a.k_head;
  const u16* const v_rows = a.v + pt.begin * a.v_token + hk * a.v_head;
  u16* const out_rows = a.out + pt.begin * a.out_token + h * a.out_head;
  const int rows_end = min(n, q0 + S::kRows), n_blocks = q0 / 32 + 1;         // blocks of keys; the last one has the diagonal
  const float sl2 = a.scale_log2;

  u16* const k_strip = reinterpret_cast<u16*>(lds_raw + wave * S::kWaveBytes);
  u16* const v_strip = k_strip + S::kStrip;
  u16* const q_lds = reinterpret_cast<u16*>(lds_raw + S::kQ);
  float* const stats = reinterpret_cast<float*>(lds_raw + S::kStat);          // [wave][maxima, sums][row]
  const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) void*)lds_raw);
  const unsigned my_lds = lds_at + (unsigned)(wave * S::kWaveBytes);

  // ---- global -> LDS, 16 rows at a time, through descriptors that end with the last row that is seen (as above; also why inline assembly)
  const int ld_sub = lane / S::kChunks, ld_pos = lane % S::kChunks;
  unsigned k_lane[S::kLoads], v_lane[S::kLoads];
#pragma unroll
  for (int j = 0; j < S::kLoads; ++j) {
    const int row = S::kRowsPerLoad * j + ld_sub;
    k_lane[j] = (unsigned)row * a.k_bytes + 16u * (unsigned)(ld_pos ^ k_swizzle<D>(row)) - 1024u * j;
    v_lane[j] = (unsigned)row * a.v_bytes + 16u * (unsigned)(ld_pos ^ v_swizzle<D>(row)) - 1024u * j;
  }
  auto load16 = [&](const u16* first, int rows, unsigned row_bytes, const unsigned (&of)[S::kLoads], unsigned to) __attribute__((always_inline)) {
    const unsigned long long at = (unsigned long long)first;
    // (through the first lane: the compiler would carry some of it in vector registers)
    const u32x4 buffer = {(unsigned)__builtin_amdgcn_readfirstlane((int)at), (unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32)) & 0xFFFFu,
                          (unsigned)__builtin_amdgcn_readfirstlane((int)bytes_of_rows<D>(rows, 16, row_bytes)), 0x00020000u};
    if constexpr (S::kLoads == 4)
      asm volatile("s_mov_b32 m0, %5\n\ts_nop 3\n\t"
                   "buffer_load_dwordx4 %0, %4, 0 offen lds\n\t"
                   "buffer_load_dwordx4 %1, %4, 0 offen offset:1024 lds\n\t"
                   "buffer_load_dwordx4 %2, %4, 0 offen offset:2048 lds\n\t"
                   "buffer_load_dwordx4 %3, %4, 0 offen offset:3072 lds" ::"v"(of[0]), "v"(of[1]), "v"(of[2]), "v"(of[3]), "s"(buffer), "s"(to)
                   : "m0", "memory");
    else
      asm volatile("s_mov_b32 m0, %3\n\ts_nop 3\n\t"
                   "buffer_load_dwordx4 %0, %2, 0 offen lds\n\t"
                   "buffer_load_dwordx4 %1, %2, 0 offen offset:1024 lds" ::"v"(of[0]), "v"(of[1]), "s"(buffer), "s"(to)
                   : "m0", "memory");
  };
  auto issue_k = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      load16(k_rows + (long long)(32 * b + 16 * i) * a.k_token, rows_end - 32 * b - 16 * i, a.k_bytes, k_lane, my_lds + 2u * (unsigned)(16 * i * D));
  };
  auto issue_v = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      load16(v_rows + (long long)(32 * b + 16 * i) * a.v_token, rows_end - 32 * b - 16 * i, a.v_bytes, v_lane, my_lds + 2u * (unsigned)(S::kStrip + 16 * i * D));
  };
  auto wait_all_but = [&](auto newest) __attribute__((always_inline)) {
    constexpr int k = decltype(newest)::value;
    __builtin_amdgcn_s_waitcnt(0x0F70 | (k & 15) | (k >> 4 << 14));
    asm volatile("" ::: "memory");
  };
  typedef std::integral_constant<int, 2 * S::kLoads> OneStrip;
  typedef std::integral_constant<int, 4 * S::kLoads> BothStrips;
  typedef std::integral_constant<int, 0> None;

  int k_off[kNK], v_off[kND];
#pragma unroll
  for (int st = 0; st < kNK; ++st) k_off[st] = l32 * D + 8 * ((2 * st) ^ (g ^ k_swizzle<D>(l32)));
  {
    const int rsub = 4 * g + ((lane & 15) >> 2), z = v_swizzle<D>(rsub);
#pragma unroll
    for (int dt = 0; dt < kND; ++dt) v_off[dt] = rsub * D + 8 * ((4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ z) + 4 * (lane & 1);
  }
  bf16x8 qf[kNK];
  auto load_q = [&](int row0, unsigned to) __attribute__((always_inline)) {              // kRowsPerLoad rows
    const int row = row0 + ld_sub;
    const unsigned long long at = (unsigned long long)(q_rows + (long long)(q0 + row0) * a.q_token);
    const u32x4 buffer = {(unsigned)__builtin_amdgcn_readfirstlane((int)at), (unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32)) & 0xFFFFu,
                          (unsigned)__builtin_amdgcn_readfirstlane((int)bytes_of_rows<D>(n - q0 - row0, S::kRowsPerLoad, a.q_bytes)), 0x00020000u};
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"((unsigned)ld_sub * a.q_bytes + 16u * (unsigned)(ld_pos ^ k_swizzle<D>(row))),
                 "s"(buffer), "s"(to)
                 : "m0", "memory");
  };
  if constexpr (kShared) {
    // the query rows: a load of each wave (of the first four at d 64), for all; the wave's first block behind it
    if (wave < 32 / S::kRowsPerLoad) load_q(S::kRowsPerLoad * wave, lds_at + (unsigned)(S::kQ + 1024 * wave));
    if (wave < n_blocks) {
      issue_k(wave);
      issue_v(wave);
      wait_all_but(BothStrips{});
    } else {
      wait_all_but(None{});
    }
    __syncthreads();
#pragma unroll
    for (int st = 0; st < kNK; ++st) qf[st] = lds_read_b128(q_lds + k_off[st]);
  } else {
    // the query rows through the strip of V, beside the first keys
#pragma unroll
    for (int j = 0; j < 32 / S::kRowsPerLoad; ++j) load_q(S::kRowsPerLoad * j, my_lds + 2u * (unsigned)S::kStrip + 1024u * j);
    issue_k(0);
    wait_all_but(OneStrip{});
#pragma unroll
    for (int st = 0; st < kNK; ++st) qf[st] = lds_read_b128(v_strip + k_off[st]);
#pragma unroll
    for (int st = 0; st < kNK; ++st) asm volatile("" : "+v"(qf[st]));    // read, before the strip is filled
    issue_v(0);
  }

  f32x16 o[kND];
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int dt = 0; dt < kND; ++dt) o[dt] = zero;
  float m = -INFINITY, l = 0.f;
  constexpr int kStep = kShared ? S::kWaves : 1;
  for (int b = kShared ? wave : 0; b < n_blocks; b += kStep) {
    const bool more = b + kStep < n_blocks;
    wait_all_but(OneStrip{});
    f32x16 s = zero;
#pragma unroll
    for (int st = 0; st < kNK; ++st) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read_b128(k_strip + k_off[st]), qf[st], s, 0, 0, 0);
    // K has been read; and a vector instruction may read a product 12 wait states after it, which the compiler does not see to in
    // another basic block
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_nop 7\n\ts_nop 7" : "+v"(s)::"memory");
    if (more) issue_k(b + kStep);
    if (b == n_blocks - 1) {                   // key 8 (r / 4) + 4 g + r % 4 of the block and row l32 of the tile
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) <= l32 - 4 * g ? s[r] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    top = max_with_other_half(top);
    if (__any(top > m)) {                       // a larger logit: what has been added up is brought onto it
      const float m_new = fmaxf(m, top), by = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * sl2);
      m = m_new;
      l *= by;
#pragma unroll
      for (int dt = 0; dt < kND; ++dt) o[dt] *= by;
    }
    const float minus = m == -INFINITY ? 0.f : -m * sl2;
    unsigned p[8];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sl2, minus)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], sl2, minus));
      l += p0 + p1;
      p[r / 2] = pack_bf16(p0, p1);
    }
    if (more) wait_all_but(OneStrip{});
    else wait_all_but(None{});
#pragma unroll
    for (int vi = 0; vi < kNV; ++vi) {
      const u32x4 pw = {p[4 * (vi % 2)], p[4 * (vi % 2) + 1], p[4 * (vi % 2) + 2], p[4 * (vi % 2) + 3]};
      o[vi / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read_vt(v_strip + v_off[vi / 2] + 16 * (vi % 2) * D, 8 * D), __builtin_bit_cast(bf16x8, pw), o[vi / 2], 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) issue_v(b + kStep);
  }

  if constexpr (kND == 4) asm volatile("s_nop 7\n\ts_nop 7" : "+v"(o[0]), "+v"(o[1]), "+v"(o[2]), "+v"(o[3]));
  else asm volatile("s_nop 7\n\ts_nop 7" : "+v"(o[0]), "+v"(o[1]));
  if constexpr (!kShared) {
    float l_row = sum_with_other_half(l), check = l_row * 0.f;
#pragma unroll
    for (int dt = 0; dt < kND; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) check = __builtin_fmaf(o[dt][r], 0.f, check);
    // what is not finite is not 0 when it is multiplied by 0: a value that the row does not see may be in it
    if (__any(!(check == 0.f))) rows_the_slow_way<D>(qf, k_rows, a.k_token, v_rows, a.v_token, q0, n, sl2, l32, g, o, l_row);
    store_rows<D>(o, 1.f / l_row, reinterpret_cast<u32x4*>(k_strip), out_rows + (long long)q0 * a.out_token, a.out_token, n - q0, lane);
    return;
  }
  // ---- the waves' results, added up: a thread has eight channels of a row
  if (wave < n_blocks) {
    l = sum_with_other_half(l);
    if (g == 0) {
      stats[64 * wave + l32] = m;
      stats[64 * wave + 32 + l32] = l;
    }
    f32x4* const left = reinterpret_cast<f32x4*>(k_strip) + lane;
#pragma unroll
    for (int k = 0; k < 4 * kND; ++k) left[64 * k] = f32x4{o[k / 4][4 * (k % 4)], o[k / 4][4 * (k % 4) + 1], o[k / 4][4 * (k % 4) + 2], o[k / 4][4 * (k % 4) + 3]};
  }
  __syncthreads();
  const int row = tid % 32, chunk = tid / 32, in_use = min(n_blocks, S::kWaves);
  if (chunk >= S::kChunks) return;
  float top = stats[row];
  for (int w = 1; w < in_use; ++w) top = fmaxf(top, stats[64 * w + row]);
  const float use = top == -INFINITY ? 0.f : top;
  float l_row = 0.f;
  f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
  for (int w = 0; w < in_use; ++w) {
    const float f = __builtin_amdgcn_exp2f((stats[64 * w + row] - use) * sl2);
    const f32x4* const left = reinterpret_cast<const f32x4*>(lds_raw + w * S::kWaveBytes) + 64 * chunk + row;
    l_row += f * stats[64 * w + 32 + row];
    lo += f * left[0];
    hi += f * left[32];
  }
  // what is not finite is not 0 when it is multiplied by 0: a value that the row does not see may be in it
  const float check = ((lo[0] + lo[1]) + (lo[2] + lo[3]) + ((hi[0] + hi[1]) + (hi[2] + hi[3]))) * 0.f + l_row * 0.f;
  if (__any(!(check == 0.f))) {
    rows_the_slow_way<D>(qf, k_rows, a.k_token, v_rows, a.v_token, q0, n, sl2, l32, g, o, l_row);
    const float inv = 1.f / l_row;
#pragma unroll
    for (int k = 0; k < 4 * kND; ++k)           // this wave's chunks
      if (k / 2 == wave && q0 + l32 < n)
        *reinterpret_cast<u32x2*>(out_rows + (long long)(q0 + l32) * a.out_token + 8 * k + 4 * g) =
            u32x2{pack_bf16(o[k / 4][4 * (k % 4)] * inv, o[k / 4][4 * (k % 4) + 1] * inv), pack_bf16(o[k / 4][4 * (k % 4) + 2] * inv, o[k / 4][4 * (k % 4) + 3] * inv)};
    return;
  }
  const float inv = 1.f / l_row;
  if (q0 + row < n)
    *reinterpret_cast<u32x4*>(out_rows + (long long)(q0 + row) * a.out_token + 8 * chunk) =
        u32x4{pack_bf16(lo[0] * inv, lo[1] * inv), pack_bf16(lo[2] * inv, lo[3] * inv), pack_bf16(hi[0] * inv, hi[1] * inv), pack_bf16(hi[2] * inv, hi[3] * inv)};
}

template <int D, int KS>
hipError_t prepare() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(prompt_kernel<D, KS>), hipFuncAttributeMaxDynamicSharedMemorySize, Shape<D, KS>::kLds);
}
template <int D, bool kShared>
hipError_t prepare_few() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(prompt_few_kernel<D, kShared>), hipFuncAttributeMaxDynamicSharedMemorySize, FewShape<D, kShared>::kLds);
}

// The grid for tiles of so many rows, `each` of them to a workgroup: every prompt may have one that is not full.
unsigned deal_out(PromptArgs& a, int rows, int each) {
  const long long tiles = ((long long)a.n_tokens + (long long)(rows - 1) * a.n_seqs) / rows;
  const unsigned items = (unsigned)(tiles * a.set_heads), per_die = (items + a.dies_per_set - 1) / a.dies_per_set;
  a.by_set_heads = divisor_of((unsigned)a.set_heads, items + (unsigned)(each * kXcds));
  return kXcds * ((per_die + each - 1) / each);
}

template <int D, bool kShared>
hipError_t launch_few(const PromptArgs& a, unsigned grid, hipStream_t s) {
  using S = FewShape<D, kShared>;
  hipLaunchKernelGGL((prompt_few_kernel<D, kShared>), dim3(grid), dim3(S::kThreads), S::kLds, s, a);
  return hipGetLastError();
}

// Four ways, by the workgroups that there would be and the mean length of the prompts; the host knows no other.
// 32 rows by eight waves: while the chip holds all of these workgroups at once, one per CU at d 128 and two at 64, or a quarter more, or 512 of long
// prompts.  Against 128 rows, d 128: 4 heads of 608 rows (76 workgroups) 8.3 and 11.6 us, 32 of 256 (256) 6.8 and 8.5, 4 of eight prompts of 295 (324) 9.6 and
// 9.1, of one of 1562 and seven of 100 (312) 14.6 and 20.0, 16 of 1024 (512) 15.9 and 16.1, 8 of 2000 (504) 21.3 and 24.2, 8 of eight prompts of 200 (448)
// 10.6 and 8.3; d 64: 32 of 512 (512) 7.5 and 8.2, 8 of one of 1562 and seven of 100 (624) 12.4 and 15.5, 4 of 32 prompts of 128 (636) 6.5 and 5.9.
// 32 rows by one wave: short prompts, where 128 rows would be more workgroups than the chip holds, most of each idle.  32/8 heads, d 128, 128 rows and 32: 56
// prompts of one row 19.7 and 6.7 us, 28 of 26 12.0 and 6.2, 64 of 64 28.7 and 22.2, 26 of 100 19.2 and 17.3; 60 of 30 and one of 1000 36.1 and 36.4, of
// 2000 57.5 and 66.7; d 64 64 of 64 17.1 and 10.7, 60 of 30 and one of 2000 34.4 and 51.4.
// 128 rows and two groups of waves that share the keys: where every workgroup has a CU to itself (a wave alone on a SIMD has the pipe wait for it half of
// the time), or nearly so and the longest of them decides, and the prompts are not too short for it.  One group and two, d 128: 32 heads of 512 rows
// 12.3 and 11.9 us, 1536 30.3 and 27.4, 4096 132 and 136, 8 of 8000 (504 workgroups) 138 and 122, 4 of 16000 (500) 270 and 233, 8 of one prompt of 1562 and
// seven of 100 (200) 23.9 and 20.5, of eight of 295 (208) 9.4 and 10.2, 16 of eight of 500 (512) 18.0 and 23.7; d 64, 4 of 16000 170 and 150.
template <int D>
hipError_t launch(PromptArgs a, hipStream_t s) {
  const long long mean = a.n_tokens / a.n_seqs;
  constexpr unsigned kFew = 256 * FewShape<D, true>::kPerCu;
  unsigned grid = deal_out(a, 32, 1);
  if (grid <= kFew + kFew / 4 || (grid <= 512 && mean >= 1024)) return launch_few<D, true>(a, grid, s);
  grid = deal_out(a, kPromptRows, 1);
  if (grid > 512 && mean <= 64) {
    grid = deal_out(a, 32, FewShape<D, false>::kItems);
    return launch_few<D, false>(a, grid, s);
  }
  if ((grid <= 256 && mean >= 192) || (grid <= 512 && mean >= 1024))
    hipLaunchKernelGGL((prompt_kernel<D, 2>), dim3(grid), dim3(Shape<D, 2>::kThreads), (Shape<D, 2>::kLds), s, a);
  else
    hipLaunchKernelGGL((prompt_kernel<D, 1>), dim3(grid), dim3(Shape<D, 1>::kThreads), (Shape<D, 1>::kLds), s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t prepare_prompt() {
  hipError_t e;
  if ((e = prepare<128, 1>()) != hipSuccess || (e = prepare<128, 2>()) != hipSuccess || (e = prepare<64, 1>()) != hipSuccess) return e;
  if ((e = prepare<64, 2>()) != hipSuccess || (e = prepare_few<64, true>()) != hipSuccess || (e = prepare_few<64, false>()) != hipSuccess) return e;
  if ((e = prepare_few<128, true>()) != hipSuccess) return e;
  return prepare_few<128, false>();
}

hipError_t launch_prompt(const PromptArgs& a, int head_dim, hipStream_t s) { return head_dim == 128 ? launch<128>(a, s) : launch<64>(a, s); }

}  // namespace kvp
