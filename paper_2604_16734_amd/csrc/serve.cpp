// Host side of the calls that serve many sequences at once: checks of the arguments and launches.  No state; no device memory is
// allocated and no stream is synchronised.
#include <atomic>
#include <cmath>

#include "serve.h"

using namespace kvp;

namespace {

bool aligned(const void* p, uintptr_t to) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % to == 0; }

bool valid_pages(const kvp_pages* p) {
  if (!p || (p->format != KVP_PAGE_BF16 && p->format != KVP_PAGE_E4M3)) return false;
  if (p->head_dim != 64 && p->head_dim != 128) return false;
  if (p->page_size < 16 || p->page_size > KVP_MAX_PAGE_SIZE || (p->page_size & (p->page_size - 1)) != 0) return false;
  if (p->n_pages < 1 || p->n_kv_heads < 1) return false;
  if ((unsigned long long)p->n_pages * (unsigned)p->n_kv_heads >= (1ull << 40) / (unsigned)p->page_size) return false;
  if (!aligned(p->k, 16) || !aligned(p->v, 16)) return false;
  if (p->format == KVP_PAGE_E4M3) return aligned(p->k_exp, 4) && aligned(p->v_exp, 4);
  return !p->k_exp && !p->v_exp;
}

Pool pool_of(const kvp_pages& p) {
  int shift = 4;
  while ((1 << shift) < p.page_size) ++shift;
  return Pool{static_cast<char*>(p.k), static_cast<char*>(p.v), static_cast<uint8_t*>(p.k_exp), static_cast<uint8_t*>(p.v_exp),
              p.n_pages, p.n_kv_heads, shift};
}

bool valid_strides(int64_t token, int64_t head) {
  return token >= 0 && token < (1 << 23) && token % 8 == 0 && head >= 0 && head < (1ll << 40) && head % 8 == 0;
}
// [n_tokens, n_heads, dim] rows that do not overlap: the rows of a token inside the distance of two tokens, or the other way round
bool separate_rows(int64_t token, int64_t head, int n_tokens, int n_heads, int dim) {
  if ((n_tokens > 1 && token < dim) || (n_heads > 1 && head < dim)) return false;
  if (n_tokens <= 1 || n_heads <= 1) return true;
  return token >= (__int128)(n_heads - 1) * head + dim || head >= (n_tokens - 1) * token + dim;       // (heads times their distance may pass 64 bits)
}

bool valid_table(const int32_t* table, int32_t width, int32_t page_size, int32_t n_seqs) {
  return aligned(table, 4) && width >= 1 && width <= (1 << 30) / page_size && n_seqs >= 1 && n_seqs <= KVP_MAX_SEQUENCES;
}

int code_of(hipError_t e) { return e == hipSuccess ? KVP_OK : KVP_EDEVICE; }

int page_rows(const kvp_pages* pages, const kvp_rows* rows, const int32_t* seq_begin, const int32_t* table, int32_t width,
              const int32_t* first, int32_t n_seqs, void* stream, bool write) {
  if (!valid_pages(pages) || !rows || !valid_table(table, width, pages->page_size, n_seqs)) return KVP_EINVAL;
  if (!aligned(seq_begin, 4) || (first && !aligned(first, 4))) return KVP_EINVAL;
  if (rows->n_tokens < 0 || (long long)rows->n_tokens * pages->n_kv_heads >= 1ll << 31) return KVP_EINVAL;
  if (!valid_strides(rows->k_token, rows->k_head) || !valid_strides(rows->v_token, rows->v_head)) return KVP_EINVAL;
  if (!write && (!separate_rows(rows->k_token, rows->k_head, rows->n_tokens, pages->n_kv_heads, pages->head_dim) ||
                 !separate_rows(rows->v_token, rows->v_head, rows->n_tokens, pages->n_kv_heads, pages->head_dim)))
    return KVP_EINVAL;
  if (rows->n_tokens == 0) return KVP_OK;
  if (!aligned(rows->k, 16) || !aligned(rows->v, 16)) return KVP_EINVAL;
  PageRowsArgs a{};
  a.pool = pool_of(*pages);
  a.k = static_cast<u16*>(rows->k);
  a.v = static_cast<u16*>(rows->v);
  a.k_token = rows->k_token; a.k_head = rows->k_head;
  a.v_token = rows->v_token; a.v_head = rows->v_head;
  a.seq_begin = seq_begin; a.table = table; a.first = first;
  a.width = width; a.n_seqs = n_seqs;
  a.n_rows = rows->n_tokens * pages->n_kv_heads;
  a.by_heads = divisor_of((unsigned)pages->n_kv_heads, (unsigned)a.n_rows);
  const bool e4m3 = pages->format == KVP_PAGE_E4M3;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return code_of(write ? launch_page_write(a, pages->head_dim, e4m3, s) : launch_page_read(a, pages->head_dim, e4m3, s));
}

// Once per device: the attributes of functions, which belong to the current device (it is the stream's).
int prepared() {
  static std::atomic<unsigned long long> done{0};
  int device = 0;
  if (hipGetDevice(&device) != hipSuccess) return KVP_EDEVICE;
  const unsigned long long bit = device < 64 ? 1ull << device : 0;
  if (done.load(std::memory_order_acquire) & bit) return KVP_OK;
  if (prepare_paged_decode() != hipSuccess || prepare_prompt() != hipSuccess) return KVP_EDEVICE;
  done.fetch_or(bit, std::memory_order_release);
  return KVP_OK;
}

bool valid_group(int32_t n_q_heads, int32_t n_kv_heads) { return n_q_heads >= 1 && n_kv_heads >= 1 && n_q_heads % n_kv_heads == 0; }
float scale_log2_of(float scale, int head_dim) { return (scale > 0.f ? scale : 1.f / std::sqrt((float)head_dim)) * 1.4426950408889634f; }
bool valid_scale(float s) { return s >= 0.f && std::isfinite(scale_log2_of(s, 64)); }      // (what the kernels multiply by)

}  // namespace

// What a decode step needs: two places for partial results per workgroup, each of a KV head's query heads.
static size_t paged_decode_bytes(const kvp_pages& p, int group) {
  return (size_t)2 * paged_decode_workgroups(p.head_dim, p.format == KVP_PAGE_E4M3) * group * (p.head_dim + 2) * sizeof(float);
}

extern "C" {

size_t kvp_paged_decode_bytes(const kvp_pages* pages, int32_t n_q_heads) {
  if (!valid_pages(pages) || !valid_group(n_q_heads, pages->n_kv_heads) || n_q_heads / pages->n_kv_heads > kDecodeGroupLimit) return 0;
  return paged_decode_bytes(*pages, n_q_heads / pages->n_kv_heads);
}

int kvp_paged_decode(const kvp_pages* pages, const void* q, int64_t q_token, int64_t q_head, int32_t n_q_heads,
                     const int32_t* table, int32_t table_width, const int32_t* lengths, int32_t n_seqs,
                     float softmax_scale, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_pages(pages) || !valid_table(table, table_width, pages->page_size, n_seqs)) return KVP_EINVAL;
  if (!valid_group(n_q_heads, pages->n_kv_heads) || n_q_heads / pages->n_kv_heads > kDecodeGroupLimit || n_q_heads > 65535) return KVP_EINVAL;
  const unsigned long long tiles = ((unsigned long long)table_width * (unsigned)pages->page_size + kPagedTile - 1) / kPagedTile;
  if (tiles * (unsigned)n_seqs > (1ull << 31) / (unsigned)pages->n_kv_heads) return KVP_EINVAL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lengths, 4) || !aligned(workspace, 16)) return KVP_EINVAL;
  if (!valid_strides(q_token, q_head) || !valid_scale(softmax_scale)) return KVP_EINVAL;
  if (workspace_bytes < kvp_paged_decode_bytes(pages, n_q_heads)) return KVP_ENOMEM;
  if (const int rc = prepared()) return rc;
  PagedDecodeArgs a{};
  const bool e4m3 = pages->format == KVP_PAGE_E4M3;
  a.pool = pool_of(*pages);
  a.q = static_cast<const u16*>(q);
  a.out = static_cast<u16*>(out);
  a.table = table; a.lengths = lengths;
  a.partial = static_cast<float*>(workspace);
  a.q_token = q_token; a.q_head = q_head;
  a.width = table_width; a.n_seqs = n_seqs; a.n_q_heads = n_q_heads;
  a.group = n_q_heads / pages->n_kv_heads;
  a.workgroups = paged_decode_workgroups(pages->head_dim, e4m3);
  a.most_keys = (long long)table_width * pages->page_size;
  a.by_heads = divisor_of((unsigned)pages->n_kv_heads, (unsigned)n_seqs * (unsigned)pages->n_kv_heads);
  a.by_group = divisor_of((unsigned)a.group, (unsigned)n_q_heads);
  a.scale_log2 = scale_log2_of(softmax_scale, pages->head_dim);
  return code_of(launch_paged_decode(a, pages->head_dim, e4m3, static_cast<hipStream_t>(stream)));
}

int kvp_page_write(const kvp_pages* pages, const kvp_rows* rows, const int32_t* seq_begin, const int32_t* table,
                   int32_t table_width, const int32_t* first, int32_t n_seqs, void* stream) {
  return page_rows(pages, rows, seq_begin, table, table_width, first, n_seqs, stream, true);
}

int kvp_page_read(const kvp_pages* pages, const kvp_rows* rows, const int32_t* seq_begin, const int32_t* table,
                  int32_t table_width, const int32_t* first, int32_t n_seqs, void* stream) {
  return page_rows(pages, rows, seq_begin, table, table_width, first, n_seqs, stream, false);
}

int kvp_prompt_attention(const kvp_prompts* p, void* stream) {
  if (!p || !valid_group(p->n_q_heads, p->n_kv_heads) || (p->head_dim != 64 && p->head_dim != 128)) return KVP_EINVAL;
  if (p->n_tokens < 0 || p->n_seqs < 1 || p->n_seqs > KVP_MAX_SEQUENCES || !aligned(p->seq_begin, 4) || !valid_scale(p->softmax_scale)) return KVP_EINVAL;
  const int64_t strides[4][2] = {{p->q_token, p->q_head}, {p->k_token, p->k_head}, {p->v_token, p->v_head}, {p->out_token, p->out_head}};
  for (const auto& s : strides)
    if (!valid_strides(s[0], s[1]) || (p->n_tokens > 1 && s[0] < p->head_dim)) return KVP_EINVAL;
  if (!separate_rows(p->out_token, p->out_head, p->n_tokens, p->n_q_heads, p->head_dim)) return KVP_EINVAL;
  if (((long long)p->n_tokens / 32 + p->n_seqs) * p->n_q_heads > (1ll << 30) - 64) return KVP_EINVAL;
  if (p->n_tokens == 0) return KVP_OK;
  if (!aligned(p->q, 16) || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->out, 16)) return KVP_EINVAL;
  if (const int rc = prepared()) return rc;
  PromptArgs a{};
  a.q = static_cast<const u16*>(p->q);
  a.k = static_cast<const u16*>(p->k);
  a.v = static_cast<const u16*>(p->v);
  a.out = static_cast<u16*>(p->out);
  a.seq_begin = p->seq_begin;
  a.q_token = p->q_token; a.q_head = p->q_head;
  a.k_token = p->k_token; a.k_head = p->k_head;
  a.v_token = p->v_token; a.v_head = p->v_head;
  a.out_token = p->out_token; a.out_head = p->out_head;
  // (of one row the distance to the next means nothing; the kernel's addresses count on one)
  auto bytes = [&](int64_t token) { return 2u * (unsigned)(token < p->head_dim ? p->head_dim : token); };
  a.q_bytes = bytes(p->q_token); a.k_bytes = bytes(p->k_token); a.v_bytes = bytes(p->v_token);
  a.n_tokens = p->n_tokens; a.n_seqs = p->n_seqs; a.n_q_heads = p->n_q_heads;
  int sets = kXcds;
  while (p->n_kv_heads % sets != 0) sets /= 2;
  a.dies_per_set = kXcds / sets;
  a.set_heads = p->n_q_heads / sets;
  a.by_group = divisor_of((unsigned)(p->n_q_heads / p->n_kv_heads), (unsigned)p->n_q_heads);
  a.scale_log2 = scale_log2_of(p->softmax_scale, p->head_dim);
  return code_of(launch_prompt(a, p->head_dim, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
