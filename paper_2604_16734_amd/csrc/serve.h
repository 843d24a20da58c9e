// Arguments of the kernels that serve many sequences at once (serve.cpp checks them, pages.hip, paged_decode.hip and prompt.hip run them).
#pragma once
#include "kvp_internal.h"
#include "pages.h"

namespace kvp {

struct Pool {
  char* k;                    // [n_pages][n_heads][page size][head_dim], bf16 or e4m3
  char* v;
  uint8_t* k_exp;             // [n_pages][n_heads][page size], e4m3 only
  uint8_t* v_exp;
  int n_pages, n_heads, shift;
};

struct PageRowsArgs {
  Pool pool;
  u16* k;                     // the rows outside the pages
  u16* v;
  long long k_token, k_head, v_token, v_head;
  const int32_t* seq_begin;
  const int32_t* table;
  const int32_t* first;       // or null
  int width, n_seqs;
  int n_rows;                 // tokens * heads, heads fastest
  Divisor by_heads;
};

struct PagedDecodeArgs {
  Pool pool;
  const u16* q;
  u16* out;                   // [n_seqs][n_q_heads][D]
  const int32_t* table;
  const int32_t* lengths;
  float* partial;             // [2 * workgroups][group][D], then [2 * workgroups][group][2]: maximum (log2 domain) and sum
  long long q_token, q_head;
  int width, n_seqs, n_q_heads, group;
  int workgroups;
  long long most_keys;        // of a sequence, by the width of the table
  Divisor by_heads;           // n_heads of the pool
  Divisor by_group;
  float scale_log2;
};
constexpr int kPagedMostWorkgroups = 512;
hipError_t prepare_paged_decode();      // function attributes on the current device
int paged_decode_workgroups(int head_dim, bool e4m3);
hipError_t launch_paged_decode(const PagedDecodeArgs& a, int head_dim, bool e4m3, hipStream_t s);

constexpr int kPromptRows = 128;       // query rows of a workgroup, where there are many
struct PromptArgs {
  const u16* q;
  const u16* k;
  const u16* v;
  u16* out;
  const int32_t* seq_begin;
  long long q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;
  unsigned q_bytes, k_bytes, v_bytes;      // from token to token
  int n_tokens, n_seqs, n_q_heads;
  int dies_per_set, set_heads;             // dies that share set_heads query heads
  Divisor by_set_heads, by_group;
  float scale_log2;
};
hipError_t prepare_prompt();            // function attributes on the current device
hipError_t launch_prompt(const PromptArgs& a, int head_dim, hipStream_t s);

hipError_t launch_page_write(const PageRowsArgs& a, int head_dim, bool e4m3, hipStream_t s);
hipError_t launch_page_read(const PageRowsArgs& a, int head_dim, bool e4m3, hipStream_t s);

}  // namespace kvp
