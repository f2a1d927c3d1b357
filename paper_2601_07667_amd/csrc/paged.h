// The paged cache: what its kernels and its entry points share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "asl.h"
#include "paged_index.h"

namespace asl {

// What asl_paged_reserve allocates.
struct PagedWorkspace {
  void* base;
  int32_t room_rows, room_dim;                         // what it was made for (room_for)
  int32_t max_seqs, max_query_rows, max_head_dim;      // the limits last asked for
  float* part;             // [part_rows][max_head_dim, a power of two >= 64] attention: unnormalised results of cut rows ...
  float2* part_mz;         // [part_rows] ... with their reference and sum
  uint32_t* arrived;       // [part_rows] zeros between calls
  int64_t part_rows;
  int4* plan;              // [2][kPagedMaxSeqs] how sequences and groups were cut
  int32_t* group;          // [kPagedMaxSeqs] the sequences' groups
  int32_t* cut;            // [1] whether any row is in pieces
  int4* forks;             // [kPagedMaxSeqs] what the bookkeeping launch of a fork leaves for the copying one
  int32_t* fresh;          // [kMaxFresh] the free pages that a call takes, in order
  uint32_t* fault;         // [1] the context's first workspace has it, for all
};

struct PagesWriteArgs {
  PageMap map;
  const int32_t* cu;       // [n + 1]
  const int32_t* rows;     // [n] rows that are written to
  const int32_t* src_rows; // [n] rows that are read, or null: k, v are dense
  const int32_t* idx;      // [idx_rows][total] or null
  const char* k;           // dense source, or the pages
  const char* v;
  char* k_pages;
  char* v_pages;
  int64_t ksh, kst, vsh, vst;  // strides of a dense source in bytes
  int32_t n, total, n_src, idx_rows;
  int32_t cpr, cpr_shift;  // 16-byte pieces of a row; the shift is -1 where that is no power of two
  int32_t tokens;          // of a workgroup (set by launch_pages_write)
};
hipError_t launch_pages_write(const PagesWriteArgs& a, int Hk, hipStream_t st);

struct PagesForkArgs {
  PageMap map;
  int32_t* table;
  int32_t* kv_len;
  int32_t* refs;           // [n_pages] rows that hold a page; 0 = free
  const int32_t* parents;  // [n]
  const int32_t* children; // [n]
  const void* const* k_ptrs;   // device arrays [n_layers], or null
  const void* const* v_ptrs;
  int4* forks;
  int32_t n, n_layers, Hk, cpr, cpr_shift;
};
hipError_t launch_pages_fork(const PagesForkArgs& a, int32_t* fresh, hipStream_t st);
hipError_t launch_pages_grow(const PageMap& map, int32_t* table, int32_t* kv_len, int32_t* refs, const int32_t* rows,
                             const int32_t* add, int n, int32_t* fresh, hipStream_t st);
hipError_t launch_pages_free(const PageMap& map, int32_t* kv_len, int32_t* refs, const int32_t* rows, int n, hipStream_t st);

struct AttendArgs {
  PageMap map;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;              // [Hq][total_q] or null
  const int32_t* rows;     // [n_seqs] or null: sequence b is row b
  const int32_t* cu_q;     // [n_seqs + 1]
  const int32_t* group_start;  // [n_groups + 1] or null
  const int32_t* prefix_len;   // [n_groups]
  int64_t qt, qh, ot, oh;  // strides of q and out in elements
  int32_t Hq, Hk, G, d;
  int32_t n_seqs, total_q, max_q_len, max_kv_len, n_groups, causal;
  int32_t key_bytes;       // of K and V of a token
  float scale;
};
hipError_t launch_attend(const PagedWorkspace& ws, const AttendArgs& a, int dtype, hipStream_t st);
hipError_t launch_attend_bf16_64(const PagedWorkspace& ws, const AttendArgs& a, hipStream_t st);
hipError_t launch_attend_bf16_128(const PagedWorkspace& ws, const AttendArgs& a, hipStream_t st);

}  // namespace asl
