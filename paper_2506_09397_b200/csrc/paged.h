// Operators over a caller's paged key-value cache (device-resident operands): launchers shared by the C entry points
// (paged_api.cu).  Every launcher only enqueues work on the given stream and returns the number of kernels it launched
// (negative: the launch failed).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace sled {

// One layer of a cache and what every request owns of it.  All pointers are device pointers.  The kernels check every
// entry that they follow: a request whose description does not hold together (lengths that do not fit its table row,
// rows outside the call, a page outside the pool, a parent that is not an earlier node) is left out and reported in
// `status`; it never leads outside the arrays.
struct PagedCache {
  const char* k;
  const char* v;
  int dtype;                  // DType of K and V
  int n_layers, n_pages, Hkv, ps, h;
  int64_t layer_bytes;        // distance between layers (eviction)
  const int32_t* table;       // [n_reqs][table_stride], table_cols entries of a row belong to the request
  int table_stride, table_cols;
  const int32_t* n_kv;        // [n_reqs]
  int n_reqs;
  int32_t* status;            // one word or null; receives a negative sled_status
};

// The queries of a call: request i owns rows cu_q[i] .. cu_q[i+1]-1, its newest keys' tokens.
struct PagedRows {
  const int32_t* cu_q;
  const int32_t* parents;     // null: a chain
  const char* q;              // [T][Hq][h], rows q_stride elements apart
  char* out;
  float* lse;                 // [T][Hq] natural logarithm, or null
  int64_t q_stride, out_stride;
  int T, Hq, group;           // group: query heads per KV head
  float scale;
};

// Attention of the rows over everything they see (list null) or over the blocks list[t][kv head][list_len], ascending,
// min(list_len, own block + 1) of them.  key_weights (optional, needs r.lse): [n_pages][Hkv][ps], added to.
// ws: paged_attention_workspace bytes.
int64_t paged_attention_workspace(int dtype, int h, int64_t rows_heads, int64_t keys, bool weigh);
int launch_paged_attention(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* key_weights, char* ws,
                           cudaStream_t s);
// the attention itself on tensor cores (bf16); scores (optional): [T][Hq][table_cols * ps] receives
// scale q.k in units of log2, -infinity where a row does not see a key, up to the request's last key
constexpr int kMaxPagedBlocks = 320;   // two on each of up to 160 SMs
int64_t paged_mma_workspace(int h);
int launch_paged_mma(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s);
// the same for fp32 caches, on CUDA cores
int64_t paged_f32_workspace(int h);
int launch_paged_f32(const PagedCache& c, const PagedRows& r, const int32_t* list, int list_len, float* scores, char* ws, cudaStream_t s);
// the same on the 5th-generation tensor cores, for requests with many query rows
int64_t paged_tc_workspace(int h);
bool paged_tc_serves(const PagedCache& c, const PagedRows& r);
int launch_paged_tc(const PagedCache& c, const PagedRows& r, char* ws, cudaStream_t s);
// adds the attention weights of the keys (bf16, head_dim 64 or 128; r.lse is set, paged_tc_serves)
int launch_paged_weigh(const PagedCache& c, const PagedRows& r, float* key_weights, cudaStream_t s);
// joins the partial results of units of unit_rows rows that were cut over `blocks` shares; desc: two words of 16 bytes a share
int launch_paged_merge(const PagedCache& c, const PagedRows& r, int unit_rows, int blocks, float* acc, float* ml, int4* desc, cudaStream_t s);
// the current device and the number of its SMs, or a negative value
constexpr int kMaxDevices = 64;
int paged_device(int* sms);
// Lets a kernel use so much dynamic shared memory, once per device; done[kMaxDevices]: what has been set.  Host threads that
// meet here set it twice, which does no harm.
template <typename Kernel>
bool allow_shared(Kernel kernel, int bytes, int dev, std::atomic<bool>* done) {
  if (done[dev].load(std::memory_order_relaxed)) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  done[dev].store(true, std::memory_order_relaxed);
  return true;
}
// bounds[page][Hkv][2][h] of the pages that hold the keys first[i] .. n_kv[i]-1 (first null: all keys)
int launch_block_bounds(const PagedCache& c, const int32_t* first, void* bounds, cudaStream_t s);
// the blocks of every (row, KV head), ascending, into list [T][Hkv][n_blocks]; scores: room for [T][Hkv][table_cols]
int launch_block_choice(const PagedCache& c, const PagedRows& r, const void* bounds, int n_blocks, int n_local, float* scores,
                        int32_t* list, cudaStream_t s);
// weights, weights_out: [n_layers][n_pages][Hkv][ps], the same array or disjoint ones; pairs: room for
// [n_layers][n_reqs][Hkv][table_cols * ps]
int launch_evict(const PagedCache& c, float* weights, float* weights_out, int64_t weight_layer, int budget, int n_sink, int n_recent,
                 int32_t* pairs, cudaStream_t s);

constexpr int kMaxTreeNodes = 128;   // nodes of one request's tree (chains have no limit)

}  // namespace sled
