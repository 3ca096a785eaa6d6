// C entry points of the operators over a paged cache: checks of what the host can see, workspaces, launches.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "../../include/sled.h"
#include "kernels.h"
#include "paged.h"

static_assert(sled::kMaxTreeNodes == SLED_MAX_TREE_NODES, "the limit stated in sled.h");

namespace {

using namespace sled;

// A workspace of more than kMostBytes bytes, or whose size does not fit 64 bits, is refused; -1 stands for it.
constexpr int64_t kMostBytes = 1LL << 60;
int64_t align256(int64_t v) { return v < 0 ? v : (v + 255) / 256 * 256; }
int64_t product(std::initializer_list<int64_t> factors) {
  int64_t n = 1;
  for (const int64_t f : factors)
    if (__builtin_mul_overflow(n, f, &n) || n > kMostBytes) return -1;
  return n;
}
int64_t sum(std::initializer_list<int64_t> parts) {
  int64_t n = 0;
  for (const int64_t p : parts) {
    if (p < 0) return -1;
    n += p;
  }
  return n;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// sizes and pointers of a cache description; layers: whether more than one layer is allowed
int check_cache(const sled_paged_kv* kv, bool need_v, bool layers) {
  if (!kv || !kv->k || (need_v && !kv->v)) return SLED_ERR_ARG;
  if (kv->dtype != SLED_F32 && kv->dtype != SLED_BF16) return SLED_ERR_ARG;
  if (kv->head_dim != 32 && kv->head_dim != 64 && kv->head_dim != 128) return SLED_ERR_ARG;
  if (kv->page_size <= 0 || kv->page_size % 16 || kv->page_size > 256) return SLED_ERR_ARG;
  if (kv->n_layers < 1 || (!layers && kv->n_layers != 1)) return SLED_ERR_ARG;
  if (kv->n_pages < 1 || kv->n_kv_heads < 1 || kv->n_kv_heads > 65535) return SLED_ERR_ARG;
  if (kv->n_reqs < 0 || kv->n_reqs > 65535 || kv->table_cols < 0 || kv->table_stride < kv->table_cols) return SLED_ERR_ARG;
  // arrays without entries need no address
  if ((kv->n_reqs > 0 && !kv->n_kv) || (kv->n_reqs > 0 && kv->table_cols > 0 && !kv->page_table)) return SLED_ERR_ARG;
  if (kv->n_layers > 65535) return SLED_ERR_ARG;
  if (!aligned(kv->k, 16) || (kv->v && !aligned(kv->v, 16)) || !aligned(kv->page_table, 4) || !aligned(kv->n_kv, 4)) return SLED_ERR_ARG;
  // rows of one layer, and keys of one request (rounded up to tiles), are counted in 32 bits
  if (static_cast<int64_t>(kv->n_pages) * kv->n_kv_heads * kv->page_size > INT32_MAX) return SLED_ERR_ARG;
  if (static_cast<int64_t>(kv->table_cols) * kv->page_size > INT32_MAX - 1024) return SLED_ERR_ARG;
  return SLED_OK;
}

int check_rows(const sled_paged_kv* kv, const void* q, int64_t q_stride, const int32_t* cu_q, int32_t n_rows, int32_t n_q_heads,
               float scale, const void* out, int64_t out_stride) {
  if (n_rows < 0 || n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % kv->n_kv_heads) return SLED_ERR_ARG;
  if (static_cast<int64_t>(n_rows) * n_q_heads > INT32_MAX) return SLED_ERR_ARG;   // (row, head) pairs are counted in 32 bits
  if (!(scale >= 0.f) || scale > 3.0e38f || !cu_q || !aligned(cu_q, 4)) return SLED_ERR_ARG;
  if (n_rows > 0 && (!q || !out)) return SLED_ERR_ARG;
  const int64_t row = static_cast<int64_t>(n_q_heads) * kv->head_dim;
  if (q_stride < row || out_stride < row || !aligned(q, 4) || !aligned(out, 4)) return SLED_ERR_ARG;
  if (kv->dtype == SLED_BF16 && (q_stride % 2 || out_stride % 2)) return SLED_ERR_ARG;
  return SLED_OK;
}

// The kernels run on the GPU that holds the cache; the caller's current device is put back.
class OnDeviceOf {
 public:
  explicit OnDeviceOf(const void* p) {
    cudaPointerAttributes attr{};
    if (cudaPointerGetAttributes(&attr, p) != cudaSuccess || attr.type != cudaMemoryTypeDevice || cudaGetDevice(&before_) != cudaSuccess) {
      int n_dev = 0;
      rc_ = cudaGetDeviceCount(&n_dev) != cudaSuccess || n_dev == 0 ? SLED_ERR_NO_DEVICE : SLED_ERR_ARG;
      cudaGetLastError();
      return;
    }
    if (attr.device != before_) {
      if (cudaSetDevice(attr.device) != cudaSuccess) { cudaGetLastError(); rc_ = SLED_ERR_DEVICE; return; }
      moved_ = true;
    }
  }
  ~OnDeviceOf() { if (moved_) cudaSetDevice(before_); }
  OnDeviceOf(const OnDeviceOf&) = delete;
  OnDeviceOf& operator=(const OnDeviceOf&) = delete;
  int rc() const { return rc_; }

 private:
  int before_ = 0, rc_ = SLED_OK;
  bool moved_ = false;
};

PagedCache cache_of(const sled_paged_kv* kv, int32_t* status) {
  PagedCache c{};
  c.k = static_cast<const char*>(kv->k);
  c.v = static_cast<const char*>(kv->v);
  c.dtype = kv->dtype == SLED_BF16 ? BF16 : F32;
  c.n_layers = kv->n_layers;
  c.n_pages = kv->n_pages;
  c.Hkv = kv->n_kv_heads;
  c.ps = kv->page_size;
  c.h = kv->head_dim;
  c.layer_bytes = static_cast<int64_t>(kv->n_pages) * kv->n_kv_heads * kv->page_size * kv->head_dim * (kv->dtype == SLED_BF16 ? 2 : 4);
  c.table = kv->page_table;
  c.table_stride = kv->table_stride;
  c.table_cols = kv->table_cols;
  c.n_kv = kv->n_kv;
  c.n_reqs = kv->n_reqs;
  c.status = status;
  return c;
}

PagedRows rows_of(const sled_paged_kv* kv, const void* q, int64_t q_stride, const int32_t* cu_q, const int32_t* parents, int32_t n_rows,
                  int32_t n_q_heads, float scale, void* out, int64_t out_stride, float* lse) {
  PagedRows r{};
  r.cu_q = cu_q;
  r.parents = parents;
  r.q = static_cast<const char*>(q);
  r.out = static_cast<char*>(out);
  r.lse = lse;
  r.q_stride = q_stride;
  r.out_stride = out_stride;
  r.T = n_rows;
  r.Hq = n_q_heads;
  r.group = n_q_heads / kv->n_kv_heads;
  r.scale = scale > 0.f ? scale : 1.f / sqrtf(static_cast<float>(kv->head_dim));
  return r;
}

int done(int n, const char* what) {
  if (n >= 0) return SLED_OK;
  std::fprintf(stderr, "sled: %s failed: %s\n", what, cudaGetErrorString(cudaPeekAtLastError()));
  cudaGetLastError();
  return SLED_ERR_DEVICE;
}

int check_workspace(const void* workspace, int64_t have, int64_t need) {
  return need < 0 || (need > 0 && (!workspace || have < need || !aligned(workspace, 256))) ? SLED_ERR_ARG : SLED_OK;
}

// the same arrays, or arrays that share no byte
bool same_or_apart(const void* a, const void* b, int64_t bytes) {
  const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
  return x == y || x + bytes <= y || y + bytes <= x;
}

int64_t lse_bytes(int32_t n_rows, int32_t n_q_heads) { return align256(product({n_rows, n_q_heads, 4})); }
int64_t list_bytes(const sled_paged_kv* kv, int32_t n_rows, int32_t n_blocks) {
  return align256(product({n_rows, kv->n_kv_heads, n_blocks, 4}));
}

int64_t attention_bytes(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, bool weigh) {
  return align256(paged_attention_workspace(kv->dtype == SLED_BF16 ? BF16 : F32, kv->head_dim, static_cast<int64_t>(n_rows) * n_q_heads,
                                            static_cast<int64_t>(kv->table_cols) * kv->page_size, weigh));
}
int64_t tree_bytes(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, bool weigh) {
  return sum({attention_bytes(kv, n_rows, n_q_heads, weigh), weigh ? lse_bytes(n_rows, n_q_heads) : 0});
}
int64_t blocks_bytes(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t n_blocks) {
  return sum({attention_bytes(kv, n_rows, n_q_heads, false), list_bytes(kv, n_rows, n_blocks), list_bytes(kv, n_rows, kv->table_cols)});
}
int64_t evict_bytes(const sled_paged_kv* kv) {
  return align256(product({kv->n_layers, kv->n_reqs, kv->n_kv_heads, kv->table_cols, kv->page_size, 4}));
}

}  // namespace

extern "C" {

int sled_attention_tree_workspace(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t weigh, int64_t* bytes) {
  if (check_cache(kv, true, false) || n_rows < 0 || n_q_heads < 1 || !bytes) return SLED_ERR_ARG;
  const int64_t n = tree_bytes(kv, n_rows, n_q_heads, weigh != 0);
  if (n < 0) return SLED_ERR_ARG;
  *bytes = n;
  return SLED_OK;
}

int sled_attention_tree(const sled_paged_kv* kv, const void* q, int64_t q_stride, const int32_t* cu_q, const int32_t* parents,
                        int32_t n_rows, int32_t n_q_heads, float scale, void* out, int64_t out_stride, float* lse, float* key_weights,
                        int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(kv, true, false);
  if (!rc) rc = check_rows(kv, q, q_stride, cu_q, n_rows, n_q_heads, scale, out, out_stride);
  if (!rc && (!aligned(parents, 4) || !aligned(lse, 4) || !aligned(key_weights, 4) || !aligned(status, 4))) rc = SLED_ERR_ARG;
  if (!rc) rc = check_workspace(workspace, workspace_bytes, tree_bytes(kv, n_rows, n_q_heads, key_weights != nullptr));
  if (rc) return rc;
  if (n_rows == 0 || kv->n_reqs == 0) return SLED_OK;
  OnDeviceOf device(kv->k);
  if (device.rc()) return device.rc();
  char* ws = static_cast<char*>(workspace);
  if (key_weights && !lse) lse = reinterpret_cast<float*>(ws + attention_bytes(kv, n_rows, n_q_heads, true));
  const PagedCache c = cache_of(kv, status);
  const PagedRows r = rows_of(kv, q, q_stride, cu_q, parents, n_rows, n_q_heads, scale, out, out_stride, lse);
  return done(launch_paged_attention(c, r, nullptr, 0, key_weights, ws, static_cast<cudaStream_t>(stream)), "sled_attention_tree");
}

int sled_evict_keys_workspace(const sled_paged_kv* kv, int64_t* bytes) {
  if (check_cache(kv, true, true) || !bytes) return SLED_ERR_ARG;
  const int64_t n = evict_bytes(kv);
  if (n < 0) return SLED_ERR_ARG;
  *bytes = n;
  return SLED_OK;
}

int sled_evict_keys(const sled_paged_kv* kv, float* key_weights, float* key_weights_out, int32_t budget, int32_t n_sink,
                    int32_t n_recent, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(kv, true, true);
  if (rc) return rc;
  const int64_t per_layer = static_cast<int64_t>(kv->n_pages) * kv->n_kv_heads * kv->page_size;
  if (!key_weights || !key_weights_out || budget < 1 || n_sink < 0 || n_recent < 0 || static_cast<int64_t>(n_sink) + n_recent > budget)
    return SLED_ERR_ARG;
  if (!aligned(key_weights, 4) || !aligned(key_weights_out, 4) || !aligned(status, 4)) return SLED_ERR_ARG;
  if (!same_or_apart(key_weights, key_weights_out, per_layer * kv->n_layers * 4)) return SLED_ERR_ARG;
  rc = check_workspace(workspace, workspace_bytes, evict_bytes(kv));
  if (rc) return rc;
  if (kv->n_reqs == 0 || kv->table_cols == 0) return SLED_OK;
  OnDeviceOf device(kv->k);
  if (device.rc()) return device.rc();
  return done(launch_evict(cache_of(kv, status), key_weights, key_weights_out, per_layer, budget, n_sink, n_recent,
                           static_cast<int32_t*>(workspace), static_cast<cudaStream_t>(stream)), "sled_evict_keys");
}

int sled_block_bounds(const sled_paged_kv* kv, const int32_t* first, void* bounds, int32_t* status, void* stream) {
  int rc = check_cache(kv, false, false);
  if (rc) return rc;
  if (!bounds || !aligned(bounds, 16) || !aligned(first, 4) || !aligned(status, 4)) return SLED_ERR_ARG;
  if (kv->n_reqs == 0 || kv->table_cols == 0) return SLED_OK;
  OnDeviceOf device(kv->k);
  if (device.rc()) return device.rc();
  return done(launch_block_bounds(cache_of(kv, status), first, bounds, static_cast<cudaStream_t>(stream)), "sled_block_bounds");
}

int sled_attention_blocks_workspace(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t n_blocks, int64_t* bytes) {
  if (check_cache(kv, true, false) || n_rows < 0 || n_q_heads < 1 || n_blocks < 1 || !bytes) return SLED_ERR_ARG;
  const int64_t n = blocks_bytes(kv, n_rows, n_q_heads, n_blocks);
  if (n < 0) return SLED_ERR_ARG;
  *bytes = n;
  return SLED_OK;
}

int sled_attention_blocks(const sled_paged_kv* kv, const void* bounds, const void* q, int64_t q_stride, const int32_t* cu_q,
                          int32_t n_rows, int32_t n_q_heads, float scale, int32_t n_blocks, int32_t n_local, void* out,
                          int64_t out_stride, int32_t* blocks, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(kv, true, false);
  if (!rc) rc = check_rows(kv, q, q_stride, cu_q, n_rows, n_q_heads, scale, out, out_stride);
  if (!rc && (!bounds || !aligned(bounds, 16) || !aligned(blocks, 4) || !aligned(status, 4) || n_local < 1 || n_blocks < n_local)) rc = SLED_ERR_ARG;
  if (!rc) rc = check_workspace(workspace, workspace_bytes, blocks_bytes(kv, n_rows, n_q_heads, n_blocks));
  if (rc) return rc;
  if (n_rows == 0 || kv->n_reqs == 0) return SLED_OK;
  OnDeviceOf device(kv->k);
  if (device.rc()) return device.rc();
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  float* scores = reinterpret_cast<float*>(ws + attention_bytes(kv, n_rows, n_q_heads, false));
  int32_t* list = blocks ? blocks : reinterpret_cast<int32_t*>(ws + attention_bytes(kv, n_rows, n_q_heads, false) + list_bytes(kv, n_rows, kv->table_cols));
  const PagedCache c = cache_of(kv, status);
  const PagedRows r = rows_of(kv, q, q_stride, cu_q, nullptr, n_rows, n_q_heads, scale, out, out_stride, nullptr);
  int n = launch_block_choice(c, r, bounds, n_blocks, n_local, scores, list, s);
  if (n >= 0) n = launch_paged_attention(c, r, list, n_blocks, nullptr, ws, s);
  return done(n, "sled_attention_blocks");
}

}  // extern "C"
