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

// sizes and pointers of a cache description; layers: whether more than one layer is allowed; codes: whether 8 bits are
int check_cache(const sled_paged_kv* kv, bool need_v, bool layers, bool codes = false) {
  if (!kv || !kv->k || (need_v && !kv->v)) return SLED_ERR_ARG;
  if (kv->dtype != SLED_F32 && kv->dtype != SLED_BF16 && !(codes && kv->dtype == SLED_E4M3)) return SLED_ERR_ARG;
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
  if (kv->dtype != SLED_F32 && (q_stride % 2 || out_stride % 2)) return SLED_ERR_ARG;
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
  c.dtype = kv->dtype == SLED_BF16 ? BF16 : kv->dtype == SLED_E4M3 ? E4M3 : F32;
  c.n_layers = kv->n_layers;
  c.n_pages = kv->n_pages;
  c.Hkv = kv->n_kv_heads;
  c.ps = kv->page_size;
  c.h = kv->head_dim;
  c.layer_bytes = static_cast<int64_t>(kv->n_pages) * kv->n_kv_heads * kv->page_size * kv->head_dim * (kv->dtype == SLED_BF16 ? 2 : kv->dtype == SLED_E4M3 ? 1 : 4);
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

bool apart(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
  return !a || !b || a_bytes <= 0 || b_bytes <= 0 || x + a_bytes <= y || y + b_bytes <= x;
}

// rows of heads of sled_rotary
int check_heads(const sled_heads* h, int32_t n_rows, int32_t head_dim, int32_t dtype) {
  const uintptr_t a = dtype == SLED_BF16 ? 2 : 4;
  if (h->n_heads < 0 || h->n_heads > 65535 || static_cast<int64_t>(n_rows) * h->n_heads > INT32_MAX) return SLED_ERR_ARG;
  if (n_rows == 0 || h->n_heads == 0) return SLED_OK;
  if (!h->in || !h->out || !aligned(h->in, a) || !aligned(h->out, a)) return SLED_ERR_ARG;
  // strides of what there is more than one of; below 2^31, so that no distance leaves 64 bits
  const int64_t in_row = n_rows > 1 ? h->in_row : 0, in_head = h->n_heads > 1 ? h->in_head : 0;
  const int64_t row = n_rows > 1 ? h->out_row : 0, head = h->n_heads > 1 ? h->out_head : 0;
  for (const int64_t s : {in_row, in_head, row, head})
    if (s < 0 || s > INT32_MAX) return SLED_ERR_ARG;
  // the places of the output are all different: rows of heads, or heads of rows
  const int64_t rows_span = (n_rows - 1) * row, heads_span = (h->n_heads - 1) * head;
  const bool heads_within = (h->n_heads == 1 || head >= head_dim) && (n_rows == 1 || row >= heads_span + head_dim);
  const bool rows_within = (n_rows == 1 || row >= head_dim) && (h->n_heads == 1 || head >= rows_span + head_dim);
  if (!heads_within && !rows_within) return SLED_ERR_ARG;
  if (h->in == h->out && (in_row != row || in_head != head)) return SLED_ERR_ARG;
  return SLED_OK;
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

int sled_page_slots(const int32_t* n_kv, const int32_t* n_keep, const int32_t* n_new, int32_t n_reqs, int32_t page_size,
                    int32_t* page_table, int32_t table_stride, int32_t table_cols, int32_t* free_pages, int32_t free_cap,
                    const int32_t* n_free, int32_t* n_kv_out, int32_t* n_free_out, int32_t* cu_q, int32_t* positions,
                    int64_t* slots, int32_t n_rows, int32_t* status, void* stream) {
  if (n_reqs < 0 || n_reqs > 65535 || page_size < 1 || table_cols < 0 || table_stride < table_cols || free_cap < 0 || n_rows < 0)
    return SLED_ERR_ARG;
  if (static_cast<int64_t>(table_cols) * page_size > INT32_MAX - 1024) return SLED_ERR_ARG;
  if (n_reqs > 0 && (!n_kv || !n_new || !n_kv_out || (table_cols > 0 && !page_table))) return SLED_ERR_ARG;
  if (!n_free || !n_free_out || !cu_q || (free_cap > 0 && !free_pages)) return SLED_ERR_ARG;
  for (const void* p : {static_cast<const void*>(n_kv), static_cast<const void*>(n_keep), static_cast<const void*>(n_new),
                        static_cast<const void*>(page_table), static_cast<const void*>(free_pages), static_cast<const void*>(n_free),
                        static_cast<const void*>(n_kv_out), static_cast<const void*>(n_free_out), static_cast<const void*>(cu_q),
                        static_cast<const void*>(positions), static_cast<const void*>(status)})
    if (!aligned(p, 4)) return SLED_ERR_ARG;
  if (!aligned(slots, 8)) return SLED_ERR_ARG;
  // blocks read the inputs while others write the outputs
  const int64_t per_req = 4LL * n_reqs, table_bytes = n_reqs > 0 ? 4LL * ((n_reqs - 1LL) * table_stride + table_cols) : 0;
  const struct { const void* p; int64_t bytes; } in[] = {{n_kv, per_req}, {n_keep, per_req}, {n_new, per_req}, {n_free, 4}},
      out[] = {{n_kv_out, per_req}, {n_free_out, 4}, {cu_q, per_req + 4}, {positions, 4LL * n_rows}, {slots, 8LL * n_rows}, {status, 4},
               {page_table, table_bytes}, {free_pages, 4LL * free_cap}};
  for (int i = 0; i < 8; ++i) {
    for (const auto& x : in)
      if (!apart(x.p, x.bytes, out[i].p, out[i].bytes)) return SLED_ERR_ARG;
    for (int j = 0; j < i; ++j)
      if (!apart(out[j].p, out[j].bytes, out[i].p, out[i].bytes)) return SLED_ERR_ARG;
  }
  OnDeviceOf device(cu_q);
  if (device.rc()) return device.rc();
  const SlotsCall a{n_kv, n_keep, n_new, n_reqs, page_size, page_table, table_stride, table_cols, free_pages, free_cap, n_free, n_kv_out, n_free_out,
                    cu_q, positions, slots, n_rows, status};
  return done(launch_page_slots(a, static_cast<cudaStream_t>(stream)), "sled_page_slots");
}

int sled_rotary_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double length, double low, double high,
                            double* frequencies, double* amplitude) {
  if (rot_dim < 2 || rot_dim > 512 || rot_dim % 2 || !frequencies || !(theta > 0) || !std::isfinite(theta)) return SLED_ERR_ARG;
  if (scaling < SLED_ROTARY_PLAIN || scaling > SLED_ROTARY_RAMP) return SLED_ERR_ARG;
  if (scaling != SLED_ROTARY_PLAIN && (!(factor > 0) || !std::isfinite(factor))) return SLED_ERR_ARG;
  if (scaling == SLED_ROTARY_BASE && rot_dim == 2) return SLED_ERR_ARG;
  const double d = rot_dim, two_pi = 6.283185307179586;
  if (scaling >= SLED_ROTARY_BANDS) {
    if (!(length > 0) || !std::isfinite(length) || !(low >= 0) || !(high > low) || !std::isfinite(high)) return SLED_ERR_ARG;
    if (scaling == SLED_ROTARY_RAMP && (!(low > 0) || !(theta > 1))) return SLED_ERR_ARG;
  }
  if (scaling == SLED_ROTARY_BASE) theta *= std::pow(factor, d / (d - 2));
  double first = 0, last = 0;
  if (scaling == SLED_ROTARY_RAMP) {      // the (real) index of the pair that makes so many turns: length theta^(-2i/d) = 2 pi turns
    const auto index = [&](double turns) { return d * std::log(length / (turns * two_pi)) / (2 * std::log(theta)); };
    first = std::fmax(std::floor(index(high)), 0.0);
    last = std::fmin(std::ceil(index(low)), d - 1);
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(theta, -2.0 * i / d);
    double s = 1;                         // how much of f stays
    if (scaling == SLED_ROTARY_LINEAR) s = 0;
    if (scaling == SLED_ROTARY_BANDS) s = std::fmin(std::fmax((length * f / two_pi - low) / (high - low), 0.0), 1.0);
    if (scaling == SLED_ROTARY_RAMP) s = 1 - std::fmin(std::fmax((i - first) / std::fmax(last - first, 0.001), 0.0), 1.0);
    frequencies[i] = s == 1 ? f : s == 0 ? f / factor : f * (s + (1 - s) / factor);
  }
  if (amplitude) *amplitude = scaling == SLED_ROTARY_RAMP && factor > 1 ? 0.1 * std::log(factor) + 1 : 1.0;
  return SLED_OK;
}

int sled_rotary(const sled_heads* q, const sled_heads* k, int32_t n_rows, int32_t head_dim, int32_t dtype, const int32_t* positions,
                const double* frequencies, int32_t rot_dim, int32_t pairs, float amplitude, int32_t transpose, void* stream) {
  if (!q || n_rows < 0 || head_dim < 2 || head_dim > 512 || head_dim % 2 || rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim) return SLED_ERR_ARG;
  if ((dtype != SLED_F32 && dtype != SLED_BF16) || (pairs != SLED_ROTARY_PAIRS && pairs != SLED_ROTARY_HALVES)) return SLED_ERR_ARG;
  if (!(std::fabs(amplitude) < INFINITY) || !frequencies || !aligned(frequencies, 8) || !aligned(positions, 4)) return SLED_ERR_ARG;
  if (n_rows > 0 && !positions) return SLED_ERR_ARG;
  int rc = check_heads(q, n_rows, head_dim, dtype);
  if (!rc && k) rc = check_heads(k, n_rows, head_dim, dtype);
  if (rc) return rc;
  const auto rows = [](const sled_heads* h) {
    return RotaryRows{static_cast<const char*>(h->in), static_cast<char*>(h->out), h->in_row, h->in_head, h->out_row, h->out_head, h->n_heads};
  };
  RotaryCall a{};
  a.q = rows(q);
  if (k) a.k = rows(k);
  if (n_rows == 0 || a.q.heads + a.k.heads == 0) return SLED_OK;
  a.n_rows = n_rows;
  a.head_dim = head_dim;
  a.half = rot_dim / 2;
  a.dtype = dtype == SLED_BF16 ? BF16 : F32;
  a.halves = pairs == SLED_ROTARY_HALVES;
  a.positions = positions;
  a.frequencies = frequencies;
  a.amplitude = amplitude;
  a.sign = transpose ? -1.f : 1.f;
  OnDeviceOf device(positions);
  if (device.rc()) return device.rc();
  return done(launch_rotary(a, static_cast<cudaStream_t>(stream)), "sled_rotary");
}

int sled_append_keys(const sled_paged_kv* kv, float* k_scale, float* v_scale, const void* k, int64_t k_stride, const void* v,
                     int64_t v_stride, int32_t rows_dtype, const int32_t* cu_q, int32_t n_rows, int32_t* status, void* stream) {
  int rc = check_cache(kv, true, false, true);
  if (rc) return rc;
  if ((rows_dtype != SLED_F32 && rows_dtype != SLED_BF16) || n_rows < 0 || !cu_q) return SLED_ERR_ARG;
  const bool codes = kv->dtype == SLED_E4M3;
  if (codes ? !k_scale || !v_scale : k_scale || v_scale || kv->dtype != rows_dtype) return SLED_ERR_ARG;
  const uintptr_t a = rows_dtype == SLED_BF16 ? 2 : 4;
  if (!aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned(cu_q, 4) || !aligned(status, 4) || !aligned(k, a) || !aligned(v, a)) return SLED_ERR_ARG;
  if (n_rows > 0 && (!k || !v)) return SLED_ERR_ARG;
  const int64_t row = static_cast<int64_t>(kv->n_kv_heads) * kv->head_dim;
  if (k_stride < row || v_stride < row || k_stride > (1LL << 40) || v_stride > (1LL << 40)) return SLED_ERR_ARG;
  if (n_rows == 0 || kv->n_reqs == 0) return SLED_OK;
  OnDeviceOf device(kv->k);
  if (device.rc()) return device.rc();
  const NewRows rows{static_cast<const char*>(k), static_cast<const char*>(v), k_stride, v_stride, rows_dtype == SLED_BF16 ? BF16 : F32, cu_q, n_rows,
                     k_scale, v_scale};
  return done(launch_append(cache_of(kv, status), rows, static_cast<cudaStream_t>(stream)), "sled_append_keys");
}

int sled_attention_scaled_workspace(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int64_t* bytes) {
  if (check_cache(kv, true, false, true) || kv->dtype != SLED_E4M3 || n_rows < 0 || n_q_heads < 1 || !bytes) return SLED_ERR_ARG;
  *bytes = align256(paged_scaled_workspace(kv->head_dim));
  return SLED_OK;
}

int sled_attention_scaled(const sled_paged_kv* kv, const float* k_scale, const float* v_scale, const void* q, int64_t q_stride,
                          const int32_t* cu_q, const int32_t* parents, int32_t n_rows, int32_t n_q_heads, float scale, void* out,
                          int64_t out_stride, float* lse, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(kv, true, false, true);
  if (!rc && kv->dtype != SLED_E4M3) rc = SLED_ERR_ARG;
  if (!rc) rc = check_rows(kv, q, q_stride, cu_q, n_rows, n_q_heads, scale, out, out_stride);
  if (!rc && (!k_scale || !v_scale || !aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned(parents, 4) || !aligned(lse, 4) || !aligned(status, 4)))
    rc = SLED_ERR_ARG;
  if (!rc) rc = check_workspace(workspace, workspace_bytes, align256(paged_scaled_workspace(kv->head_dim)));
  if (rc) return rc;
  if (n_rows == 0 || kv->n_reqs == 0) return SLED_OK;
  OnDeviceOf device(kv->k);
  if (device.rc()) return device.rc();
  const PagedCache c = cache_of(kv, status);
  const PagedRows r = rows_of(kv, q, q_stride, cu_q, parents, n_rows, n_q_heads, scale, out, out_stride, lse);
  return done(launch_paged_scaled(c, CacheScales{k_scale, v_scale}, r, static_cast<char*>(workspace), static_cast<cudaStream_t>(stream)),
              "sled_attention_scaled");
}

}  // extern "C"
