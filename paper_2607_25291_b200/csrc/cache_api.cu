// The C entry points of generation from a paged cache (include/cosa.h): argument checks, defaults, kernel dispatch.
#include <math.h>

#include <nvtx3/nvToolsExt.h>

#include "cache.cuh"

namespace cosa {
namespace {

struct NvtxRange {
  explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
  ~NvtxRange() { nvtxRangePop(); }
};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// (a kernel that meets a misaligned word faults)
template <typename... T>
bool whole_words(const T*... p) { return (((reinterpret_cast<uintptr_t>(p) & (sizeof(T) - 1)) == 0) && ...); }
bool power_of_two(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2_of(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

int check_pages(int page_size, int num_pages, int table_stride) {
  if (!power_of_two(page_size) || page_size < 8 || page_size > 65536 || num_pages < 1 || table_stride < 1) return COSA_ERR_INVALID_ARG;
  if ((long long)num_pages * page_size > 0x7fffffffLL) return COSA_ERR_UNSUPPORTED;   // slots are 32-bit
  if ((long long)table_stride * page_size > 0x40000000LL) return COSA_ERR_UNSUPPORTED;   // and so are lengths, with room to round up
  return COSA_OK;
}

// `pools`: the call touches k and v
int view_of(const cosa_cache* c, bool pools, CacheView* v) {
  if (!c) return COSA_ERR_INVALID_ARG;
  if (c->dtype != COSA_BF16 && c->dtype != COSA_F16) return COSA_ERR_UNSUPPORTED;
  if (c->cache_dtype != c->dtype && c->cache_dtype != COSA_E4M3) return COSA_ERR_UNSUPPORTED;
  if (c->d != 64 && c->d != 128) return COSA_ERR_UNSUPPORTED;
  if (c->hkv < 1) return COSA_ERR_INVALID_ARG;
  int rc = check_pages(c->page_size, c->num_pages, c->table_stride);
  if (rc != COSA_OK) return rc;
  *v = CacheView{};
  v->e4m3 = c->cache_dtype == COSA_E4M3;
  if (pools) {
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return COSA_ERR_INVALID_ARG;
    if (v->e4m3 && (!c->k_scale || !c->v_scale)) return COSA_ERR_INVALID_ARG;
  }
  if (c->k_bounds && !aligned16(c->k_bounds)) return COSA_ERR_INVALID_ARG;
  if (!whole_words(c->page_table, c->k_scale, c->v_scale)) return COSA_ERR_INVALID_ARG;
  v->k = c->k; v->v = c->v; v->bounds = c->k_bounds;
  v->table = c->page_table; v->k_scale = c->k_scale; v->v_scale = c->v_scale;
  v->table_stride = c->table_stride; v->num_pages = c->num_pages;
  v->page_size = c->page_size; v->page_shift = log2_of(c->page_size);
  v->hkv = c->hkv; v->d = c->d; v->f16 = c->dtype == COSA_F16;
  v->token_stride = c->d; v->head_stride = (long long)c->page_size * c->d; v->page_stride = v->head_stride * c->hkv;
  const int64_t* s = c->strides;
  if (s[0] != 0 || s[1] != 0 || s[2] != 0) {
    const int unit = v->e4m3 ? 16 : 8;                       // elements of 16 bytes
    if (s[2] < c->d || s[2] % unit != 0) return COSA_ERR_INVALID_ARG;
    if (c->hkv > 1 && (s[1] < c->d || s[1] % unit != 0)) return COSA_ERR_INVALID_ARG;
    if (c->num_pages > 1 && (s[0] < c->d || s[0] % unit != 0)) return COSA_ERR_INVALID_ARG;
    v->page_stride = c->num_pages > 1 ? s[0] : v->page_stride;
    v->head_stride = c->hkv > 1 ? s[1] : v->head_stride;
    v->token_stride = s[2];
  }
  return COSA_OK;
}

// two element strides from the options; both zero: rows of d, `inner` to the outer index
int strides2(const int64_t* given, int inner, int d, bool outer_moves, long long* outer_out, long long* inner_out) {
  *outer_out = (long long)inner * d;
  *inner_out = d;
  if (given[0] == 0 && given[1] == 0) return COSA_OK;
  if (inner > 1 && (given[1] < d || given[1] % 8 != 0)) return COSA_ERR_INVALID_ARG;
  if (outer_moves && (given[0] < d || given[0] % 8 != 0)) return COSA_ERR_INVALID_ARG;
  *outer_out = given[0];
  *inner_out = given[1];
  return COSA_OK;
}

int scratch_for(const cosa_decode_options& o, size_t need, void** out) {
  *out = nullptr;
  if (need == 0) return COSA_OK;
  if (o.workspace) {
    if (o.workspace_bytes < need || !aligned16(o.workspace)) return COSA_ERR_WORKSPACE;
    *out = o.workspace;
    return COSA_OK;
  }
  return own_scratch(need, out);
}

int check_queries(const CacheView& c, const void* q, int batch, int hq, const int32_t* lens) {
  if (!q || !lens || !c.table || !aligned16(q) || !whole_words(lens)) return COSA_ERR_INVALID_ARG;
  if (batch < 1 || hq < 1 || hq % c.hkv != 0) return COSA_ERR_INVALID_ARG;
  if (batch > 65535 || (long long)batch * hq > 0x7fffffffLL) return COSA_ERR_UNSUPPORTED;
  return COSA_OK;
}

cosa_decode_options options_of(const cosa_decode_options* opt) {
  cosa_decode_options o{};
  if (opt) o = *opt;
  return o;
}

// pages that cosa_decode_select keeps of a request with n of them
int kept_pages(long long budget_fx, const cosa_decode_options& o, int n) {
  long long k = budget_count_fx(budget_fx, n);
  if (o.min_pages > k) k = o.min_pages;
  if ((long long)o.keep_first + o.keep_last > k) k = (long long)o.keep_first + o.keep_last;
  return (int)(k < n ? k : n);
}

}  // namespace

cudaError_t prefer_shared(const void* kernel, SmemLimit* state) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  if (state->bytes[dev].load(std::memory_order_acquire)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (e == cudaSuccess) state->bytes[dev].store(1, std::memory_order_release);
  return e;
}
}  // namespace cosa

using namespace cosa;

extern "C" {

size_t cosa_cache_bytes(void) { return sizeof(cosa_cache); }
size_t cosa_decode_options_bytes(void) { return sizeof(cosa_decode_options); }

int cosa_page_plan(const int32_t* lens, const int32_t* grow, int32_t batch, int32_t page_size, int32_t* page_table, int32_t table_stride,
                   int32_t* free_ring, int32_t num_pages, const int64_t* ring_state, int32_t* out_lens, int64_t* out_ring_state,
                   int32_t* out_starts, int32_t* out_slots, int32_t* out_positions, int32_t* out_requests, int32_t max_tokens, void* stream) {
  NvtxRange range("cosa_page_plan");
  if (!lens || !grow || !page_table || !free_ring || !ring_state || !out_lens || !out_ring_state || !out_starts) return COSA_ERR_INVALID_ARG;
  if (batch < 1 || max_tokens < 0 || (max_tokens > 0 && !out_slots)) return COSA_ERR_INVALID_ARG;
  if (!whole_words(lens, grow, page_table, free_ring, ring_state, out_lens, out_ring_state, out_starts, out_slots, out_positions, out_requests)) return COSA_ERR_INVALID_ARG;
  if (out_lens == lens || out_lens == grow || out_starts == lens || out_starts == grow || out_ring_state == ring_state) return COSA_ERR_INVALID_ARG;
  int rc = check_pages(page_size, num_pages, table_stride);
  if (rc != COSA_OK) return rc;
  if (batch > kMaxPlanRequests) return COSA_ERR_UNSUPPORTED;
  PlanParams p{};
  p.lens = lens; p.grow = grow; p.table = page_table; p.ring = free_ring;
  p.ring_state = reinterpret_cast<const long long*>(ring_state);
  p.out_lens = out_lens; p.out_starts = out_starts; p.out_slots = out_slots; p.out_positions = out_positions; p.out_requests = out_requests;
  p.out_ring_state = reinterpret_cast<long long*>(out_ring_state);
  p.batch = batch; p.page_size = page_size; p.page_shift = log2_of(page_size); p.table_stride = table_stride;
  p.num_pages = num_pages; p.max_tokens = max_tokens;
  cudaError_t e = launch_page_plan(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? COSA_OK : cuda_fail(e, "page plan launch");
}

int cosa_cache_append_ex(const cosa_cache* cache, const void* k_new, const void* v_new, const int32_t* slots, int32_t tokens, void* stream,
                         const cosa_decode_options* opt) {
  NvtxRange range("cosa_cache_append");
  AppendParams p{};
  int rc = view_of(cache, true, &p.c);
  if (rc != COSA_OK) return rc;
  if (tokens < 0) return COSA_ERR_INVALID_ARG;
  if (tokens == 0) return COSA_OK;
  if (!k_new || !v_new || !slots || !aligned16(k_new) || !aligned16(v_new) || !whole_words(slots)) return COSA_ERR_INVALID_ARG;
  const cosa_decode_options o = options_of(opt);
  rc = strides2(o.new_strides, p.c.hkv, p.c.d, tokens > 1, &p.new_token, &p.new_head);
  if (rc != COSA_OK) return rc;
  p.k_new = k_new; p.v_new = v_new; p.slots = slots; p.tokens = tokens;
  cudaError_t e = launch_cache_append(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? COSA_OK : cuda_fail(e, "append launch");
}

int cosa_cache_append(const cosa_cache* cache, const void* k_new, const void* v_new, const int32_t* slots, int32_t tokens, void* stream) {
  return cosa_cache_append_ex(cache, k_new, v_new, slots, tokens, stream, nullptr);
}

int cosa_decode_select_ex(const cosa_cache* cache, const void* q, int32_t batch, int32_t hq, const int32_t* lens, float budget,
                          int32_t* out_pages, int32_t* out_count, int32_t list_stride, void* stream, const cosa_decode_options* opt) {
  NvtxRange range("cosa_decode_select");
  SelectParams p{};
  int rc = view_of(cache, false, &p.c);
  if (rc == COSA_OK) rc = check_queries(p.c, q, batch, hq, lens);
  if (rc != COSA_OK) return rc;
  if (!p.c.bounds || !out_pages || !out_count || !whole_words(out_pages, out_count)) return COSA_ERR_INVALID_ARG;
  if (!(budget > 0.f) || budget > 1.f) return COSA_ERR_INVALID_ARG;
  const cosa_decode_options o = options_of(opt);
  if (o.min_pages < 0 || o.keep_first < 0 || o.keep_last < 0) return COSA_ERR_INVALID_ARG;
  p.budget_fx = budget_to_fx(budget);
  if (list_stride < kept_pages(p.budget_fx, o, p.c.table_stride)) return COSA_ERR_INVALID_ARG;
  if ((long long)p.c.table_stride * hq > 0x7fffffffLL) return COSA_ERR_UNSUPPORTED;   // a request's pages and heads are counted in 32 bits
  rc = strides2(o.q_strides, hq, p.c.d, batch > 1, &p.q_request, &p.q_head);
  if (rc != COSA_OK) return rc;
  void* ws = nullptr;
  rc = scratch_for(o, decode_select_scratch(batch, hq, p.c.hkv, p.c.table_stride), &ws);
  if (rc != COSA_OK) return rc;
  p.q = q; p.lens = lens; p.out_pages = out_pages; p.out_count = out_count;
  p.batch = batch; p.hq = hq; p.group = hq / p.c.hkv; p.list_stride = list_stride;
  p.min_pages = o.min_pages; p.keep_first = o.keep_first; p.keep_last = o.keep_last;
  p.scores = static_cast<float*>(ws);
  cudaError_t e = launch_decode_select(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? COSA_OK : cuda_fail(e, "page selection launch");
}

int cosa_decode_select(const cosa_cache* cache, const void* q, int32_t batch, int32_t hq, const int32_t* lens, float budget,
                       int32_t* out_pages, int32_t* out_count, int32_t list_stride, void* stream) {
  return cosa_decode_select_ex(cache, q, batch, hq, lens, budget, out_pages, out_count, list_stride, stream, nullptr);
}

int cosa_decode_attention_ex(const cosa_cache* cache, const void* q, int32_t batch, int32_t hq, const int32_t* lens, const int32_t* pages,
                             const int32_t* count, int32_t list_stride, void* out, float* out_lse, void* stream,
                             const cosa_decode_options* opt) {
  NvtxRange range("cosa_decode_attention");
  DecodeParams p{};
  int rc = view_of(cache, true, &p.c);
  if (rc == COSA_OK) rc = check_queries(p.c, q, batch, hq, lens);
  if (rc != COSA_OK) return rc;
  if (!out || !aligned16(out) || (pages && (!count || list_stride < 1)) || !whole_words(pages, count, out_lse)) return COSA_ERR_INVALID_ARG;
  const cosa_decode_options o = options_of(opt);
  if (o.window < 0 || o.ctas < 0 || !(o.softmax_scale >= 0.f)) return COSA_ERR_INVALID_ARG;
  if (o.impl != 0 && o.impl != 1) return COSA_ERR_UNSUPPORTED;
  rc = strides2(o.q_strides, hq, p.c.d, batch > 1, &p.q_request, &p.q_head);
  if (rc == COSA_OK) rc = strides2(o.out_strides, hq, p.c.d, batch > 1, &p.out_request, &p.out_head);
  if (rc != COSA_OK) return rc;
  p.q = q; p.lens = lens; p.pages = pages; p.count = count; p.out = out; p.lse = out_lse;
  p.batch = batch; p.hq = hq; p.group = hq / p.c.hkv; p.list_stride = list_stride; p.window = o.window; p.ctas = o.ctas;
  p.scale = o.softmax_scale > 0.f ? o.softmax_scale : (float)(1.0 / sqrt((double)p.c.d));
  p.wait_budget = o.wait_cycles > 0 ? (long long)o.wait_cycles : (1LL << 31);
  // boxes of a list, at least 8 tokens each, are counted in 32 bits
  if (pages && ((long long)list_stride << (p.c.page_shift - 3)) > 0x7fffffffLL) return COSA_ERR_UNSUPPORTED;
  // tiles of a request or list, at least 16 tokens each, are counted in 32 bits over its KV heads and chunks of query heads
  const long long longest = (long long)(pages && list_stride > p.c.table_stride ? list_stride : p.c.table_stride) << p.c.page_shift;
  if ((longest + 15) / 16 * ((hq + 7) / 8 + p.c.hkv) > 0x7fffffffLL) return COSA_ERR_UNSUPPORTED;
  p.status = device_status_word();
  if (!p.status) return cuda_fail(cudaGetLastError(), "device status word");
  cudaError_t e;
  if (o.impl == 1) {
    e = launch_decode_check(p, static_cast<cudaStream_t>(stream));
  } else {
    void* ws = nullptr;
    rc = scratch_for(o, decode_attention_scratch(p.group, p.c.d), &ws);
    if (rc != COSA_OK) return rc;
    p.partials = static_cast<float*>(ws);
    p.counters = o.workspace || device_sm_count() > kDecodeCounters ? nullptr : decode_counters();
    e = launch_decode_attention(p, static_cast<cudaStream_t>(stream));
  }
  return e == cudaSuccess ? COSA_OK : cuda_fail(e, "decode attention launch");
}

int cosa_decode_attention(const cosa_cache* cache, const void* q, int32_t batch, int32_t hq, const int32_t* lens, const int32_t* pages,
                          const int32_t* count, int32_t list_stride, void* out, float* out_lse, void* stream) {
  return cosa_decode_attention_ex(cache, q, batch, hq, lens, pages, count, list_stride, out, out_lse, stream, nullptr);
}

size_t cosa_decode_workspace_bytes(int op, const cosa_cache* cache, int32_t batch, int32_t hq, const cosa_decode_options* opt) {
  const bool check = opt && opt->impl == 1;
  CacheView c;
  if (view_of(cache, false, &c) != COSA_OK || batch < 1 || hq < 1 || hq % c.hkv != 0) return 0;
  const size_t select = op == 1 ? 0 : decode_select_scratch(batch, hq, c.hkv, c.table_stride);
  const size_t attention = op == 0 || check ? 0 : decode_attention_scratch(hq / c.hkv, c.d);
  return select > attention ? select : attention;
}

}  // extern "C"
