// cosa_page_plan: pages and slots of a step from the lengths of its requests.
//
// Three prefix sums over the requests decide everything: of the tokens asked for (where a request's tokens begin), of the pages
// needed (who is served, and which free pages go to whom), of the pages given back (where they go behind the free ones).  Every CTA
// takes all three by itself -- 8 bytes a request, from L2 -- and then its share of the tokens and pages, each of which finds its
// request by bisection in shared memory.  No CTA waits for another, and nothing that one writes is read by another: new pages come
// from the ring, old ones from entries of the table that the call leaves alone, and the ring has room for what is given back
// behind what is handed out (pages are either free or held).
#include <algorithm>

#include "cache.cuh"

namespace cosa {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kTokensPerCta = 4 * kThreads;   // four tokens a thread
constexpr int kEnded = -2, kDoesNotFit = -1;

__device__ __forceinline__ long long warp_inclusive(long long x) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// exclusive prefix sum over the threads of the CTA, and the total; `part`: a word a warp, of its own for every sum
__device__ __forceinline__ long long block_scan(long long x, long long* part, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long in = warp_inclusive(x);
  if (lane == 31) part[warp] = in;
  __syncthreads();
  const long long up_to = warp_inclusive(lane < kWarps ? part[lane] : 0);
  *total = __shfl_sync(0xffffffffu, up_to, kWarps - 1);
  const long long before = __shfl_sync(0xffffffffu, up_to, max(warp - 1, 0));
  return (warp ? before : 0) + in - x;
}

__device__ __forceinline__ int clip(long long x) { return x > 0x7fffffffLL ? 0x7fffffff : (int)x; }

// first request whose inclusive sum exceeds x (x below the last sum)
__device__ __forceinline__ int find(const int* ends, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

__global__ void __launch_bounds__(kThreads) page_plan_kernel(PlanParams p, bool quads) {
  extern __shared__ int smem[];
  __shared__ long long parts[3][kWarps], s_head, s_tail;
  __shared__ int s_first, s_last, s_free, s_used[kWarps];
  int* token_end = smem;                     // [batch] inclusive sums: tokens asked for,
  int* page_end = token_end + p.batch;       // pages needed by requests that fit,
  int* back_end = page_end + p.batch;        // pages given back
  int* held_len = back_end + p.batch;        // tokens held, or -1 - tokens of a request that is not served
  chain_next();
  chain_wait();
  const int tid = threadIdx.x, per = (p.batch + kThreads - 1) / kThreads, b0 = min(p.batch, tid * per), b1 = min(p.batch, b0 + per);
  auto pages_of = [&](long long tokens) { return (tokens + p.page_size - 1) >> p.page_shift; };
  if (tid == kThreads - 1) {                 // (the last warp has the fewest requests)
    const long long head = p.ring_state[0], tail = p.ring_state[1];
    s_head = head;
    s_tail = tail;
    s_free = (int)max(0LL, min((long long)p.num_pages, tail - head));
    s_first = (int)(((head % p.num_pages) + p.num_pages) % p.num_pages);
    s_last = (int)(((tail % p.num_pages) + p.num_pages) % p.num_pages);
  }
  long long asked = 0, tokens;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) {
    const int len = max(0, p.lens[b]), grow = p.grow[b];
    held_len[b] = len;
    page_end[b] = grow;
    asked += max(0, grow);
  }
  long long end = block_scan(asked, parts[0], &tokens), need = 0, back = 0, needed, backs;
  for (int b = b0; b < b1; ++b) {
    const int len = held_len[b], grow = page_end[b];
    end += max(0, grow);
    token_end[b] = clip(end);
    const long long held = pages_of(len), then = pages_of((long long)len + max(0, grow));
    const bool fits = then <= p.table_stride && end <= p.max_tokens;
    if (grow < 0) back += min((long long)p.table_stride, held);
    else if (fits) need += then - held;
    page_end[b] = grow < 0 ? kEnded : (fits ? (int)(then - held) : kDoesNotFit);
  }
  long long need_end = block_scan(need, parts[1], &needed), back_sum = block_scan(back, parts[2], &backs);
  int used = 0;
  for (int b = b0; b < b1; ++b) {
    const int mine = page_end[b], len = held_len[b], asked_here = token_end[b] - (b > b0 ? token_end[b - 1] : clip(end - asked));
    if (mine > 0) need_end += mine;
    const bool served = mine == 0 || (mine > 0 && need_end <= s_free);
    if (served && mine > 0) used = (int)need_end;
    page_end[b] = clip(need_end);
    if (mine == kEnded) back_sum += min((long long)p.table_stride, pages_of(len));
    back_end[b] = clip(back_sum);
    if (!served) held_len[b] = -1 - len;
    if (blockIdx.x == 0) {
      p.out_lens[b] = mine == kEnded ? 0 : (served ? len + asked_here : len);
      p.out_starts[b + 1] = token_end[b];
    }
  }
  // pages handed out: the largest sum among the requests served (sums grow along the requests)
  used = __reduce_max_sync(0xffffffffu, used);
  if ((tid & 31) == 0) s_used[tid >> 5] = used;
  __syncthreads();
  used = __reduce_max_sync(0xffffffffu, s_used[tid & (kWarps - 1)]);
  if (blockIdx.x == 0 && tid == 0) {
    p.out_starts[0] = 0;
    p.out_ring_state[0] = s_head + used;
    p.out_ring_state[1] = s_tail + backs;
  }
  const int first = s_first, last = s_last;
  auto ring_at = [&](int from, int i) {
    const long long at = (long long)from + i;
    return (int)(at >= p.num_pages ? at - p.num_pages : at);
  };
  const int stride = gridDim.x * kThreads, me = blockIdx.x * kThreads + tid;
  for (int e = me; e < used; e += stride) {
    const int b = find(page_end, p.batch, e), base = b ? page_end[b - 1] : 0;
    p.table[(long long)b * p.table_stride + (int)pages_of(held_len[b]) + (e - base)] = p.ring[ring_at(first, e)];
  }
  for (int e = me; e < (int)min(backs, (long long)p.num_pages); e += stride) {
    const int b = find(back_end, p.batch, e), base = b ? back_end[b - 1] : 0;
    p.ring[ring_at(last, e)] = p.table[(long long)b * p.table_stride + (e - base)];
  }
  // four tokens a thread: their requests lie side by side, and most of them in one page
  for (long long t0 = 4LL * me; t0 < p.max_tokens; t0 += 4LL * stride) {
    int slot[4], pos[4], req[4], b = t0 < tokens ? find(token_end, p.batch, (int)t0) : 0, page = -1, page_at = -1, page_req = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long t = t0 + i;
      slot[i] = pos[i] = req[i] = -1;
      if (t >= tokens || t >= p.max_tokens) continue;
      while (t >= token_end[b]) ++b;         // (ends: the last sum exceeds t)
      req[i] = b;
      const int len = held_len[b];
      if (len < 0) continue;
      pos[i] = len + (int)t - (b ? token_end[b - 1] : 0);
      const int at = pos[i] >> p.page_shift;
      if (at != page_at || b != page_req) {
        const int held = (int)pages_of(len);
        page = at < held ? p.table[(long long)b * p.table_stride + at] : p.ring[ring_at(first, (b ? page_end[b - 1] : 0) + at - held)];
        page_at = at;
        page_req = b;
      }
      slot[i] = (int)(((long long)page << p.page_shift) + (pos[i] & (p.page_size - 1)));
    }
    if (quads && t0 + 4 <= p.max_tokens) {
      *reinterpret_cast<int4*>(p.out_slots + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      if (p.out_positions) *reinterpret_cast<int4*>(p.out_positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      if (p.out_requests) *reinterpret_cast<int4*>(p.out_requests + t0) = make_int4(req[0], req[1], req[2], req[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (t0 + i >= p.max_tokens) continue;
        p.out_slots[t0 + i] = slot[i];
        if (p.out_positions) p.out_positions[t0 + i] = pos[i];
        if (p.out_requests) p.out_requests[t0 + i] = req[i];
      }
    }
  }
}

SmemLimit g_limit;
}  // namespace

cudaError_t launch_page_plan(const PlanParams& p, cudaStream_t st) {
  const size_t smem = (size_t)p.batch * 16;
  // (48 KB without asking are for this and the kernel's fixed half KB together)
  cudaError_t e = smem > 40 * 1024 ? raise_smem_limit((const void*)page_plan_kernel, &g_limit, kMaxPlanRequests * 16) : cudaSuccess;
  if (e != cudaSuccess) return e;
  const int grid = std::max(1, std::min(device_sm_count(), (p.max_tokens + kTokensPerCta - 1) / kTokensPerCta));
  const auto at16 = [](const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
  return launch_chained(page_plan_kernel, dim3(grid), kThreads, smem, st, p, at16(p.out_slots) && at16(p.out_positions) && at16(p.out_requests));
}

}  // namespace cosa
