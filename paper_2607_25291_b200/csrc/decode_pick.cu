// cosa_decode_select, second part: the K pages of largest rank of every (request, KV head).
//
// A CTA takes a row: maxima of the heads' scores, ranks r[j] = max_g (M[g][j] - max M[g]), the K-th largest of them by a histogram of 2,048 bins and, in its
// bin, by comparing each with each (or, among many, by three rounds of a radix histogram over the bits: 11, 11 and 10), and the kept pages in
// ascending order by a prefix sum.  Bound: the latency of a dozen steps one after the other, and the instructions in them: 2,048 pages of four heads
// take 6.9 us, launch included.  (Clusters of up to eight CTAs for long rows, the ranks sent to the first: 16 requests of 16,384 pages 328 us a call
// against 247, one request of 8,192 pages 24.0 against 22.2.)
#include <algorithm>

#include "cache.cuh"
#include "ptx_sm100.cuh"
#include "warp_mma.cuh"

namespace cosa {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kBins = 2048;
constexpr int kHeadsAtOnce = 4;
constexpr size_t kMostShared = 200 * 1024;

// order-preserving bits of a float (-inf lowest; no NaN)
__device__ __forceinline__ uint32_t rank_bits(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// exclusive prefix sum over the CTA (two sums below 65536 in one word), and the total
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* part, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t in = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, in, o);
    if (lane >= o) in += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = in;
  __syncthreads();
  uint32_t ahead = lane < kWarps ? part[lane] : 0u;
#pragma unroll
  for (int o = 1; o < kWarps; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, ahead, o);
    if (lane >= o) ahead += y;
  }
  *total = __shfl_sync(0xffffffffu, ahead, kWarps - 1);
  const uint32_t before = __shfl_sync(0xffffffffu, ahead, max(warp - 1, 0));
  return (warp ? before : 0u) + in - x;
}
__device__ __forceinline__ void copy_16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
}
// Bins of the ranks r <= 0: 64 for every power of two that |r| can lie between, from 2^-16 to 2^16; what is larger (and the pages kept whatever their
// score) in the last one, what is smaller in the first.  Neighbouring ranks of a few thousand pages then share a bin with a dozen others at most.
constexpr int kFirstBin = (127 - 16) << 6, kBinShift = 17;
__device__ __forceinline__ int bin_of(uint32_t key) {
  return key & 0x80000000u ? kBins - 1 : kBins - 1 - min(max((int)((0x7fffffffu - key) >> kBinShift) - kFirstBin, 0), kBins - 1);
}

// kCopied: this CTA's scores fit shared memory and are copied there in one go
template <bool kCopied>
__global__ void __launch_bounds__(kThreads) decode_pick_kernel(SelectParams p, bool keys_shared) {
  extern __shared__ __align__(16) char smem[];
  __shared__ uint32_t s_part[kWarps];
  __shared__ __align__(16) float s_tops[2][kWarps][kHeadsAtOnce];
  __shared__ int s_digit, s_left, s_same, s_listed;
  const CacheView& c = p.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x, b = row / c.hkv, pitch = score_pitch(c.table_stride);
  // shared: histogram; ranks; scores
  int* hist = reinterpret_cast<int*>(smem);
  uint32_t* keys = reinterpret_cast<uint32_t*>(hist + kBins);
  float* here = reinterpret_cast<float*>(keys + (keys_shared ? pitch : 0));
  if (!keys_shared) keys = reinterpret_cast<uint32_t*>(p.scores + (long long)p.batch * p.hq * pitch) + (long long)row * pitch;
  chain_next();
  // (the lengths were there before the kernel that scores let this one begin)
  const int n = (int)((clamped_len(p.lens[b], c) + c.page_size - 1) >> c.page_shift);
  const int keep = n == 0 ? 0 : (int)min((long long)n, max((long long)max(budget_count_fx(p.budget_fx, n), p.min_pages), (long long)p.keep_first + p.keep_last));
  const int quads = (n + 3) / 4;                                                  // four pages a thread at a time
  const float* m = p.scores + (long long)row * p.group * pitch;
  int m_pitch = pitch;
  *reinterpret_cast<int4*>(hist + tid * 4) = make_int4(0, 0, 0, 0);
  if (tid == 0) s_listed = 0;
  static_assert(kBins == 4 * kThreads);
  chain_wait();
  if constexpr (kCopied) {
    for (int i = tid; i < quads; i += kThreads)
      for (int g = 0; g < p.group; ++g) copy_16(here + (g * quads + i) * 4, m + (long long)g * pitch + i * 4);
    asm volatile("cp.async.wait_all;" ::: "memory");                              // (a thread reads what it has copied itself)
    m = here;
    m_pitch = quads * 4;
  }
  // ---- some heads at a time: their maxima, and with them the ranks
  for (int g0 = 0; g0 < p.group; g0 += kHeadsAtOnce) {
    const float* mg = m + (long long)g0 * m_pitch;
    float top[kHeadsAtOnce];
#pragma unroll
    for (int g = 0; g < kHeadsAtOnce; ++g) top[g] = -INFINITY;
    for (int i = tid; i < quads; i += kThreads) {
      const int there = n - i * 4;                                             // pages of the quad that are there
#pragma unroll
      for (int g = 0; g < kHeadsAtOnce; ++g)
        if (g0 + g < p.group) {
          const float4 x = *reinterpret_cast<const float4*>(mg + (long long)g * m_pitch + i * 4);
          top[g] = fmaxf(top[g], fmaxf(fmaxf(x.x, there > 1 ? x.y : -INFINITY), fmaxf(there > 2 ? x.z : -INFINITY, there > 3 ? x.w : -INFINITY)));
        }
    }
    float (&tops)[kWarps][kHeadsAtOnce] = s_tops[(g0 / kHeadsAtOnce) & 1];
#pragma unroll
    for (int g = 0; g < kHeadsAtOnce; ++g) {
      const float x = ptx::warp_max(top[g]);
      if (lane == 0) tops[warp][g] = x;
    }
    __syncthreads();
    const float4 others = *reinterpret_cast<const float4*>(tops[lane % kWarps]);
    top[0] = ptx::warp_max(others.x); top[1] = ptx::warp_max(others.y); top[2] = ptx::warp_max(others.z); top[3] = ptx::warp_max(others.w);
    // A page that holds the maximum ranks 0 whatever that maximum is (inf - inf would be no number, and be passed over); a head without a score above -inf has
    // none: NaN equals nothing and gives no ranks
#pragma unroll
    for (int g = 0; g < kHeadsAtOnce; ++g)
      if (top[g] == -INFINITY) top[g] = NAN;
    auto rank = [](float x, float top) { return x == top ? 0.f : __fsub_rn(x, top); };
    const bool begin = g0 == 0, end = g0 + kHeadsAtOnce >= p.group;
    float* so_far = reinterpret_cast<float*>(keys);                               // (until they are whole the ranks lie where the keys will)
    for (int i = tid; i < quads; i += kThreads) {
      float4 r = begin ? make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY) : *reinterpret_cast<const float4*>(so_far + i * 4);
#pragma unroll
      for (int g = 0; g < kHeadsAtOnce; ++g)
        if (g0 + g < p.group) {
          const float4 x = *reinterpret_cast<const float4*>(mg + (long long)g * m_pitch + i * 4);
          r.x = fmaxf(r.x, rank(x.x, top[g])); r.y = fmaxf(r.y, rank(x.y, top[g]));
          r.z = fmaxf(r.z, rank(x.z, top[g])); r.w = fmaxf(r.w, rank(x.w, top[g]));
        }
      if (!end) {
        *reinterpret_cast<float4*>(so_far + i * 4) = r;
        continue;
      }
      const float rs[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = i * 4 + e;
        if (j < n) {
          const uint32_t key = j < p.keep_first || j >= n - p.keep_last ? rank_bits(INFINITY) : rank_bits(__fadd_rn(rs[e], 0.f));   // (no negative zeros: equal ranks are equal bits)
          atomicAdd(&hist[bin_of(key)], 1);
          keys[j] = key;
        }
      }
    }
  }
  __syncthreads();

  // ---- the K-th largest: keys from `low` to `high` share its bin, and of those the larger ones, or the first `left` of equal ones, are kept
  int32_t* out = p.out_pages + (long long)row * p.list_stride;
  uint32_t low = 0, high = 0xffffffffu, bound = 0, mask = 0, total;
  int left = keep;                                                                // to be kept of those that agree with `bound` in `mask`
  auto digit = [&](int bins) {                                                    // of the histogram: the bin of the left-th largest
    const int per = bins / kThreads, top = bins - 1 - tid * per;
    int own = 0;
    for (int i = 0; i < per; ++i) own += hist[top - i];
    int above = (int)block_scan((uint32_t)own, s_part, &total);
    if (above < left && above + own >= left)
      for (int i = 0; i < per; ++i) {
        if (above + hist[top - i] >= left) { s_digit = top - i; s_left = left - above; s_same = hist[top - i]; break; }
        above += hist[top - i];
      }
    __syncthreads();
    left = s_left;
  };
  if (keep < n && keep > 0) {
    digit(kBins);
    const int bin = s_digit, same = s_same;
    const uint32_t edge = 0x7fffffffu - ((uint32_t)(kFirstBin + kBins - 1 - bin) << kBinShift);
    if (bin != kBins - 1) high = edge;
    if (bin != 0) low = edge - ((1u << kBinShift) - 1u);
    if (same > left && same <= kThreads) {
      // few in the bin: each finds its place among them by comparison (larger first, then by index), and says in its key whether it is kept
      uint2* listed = reinterpret_cast<uint2*>(hist);
      for (int i = tid; i * 4 < n; i += kThreads)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = i * 4 + e;
          const uint32_t key = j < n ? keys[j] : 0u;
          if (j < n && key >= low && key <= high) listed[atomicAdd(&s_listed, 1)] = make_uint2(key, (uint32_t)j);
        }
      __syncthreads();
      if (tid < same) {
        const uint2 me = listed[tid];
        int ahead = 0;
        for (int i = 0; i < same; ++i) {
          const uint2 x = listed[i];
          ahead += x.x > me.x || (x.x == me.x && x.y < me.y);
        }
        keys[me.y] = ahead < left ? 0xffffffffu : 0u;
      }
      bound = mask = 0xffffffffu;
      left = n;
      __syncthreads();
    } else if (same > left) {
      // many, equal ones perhaps: by the bits of the keys
#pragma unroll 1
      for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bins = round == 2 ? 1024 : 2048;
        __syncthreads();
        for (int i = tid; i < bins; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kThreads) {
          const uint32_t key = keys[j];
          if (key >= low && key <= high && (key & mask) == bound) atomicAdd(&hist[(key >> shift) & (bins - 1)], 1);
        }
        __syncthreads();
        digit(bins);
        bound |= (uint32_t)s_digit << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        if (s_same == left) break;                                                // all that agree so far are kept
      }
    }
  }
  // ---- the list: larger ranks, and of those that agree the first `left`
  int kept_before = 0, same_before = 0;
  for (int j0 = 0; j0 < n; j0 += kThreads * 4) {
    uint32_t own = 0;
    bool over[4], agrees[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + tid * 4 + e;
      const uint32_t key = j < n ? keys[j] : 0u;
      const bool in = j < n && keep > 0 && key >= low && key <= high;
      over[e] = (j < n && keep > 0 && key > high) || (in && (key & mask) > bound);
      agrees[e] = in && (key & mask) == bound;
      own += (over[e] ? 1u << 16 : 0u) + (agrees[e] ? 1u : 0u);
    }
    const uint32_t before = block_scan(own, s_part, &total);
    int larger = kept_before + (int)(before >> 16), same = same_before + (int)(before & 0xffffu);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (over[e] || (agrees[e] && same < left)) out[larger + min(same, left)] = j0 + tid * 4 + e;
      larger += over[e];
      same += agrees[e];
    }
    kept_before += (int)(total >> 16);
    same_before += (int)(total & 0xffffu);
  }
  for (int i = keep + tid; i < p.list_stride; i += kThreads) out[i] = -1;
  if (tid == 0) p.out_count[row] = keep;
}

// How a call is laid out: whether a row's ranks and scores fit shared memory
struct Layout { bool keys_shared, copied; size_t smem; };
Layout layout_of(int group, int table_stride) {
  Layout L{};
  const int pitch = score_pitch(table_stride);
  const size_t fixed = kBins * 4, keys = (size_t)pitch * 4, scores = keys * group;
  L.keys_shared = fixed + keys <= kMostShared;
  L.copied = L.keys_shared && fixed + keys + scores <= kMostShared;
  L.smem = fixed + (L.keys_shared ? keys : 0) + (L.copied ? scores : 0);
  return L;
}

}  // namespace

// scores of every query head and page, and ranks that do not fit shared memory
size_t decode_select_scratch(int batch, int hq, int hkv, int table_stride) {
  return (size_t)batch * ((size_t)hq + (layout_of(hq / hkv, table_stride).keys_shared ? 0 : hkv)) * score_pitch(table_stride) * 4;
}

cudaError_t launch_decode_pick(const SelectParams& p, cudaStream_t st) {
  static SmemLimit limit[2], preferred[2];
  const Layout L = layout_of(p.group, p.c.table_stride);
  auto kernel = L.copied ? decode_pick_kernel<true> : decode_pick_kernel<false>;
  cudaError_t e = L.smem > 40 * 1024 ? raise_smem_limit((const void*)kernel, &limit[L.copied], L.smem) : cudaSuccess;
  if (e == cudaSuccess) e = prefer_shared((const void*)kernel, &preferred[L.copied]);
  if (e != cudaSuccess) return e;
  return launch_chained(kernel, dim3(p.batch * p.c.hkv), kThreads, L.smem, st, p, L.keys_shared);
}

}  // namespace cosa
