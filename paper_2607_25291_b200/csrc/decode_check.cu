// One-token attention over a paged cache on CUDA cores: a second opinion for the fast kernel (impl = 1), written from the
// formula alone.  A CTA takes one (request, query head); its eight warps take the tokens in turns, d/32 channels a lane, with a running
// maximum and sum each, and are joined in shared memory.
#include "cache.cuh"

namespace cosa {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ float e4m3_value(uint8_t x) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(x, __NV_E4M3)));
}

template <bool F16>
__global__ void __launch_bounds__(kWarps * 32) decode_check_kernel(DecodeParams p) {
  using H = Half16<F16>;
  using T = typename H::T;
  __shared__ float s_top[kWarps], s_sum[kWarps], s_out[kWarps][kHeadDim];
  chain_next();
  chain_wait();
  if (__syncthreads_or(threadIdx.x == 0 && *p.status != 0)) return;
  const CacheView& c = p.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.y, hq = blockIdx.x, h = hq / p.group, per = c.d / 32;
  const long long len = clamped_len(p.lens[b], c), from = p.window > 0 && len > p.window ? len - p.window : 0;
  const int32_t* list = p.pages ? p.pages + ((long long)b * c.hkv + h) * p.list_stride : nullptr;
  const int entries = list ? min(max(0, p.count[b * c.hkv + h]), p.list_stride) : 0;
  const long long total = list ? (long long)entries << c.page_shift : len;
  const float ks = c.e4m3 ? c.k_scale[h] : 1.f, vs = c.e4m3 ? c.v_scale[h] : 1.f;
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, top = -INFINITY, sum = 0.f;
  for (int i = 0; i < per; ++i) q[i] = H::widen1(static_cast<const T*>(p.q)[b * p.q_request + hq * p.q_head + lane * per + i]);
  for (long long i = warp; i < total; i += kWarps) {
    long long t = i;
    if (list) {
      const int j = list[i >> c.page_shift];
      if (j < 0 || j >= c.table_stride) continue;
      t = ((long long)j << c.page_shift) + (i & (c.page_size - 1));
    }
    if (t < from || t >= len) continue;
    const int page = c.table[(long long)b * c.table_stride + (t >> c.page_shift)];
    const bool there = page >= 0 && page < c.num_pages;      // (a page that is none reads as zeros, as the fast kernel has it)
    const long long at = there ? page * c.page_stride + h * c.head_stride + (t & (c.page_size - 1)) * c.token_stride + lane * per : 0;
    auto value = [&](const void* pool, float scale, int i) {
      if (!there) return 0.f;
      return c.e4m3 ? e4m3_value(static_cast<const uint8_t*>(pool)[at + i]) * scale : H::widen1(static_cast<const T*>(pool)[at + i]);
    };
    float x = 0.f;
    for (int i = 0; i < per; ++i) x += q[i] * value(c.k, ks, i);
    for (int s = 16; s > 0; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    x *= p.scale;
    const float now = fmaxf(top, x), ref = now == -INFINITY ? 0.f : now, keep = expf(top - ref), w = expf(x - ref);
    top = now;
    sum = sum * keep + w;
    for (int i = 0; i < per; ++i) o[i] = o[i] * keep + w * value(c.v, vs, i);
  }
  if (lane == 0) { s_top[warp] = top; s_sum[warp] = sum; }
  for (int i = 0; i < per; ++i) s_out[warp][lane * per + i] = o[i];
  __syncthreads();
  if (warp == 0) {
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_top[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    sum = 0.f;
    for (int w = 0; w < kWarps; ++w) sum += s_sum[w] * expf(s_top[w] - ref);
    for (int i = 0; i < per; ++i) {
      float x = 0.f;
      for (int w = 0; w < kWarps; ++w) x += s_out[w][lane * per + i] * expf(s_top[w] - ref);
      static_cast<T*>(p.out)[b * p.out_request + hq * p.out_head + lane * per + i] = H::narrow1(sum == 0.f ? 0.f : x / sum);
    }
    if (p.lse && lane == 0) p.lse[(long long)b * p.hq + hq] = sum == 0.f ? -INFINITY : ref + logf(sum);
  }
}

}  // namespace

cudaError_t launch_decode_check(const DecodeParams& p, cudaStream_t st) {
  if (p.batch > 65535) return cudaErrorInvalidValue;
  return launch_chained(p.c.f16 ? decode_check_kernel<true> : decode_check_kernel<false>, dim3(p.hq, p.batch), kWarps * 32, 0, st, p);
}

}  // namespace cosa
