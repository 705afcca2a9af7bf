// cosa_cache_append: a step's keys and values into the pages, with the pages' bounds.
//
// A warp takes one KV head of a few tokens: eight channels (16 bytes) a lane, so that d/8 lanes hold a row and a warp two rows (four of
// 64 channels).  Without bounds the tokens are independent.  With bounds the unit is a run: consecutive slots inside one
// page.  The warp in whose share a run begins writes all of it and folds it into the page's minima and maxima, so
// that no two warps touch one page's bounds and no atomics are needed.  That wants pages that are many: 32,768 tokens of 8 heads take 46.6 us in pages of 64, 54 in pages
// of 256, but 136 in pages of 1,024 and 379 in pages of 4,096, whose few warps have long runs.
//
// Bound: memory.  32,767 tokens of 8 heads of 128 channels: 46.0 us with bounds (5.8 TB/s, 91 % of the copy rate), 43.2 without (96 %).
#include <algorithm>

#include "cache.cuh"
#include "ptx_sm100.cuh"

namespace cosa {
namespace {

constexpr int kThreads = 128;
// Rows of a lane in flight together, and CTAs an SM.  Runs are few and long (32,767 tokens of prompts in 64-token pages: 49.7 us with four, 47.1 with eight and
// 45.9 in CTAs of 128 threads; into e4m3 44.6 with four, 41.3 with eight); tokens by themselves are many warps with little to do (10,015 tokens into e4m3: 13.7 us with
// four and six CTAs, 13.1 with two and eight; 1,000 tokens 5.2 and 4.3).  Warps that stay, with a batch on its way while one is written, were slower by up to a quarter
template <bool kBounds> constexpr int kInFlight = kBounds ? 8 : 2;
template <bool kBounds> constexpr int kCtasPerSm = kBounds ? 4 : 8;

// Quotients by a scale common to many numbers, two at a time: q = x r, q + (x - q s) r with r = 1/s rounded to nearest is x/s rounded to nearest
// (P. Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990, theorem on division), as long as nothing under- or
// overflows on the way; scales for which that could be are divided by.  What is lost where the quotient itself is below float32's normal
// range rounds to zero in e4m3 all the same.
struct Scale {
  float s, r;
  bool plain;
};
__device__ __forceinline__ Scale scale_of(const float* s) {
  const float x = *s;
  return Scale{x, __frcp_rn(x), !(fabsf(x) > 0x1p-60f && fabsf(x) < 0x1p60f)};
}
// eight numbers; what could overflow is divided as well
template <bool F16>
__device__ __forceinline__ uint2 to_e4m3(uint4 x, const Scale& by) {
  using H = Half16<F16>;
  using T2 = typename H::T2;
  const T2* h = reinterpret_cast<const T2*>(&x);
  const uint32_t limit = F16 ? 0x7bff7bffu : 0x5d805d80u;                         // the largest f16; 2^60
  const T2 most = __hmax2(__hmax2(__habs2(h[0]), __habs2(h[1])), __hmax2(__habs2(h[2]), __habs2(h[3])));
  const bool slow = by.plain || !__hble2(most, *reinterpret_cast<const T2*>(&limit));
  if (slow) {
    // (words move up, so that none is found by an index: with arrays the other way went through local memory too, 16.2 us instead of 13.1 at 10,015 tokens)
    unsigned long long y = 0;
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
      const float2 w = H::widen(*reinterpret_cast<const T2*>(&x.x));
      const unsigned long long z = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(w.x, by.s), __fdiv_rn(w.y, by.s)), __NV_SATFINITE, __NV_E4M3);   // (beyond +-448: +-448)
      y = y >> 16 | z << 48;
      x.x = x.y; x.y = x.z; x.z = x.w;
    }
    return make_uint2((uint32_t)y, (uint32_t)(y >> 32));
  }
  const unsigned long long r = ptx::pack_f32x2(by.r, by.r), s = ptx::pack_f32x2(-by.s, -by.s);
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 w = H::widen(h[i]);
    const unsigned long long a = ptx::pack_f32x2(w.x, w.y), q = ptx::mul_f32x2(a, r);
    float2 z;
    ptx::unpack_f32x2(ptx::fma_f32x2(ptx::fma_f32x2(q, s, a), r, q), z.x, z.y);
    y[i] = __nv_cvt_float2_to_fp8x2(z, __NV_SATFINITE, __NV_E4M3);
  }
  return make_uint2(y[0] | (y[1] << 16), y[2] | (y[3] << 16));
}

template <bool F16, bool E4M3>
__device__ __forceinline__ void store_row(char* at, uint4 x, const Scale& scale) {
  if constexpr (E4M3) *reinterpret_cast<uint2*>(at) = to_e4m3<F16>(x, scale);
  else *reinterpret_cast<uint4*>(at) = x;
}

template <bool F16>
__device__ __forceinline__ void fold(uint4& low, uint4& high, uint4 x) {
  using T2 = typename Half16<F16>::T2;
  T2 *l = reinterpret_cast<T2*>(&low), *h = reinterpret_cast<T2*>(&high);
  const T2* v = reinterpret_cast<const T2*>(&x);
#pragma unroll
  for (int i = 0; i < 4; ++i) { l[i] = __hmin2(l[i], v[i]); h[i] = __hmax2(h[i], v[i]); }
}

// kBounds: with the pages' minima and maxima
template <bool F16, bool E4M3, bool kBounds>
__global__ void __launch_bounds__(kThreads, kCtasPerSm<kBounds>) cache_append_kernel(AppendParams p, int share) {
  using T = typename Half16<F16>::T;
  constexpr int kDeep = kInFlight<kBounds>;
  chain_next();
  chain_wait();
  const CacheView& c = p.c;
  const int lane = threadIdx.x & 31, per_row = c.d / 8, rows = 32 / per_row, sub = lane / per_row, chunk = lane % per_row;
  const long long w = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int h = (int)(w % c.hkv);
  const long long t0 = w / c.hkv * share;
  if (t0 >= p.tokens) return;
  const int t1 = (int)min((long long)p.tokens, t0 + share);
  Scale ks{}, vs{};
  if constexpr (E4M3) { ks = scale_of(c.k_scale + h); vs = scale_of(c.v_scale + h); }
  // (addresses: all that is the same for a warp's rows once, and factors without a sign)
  constexpr unsigned long long kElement = E4M3 ? 1 : 2;
  const long long new_at = h * p.new_head + chunk * 8, pool_at = (h * c.head_stride + chunk * 8) * (long long)kElement;
  const char* kn = reinterpret_cast<const char*>(static_cast<const T*>(p.k_new) + new_at);
  const char* vn = reinterpret_cast<const char*>(static_cast<const T*>(p.v_new) + new_at);
  char *kc = static_cast<char*>(c.k) + pool_at, *vc = static_cast<char*>(c.v) + pool_at;
  const unsigned space = (unsigned)min((long long)c.num_pages << c.page_shift, 0x7fffffffLL + 1), in_page = c.page_size - 1;   // (as a number without a sign a slot below zero lies past it)
  const unsigned long long new_token = (unsigned long long)p.new_token * 2, page_bytes = c.page_stride * kElement, token_bytes = c.token_stride * kElement;
  auto load = [&](const char* x, unsigned t) { return *reinterpret_cast<const uint4*>(x + t * new_token); };
  auto row_at = [&](unsigned slot) { return (slot >> c.page_shift) * page_bytes + (slot & in_page) * token_bytes; };
  if constexpr (!kBounds) {
    for (int t = (int)t0 + sub; t < t1; t += rows * kDeep) {
      int slot[kDeep];
      uint4 k[kDeep], v[kDeep];
#pragma unroll
      for (int i = 0; i < kDeep; ++i) slot[i] = t + i * rows < t1 ? p.slots[t + i * rows] : -1;
#pragma unroll
      for (int i = 0; i < kDeep; ++i)
        if (t + i * rows < t1) { k[i] = load(kn, t + i * rows); v[i] = load(vn, t + i * rows); }
#pragma unroll
      for (int i = 0; i < kDeep; ++i)
        if ((unsigned)slot[i] < space) {
          const unsigned long long at = row_at(slot[i]);
          store_row<F16, E4M3>(kc + at, k[i], ks);
          store_row<F16, E4M3>(vc + at, v[i], vs);
        }
    }
  } else {
    // a run begins where the slot is not the one after its predecessor's, or begins a page
    auto begins = [&](int t) {
      if (t >= t1) return false;
      const int slot = p.slots[t];
      if ((unsigned)slot >= space) return false;
      return t == 0 || (slot & (c.page_size - 1)) == 0 || p.slots[t - 1] != slot - 1;
    };
    for (int t = (int)t0; t < t1;) {
      const uint32_t found = __ballot_sync(0xffffffffu, begins(t + lane));
      if (!found) { t += 32; continue; }
      t += __ffs(found) - 1;
      const int first = p.slots[t], most = min(p.tokens - t, c.page_size - (first & (c.page_size - 1)));
      int len = 1;
      while (len < most) {        // how far the run goes
        const int i = len + lane;
        const uint32_t off = __ballot_sync(0xffffffffu, i >= most || p.slots[t + i] != first + i);
        if (off) { len += __ffs(off) - 1; break; }
        len += 32;
      }
      T* bounds = static_cast<T*>(c.bounds) + ((long long)(first >> c.page_shift) * c.hkv + h) * 2 * c.d + chunk * 8;
      uint4 low, high;
      if ((first & (c.page_size - 1)) == 0) {
        const uint32_t inf = F16 ? 0x7c007c00u : 0x7f807f80u;
        low = make_uint4(inf, inf, inf, inf);
        high = make_uint4(inf | 0x80008000u, inf | 0x80008000u, inf | 0x80008000u, inf | 0x80008000u);
      } else {
        low = *reinterpret_cast<const uint4*>(bounds);
        high = *reinterpret_cast<const uint4*>(bounds + c.d);
      }
      for (int i0 = sub; i0 < len; i0 += rows * kDeep) {
        uint4 k[kDeep], v[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
          if (i0 + i * rows < len) { k[i] = load(kn, t + i0 + i * rows); v[i] = load(vn, t + i0 + i * rows); }
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
          if (i0 + i * rows < len) {
            fold<F16>(low, high, k[i]);
            const unsigned long long at = row_at(first + i0 + i * rows);
            store_row<F16, E4M3>(kc + at, k[i], ks);
            store_row<F16, E4M3>(vc + at, v[i], vs);
          }
      }
      for (int o = per_row; o < 32; o <<= 1) {
        uint4 x, y;
        x.x = __shfl_xor_sync(0xffffffffu, low.x, o); x.y = __shfl_xor_sync(0xffffffffu, low.y, o);
        x.z = __shfl_xor_sync(0xffffffffu, low.z, o); x.w = __shfl_xor_sync(0xffffffffu, low.w, o);
        y.x = __shfl_xor_sync(0xffffffffu, high.x, o); y.y = __shfl_xor_sync(0xffffffffu, high.y, o);
        y.z = __shfl_xor_sync(0xffffffffu, high.z, o); y.w = __shfl_xor_sync(0xffffffffu, high.w, o);
        uint4 unused = x;
        fold<F16>(low, unused, x);
        unused = y;
        fold<F16>(unused, high, y);
      }
      if (sub == 0) {
        *reinterpret_cast<uint4*>(bounds) = low;
        *reinterpret_cast<uint4*>(bounds + c.d) = high;
      }
      t += len;
    }
  }
}

}  // namespace

cudaError_t launch_cache_append(const AppendParams& p, cudaStream_t st) {
  // tokens a warp: one where there are few, so that they are written side by side; two batches, or a page of 64, where there are many
  const int most = p.c.bounds ? 64 : 4 * 32 / (p.c.d / 8);
  const int share = (int)std::min<long long>(most, std::max<long long>(1, (long long)p.tokens * p.c.hkv / 8192));
  const long long warps = ((long long)p.tokens + share - 1) / share * p.c.hkv, ctas = (warps + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  auto kernel = p.c.f16 ? (p.c.e4m3 ? (p.c.bounds ? cache_append_kernel<true, true, true> : cache_append_kernel<true, true, false>)
                                    : (p.c.bounds ? cache_append_kernel<true, false, true> : cache_append_kernel<true, false, false>))
                        : (p.c.e4m3 ? (p.c.bounds ? cache_append_kernel<false, true, true> : cache_append_kernel<false, true, false>)
                                    : (p.c.bounds ? cache_append_kernel<false, false, true> : cache_append_kernel<false, false, false>));
  return launch_chained(kernel, dim3((unsigned)ctas), kThreads, 0, st, p, share);
}

}  // namespace cosa
