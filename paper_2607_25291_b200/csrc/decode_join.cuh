// The last step of cosa_decode_attention: a row whose pieces lie in several CTAs.
#pragma once

#include "cache.cuh"
#include "ptx_sm100.cuh"

namespace cosa {

// Joins the pieces of query head `head` of one (request b, KV head h, chunk ch of query heads), one in each of CTAs `first` to `last`, and writes its
// output: a warp, d / 32 channels a lane.  Piece 1 of the first CTA, piece 0 of the others.  They come from other SMs and are read past L1, eight
// while the eight before are added up: nothing but latency is spent here.
template <bool F16, int D>
__device__ __forceinline__ void join_head(const DecodeParams& p, const float* data, int slot_heads, int per_chunk, int first, int last, int b, int h, int ch, int head) {
  using H = Half16<F16>;
  constexpr int kVec = D / 32, kDeep = 8;
  const int lane = threadIdx.x & 31, size = slot_heads * (D + 4), n = last - first + 1;
  const float* of_head = data + (long long)first * 2 * size + head * D + lane * kVec;
  auto offset = [&](int i) { return (long long)(i == 0 ? 1 : 2 * i) * size; };
  auto load = [&](int i0, float (&x)[kDeep][kVec]) {
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const float* from = of_head + offset(min(i0 + i, n - 1));                   // (past the last: the last again, with no weight)
      if constexpr (kVec == 4) *reinterpret_cast<float4*>(x[i]) = __ldcg(reinterpret_cast<const float4*>(from));
      else *reinterpret_cast<float2*>(x[i]) = __ldcg(reinterpret_cast<const float2*>(from));
    }
  };
  float x[kDeep][kVec], next[kDeep][kVec], most = -INFINITY, sum = 0.f, out[kVec];
  load(0, x);
#pragma unroll
  for (int v = 0; v < kVec; ++v) out[v] = 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += 32) {                                            // by the rule by which the pieces themselves were computed
    const float* mine = data + (long long)first * 2 * size + offset(min(i0 + lane, n - 1)) + slot_heads * D + head;
    const float top = i0 + lane < n ? __ldcg(mine) : -INFINITY, l = i0 + lane < n ? __ldcg(mine + slot_heads) : 0.f;
    float now = fmaxf(most, top);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, o));
    const float ref = now == -INFINITY ? 0.f : now, keep = ptx::ex2_approx(most - ref), weight = ptx::ex2_approx(top - ref);
    most = now;
    float part = weight * l;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    sum = sum * keep + part;
#pragma unroll
    for (int v = 0; v < kVec; ++v) out[v] *= keep;
#pragma unroll 1
    for (int i1 = 0; i1 < 32 && i0 + i1 < n; i1 += kDeep) {
      const int ahead = i0 + i1 + kDeep;
      if (ahead < n) load(ahead, next);
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        const float w = __shfl_sync(0xffffffffu, weight, i1 + i);
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
          out[v] = i0 + i1 + i < n ? fmaf(w, x[i][v], out[v]) : out[v];           // (past the last piece the last comes again; one of no weight may hold no number, and says so)
          x[i][v] = next[i][v];
        }
      }
    }
  }
  const float inv = (p.c.e4m3 ? p.c.v_scale[h] : 1.f) / sum;                       // (a sum of zero: no tokens in effect; one that is no number goes on to the outputs)
  const int hq = h * p.group + ch * per_chunk + head;
  typename H::T* dst = static_cast<typename H::T*>(p.out) + b * p.out_request + (long long)hq * p.out_head + lane * kVec;
#pragma unroll
  for (int v = 0; v < kVec; v += 2) *reinterpret_cast<typename H::T2*>(dst + v) = H::narrow(sum == 0.f ? 0.f : out[v] * inv, sum == 0.f ? 0.f : out[v + 1] * inv);
  if (p.lse && lane == 0) p.lse[(long long)b * p.hq + hq] = sum == 0.f ? -INFINITY : most * 0.6931471805599453f + logf(sum);
}

}  // namespace cosa
