// cosa_decode_select, first part: scores of pages.
//
// M[g][j] = sum_c max(q_c low_jc, q_c high_jc) for the query heads of a group and every page (the criterion of J. Tang et al., "Quest: query-aware
// sparsity for efficient long-context LLM inference", 2024).  With q split into its positive and its
// negative part the maximum is one multiplication and one addition of a product with zero, exact in float32 (products of two 16-bit
// numbers have at most 22 bits), two channels an instruction; the tree of additions that follows is part of the operator's definition.
// d/8 lanes take a page (eight channels of minima and maxima each).
//
// Bound: memory (4 d bytes a page and KV head); the instructions, 64 a page for four heads, take the SMs some three quarters of that time.
// All rows -- (request, KV head, four heads) -- lie one behind the other and every warp takes an equal run of pages, copied asynchronously into a
// ring of its own.  (One cluster of CTAs a row, which kept the sums in shared memory and picked the pages as well: 24 contexts of 300 to 64K
// tokens in 16-token pages 52 us.)  What picks the pages is decode_pick.cu.
#include <algorithm>

#include "cache.cuh"
#include "ptx_sm100.cuh"

namespace cosa {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kAtOnce = 4;                // heads worked on together
constexpr int kStages = 2, kStageBytes = 4096;                                   // bounds in flight, by warp

__device__ __forceinline__ void copy_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kOpen> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kOpen) : "memory"); }

// A stage's pages by the definition as it stands, for bounds that are not finite: heads one after the other.  `m`: the first page's sum of the
// first of the heads.
template <bool F16, int D>
__device__ __forceinline__ void score_as_defined(uint32_t stage, const typename Half16<F16>::T* q, long long q_head, int heads, float* m, int m_stride, int pages) {
  using H = Half16<F16>;
  constexpr int kLanes = D / 8, kPages = 32 / kLanes, kPageBytes = 4 * D;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, chunk = lane % kLanes;
#pragma unroll 1
  for (int j = sub; j < kStageBytes / kPageBytes; j += kPages) {
    const uint32_t at = stage + j * kPageBytes + chunk * 16;
    const uint4 low = ptx::ld_shared_128(at), high = ptx::ld_shared_128(at + 2 * D);
#pragma unroll 1
    for (int g = 0; g < min(heads, kAtOnce); ++g) {
      const uint4 w = *reinterpret_cast<const uint4*>(q + g * q_head);
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 a = H::widen(reinterpret_cast<const typename H::T2*>(&w)[i]), l = H::widen(reinterpret_cast<const typename H::T2*>(&low)[i]),
                     h = H::widen(reinterpret_cast<const typename H::T2*>(&high)[i]);
        x[2 * i] = fmaxf(__fmul_rn(a.x, l.x), __fmul_rn(a.x, h.x));
        x[2 * i + 1] = fmaxf(__fmul_rn(a.y, l.y), __fmul_rn(a.y, h.y));
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < o; ++i) x[i] = __fadd_rn(x[i], x[i + o]);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) x[0] = __fadd_rn(x[0], __shfl_xor_sync(0xffffffffu, x[0], o));
      if (chunk == 0 && j < pages) m[(long long)g * m_stride + j] = x[0];
    }
  }
}

template <bool F16, int D>
__global__ void __launch_bounds__(kThreads, 2) decode_select_kernel(SelectParams p, int chunks, bool many) {
  using H = Half16<F16>;
  using T = typename H::T;
  constexpr int kLanes = D / 8, kPages = 32 / kLanes;                             // lanes a page, pages a warp side by side
  constexpr int kPageBytes = 4 * D, kStagePages = kStageBytes / kPageBytes, kSteps = kStagePages / kPages;
  extern __shared__ __align__(16) char smem[];
  __shared__ DivisionRoom<kThreads> room;
  const CacheView& c = p.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / kLanes, chunk = lane % kLanes;
  const int per_unit = c.hkv * chunks, pitch = score_pitch(c.table_stride);
  chain_wait();
  chain_next();                                                                   // (only now: the kernel that picks reads the lengths before it waits)
  auto pages_of = [&](int b) { return (int)((clamped_len(p.lens[b], c) + c.page_size - 1) >> c.page_shift); };
  auto fetch_unit = [&](int b) { return make_int2(pages_of(b), 0); };
  auto unit_pages = [&](int2 x) { return UnitSize{x.x * per_unit, x.x, 0}; };
  // (a few pages a warp while there are warps: the way to the first page is what a short call waits for)
  const int me = blockIdx.x * kWarps + warp;
  Division div{};
  RunStart run;
  if (!many) run = divide_few(p.batch, fetch_unit, unit_pages, (int)gridDim.x * kWarps, kPages, me, div);
  else run = divide_many<kThreads>(p.batch, fetch_unit, unit_pages, (int)gridDim.x * kWarps, kPages, me, div, &room);
  int count = run_length(div, me);
  if (count == 0) return;
  int b = run.unit, n = run.size.a;
  int sub_row = run.in_unit <= 0x7fffffffLL ? (int)run.in_unit / n : (int)(run.in_unit / n), j = (int)(run.in_unit - (long long)sub_row * n);   // row of the request, first page
  const uint32_t ring = ptx::smem_u32(smem) + warp * kStages * kStageBytes;

  const uint32_t step = (uint32_t)c.hkv * kPageBytes;                             // bytes from a page to the next
  auto look_up = [&](const int32_t* table, int at, int pages) { return at < pages ? (uint32_t)min(max(table[at], 0), c.num_pages - 1) : 0u; };
  while (count > 0) {                                                             // pieces of rows
    const int h = chunks == 1 ? sub_row : sub_row / chunks, g0 = (sub_row - h * chunks) * kAtOnce, pages = min(count, n - j);
    const int32_t* table = c.table + (long long)b * c.table_stride + j;
    uint32_t page_now = look_up(table, lane, pages), page_next = look_up(table, 32 + lane, pages);
    uint4 q[kAtOnce];
    const T* q_at = static_cast<const T*>(p.q) + b * p.q_request + ((long long)h * p.group + g0) * p.q_head + chunk * 8;
#pragma unroll
    for (int g = 0; g < kAtOnce; ++g) q[g] = g0 + g < p.group ? *reinterpret_cast<const uint4*>(q_at + g * p.q_head) : make_uint4(0, 0, 0, 0);
    const char* bounds = static_cast<const char*>(c.bounds) + (long long)h * kPageBytes + lane * 16 % kPageBytes;
    int fetched = 0;
    uint32_t to = ring;
    auto fetch = [&]() {                                                          // the next stage of pages
      if (fetched < pages) {
        if (fetched > 0 && (fetched & 31) == 0) {
          page_now = page_next;
          page_next = look_up(table, fetched + 32 + lane, pages);
        }
#pragma unroll
        for (int i = 0; i < kStageBytes / 512; ++i) {                             // 512 bytes: one page, or two
          const int at = i * (512 / kPageBytes) + lane * 16 / kPageBytes;
          const uint32_t page = __shfl_sync(0xffffffffu, page_now, (fetched & 31) + at);
          if (fetched + at < pages) copy_16(to + i * 512 + lane * 16, bounds + (unsigned long long)page * step);
        }
        fetched += kStagePages;
        to = to == ring + (kStages - 1) * kStageBytes ? ring : to + kStageBytes;
      }
      copies_end_group();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch();
    unsigned long long qn[kAtOnce][4], qp[kAtOnce][4];                            // negative and positive parts
#pragma unroll
    for (int g = 0; g < kAtOnce; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = H::widen(reinterpret_cast<const typename H::T2*>(&q[g])[i]);
        qn[g][i] = ptx::pack_f32x2(fminf(x.x, 0.f), fminf(x.y, 0.f));
        qp[g][i] = ptx::pack_f32x2(fmaxf(x.x, 0.f), fmaxf(x.y, 0.f));
      }
    // sums over a lane's channels, (x_i + x_i+4) + (x_i+2 + x_i+6) for i = 0 and 1, and over the lanes of a page: at the first two additions a
    // lane goes on with half of the heads, at the others with half of the stage's steps
    constexpr int kTop = kLanes / 2;
    const bool b1 = chunk & kTop, b2 = chunk & (kTop / 2);
    const int gz = g0 + (b1 ? 2 : 0) + (b2 ? 1 : 0);
    auto over_channels = [&](const unsigned long long (&y)[4]) {
      float even, odd;
      ptx::unpack_f32x2(ptx::add_f32x2(ptx::add_f32x2(y[0], y[2]), ptx::add_f32x2(y[1], y[3])), even, odd);
      return __fadd_rn(even, odd);
    };
    auto over_heads = [&](const float (&x)[kAtOnce]) {
      const float s0 = b1 ? x[0] : x[2], s1 = b1 ? x[1] : x[3];
      const float w0 = __fadd_rn(b1 ? x[2] : x[0], __shfl_xor_sync(0xffffffffu, s0, kTop));
      const float w1 = __fadd_rn(b1 ? x[3] : x[1], __shfl_xor_sync(0xffffffffu, s1, kTop));
      return __fadd_rn(b2 ? w1 : w0, __shfl_xor_sync(0xffffffffu, b2 ? w0 : w1, kTop / 2));
    };
    float* m = p.scores + ((long long)(b * c.hkv + h) * p.group + gz) * pitch + j;
    uint32_t stage = ring;
    for (int k = 0; k < pages; k += kStagePages) {
      fetch();
      copies_wait<kStages - 1>();
      __syncwarp();
      float z[kSteps];
      bool odd = false;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const uint32_t at = stage + (i * kPages + sub) * kPageBytes + chunk * 16;
        const uint4 low = ptx::ld_shared_128(at), high = ptx::ld_shared_128(at + 2 * D);
        unsigned long long lo[4], hi[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 x = H::widen(reinterpret_cast<const typename H::T2*>(&low)[w]), y = H::widen(reinterpret_cast<const typename H::T2*>(&high)[w]);
          lo[w] = ptx::pack_f32x2(x.x, x.y);
          hi[w] = ptx::pack_f32x2(y.x, y.y);
        }
        float x[kAtOnce];
#pragma unroll
        for (int g = 0; g < kAtOnce; ++g) {
          unsigned long long y[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) y[w] = ptx::fma_f32x2(qp[g][w], hi[w], ptx::mul_f32x2(qn[g][w], lo[w]));
          x[g] = over_channels(y);
        }
        z[i] = over_heads(x);
      }
      int first = 0, had = kSteps;                                                // steps that this lane ends with: z[0 ..] are first ..
#pragma unroll
      for (int o = kTop / 4; o > 0; o >>= 1) {
        had /= 2;
        const bool up = chunk & o;
        first += up ? had : 0;
#pragma unroll
        for (int i = 0; i < kSteps / 2; ++i)
          if (i < had) z[i] = __fadd_rn(up ? z[i + had] : z[i], __shfl_xor_sync(0xffffffffu, up ? z[i] : z[i + had], o));
      }
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        if (i < had) {
          const int at = k + (first + i) * kPages + sub;
          odd |= z[i] != z[i] && at < pages;
          if (at < pages && gz < p.group) m[at] = z[i];
        }
      if (__any_sync(0xffffffffu, odd)) {                                         // an infinite bound met the part of q that is zero
        __syncwarp();
        score_as_defined<F16, D>(stage, q_at, p.q_head, p.group - g0, m + (long long)(g0 - gz) * pitch + k, pitch, pages - k);
      }
      __syncwarp();                                                               // the stage may be overwritten
      stage = stage == ring + (kStages - 1) * kStageBytes ? ring : stage + kStageBytes;
    }
    count -= pages;
    j = 0;
    if (count > 0 && ++sub_row == per_unit) {
      sub_row = 0;
      do n = pages_of(++b); while (n == 0 && b + 1 < p.batch);
    }
  }
}

template <bool F16, int D>
cudaError_t launch(const SelectParams& p, cudaStream_t st) {
  static SmemLimit limit, preferred;
  auto kernel = decode_select_kernel<F16, D>;
  constexpr size_t smem = kWarps * kStages * kStageBytes;
  cudaError_t e = raise_smem_limit((const void*)kernel, &limit, smem);
  if (e == cudaSuccess) e = prefer_shared((const void*)kernel, &preferred);
  if (e != cudaSuccess) return e;
  const int chunks = (p.group + kAtOnce - 1) / kAtOnce, sms = device_sm_count();
  if (sms <= 0) return cudaErrorInvalidDevice;
  const long long most = (long long)p.batch * p.c.table_stride * p.c.hkv * chunks, per_cta = kWarps * (32 / (D / 8));
  const int grid = (int)std::max(1LL, std::min<long long>(2 * sms, (most + per_cta - 1) / per_cta));
  return launch_chained(kernel, dim3(grid), kThreads, smem, st, p, chunks, p.batch > kFewUnits || most > 0x7fffffffLL);
}

}  // namespace

cudaError_t launch_decode_select(const SelectParams& p, cudaStream_t st) {
  cudaError_t e;
  if (p.c.d == 128) e = p.c.f16 ? launch<true, 128>(p, st) : launch<false, 128>(p, st);
  else e = p.c.f16 ? launch<true, 64>(p, st) : launch<false, 64>(p, st);
  return e == cudaSuccess ? launch_decode_pick(p, st) : e;
}

}  // namespace cosa
