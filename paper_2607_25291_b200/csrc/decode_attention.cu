// cosa_decode_attention: one new token of each request over its cached tokens.
//
// Mathematics.  A KV head's keys and values are read once for the whole group of query heads.  With S = K q^T (keys x heads) a tile
// updates m' = max(m, max S), l = 2^(m-m') l + sum 2^(S-m'), O = 2^(m-m') O + V^T 2^(S-m') (logits in base 2); pieces of a row are
// joined by the same rule.  Both products have keys or channels as the 16 rows of m16n8k16 and eight heads as its
// columns: groups up to eight waste no row, where a 128-row tcgen05 tile would be empty but for one to sixteen rows.
//
// Bound: memory.  2 len hkv d elements are read and 4 flops done for every element and head of the group, some 4 to 16 per byte.  Over an 8-bit cache the
// products and conversions come near it, with 16 heads a KV head they are the bound (128K tokens: 50 us of 42 with 4 heads, 74 with 16; in bf16 86 and 99 of 83).
//
// Division.  All rows -- (request, KV head, chunk of 16 query heads) -- lie one behind the other as tiles of 4 KB of K and 4 KB of V, and every warp that
// multiplies takes an equal run of tiles, wherever rows begin and end: no SM idles behind a long request.  The runs are found from the
// lengths on the device, by every warp for itself where there are few requests.  A CTA an SM: eight warps multiply, each on its own ring
// of tiles, and eight fetch, one for each of them, a box of one page (or part of one) a TMA copy; a tile costs a warp that fetches some 750 cycles
// and one that multiplies 1,050 (bf16, four heads), of the 2,700 that memory takes to bring eight.  With both in one warp 128K tokens took 95.9 us,
// with two kinds 92.2.  No barrier of the CTA until a run is through.  A row inside one run is written at once; pieces are joined in shared memory where
// the row ends inside the CTA, otherwise by the CTA that comes last (or by decode_join.cu), in the order of the pieces in any case.
//
// Measured, device times of calls that take turns on three inputs: 128K tokens of 8 KV heads in bf16 86.0 us (6.2 TB/s, 96 % of the copy rate; reading
// alone the memory gives up to 7.7 TB/s between the first tiles, 4 us, and the last), 48 requests of 500 to 32K tokens in e4m3 122.2 us (6.2 TB/s), one
// request of one token 5.4 us.
#include <algorithm>

#include "decode_join.cuh"
#include "tile_maps.cuh"
#include "warp_mma.cuh"

namespace cosa {
namespace {

constexpr int kWarps = 8, kThreads = 2 * kWarps * 32, kTileBytes = 4096, kStageBytes = 2 * kTileBytes;   // warps that multiply; behind them as many that fetch
// Of a tile in flight: flags; request, KV head, chunk; of its boxes (at most 8) the rows attended to; the next row's request, KV head, chunk; the row's first
// tile, counted over the whole call, and how many it has
constexpr int kMetaWords = 20;
constexpr int kRegsMultiply = 184, kRegsFetch = 72;   // registers a thread: together at most what the CTA is launched with (checked before the launch)
constexpr int kPieceWords = 7;   // of a piece of a row: the row (-1: no piece), request, KV head, chunk, whether the row ends in it, the row's first tile, their number
constexpr int kMinTiles = 2;     // tiles a warp takes at least
// Tiles in flight a warp: 128 KB an SM.  More only lengthens the queues, in which some SMs then fall behind others (128K tokens 91.7 us with three, 87.4
// with two; 48 ragged requests in e4m3 128.7 and 123.7)
constexpr int kStages = 2;
constexpr int kDivisionWords = 2 + 2 * 6;   // tiles of a run, runs with one more; of each unfinished row: first and last CTA, request, KV head, chunk, whether to join it
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
enum Flags { kFull = 1, kFirst = 2, kLast = 4, kFromStart = 8 };   // of a tile: no row masked; first of this run's piece; last of the row; the piece begins the row

struct Maps { CUtensorMap k, v; };
struct Shape {                    // what the launcher works out
  int units, per_unit;            // rows come in units of one length: requests, or with lists (request, KV head)s
  int chunks;                     // chunks of query heads
  int box_rows, box_shift;        // tokens a box
  int boxes_shift;                // log2 boxes a tile
  int page_boxes_shift;           // log2 boxes a page
  bool whole_rows;                // a row lies in one CTA: nothing to be joined behind the kernel
  bool many;                      // too many units, or tiles, for one warp to sum up
  int slot_heads;                 // query heads a piece holds in shared memory
  int slots_bytes;
  DecodeParts parts;
  int* counters;                  // [CTAs] pieces that have been left of the row that begins in a CTA, zero between calls; nullptr: decode_join.cu joins
};

template <bool E4M3, int D> struct Tile {
  static constexpr int kRowBytes = D * (E4M3 ? 1 : 2), kRows = kTileBytes / kRowBytes, kSubs = kRows / 16;
};

// tiles of a unit, and what they cover
struct Unit { int tiles, first, len, from, boxes; };
template <int kRows>
__device__ __forceinline__ Unit unit_of(const DecodeParams& p, const Shape& s, int len, int entries) {
  Unit x;
  x.len = clamped_len(len, p.c);
  x.from = p.window > 0 && x.len > p.window ? x.len - p.window : 0;
  x.first = 0;
  if (p.pages) {
    x.boxes = x.len ? min(max(entries, 0), p.list_stride) << s.page_boxes_shift : 0;
    x.tiles = (x.boxes + (1 << s.boxes_shift) - 1) >> s.boxes_shift;
  } else {
    x.first = x.from / kRows;
    x.tiles = (x.len + kRows - 1) / kRows - x.first;
    x.boxes = (x.len + s.box_rows - 1) >> s.box_shift;
  }
  return x;
}

template <bool F16, bool E4M3, int D, int NT>
__global__ void __launch_bounds__(kThreads, 1) decode_attention_kernel(DecodeParams p, Shape s, const __grid_constant__ Maps maps) {
  using T = Tile<E4M3, D>;
  using H = Half16<F16>;
  using HP = Half16<F16 || E4M3>;            // 8-bit caches are multiplied as f16, which holds their numbers exactly
  constexpr int kHeads = NT * 8, kSteps = D / 16;
  // Weights that are multiplied as f16 are taken against the maximum less 15, so that they reach up to 2^15: f16 ends at 2^16 and has no exponents below 2^-24, where
  // weights of at most 1 would be lost behind a token 17 above them (2^-25 of the largest each, 0.4 % of a row of 128K tokens).  So they are not before 2^-40 of it.  `top`
  // is the lowered maximum everywhere: outputs and sums of a row's pieces grow alike.  Logits beyond 2^22, which differ by halves, are left as they are
  constexpr float kLift = F16 || E4M3 ? 15.f : 0.f;
  // where a channel of a piece lies in shared memory: heads that are written together (two apart) in banks of their own
  auto piece_at = [](int head, int ch) { return head * D + (E4M3 ? ch ^ ((head & 2) << 3) ^ ((head & 4) >> 2) : ch ^ ((head & 6) << 2)); };
  extern __shared__ __align__(1024) char smem[];
  const CacheView& c = p.c;
  const int tid = threadIdx.x, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const bool fetches = tid >= kWarps * 32;
  const int warp = (tid >> 5) & (kWarps - 1);                                 // of those that multiply, or of those that fetch for them
  const int ring_bytes = kStages * kStageBytes;
  const int slot_floats = s.slot_heads * (D + 2);
  char* slots = smem + kWarps * ring_bytes;                                   // the warps' pieces of rows that began before their run
  uint64_t* bars = reinterpret_cast<uint64_t*>(slots + s.slots_bytes);        // [warp][2][stages]: tile arrived, tile worked off
  int* metas = reinterpret_cast<int*>(bars + kWarps * 2 * kStages);
  int* pieces = metas + kWarps * kStages * kMetaWords;                       // [warp][2]: the piece of a row begun before, of one that goes on
  int* counts = pieces + kWarps * 2 * kPieceWords;                            // [warp] tiles
  int* division = counts + kWarps;                                            // tiles of a run, runs with one more; where the CTA's unfinished rows are joined
  volatile int* abort_flag = division + kDivisionWords;
  auto* room = reinterpret_cast<DivisionRoom<kThreads>*>(slots);              // (before the slots are used)
  const bool lists = p.pages != nullptr;
  const uint32_t ring = ptx::smem_u32(smem) + warp * ring_bytes, full0 = ptx::smem_u32(bars + warp * 2 * kStages), empty0 = full0 + kStages * 8;
  int* meta = metas + warp * kStages * kMetaWords;

  // What comes next in the stream may begin to launch: it waits for this kernel itself
  chain_next();
  if (tid == 0) { ptx::prefetch_tensormap(&maps.k); ptx::prefetch_tensormap(&maps.v); }
  if (tid < kWarps * 2) pieces[tid * kPieceWords] = -1;
  if (tid < 2) division[2 + tid * 6] = -1;
  if (tid == 0) *abort_flag = 0;
  if (fetches) {
    if (lane < 2 * kStages) ptx::mbar_init(full0 + lane * 8, 1);
    ptx::mbar_fence_init();
    __syncwarp();
  }
  chain_wait();

  const int boxes = 1 << s.boxes_shift, box_bytes = s.box_rows * T::kRowBytes;
  const int stopped = *p.status;
  auto len_of = [&](int u) { return p.lens[lists ? u / c.hkv : u]; };
  auto entries_of = [&](int u) { return lists ? p.count[u] : 0; };
  // (below 2^31: larger calls are refused)
  auto fetch_unit = [&](int u) { return make_int2(len_of(u), entries_of(u)); };
  auto unit_tiles = [&](int2 x) { return UnitSize{unit_of<T::kRows>(p, s, x.x, x.y).tiles * s.per_unit, x.x, x.y}; };
  const int me = blockIdx.x * kWarps + warp;
  const bool many = s.many;
  Division div{};
  RunStart run{};
  if (many) run = divide_many<kThreads>(s.units, fetch_unit, unit_tiles, (int)gridDim.x * kWarps, kMinTiles, me, div, room);
  bool ok = true;
  if (fetches) {
    // ================================================================ fetching
    int count;
    if (s.whole_rows) {                                                         // each CTA as many rows, its warps equal runs of their tiles
      FewUnits f{};
      f.load(s.units, fetch_unit, unit_tiles);
      const int rows = s.units * s.per_unit;
      const int first = f.before_row(rows * (int)blockIdx.x / (int)gridDim.x, s.per_unit);
      const int tiles = f.before_row(rows * ((int)blockIdx.x + 1) / (int)gridDim.x, s.per_unit) - first;
      count = tiles / kWarps + (warp < tiles % kWarps ? 1 : 0);                 // (warps without a tile come last: pieces of a row lie side by side)
      run = f.seek(first + tiles / kWarps * warp + min(warp, tiles % kWarps));
      div.empty = f.empty;
    } else {
      if (!many) run = divide_few(s.units, fetch_unit, unit_tiles, (int)gridDim.x * kWarps, kMinTiles, me, div);
      count = run_length(div, me);
    }
    if (stopped) count = 0;
    if (lane == 0) counts[warp] = count;
    if (warp == 0 && lane == 0) { division[0] = (int)div.each; division[1] = (int)div.more; }
    int tile = (int)div.each * me + min(me, (int)div.more);                     // the next one, counted over the call (where rows are joined by counters)
    // what is fetched: a row (request, KV head, chunk of query heads) and 32 boxes of it; `ahead`, the next 32 in the walk, is being looked up
    struct Place { int b, h, ch, base; Unit unit; };
    Place at{}, ahead{};
    int left = 0, box = 0, page_now = 0, token_now = -1, page_ahead = 0, token_ahead = -1, len_next = 0, entries_next = 0;
    auto look_up = [&](const Place& x, int& page, int& token) {                 // one box a lane: first token (-1: not to be fetched) and page
      const int i = x.base + lane;
      token = -1;
      page = 0;
      if (i < x.unit.boxes) {
        if (lists) {
          const int j = p.pages[(long long)(x.b * c.hkv + x.h) * p.list_stride + (i >> s.page_boxes_shift)];
          if (j >= 0 && j < c.table_stride) token = (j << c.page_shift) + ((i & ((1 << s.page_boxes_shift) - 1)) << s.box_shift);
        } else {
          token = i << s.box_shift;
        }
        if (token >= x.unit.len || token + s.box_rows <= x.unit.from) token = -1;
        if (token >= 0) page = c.table[(long long)x.b * c.table_stride + (token >> c.page_shift)];
      }
    };
    auto next_window = [&]() {                                                  // `at` becomes `ahead`, and `ahead` what comes after it
      at = ahead;
      page_now = page_ahead;
      token_now = token_ahead;
      ahead.base += 32;
      if (ahead.base >= (at.unit.first + at.unit.tiles) << s.boxes_shift) {
        if (++ahead.ch == s.chunks) {
          ahead.ch = 0;
          if (++ahead.h == c.hkv) { ahead.h = 0; ++ahead.b; }
          if (lists || ahead.h == 0)
            for (;;) {
              if (ahead.b >= p.batch) { ahead.unit = Unit{}; break; }           // (past the last run)
              ahead.unit = unit_of<T::kRows>(p, s, len_next, entries_next);
              const int u = lists ? ahead.b * c.hkv + ahead.h + 1 : ahead.b + 1;
              if (u < s.units) { len_next = len_of(u); entries_next = entries_of(u); }
              if (ahead.unit.tiles > 0) break;
              if (!lists) ++ahead.b;
              else if (++ahead.h == c.hkv) { ahead.h = 0; ++ahead.b; }
            }
        }
        ahead.base = (ahead.unit.first << s.boxes_shift) & ~31;
      }
      look_up(ahead, page_ahead, token_ahead);
    };
    if (count > 0) {
      const int u = run.unit;
      ahead.unit = unit_of<T::kRows>(p, s, run.size.a, run.size.b);
      if (u + 1 < s.units) { len_next = len_of(u + 1); entries_next = entries_of(u + 1); }
      const int sub_row = run.in_unit <= 0x7fffffffLL ? (int)run.in_unit / ahead.unit.tiles : (int)(run.in_unit / ahead.unit.tiles);
      const int skip = (int)(run.in_unit - (long long)sub_row * ahead.unit.tiles);
      if (lists) { ahead.b = u / c.hkv; ahead.h = u - ahead.b * c.hkv; ahead.ch = sub_row; }
      else { ahead.b = u; ahead.h = s.chunks == 1 ? sub_row : sub_row / s.chunks; ahead.ch = sub_row - ahead.h * s.chunks; }
      left = ahead.unit.tiles - skip;
      box = (ahead.unit.first + skip) << s.boxes_shift;
      ahead.base = box & ~31;
      look_up(ahead, page_ahead, token_ahead);
    }
    bool piece_begins = true, fetching = false;
    const uint64_t once = ptx::l2_policy_evict_first();                         // (a step reads a layer's cache once: 200 windows 42.8 -> 39.5 us, lists 49.9 -> 48.5)
    auto issue = [&](int stage) {
      if (left == 0 || box - at.base == 32 || !fetching) {
        fetching = true;
        next_window();
        if (left == 0) {
          left = at.unit.tiles;
          box = at.unit.first << s.boxes_shift;
          piece_begins = true;
        }
      }
      const int i = box - at.base, token = __shfl_sync(0xffffffffu, token_now, i + (lane & (boxes - 1)));
      const int low = token < 0 ? 0 : max(0, at.unit.from - token), high = token < 0 ? 0 : min(s.box_rows, at.unit.len - token);
      const uint32_t here = __ballot_sync(0xffffffffu, lane < boxes && token >= 0);
      const bool full = __all_sync(0xffffffffu, low == 0 && high == s.box_rows);
      int* m = meta + stage * kMetaWords;
      --left;
      if (lane < boxes) m[4 + lane] = low | (high << 16);
      if (lane == 0) {
        *reinterpret_cast<int4*>(m) = make_int4((full ? kFull : 0) | (piece_begins ? kFirst : 0) | (left == 0 ? kLast : 0) |
                                                    (box == at.unit.first << s.boxes_shift ? kFromStart : 0),
                                                at.b, at.h, at.ch);
        *reinterpret_cast<int4*>(m + 12) = make_int4(ahead.b, ahead.h, ahead.ch, 0);   // (behind the row's last tile: the next row)
        *reinterpret_cast<int2*>(m + 16) = make_int2(tile - ((box >> s.boxes_shift) - at.unit.first), at.unit.tiles);
      }
      piece_begins = false;
      ++tile;
      __syncwarp();
      const uint32_t bar = full0 + stage * 8, dst = ring + stage * kStageBytes;
      if (ptx::elect_one()) ptx::mbar_expect_tx(bar, __popc(here) * 2 * box_bytes);
      __syncwarp();
      for (int j = 0; j < boxes; ++j) {
        if (!((here >> j) & 1)) continue;
        const int page = __shfl_sync(0xffffffffu, page_now, i + j), row = __shfl_sync(0xffffffffu, token_now, i + j) & (c.page_size - 1);
        if (ptx::elect_one()) {
          ptx::tma_load_5d(dst + j * box_bytes, &maps.k, 0, row, 0, at.h, page, bar, once);
          ptx::tma_load_5d(dst + kTileBytes + j * box_bytes, &maps.v, 0, row, 0, at.h, page, bar, once);
        }
      }
      box += boxes;
    };
    const bool short_budget = ptx::wait_budget_is_short(p.wait_budget);
    int issued = 0, stage = 0, round = 0;                                       // round: how often the ring has been filled
    bool met = false, stop = false;
    // (all stages at first; the CTA meets before any of them is waited for, and those that multiply learn what there is for them)
    for (;;) {
      if (!met && (issued == kStages || issued == count)) {
        stop = __syncthreads_or(stopped);
        if (!stop) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFetch));
        met = true;
        if (stop) break;
      }
      if (issued == count) break;
      if (round > 0) {
        const uint32_t bar = empty0 + stage * 8, parity = (round - 1) & 1;
        ok = short_budget ? ptx::mbar_poll_warp(bar, parity, abort_flag, max(p.wait_budget, 1LL << 24)) : ptx::mbar_wait_warp(bar, parity, abort_flag, p.wait_budget);
        if (!ok) break;
      }
      issue(stage);
      ++issued;
      if (++stage == kStages) { stage = 0; ++round; }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicExch(p.status, (int32_t)COSA_ERR_DEVICE_TIMEOUT);
    }
    // What is in flight arrives on its own, given up or not, and is waited for before the shared memory goes to another CTA
    for (int i = max(0, issued - kStages); i < issued; ++i) ptx::mbar_wait_noabort(full0 + i % kStages * 8, i / kStages & 1);
    if (stop) return;
    // ---- rows without a token
    if (div.empty)
      for (int u0 = me * 32; u0 < s.units; u0 += gridDim.x * kWarps * 32) {
        const bool none = u0 + lane < s.units && unit_of<T::kRows>(p, s, len_of(u0 + lane), entries_of(u0 + lane)).tiles == 0;
        for (uint32_t found = __ballot_sync(0xffffffffu, none); found; found &= found - 1) {
          const int u = u0 + __ffs(found) - 1, n = lists ? p.group : p.hq;
          const int rb = lists ? u / c.hkv : u, h0 = lists ? u % c.hkv * p.group : 0;
          for (int i = lane; i < n * (D / 8); i += 32)
            *reinterpret_cast<uint4*>(static_cast<typename H::T*>(p.out) + rb * p.out_request + (long long)(h0 + i / (D / 8)) * p.out_head + i % (D / 8) * 8) =
                make_uint4(0, 0, 0, 0);
          if (p.lse)
            for (int i = lane; i < n; i += 32) p.lse[(long long)rb * p.hq + h0 + i] = -INFINITY;
        }
      }
  } else {
    // ================================================================ multiplying
    if (__syncthreads_or(stopped)) return;
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsMultiply));
    const int count = counts[warp];
    uint32_t q[NT][kSteps][2];
    auto load_q = [&](int b, int h, int ch) {
      const int heads = min(kHeads, p.group - ch * kHeads);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const bool there = n * 8 + g < heads;
        const typename H::T* src = static_cast<const typename H::T*>(p.q) + b * p.q_request + (long long)(h * p.group + ch * kHeads + n * 8 + (there ? g : 0)) * p.q_head;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          if constexpr (E4M3) {                  // channels 4t .. 4t+3 of a step, the order in which the cache's bytes come
            const uint2 x = there ? *reinterpret_cast<const uint2*>(src + 16 * j + 4 * t4) : make_uint2(0, 0);
            q[n][j][0] = x.x;
            q[n][j][1] = x.y;
          } else {
            q[n][j][0] = there ? *reinterpret_cast<const uint32_t*>(src + 16 * j + 2 * t4) : 0u;
            q[n][j][1] = there ? *reinterpret_cast<const uint32_t*>(src + 16 * j + 8 + 2 * t4) : 0u;
          }
        }
      }
    };
    // ---- the products
    // address of 16 bytes of a tile: chunk of the row of `key`
    auto chunk_at = [&](int key, int chunk) -> uint32_t {
      if constexpr (T::kRowBytes == 256) {      // a box: 64 channels of every row, then the other 64
        const int j = key >> s.box_shift, r = key & (s.box_rows - 1);
        return j * box_bytes + (chunk >> 3) * (box_bytes >> 1) + r * 128 + (((chunk ^ r) & 7) << 4);
      } else if constexpr (T::kRowBytes == 128) {
        return key * 128 + (((chunk ^ key) & 7) << 4);
      } else {
        return key * 64 + (((chunk ^ (key >> 1)) & 3) << 4);
      }
    };
    float o[NT][kSteps][4], top[NT][2], l[NT][2], scale[NT][2];
    int b = 0, kvh = 0, ch = 0, head0 = 0, heads = 0, from_start = 0, row_first = 0, row_tiles = 0;
    int stage = 0, parity = 0;
    for (int done = 0; done < count; ++done) {
      // (a short budget is kept to by polling: a wait that may suspend can outlast it)
      ok = ptx::wait_budget_is_short(p.wait_budget) ? ptx::mbar_poll_warp(full0 + stage * 8, parity, abort_flag, p.wait_budget)
                                                    : ptx::mbar_wait_warp(full0 + stage * 8, parity, abort_flag, p.wait_budget);
      if (!ok) break;
      const int* m = meta + stage * kMetaWords;
      const int flags = m[0];
      if (flags & kFirst) {
        b = m[1];
        kvh = m[2];
        ch = m[3];
        from_start = flags & kFromStart;
        row_first = m[16];
        row_tiles = m[17];
        if (done == 0) load_q(b, kvh, ch);
        head0 = kvh * p.group + ch * kHeads;
        heads = min(kHeads, p.group - ch * kHeads);
        const float scale_kv = p.scale * kLog2e * (E4M3 ? c.k_scale[kvh] : 1.f);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          scale[n][0] = scale[n][1] = scale_kv;
          if constexpr (E4M3 && !F16) {
            // bf16 queries as f16, each head divided by a power of two so that its largest element lies in [1, 2): exact but for elements below 2^-14
            // of that, whose last bits are lost
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float2 x = H::widen(*reinterpret_cast<const typename H::T2*>(&q[n][j][i]));
                most = fmaxf(most, fmaxf(fabsf(x.x), fabsf(x.y)));
              }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int e = most > 0.f ? min(126, max(-126, (int)(__float_as_uint(most) >> 23) - 127)) : 0;
            const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float2 x = H::widen(*reinterpret_cast<const typename H::T2*>(&q[n][j][i]));
                const __half2 y = __floats2half2_rn(x.x * down, x.y * down);
                q[n][j][i] = *reinterpret_cast<const uint32_t*>(&y);
              }
            scale[n][0] *= __shfl_sync(0xffffffffu, up, 8 * t4);
            scale[n][1] *= __shfl_sync(0xffffffffu, up, 8 * t4 + 4);
          }
          top[n][0] = top[n][1] = -INFINITY;
          l[n][0] = l[n][1] = 0.f;
#pragma unroll
          for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][j][i] = 0.f;
        }
      }
      const uint32_t kt = ring + stage * kStageBytes, vt = kt + kTileBytes;
      if (!(flags & kFull)) {
        // rows that are not attended to: whatever they hold, their weight of zero must meet a number
        constexpr int kChunks = T::kRowBytes / 16;
        for (int i = lane; i < T::kRows * kChunks; i += 32) {
          const int key = i / kChunks, range = m[4 + (key >> s.box_shift)], r = key & (s.box_rows - 1);
          if (r < (range & 0xffff) || r >= (range >> 16))
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vt + chunk_at(key, i % kChunks)), "r"(0) : "memory");
        }
        __syncwarp();
      }
      float x[T::kSubs][NT][4];
#pragma unroll
      for (int u16 = 0; u16 < T::kSubs; ++u16) {
        float y[NT][4];                                                         // (two sums: half as many products wait for one another)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[u16][n][i] = y[n][i] = 0.f;
        const int key = u16 * 16 + (lane & 15);
        if constexpr (E4M3) {
#pragma unroll
          for (int j = 0; j < kSteps; j += 2) {
            uint32_t r[4];
            ptx::ldmatrix_x4(r, kt + chunk_at(key, j + (lane >> 4)));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t a[4] = {ptx::e4m3x2_to_f16x2((uint16_t)r[2 * i]), ptx::e4m3x2_to_f16x2((uint16_t)r[2 * i + 1]),
                                     ptx::e4m3x2_to_f16x2((uint16_t)(r[2 * i] >> 16)), ptx::e4m3x2_to_f16x2((uint16_t)(r[2 * i + 1] >> 16))};
#pragma unroll
              for (int n = 0; n < NT; ++n) ptx::mma_16x8x16<true>(i ? y[n] : x[u16][n], a, q[n][j + i][0], q[n][j + i][1]);
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            uint32_t a[4];
            ptx::ldmatrix_x4(a, kt + chunk_at(key, 2 * j + (lane >> 4)));
#pragma unroll
            for (int n = 0; n < NT; ++n) ptx::mma_16x8x16<F16>(j & 1 ? y[n] : x[u16][n], a, q[n][j][0], q[n][j][1]);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[u16][n][i] += y[n][i];
      }
      if ((flags & kLast) && done + 1 < count) load_q(m[12], m[13], m[14]);      // the next row's queries, while this one is brought to its end
#pragma unroll
      for (int u16 = 0; u16 < T::kSubs; ++u16) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[u16][n][i] *= scale[n][i & 1];
        if (!(flags & kFull)) {
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const int key = u16 * 16 + g + 4 * i, range = m[4 + (key >> s.box_shift)], r = key & (s.box_rows - 1);
            if (r < (range & 0xffff) || r >= (range >> 16))
#pragma unroll
              for (int n = 0; n < NT; ++n) x[u16][n][i] = x[u16][n][i + 1] = -INFINITY;
          }
        }
      }
      float ref[NT][2], keep[NT][2];
      bool moved = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float now = -INFINITY;
#pragma unroll
          for (int u16 = 0; u16 < T::kSubs; ++u16) now = fmaxf(now, fmaxf(x[u16][n][i], x[u16][n][i + 2]));
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, off));
          now = fmaxf(top[n][i], kLift && fabsf(now) < 0x1p22f ? now - kLift : now);
          ref[n][i] = now == -INFINITY ? 0.f : now;
          keep[n][i] = ptx::ex2_approx(top[n][i] - ref[n][i]);
          moved |= now != top[n][i];
          top[n][i] = now;
        }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          l[n][0] *= keep[n][0];
          l[n][1] *= keep[n][1];
#pragma unroll
          for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][j][i] *= keep[n][i & 1];
        }
      }
#pragma unroll
      for (int u16 = 0; u16 < T::kSubs; ++u16) {
        // Weights as two 16-bit terms, the second what rounding to the first leaves: one term alone would add 2^-9 (bf16) or 2^-12 (f16) to the output's own
        // rounding.  The second product costs nothing over a 16-bit cache, where memory is the bound, and little over an 8-bit one (one term and two, bf16 outputs: 48
        // ragged requests 120.7 and 122.2 us, in a loop of seconds under the power cap 127.3 and 132.0; 128K tokens 49.7 and 53.5, with 16 heads a KV head 64 and 75)
        uint32_t big[NT][2], rest[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float w0 = ptx::ex2_approx(x[u16][n][2 * i] - ref[n][0]), w1 = ptx::ex2_approx(x[u16][n][2 * i + 1] - ref[n][1]);
            l[n][0] += w0;
            l[n][1] += w1;
            const typename HP::T2 hi = HP::narrow(w0, w1);
            big[n][i] = ptx::transpose_8x8(*reinterpret_cast<const uint32_t*>(&hi));
            const float2 back = HP::widen(hi);
            const typename HP::T2 lo = HP::narrow(w0 - back.x, w1 - back.y);
            rest[n][i] = ptx::transpose_8x8(*reinterpret_cast<const uint32_t*>(&lo));
          }
        if constexpr (E4M3) {
          const int key = u16 * 16 + (lane & 15);
#pragma unroll
          for (int j = 0; j < kSteps; j += 2) {
            uint32_t r[4];
            ptx::ldmatrix_x4_trans(r, vt + chunk_at(key, j + (lane >> 4)));
#pragma unroll
            for (int i = 0; i < 2; ++i) {      // even channels are rows 0-7, odd ones rows 8-15
              const uint32_t first = __byte_perm(r[2 * i], 0, 0x3120), second = __byte_perm(r[2 * i + 1], 0, 0x3120);
              const uint32_t a[4] = {ptx::e4m3x2_to_f16x2((uint16_t)first), ptx::e4m3x2_to_f16x2((uint16_t)(first >> 16)),
                                     ptx::e4m3x2_to_f16x2((uint16_t)second), ptx::e4m3x2_to_f16x2((uint16_t)(second >> 16))};
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                ptx::mma_16x8x16<true>(o[n][j + i], a, big[n][0], big[n][1]);
                ptx::mma_16x8x16<true>(o[n][j + i], a, rest[n][0], rest[n][1]);
              }
            }
          }
        } else {
          const int key = u16 * 16 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
          for (int j = 0; j < kSteps; j += 2) {      // (two steps' first terms, then their second ones: no product waits for the one before it)
            uint32_t a[2][4];
            ptx::ldmatrix_x4_trans(a[0], vt + chunk_at(key, 2 * j + ((lane >> 3) & 1)));
            ptx::ldmatrix_x4_trans(a[1], vt + chunk_at(key, 2 * j + 2 + ((lane >> 3) & 1)));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              ptx::mma_16x8x16<F16>(o[n][j], a[0], big[n][0], big[n][1]);
              ptx::mma_16x8x16<F16>(o[n][j + 1], a[1], big[n][0], big[n][1]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              ptx::mma_16x8x16<F16>(o[n][j], a[0], rest[n][0], rest[n][1]);
              ptx::mma_16x8x16<F16>(o[n][j + 1], a[1], rest[n][0], rest[n][1]);
            }
          }
        }
      }
      if (!(flags & kFull)) ptx::fence_proxy_async_smem();                      // the zeros written above come before the next copy into this stage
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(empty0 + stage * 8);
      if (++stage == kStages) { stage = 0; parity ^= 1; }
      if (!(flags & kLast) && done + 1 < count) continue;

      // ---- the end of this run's piece of the row
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], off);
      if ((flags & kLast) && from_start) {                                      // the whole row
        const float vs = E4M3 ? c.v_scale[kvh] : 1.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          // (a sum of zero: no logit above -inf, and no tokens in effect; one that is no number goes on to the outputs)
          const bool none0 = l[n][0] == 0.f, none1 = l[n][1] == 0.f;
          const float inv0 = vs / l[n][0], inv1 = vs / l[n][1];
          const int head = n * 8 + g;
          typename H::T* dst = static_cast<typename H::T*>(p.out) + b * p.out_request + (long long)(head0 + head) * p.out_head;
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            const typename H::T2 first = H::narrow(none0 ? 0.f : o[n][j][0] * inv0, none1 ? 0.f : o[n][j][1] * inv1),
                                 second = H::narrow(none0 ? 0.f : o[n][j][2] * inv0, none1 ? 0.f : o[n][j][3] * inv1);
            const uint32_t x0 = ptx::transpose_8x8(*reinterpret_cast<const uint32_t*>(&first)), x1 = ptx::transpose_8x8(*reinterpret_cast<const uint32_t*>(&second));
            if (head < heads) {
              if constexpr (E4M3) {
                *reinterpret_cast<uint2*>(dst + 16 * j + 4 * t4) = make_uint2(__byte_perm(x0, x1, 0x5410), __byte_perm(x0, x1, 0x7632));
              } else {
                *reinterpret_cast<uint32_t*>(dst + 16 * j + 2 * t4) = x0;
                *reinterpret_cast<uint32_t*>(dst + 16 * j + 8 + 2 * t4) = x1;
              }
            }
          }
          if (p.lse && g == 0)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (n * 8 + 2 * t4 + i < heads)
                p.lse[(long long)b * p.hq + head0 + n * 8 + 2 * t4 + i] = l[n][i] == 0.f ? -INFINITY : top[n][i] * kLn2 + logf(l[n][i]);
        }
      } else {
        // piece 1 (begins its row, which goes on) is the run's last: it takes the place of the ring
        const int which = from_start ? 1 : 0;
        float* dst = reinterpret_cast<float*>(which ? smem + warp * ring_bytes : slots + warp * slot_floats * 4);
        __syncwarp();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int head = n * 8 + 2 * t4 + i;
            if (head < heads) {
              if (g == 0) { dst[s.slot_heads * D + head] = top[n][i]; dst[s.slot_heads * (D + 1) + head] = l[n][i]; }
#pragma unroll
              for (int j = 0; j < kSteps; ++j) {
                dst[piece_at(head, 16 * j + (E4M3 ? 2 * g : g))] = o[n][j][i];
                dst[piece_at(head, 16 * j + (E4M3 ? 2 * g + 1 : g + 8))] = o[n][j][2 + i];
              }
            }
          }
        if (lane == 0) {
          int* x = pieces + (warp * 2 + which) * kPieceWords;
          x[0] = (b * c.hkv + kvh) * s.chunks + ch;
          x[1] = b;
          x[2] = kvh;
          x[3] = ch;
          x[4] = (flags & kLast) ? 1 : 0;
          x[5] = row_first;
          x[6] = row_tiles;
        }
      }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicExch(p.status, (int32_t)COSA_ERR_DEVICE_TIMEOUT);
    }
    ptx::bar_sync(1, kWarps * 32);
    if (*abort_flag) return;

    // ================================================================ rows whose pieces meet in this CTA, and those that go on in others
    // (a warp takes a row and query head, a lane channels 32 apart)
    constexpr int kVec = D / 32;
    const uint32_t going = __ballot_sync(0xffffffffu, lane < kWarps && pieces[lane * 2 * kPieceWords] >= 0);
    const uint32_t ending = __ballot_sync(0xffffffffu, lane < kWarps && pieces[lane * 2 * kPieceWords] >= 0 && pieces[lane * 2 * kPieceWords + 4]);
    const uint32_t begun = __ballot_sync(0xffffffffu, lane < kWarps && pieces[(lane * 2 + 1) * kPieceWords] >= 0);
    DecodePart* part = s.parts.part + blockIdx.x;
    if (tid < 2 && !(tid == 0 ? (going & 1) : begun)) part->piece[tid].row = -1;
    int job = 0;
    for (uint32_t starts = (going & 1) | (begun << 1); starts; starts &= starts - 1) {   // bit 0: a row begun before this CTA; bit w + 1: one begun in warp w
      const int which = (starts & 1) ? 0 : 1, w0 = which ? __ffs(starts) - 2 : 0;
      // the pieces follow one another in the warps behind, up to the one where the row ends
      const uint32_t behind = which ? ~((2u << w0) - 1u) : ~0u, stop = ~going & behind & ((1u << kWarps) - 1u), end = ending & behind;
      const int before_stop = stop ? __ffs(stop) - 2 : kWarps - 1, at_end = end ? __ffs(end) - 1 : kWarps;
      const int last = min(before_stop, at_end);
      const bool ends = at_end == last, whole = which && ends;
      const int* x = pieces + (w0 * 2 + which) * kPieceWords;
      const int rb = x[1], rh = x[2], rch = x[3], h0 = rh * p.group + rch * kHeads, hn = min(kHeads, p.group - rch * kHeads);
      if (which && !whole) { if (tid == 0) part->piece[1] = DecodePiece{x[0], rb, rh, rch, 0}; }
      else if (which) { if (tid == 0 && !((starts >> 1) & ~((1u << w0)))) part->piece[1].row = -1; }
      else if (tid == 0) part->piece[0] = DecodePiece{x[0], rb, rh, rch, ends ? 1 : 0};
      if (!whole && tid == 0) {                                                 // the CTAs in which the row's first and last tile are
        const int each = division[0], longer = division[1] * (each + 1);
        auto cta_of = [&](int t) { return (t < longer ? t / (each + 1) : division[1] + (t - longer) / each) / kWarps; };
        int* y = division + 2 + which * 6;
        y[0] = cta_of(x[5]);
        y[1] = cta_of(x[5] + x[6] - 1);
        y[2] = rb;
        y[3] = rh;
        y[4] = rch;
      }
      for (int head = (warp - job) & (kWarps - 1); head < hn; head += kWarps) {
        auto piece = [&](int w) { return reinterpret_cast<const float*>(w == w0 && which ? smem + w * ring_bytes : slots + w * slot_floats * 4); };
        const int n = last - w0 + 1;                                            // a lane looks at a piece's maximum and sum, then all at its channels
        const float* of_lane = piece(w0 + min(lane, n - 1));
        const float top = lane < n ? of_lane[s.slot_heads * D + head] : -INFINITY, most = ptx::warp_max(top), ref = most == -INFINITY ? 0.f : most;
        const float weight = ptx::ex2_approx(top - ref);
        float sum_l = lane < n ? weight * of_lane[s.slot_heads * (D + 1) + head] : 0.f, sum_o[kVec];
#pragma unroll
        for (int off = 4; off > 0; off >>= 1) sum_l += __shfl_xor_sync(0xffffffffu, sum_l, off);
        sum_l = __shfl_sync(0xffffffffu, sum_l, 0);                             // (eight pieces at most)
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum_o[i] = 0.f;
#pragma unroll 2
        for (int k = 0; k < n; ++k) {
          const float* y = piece(w0 + k);
          const float w = __shfl_sync(0xffffffffu, weight, k);
#pragma unroll
          for (int i = 0; i < kVec; ++i) sum_o[i] += w * y[piece_at(head, i * 32 + lane)];
        }
        if (whole) {
          const float inv = (E4M3 ? c.v_scale[rh] : 1.f) / sum_l;
          typename H::T* dst = static_cast<typename H::T*>(p.out) + rb * p.out_request + (long long)(h0 + head) * p.out_head + lane;
#pragma unroll
          for (int i = 0; i < kVec; ++i) dst[i * 32] = H::narrow1(sum_l == 0.f ? 0.f : sum_o[i] * inv);
          if (p.lse && lane == 0) p.lse[(long long)rb * p.hq + h0 + head] = sum_l == 0.f ? -INFINITY : most * kLn2 + logf(sum_l);
        } else {
          float* to = s.parts.data + ((long long)blockIdx.x * 2 + which) * s.slot_heads * (D + 4);
#pragma unroll
          for (int i = 0; i < kVec; ++i) to[head * D + i * 32 + lane] = sum_o[i];
          if (lane == 0) { to[s.slot_heads * D + head] = most; to[s.slot_heads * (D + 1) + head] = sum_l; }
        }
      }
      job += hn;
    }
    if (!s.counters) return;
    // the CTA that leaves a row's last piece joins it (in the order of the pieces, whoever is last)
    ptx::bar_sync(1, kWarps * 32);
    if (tid < 2) {
      int* y = division + 2 + tid * 6;
      y[5] = 0;
      if (y[0] >= 0 && ptx::count_acq_rel(s.counters + y[0]) == y[1] - y[0]) {  // (before it lies all that this CTA has left, behind it what the others have)
        s.counters[y[0]] = 0;
        y[5] = 1;
      }
    }
    ptx::bar_sync(1, kWarps * 32);
    const int heads0 = division[2 + 5] ? min(kHeads, p.group - division[2 + 4] * kHeads) : 0, heads1 = division[8 + 5] ? min(kHeads, p.group - division[8 + 4] * kHeads) : 0;
#pragma unroll 1
    for (int i = warp; i < heads0 + heads1; i += kWarps) {
      const int* y = division + (i < heads0 ? 2 : 8);
      join_head<F16, D>(p, s.parts.data, s.slot_heads, kHeads, y[0], y[1], y[2], y[3], y[4], i < heads0 ? i : i - heads0);
    }
  }
}

// a tensor map over one pool: (columns of 128 bytes at most, tokens of a page, column blocks, heads, pages)
bool make_pool_map(CUtensorMap* map, const void* base, const CacheView& c, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const int es = c.e4m3 ? 1 : 2, row = c.d * es, inner = row < 128 ? row : 128;
  const cuuint64_t dims[5] = {(cuuint64_t)(inner / es), (cuuint64_t)c.page_size, (cuuint64_t)(row / inner), (cuuint64_t)c.hkv, (cuuint64_t)c.num_pages};
  const cuuint64_t strides[4] = {(cuuint64_t)c.token_stride * es, (cuuint64_t)inner, (cuuint64_t)c.head_stride * es, (cuuint64_t)c.page_stride * es};
  const cuuint32_t box[5] = {(cuuint32_t)(inner / es), (cuuint32_t)box_rows, (cuuint32_t)(row / inner), 1, 1}, one[5] = {1, 1, 1, 1, 1};
  return fn(map, c.e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, const_cast<void*>(base), dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, inner == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int log2_int(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}
int heads_per_chunk(int group) { return group <= 8 ? 8 : 16; }

template <bool F16, bool E4M3, int D, int NT>
cudaError_t launch(const DecodeParams& p, Shape s, int grid, const Maps& maps, cudaStream_t st) {
  static SmemLimit limit;
  // the slots' place first holds the sums over many units
  const size_t slots = (size_t)kWarps * s.slot_heads * (D + 2) * 4, begin = sizeof(DivisionRoom<kThreads>);
  s.slots_bytes = (int)((std::max(slots, begin) + 15) / 16 * 16);
  const size_t fixed = s.slots_bytes + (kWarps * 2 * kPieceWords + kWarps + kDivisionWords + 4) * 4, per_stage = kWarps * (kStageBytes + 16 + kMetaWords * 4);
  const size_t smem = fixed + kStages * per_stage;
  if (smem > 227 * 1024) return cudaErrorInvalidConfiguration;
  auto kernel = decode_attention_kernel<F16, E4M3, D, NT>;
  cudaError_t e = raise_smem_limit((const void*)kernel, &limit, smem);
  if (e != cudaSuccess) return e;
  // the split of the registers must not exceed what the CTA is launched with: a warp would wait for its share for good
  static const bool enough = [&] {
    cudaFuncAttributes attr{};
    return cudaFuncGetAttributes(&attr, (const void*)kernel) == cudaSuccess && attr.numRegs * 2 >= kRegsMultiply + kRegsFetch;
  }();
  if (!enough) return cudaErrorInvalidConfiguration;
  return launch_chained(kernel, dim3(grid), kThreads, smem, st, p, s, maps);
}

}  // namespace

size_t decode_attention_scratch(int group, int d) {
  int sms = device_sm_count();
  if (sms <= 0) sms = 160;
  return (size_t)sms * (2 * std::min(group, heads_per_chunk(group)) * (d + 4) * sizeof(float) + sizeof(DecodePart));
}

cudaError_t launch_decode_attention(const DecodeParams& p, cudaStream_t st) {
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorInvalidDevice;
  const CacheView& c = p.c;
  const int tile_rows = kTileBytes / (c.d * (c.e4m3 ? 1 : 2)), per_chunk = heads_per_chunk(p.group);
  Shape s{};
  s.chunks = (p.group + per_chunk - 1) / per_chunk;
  s.units = p.pages ? p.batch * c.hkv : p.batch;
  s.per_unit = p.pages ? s.chunks : c.hkv * s.chunks;
  s.box_rows = std::min(c.page_size, tile_rows);
  s.box_shift = log2_int(s.box_rows);
  s.boxes_shift = log2_int(tile_rows / s.box_rows);
  s.page_boxes_shift = c.page_shift - s.box_shift;
  s.slot_heads = std::min(p.group, per_chunk);
  // no more CTAs than the longest rows that the tables allow could use
  long long row_tokens = p.pages ? (long long)p.list_stride << c.page_shift : (long long)c.table_stride << c.page_shift;
  if (p.window > 0 && !p.pages) row_tokens = std::min<long long>(row_tokens, (long long)p.window + tile_rows);
  const long long row_tiles = (row_tokens + tile_rows - 1) / tile_rows;
  const long long useful = (row_tiles * s.units * s.per_unit / kMinTiles + kWarps - 1) / kWarps;
  const int ctas = p.ctas > 0 ? std::min(p.ctas, sms) : sms;
  const long long rows = (long long)s.units * s.per_unit;
  // Rows of few tiles, and few of them: a CTA takes whole ones, nothing is joined through global memory, and no second kernel is launched for it where a workspace is the
  // caller's (three requests of up to 201 tokens of 8 heads: 8.9 us to 6.8, now 5.9).  Whole rows and equal runs, us, for rows of 4, 8, 16 and 32 tiles each:
  // 8 rows of 4 heads 5.7 / 6.5 / 7.7 / 9.4 and 7.9 / 7.4 / 7.5 / 9.9; 128 rows 6.1 / 7.0 / 8.3 / 10.0 and 8.3 / 7.9 / 8.0 / 11.6; 296 rows, two a CTA,
  // 7.1 / 8.4 / 10.1 / 13.4 and 8.6 / 8.1 / 9.8 / 13.1; 32 rows of 16 heads 7.6 / 8.9 / 10.5 / 12.8 and 12.5 / 10.9 / 10.2 / 13.9, in e4m3 8.4 / 9.8 / 12.2 / 15.8 and
  // 14.3 / 12.7 / 11.8 / 15.8.  (Tiles are those of the longest row that the table could hold: the lengths are on the device)
  s.many = s.units > kFewUnits || row_tiles * rows > 0x7fffffffLL;
  s.whole_rows = row_tiles <= 32 && !s.many && rows <= 2 * ctas;
  const int grid = (int)std::max(1LL, std::min<long long>(ctas, s.whole_rows ? rows : useful));
  s.parts.data = p.partials;
  s.parts.part = reinterpret_cast<DecodePart*>(p.partials + (size_t)sms * 2 * s.slot_heads * (c.d + 4));
  // (counters where the library's own scratch is used, which calls that may overlap do not share, and tiles are counted in 32 bits)
  s.counters = grid > 1 && !s.whole_rows && row_tiles * rows <= 0x7fffffffLL ? p.counters : nullptr;
  Maps maps;
  if (!make_pool_map(&maps.k, c.k, c, s.box_rows) || !make_pool_map(&maps.v, c.v, c, s.box_rows)) return cudaErrorInvalidValue;
  const bool wide = p.group > 8;
  cudaError_t e;
#define COSA_DECODE(f16, e4m3)                                                                                             \
  e = c.d == 128 ? (wide ? launch<f16, e4m3, 128, 2>(p, s, grid, maps, st) : launch<f16, e4m3, 128, 1>(p, s, grid, maps, st)) \
                 : (wide ? launch<f16, e4m3, 64, 2>(p, s, grid, maps, st) : launch<f16, e4m3, 64, 1>(p, s, grid, maps, st))
  if (c.f16) {
    if (c.e4m3) COSA_DECODE(true, true); else COSA_DECODE(true, false);
  } else {
    if (c.e4m3) COSA_DECODE(false, true); else COSA_DECODE(false, false);
  }
#undef COSA_DECODE
  if (e != cudaSuccess || grid == 1 || s.whole_rows || s.counters) return e;
  return launch_decode_join(p, s.parts, grid, s.slot_heads, per_chunk, st);
}

}  // namespace cosa
