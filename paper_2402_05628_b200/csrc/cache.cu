// The paged 8-bit cache: the plan of a step (block tables, slot map, positions) and the write of K / V rows.
#include <cuda_bf16.h>

#include "cache.cuh"
#include "f32x2.cuh"
#include "kernels.h"

namespace repq {
namespace cache {

repq_status check(const repq_cache& c, const char* who) {
  REPQ_REQUIRE(c.num_blocks > 0 && c.kv_heads > 0, REPQ_INVALID_ARG, "%s: num_blocks and kv_heads must be positive", who);
  REPQ_REQUIRE(c.k_codes && c.v_codes && c.k_scale && c.v_scale, REPQ_INVALID_ARG, "%s: NULL cache pointer", who);
  REPQ_REQUIRE(c.block_size == 16 || c.block_size == 32 || c.block_size == 64 || c.block_size == 128, REPQ_UNSUPPORTED,
               "%s: block_size %d is not 16, 32, 64 or 128", who, c.block_size);
  REPQ_REQUIRE(c.d_h >= 16 && c.d_h <= 128 && c.d_h % 16 == 0, REPQ_UNSUPPORTED, "%s: d_h %d is not a multiple of 16 up to 128", who, c.d_h);
  REPQ_REQUIRE(int64_t(c.num_blocks) * c.block_size <= INT32_MAX, REPQ_UNSUPPORTED, "%s: slots of the cache pass 32 bits", who);
  REPQ_REQUIRE(int64_t(c.num_blocks) * c.kv_heads <= INT32_MAX, REPQ_UNSUPPORTED, "%s: scales of the cache pass 32 bits", who);
  REPQ_REQUIRE(int64_t(c.num_blocks) * c.kv_heads * c.block_size * c.d_h < (int64_t(1) << 36), REPQ_UNSUPPORTED, "%s: K or V codes of 64 GiB", who);
  REPQ_REQUIRE(aligned(c.k_codes, 16) && aligned(c.v_codes, 16) && aligned(c.k_scale, 4) && aligned(c.v_scale, 4), REPQ_ALIGNMENT,
               "%s: cache codes must be 16-byte aligned", who);
  return REPQ_OK;
}

namespace {

// ---- plan.  What it costs is the latency of a few dependent reads (8 us for 300 requests and as many as 8000 tokens), so there is one kernel and nothing for its CTAs to wait on: every CTA forms the two
// prefix sums (tokens, fresh blocks) over all requests for itself, and then writes its share of the slots, CTA 0 and its neighbours also the table entries of
// their share of the requests.
constexpr int kPlanThreads = 512;
constexpr int kPlanSlots = 2048;                 // slots of a CTA

__device__ __forceinline__ int ceil_div_pow2(int n, int shift) { return (n >> shift) + ((n & ((1 << shift) - 1)) != 0); }

struct PlanOne { int kv, q, old_blocks, fresh, lost; };
__device__ __forceinline__ PlanOne plan_one(const repq_cache_plan_desc& d, int b, int shift) {
  PlanOne o;
  o.kv = max(__ldg(d.kv_lens + b), 0);
  o.q = max(__ldg(d.q_lens + b), 0);
  o.old_blocks = ceil_div_pow2(o.kv, shift);
  const int all = ceil_div_pow2(o.kv + o.q, shift), in = min(all, d.table_width);
  o.fresh = max(in - o.old_blocks, 0);
  o.lost = max(all - max(in, o.old_blocks), 0);
  return o;
}

__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(const __grid_constant__ repq_cache_plan_desc d, int shift) {
  __shared__ int first_token[kPlanThreads + 1], first_block[kPlanThreads];
  __shared__ int warp_sums[4][kPlanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dependency_wait();
  grid_dependency_trigger();
  const int per = (d.requests + kPlanThreads - 1) / kPlanThreads;        // consecutive requests of a thread
  const int b0 = min(tid * per, d.requests), b1 = min(b0 + per, d.requests);
  int tokens = 0, blocks = 0, lost = 0, longest = 0;
  for (int b = b0; b < b1; ++b) {
    const PlanOne o = plan_one(d, b, shift);
    tokens += o.q;
    blocks += o.fresh;
    lost += o.lost;
    longest = max(longest, o.kv + o.q);
  }
  int st = tokens, sb = blocks;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, st, o), c = __shfl_up_sync(0xffffffffu, sb, o);
    if (lane >= o) { st += a; sb += c; }
  }
  lost = __reduce_add_sync(0xffffffffu, lost);
  longest = __reduce_max_sync(0xffffffffu, longest);
  if (lane == 31) { warp_sums[0][warp] = st; warp_sums[1][warp] = sb; warp_sums[2][warp] = lost; warp_sums[3][warp] = longest; }
  __syncthreads();
  int before_t = 0, before_b = 0, total_t = 0, total_b = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    const int a = warp_sums[0][w], c = warp_sums[1][w];
    if (w < warp) { before_t += a; before_b += c; }
    total_t += a;
    total_b += c;
  }
  st += before_t - tokens;                       // sums before this thread's requests
  sb += before_b - blocks;
  first_token[tid] = st;
  first_block[tid] = sb;
  const int head = min(max(__ldg(d.free_head), 0), d.free_blocks);
  const int room = d.free_blocks - head;         // entries that are left
  if (blockIdx.x == 0) {
    int t = st;
    for (int b = b0; b < b1; ++b) {
      const PlanOne o = plan_one(d, b, shift);
      d.cu_q[b] = t;
      d.kv_lens_out[b] = o.kv + o.q;
      t += o.q;
    }
    if (tid == 0) {
      d.cu_q[d.requests] = total_t;
      d.free_head_out[0] = head + min(total_b, room);
      if (d.totals) {
        int missing = 0, most = 0;
        for (int w = 0; w < kPlanThreads / 32; ++w) { missing += warp_sums[2][w]; most = max(most, warp_sums[3][w]); }
        d.totals[0] = total_t;
        d.totals[1] = min(total_b, room);
        d.totals[2] = missing + max(total_b - room, 0);
        d.totals[3] = most;
      }
    }
  }
  // fresh table entries: the groups of consecutive requests of the threads, dealt to the CTAs; a thread writes those of its own group
  if (tid % gridDim.x == blockIdx.x) {
    int e = sb;
    for (int b = b0; b < b1; ++b) {
      const PlanOne o = plan_one(d, b, shift);
      int32_t* row = d.block_table + b * d.ld_table + o.old_blocks;
      for (int i = 0; i < o.fresh; ++i, ++e) row[i] = e < room ? __ldg(d.free_list + head + e) : -1;
    }
  }
  __syncthreads();
  const int s0 = blockIdx.x * kPlanSlots;
  for (int s = s0 + tid; s < min(s0 + kPlanSlots, d.slots); s += kPlanThreads) {
    int slot = -1, pos = -1;
    if (s < total_t) {
      int lo = 0, hi = kPlanThreads - 1;         // the last group that starts at or before s
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first_token[mid] <= s) lo = mid; else hi = mid - 1;
      }
      int t = first_token[lo], e = first_block[lo], b = lo * per;
      PlanOne o = plan_one(d, b, shift);
      while (s >= t + o.q) {
        t += o.q;
        e += o.fresh;
        o = plan_one(d, ++b, shift);
      }
      pos = o.kv + s - t;
      const int j = pos >> shift;
      int page = -1;
      if (j < d.table_width) {
        if (j < o.old_blocks) page = d.block_table[b * d.ld_table + j];
        else if (e + j - o.old_blocks < room) page = __ldg(d.free_list + head + e + j - o.old_blocks);
      }
      if (page >= 0) slot = (page << shift) + (pos & ((1 << shift) - 1));
    }
    d.slot_map[s] = slot;
    if (d.positions) d.positions[s] = pos;
  }
}

// ---- write.  Bytes are all there is to it (a row read, a row of codes written), but a block's scale needs all of the rows that it gets ("run": rows
// of consecutive slots in one block).  A CTA takes a window of tokens and K or V of one head; the window's runs are found by a vote.  A run that
// fits a warp's registers (16 rows of 128 channels) is a warp's; a longer one is shared by the CTA's warps, which join their
// maxima in shared memory.  Either way every row is read once, all its loads in flight together (a run per warp whatever its length, read
// twice where it did not fit: 75 us for 2400 tokens of 32 heads of 128 channels in blocks of 64, 33 now, 26 back to back).  The bytes of that take 9 us at the memory's
// rate; what bounds it now is 20 instructions an element (issue slots busy 54 %) and the latency of slot map, scale and rows one after the other.
constexpr int kHeld = 8;                          // pieces of eight elements that a thread holds
constexpr int kMostWindow = 64;

struct WriteParams {
  repq_cache c;
  const void* x[2];
  int64_t st[2], sh[2];
  const int32_t* slots;
  int tokens, shift, window;
  int pieces, by_pieces;                          // pieces of a row; n / pieces = n * by_pieces >> 16 for n < 2048
};

// round(x / s) to a code, as the IEEE quotient rounds, a NaN to 128 ...
__device__ __forceinline__ uint32_t exact_code(float x, float s) {
  const float q = fminf(fmaxf(rintf(__fdiv_rn(x, s)), -127.f), 127.f);
  return x == x ? uint32_t(int(q) + 128) : 128u;
}
static __device__ __noinline__ uint2 exact_codes(float4 a, float4 b, float s) {
  return make_uint2(exact_code(a.x, s) | exact_code(a.y, s) << 8 | exact_code(a.z, s) << 16 | exact_code(a.w, s) << 24,
                    exact_code(b.x, s) | exact_code(b.y, s) << 8 | exact_code(b.z, s) << 16 | exact_code(b.w, s) << 24);
}
// ... of eight elements: x * (1 / s) is within 2^-15 of the quotient where codes are, so only pieces with a value near a tie (or an infinity
// or NaN) are divided, one in some 600; all other roundings are those of the float adder (1.5 * 2^23 + 128, whose low byte is the code).
// (A division of every element inlined: 38 instructions an element, 49 us for what takes 9 at the memory's rate.)
__device__ __forceinline__ uint2 codes_of(const float (&f)[8], float s, float inv) {
  constexpr float kMagic = 12582912.f + 128.f;
  const f32x2 inv2 = splat2(inv), up = splat2(kMagic), down = splat2(-kMagic);
  uint32_t u[8];
  float far = 0.f;                                 // from the code, the farthest of them
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f32x2 t = mul2(pack2(f[2 * k], f[2 * k + 1]), inv2), q = add2(t, up), off = fma2(add2(q, down), splat2(-1.f), t);
    float q0, q1, o0, o1;
    unpack2(q, q0, q1);
    unpack2(off, o0, o1);
    asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(far) : "f"(fabsf(o0)), "f"(fabsf(o1)));
    u[2 * k] = __float_as_uint(q0);
    u[2 * k + 1] = __float_as_uint(q1);
  }
  if (!(far < 0.4999f)) return exact_codes(make_float4(f[0], f[1], f[2], f[3]), make_float4(f[4], f[5], f[6], f[7]), s);
  return make_uint2(__byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(u[4], u[5], 0x0040), __byte_perm(u[6], u[7], 0x0040), 0x5410));
}

template <typename T> struct Piece;               // eight elements
template <> struct Piece<__nv_bfloat16> {
  uint4 r;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() { r = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  // largest magnitude (NaN left out)
  __device__ __forceinline__ float top() const {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&r);
    const __nv_bfloat162 m = __hmax2(__hmax2(__habs2(h[0]), __habs2(h[1])), __hmax2(__habs2(h[2]), __habs2(h[3])));
    return fmaxf(__low2float(m), __high2float(m));
  }
};
template <> struct Piece<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ float top() const {
    return fmaxf(fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(a.z), fabsf(a.w))), fmaxf(fmaxf(fabsf(b.x), fabsf(b.y)), fmaxf(fabsf(b.z), fabsf(b.w))));
  }
};

// A run's rows, by `kThreads` threads of which this is number `t`: a warp, or the whole CTA (`tops`: a word per warp in shared memory).
template <typename T, int kThreads, bool kEven>
__device__ __forceinline__ void write_run(const WriteParams& P, int head, int kv, int t0, int slot0, int rows, int t, uint32_t* tops) {
  const int lane = t & 31, bs = 1 << P.shift, off = slot0 & (bs - 1), page = slot0 >> P.shift;
  const int64_t tile = int64_t(page) * P.c.kv_heads + head;
  const int64_t st = kv ? P.st[1] : P.st[0];
  const T* x = static_cast<const T*>(kv ? P.x[1] : P.x[0]) + head * (kv ? P.sh[1] : P.sh[0]) + t0 * st;
  uint8_t* codes = (kv ? P.c.v_codes : P.c.k_codes) + (tile << P.shift) * P.c.d_h;
  float* scale = (kv ? P.c.v_scale : P.c.k_scale) + tile;
  const int n = rows * P.pieces;
  // (kEven: the threads' pieces of a row are whole rows, so a thread's pieces lie at a fixed step)
  const T* x0 = x + (t * P.by_pieces >> 16) * st + 8 * (t - (t * P.by_pieces >> 16) * P.pieces);
  const int64_t step = (kThreads * P.by_pieces >> 16) * st;
  Piece<T> held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int e = t + kThreads * i;
    if (e < n) held[i].load(kEven ? x0 + i * step : x + (e * P.by_pieces >> 16) * st + 8 * (e - (e * P.by_pieces >> 16) * P.pieces));
    else held[i].clear();
  }
  const float before = off ? *scale : 0.f;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) top = fmaxf(top, held[i].top());
  top = fminf(top, 3.402823466e38f);
  // (magnitudes order as their bits do)
  uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
  if (kThreads > 32) {
    if (lane == 0) tops[t >> 5] = bits;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) bits = max(bits, tops[w]);
  }
  const float after = fmaxf(before, fmaxf(__fmul_rn(__uint_as_float(bits), 1.0f / 127.0f), 0x1p-60f));
  if (after > before) {
    if (off) {                                     // the block's earlier rows move to the wider scale
      const float ratio = __fdiv_rn(before, after);
      uint32_t* w = reinterpret_cast<uint32_t*>(codes);
#pragma unroll 1
      for (int e = t; e < (off * P.c.d_h) >> 2; e += kThreads) {
        const uint32_t u = w[e];
        uint32_t o = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float c = fminf(fmaxf(rintf(__fmul_rn(float(int((u >> (8 * k)) & 255u) - 128), ratio)), -127.f), 127.f);
          o |= uint32_t(int(c) + 128) << (8 * k);
        }
        w[e] = o;
      }
    }
    if (kThreads > 32) __syncthreads();            // (every warp has read the scale)
    if (t == 0) *scale = after;
  }
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(after));
  uint2* to = reinterpret_cast<uint2*>(codes + off * P.c.d_h);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int e = t + kThreads * i;
    if (e >= n) break;
    float f[8];
    held[i].get(f);
    to[e] = codes_of(f, after, inv);               // (rows of codes are dense: piece e of the run is 8 e bytes in)
  }
}

template <typename T, int kThreads, bool kEven>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 768 / kThreads : 512 / kThreads) cache_write_kernel(const __grid_constant__ WriteParams P) {
  constexpr int kWarps = kThreads / 32, kFits = 32 * kHeld;             // pieces of a warp
  __shared__ uint32_t tops[2][kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int head = blockIdx.y, kv = blockIdx.z, bs = 1 << P.shift;
  const int t_end = min((int(blockIdx.x) + 1) * P.window, P.tokens);
  const int64_t slots = int64_t(P.c.num_blocks) << P.shift;
  grid_dependency_wait();
  grid_dependency_trigger();
  // (every warp finds the runs for itself: no barriers)
  int nth = 0, shared = 0;
#pragma unroll 1
  for (int w0 = int(blockIdx.x) * P.window; w0 < t_end; w0 += 32) {
    const int t = w0 + lane;
    const int s = t < P.tokens ? __ldg(P.slots + t) : -1, edge = lane == 0 && t > 0 && t < P.tokens ? __ldg(P.slots + t - 1) : -2;
    int ahead = __shfl_up_sync(0xffffffffu, s, 1);
    if (lane == 0) ahead = edge;
    const bool there = s >= 0 && s < slots, starts = there && ((s & (bs - 1)) == 0 || ahead != s - 1);
    uint32_t todo = __ballot_sync(0xffffffffu, starts && t < t_end);
    const uint32_t breaks = __ballot_sync(0xffffffffu, starts || !there);
#pragma unroll 1
    while (todo) {
      const int l0 = __ffs(todo) - 1, t0 = w0 + l0;
      todo &= todo - 1;
      const int slot0 = __shfl_sync(0xffffffffu, s, l0);
      const uint32_t after = l0 == 31 ? 0u : breaks >> (l0 + 1);
      int rows = after ? __ffs(after) : 32 - l0;   // up to what breaks the run, or to the end of these tokens
      if (!after) {
        const int most = min(bs - (slot0 & (bs - 1)), P.tokens - t0);
#pragma unroll 1
        for (; rows < most; rows += 32) {
          const bool in = rows + lane < most && __ldg(P.slots + t0 + rows + lane) == slot0 + rows + lane;
          const uint32_t m = ~__ballot_sync(0xffffffffu, in);
          if (m) { rows += __ffs(m) - 1; break; }
        }
        rows = min(rows, most);
      }
      if (rows * P.pieces <= kFits) {
        if (nth++ % kWarps == warp) write_run<T, 32, kEven>(P, head, kv, t0, slot0, rows, lane, nullptr);
      } else {
        // (two sets of words in turn: a warp may be a run ahead of those that still read)
        write_run<T, kThreads, kEven>(P, head, kv, t0, slot0, rows, tid, tops[shared++ & 1]);
      }
    }
  }
}

template <typename T>
repq_status launch_write(const WriteParams& P, cudaStream_t st) {
  const dim3 grid((P.tokens + P.window - 1) / P.window, P.c.kv_heads, 2);
  // four warps hold 64 rows of 128 channels
  const bool even = 32 % P.pieces == 0;
  if (P.shift <= 6 && even) REPQ_CUDA(launch_chained(cache_write_kernel<T, 128, true>, grid, dim3(128), 0, st, P));
  else if (P.shift <= 6) REPQ_CUDA(launch_chained(cache_write_kernel<T, 128, false>, grid, dim3(128), 0, st, P));
  else if (even) REPQ_CUDA(launch_chained(cache_write_kernel<T, 256, true>, grid, dim3(256), 0, st, P));
  else REPQ_CUDA(launch_chained(cache_write_kernel<T, 256, false>, grid, dim3(256), 0, st, P));
  note_launch();
  return REPQ_OK;
}

}  // namespace
}  // namespace cache
}  // namespace repq

using namespace repq;

extern "C" repq_status repq_cache_plan(const repq_cache_plan_desc* d, void* stream) {
  REPQ_REQUIRE(d != nullptr, REPQ_INVALID_ARG, "repq_cache_plan: NULL descriptor");
  REPQ_REQUIRE(d->requests >= 0 && d->table_width >= 0 && d->free_blocks >= 0 && d->slots >= 0, REPQ_INVALID_ARG,
               "repq_cache_plan: negative size");
  const int bs = d->block_size;
  REPQ_REQUIRE(bs == 16 || bs == 32 || bs == 64 || bs == 128, REPQ_UNSUPPORTED, "repq_cache_plan: block_size %d is not 16, 32, 64 or 128", bs);
  REPQ_REQUIRE(d->cu_q && d->free_head && d->free_head_out, REPQ_INVALID_ARG, "repq_cache_plan: NULL pointer");
  REPQ_REQUIRE(d->requests == 0 || (d->kv_lens && d->q_lens && d->kv_lens_out), REPQ_INVALID_ARG, "repq_cache_plan: NULL lengths");
  REPQ_REQUIRE(d->requests == 0 || (d->kv_lens_out != d->kv_lens && d->kv_lens_out != d->q_lens), REPQ_INVALID_ARG,
               "repq_cache_plan: kv_lens_out must not be an input (every CTA reads all lengths)");
  REPQ_REQUIRE(d->free_head_out != d->free_head, REPQ_INVALID_ARG, "repq_cache_plan: free_head_out must not be free_head");
  REPQ_REQUIRE(d->table_width == 0 || d->requests == 0 || d->block_table, REPQ_INVALID_ARG, "repq_cache_plan: NULL block_table");
  REPQ_REQUIRE(d->free_blocks == 0 || d->free_list, REPQ_INVALID_ARG, "repq_cache_plan: NULL free_list");
  REPQ_REQUIRE(d->slots == 0 || d->slot_map, REPQ_INVALID_ARG, "repq_cache_plan: NULL slot_map");
  REPQ_REQUIRE(d->ld_table >= d->table_width, REPQ_INVALID_ARG, "repq_cache_plan: ld_table is smaller than table_width");
  const int shift = bs == 16 ? 4 : bs == 32 ? 5 : bs == 64 ? 6 : 7;
  const int grid = d->slots > cache::kPlanSlots ? (d->slots + cache::kPlanSlots - 1) / cache::kPlanSlots : 1;
  REPQ_CUDA(launch_chained(cache::cache_plan_kernel, dim3(grid), dim3(cache::kPlanThreads), 0, static_cast<cudaStream_t>(stream), *d, shift));
  note_launch();
  return REPQ_OK;
}

extern "C" repq_status repq_cache_write(const repq_cache_write_desc* d, void* stream) {
  REPQ_REQUIRE(d != nullptr, REPQ_INVALID_ARG, "repq_cache_write: NULL descriptor");
  REPQ_TRY(cache::check(d->cache, "repq_cache_write"));
  REPQ_REQUIRE(d->tokens >= 0, REPQ_INVALID_ARG, "repq_cache_write: negative number of tokens");
  REPQ_REQUIRE(d->dtype == REPQ_F32 || d->dtype == REPQ_BF16, REPQ_INVALID_ARG, "repq_cache_write: dtype %d", d->dtype);
  if (d->tokens == 0) return REPQ_OK;
  REPQ_REQUIRE(d->k && d->v && d->slot_map, REPQ_INVALID_ARG, "repq_cache_write: NULL pointer");
  const int64_t unit = d->dtype == REPQ_F32 ? 4 : 2;
  REPQ_REQUIRE(aligned(d->k, 16) && aligned(d->v, 16) && (d->k_stride_token | d->k_stride_head | d->v_stride_token | d->v_stride_head) * unit % 16 == 0,
               REPQ_ALIGNMENT, "repq_cache_write: rows of k and v must be 16-byte aligned");
  cache::WriteParams P;
  P.c = d->cache;
  P.x[0] = d->k; P.st[0] = d->k_stride_token; P.sh[0] = d->k_stride_head;
  P.x[1] = d->v; P.st[1] = d->v_stride_token; P.sh[1] = d->v_stride_head;
  P.slots = d->slot_map;
  P.tokens = d->tokens;
  P.shift = cache::log2_block(d->cache.block_size);
  P.pieces = d->cache.d_h / 8;
  P.by_pieces = (65536 + P.pieces - 1) / P.pieces;
  // windows such that there are some sixteen CTAs per SM, of 64 tokens at most (2400 tokens of 32 heads: 33 us with windows of 64, 36 with 128,
  // 51 with 4); four tokens where there are few (a warp each; 64 single tokens of 32 heads 11 us, 31 with one window)
  const int64_t per = int64_t(d->tokens) * d->cache.kv_heads / (int64_t(sm_count()) * 8);
  P.window = 4;
  while (P.window < per && P.window < cache::kMostWindow) P.window *= 2;
  REPQ_REQUIRE(d->cache.kv_heads <= 65535, REPQ_UNSUPPORTED, "repq_cache_write: too many heads");
  return d->dtype == REPQ_F32 ? cache::launch_write<float>(P, static_cast<cudaStream_t>(stream))
                              : cache::launch_write<__nv_bfloat16>(P, static_cast<cudaStream_t>(stream));
}
