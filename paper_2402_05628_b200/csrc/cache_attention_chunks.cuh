// Attention over the 8-bit cache for chunks of prompts: many rows per key / value head, on tcgen05.
//
// A CTA takes 256 rows of one key / value head of a request (token x group) as two tiles of 128, and walks the keys they see in steps
// of 128.  Four warps turn the codes of a step into f16 tiles of shared memory (code - 128 is exact), K as it comes, V as the MN-major
// operand of the same layout.  Per tile S = Q K^T goes to 128 columns of tensor memory; a thread per row forms weights 16
// columns at a time and writes them, f16, over columns it has read, from where O += P V takes them.  The two tiles alternate: one's
// softmax runs under the other's MMAs.
//
// With x = S alpha k_scale log2 e (queries scaled per row to f16's range by a power of two) and lv = log2 v_scale, both per
// 16 keys, weights are w = 2^(x + lv - m + 7): the value scales go into the exponent, so no product per key is spent on them, and
// the sum is Z = sum w / v_scale, a product per 16 keys.  m follows the largest x + lv of the row at a distance of up to 8, so w
// is at most 2^15 and the accumulator is rescaled rarely; weights have 11 bits down to 2^-21 of the largest.
//
// Items (request, row pair, head; the longest of a request first) are handed out by a counter; where there are fewer of them than SMs, each
// is cut along the keys and joined by the part that finishes last, parts in order.
// Roles: two groups of four softmax warps, four conversion warps, one warp that issues MMAs, one that fetches items.  Every wait is
// bounded; when one runs out all roles leave, MMAs in flight are drained and tensor memory is freed.
#pragma once
#include "cache_attention.cuh"
#include "f32x2.cuh"
#include "tc_ptx.cuh"

namespace repq {
namespace cache {
namespace chunks {

using namespace tc;

constexpr int kTileRows = 128, kPair = 2 * kTileRows, kKeys = 128;
constexpr int kSoftWarps = 8, kConvWarps = 4;
constexpr int kMmaWarp = kSoftWarps + kConvWarps, kItemWarp = kMmaWarp + 1;
constexpr int kThreads = 32 * (kItemWarp + 1);
constexpr float kLift = 7.f, kLag = 8.f;
constexpr float kLn2 = 0.6931471805599453f;

struct Item { int b, h, row0, q0, before, n_rows, j0, end[2], part, id; };   // before: tokens ahead of the request's first query

struct ChunkParams {
  AttendParams a;
  int few;                               // requests of at most this many rows are not this kernel's
  int32_t* tickets;                      // [2]: next item, CTAs that are done
  int32_t* status;
};

template <int kSteps>
struct Shared {
  static constexpr int kBlocks = (kSteps + 3) / 4;                       // blocks of 64 channels
  static constexpr uint32_t kTile = kBlocks * 128 * 128;                 // 128 rows of 128 bytes per block
  alignas(1024) uint8_t q[2][kTile];
  alignas(1024) uint8_t k[2][kTile];
  alignas(1024) uint8_t v[2][kTile];
  float4 scale[4][8];                    // per step (four in turn) and 16 keys: k_scale, log2 v_scale, 1 / v_scale
  Item item[2];
  long long first[kThreads + 1];
  int last[2];
  alignas(8) uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_full[2], s_full[2], p_full[2], pv_done[2], o_empty[2], item_full[2],
      item_empty[2], done;
  uint32_t tmem_base;
  volatile int abort;
};

__device__ __forceinline__ bool wait_for(uint64_t& bar, uint32_t parity, volatile int* abort, int code, int32_t* status) {
  return tc::mbar_wait<false>(smem_u32(&bar), parity & 1u, abort, code, status);
}

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// row pairs of a request (per key / value head)
__device__ __forceinline__ int pairs_of(const ChunkParams& P, const Request& rq) {
  const int rows = rq.q_len * P.a.group;
  return rows > P.few ? (rows + kPair - 1) / kPair : 0;
}

// place of 16-byte piece `c` (eight channels) of row `r` in a swizzled tile
__device__ __forceinline__ uint32_t piece_at(int r, int c) {
  return uint32_t(c >> 3) * (128u * 128u) + uint32_t(r) * 128u + (uint32_t((c ^ r) & 7) << 4);
}

// 16 neighbouring values of an output row.
__device__ __forceinline__ int store16(const AttendParams& P, int token, int head, int d, const float (&v)[16]) {
  const int64_t at = token * P.ldo + head * P.o_sh;
  if (P.out_kind == REPQ_OUT_BF16) {
    uint4* o = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(P.out) + at + d);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    o[0] = make_uint4(w[0], w[1], w[2], w[3]);
    o[1] = make_uint4(w[4], w[5], w[6], w[7]);
    return 0;
  }
  int sum = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += store_pair(P, token, head, d + 2 * i, v[2 * i], v[2 * i + 1]);
  return sum;
}

template <int kSteps>
__global__ void __launch_bounds__(kThreads, 1) cache_chunks_kernel(const __grid_constant__ ChunkParams P) {
  using Sh = Shared<kSteps>;
  constexpr int dh = 16 * kSteps;
  constexpr int kPart = kTileRows * (dh + 2);             // floats of a tile's part
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Sh& S = *reinterpret_cast<Sh*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&S.k_full[i]), kConvWarps);
      mbar_init(smem_u32(&S.k_empty[i]), 1);
      mbar_init(smem_u32(&S.v_full[i]), kConvWarps);
      mbar_init(smem_u32(&S.v_empty[i]), 1);
      mbar_init(smem_u32(&S.q_full[i]), 4);
      mbar_init(smem_u32(&S.s_full[i]), 1);
      mbar_init(smem_u32(&S.p_full[i]), 4);
      mbar_init(smem_u32(&S.pv_done[i]), 1);
      mbar_init(smem_u32(&S.o_empty[i]), 4);
      mbar_init(smem_u32(&S.item_full[i]), 1);
      mbar_init(smem_u32(&S.item_empty[i]), kSoftWarps + kConvWarps + 1);
    }
    mbar_init(smem_u32(&S.done), 1);
    S.abort = 0;
    if (smem_u32(smem_raw) & 1023u) {
      atomicCAS(P.status, 0, 100);
      S.abort = 1;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = S.tmem_base;
  volatile int* abort = &S.abort;
  grid_dependency_wait();
  grid_dependency_trigger();

  // ---- the line of items: requests in order
  const int per = (P.a.requests + kThreads - 1) / kThreads;
  {
    long long n = 0;
    for (int b = tid * per; b < min((tid + 1) * per, P.a.requests); ++b) n += (long long)pairs_of(P, request_of(P.a, b)) * P.a.c.kv_heads;
    long long before = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long a = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += a;
    }
    if (lane == 31) S.first[warp] = before;
    __syncthreads();
    for (int w = 0; w < warp; ++w) before += S.first[w];
    __syncthreads();
    S.first[tid + 1] = before;
    if (tid == 0) S.first[0] = 0;
    __syncthreads();
  }
  const long long items = S.first[kThreads];
  // parts of an item along the keys
  const int parts = items > 0 && items * 2 <= (long long)gridDim.x ? int((long long)gridDim.x / items) : 1;

  // What every role but the fetching warp does with an item: read it, hand the slot back.
  auto next_item = [&](int it, Item& x) {
    if (!wait_for(S.item_full[it & 1], uint32_t(it >> 1), abort, 101, P.status)) { x.b = -1; }
    else x = S.item[it & 1];
    x.b = __shfl_sync(0xffffffffu, x.b, 0);               // (all lanes leave together)
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&S.item_empty[it & 1]));
    return x.b >= 0;
  };

  if (warp == kItemWarp) {
    // ---------------------------------------------------------------- items
    for (int it = 0;; ++it) {
      bool ok = it < 2 || wait_for(S.item_empty[it & 1], uint32_t((it >> 1) - 1), abort, 102, P.status);
      ok = __all_sync(0xffffffffu, ok);
      if (lane == 0) {
        Item x = {};
        x.b = -1;
        const long long ticket = ok ? atomicAdd(P.tickets, 1) : items * parts;
        if (ticket < items * parts) {
          const long long id = ticket / parts;
          int lo = 0, hi = kThreads - 1;
          while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (S.first[mid] <= id) lo = mid; else hi = mid - 1;
          }
          long long start = S.first[lo];
          int b = lo * per;
          Request rq = request_of(P.a, b);
          int pairs = pairs_of(P, rq);
          while (id >= start + (long long)pairs * P.a.c.kv_heads) {
            start += (long long)pairs * P.a.c.kv_heads;
            rq = request_of(P.a, ++b);
            pairs = pairs_of(P, rq);
          }
          const int local = int(id - start), up = local / P.a.c.kv_heads;
          x.b = b;
          x.h = local - up * P.a.c.kv_heads;
          x.row0 = (pairs - 1 - up) * kPair;
          x.q0 = rq.q0;
          x.before = rq.kv - rq.q_true;
          x.n_rows = rq.q_len * P.a.group;
          x.part = int(ticket - id * parts);
          x.id = int(id);
          int steps[2], most = 0;
          for (int i = 0; i < 2; ++i) {
            const int rows = min(x.n_rows - x.row0 - i * kTileRows, kTileRows);
            const int seen = rows > 0 ? min(min(x.before + (x.row0 + i * kTileRows + rows - 1) / P.a.group + 1, rq.kv), P.a.max_kv) : 0;
            steps[i] = seen > 0 ? (seen + kKeys - 1) / kKeys : 0;
            most = max(most, steps[i]);
          }
          x.j0 = int((long long)most * x.part / parts);
          const int j1 = int((long long)most * (x.part + 1) / parts);
          for (int i = 0; i < 2; ++i) x.end[i] = max(min(steps[i], j1), x.j0);
        }
        S.item[it & 1] = x;
        ok = x.b >= 0;
      }
      ok = __shfl_sync(0xffffffffu, ok, 0);
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&S.item_full[it & 1]));
      if (!ok) break;
    }
    if (lane == 0 && atomicAdd(P.tickets + 1, 1) == int(gridDim.x) - 1) {     // the counters for the next call
      P.tickets[0] = 0;
      P.tickets[1] = 0;
    }
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMAs
    const bool issues = elect_one();
    // D = f32, A and B f16; S: both K-major, N = 128; P V: A in tensor memory, B MN-major, N = d_h
    constexpr uint32_t idesc_s = (1u << 4) | (uint32_t(kKeys >> 3) << 17) | (uint32_t(kTileRows >> 4) << 24);
    constexpr uint32_t idesc_o = (1u << 4) | (1u << 16) | (uint32_t(dh >> 3) << 17) | (uint32_t(kTileRows >> 4) << 24);
    const uint64_t dq0 = smem_desc_sw128(smem_u32(S.q[0])), dk0 = smem_desc_sw128(smem_u32(S.k[0])),
                   dv0 = smem_desc_sw128(smem_u32(S.v[0]), 128 * 128);
    uint32_t kg = 0, vg = 0;                              // steps of K and V taken
    uint32_t ph_q = 0, ph_p = 0, ph_o = 0;                // a bit per tile
    bool ok = true;
    Item x;
    for (int it = 0; ok && next_item(it, x); ++it) {
      const int n = max(x.end[0], x.end[1]) - x.j0;
      if (n <= 0) continue;
      auto issue_s = [&](int i, uint32_t slot) {
        if (issues) {
          const uint64_t a = dq0 + uint64_t(i * (Sh::kTile >> 4)), b = dk0 + uint64_t(slot * (Sh::kTile >> 4));
#pragma unroll
          for (int s = 0; s < kSteps; ++s) {
            const uint32_t off = uint32_t(s >> 2) * (128 * 128 / 16) + uint32_t(s & 3) * 2;
            umma_f16(tmem + uint32_t(i * 128), a + off, b + off, idesc_s, s != 0 ? 1u : 0u);
          }
          umma_commit(smem_u32(&S.s_full[i]));
        }
        __syncwarp();
      };
      // a step's keys: both tiles' S
      auto keys_ready = [&]() {
        ok = ok && wait_for(S.k_full[kg & 1], kg >> 1, abort, 103, P.status);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        return ok;
      };
      if (!keys_ready()) break;
      for (int i = 0; i < 2 && ok; ++i) {
        if (x.end[i] <= x.j0) continue;
        ok = __all_sync(0xffffffffu, wait_for(S.q_full[i], ph_q >> i, abort, 104, P.status));
        if (!ok) break;
        ph_q ^= 1u << i;
        tc_fence_after();
        issue_s(i, kg & 1);
      }
      if (!ok) break;
      if (issues) umma_commit(smem_u32(&S.k_empty[kg & 1]));
      __syncwarp();
      ++kg;
      for (int j = 0; j < n && ok; ++j, ++vg) {
        const bool more = j + 1 < n;
        bool keys = false, values = false;
        for (int i = 0; i < 2; ++i) {
          if (x.j0 + j >= x.end[i]) continue;
          ok = wait_for(S.p_full[i], ph_p >> i, abort, 105, P.status);
          if (ok && !values) { ok = wait_for(S.v_full[vg & 1], vg >> 1, abort, 106, P.status); values = true; }
          if (ok && j == 0) ok = wait_for(S.o_empty[i], (ph_o >> i) ^ 1u, abort, 107, P.status);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          ph_p ^= 1u << i;
          if (j == 0) ph_o ^= 1u << i;
          tc_fence_after();
          if (issues) {
            const uint64_t b = dv0 + uint64_t((vg & 1) * (Sh::kTile >> 4));
#pragma unroll
            for (int s = 0; s < kKeys / 16; ++s)
              umma_f16_ts(tmem + 256u + uint32_t(i * 128), tmem + uint32_t(i * 128 + 8 * s), b + uint64_t(16 * 128 / 16 * s), idesc_o, j != 0 || s != 0 ? 1u : 0u);
            umma_commit(smem_u32(&S.pv_done[i]));
          }
          __syncwarp();
          if (x.j0 + j + 1 < x.end[i]) {
            if (!keys) { if (!keys_ready()) break; keys = true; }
            issue_s(i, kg & 1);
          }
        }
        if (!ok) break;
        if (issues) {
          umma_commit(smem_u32(&S.v_empty[vg & 1]));
          if (more) umma_commit(smem_u32(&S.k_empty[kg & 1]));
        }
        __syncwarp();
        if (more) ++kg;
      }
    }
    if (issues) umma_commit(smem_u32(&S.done));
    __syncwarp();
    mbar_drain(smem_u32(&S.done), 0);
  } else if (warp >= kSoftWarps && warp < kMmaWarp) {
    // ---------------------------------------------------------------- codes to f16 tiles
    const int t = tid - 32 * kSoftWarps;
    constexpr int kPer = kSteps;                          // pieces of 16 codes: 128 rows x kSteps over 128 threads
    const AttendParams& A = P.a;
    uint32_t kg = 0, vg = 0;
    bool ok = true;
    Item x;
    for (int it = 0; ok && next_item(it, x); ++it) {
      const int n = max(x.end[0], x.end[1]) - x.j0;
      if (n <= 0) continue;
      const int32_t* table = A.table + x.b * A.ld_table;
      const int seen = min(min(x.before + (min(x.row0 + kPair, x.n_rows) - 1) / A.group + 1, A.max_kv), int(min((long long)A.table_width << A.shift, (long long)INT32_MAX)));
      int page[kPer];
      auto pages_of = [&](int j) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int key = (x.j0 + j) * kKeys + (i * 128 + t) / kSteps;
          page[i] = key < seen ? __ldg(table + (key >> A.shift)) : -1;
        }
      };
      uint4 raw[kPer];
      auto fetch = [&](const uint8_t* codes, int j) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int e = i * 128 + t, r = e / kSteps, p = e - r * kSteps;
          const int key = (x.j0 + j) * kKeys + r;
          raw[i] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
          if (unsigned(page[i]) < unsigned(A.c.num_blocks)) {
            const int64_t row = ((int64_t(page[i]) * A.c.kv_heads + x.h) << A.shift) + (key & ((1 << A.shift) - 1));
            raw[i] = __ldg(reinterpret_cast<const uint4*>(codes + row * dh) + p);
          }
        }
      };
      auto convert = [&](uint8_t* tile) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int e = i * 128 + t, r = e / kSteps, p = e - r * kSteps;
          const uint4 a = make_uint4(codes_lo(raw[i].x), codes_hi(raw[i].x), codes_lo(raw[i].y), codes_hi(raw[i].y));
          const uint4 b = make_uint4(codes_lo(raw[i].z), codes_hi(raw[i].z), codes_lo(raw[i].w), codes_hi(raw[i].w));
          const bool odd = (p >> 2) & 1;                  // (the second block's lanes write their halves the other way round: no bank conflicts)
          *reinterpret_cast<uint4*>(tile + piece_at(r, 2 * p + (odd ? 1 : 0))) = odd ? b : a;
          *reinterpret_cast<uint4*>(tile + piece_at(r, 2 * p + (odd ? 0 : 1))) = odd ? a : b;
        }
        fence_async_smem();
        __syncwarp();
      };
      // the scales of eight groups of 16 keys
      float4 sc = make_float4(1.f, -CUDART_INF_F, 0.f, 0.f);
      auto fetch_scales = [&](int j) {
        if (t < 8) {
          const int key = (x.j0 + j) * kKeys + 16 * t;
          const int pg = key < seen ? __ldg(table + (key >> A.shift)) : -1;
          sc = make_float4(1.f, -CUDART_INF_F, 0.f, 0.f);                    // (tokens of a missing block weigh nothing)
          if (unsigned(pg) < unsigned(A.c.num_blocks)) {
            const int64_t at = int64_t(pg) * A.c.kv_heads + x.h;
            const float vs = __ldg(A.c.v_scale + at);
            sc = make_float4(__ldg(A.c.k_scale + at), lg2(vs), __fdividef(1.f, vs), 0.f);
          }
        }
      };
      pages_of(0);
      fetch(A.c.k_codes, 0);
      fetch_scales(0);
      for (int j = 0; j < n; ++j) {
        if (!(ok = __all_sync(0xffffffffu, wait_for(S.k_empty[kg & 1], (kg >> 1) ^ 1u, abort, 108, P.status)))) break;
        if (t < 8) S.scale[kg & 3][t] = sc;
        convert(S.k[kg & 1]);
        if (lane == 0) mbar_arrive(smem_u32(&S.k_full[kg & 1]));
        ++kg;
        fetch(A.c.v_codes, j);
        if (j + 1 < n) fetch_scales(j + 1);
        if (!(ok = __all_sync(0xffffffffu, wait_for(S.v_empty[vg & 1], (vg >> 1) ^ 1u, abort, 109, P.status)))) break;
        convert(S.v[vg & 1]);
        if (lane == 0) mbar_arrive(smem_u32(&S.v_full[vg & 1]));
        ++vg;
        if (j + 1 < n) {
          pages_of(j + 1);
          fetch(A.c.k_codes, j + 1);
        }
      }
    }
  } else if (warp < kSoftWarps) {
    // ---------------------------------------------------------------- softmax, a thread per row
    const AttendParams& A = P.a;
    const int i = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lanes = uint32_t(quarter * 32) << 16;
    const uint32_t t_s = tmem + lanes + uint32_t(i * 128), t_o = tmem + lanes + 256u + uint32_t(i * 128);
    uint32_t ph_s = 0, ph_pv = 0;                         // phases waited for
    uint32_t kg = 0;                                      // steps of K in all items (both tiles count alike)
    auto tile_barrier = [&]() {                           // of the tile's four warps
      if (i == 0) asm volatile("bar.sync 1, 128;" ::: "memory");
      else asm volatile("bar.sync 2, 128;" ::: "memory");
    };
    bool ok = true;
    Item x;
    for (int it = 0; ok && next_item(it, x); ++it) {
      const int n_both = max(max(x.end[0], x.end[1]) - x.j0, 0), n = x.end[i] - x.j0;
      const int row = x.row0 + i * kTileRows + r;
      const bool in = row < x.n_rows;
      const int row_token = row / A.group, token = x.q0 + row_token, head = x.h * A.group + row - row_token * A.group;
      const int limit = in ? min(x.before + row_token + 1, A.max_kv) : 0;
      float m = -CUDART_INF_F, z = 0.f;
      if (n > 0) {
        // ---- queries to f16, the row's largest element in [2^8, 2^9)
        float back;
        {
          const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(A.q) + token * A.q_st + head * A.q_sh;
          float top = 0.f;
#pragma unroll 4
          for (int c = 0; c < 2 * kSteps; ++c) {
            const uint4 w = in ? __ldg(reinterpret_cast<const uint4*>(p) + c) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              top = max3(top, __uint_as_float((u[e] << 16) & 0x7fffffffu), __uint_as_float(u[e] & 0x7fff0000u));
          }
          const int e2 = min(max(int(__float_as_uint(top) >> 23) - 127 - 8, -110), 110);
          const float down = __uint_as_float(uint32_t(127 - e2) << 23);
          back = __uint_as_float(uint32_t(127 + e2) << 23) * A.scale;
#pragma unroll 4
          for (int c = 0; c < 2 * kSteps; ++c) {          // (read again, from L1)
            const uint4 w = in ? __ldg(reinterpret_cast<const uint4*>(p) + c) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              h[e] = bits_of(__floats2half2_rn(__uint_as_float(u[e] << 16) * down, __uint_as_float(u[e] & 0xffff0000u) * down));
            *reinterpret_cast<uint4*>(S.q[i] + piece_at(r, c)) = make_uint4(h[0], h[1], h[2], h[3]);
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&S.q_full[i]));
        }
        for (int j = 0; j < n; ++j) {
          if (!(ok = __all_sync(0xffffffffu, wait_for(S.s_full[i], ph_s, abort, 110, P.status)))) break;
          ph_s ^= 1u;
          tc_fence_after();
          const int sees = limit - (x.j0 + j) * kKeys;    // columns of this step
          const bool masked = __any_sync(0xffffffffu, sees < kKeys);
          const float4* scale = S.scale[(kg + j) & 3];
          uint32_t buf[2][16];
          tmem_ld16(t_s, buf[0]);
#pragma unroll
          for (int c = 0; c < kKeys / 16; ++c) {          // 16 keys: a block of tokens, or a part of one
            uint32_t (&s)[16] = buf[c & 1];
            tmem_ld_wait(s);
            if (c + 1 < kKeys / 16) tmem_ld16(t_s + 16u * (c + 1), buf[(c + 1) & 1]);
            if (masked) {
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (16 * c + e >= sees) s[e] = 0xff800000u;
            }
            const float4 g = scale[c];
            const float f = g.x * back;
            float top = __uint_as_float(s[0]);
#pragma unroll
            for (int e = 1; e < 15; e += 2) top = max3(top, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
            top = fmaf(fmaxf(top, __uint_as_float(s[15])), f, g.y);
            if (__any_sync(0xffffffffu, top > m + kLag)) {
              // m rises: what has been summed and written so far is brought down
              if (c + 1 < kKeys / 16) tmem_ld_wait(buf[(c + 1) & 1]);   // (no registers in flight past this point)
              const float up = top > m + kLag ? top : m;
              const float down = m == -CUDART_INF_F ? 0.f : ex2(m - up);
              z *= down;
              m = up;
              const __half2 dh2 = __float2half2_rn(down);
#pragma unroll 1
              for (int b = 0; b < (c + 1) / 2; ++b) {     // (an odd last group's eight columns with what follows them)
                uint32_t w[16];
                tmem_ld16(t_s + 16u * b, w);
                tmem_ld_wait(w);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                  if (16 * b + e < 8 * c) w[e] = bits_of(__hmul2(half2_of(w[e]), dh2));
                tmem_st16(t_s + 16u * b, w);
              }
              if (j > 0) {
                // (the phase of the step before: nothing else waits for it in between)
                if (!(ok = __all_sync(0xffffffffu, wait_for(S.pv_done[i], ph_pv ^ 1u, abort, 111, P.status)))) break;
                tc_fence_after();
#pragma unroll 1
                for (int b = 0; b < kSteps; ++b) {
                  uint32_t w[16];
                  tmem_ld16(t_o + 16u * b, w);
                  tmem_ld_wait(w);
#pragma unroll
                  for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * down);
                  tmem_st16(t_o + 16u * b, w);
                }
              }
              tmem_st_wait();
            }
            const float base = m == -CUDART_INF_F ? 0.f : kLift - m;
            const f32x2 ff = splat2(f), bb = splat2(base + g.y);
            f32x2 sum = splat2(0.f);
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float a, b;
              unpack2(fma2(pack2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), ff, bb), a, b);
              a = ex2(a);
              b = ex2(b);
              sum = add2(sum, pack2(a, b));
              w[e] = bits_of(__floats2half2_rn(a, b));
            }
            float a, b;
            unpack2(sum, a, b);
            z = fmaf(a + b, g.z, z);
            tmem_st8(t_s + 8u * c, w);
          }
          if (!ok) break;
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&S.p_full[i]));
          ph_pv ^= 1u;                                    // this step's completion comes next
        }
        if (!ok) break;
        ok = __all_sync(0xffffffffu, wait_for(S.pv_done[i], ph_pv ^ 1u, abort, 112, P.status));
        if (!ok) break;
        tc_fence_after();
      }
      kg += uint32_t(n_both);

      // ---- the row
      const bool whole = parts == 1;
      float* part = A.partials + (int64_t(x.id) * parts * 2 + x.part * 2 + i) * kPart;
      bool writes = whole;
      if (!whole) {
        if (n > 0) {
#pragma unroll
          for (int b = 0; b < kSteps; ++b) {
            uint32_t w[16];
            tmem_ld16(t_o + 16u * b, w);
            tmem_ld_wait(w);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              __stcg(reinterpret_cast<uint4*>(part) + (4 * b + e) * kTileRows + r, make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]));
          }
        }
        __stcg(reinterpret_cast<float2*>(part + kTileRows * dh) + r, make_float2(n > 0 ? m : -CUDART_INF_F, n > 0 ? z : 0.f));
        __threadfence();
        tile_barrier();
        if (r == 0) {
          const int seen = atomicAdd(A.counters + 2 * x.id + i, 1);
          S.last[i] = seen == parts - 1;
          if (seen == parts - 1) A.counters[2 * x.id + i] = 0;
        }
        tile_barrier();
        writes = S.last[i] != 0;
        if (writes) __threadfence();
      }
      if (writes) {
        const float* p0 = A.partials + (int64_t(x.id) * parts * 2 + i) * kPart;
        float zt = z, mt = m;
        if (!whole) {
          mt = -CUDART_INF_F;
          for (int p = 0; p < parts; ++p) mt = fmaxf(mt, __ldcg(reinterpret_cast<const float2*>(p0 + int64_t(2 * p) * kPart + kTileRows * dh) + r).x);
          zt = 0.f;
          for (int p = 0; p < parts; ++p) {
            const float2 mz = __ldcg(reinterpret_cast<const float2*>(p0 + int64_t(2 * p) * kPart + kTileRows * dh) + r);
            if (mz.x > -CUDART_INF_F) zt = fmaf(ex2(mz.x - mt), mz.y, zt);
          }
        }
        const float inv = zt > 0.f ? __fdividef(1.f, zt) : zt == 0.f ? 0.f : CUDART_NAN_F;
        int sum = 0;
#pragma unroll
        for (int b = 0; b < kSteps; ++b) {
          float v[16];
          if (whole) {
            uint32_t w[16] = {};
            if (n > 0) {
              tmem_ld16(t_o + 16u * b, w);
              tmem_ld_wait(w);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(w[e]) * inv;
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = 0.f;
            for (int p = 0; p < parts; ++p) {
              const float* pp = p0 + int64_t(2 * p) * kPart;
              const float mp = __ldcg(reinterpret_cast<const float2*>(pp + kTileRows * dh) + r).x;
              if (mp == -CUDART_INF_F) continue;          // (saw nothing, wrote nothing)
              const float f = ex2(mp - mt) * inv;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float4 w = __ldcg(reinterpret_cast<const float4*>(pp) + (4 * b + e) * kTileRows + r);
                v[4 * e] = fmaf(f, w.x, v[4 * e]);
                v[4 * e + 1] = fmaf(f, w.y, v[4 * e + 1]);
                v[4 * e + 2] = fmaf(f, w.z, v[4 * e + 2]);
                v[4 * e + 3] = fmaf(f, w.w, v[4 * e + 3]);
              }
            }
          }
          if (in) sum += store16(A, token, head, 16 * b, v);
        }
        if (in && A.out_row_sum) atomicAdd(A.out_row_sum + token, sum);
        if (in && A.lse) A.lse[int64_t(token) * A.heads + head] = zt > 0.f ? (mt - kLift + log2f(zt)) * kLn2 : zt == 0.f ? -CUDART_INF_F : CUDART_NAN_F;
      }
      if (n > 0) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.o_empty[i]));
      }
      __syncwarp();
    }
  }

  // ------------------------------------------------------------------ teardown
  if (warp < kSoftWarps) tmem_st_wait();
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

template <int kSteps>
repq_status launch(const AttendParams& A, const ChunksPlan& plan, int few, void* workspace, cudaStream_t st) {
  constexpr size_t smem = sizeof(Shared<kSteps>);
  static_assert(smem <= 227 * 1024, "shared storage exceeds an SM's");
  REPQ_TRY((allow_smem<cache_chunks_kernel<kSteps>>(int(smem))));
  ChunkParams P;
  P.a = A;
  P.few = few;
  P.tickets = static_cast<int32_t*>(workspace);
  P.a.counters = P.tickets + 2;
  P.a.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + plan.counter_bytes);
  P.status = device_status_word();
  REPQ_REQUIRE(P.status != nullptr, REPQ_CUDA_ERROR, "repq_cache_attention: no device status word");
  REPQ_CUDA(launch_chained(cache_chunks_kernel<kSteps>, dim3(plan.ctas), dim3(kThreads), smem, st, P));
  note_launch();
  return REPQ_OK;
}

}  // namespace chunks
}  // namespace cache
}  // namespace repq
