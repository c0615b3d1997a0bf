// What decode over the bf16 cache and over the 8-bit cache have in common: the list of K/V rows and the blocks' places in it, the
// merge of pieces, the groups of layers that share a donor, the workspace.  (kvp_decode.cu describes the design.)
#pragma once
#include <math.h>

#include <algorithm>

#include "kvp_deal.h"
#include "kvp_host.h"
#include "kvp_sm100.cuh"

namespace kvp {
namespace {

constexpr int GRAN = 16;           // tokens per ring stage
constexpr int MAX_DEC_GROUPS = 64, FEW_DEC_GROUPS = 8;   // a launch of few groups has a parameter block of 1 KB, not 8: 0.6 us less to launch
constexpr int MAX_MEMBERS = 4;     // layers of a donor group served by one pass (rows = members * G <= 16)

struct DecSizes {
  const int32_t* block_table;  // [B, max_pages]
  const int32_t* lengths;      // [B]
  float* part_o;               // [pieces][rows][DH]
  float* part_ml;              // [pieces][rows][2]
  int rows;                    // query rows of the largest group
  int n_groups, B, Hq, Hkv, page_size, max_pages, n_pages;
  int fit;                     // blocks that fit on the device
  int max_shares;              // most shares of the list
  int by_units;                // the lists are short at any length: whole units are dealt out, no sums are formed
  int num_splits;              // > 0: the caller's split count instead; a block is one (unit, split)
  int io_f32;                  // queries are read and outputs written as fp32 (rounded to bf16 on load / widened on store)
  float scale_log2;
};

__device__ __forceinline__ int clamp_length(const DecSizes& p, int len) { return min(max(len, 1), p.max_pages * p.page_size); }
__device__ __forceinline__ int clamped_length(const DecSizes& p, int b) { return clamp_length(p, p.lengths[b]); }
__device__ __forceinline__ int granules_of(int len) { return (len + GRAN - 1) / GRAN; }

// Over the batch, formed by one warp: granules (of one KV head) of the sequences before b_before, of all, and of the longest.
// len0: the length (unclamped) of the lane's sequence among the first 32.
__device__ __forceinline__ void sum_granules(const DecSizes& p, int len0, int b_before, int& before, int& all, int& longest) {
  const int lane = threadIdx.x & 31;
  int sum = 0, most = 0, first = 0;
  for (int b = lane; b < p.B; b += 32) {
    const int n = granules_of(clamp_length(p, b < 32 ? len0 : p.lengths[b]));
    sum += n;
    most = max(most, n);
    first += b < b_before ? n : 0;
  }
  all = __reduce_add_sync(0xffffffffu, sum);
  longest = __reduce_max_sync(0xffffffffu, most);
  before = b_before > 0 ? __reduce_add_sync(0xffffffffu, first) : 0;
}
// The lengths of the first 32 sequences, one a lane, before the kernels ahead have finished (through L2: no line of them may
// stay in L1, later loads must see what those kernels write).  What was worked out from them holds if they are still the same
// behind the wait, and is worked out again if not: the lengths of a step are in place long before.  Batches of more than 32
// only look behind it.  (From the wait to a block's first data went 4.2 to 6 us, most of it this arithmetic out of a cold
// instruction cache.  Append, decode and merge, us: 8 sequences of 8K-16K in four layers 133.4 -> 130.0, 15 of 2K-4K in six
// 40.5 -> 37.0, 8 of 12K in five 67.3 -> 63.3, 28 of 1000 in three 30.4 -> 28.3.)
__device__ __forceinline__ int early_length(const DecSizes& p) {
  const int lane = threadIdx.x & 31;
  return lane < p.B ? __ldcg(p.lengths + lane) : 0;
}
// The first T mod n of n shares of a list of T granules hold one more than the others.
struct Dealt {
  uint32_t q, r;
  __device__ __forceinline__ Dealt(long long total, uint32_t n) : q(uint32_t(div_places(total, n))), r(uint32_t(total - (long long)q * n)) {}
  __device__ __forceinline__ long long begin(uint32_t i) const { return (long long)i * q + min(i, r); }
  __device__ __forceinline__ uint32_t size(uint32_t i) const { return q + (i < r ? 1u : 0u); }
  __device__ __forceinline__ int share_of(long long g) const {
    const long long longer = (long long)r * (q + 1);
    return g < longer ? int(div_places(g, q + 1)) : int(r + div_places(g - longer, q));
  }
};

// 16-byte asynchronous copy; with src_bytes == 0 nothing is read and the destination is filled with zeros
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ln(l 2^m), with the sum of the two logarithms and the constant kept to twice the precision before the only rounding
__device__ __forceinline__ float log_sum(float m, float l) {
  const float t = log2f(l), s = m + t, b = s - m;
  const float low = (m - (s - b)) + (t - b);          // s + low == m + t
  constexpr double kLn2 = 0.693147180559945309417;
  constexpr float hi = float(kLn2), lo = float(kLn2 - double(hi));
  return fmaf(s, hi, fmaf(s, lo, low * hi));
}

// All shares alike
template <int DH>
struct EvenDeal : Dealt {
  static __device__ __forceinline__ int shares(const DecSizes& p, long long total) { return shares_for(DH, p.fit, p.max_shares, total); }
  __device__ __forceinline__ EvenDeal(const DecSizes&, long long total, int n) : Dealt(total, n) {}
};

// Merges the pieces of the units that more than one share holds and writes bf16 outputs and LSE.  Eight warps per block;
// `wpr` of them share a row of a unit (one where a unit has few pieces, eight where it has many), each lane four
// columns.  Bound: latency; the pieces are in L2.
constexpr int COMBINE_THREADS = 256;
// EMPTY: there may be units without a token, whose pieces have no sum: output 0, LSE -infinity.
template <int DH, bool EMPTY, typename Params, typename Deal = EvenDeal<DH>>
__global__ void __launch_bounds__(COMBINE_THREADS) decode_combine_kernel(const __grid_constant__ Params p, int wpr) {
  constexpr int LANES = DH / 4;               // lanes per piece and row
  constexpr int PER_WARP = 32 / LANES;        // pieces a warp takes at a time
  __shared__ float s_m[COMBINE_THREADS / 32], s_l[COMBINE_THREADS / 32];
  __shared__ float4 s_o[COMBINE_THREADS / 32][LANES];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rows_per_block = (COMBINE_THREADS / 32) / wpr;
  const int G = p.Hq / p.Hkv;
  const int unit = blockIdx.x;
  const int hk = unit % p.Hkv, b = unit / p.Hkv % p.B, gi = unit / p.Hkv / p.B;
  const auto& grp = p.grp[gi];
  const int R = grp.n_members * G;
  const int row = blockIdx.y * rows_per_block + warp / wpr;
  grid_dep_launch();
  int w0 = 0, w1 = 0;                         // shares (or splits) that hold the unit
  if (p.num_splits > 0) {
    w0 = unit * p.num_splits;
    w1 = w0 + p.num_splits - 1;
    grid_dep_wait();
  } else {
    int len0 = 0;
    for (bool behind = p.B > 32;; behind = true) {
      if (behind) grid_dep_wait();
      const int now = early_length(p);
      if (behind && p.B <= 32 && __all_sync(0xffffffffu, now == len0)) break;
      len0 = now;
      int before, all, longest;
      sum_granules(p, len0, b, before, all, longest);
      const long long granules = (long long)all * p.Hkv * p.n_groups;
      if (dealt_by_units(DH, granules, (long long)p.n_groups * p.B * p.Hkv, longest, p.fit)) {
        w0 = w1 = 0;                          // finished by the blocks that held them
      } else {
        const int len = b < 32 ? __shfl_sync(0xffffffffu, len0, b) : p.lengths[b];
        const int rest = unit_rest(DH, granules, p.fit), ng = granules_of(clamp_length(p, len));
        const long long per_group = ((long long)all + (long long)p.B * rest) * p.Hkv, total = per_group * p.n_groups;
        const int n = Deal::shares(p, total);
        const long long first = gi * per_group + ((long long)before + (long long)b * rest) * p.Hkv + (long long)hk * (ng + rest);
        const Deal dealt(p, total, n);
        w0 = dealt.share_of(first);
        w1 = dealt.share_of(first + ng - 1);
      }
      if (behind) break;
    }
    if (w0 == w1) return;                     // finished by the block that had the share
  }
  if (blockIdx.y * rows_per_block >= R) return;
  const int sub = lane / LANES, col = (lane % LANES) * 4;
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (row < R) {
    constexpr int UNROLL = 4;                 // pieces in flight per lane
    const int step = wpr * PER_WARP;
    for (int w = w0 + (warp % wpr) * PER_WARP + sub; w <= w1; w += step * UNROLL) {
      float2 ml[UNROLL];
      float4 o[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int wu = w + u * step;
        ml[u] = make_float2(-INFINITY, 0.f);
        if (wu <= w1) {
          const size_t piece = p.num_splits > 0 ? size_t(wu) : size_t(wu) * 2 + (wu == w0 ? 1 : 0);
          ml[u] = *reinterpret_cast<const float2*>(p.part_ml + (piece * p.rows + row) * 2);
          o[u] = *reinterpret_cast<const float4*>(p.part_o + (piece * p.rows + row) * DH + col);
        }
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (ml[u].x == -INFINITY) continue;   // an empty split
        const float mn = fmaxf(m, ml[u].x);
        const float fa = m == -INFINITY ? 0.f : fast_exp2(m - mn), fb = fast_exp2(ml[u].x - mn);
        acc.x = acc.x * fa + o[u].x * fb;
        acc.y = acc.y * fa + o[u].y * fb;
        acc.z = acc.z * fa + o[u].z * fb;
        acc.w = acc.w * fa + o[u].w * fb;
        l = l * fa + ml[u].y * fb;
        m = mn;
      }
    }
  }
  auto merge = [&](float om, float ol, const float4& oo) {
    if (om == -INFINITY) return;
    const float mn = fmaxf(m, om);
    const float fa = m == -INFINITY ? 0.f : fast_exp2(m - mn), fb = fast_exp2(om - mn);
    acc.x = acc.x * fa + oo.x * fb;
    acc.y = acc.y * fa + oo.y * fb;
    acc.z = acc.z * fa + oo.z * fb;
    acc.w = acc.w * fa + oo.w * fb;
    l = l * fa + ol * fb;
    m = mn;
  };
  if (PER_WARP == 2) {                        // the two halves of the warp hold different pieces
    const float om = __shfl_xor_sync(0xffffffffu, m, 16), ol = __shfl_xor_sync(0xffffffffu, l, 16);
    const float4 oo = make_float4(__shfl_xor_sync(0xffffffffu, acc.x, 16), __shfl_xor_sync(0xffffffffu, acc.y, 16),
                                  __shfl_xor_sync(0xffffffffu, acc.z, 16), __shfl_xor_sync(0xffffffffu, acc.w, 16));
    merge(om, ol, oo);
  }
  if (wpr > 1) {                              // the block's warps hold pieces of one row (uniform: every thread arrives)
    if (lane < LANES) s_o[warp][lane] = acc;
    if (lane == 0) {
      s_m[warp] = m;
      s_l[warp] = l;
    }
    __syncthreads();
    if (warp % wpr != 0) return;
    for (int k = 1; k < wpr; ++k) merge(s_m[warp + k], s_l[warp + k], s_o[warp + k][lane % LANES]);
  }
  if (row < R && lane < LANES) {
    const int mem = row / G;
    const size_t head = size_t(b) * p.Hq + hk * G + row % G;
    const float inv = EMPTY && l == 0.f ? 0.f : 1.f / l;
    const uint2 v = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));   // rounded to bf16 either way
    if (p.io_f32)
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(grp.o[mem]) + head * DH + col) =
          make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
    else
      *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(grp.o[mem]) + head * DH + col) = v;
    if (lane == 0) grp.lse[mem][head] = EMPTY && l == 0.f ? -INFINITY : log_sum(m, l);
  }
}

inline int check_desc(const kvp_decode_desc* d) {
  if (d == nullptr) return KVP_ERR_INVALID_ARG;
  if (d->L < 1 || d->B < 1 || d->Hq < 1 || d->Hkv < 1 || d->max_pages < 1 || d->n_pages < 1 || d->num_splits < 0)
    return KVP_ERR_INVALID_ARG;
  if (d->dtype != KVP_BF16 && d->dtype != KVP_F32) return KVP_ERR_UNSUPPORTED;
  if ((d->dh != 64 && d->dh != 128) || d->Hq % d->Hkv != 0 || d->Hq / d->Hkv > 16 || d->page_size < GRAN ||
      d->page_size % GRAN != 0)
    return KVP_ERR_UNSUPPORTED;
  return KVP_OK;
}

// Sub-groups of at most min(MAX_MEMBERS, 16 / G) layers that share a donor inside [begin, end).
struct SubGroup {
  int owner;
  int members[MAX_MEMBERS];
  int n;
};

inline int build_groups(const kvp_decode_desc* d, const int32_t* donor, int begin, int end, SubGroup* out, int max_out) {
  const int G = d->Hq / d->Hkv;
  int per = 16 / G;
  if (per > MAX_MEMBERS) per = MAX_MEMBERS;
  int n_out = 0;
  for (int own = 0; own < d->L; ++own) {
    if (donor[own] != own) continue;
    SubGroup cur;
    cur.owner = own;
    cur.n = 0;
    for (int l = begin > own ? begin : own; l < end; ++l) {
      if (donor[l] != own) continue;
      cur.members[cur.n++] = l;
      if (cur.n == per) {
        if (n_out == max_out) return -1;
        out[n_out++] = cur;
        cur.n = 0;
      }
    }
    if (cur.n > 0) {
      if (n_out == max_out) return -1;
      out[n_out++] = cur;
    }
  }
  return n_out;
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Pieces and their bytes.  When the library chooses: two for each share of the list at its longest; with the
// caller's split count: one for every (unit, split).  One launch holds at most MAX_DEC_GROUPS sub-groups and launches
// reuse the space.
struct DealBy {
  int fit;      // blocks that fit on the device
  int rounds;   // shares at most, in as many
};
inline size_t piece_bytes(const kvp_decode_desc* d, size_t pieces, int rows) {
  return align256(pieces * rows * d->dh * 4) + align256(pieces * rows * 2 * 4);
}
inline long long longest_unit(const kvp_decode_desc* d) { return (long long)d->max_pages * d->page_size / GRAN; }
inline long long longest_list(const kvp_decode_desc* d, int n_groups) { return (long long)n_groups * d->B * d->Hkv * longest_unit(d); }
struct Scratch {
  int max_shares = 0, rows = 0;
  size_t pieces = 0, bytes = 0;
};
// limit > 0: fewer shares until the pieces fit into that many bytes
inline Scratch plan_scratch(const kvp_decode_desc* d, const SubGroup* subs, int n_sub, size_t limit, DealBy by) {
  Scratch s;
  const int per_launch = n_sub < MAX_DEC_GROUPS ? n_sub : MAX_DEC_GROUPS;
  for (int i = 0; i < n_sub; ++i) s.rows = std::max(s.rows, subs[i].n * (d->Hq / d->Hkv));
  const long long longest = longest_list(d, per_launch);
  s.max_shares = shares_for(d->dh, by.fit, by.fit * by.rounds, longest + (long long)per_launch * d->B * d->Hkv * unit_rest(d->dh, longest, by.fit));
  for (;;) {
    s.pieces = d->num_splits > 0 ? size_t(per_launch) * d->B * d->Hkv * d->num_splits : size_t(s.max_shares) * 2;
    s.bytes = piece_bytes(d, s.pieces, s.rows);
    if (limit == 0 || s.bytes <= limit || d->num_splits > 0 || s.max_shares == 1) return s;
    s.max_shares = (s.max_shares + 1) / 2;
  }
}
// bytes for decoding layers [begin, end); 0 when the request cannot be served at all
inline size_t decode_scratch_bytes(const kvp_decode_desc* d, const int32_t* donor, int begin, int end, DealBy by) {
  static thread_local SubGroup tmp[4096];
  const int n_sub = build_groups(d, donor, begin, end, tmp, 4096);
  return n_sub <= 0 ? 0 : plan_scratch(d, tmp, n_sub, 0, by).bytes;
}

}  // namespace
}  // namespace kvp
