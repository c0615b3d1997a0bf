// Appending any number of tokens to the paged cache: K rotated by the token's position on the way in, the queries of the same
// tokens rotated beside it, and K and V stored as bf16 or in 8 bits (kvp_cache8.h).  One launch for up to 64 layers.
//
// Bound: HBM for prompts (every element is read and written once, 16 bytes a load), latency for token steps.  Positions are per
// sequence, so the angle is formed on the device: pos times the frequency as a 64-bit fraction of a turn, whose wrap-around is the
// range reduction; sine and cosine are taken of its upper 32 bits as a float, and what that float leaves off is applied as a
// first-order correction.
// Measured (us; in brackets the bytes at the copy rate): prompts of 12000 tokens, four layers, queries with them, bf16 169 to 171 (165), fp32
// 329 (308), bf16 without queries 53 (45); 30400 tokens behind begun blocks into 8 bits 437 to 445 (390), without queries 203 (86: the
// barrier and two heads in flight a block); 32 tokens of eight layers, device time in a graph, 4.5 bf16, 4.8 in 8 bits.
#include <math.h>

#include <algorithm>

#include "kvp_cache8.cuh"
#include "kvp_host.h"
#include "kvp_rope_freq.h"

namespace kvp {
namespace {

constexpr int APP_THREADS = 256;
// Blocks per SM, by registers.  (Token kernel with five, whose last blocks wait for the others: 32 tokens of eight layers 5.4 us instead
// of 4.5.  Runs of 30400 tokens in four layers: dh 64 with four 149 us instead of 136; dh 128 with five, which spills, 462 instead of 433.)
constexpr int ONES_AN_SM = 6, RUNS_A_WAVE = 4;
template <int DH, bool ONE_WAVE>
constexpr int RUNS_AN_SM = DH == 64 && !ONE_WAVE ? 5 : RUNS_A_WAVE;
// Heads that a block of runs has in flight.  (K's and V's in 8 bits: with four, registers spill.)
template <bool BITS8>
constexpr int KV_HEADS = BITS8 ? 2 : 4;
constexpr int Q_HEADS = 4;
constexpr int MANY_LAYERS = 64, FEW_LAYERS = 8;    // a launch of few layers has a parameter block of 1 KB, not 5

struct AppLayer {
  const void* q;                 // [T,Hq,dh] bf16 or (F32) fp32; null: no queries
  void* q_out;
  const void *k_new, *v_new;     // [T,Hkv,dh]; null: a consumer
  void *k_cache, *v_cache;       // [n_pages][Hkv][page_size][dh], bf16 or e4m3
  uint8_t *k_scale, *v_scale;    // [n_pages][Hkv][page_size / 16]
};
struct AppSizes {
  const int32_t* block_table;    // [B, max_pages]
  const int32_t* lengths;        // [B]
  const int32_t* first;          // [B + 1], or null: one token a sequence
  int B, T, Hq, Hkv, page_size, max_pages, n_pages;
  int rotate;
  int kv_slices, q_slices;       // of runs: blocks that share K's and V's heads of a block of positions, and its query heads (0: the same blocks do both)
  uint64_t turns[64];            // rope_turns
};
template <int NL>
struct AppParams : AppSizes {
  AppLayer at[NL];
};

// eight consecutive elements as bf16
template <bool F32>
__device__ __forceinline__ uint4 load_eight(const void* base, size_t at) {
  if constexpr (F32) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
    const float4 a = p[0], b = p[1];
    return make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
  }
  return *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(base) + at);
}
// eight floats rounded to bf16, stored as such or widened
template <bool F32>
__device__ __forceinline__ void store_eight(void* base, size_t at, const float (&f)[8]) {
  const uint4 v = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  if constexpr (F32) {
    float4* p = reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + at);
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
    p[0] = make_float4(lo(v.x), hi(v.x), lo(v.y), hi(v.y));
    p[1] = make_float4(lo(v.z), hi(v.z), lo(v.w), hi(v.w));
  } else {
    *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(base) + at) = v;
  }
}
__device__ __forceinline__ void widen(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// cosine and sine of pos * turns (turns: 64-bit fraction of a turn)
__device__ __forceinline__ float2 turn_of(uint64_t turns, int pos) {
  const int t = int((turns * uint64_t(pos)) >> 32);                  // signed 2^-32 of a turn
  const float a = __int2float_rn(t);
  const float d = float(t - __float2int_rz(a)) * 1.4629180792671596e-9f;   // what a leaves off (up to 64), in radians
  float s, c;
  sincospif(a * 4.656612873077393e-10f, &s, &c);                     // 2^-31 of half a turn
  return make_float2(fmaf(-d, s, c), fmaf(d, c, s));
}
__device__ __forceinline__ void turn_pairs(float (&f)[8], const float2 (&cs)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float a = f[2 * k], b = f[2 * k + 1];
    f[2 * k] = fmaf(a, cs[k].x, -(b * cs[k].y));
    f[2 * k + 1] = fmaf(a, cs[k].y, b * cs[k].x);
  }
}

// Largest finite magnitude, as bits.  What is not finite becomes NaN (e4m3 has no infinity) and does not count.
__device__ __forceinline__ uint32_t finite_amax(float (&f)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t bits = __float_as_uint(f[k]) & 0x7fffffffu;
    if (bits >= 0x7f800000u) f[k] = __uint_as_float(0x7fffffffu);
    else m = max(m, bits);
  }
  return m;
}
__device__ __forceinline__ uint2 quantise(const float (&f)[8], int e) {
  const float s = __uint_as_float(power_bits(-e));
  return make_uint2(f32x4_to_e4m3(f[0] * s, f[1] * s, f[2] * s, f[3] * s), f32x4_to_e4m3(f[4] * s, f[5] * s, f[6] * s, f[7] * s));
}

// One token a sequence.  A head row of DH elements is DH / 8 lanes; a CTA takes 256 / (DH / 8) of the rows of one token and layer
// (K heads, V heads, query heads).  The length, the page and the angles are worked out before the kernels ahead have finished
// (through L2: no line may stay in L1) and again behind the wait if the length or the page is not the same there, so that one
// latency lies between the wait and the stores: the rows, the length, the page and the block's scale are asked for at once.
template <int DH, bool BITS8, bool F32, int NL>
__global__ void __launch_bounds__(APP_THREADS, ONES_AN_SM) append_one_kernel(const __grid_constant__ AppParams<NL> p) {
  constexpr int LANES = DH / 8;
  const AppLayer& at = p.at[blockIdx.y];
  const int b = blockIdx.x, c = threadIdx.x % LANES;
  const int row = blockIdx.z * (APP_THREADS / LANES) + threadIdx.x / LANES;
  grid_dep_launch();
  const int kv_rows = at.k_new != nullptr ? 2 * p.Hkv : 0, rows = kv_rows + (at.q != nullptr ? p.Hq : 0);
  const bool there = row < rows;
  const bool is_q = row >= kv_rows, is_v = !is_q && row >= p.Hkv;
  const int head = is_q ? row - kv_rows : is_v ? row - p.Hkv : row, heads = is_q ? p.Hq : p.Hkv;
  const size_t in = (size_t(b) * heads + head) * DH + c * 8;
  const int cap = p.max_pages * p.page_size;
  float2 cs[4];
  auto angles = [&](int pos) {
    if (!p.rotate) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) cs[k] = turn_of(p.turns[c * 4 + k], pos);
  };
  auto page_at = [&](int pos) { return pos >= 0 && pos < cap ? __ldcg(p.block_table + size_t(b) * p.max_pages + pos / p.page_size) : -1; };
  uint8_t* const scale = BITS8 ? (is_v ? at.v_scale : at.k_scale) : nullptr;
  auto block_of = [&](int page, int pos) {
    return (size_t(page) * p.Hkv + head) * (p.page_size / CACHE_BLOCK) + pos % p.page_size / CACHE_BLOCK;
  };
  auto scale_at = [&](int page, int pos) -> int {        // exponent of a block that older tokens began
    const bool begun = BITS8 && there && !is_q && page >= 0 && page < p.n_pages && pos % CACHE_BLOCK > 0;
    return begun ? exponent_of_byte(scale[block_of(page, pos)]) : LEAST_SCALE;
  };
  int pos = __ldcg(p.lengths + b) - 1;
  int page = page_at(pos);
  angles(pos);
  grid_dep_wait();
  uint4 raw = make_uint4(0u, 0u, 0u, 0u);
  if (there) raw = load_eight<F32>(is_q ? at.q : is_v ? at.v_new : at.k_new, in);
  const int pos_now = p.lengths[b] - 1, page_now = page_at(pos);
  int e_old = scale_at(page, pos);
  if (pos_now != pos || page_now != page) {              // (the whole block)
    pos = pos_now;
    page = page_at(pos);
    angles(pos);
    e_old = scale_at(page, pos);
  }
  if (pos < 0 || pos >= cap) return;                     // (the whole block)
  const bool stored = there && !is_q && page >= 0 && page < p.n_pages;
  const int older = pos % CACHE_BLOCK;
  const size_t block = stored ? block_of(page, pos) : 0;
  float f[8];
  widen(raw, f);
  if (p.rotate && !is_v) turn_pairs(f, cs);
  if (there && is_q) store_eight<F32>(at.q_out, in, f);
  void* const cache = is_v ? at.v_cache : at.k_cache;
  const size_t first_elem = block * CACHE_BLOCK * DH + c * 8;      // of the block's first token
  if constexpr (BITS8) {
    uint32_t amax = finite_amax(f);
#pragma unroll
    for (int s = LANES / 2; s > 0; s >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, s));
    if (stored) {
      const int e = max(e_old, scale_exponent(amax));
      uint8_t* const codes = reinterpret_cast<uint8_t*>(cache) + first_elem;
      if (older > 0 && e > e_old) {
        const float factor = __uint_as_float(power_bits(e_old - e));
        for (int r = 0; r < older; ++r) {
          uint2* const w = reinterpret_cast<uint2*>(codes + r * DH);
          *w = make_uint2(rescale_e4m3(w->x, factor), rescale_e4m3(w->y, factor));
        }
      }
      *reinterpret_cast<uint2*>(codes + older * DH) = quantise(f, e);
      if (c == 0) scale[block] = uint8_t(e + 127);
    }
  } else if (stored) {
    store_eight<false>(cache, first_elem + older * DH, f);
  }
}

// Runs of tokens of every sequence.  A CTA takes one block of 16 positions of a sequence that new tokens fall into, in one layer
// (and where there is room, some of its heads).  A thread keeps one row and one slice of eight elements and goes through the heads,
// so that its sines and cosines stay in registers.  In 8 bits the largest magnitude of a block and head is exchanged through
// shared memory.  (A warp for all 16 rows of a head instead, with the angles in shared memory: prompts 211 and 492 us.  All blocks
// found by a search over the sequences: 64 runs of 4 tokens 22 us instead of 8.5.)
template <int DH, bool BITS8, bool F32, bool ONE_WAVE, int NL>
__global__ void __launch_bounds__(APP_THREADS, RUNS_AN_SM<DH, ONE_WAVE>) append_runs_kernel(const __grid_constant__ AppParams<NL> p) {
  constexpr int LANES = DH / 8, TEAM = CACHE_BLOCK * LANES, TEAMS = APP_THREADS / TEAM, TEAM_WARPS = TEAM / 32, HEADS = KV_HEADS<BITS8>, FLY = HEADS / TEAMS, Q_FLY = Q_HEADS / TEAMS;
  __shared__ uint32_t s_amax[2][TEAMS][FLY][TEAM_WARPS];
  __shared__ int2 s_found;
  const AppLayer& at = p.at[blockIdx.y];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int team = threadIdx.x / TEAM, r = threadIdx.x % TEAM / LANES, c = threadIdx.x % LANES;
  const int cap = p.max_pages * p.page_size;
  if (ONE_WAVE) grid_dep_launch();

  // The sequence and its block of positions: the first B blocks of the grid take the first one of each sequence, the others look
  // theirs up among the rest.
  int b = -1, base = 0;                            // sequence, the block's first position
  int r_lo = 0, r_hi = 0, row0 = 0;                // its rows that are new, and the row of T that its first one would be
  struct Ends {
    int r0, r1, len;
  };
  auto load = [&](int i) { return i < p.B ? Ends{__ldcg(p.first + i), __ldcg(p.first + i + 1), __ldcg(p.lengths + i)} : Ends{0, 0, 0}; };
  auto span = [&](const Ends& e, int& l, int& h, long long& tp) {   // rows of T outside [0, T) do not exist
    tp = (long long)e.len - e.r1;
    l = int(min((long long)cap, max(0LL, max((long long)e.r0, 0LL) + tp)));
    h = int(min((long long)cap, max(0LL, min((long long)e.r1, (long long)p.T) + tp)));
  };
  auto take = [&](int seq, int nth) {              // its nth block, if it has one
    int lo, hi;
    long long to_pos;
    span(load(seq), lo, hi, to_pos);
    base = (lo / CACHE_BLOCK + nth) * CACHE_BLOCK;
    b = base < hi && lo < hi ? seq : -1;
    r_lo = max(lo - base, 0);
    r_hi = min(hi - base, CACHE_BLOCK);
    row0 = int(base - to_pos);
  };
  auto locate = [&]() {
    if (int(blockIdx.x) < p.B) return take(blockIdx.x, 0);
    __syncthreads();
    if (threadIdx.x == 0) s_found = int2{-1, 0};
    __syncwarp();
    if (warp == 0) {
      int before = 0;
      Ends e = load(lane);
      for (int b0 = 0; b0 < p.B; b0 += 32) {
        Ends next = e;
        if (b0 + 32 < p.B) next = load(b0 + 32 + lane);
        int l, h;
        long long tp;
        span(e, l, h, tp);
        const int n = h > l ? (h - 1) / CACHE_BLOCK - l / CACHE_BLOCK : 0;   // blocks behind the first
        int upto = n;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, upto, s);
          if (lane >= s) upto += v;
        }
        const int unit = int(blockIdx.x) - p.B - before;
        if (unit < upto && unit >= upto - n) s_found = int2{b0 + lane, unit - (upto - n) + 1};
        if (__any_sync(0xffffffffu, unit < upto)) break;
        before += __shfl_sync(0xffffffffu, upto, 31);
        e = next;
      }
    }
    __syncthreads();
    b = -1;
    if (s_found.x >= 0) take(s_found.x, s_found.y);
  };
  float2 cs[4];
  auto angles = [&]() {
    if (!p.rotate) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) cs[k] = turn_of(p.turns[c * 4 + k], base + r);
  };
  // As in decode, where all blocks come up at once: from what is there before the kernels ahead have finished, and again behind the
  // wait; the angles are kept if the place is still the same.
  if constexpr (ONE_WAVE) {
    for (int behind = 0, angles_of = -1; behind < 2; ++behind) {   // (one copy of the code)
      if (behind != 0) grid_dep_wait();
      locate();
      if (b >= 0 && base != angles_of) angles();
      angles_of = b >= 0 ? base : -1;
    }
  } else {
    grid_dep_wait();
    locate();
    if (b >= 0) angles();
  }
  if (b < 0) {
    if (!ONE_WAVE) grid_dep_launch();
    return;
  }
  const bool mine = r >= r_lo && r < r_hi;             // this thread's row is new
  const int older = r_lo;                              // rows of the block that older tokens have
  const int page = p.block_table[size_t(b) * p.max_pages + base / p.page_size];
  const size_t row = size_t(row0 + r);                 // of T (where the row is new)
  const bool does_kv = int(blockIdx.z) < p.kv_slices, does_q = p.q_slices == 0 || !does_kv;

  if (does_kv && at.k_new != nullptr && page >= 0 && page < p.n_pages) {
    // groups of HEADS K heads, then of V heads
    const int groups = (p.Hkv + HEADS - 1) / HEADS, per_page = p.page_size / CACHE_BLOCK;
    const size_t page_block = size_t(page) * p.Hkv * per_page + base % p.page_size / CACHE_BLOCK;
    int buf = 0;
    for (int group = blockIdx.z; group < 2 * groups; group += p.kv_slices, buf ^= 1) {
      const bool is_v = group >= groups;
      const int head = (is_v ? group - groups : group) * HEADS + team;         // and every TEAMS-th behind it
      const int heads = (p.Hkv - head + TEAMS - 1) / TEAMS;                    // that there are of those (or fewer than one)
      const size_t block = page_block + size_t(head) * per_page, next_block = size_t(TEAMS) * per_page;
      uint8_t* const scale = BITS8 ? (is_v ? at.v_scale : at.k_scale) + block : nullptr;
      const size_t in = (row * p.Hkv + head) * DH + c * 8;
      uint4 raw[FLY];
      uint32_t held[FLY];                          // scales of a block that older tokens began
#pragma unroll
      for (int u = 0; u < FLY; ++u) {
        raw[u] = make_uint4(0u, 0u, 0u, 0u);
        held[u] = 0;
        if (u < heads) {
          if (mine) raw[u] = load_eight<F32>(is_v ? at.v_new : at.k_new, in + u * TEAMS * DH);
          if (BITS8 && older > 0) held[u] = scale[u * next_block];
        }
      }
      auto turned = [&](int u, float (&f)[8]) {
        widen(raw[u], f);
        if (p.rotate && !is_v) turn_pairs(f, cs);
      };
      if constexpr (BITS8) {
#pragma unroll
        for (int u = 0; u < FLY; ++u) {            // (rotated again below: kept, four heads' floats would leave room for three blocks an SM)
          float f[8];
          turned(u, f);
          const uint32_t m = __reduce_max_sync(0xffffffffu, finite_amax(f));
          if (lane == 0) s_amax[buf][team][u][warp % TEAM_WARPS] = m;
        }
        __syncthreads();
      }
      const size_t elem = (block * CACHE_BLOCK + r) * DH + c * 8, next_elem = next_block * CACHE_BLOCK * DH;
#pragma unroll
      for (int u = 0; u < FLY; ++u) {
        if (u >= heads) break;
        void* const cache = is_v ? at.v_cache : at.k_cache;
        float f[8];
        turned(u, f);
        if constexpr (BITS8) {
          uint32_t amax = 0;
#pragma unroll
          for (int w = 0; w < TEAM_WARPS; ++w) amax = max(amax, s_amax[buf][team][u][w]);
          const int e_old = older > 0 ? exponent_of_byte(held[u]) : LEAST_SCALE, e = max(e_old, scale_exponent(amax));
          uint2* const codes = reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(cache) + elem + u * next_elem);
          if (mine) {
            finite_amax(f);
            *codes = quantise(f, e);
          } else if (r < older && e > e_old) {
            const float factor = __uint_as_float(power_bits(e_old - e));
            *codes = make_uint2(rescale_e4m3(codes->x, factor), rescale_e4m3(codes->y, factor));
          }
          if (threadIdx.x % TEAM == 0) scale[u * next_block] = uint8_t(e + 127);   // (all have read the old one)
        } else {
          if (mine) store_eight<false>(cache, elem + u * next_elem, f);
        }
      }
    }
  }
  if (does_q && at.q != nullptr && mine) {
    const int first = int(blockIdx.z) - (p.q_slices == 0 ? 0 : p.kv_slices), step = p.q_slices == 0 ? p.kv_slices : p.q_slices;
    for (int head = first * Q_HEADS + team; head < p.Hq; head += step * Q_HEADS) {
      const size_t in = (row * p.Hq + head) * DH + c * 8;
      const int heads = (p.Hq - head + TEAMS - 1) / TEAMS;
      uint4 raw[Q_FLY];
#pragma unroll
      for (int u = 0; u < Q_FLY; ++u)
        if (u < heads) raw[u] = load_eight<F32>(at.q, in + u * TEAMS * DH);
#pragma unroll
      for (int u = 0; u < Q_FLY; ++u) {
        if (u >= heads) break;
        float f[8];
        widen(raw[u], f);
        if (p.rotate) turn_pairs(f, cs);
        store_eight<F32>(at.q_out, in + u * TEAMS * DH, f);
      }
    }
  }
  if (!ONE_WAVE) grid_dep_launch();
}

template <bool BITS8, bool F32, int NL>
cudaError_t launch_tokens(const AppParams<MANY_LAYERS>& all, int n, int dh, cudaStream_t stream) {
  AppParams<NL> p;
  static_cast<AppSizes&>(p) = all;
  std::copy(all.at, all.at + n, p.at);
  if (all.first == nullptr) {
    const int rows = 2 * all.Hkv + all.Hq;
    const int per = APP_THREADS / (dh / 8);
    return launch_kernel(dh == 128 ? append_one_kernel<128, BITS8, F32, NL> : append_one_kernel<64, BITS8, F32, NL>, dim3(all.B, n, (rows + per - 1) / per), APP_THREADS,
                         0, stream, 1, p);
  }
  // a block of the grid for each sequence, and for each block of positions behind the first that n tokens fall into: (n + 14) / 16
  const long long most = all.B + (all.T + 14LL * std::min(all.B, all.T)) / CACHE_BLOCK;
  // Where there is room for them, blocks of their own for the queries, and heads over several blocks, four each.
  const int room = int(std::min(64LL, ((long long)RUNS_A_WAVE * sm_count() + most * n - 1) / (most * n)));
  const int kv = 2 * ((all.Hkv + KV_HEADS<BITS8> - 1) / KV_HEADS<BITS8>), q = all.at[0].q != nullptr ? (all.Hq + Q_HEADS - 1) / Q_HEADS : 0;
  p.kv_slices = std::max(1, std::min(kv, q > 0 ? room * 2 * kv / (2 * kv + q) : room));
  p.q_slices = q > 0 ? std::max(0, std::min(q, room - p.kv_slices)) : 0;
  const dim3 grid(unsigned(most), n, p.kv_slices + p.q_slices);
  const bool one_wave = most * n * grid.z <= (long long)RUNS_A_WAVE * sm_count();
  auto* const kernel = one_wave ? (dh == 128 ? append_runs_kernel<128, BITS8, F32, true, NL> : append_runs_kernel<64, BITS8, F32, true, NL>)
                                : (dh == 128 ? append_runs_kernel<128, BITS8, F32, false, NL> : append_runs_kernel<64, BITS8, F32, false, NL>);
  return launch_kernel(kernel, grid, APP_THREADS, 0, stream, 1, p);
}

template <bool BITS8, bool F32>
cudaError_t launch_tokens(const AppParams<MANY_LAYERS>& p, int n, int dh, cudaStream_t stream) {
  return n <= FEW_LAYERS ? launch_tokens<BITS8, F32, FEW_LAYERS>(p, n, dh, stream) : launch_tokens<BITS8, F32, MANY_LAYERS>(p, n, dh, stream);
}

}  // namespace
}  // namespace kvp

using namespace kvp;

extern "C" int kvp_cache_append_tokens(const kvp_decode_desc* d, const int32_t* donor, int32_t T, const int32_t* first, float theta,
                                       const void* const* q, void* const* q_out, const void* const* k_new, const void* const* v_new,
                                       void* const* k_cache, void* const* v_cache, uint8_t* const* k_scale, uint8_t* const* v_scale,
                                       const int32_t* block_table, const int32_t* lengths, kvp_stream_t stream_) {
  if (d == nullptr || donor == nullptr || k_new == nullptr || v_new == nullptr || k_cache == nullptr || v_cache == nullptr ||
      block_table == nullptr || lengths == nullptr || (q == nullptr) != (q_out == nullptr) || (k_scale == nullptr) != (v_scale == nullptr))
    return KVP_ERR_INVALID_ARG;
  if (d->L < 1 || d->B < 1 || d->Hq < 1 || d->Hkv < 1 || d->max_pages < 1 || d->n_pages < 1 || T < 0 || (first == nullptr && T != d->B) ||
      !(theta == 0.f || (theta > 1.f && theta < INFINITY)))
    return KVP_ERR_INVALID_ARG;
  if (d->dtype != KVP_BF16 && d->dtype != KVP_F32) return KVP_ERR_UNSUPPORTED;
  if ((d->dh != 64 && d->dh != 128) || d->Hq % d->Hkv != 0 || d->page_size < CACHE_BLOCK || d->page_size % CACHE_BLOCK != 0 ||
      (long long)d->max_pages * d->page_size > 0x7fffffffLL || d->Hq > (1 << 16))
    return KVP_ERR_UNSUPPORTED;
  for (int l = 0; l < d->L; ++l)
    if (donor[l] < 0 || donor[l] > l || donor[donor[l]] != donor[l]) return KVP_ERR_BAD_DONOR;
  if (T == 0) return KVP_OK;           // (tensors without rows have no memory)
  const bool bits8 = k_scale != nullptr;
  for (int l = 0; l < d->L; ++l) {     // all of them before anything is launched
    if (q != nullptr) {
      if (q[l] == nullptr || q_out[l] == nullptr) return KVP_ERR_INVALID_ARG;
      if (!aligned16(q[l]) || !aligned16(q_out[l])) return KVP_ERR_UNSUPPORTED;
    }
    if (donor[l] != l) continue;       // consumers store nothing (Eq. 3)
    if (k_new[l] == nullptr || v_new[l] == nullptr || k_cache[l] == nullptr || v_cache[l] == nullptr || (bits8 && (k_scale[l] == nullptr || v_scale[l] == nullptr)))
      return KVP_ERR_INVALID_ARG;
    if (!aligned16(k_new[l]) || !aligned16(v_new[l]) || !aligned16(k_cache[l]) || !aligned16(v_cache[l])) return KVP_ERR_UNSUPPORTED;
  }
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  AppParams<MANY_LAYERS> p;
  p.block_table = block_table;
  p.lengths = lengths;
  p.first = first;
  p.B = d->B;
  p.T = T;
  p.Hq = d->Hq;
  p.Hkv = d->Hkv;
  p.page_size = d->page_size;
  p.max_pages = d->max_pages;
  p.n_pages = d->n_pages;
  p.rotate = theta != 0.f;
  if (p.rotate) rope_turns(double(theta), d->dh, p.turns);
  int n = 0;
  for (int l = 0; l <= d->L; ++l) {
    if (l < d->L && (q != nullptr || donor[l] == l)) {
      AppLayer& a = p.at[n++];
      const bool owner = donor[l] == l;
      a = AppLayer{q ? q[l] : nullptr, q ? q_out[l] : nullptr, owner ? k_new[l] : nullptr, owner ? v_new[l] : nullptr, owner ? k_cache[l] : nullptr,
                   owner ? v_cache[l] : nullptr, owner && bits8 ? k_scale[l] : nullptr, owner && bits8 ? v_scale[l] : nullptr};
    }
    if (n == MANY_LAYERS || (l == d->L && n > 0)) {
      const bool f32 = d->dtype == KVP_F32;
      const cudaError_t e = bits8 ? (f32 ? launch_tokens<true, true>(p, n, d->dh, stream) : launch_tokens<true, false>(p, n, d->dh, stream))
                                  : (f32 ? launch_tokens<false, true>(p, n, d->dh, stream) : launch_tokens<false, false>(p, n, d->dh, stream));
      if (e != cudaSuccess) return KVP_ERR_CUDA;
      n = 0;
    }
  }
  return KVP_OK;
}
