// Appending any number of tokens to the paged cache: K rotated by the token's position on the way in, the queries of the same
// tokens rotated beside it, and K and V stored as bf16 or in 8 bits (kvp_cache8.h).  One launch for up to 64 layers.
//
// Bound: HBM for prompts (every element is read and written once: 16-byte loads, a warp's all in flight before the first is
// used), latency for token steps (lengths -> block table -> store).  Positions are per sequence, so the angle is formed on the
// device: pos times the frequency as a 64-bit fraction of a turn, whose wrap-around is the range reduction; sine and cosine are
// taken of its upper 32 bits as a float, and what that float leaves off is applied as a first-order correction.
#include <math.h>

#include <algorithm>

#include "kvp_cache8.cuh"
#include "kvp_host.h"
#include "kvp_rope_freq.h"

namespace kvp {
namespace {

constexpr int APP_THREADS = 256, APP_WARPS = APP_THREADS / 32;
constexpr int MANY_LAYERS = 64, FEW_LAYERS = 8;    // a launch of few layers has a parameter block of 1 KB, not 5

struct AppLayer {
  const void* q;                 // [T,Hq,dh] bf16 or (io_f32) fp32; null: no queries
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
  int io_f32, rotate;
  uint64_t turns[64];            // rope_turns
};
template <int NL>
struct AppParams : AppSizes {
  AppLayer at[NL];
};

// eight consecutive elements as bf16
__device__ __forceinline__ uint4 load_eight(const void* base, size_t at, int f32) {
  if (f32) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
    const float4 a = p[0], b = p[1];
    return make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
  }
  return *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(base) + at);
}
// eight floats rounded to bf16, stored as such or widened
__device__ __forceinline__ void store_eight(void* base, size_t at, int f32, const float (&f)[8]) {
  const uint4 v = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  if (f32) {
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
// (K heads, V heads, query heads).  The rows are asked for before the lengths are there.
template <int DH, bool BITS8, int NL>
__global__ void __launch_bounds__(APP_THREADS) append_one_kernel(const __grid_constant__ AppParams<NL> p) {
  constexpr int LANES = DH / 8;
  const AppLayer& at = p.at[blockIdx.y];
  const int b = blockIdx.x, c = threadIdx.x % LANES;
  int row = blockIdx.z * (APP_THREADS / LANES) + threadIdx.x / LANES;
  grid_dep_launch();
  grid_dep_wait();
  const int kv_rows = at.k_new != nullptr ? 2 * p.Hkv : 0, rows = kv_rows + (at.q != nullptr ? p.Hq : 0);
  if (blockIdx.z * (APP_THREADS / LANES) >= rows) return;          // (the whole block)
  const bool there = row < rows;
  const bool is_q = row >= kv_rows, is_v = !is_q && row >= p.Hkv;
  const int head = is_q ? row - kv_rows : is_v ? row - p.Hkv : row, heads = is_q ? p.Hq : p.Hkv;
  const size_t in = (size_t(b) * heads + head) * DH + c * 8;
  uint4 raw = make_uint4(0u, 0u, 0u, 0u);
  if (there) raw = load_eight(is_q ? at.q : is_v ? at.v_new : at.k_new, in, p.io_f32);
  const int pos = p.lengths[b] - 1;
  if (pos < 0 || pos >= p.max_pages * p.page_size) return;         // (the whole block)
  const int page = p.block_table[size_t(b) * p.max_pages + pos / p.page_size];
  const bool stored = there && !is_q && page >= 0 && page < p.n_pages;
  const int slot = pos % p.page_size, older = pos % CACHE_BLOCK;
  const size_t block = (size_t(stored ? page : 0) * p.Hkv + (is_q ? 0 : head)) * (p.page_size / CACHE_BLOCK) + slot / CACHE_BLOCK;
  uint8_t* const scale = BITS8 ? (is_v ? at.v_scale : at.k_scale) : nullptr;
  int e_old = LEAST_SCALE;
  if (BITS8 && stored && older > 0) e_old = exponent_of_byte(scale[block]);
  float f[8];
  widen(raw, f);
  if (p.rotate && !is_v && there) {
    float2 cs[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) cs[k] = turn_of(p.turns[c * 4 + k], pos);
    turn_pairs(f, cs);
  }
  if (there && is_q) store_eight(at.q_out, in, p.io_f32, f);
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
    store_eight(cache, first_elem + older * DH, 0, f);
  }
}

// Runs of tokens of every sequence.  A CTA takes one block of 16 positions of a sequence that new tokens fall into, in one layer
// (and every gridDim.z-th head): it finds its block by a prefix sum over the sequences, forms the 16 rows' sines and cosines
// once, and its warps take the heads in turn, a warp all 16 rows of one, so that the largest magnitude of a block and head and
// the rounding to its scale stay in registers.
template <int DH, bool BITS8, int NL>
__global__ void __launch_bounds__(APP_THREADS, 2) append_runs_kernel(const __grid_constant__ AppParams<NL> p) {
  constexpr int LANES = DH / 8, ROWS = 32 / LANES, ITERS = CACHE_BLOCK / ROWS;   // lanes a row, rows at a time
  __shared__ float2 s_turn[CACHE_BLOCK][DH / 2];
  __shared__ int s_sum[APP_WARPS], s_found[2];
  const AppLayer& at = p.at[blockIdx.y];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cap = p.max_pages * p.page_size;
  grid_dep_wait();
  // positions of sequence b that its new tokens take: [lo, hi); rows of T outside [0, T) do not exist
  auto span = [&](int b, int& lo, int& hi) {
    const long long r0 = p.first[b], r1 = p.first[b + 1], len = p.lengths[b], to_pos = len - r1;   // position of row r: r + to_pos
    lo = int(min((long long)cap, max(0LL, max(r0, 0LL) + to_pos)));
    hi = int(min((long long)cap, max(0LL, min(r1, (long long)p.T) + to_pos)));
  };
  if (threadIdx.x == 0) s_found[0] = -1;
  int before = 0;
  for (int b0 = 0; b0 < p.B; b0 += APP_THREADS) {
    const int b = b0 + threadIdx.x;
    int n = 0;
    if (b < p.B) {
      int lo, hi;
      span(b, lo, hi);
      if (hi > lo) n = (hi - 1) / CACHE_BLOCK - lo / CACHE_BLOCK + 1;
    }
    int upto = n;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, s);
      if (lane >= s) upto += v;
    }
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
    int ahead = before;
#pragma unroll
    for (int w = 0; w < APP_WARPS; ++w) {
      ahead += w < warp ? s_sum[w] : 0;
      before += s_sum[w];
    }
    const int unit = int(blockIdx.x) - ahead;
    if (unit < upto && unit >= upto - n) {
      s_found[0] = b;
      s_found[1] = unit - (upto - n);
    }
    __syncthreads();
    if (s_found[0] >= 0) break;
  }
  if (s_found[0] < 0) {
    grid_dep_launch();
    return;
  }
  const int b = s_found[0];
  int lo, hi;
  span(b, lo, hi);
  const int base = (lo / CACHE_BLOCK + s_found[1]) * CACHE_BLOCK;   // the block's first position
  const int r_lo = max(lo - base, 0), r_hi = min(hi - base, CACHE_BLOCK);   // its rows that are new
  const long long row0 = (long long)base - p.lengths[b] + p.first[b + 1];   // row of T at `base` (may be negative)
  const int page = p.block_table[size_t(b) * p.max_pages + base / p.page_size];
  if (p.rotate) {
    for (int i = threadIdx.x; i < CACHE_BLOCK * (DH / 2); i += APP_THREADS) s_turn[i / (DH / 2)][i % (DH / 2)] = turn_of(p.turns[i % (DH / 2)], base + i / (DH / 2));
  }
  __syncthreads();
  const int rr = lane / LANES, c = lane % LANES;
  const int kv_rows = at.k_new != nullptr ? 2 * p.Hkv : 0, rows = kv_rows + (at.q != nullptr ? p.Hq : 0);
  const bool paged = page >= 0 && page < p.n_pages;
  for (int row = int(blockIdx.z) * APP_WARPS + warp; row < rows; row += int(gridDim.z) * APP_WARPS) {
    const bool is_q = row >= kv_rows, is_v = !is_q && row >= p.Hkv;
    if (!is_q && !paged) continue;
    const int head = is_q ? row - kv_rows : is_v ? row - p.Hkv : row, heads = is_q ? p.Hq : p.Hkv;
    const void* const src = is_q ? at.q : is_v ? at.v_new : at.k_new;
    auto in = [&](int r) { return (size_t(row0 + r) * heads + head) * DH + c * 8; };
    uint4 raw[ITERS];
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
      const int r = i * ROWS + rr;
      raw[i] = make_uint4(0u, 0u, 0u, 0u);
      if (r >= r_lo && r < r_hi) raw[i] = load_eight(src, in(r), p.io_f32);
    }
    auto rotated = [&](int i, float (&f)[8]) {
      widen(raw[i], f);
      if (p.rotate && !is_v) {
        float2 cs[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) cs[k] = s_turn[i * ROWS + rr][c * 4 + k];
        turn_pairs(f, cs);
      }
    };
    const size_t block = (size_t(is_q ? 0 : page) * p.Hkv + head) * (p.page_size / CACHE_BLOCK) + base % p.page_size / CACHE_BLOCK;
    void* const cache = is_v ? at.v_cache : at.k_cache;
    const size_t first_elem = block * CACHE_BLOCK * DH + c * 8;
    if (BITS8 && !is_q) {
      uint8_t* const scale = is_v ? at.v_scale : at.k_scale;
      uint8_t* const codes = reinterpret_cast<uint8_t*>(cache) + first_elem;
      const int e_old = r_lo > 0 ? exponent_of_byte(scale[block]) : LEAST_SCALE;
      float f[ITERS][8];
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < ITERS; ++i) {
        rotated(i, f[i]);
        amax = max(amax, finite_amax(f[i]));
      }
      amax = __reduce_max_sync(0xffffffffu, amax);
      const int e = max(e_old, scale_exponent(amax));
      if (r_lo > 0 && e > e_old) {
        const float factor = __uint_as_float(power_bits(e_old - e));
        for (int r = rr; r < r_lo; r += ROWS) {
          uint2* const w = reinterpret_cast<uint2*>(codes + r * DH);
          *w = make_uint2(rescale_e4m3(w->x, factor), rescale_e4m3(w->y, factor));
        }
      }
#pragma unroll
      for (int i = 0; i < ITERS; ++i) {
        const int r = i * ROWS + rr;
        if (r >= r_lo && r < r_hi) *reinterpret_cast<uint2*>(codes + r * DH) = quantise(f[i], e);
      }
      __syncwarp();                                                // (every lane has read the old scale)
      if (lane == 0) scale[block] = uint8_t(e + 127);
    } else {
#pragma unroll
      for (int i = 0; i < ITERS; ++i) {
        const int r = i * ROWS + rr;
        float f[8];
        rotated(i, f);
        if (r >= r_lo && r < r_hi) {
          if (is_q) store_eight(at.q_out, in(r), p.io_f32, f);
          else store_eight(cache, first_elem + r * DH, 0, f);
        }
      }
    }
  }
  grid_dep_launch();
}

template <bool BITS8, int NL>
cudaError_t launch_tokens(const AppParams<MANY_LAYERS>& all, int n, int dh, cudaStream_t stream) {
  AppParams<NL> p;
  static_cast<AppSizes&>(p) = all;
  std::copy(all.at, all.at + n, p.at);
  const int rows = 2 * all.Hkv + all.Hq;
  if (all.first == nullptr) {
    const int per = APP_THREADS / (dh / 8);
    return launch_kernel(dh == 128 ? append_one_kernel<128, BITS8, NL> : append_one_kernel<64, BITS8, NL>, dim3(all.B, n, (rows + per - 1) / per), APP_THREADS,
                         0, stream, 1, p);
  }
  // blocks that n >= 1 tokens fall into: at most n, and at most (n + 14) / 16 + 1
  const long long live = std::min(all.B, all.T), most = std::min((long long)all.T, (all.T + 30 * live) / CACHE_BLOCK);
  const int slices = int(std::max(1LL, std::min((long long)(rows + APP_WARPS - 1) / APP_WARPS, 2LL * sm_count() / std::max(1LL, most * n))));
  return launch_kernel(dh == 128 ? append_runs_kernel<128, BITS8, NL> : append_runs_kernel<64, BITS8, NL>, dim3(unsigned(most), n, slices), APP_THREADS, 0, stream,
                       1, p);
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
  p.io_f32 = d->dtype == KVP_F32;
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
      const cudaError_t e = n <= FEW_LAYERS ? (bits8 ? launch_tokens<true, FEW_LAYERS>(p, n, d->dh, stream) : launch_tokens<false, FEW_LAYERS>(p, n, d->dh, stream))
                                            : (bits8 ? launch_tokens<true, MANY_LAYERS>(p, n, d->dh, stream) : launch_tokens<false, MANY_LAYERS>(p, n, d->dh, stream));
      if (e != cudaSuccess) return KVP_ERR_CUDA;
      n = 0;
    }
  }
  return KVP_OK;
}
