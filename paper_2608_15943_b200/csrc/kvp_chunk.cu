// Attention of the new tokens of every sequence (one, a few drafted ones, a piece of a prompt) over the shared paged cache they
// have been appended to, bf16 or 8 bits, with or without a sliding window and first tokens that stay visible.
//
// The query rows of a sequence and KV head are laid out token by token: the G heads of a token in each of the layers that
// share the donor.  128 of them are a tile, two tiles a unit; a unit walks the cached keys that any of its rows sees, 64 a step,
// and each K/V block that it brings in serves both tiles, all heads and all layers.  The steps of all units form one list, which the
// CTAs (one an SM) deal out among themselves from the lengths on the device: whole units in rounds where there are many, equal shares
// of the list where there are few; a unit that ends up in several shares is merged by a second kernel.  So one long context
// occupies the whole device, and prompts of any lengths leave no SM behind.
//   warp 0        TMA producer: K and V blocks, page by page (8-bit cache: the codes into a ring of their own, and their scales)
//   warps 1, 2    tcgen05.mma issuers, one per tile: S = Q K^T into one of two 64-column score buffers, O += P V with P from TMEM
//   warp 3        lays out the CTA's pieces of units, and looks through the V blocks that not every row sees in full
//   warps 4-11    softmax, a warpgroup per tile, a thread per row; then O out of TMEM to the outputs or to the unit's partial sums,
//                 while the rows of the next piece come into shared memory.  Where a unit has one tile alone, both warpgroups have
//                 it, take every other step each, and put their two sums together at the end.
//   warps 12-15   (8-bit cache only) V's codes to f16, which holds them exactly.  K's are operands as they are; the scales are applied
//                 to the scores and to the weights of V.
// What bounds it.  Drafts (2-8 tokens of 16 sequences of 4K-16K, 16 to 64 rows a unit): memory in bf16, 228 us, 5.8 TB/s; over the
// 8-bit cache, 243 us, the chain of a step (scores out of TMEM, maximum, exponentials and weights, P, product; some 2900 cycles for
// every other step of each half), beside the conversion of V on the same schedulers.  Prompts: the 1000 W of the board (1.67 to 1.8 GHz; 1190
// TFLOP/s over 64K tokens in a burst of 15.7 ms, 1050 over seconds); ahead of it the exponentials (1024 of 1800 cycles a step of two tiles) and the
// products of 64 columns, which read Q again for each (1280).  Heads of 64 over 8 bits: the chain, 2700 cycles a step at full clock.
// Left out: a quarter of the exponentials as polynomials on the multipliers (no faster in bf16, registers spill in 8 bits);
// turns for the two tiles' exponentials (5 to 15% slower); the next piece's queries asked for ahead of the last step (5% slower).
// Masked places.  A score that a row does not see is -infinity before the maximum.  In V, rows that no row of the unit sees (slots
// behind the sequence, freed pages before the window: anything may be there) are not read and are zeros in shared memory.  A
// visible row of V with an infinity or NaN in it must reach the rows that see it and no other, which 0 * NaN in a matrix product
// does not give: in blocks with any masking such rows are taken out, and the softmax threads add them to O by themselves.
#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "kvp_cache8.cuh"
#include "kvp_chunk_rows.h"
#include "kvp_decode_list.cuh"
#include "kvp_host.h"
#include "kvp_sm100.cuh"

namespace kvp {
namespace {

constexpr int TILE = CHUNK_TILE;          // query rows of a tile (TMEM lanes)
constexpr int STEP = 64;                  // keys per step
constexpr int BATCH = 8;                  // steps whose pages the producer's lanes hold: four blocks of 16 keys a step
constexpr int CHUNK_MEMBERS = 8;          // layers of a donor group in one tile
constexpr int MANY_CHUNK_GROUPS = 16, FEW_CHUNK_GROUPS = 4;
constexpr uint32_t Q_HALF = TILE * 128;   // one [128 rows x 128 B] block of Q
constexpr uint32_t KV_HALF = STEP * 128;
constexpr float kRescaleBy = 8.0f;        // log2: O is rescaled when the maximum has moved by more
// A product is scaled and the (rounded) maximum taken off in one operation, which is exact until its end: the largest score comes out as
// what the maximum was rounded by, and from 2^31 on that is more than exponents hold.  So rows with a maximum beyond FAR, where scores are 1/2
// and more apart, and off by more than that, are scaled by the power of two in the scale alone, of which the difference to the largest is
// exact.  (Difference first and scaled then, for every row: prompts under a window 2220 -> 2270 us.  A branch for such rows: 2350.)
constexpr float FAR = 8388608.f;
// Places of the list behind the steps of a unit, for its start, its output and its merge, 8900 cycles where a step of two tiles takes 1800
// (3: drafts and prompts under a window 1% slower; 8: short prompts 1%); least places of a share.
constexpr int REST = 6, LEAST_SHARE = 8;

__device__ int g_chunk_status;

constexpr int PIECES = 4, PIECES_BYTES = 512;       // the ring of pieces
// The scales of a step of the 8-bit cache, a block of 16 keys each: K's and V's powers of two, and V's exponents.  A step's stay until
// its product has been issued: K is asked for one step ahead of V at the most, and V's rings hold fewer steps than there are places.
struct Scales {
  float4 k, v, e;
};
constexpr int SCALES = 16;

template <int DH, bool BITS8>
struct ChunkSmem {
  static constexpr int K_STAGES = BITS8 ? (DH == 128 ? 6 : 8) : (DH == 128 ? 5 : 8);
  static constexpr int V_STAGES = BITS8 ? 4 : K_STAGES;
  static constexpr int RAW_STAGES = BITS8 ? (DH == 128 ? 6 : 8) : 0;                       // V's codes
  static constexpr int Q_BYTES = TILE * DH * 2, V_BYTES = STEP * DH * 2, K_BYTES = BITS8 ? STEP * DH : V_BYTES, RAW_BYTES = STEP * DH;
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = OFF_Q + 2 * Q_BYTES;
  static constexpr int OFF_V = OFF_K + K_STAGES * K_BYTES;
  static constexpr int OFF_RAW = OFF_V + V_STAGES * V_BYTES;
  static constexpr int OFF_BAR = OFF_RAW + RAW_STAGES * RAW_BYTES;
  static constexpr int BARRIERS = 2 + 2 * K_STAGES + 3 * V_STAGES + 14 + 2 * PIECES + 2 * RAW_STAGES;
  static constexpr int OFF_BAD = OFF_BAR + (BARRIERS + 2) / 2 * 16;   // [V_STAGES][4] rows of V that are left to the softmax threads
  static constexpr int OFF_SCALE = OFF_BAD + V_STAGES * 32;     // [SCALES]
  static constexpr int OFF_PIECES = OFF_SCALE + (BITS8 ? SCALES * int(sizeof(Scales)) : 0);
  static constexpr int TOTAL = OFF_PIECES + PIECES_BYTES + 1024;      // room for the alignment
  static constexpr int THREADS = BITS8 ? 512 : 384;
  // 8-bit cache: registers of a thread at launch, of the softmax threads, and what stays with each of the others
  static constexpr int LAUNCH_REGS = 128, SOFTMAX_REGS = 192, OTHER_REGS = 64;
  static_assert(256 * SOFTMAX_REGS + 256 * OTHER_REGS <= 512 * LAUNCH_REGS, "registers of a CTA");
};
static_assert(ChunkSmem<128, false>::TOTAL <= 232448 && ChunkSmem<128, true>::TOTAL <= 232448, "shared memory of a CTA");
static_assert(ChunkSmem<64, true>::RAW_STAGES + ChunkSmem<64, true>::V_STAGES + 1 < SCALES && ChunkSmem<128, true>::RAW_STAGES + ChunkSmem<128, true>::V_STAGES + 1 < SCALES,
              "rings of the 8-bit cache");

// A unit that more than one share holds, noted by the CTA of its second share
struct Merge {
  int g, hk, b, pair;
  int w0, w1;                              // its shares (w0 < 0: nothing to merge)
  int pad[2];
};

struct ChunkSizes {
  const int32_t *block_table, *lengths, *first;
  Merge* merges;                           // [shares]
  float* part_o;                           // [2 * shares][256][DH]
  float* part_ml;                          // [2 * shares][256][2]
  int B, T, Hq, Hkv, G, page_size, max_pages, n_pages;
  int n_groups;
  int kind[MANY_CHUNK_GROUPS];             // groups of as many layers have the same list: its number
  int n_kinds;
  Rows rows[CHUNK_MEMBERS], heads;         // of each list; G, the query heads of a KV head, the same way
  int window, sinks;                       // window 0: none
  int box;                                 // keys of a TMA box: 64, 32 or 16
  int io_f32;
  float scale, scale_power, scale_rest;    // of the products, for powers of 2: a power of two times 1 to 2
};
struct ChunkGroup {
  CUtensorMap map_k, map_v;
  const void* q[CHUNK_MEMBERS];
  void* o[CHUNK_MEMBERS];
  float* lse[CHUNK_MEMBERS];
  const void* v_pool;
  const uint8_t *k_scale, *v_scale;
};
template <int NG>
struct ChunkParams : ChunkSizes {
  ChunkGroup grp[NG];
};

// ---------------------------------------------------------------------------------------------
// the list of steps
// ---------------------------------------------------------------------------------------------
// The rows of a sequence that are computed: tokens before position 0 or behind the table's capacity are left out.
struct Span {
  int row0, n;       // rows of q
  int pos0;          // position of the first
};
__device__ __forceinline__ Span span_of(const ChunkSizes& p, int b) {
  Span s;
  int end;
  if (p.first != nullptr) {
    s.row0 = min(max(p.first[b], 0), p.T);
    end = min(max(p.first[b + 1], s.row0), p.T);
  } else {
    s.row0 = b;
    end = b + 1;
  }
  s.n = end - s.row0;
  s.pos0 = max(p.lengths[b], 0) - s.n;
  const int early = max(0, -s.pos0);
  s.row0 += early;
  s.n -= early;
  s.pos0 += early;
  s.n = max(0, min(s.n, p.max_pages * p.page_size - s.pos0));
  return s;
}
// The keys that a pair of tiles walks
struct Walked {
  int pos_first, pos_last_a, pos_last;   // positions of the first row, of tile A's last and of the last
  int sink_blocks, from;                 // blocks of first tokens, then blocks from `from` on
  int n, n_a;                            // steps, and those of tile A
};
__device__ __forceinline__ int pairs_of(const Span& s, const Rows& R) { return units_of_rows(s.n * R.n); }
__device__ __forceinline__ Walked walked(const ChunkSizes& p, const Span& s, const Rows& R, int pair) {
  Walked w;
  const int row0 = pair * 2 * TILE;
  auto token = [&](int row) { return min(s.n - 1, R.token(row)); };
  w.pos_first = s.pos0 + token(row0);
  w.pos_last_a = s.pos0 + token(row0 + TILE - 1);
  w.pos_last = s.pos0 + token(row0 + 2 * TILE - 1);
  const int end_a = w.pos_last_a / STEP + 1, end = w.pos_last / STEP + 1;
  w.sink_blocks = p.window > 0 ? min((p.sinks + STEP - 1) / STEP, end) : 0;
  w.from = p.window > 0 ? max(max(0, w.pos_first - p.window + 1) / STEP, w.sink_blocks) : 0;
  w.n = w.sink_blocks + max(0, end - w.from);
  w.n_a = min(w.sink_blocks, end_a) + max(0, end_a - w.from);
  return w;
}
// Of the lane's sequence b (nothing behind the last), a warp together: places, units of a KV head, steps of the longest.
struct Listed {
  long long places;
  int pairs, longest;
};
__device__ __forceinline__ Listed listed(const ChunkSizes& p, int b, const Rows& R) {
  const int lane = lane_id();
  Span s{0, 0, 0};
  if (b < p.B) s = span_of(p, b);
  Listed l{0, pairs_of(s, R), 0};
  const bool few = l.pairs <= 2;
  if (few)
    for (int i = 0; i < l.pairs; ++i) {
      const int n = walked(p, s, R, i).n;
      l.places += n + REST;
      l.longest = max(l.longest, n);
    }
  for (uint32_t left = __ballot_sync(0xffffffffu, !few); left != 0; left &= left - 1) {
    const int of = __ffs(left) - 1;
    const Span t{__shfl_sync(0xffffffffu, s.row0, of), __shfl_sync(0xffffffffu, s.n, of), __shfl_sync(0xffffffffu, s.pos0, of)};
    const int n = __shfl_sync(0xffffffffu, l.pairs, of);
    long long mine = 0;
    int longest = 0;
    for (int i = lane; i < n; i += 32) {
      const int steps = walked(p, t, R, i).n;
      mine += steps + REST;
      longest = max(longest, steps);
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) mine += __shfl_xor_sync(0xffffffffu, mine, d);
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (lane == of) l.places = mine, l.longest = longest;
  }
  return l;
}
__device__ __forceinline__ long long warp_scan(long long v) {   // inclusive
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const long long o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane_id() >= d) v += o;
  }
  return v;
}
// What a CTA gets: whole units `first`, first + gridDim.x, ... below `rounds_end`, then a share of the list behind them.
struct Share {
  int g, hk, b, pair;
  int off;           // places of the unit that belong to earlier shares
  int left;          // places of the share
  long long rounds_end;
};
// Sums over 32 sequences each, then over all before them, i <= n32 = ceil(B / 32): of places [kind][i], and of units [kind][i]; longest
// unit of each 32.  All warps of the block.
struct Sums {
  long long *places, *units;
  int* longest;
  int n32;
  __device__ __forceinline__ Sums(void* at, const ChunkSizes& p) : places(static_cast<long long*>(at)), n32((p.B + 31) / 32) {
    units = places + p.n_kinds * (n32 + 1);
    longest = reinterpret_cast<int*>(units + p.n_kinds * (n32 + 1));
  }
  __device__ __forceinline__ void* end(const ChunkSizes& p) const { return longest + (p.n_kinds * n32 + 1) / 2 * 2; }
  __device__ __forceinline__ long long all_places(int kind) const { return places[kind * (n32 + 1) + n32]; }
  __device__ __forceinline__ long long all_units(int kind) const { return units[kind * (n32 + 1) + n32]; }
};
__device__ __forceinline__ long long warp_sum(long long v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ void list_sums(const ChunkSizes& p, const Sums& s, int warps) {
  const int warp = threadIdx.x >> 5, lane = lane_id();
  for (int i = warp; i < s.n32 * p.n_kinds; i += warps) {
    const int kind = i / s.n32, at = i % s.n32;
    const Listed l = listed(p, at * 32 + lane, p.rows[kind]);
    const long long places = warp_sum(l.places), units = warp_sum(l.pairs);
    const int longest = __reduce_max_sync(0xffffffffu, l.longest);
    if (lane == 0) {
      s.places[kind * (s.n32 + 1) + at] = places;
      s.units[kind * (s.n32 + 1) + at] = units;
      s.longest[i] = longest;
    }
  }
  __syncthreads();
  for (int k = warp; k < 2 * p.n_kinds; k += warps) {
    long long* const of = s.places + k * (s.n32 + 1);       // (units follow places)
    long long before = 0;
    for (int i0 = 0; i0 < s.n32; i0 += 32) {
      const int i = i0 + lane;
      const long long v = i < s.n32 ? of[i] : 0, up = warp_scan(v);
      if (i < s.n32) of[i] = before + up - v;
      before += __shfl_sync(0xffffffffu, up, 31);
    }
    __syncwarp();
    if (lane == 0) of[s.n32] = before;
  }
  __syncthreads();
}
// the last of sums[0 .. n) that is at or below `at`, by a warp
__device__ __forceinline__ int last_below(const long long* sums, int n, long long at) {
  int i = 0;
  for (int i0 = 0; i0 < n; i0 += 32) {
    const uint32_t below = __ballot_sync(0xffffffffu, i0 + lane_id() < n && sums[i0 + lane_id()] <= at);
    if (below == 0) break;
    i = i0 + 31 - __clz(below);
  }
  return i;
}
// How the list is dealt out.  Many units: whole, in rounds of one a CTA, so that CTAs that run together read the same keys at the same
// time, out of L2; as many as give no CTA more than a fair part, and not the last two.  What is left is cut into shares that even out
// what the rounds gave.  Not where a unit is longer than an eighth of a CTA's work (what is left would not even that out), or where
// there are few: equal shares of the whole list.
// (Pieces of prompts behind 2K to 8K tokens, read out of memory: 8.3 GB with equal shares of the list.)
// Few and short units: whole, one a CTA, up to WHOLE_UP_TO steps more than an equal share has.  (Four tokens behind 100-300, 400-600, 900-1100 and
// 1900-2100 of 8 sequences: 16.6, 19.5, 22.7 and 24.5 us; cut, 22.0, 22.2, 22.8 and 24.5; whole up to 32 more 16.6, 19.5, 24.2 and 34.8.)
constexpr int ROUNDS_FROM = 4, ROUNDS_LEFT = 2, WHOLE_UP_TO = 8;
struct Deal {
  long long rounds_end;        // units that are dealt out whole
  long long base;              // their places
  long long total;             // places behind them
  int n;                       // shares of these
  bool even;                   // all alike, or from places `begin` on
  long long* begin;            // [n + 1]
  __device__ __forceinline__ long long first(int w) const { return even ? Dealt(total, n).begin(w) : begin[w]; }
  __device__ __forceinline__ int share_of(long long at) const { return even ? Dealt(total, n).share_of(at) : last_below(begin, n, at); }
};
// The place `at` of the list, by a warp: group, KV head, sequence; what is left is inside the sequence's.
struct Found {
  int g, hk, b;
  long long left;
};
__device__ __forceinline__ Found find(const ChunkSizes& p, const Sums& s, long long at) {
  Found f{0, 0, 0, at};
  for (;; ++f.g) {
    const long long group = s.all_places(p.kind[f.g]) * p.Hkv;
    if (f.left < group) break;
    f.left -= group;
  }
  const int kind = p.kind[f.g];
  f.hk = int(div_places(f.left, s.all_places(kind)));
  f.left -= f.hk * s.all_places(kind);
  const int row = kind * (s.n32 + 1), i = last_below(s.places + row, s.n32, f.left);
  f.left -= s.places[row + i];
  const long long mine = listed(p, i * 32 + lane_id(), p.rows[kind]).places, up = warp_scan(mine);
  const int of = __ffs(__ballot_sync(0xffffffffu, up > f.left)) - 1;
  f.left -= __shfl_sync(0xffffffffu, up - mine, of);
  f.b = i * 32 + of;
  return f;
}
// By all warps of the block; `room` bytes of shared memory behind the sums.
__device__ __forceinline__ Deal deal_out(const ChunkSizes& p, const Sums& s, int room, int warps) {
  const int lane = lane_id(), warp = threadIdx.x >> 5, n = int(gridDim.x);
  Deal d{0, 0, 0, 0, true, static_cast<long long*>(s.end(p))};
  long long units = 0;
  int longest = 0;
  for (int g = 0; g < p.n_groups; ++g) {
    d.total += s.all_places(p.kind[g]) * p.Hkv;
    units += s.all_units(p.kind[g]) * p.Hkv;
  }
  for (int i = lane; i < s.n32 * p.n_kinds; i += 32) longest = max(longest, s.longest[i]);
  longest = __reduce_max_sync(0xffffffffu, longest);
  if (units <= n && longest <= div_places(d.total, n) + WHOLE_UP_TO) {
    d.rounds_end = units;
    d.base = d.total;
  } else if (units >= (long long)ROUNDS_FROM * n && (long long)longest * 8 * n <= d.total) {
    // what the rounds give each CTA, from the places of every unit of a KV head
    int* const cost = reinterpret_cast<int*>(d.begin + n + 1);
    long long all = 0;
    for (int kind = 0; kind < p.n_kinds; ++kind) all += s.all_units(kind);
    if ((all + 1) * 4 + (n + 1) * 8 <= room) {
      for (int kind = 0, at = 0; kind < p.n_kinds; at += int(s.all_units(kind)), ++kind) {
        const Rows rows = p.rows[kind];
        for (int i = warp; i < s.n32; i += warps) {
          const Span mine = i * 32 + lane < p.B ? span_of(p, i * 32 + lane) : Span{0, 0, 0};
          const int pairs = pairs_of(mine, rows);
          const int to = at + int(s.units[kind * (s.n32 + 1) + i] + warp_scan(pairs) - pairs);
          const bool few = pairs <= 2;
          if (few)
            for (int pair = 0; pair < pairs; ++pair) cost[to + pair] = walked(p, mine, rows, pair).n + REST;
          for (uint32_t left = __ballot_sync(0xffffffffu, !few); left != 0; left &= left - 1) {
            const int of = __ffs(left) - 1;
            const Span t{__shfl_sync(0xffffffffu, mine.row0, of), __shfl_sync(0xffffffffu, mine.n, of), __shfl_sync(0xffffffffu, mine.pos0, of)};
            const int many = __shfl_sync(0xffffffffu, pairs, of), from = __shfl_sync(0xffffffffu, to, of);
            for (int pair = lane; pair < many; pair += 32) cost[from + pair] = walked(p, t, rows, pair).n + REST;
          }
        }
      }
      int* const rounds = cost + all;
      if (threadIdx.x == 0) *rounds = int(div_places(units, n)) - ROUNDS_LEFT;
      __syncthreads();
      // the CTA's places in the first `most` rounds, as long as they are no more than a fair part of all
      const long long fair = div_places(d.total, n);
      auto take = [&](int most, int& taken) {
        long long mine = 0, in = threadIdx.x;                  // unit of the KV head `g`, hk
        int g = 0, hk = 0, at = 0;
        for (taken = 0; taken < most; ++taken, in += n) {
          while (in >= s.all_units(p.kind[g])) {
            in -= s.all_units(p.kind[g]);
            if (++hk == p.Hkv) {
              hk = 0;
              ++g;
              at = 0;
              for (int kind = 0; kind < p.kind[g]; ++kind) at += int(s.all_units(kind));
            }
          }
          if (mine + cost[at + in] > fair) break;
          mine += cost[at + in];
        }
        return mine;
      };
      const bool is_cta = int(threadIdx.x) < n;
      int taken = 0;
      if (is_cta) {
        take(int(div_places(units, n)) - ROUNDS_LEFT, taken);
        atomicMin(rounds, taken);
      }
      __syncthreads();
      d.rounds_end = (long long)*rounds * n;
      if (is_cta) d.begin[threadIdx.x] = fair - take(*rounds, taken);
      __syncthreads();
      if (warp == 0) {                                         // sums, then in proportion: they come to what is left
        long long sum = 0;
        for (int i0 = 0; i0 < n; i0 += 32) {
          const long long v = i0 + lane < n ? d.begin[i0 + lane] : 0, up = warp_scan(v);
          __syncwarp();
          if (i0 + lane < n) d.begin[i0 + lane] = sum + up - v;
          sum += __shfl_sync(0xffffffffu, up, 31);
        }
        __syncwarp();
        const long long left = sum + (d.total - n * fair);
        const double part = sum > 0 ? double(left) / double(sum) : 0.;
        for (int i = lane; i < n; i += 32) d.begin[i] = min(left, (long long)(double(d.begin[i]) * part));
        if (lane == 0) d.begin[n] = left;
      }
      d.even = false;
      __syncthreads();
      d.base = d.total - d.begin[n];
    }
  }
  d.total -= d.base;
  d.n = d.even ? int(min((long long)n, max(d.total > 0 ? 1ll : 0ll, d.total / LEAST_SHARE))) : n;
  return d;
}
// The share of this CTA, by one warp; writes the note for the merge.
__device__ __forceinline__ Share find_share(const ChunkSizes& p, const Sums& s, const Deal& d) {
  const int lane = lane_id(), w = int(blockIdx.x);
  Share out{0, 0, 0, 0, 0, 0, d.rounds_end};
  Merge note{0, 0, 0, 0, -1, -1, {0, 0}};
  const long long begin = w < d.n ? d.first(w) : 0, size = w < d.n ? (w + 1 < d.n ? d.first(w + 1) : d.total) - begin : 0;
  if (size > 0) {
    const Found f = find(p, s, d.base + begin);
    out.g = f.g;
    out.hk = f.hk;
    out.b = f.b;
    long long at = f.left;
    const Span span = span_of(p, f.b);
    const Rows R = p.rows[p.kind[f.g]];
    const int pairs = pairs_of(span, R);
    for (int pair0 = 0;; pair0 += 32) {
      const int pair = pair0 + lane;
      const long long cost = pair < pairs ? walked(p, span, R, pair).n + REST : 0, sum = warp_scan(cost);
      const long long all = __shfl_sync(0xffffffffu, sum, 31);
      if (at >= all && pair0 + 32 < pairs) {
        at -= all;
        continue;
      }
      const int first = __ffs(__ballot_sync(0xffffffffu, sum > at)) - 1;
      at -= __shfl_sync(0xffffffffu, sum - cost, first);
      out.pair = pair0 + first;
      break;
    }
    out.off = int(at);
    out.left = int(size);                  // (2^31 steps of a CTA would take most of an hour)
    // the unit goes on from an earlier share: the first that begins inside it notes it
    const int steps = walked(p, span, R, out.pair).n;
    if (out.off > 0 && out.off < steps) {
      const int w0 = d.share_of(begin - out.off);
      // (the next one may be empty, and then begins where the first that is not does)
      if (d.first(w0 + 1) == begin) note = Merge{out.g, out.hk, out.b, out.pair, w0, d.share_of(begin - out.off + steps - 1), {0, 0}};
    }
  }
  // (an empty share may lie between two of a unit's)
  if (size == 0 && w < d.n)
    for (int row = lane; row < 2 * TILE; row += 32) *reinterpret_cast<float2*>(p.part_ml + (size_t(2 * w) * (2 * TILE) + row) * 2) = make_float2(-INFINITY, 0.f);
  if (lane == 0) p.merges[w] = note;
  return out;
}

// A share's pieces, one after the other: what the roles need of them, laid out by warp 3 in a ring in shared memory.
struct Piece {
  int n;                       // steps; 0: there are no more pieces
  int g, hk, b;
  int row0;                    // row of q of the sequence's first token
  int pos0;                    // its position
  int duo;                     // one tile: both halves of the CTA have its rows, and take every other step each; 2: rows of half a tile,
                               // in its second half for half 1, so that softmax works on all four quarters of the SM
  int n_x[2];                  // steps that each half takes
  int rows[2];                 // rows of its tile
  int token[2], in[2];         // the tile's first: its token, and which of the token's rows
  int pos_first, pos_last;     // positions of the unit's rows
  int sinks, at_sinks, at;     // step i is block at_sinks + i for i < sinks, at + i from there on
  int2 clear, clear_x[2];      // steps i, x <= i < y, in which all rows (the half's rows) see every key
  int whole, slot;             // the unit has no other piece; otherwise the place of its partial sums
  __device__ __forceinline__ int block(int i) const { return (i < sinks ? at_sinks : at) + i; }
  // no row of the unit sees any of n keys from `key` on
  __device__ __forceinline__ bool unseen(const ChunkSizes& p, int key, int n) const {
    return key > pos_last || (p.window > 0 && key + n - 1 <= pos_first - p.window && key >= p.sinks);
  }
};
static_assert(PIECES * sizeof(Piece) <= PIECES_BYTES && sizeof(Piece) % 8 == 0, "the ring of pieces");

struct Pieces {
  Share share;                 // where the share begins
  int g, hk, b, pair, off, left;
  long long unit;              // the next of the whole ones; from rounds_end on: the share's
  __device__ __forceinline__ explicit Pieces(const Share& s) : share(s), g(0), hk(0), b(0), pair(0), off(0), left(0), unit(blockIdx.x) {}
  // k units further on, by a warp together
  __device__ __forceinline__ void advance(const ChunkSizes& p, long long k) {
    k += pair;
    for (;;) {
      const int pairs = b + lane_id() < p.B ? pairs_of(span_of(p, b + lane_id()), p.rows[p.kind[g]]) : 0;
      const long long up = warp_scan(pairs);
      const uint32_t hit = __ballot_sync(0xffffffffu, up > k);
      if (hit != 0) {
        const int of = __ffs(hit) - 1;
        pair = int(k - __shfl_sync(0xffffffffu, up - pairs, of));
        b += of;
        return;
      }
      k -= __shfl_sync(0xffffffffu, up, 31);
      b += 32;
      if (b >= p.B) {
        b = 0;
        if (++hk == p.Hkv) {
          hk = 0;
          ++g;
        }
      }
    }
  }
  // The next piece, by a warp together; lane 0 writes it down.
  __device__ __forceinline__ void next(const ChunkSizes& p, Piece& out) {
    const int lane = lane_id();
    for (;;) {
      if (unit < share.rounds_end) {          // a whole unit, a round behind the last one
        advance(p, unit == blockIdx.x ? unit : (long long)gridDim.x);
        unit += gridDim.x;
        off = 0;
        left = INT_MAX;
      } else if (share.left >= 0) {           // on to the share
        g = share.g;
        hk = share.hk;
        b = share.b;
        pair = share.pair;
        off = share.off;
        left = share.left;
        share.left = -1;
        unit = LLONG_MAX;
      }
      if (left <= 0) break;
      const bool in_rounds = unit != LLONG_MAX;
      const Rows R = p.rows[p.kind[g]];
      const Span span = span_of(p, b);
      if (!in_rounds && pair >= pairs_of(span, R)) {        // on to the next sequence that has rows
        advance(p, 0);
        continue;
      }
      const Walked w = walked(p, span, R, pair);
      const int c0 = off, c1 = min(w.n, off + left);
      const int now = pair;
      left -= min(left, w.n + REST - off);
      off = 0;
      ++pair;
      if (in_rounds) pair = now;              // (the place that the next round is counted from)
      if (c0 >= c1) continue;
      if (lane == 0) {
        const int row = now * 2 * TILE, n_rows = span.n * R.n;
        const bool duo = row + TILE >= n_rows;
        auto clear = [&](int pos_first, int pos_last) {      // (blocks of first tokens count as masked)
          const int begin = p.window > 0 && pos_last >= p.window ? (pos_last - p.window) / STEP + 1 : 0, end = (pos_first + 1) / STEP;
          return make_int2(w.sink_blocks + max(begin - w.from, 0) - c0, w.sink_blocks + end - w.from - c0);
        };
        out.g = g;
        out.hk = hk;
        out.b = b;
        out.row0 = span.row0;
        out.pos0 = span.pos0;
        out.duo = !duo ? 0 : n_rows - row <= TILE / 2 ? 2 : 1;
        for (int x = 0; x < 2; ++x) {
          const int first = row + (duo ? 0 : x * TILE);
          out.rows[x] = min(TILE, n_rows - first);
          out.token[x] = R.token(first);
          out.in[x] = first - out.token[x] * R.n;
        }
        const int n = c1 - c0;
        out.n_x[0] = duo ? (n + 1) / 2 : max(0, min(c1, w.n_a) - c0);
        out.n_x[1] = duo ? n / 2 : n;
        out.pos_first = w.pos_first;
        out.pos_last = w.pos_last;
        out.sinks = w.sink_blocks - c0;
        out.at_sinks = c0;
        out.at = w.from - w.sink_blocks + c0;
        out.clear = clear(w.pos_first, w.pos_last);
        out.clear_x[0] = duo ? out.clear : clear(w.pos_first, w.pos_last_a);
        out.clear_x[1] = duo ? out.clear : clear(span.pos0 + out.token[1], w.pos_last);
        out.whole = c0 == 0 && c1 == w.n;
        out.slot = 2 * int(blockIdx.x) + (c0 == 0 ? 1 : 0);
        out.n = n;
      }
      return;
    }
    if (lane == 0) out.n = 0;
  }
};

// ---------------------------------------------------------------------------------------------
// pieces of the kernel
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t tmem_ld_x1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr) : "memory");
  return r;
}
__device__ __forceinline__ void tmem_st_x4(uint32_t taddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float4 tmem_ld_x4(uint32_t taddr) {
  uint32_t a, b, c, d;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(taddr) : "memory");
  tmem_ld_wait();
  return make_float4(__uint_as_float(a), __uint_as_float(b), __uint_as_float(c), __uint_as_float(d));
}
// A number that is the same in the whole warp, so that the compiler knows it: what follows from it stays in uniform registers, from
// which tensor and copy instructions take their operands (moved there one by one, they cost the issuing warps half their time).
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ int2 uniform(int2 v) { return make_int2(uniform(v.x), uniform(v.y)); }
// A bounded wait of a whole warp: true in all lanes or in none (the roles that use warp-wide operations go on or leave together).
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int* err) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, err)); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t f32x4_to_e5m2(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return uint32_t(lo) | uint32_t(hi) << 16;
}
// Lane t of a quad holds four 16-byte parts of its row: of the parts t of the quad's four rows, row j's comes to v[4 j].
__device__ __forceinline__ void swap_in_quads(uint32_t* v, int t) {
#pragma unroll
  for (int bit = 1; bit <= 2; bit *= 2)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c & bit) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t &a = v[4 * c + i], &b = v[4 * (c | bit) + i];
        const uint32_t got = __shfl_xor_sync(0xffffffffu, t & bit ? a : b, bit);
        if (t & bit) a = got; else b = got;
      }
    }
}
// Sixteen e4m3 numbers: whether one of them is NaN, and all times 2^-8 as f16.  The bits of a finite one, its exponent and mantissa
// one place down from a half's upper byte, are that f16 number (subnormal ones too).  (The conversion instruction takes some
// seven others, and NaN with it: drafts of 16 sequences 526 us with it for K and V, 310 with K as an operand and V so.)
__device__ __forceinline__ uint32_t any_nan(const uint4& c) {
  const uint32_t m = 0x7f7f7f7fu, one = 0x01010101u;
  return (((c.x & m) + one) | ((c.y & m) + one) | ((c.z & m) + one) | ((c.w & m) + one)) & 0x80808080u;
}
// Of four columns' codes the even ones in one word and the odd ones in the other, which takes no permutation of bytes: so columns 4 i
// + 1 and 4 i + 2 are in each other's place, and whoever reads O puts them back.
__device__ __forceinline__ void widen16(const uint4& c, uint4 (&out)[2]) {
  auto even = [](uint32_t w) { return (w << 8 & 0x80008000u) | (w << 7 & 0x3f803f80u); };
  auto odd = [](uint32_t w) { return (w & 0x80008000u) | (w >> 1 & 0x3f803f80u); };
  out[0] = make_uint4(even(c.x), odd(c.x), even(c.y), odd(c.y));
  out[1] = make_uint4(even(c.z), odd(c.z), even(c.w), odd(c.w));
}
__device__ __forceinline__ uint32_t nan_too(uint32_t two) {       // 480 * 2^-8 is what NaN's bits come out as
  return two | ((two & 0x3f80u) == 0x3f80u ? 0x7f80u : 0) | ((two & 0x3f800000u) == 0x3f800000u ? 0x7f800000u : 0);
}
__device__ __forceinline__ void put_nan(uint4 (&out)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) out[i] = make_uint4(nan_too(out[i].x), nan_too(out[i].y), nan_too(out[i].z), nan_too(out[i].w));
}
// D[tmem] (+)= A[smem] * B[smem], 8-bit floating-point numbers
__device__ __forceinline__ void umma8_ss_w(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate, uint32_t leader) {
  asm volatile(
      "{\n"
      " .reg .pred p, q;\n"
      " .reg .b64 da, db;\n"
      " mov.b64 da, {%1, %3};\n"
      " mov.b64 db, {%2, %3};\n"
      " setp.ne.b32 p, %5, 0;\n"
      " setp.ne.b32 q, %6, 0;\n"
      " @q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n"
      "}\n" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
// upper word of the descriptor of a K-major tile of 64-byte rows with the 64-byte swizzle: 512 bytes between groups of eight rows
constexpr uint32_t DESC_HI_SW64 = (512u >> 4) | (1u << 14) | (4u << 29);

// O of this thread's row += p_j V_j for the keys `left` of a block, from the pool itself.  P is in TMEM by now, as the product takes
// it; `fresh`: O holds nothing yet.  A warp together.
template <int DH, bool BITS8>
__device__ __noinline__ void add_rows(const ChunkSizes& p, const ChunkGroup& grp, int b, int hk, int key0, unsigned long long left, unsigned long long seen,
                                      uint32_t tm_p, uint32_t tm_o, bool fresh) {
  for (int h = 0; h < DH / 32; ++h) {
    uint32_t acc[32];
    if (fresh) {
#pragma unroll
      for (int i = 0; i < 32; ++i) acc[i] = 0;
    } else {
      tmem_ld_x32(tm_o + h * 32, acc);
      tmem_ld_wait();
    }
    for (unsigned long long rest = left; rest != 0; rest &= rest - 1) {
      const int j = __ffsll(rest) - 1, key = key0 + j;
      const uint32_t two = tmem_ld_x1(tm_p + (j >> 1));
      tmem_ld_wait();
      const float2 pf = f16x2_to_f32(two);
      const float pj = BITS8 ? (j & 1 ? pf.y : pf.x) : __uint_as_float(j & 1 ? two & 0xffff0000u : two << 16);
      const int page = p.block_table[size_t(b) * p.max_pages + key / p.page_size];
      const bool takes = unsigned(page) < unsigned(p.n_pages) && (seen >> j & 1) != 0;
      const size_t row = takes ? (size_t(page) * p.Hkv + hk) * p.page_size + key % p.page_size : 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float2 v;
        if (BITS8) {
          v = f16x2_to_f32(e4m3x2_to_f16x2(reinterpret_cast<const uint16_t*>(grp.v_pool)[(row * DH + h * 32) / 2 + i]));
          v.x *= 0.00390625f, v.y *= 0.00390625f;
        } else {
          const uint32_t bits = reinterpret_cast<const uint32_t*>(grp.v_pool)[(row * DH + h * 32) / 2 + i];
          v = make_float2(__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u));
        }
        const int at0 = !BITS8 ? 2 * i : i / 2 * 4 + (i & 1), at1 = at0 + (BITS8 ? 2 : 1);        // (as widen16 leaves the columns)
        if (takes) {
          acc[at0] = __float_as_uint(fmaf(pj, v.x, __uint_as_float(acc[at0])));
          acc[at1] = __float_as_uint(fmaf(pj, v.y, __uint_as_float(acc[at1])));
        }
      }
      __syncwarp();      // (the next load of TMEM is one of the whole warp)
    }
    tmem_st_x32(tm_o + h * 32, acc);
  }
  tmem_st_wait();
}

// Steps that scores run ahead of the products with P: a score buffer is free once the product of its tile's step before last has been issued.
template <int KS>
__device__ __forceinline__ int scores_ahead(bool duo) {
  static_assert(KS > 2, "");
  return !duo ? 2 : KS > 4 ? 4 : KS - 1;
}
// ---------------------------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------------------------
template <int DH, bool BITS8, int NG>
__global__ void __launch_bounds__(ChunkSmem<DH, BITS8>::THREADS, 1) chunk_kernel(const __grid_constant__ ChunkParams<NG> p) {
  using L = ChunkSmem<DH, BITS8>;
  constexpr int KS = L::K_STAGES, VS = L::V_STAGES, RS = L::RAW_STAGES;
  constexpr int HALVES = DH / 64;      // 64-column (128-byte) blocks of a row

  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* const q_full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);   // [2] per tile: its rows have come (4 arrivals)
  uint64_t* const k_full = q_full + 2;          // [KS]
  uint64_t* const k_empty = k_full + KS;        // [KS]
  uint64_t* const v_full = k_empty + KS;        // [VS]
  uint64_t* const v_empty = v_full + VS;        // [VS]
  uint64_t* const v_fixed = v_empty + VS;       // [VS] warp 3 has looked through the block (8 bits: the converting warps have, at v_full)
  uint64_t* const s_full = v_fixed + VS;        // [2][2] per tile and score buffer
  uint64_t* const p_ready = s_full + 4;         // [2][2] (4 arrivals)
  uint64_t* const pv_done = p_ready + 4;        // [2] one completion per step's product
  uint64_t* const o_done = pv_done + 2;         // [2] a piece's last product
  uint64_t* const duo_ml = o_done + 2;          // the halves of a duo have left their rows' maxima and sums (8 arrivals),
  uint64_t* const duo_free = duo_ml + 1;        // and have read each other's O (8 arrivals)
  uint64_t* const piece_full = duo_free + 1;    // [PIECES]
  uint64_t* const piece_empty = piece_full + PIECES;   // [PIECES] (an arrival of each warp that reads them)
  uint64_t* const raw_full = piece_empty + PIECES;     // [RS]
  uint64_t* const raw_empty = raw_full + RS;    // [RS] (4 arrivals)
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(q_full + L::BARRIERS);
  Piece* const s_pieces = reinterpret_cast<Piece*>(smem + L::OFF_PIECES);
  unsigned long long* const s_bad = reinterpret_cast<unsigned long long*>(smem + L::OFF_BAD);
  Scales* const s_scales = reinterpret_cast<Scales*>(smem + L::OFF_SCALE);

  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  int* const err = &g_chunk_status;

  if (threadIdx.x == 0) {
    mbar_init(duo_ml, 8);
    mbar_init(duo_free, 8);
    for (int i = 0; i < PIECES; ++i) {
      mbar_init(&piece_full[i], 1);
      mbar_init(&piece_empty[i], L::THREADS / 32 - 1);
    }
    for (int i = 0; i < KS; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 2);
    }
    for (int i = 0; i < VS; ++i) {
      mbar_init(&v_full[i], BITS8 ? 4 : 1);
      mbar_init(&v_empty[i], BITS8 ? 2 : 3);    // both issuing warps, and warp 3: nobody may fall a round of the ring behind
      mbar_init(&v_fixed[i], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_ready[i], 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 4);
      mbar_init(&pv_done[i], 1);
      mbar_init(&o_done[i], 1);
    }
    for (int i = 0; i < RS; ++i) {
      mbar_init(&raw_full[i], 1);
      mbar_init(&raw_empty[i], 4);
    }
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = uniform(*tmem_slot);
  grid_dep_wait();
  const Sums sums(smem + L::OFF_Q, p);          // (no query, K or V has been loaded)
  list_sums(p, sums, L::THREADS / 32);
  Share share{0, 0, 0, 0, 0, 0, 0};
  {
    const Deal deal = deal_out(p, sums, L::OFF_BAR - L::OFF_Q - int(static_cast<uint8_t*>(sums.end(p)) - (smem + L::OFF_Q)), L::THREADS / 32);
    if (warp == 3) share = find_share(p, sums, deal);
  }
  fence_proxy_async_smem();     // (at 16384 sequences the sums reach into K's stages)
  __syncthreads();
  uint32_t at = 0;      // steps of earlier pieces: ring positions of this piece's first
  uint32_t it = 0;      // pieces so far
  bool ok = true;
  // The piece that the role is at; it stays in the ring until the role gives it back.
  auto piece_at = [&](uint32_t i) -> const Piece* {
    ok = ok && warp_wait(&piece_full[i % PIECES], (i / PIECES) & 1, err);
    const Piece* const of = s_pieces + i % PIECES;
    return ok && uniform(of->n) > 0 ? of : nullptr;
  };
  auto give_back = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(&piece_empty[it % PIECES]);
    ++it;
  };
  // tile X: score buffer u at [X*128 + u*64, +64) with P over its first 32 columns; O at [256 + X*128, +DH)

  if (warp < 4) {
    if constexpr (BITS8) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::OTHER_REGS));
  }
  if (warp == 0) {
    // ------------------------------ K and V, or their codes ------------------------------
    const uint32_t leader = elect_one();    // the whole warp runs the loop; one lane issues
    while (const Piece* const piece = piece_at(it)) {
      const ChunkGroup& grp = p.grp[uniform(piece->g)];
      const int n = uniform(piece->n), hk = uniform(piece->hk);
      // Four lanes a step, a block of 16 keys each: rows of the pool (-1: no row of the unit sees any of the box's keys), and scales.
      // Pages are asked for two batches ahead, scales one.
      const int sub = lane & 3;
      const int none = p.n_pages * p.Hkv * p.page_size, per_box = p.box / 16;        // (behind the pool: TMA fills in zeros)
      auto box_key = [&](int i) { return (piece->block(i) * STEP + sub * 16) / p.box * p.box; };
      auto page_of = [&](int batch) -> int {
        const int i = batch * BATCH + (lane >> 2);
        if (i >= n) return -1;
        const int key = box_key(i);
        if (piece->unseen(p, key, p.box)) return -1;
        const int page = p.block_table[size_t(piece->b) * p.max_pages + key / p.page_size];
        return unsigned(page) < unsigned(p.n_pages) ? page : -2;
      };
      auto row_of = [&](int batch, int page) -> int {
        const int i = batch * BATCH + (lane >> 2);
        return page >= 0 ? (page * p.Hkv + hk) * p.page_size + box_key(i) % p.page_size : none;
      };
      auto boxes_of = [&](int page) -> uint32_t { return __ballot_sync(0xffffffffu, page != -1 && sub % per_box == 0); };
      auto scales_of = [&](int batch, int page) -> uint32_t {  // K's and V's
        const int i = batch * BATCH + (lane >> 2);
        if (!BITS8 || i >= n || page < 0) return 0x7f;         // (V's the smallest: the zeros of a missing page raise no reference of the weights)
        const size_t block = (size_t(page) * p.Hkv + hk) * (p.page_size / CACHE_BLOCK) + (piece->block(i) * STEP + sub * 16) % p.page_size / CACHE_BLOCK;
        return grp.k_scale[block] | uint32_t(grp.v_scale[block]) << 8;
      };
      // K or V of a step, whose pages are in lanes lane0 .. lane0 + 3
      auto load = [&](int i, int row, uint32_t boxes, auto is_v) -> bool {
        constexpr bool v = decltype(is_v)::value;
        constexpr uint32_t ring = !v ? KS : BITS8 ? RS : VS;
        const uint32_t j = at + i, s = j % ring, lane0 = (i % BATCH) * 4;
        uint64_t* const full = !v ? &k_full[s] : BITS8 ? &raw_full[s] : &v_full[s];
        if (!warp_wait(!v ? &k_empty[s] : BITS8 ? &raw_empty[s] : &v_empty[s], ((j / ring) & 1) ^ 1, err)) return false;
        boxes = boxes >> lane0 & 15;
        if constexpr (BITS8) __syncwarp();           // (the scales are written)
        mbar_expect_tx_e(full, uint32_t(__popc(boxes)) * p.box * DH * (BITS8 ? 1 : 2), leader);
        uint8_t* const tile = smem + (!v ? L::OFF_K + s * L::K_BYTES : BITS8 ? L::OFF_RAW + s * L::RAW_BYTES : L::OFF_V + s * L::V_BYTES);
        const CUtensorMap* const map = v ? &grp.map_v : &grp.map_k;
        for (int b = 0; b < 4; b += per_box) {
          const int y = __shfl_sync(0xffffffffu, row, lane0 + b);
          if constexpr (BITS8) {
            tma_load_2d_e(tile + b * 16 * DH, map, full, 0, y, leader & boxes >> b);
          } else {
#pragma unroll
            for (int h = 0; h < HALVES; ++h) tma_load_2d_e(tile + h * KV_HALF + b * 16 * 128, map, full, h * 64, y, leader & boxes >> b);
          }
        }
        return true;
      };
      constexpr std::false_type is_k;
      constexpr std::true_type is_v;
      if constexpr (BITS8) {
        // K and V side by side: V's way is the longer one.
        int page = page_of(0), page1 = page_of(1);
        uint32_t scales = scales_of(0, page);
        for (int batch = 0; batch * BATCH < n && ok; ++batch) {
          const int page2 = page_of(batch + 2);
          const uint32_t scales1 = scales_of(batch + 1, page1);
          const int mine = batch * BATCH + (lane >> 2), row = row_of(batch, page);
          const uint32_t boxes = boxes_of(page);
          for (int i = batch * BATCH; i < min(n, (batch + 1) * BATCH) && ok; ++i) {
            if (mine == i) {               // (ahead of K, which the scores wait for)
              float* const of = reinterpret_cast<float*>(s_scales + (at + i) % SCALES) + sub;
              of[0] = __uint_as_float(power_bits(exponent_of_byte(scales & 255)));
              of[4] = __uint_as_float(power_bits(exponent_of_byte(scales >> 8)));
              of[8] = float(exponent_of_byte(scales >> 8));
            }
            ok = load(i, row, boxes, is_k) && load(i, row, boxes, is_v);
          }
          page = page1;
          page1 = page2;
          scales = scales1;
        }
      } else {
        // K as far ahead of V as the scores run ahead of the products: both rings are then full of what is to come.
        const int ahead = scores_ahead<KS>(uniform(piece->duo) != 0);
        int page1 = page_of(0), page2 = page_of(1), row0 = none, row1 = row_of(0, page1);
        uint32_t boxes0 = 0, boxes1 = boxes_of(page1);
        for (int i = 0; i < ahead && i < n && ok; ++i) ok = load(i, row1, boxes1, is_k);
        for (int batch = 0; batch * BATCH < n && ok; ++batch) {
          const int page3 = page_of(batch + 2);
          row0 = row1;
          boxes0 = boxes1;
          row1 = row_of(batch + 1, page2);
          boxes1 = boxes_of(page2);
          const int end = (batch + 1) * BATCH;
          for (int i = batch * BATCH; i < min(n, end) && ok; ++i) {
            const bool next = i + ahead >= end;
            if (i + ahead < n) ok = load(i + ahead, next ? row1 : row0, next ? boxes1 : boxes0, is_k);
            ok = ok && load(i, row0, boxes0, is_v);
          }
          page2 = page3;
        }
      }
      at += n;
      give_back();
    }
    grid_dep_launch();
  } else if (warp == 1 || warp == 2) {
    // ------------------------------ MMA issuer of tile x ------------------------------
    const uint32_t leader = elect_one();
    // The types of A and B are in bits 7 and 10: bf16; 8-bit cache: P and V in f16, K in e4m3 with Q's two parts in e4m3 and e5m2.
    constexpr uint32_t no_types = ~((1u << 7) | (1u << 10));
    constexpr uint32_t idesc_qk = BITS8 ? umma_idesc_bf16(TILE, STEP, 0, 0) & no_types : umma_idesc_bf16(TILE, STEP, 0, 0);
    constexpr uint32_t idesc_pv = BITS8 ? umma_idesc_bf16(TILE, DH, 0, 1) & no_types : umma_idesc_bf16(TILE, DH, 0, 1);
    constexpr uint32_t hi = desc_hi_sw128(1024);
    constexpr uint32_t hi8 = DH == 128 ? hi : DESC_HI_SW64;        // rows of e4m3 numbers
    const uint32_t k_base = smem_u32(smem + L::OFF_K), v_base = smem_u32(smem + L::OFF_V);
    const int x = warp - 1;
    const uint32_t q_lo = desc_lo_sw128(smem_u32(smem + L::OFF_Q + x * L::Q_BYTES), 0);
    const uint32_t tm_s = tmem_base + x * 128, tm_o = tmem_base + 256 + x * 128;
    uint32_t done = 0, n_done = 0;    // steps of earlier pieces in which this tile took part; those pieces
    while (const Piece* const piece = piece_at(it)) {
      const int n = uniform(piece->n), n_x = uniform(piece->n_x[x]);
      const bool duo = uniform(piece->duo) != 0;
      const int2 clear = uniform(piece->clear);
      // (the tile's steps are i itself, or those of its parity)
      auto takes = [&](int i) { return duo ? (i & 1) == x : i < n_x; };
      auto own = [&](int i) { return done + (duo ? i >> 1 : i); };
      auto k_come = [&](int i) -> bool { return warp_wait(&k_full[(at + i) % KS], ((at + i) / KS) & 1, err); };
      // K of step i has come: scores, where the tile takes part
      auto scores = [&](int i) {
        if (!takes(i)) return;
        const uint32_t u = own(i) & 1, k_lo = desc_lo_sw128(k_base + (at + i) % KS * L::K_BYTES, 0);
        if constexpr (BITS8) {
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int ks = 0; ks < DH / 32; ++ks)
              umma8_ss_w(tm_s + u * STEP, desc_lo_add(q_lo, part * (TILE * DH) + ks * 32), desc_lo_add(k_lo, ks * 32), hi8, idesc_qk | (part << 7), (part | ks) != 0, leader);
        } else {
#pragma unroll
          for (int ks = 0; ks < DH / 16; ++ks)
            umma_ss_w(tm_s + u * STEP, desc_lo_add(q_lo, (ks / 4) * Q_HALF + (ks % 4) * 32), desc_lo_add(k_lo, (ks / 4) * KV_HALF + (ks % 4) * 32), hi, idesc_qk, ks != 0,
                      leader);
        }
        umma_commit(&s_full[2 * x + u], leader);
      };
      // stages go back: behind this warp's products with them, or at once where it has none
      auto release = [&](uint64_t* bar, bool taken) {
        if (taken)
          umma_commit(bar, leader);
        else if (leader)
          mbar_arrive(bar);
      };
      if (n_x > 0 && !warp_wait(&q_full[x], n_done & 1, err)) { ok = false; break; }
      const int ahead = scores_ahead<KS>(duo);
      for (int i = 0; i < ahead && i < n && ok; ++i) {
        ok = k_come(i);
        if (!ok) break;
        tc_fence_after_sync();
        scores(i);
        release(&k_empty[(at + i) % KS], takes(i));
      }
      for (int i = 0; i < n && ok; ++i) {
        // (everything that the products and the next scores wait for ahead of P, which comes last)
        const uint32_t s = (at + i) % VS;
        const bool further = i + ahead < n;
        if (!warp_wait(&v_full[s], ((at + i) / VS) & 1, err) || (further && !k_come(i + ahead))) { ok = false; break; }
        const bool mine = takes(i);
        if (mine) {
          const uint32_t k = own(i), u = k & 1, v_lo = desc_lo_sw128(v_base + s * L::V_BYTES, KV_HALF);
          uint32_t add = k != done;
          if (i < clear.x || i >= clear.y) {
            if (!BITS8 && !warp_wait(&v_fixed[s], ((at + i) / VS) & 1, err)) { ok = false; break; }
            // (the softmax threads have begun O with the rows that they add themselves)
            if (k == done) add = (s_bad[s * 4] | s_bad[s * 4 + 1] | s_bad[s * 4 + 2] | s_bad[s * 4 + 3]) != 0;
          }
          if (!warp_wait(&p_ready[2 * x + u], (k >> 1) & 1, err)) { ok = false; break; }
          tc_fence_after_sync();
#pragma unroll
          for (int ks = 0; ks < STEP / 16; ++ks)
            umma_ts_w(tm_o, tm_s + u * STEP + ks * 8, desc_lo_add(v_lo, ks * 2048), hi, idesc_pv, ks == 0 ? add : 1u, leader);
          umma_commit(&pv_done[x], leader);
          if (k + 1 == done + n_x) umma_commit(&o_done[x], leader);
        }
        if (further) {
          if (!mine) tc_fence_after_sync();
          scores(i + ahead);
          release(&k_empty[(at + i + ahead) % KS], takes(i + ahead));
        }
        release(&v_empty[s], mine);
      }
      at += n;
      done += n_x;
      n_done += n_x > 0 ? 1 : 0;
      give_back();
    }
  } else if (warp == 3) {
    // ------------------------------ the pieces; V blocks with masking ------------------------------
    Pieces pieces(share);
    // A piece is laid out one ahead of the one whose V blocks are looked through.
    auto lay_out = [&](uint32_t i) {
      ok = ok && warp_wait(&piece_empty[i % PIECES], ((i / PIECES) & 1) ^ 1, err);
      if (!ok) return false;
      Piece* const of = s_pieces + i % PIECES;
      pieces.next(p, *of);
      __syncwarp();
      const bool some = uniform(of->n) > 0;
      if (lane == 0) mbar_arrive(&piece_full[i % PIECES]);
      return some;
    };
    bool more = lay_out(0);
    while (more) {
      const Piece* const piece = s_pieces + it % PIECES;
      const int n = uniform(piece->n);
      // (behind the first steps of a long piece, whose blocks may have masks that its products wait for)
      const int lay_at = !BITS8 && n > 8 ? 2 : 0;
      if (lay_at == 0) more = lay_out(it + 1);
      if constexpr (!BITS8) {
        constexpr int CHUNKS = DH / 8;       // 16-byte pieces of a row
        const int2 clear = uniform(piece->clear);
        for (int i = 0; i < n && ok; ++i) {
          const uint32_t s = (at + i) % VS;
          if (lay_at > 0 && i == lay_at) more = lay_out(it + 1);
          ok = ok && warp_wait(&v_full[s], ((at + i) / VS) & 1, err);
          if (!ok) break;
          if (i < clear.x || i >= clear.y) {
            const int block = piece->block(i);
            uint8_t* const v = smem + L::OFF_V + s * L::V_BYTES;
            unsigned long long bad = 0;
#pragma unroll
            for (int part = 0; part < 2; ++part) {
              const int r = part * 32 + lane;
              const bool dead = piece->unseen(p, block * STEP + r, 1);
              uint32_t most = 0;               // largest magnitudes, as bits
              if (!dead)
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                  const uint4 w = *reinterpret_cast<const uint4*>(v + (c / 8) * KV_HALF + sw128_offset(r, c % 8));
                  constexpr uint32_t no_sign = 0x7fff7fffu;
                  most = __vimax3_s16x2(most, w.x & no_sign, w.y & no_sign);
                  most = __vimax3_s16x2(most, w.z & no_sign, w.w & no_sign);
                }
              const bool odd = (most & 0xffffu) >= 0x7f80u || most >= 0x7f800000u;
              if (dead || odd)
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) *reinterpret_cast<uint4*>(v + (c / 8) * KV_HALF + sw128_offset(r, c % 8)) = make_uint4(0, 0, 0, 0);
              bad |= (unsigned long long)__ballot_sync(0xffffffffu, odd) << (32 * part);
            }
            if (lane < 4) s_bad[s * 4 + lane] = lane == 0 ? bad : 0;
            fence_proxy_async_smem();
          }
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&v_fixed[s]);
            mbar_arrive(&v_empty[s]);
          }
        }
        at += n;
      }
      more = more && ok;
      ++it;
    }
  } else if (warp < 12) {
    // ------------------------------ softmax of tile x, and its rows of the outputs ------------------------------
    if constexpr (BITS8) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::SOFTMAX_REGS));
    const int x = (warp - 4) >> 2, quarter = warp & 3;
    // the warp's first row of a piece, at its TMEM lanes (below 0: none)
    auto first_row = [&](const Piece* of) { return quarter * 32 - (of->duo == 2 && x == 1 ? TILE / 2 : 0); };
    const uint32_t lane_sel = uint32_t(quarter * 32) << 16;
    const uint32_t tm_s = tmem_base + x * 128 + lane_sel, tm_o = tmem_base + 256 + x * 128 + lane_sel;
    float c_next = 1.f;                  // 8 bits: a power of two, which takes back what the thread's row has been multiplied by
    uint32_t done = 0, n_done = 0, n_duo = 0;       // steps of earlier pieces in which this tile took part; those pieces; duos
    // The warp's query rows of a piece go to their places: every product with the last one's has been seen to complete.  Four lanes a row,
    // and four rows one after the other: a row a lane, its 16-byte parts were as many lines each (3200 cycles a piece, and its output
    // the same way 5400).
    // Rows that a tile has not are zeros, and their products then take little of the power that bounds large calls.
    bool clean = false;                  // all of the warp's are zeros
    const int t = lane & 3, quad = lane & ~3;
    auto of_row = [&](const void* own, int j) {            // row quad + j's
      return reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(own), quad + j));
    };
    auto ask_q = [&](const Piece* of) {
      const int r0 = uniform(first_row(of)), r = r0 + lane;
      if (of->n_x[x] == 0) return;
      if (r0 < 0 || r0 >= of->rows[x]) {
        for (int i = lane; !clean && i < 32 * DH / 8; i += 32) {
          const int row = quarter * 32 + i / (DH / 8), c = i % (DH / 8);
          *reinterpret_cast<uint4*>(smem + L::OFF_Q + x * L::Q_BYTES + (BITS8 ? quarter * 32 * DH + (c & 1) * (TILE * DH) + i / 2 * 16 : (c / 8) * Q_HALF + sw128_offset(row, c % 8))) = make_uint4(0, 0, 0, 0);
        }
        clean = true;
        return;
      }
      clean = false;
      const void* own = nullptr;
      if (r < of->rows[x]) {
        const Rows R = p.rows[p.kind[of->g]];
        const int more = R.token(of->in[x] + r), in = of->in[x] + r - more * R.n, member = p.heads.token(in);
        const size_t elem = (size_t(of->row0 + of->token[x] + more) * p.Hq + of->hk * p.G + in - member * p.G) * DH;
        own = static_cast<const uint8_t*>(p.grp[of->g].q[member]) + elem * (p.io_f32 ? 4 : 2);
      }
      uint8_t* const tile = smem + L::OFF_Q + x * L::Q_BYTES;
      auto eight = [&](const uint8_t* row, int c) -> uint4 {               // as bf16
        if (!p.io_f32) return reinterpret_cast<const uint4*>(row)[c];
        const float4* const src = reinterpret_cast<const float4*>(row) + 2 * c;
        const float4 a = src[0], b = src[1];
        return make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
      };
#pragma unroll 1
      for (int j = 0; j < 4; ++j) {
        const uint8_t* const row = of_row(own, j);
        const int at_row = quarter * 32 + quad + j;
        if constexpr (BITS8) {
          // A number as the sum of two, e4m3 and e5m2, which both go into products with K as it is: a bf16 number's eight bits are
          // four and three (what is left by rounding to four bits is eight steps of the eighth at the most).  By a power of two a
          // row, the largest to 2^7 (no further than by 2^120): exact for all elements down to 2^-13 of it.  Below that e4m3's steps
          // stay 2^-9 and leave more than three bits: off by 2^-21 of the largest at most, where a product with it is rounded by 2^-24.
          // (Three parts in e5m2 are exact to 2^-23 of it, but take 32 KB from the rings at heads of 128: drafts 309 us instead of 249.)
          uint4 v[DH / 64][2];
          float most = 0.f;
#pragma unroll
          for (int c = 0; c < DH / 64; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              v[c][e] = row != nullptr ? eight(row, 2 * (4 * c + t) + e) : make_uint4(0, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t two = i == 0 ? v[c][e].x : i == 1 ? v[c][e].y : i == 2 ? v[c][e].z : v[c][e].w;
                most = fmaxf(most, fmaxf(fabsf(__uint_as_float(two << 16)), fabsf(__uint_as_float(two & 0xffff0000u))));
              }
            }
          most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
          most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
          const int up = min(max(7 + 127 - int(__float_as_uint(most) >> 23), -120), 120);
          const float power = __uint_as_float(uint32_t(up + 127) << 23);
          if (t == j) c_next = p.scale_power * __uint_as_float(uint32_t(127 - up) << 23);
          {
#pragma unroll
            for (int c = 0; c < DH / 64; ++c) {
              uint32_t hi[4], lo[4];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                  const uint32_t a = i == 0 ? v[c][e].x : v[c][e].z, b = i == 0 ? v[c][e].y : v[c][e].w;
                  float f[4] = {__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)};
#pragma unroll
                  for (int k = 0; k < 4; ++k) f[k] = fabsf(f[k]) < INFINITY ? f[k] * power : NAN;
                  hi[2 * e + i] = f32x4_to_e4m3(f[0], f[1], f[2], f[3]);
                  const float2 y = f16x2_to_f32(e4m3x2_to_f16x2(uint16_t(hi[2 * e + i]))), z = f16x2_to_f32(e4m3x2_to_f16x2(uint16_t(hi[2 * e + i] >> 16)));
                  lo[2 * e + i] = f32x4_to_e5m2(f[0] - y.x, f[1] - y.y, f[2] - z.x, f[3] - z.y);
                }
              }
              const int part = 4 * c + t;
              const uint32_t at8 = DH == 128 ? sw128_offset(at_row, part) : at_row * 64u + ((part ^ (at_row >> 1 & 3)) << 4);
              *reinterpret_cast<uint4*>(tile + at8) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
              *reinterpret_cast<uint4*>(tile + TILE * DH + at8) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
          }
        } else {
#pragma unroll
          for (int c4 = 0; c4 < DH / 8; c4 += 4) {
            const int c = c4 + t;
            uint8_t* const place = tile + (c / 8) * Q_HALF + sw128_offset(at_row, c % 8);
            if (row == nullptr)
              *reinterpret_cast<uint4*>(place) = make_uint4(0, 0, 0, 0);
            else if (p.io_f32)
              *reinterpret_cast<uint4*>(place) = eight(row, c);
            else
              cp_async16(smem_u32(place), row + c * 16, 16);
          }
        }
      }
      cp_async_commit();
    };
    auto give_q = [&](const Piece* of) {
      if (of->n_x[x] == 0) return;
      cp_async_wait<0>();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[x]);
    };
    const Piece* piece = piece_at(0);
    if (piece != nullptr) {
      ask_q(piece);
      give_q(piece);
    }
    while (piece != nullptr) {
      const int r0 = uniform(first_row(piece)), r = r0 + lane;
      const bool any = r0 >= 0 && r0 < piece->rows[x];      // (the same in the whole warp)
      const bool duo = uniform(piece->duo) != 0, apart = uniform(piece->duo) == 2;
      const int2 pair_clear = uniform(piece->clear), clear = uniform(piece->clear_x[x]);
      const int n_x = uniform(piece->n_x[x]);
      const float c_row = c_next;
      float m_used = -INFINITY;          // running maximum (log2 domain) that the exponentials are taken against,
      float c_used = 0.f, nm = 0.f;      // the factor of the scores (8 bits: beside K's powers), what is added to them,
      float limit = 0.f;                 // and how far above it a score moves it (log2)
      float d_used = -INFINITY;          // 8 bits: what O is in units of, relative to the maximum (log2; of the size of V's powers)
      const float c_all = BITS8 ? p.scale_rest : p.scale, c_far = BITS8 ? 1.f : p.scale_power;
      auto refer_to = [&](float largest) {                      // (8 bits: in units of powers of two)
        const float c = fabsf(largest * c_all) > FAR ? c_far : c_all;
        const bool none = largest == -INFINITY;                 // (a row that has seen nothing yet: all terms are 0)
        m_used = largest * c_all;
        c_used = BITS8 ? c_row * c : c;
        nm = none ? 0.f : -(largest * c);
        limit = none ? -FLT_MAX : kRescaleBy;
      };
      uint64_t l2 = 0ull, l2b = 0ull;
      for (int k = 0; k < n_x; ++k) {
        const int i = duo ? 2 * k + x : k;
        const uint32_t u = (done + k) & 1;
        ok = warp_wait(&s_full[2 * x + u], ((done + k) >> 1) & 1, err);
        if (!ok) break;
        tc_fence_after_sync();
        const uint32_t tm_su = tm_s + u * STEP;
        bool rescale = false;
        float alpha = 1.f;
        unsigned long long seen = ~0ull;
        if (any) {
          float4 kp, vp, ve;
          if constexpr (BITS8) {
            const Scales& of = s_scales[(at + i) % SCALES];
            kp = of.k, vp = of.v, ve = of.e;
          }
          uint32_t sv[STEP];
          tmem_ld_x32(tm_su, *reinterpret_cast<uint32_t(*)[32]>(&sv[0]));
          tmem_ld_x32(tm_su + 32, *reinterpret_cast<uint32_t(*)[32]>(&sv[32]));
          tmem_ld_wait();
          if (i < clear.x || i >= clear.y) {
            const int key0 = piece->block(i) * STEP;
            const int pos = piece->pos0 + piece->token[x] + p.rows[p.kind[piece->g]].token(piece->in[x] + min(r, piece->rows[x] - 1));
            auto below = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };
            seen = below(pos - key0 + 1);
            if (p.window > 0) seen &= ~below(pos - p.window + 1 - key0) | below(p.sinks - key0);
            const uint32_t lo = uint32_t(seen), up = uint32_t(seen >> 32);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if ((lo >> j & 1) == 0) sv[j] = 0xff800000u;        // -inf
              if ((up >> j & 1) == 0) sv[32 + j] = 0xff800000u;
            }
          }
          float mp[4];
          if constexpr (BITS8) {
            // A score is its product times K's power, a weight of V the probability times V's: 2^(s + e), in f16, relative to
            // the maximum and d_used, which rises (and O falls) where a weight would leave f16's upper range.  So scales cost no rounding, and a
            // weight has 11 bits unless it is below 2^-21 of the largest.
#pragma unroll
            for (int j = 0; j < 4; ++j) mp[j] = fmaxf(__uint_as_float(sv[16 * j]), __uint_as_float(sv[16 * j + 1]));
#pragma unroll
            for (int g = 2; g < 16; g += 2)
#pragma unroll
              for (int j = 0; j < 4; ++j) mp[j] = fmax3(mp[j], __uint_as_float(sv[16 * j + g]), __uint_as_float(sv[16 * j + g + 1]));
            const float k4[4] = {kp.x, kp.y, kp.z, kp.w};
            float cg[4], x4[4];          // factors of the blocks' scores (not zero: a masked score is -infinity times this), their largest
            auto scaled = [&]() {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                cg[j] = fmaxf(c_used * k4[j], FLT_MIN);
                x4[j] = fmaf(mp[j], cg[j], nm);
              }
              return fmaxf(fmaxf(x4[0], x4[1]), fmaxf(x4[2], x4[3]));
            };
            if (k == 0 || scaled() > limit) {
              float largest = -INFINITY;
#pragma unroll
              for (int j = 0; j < 4; ++j) largest = fmaxf(largest, mp[j] * fmaxf(c_row * k4[j], FLT_MIN));
              const float m_before = m_used;
              refer_to(largest);
              scaled();
              if (k > 0) {
                const float rise = m_used - m_before, f = fast_exp2(-rise);
                d_used -= rise;
                l2 = fmul2(l2, pack_f2(f, f));
                l2b = fmul2(l2b, pack_f2(f, f));
              }
            }
            const float d_step = fmaxf(fmaxf(x4[0] + ve.x, x4[1] + ve.y), fmaxf(x4[2] + ve.z, x4[3] + ve.w));
            if (k == 0) {
              d_used = d_step - 7.f;
            } else if (d_step > d_used + 15.f) {
              alpha = fast_exp2(d_used - (d_step - 7.f));
              d_used = d_step - 7.f;
              rescale = true;
            }
            const float unit = m_used == -INFINITY ? 0.f : fast_exp2(-d_used);
            // (finite: scales of blocks that the row does not see are of any size, and its probabilities there 0)
            constexpr float most = 3.4028235e38f;
            const float fg[4] = {fminf(unit * vp.x, most), fminf(unit * vp.y, most), fminf(unit * vp.z, most), fminf(unit * vp.w, most)};
            const uint64_t nm2 = pack_f2(nm, nm);
#pragma unroll
            for (int g = 0; g < STEP / 32; ++g) {
              uint32_t pk[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const int of16 = g * 2 + j / 8;
                const uint64_t e2 = ffma2(pack_f2(__uint_as_float(sv[g * 32 + 2 * j]), __uint_as_float(sv[g * 32 + 2 * j + 1])), pack_f2(cg[of16], cg[of16]), nm2);
                const uint64_t e = pack_f2(fast_exp2(f2_lo(e2)), fast_exp2(f2_hi(e2)));
                if (j & 1) l2b = fadd2(l2b, e); else l2 = fadd2(l2, e);
                const uint64_t w = fmul2(e, pack_f2(fg[of16], fg[of16]));
                pk[j] = pack_f16(f2_lo(w), f2_hi(w));
              }
              tmem_st_x16(tm_su + g * 16, pk);
            }
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) mp[j] = fmaxf(__uint_as_float(sv[2 * j]), __uint_as_float(sv[2 * j + 1]));
#pragma unroll
            for (int g = 8; g < STEP; g += 8)
#pragma unroll
              for (int j = 0; j < 4; ++j) mp[j] = fmax3(mp[j], __uint_as_float(sv[g + 2 * j]), __uint_as_float(sv[g + 2 * j + 1]));
            const float largest = fmaxf(fmaxf(mp[0], mp[1]), fmaxf(mp[2], mp[3]));
            if (k == 0) {
              refer_to(largest);
            } else if (fmaf(largest, c_used, nm) > limit) {
              const float m_before = m_used;
              refer_to(largest);
              alpha = fast_exp2(m_before - m_used);
              l2 = fmul2(l2, pack_f2(alpha, alpha));
              l2b = fmul2(l2b, pack_f2(alpha, alpha));
              rescale = true;
            }
            const uint64_t c2 = pack_f2(c_used, c_used);
            const uint64_t nm2 = pack_f2(nm, nm);
#pragma unroll
            for (int g = 0; g < STEP / 32; ++g) {
              uint32_t pk[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const uint64_t e2 = ffma2(pack_f2(__uint_as_float(sv[g * 32 + 2 * j]), __uint_as_float(sv[g * 32 + 2 * j + 1])), c2, nm2);
                const uint64_t e = pack_f2(fast_exp2(f2_lo(e2)), fast_exp2(f2_hi(e2)));
                if (j & 1) l2b = fadd2(l2b, e); else l2 = fadd2(l2, e);
                pk[j] = pack_bf16(f2_lo(e), f2_hi(e));
              }
              tmem_st_x16(tm_su + g * 16, pk);    // P as bf16 pairs over the first 32 columns of this score buffer
            }
          }
        }
        // O may still be receiving the last step's product: a rescale waits for it first.
        if (k > 0 && __any_sync(0xffffffffu, rescale)) {
          if (!warp_wait(&pv_done[x], (done + k - 1) & 1, err)) { ok = false; break; }
          tc_fence_after_sync();
#pragma unroll
          for (int g = 0; g < DH / 32; ++g) {
            uint32_t tmp[32];
            tmem_ld_x32(tm_o + g * 32, tmp);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) tmp[j] = __float_as_uint(__uint_as_float(tmp[j]) * alpha);
            tmem_st_x32(tm_o + g * 32, tmp);
          }
        }
        tmem_st_wait();
        if (i < pair_clear.x || i >= pair_clear.y) {
          const uint32_t s = (at + i) % VS;
          // (V first: only then is v_fixed past the stage's last use)
          if (!warp_wait(&v_full[s], ((at + i) / VS) & 1, err) || (!BITS8 && !warp_wait(&v_fixed[s], ((at + i) / VS) & 1, err))) { ok = false; break; }
          const unsigned long long bad = s_bad[s * 4] | s_bad[s * 4 + 1] | s_bad[s * 4 + 2] | s_bad[s * 4 + 3];
          if (bad != 0) {
            if (k > 0 && !warp_wait(&pv_done[x], (done + k - 1) & 1, err)) { ok = false; break; }
            tc_fence_after_sync();
            add_rows<DH, BITS8>(p, p.grp[piece->g], piece->b, piece->hk, piece->block(i) * STEP, bad, any ? seen : 0ull, tm_su, tm_o, k == 0);
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[2 * x + u]);
      }
      if (!ok) break;
      const Piece* const next = piece_at(it + 1);
      if (!ok) break;
      if (next != nullptr && !apart) ask_q(next);
      float m = m_used, l = (f2_lo(l2) + f2_hi(l2)) + (f2_lo(l2b) + f2_hi(l2b));
      if (n_x > 0) {
        if (!warp_wait(&o_done[x], n_done & 1, err)) break;
        tc_fence_after_sync();
        ++n_done;
      }
      // (8 bits: O is in units of its own, and V in shared memory 2^-8 of its codes)
      const float unit = !BITS8 ? 1.f : m == -INFINITY ? 0.f : fast_exp2(d_used + 8.f);
      float mine = unit, others = 0.f;
      // A duo's halves have the same rows, and each puts half of the columns together.  Maxima and sums are exchanged, and O read, by way
      // of TMEM (over a score buffer: the next piece has not begun); where the rows are at other lanes, by the room of the queries.
      auto shared_row = [&](int y) { return smem + L::OFF_Q + y * L::Q_BYTES + r * (DH * 2); };       // of half y: DH / 2 columns that it leaves to the other
      auto shared_ml = [&](int y) { return reinterpret_cast<float4*>(smem + L::OFF_Q + y * L::Q_BYTES + TILE / 2 * (DH * 2)) + r; };
      if (duo) {
        if (!apart) {
          tmem_st_x4(tm_s, __float_as_uint(m), __float_as_uint(l), __float_as_uint(unit), 0);
          tmem_st_wait();
        } else if (any) {
          *shared_ml(x) = make_float4(m, l, unit, 0.f);
          for (int h = 0; h < DH / 64 && n_x > 0; ++h) {
            uint32_t tmp[32];
            tmem_ld_x32(tm_o + ((x ^ 1) * (DH / 64) + h) * 32, tmp);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; ++j)
              *reinterpret_cast<uint4*>(shared_row(x) + (((h * 8 + j) ^ (r & 7)) << 4)) = make_uint4(tmp[4 * j], tmp[4 * j + 1], tmp[4 * j + 2], tmp[4 * j + 3]);
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(duo_ml);
        if (!warp_wait(duo_ml, n_duo & 1, err)) break;
        tc_fence_after_sync();
        const float4 other = !apart ? tmem_ld_x4(x == 0 ? tm_s + 128 : tm_s - 128) : any ? *shared_ml(x ^ 1) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        const float top = fmaxf(m, other.x);
        mine = m == -INFINITY ? 0.f : fast_exp2(m - top);
        others = other.x == -INFINITY ? 0.f : fast_exp2(other.x - top);
        l = l * mine + other.y * others;
        m = top;
        mine *= unit;
        others *= other.z;
      }
      // (the next piece's first scores run beside what is left of this one; those of a duo are over the halves' notes)
      if (!duo && next != nullptr) give_q(next);
      if (any) {
        const ChunkGroup& grp = p.grp[piece->g];
        const bool there = r < piece->rows[x], whole = piece->whole;
        const Rows R = p.rows[p.kind[piece->g]];
        const int more = R.token(piece->in[x] + r), in = piece->in[x] + r - more * R.n, member = p.heads.token(in);
        const size_t head = size_t(piece->row0 + piece->token[x] + more) * p.Hq + piece->hk * p.G + in - member * p.G;
        const size_t part = size_t(piece->slot) * (2 * TILE) + (duo ? 0 : x * TILE) + r;
        const float inv_l = l == 0.f ? 0.f : 1.f / l;
        if (there && !(duo && x == 1)) {
          if (whole)
            grp.lse[member][head] = l == 0.f ? -INFINITY : log_sum(m, l);
          else
            *reinterpret_cast<float2*>(p.part_ml + part * 2) = make_float2(m, l);
        }
        void* own = nullptr;
        if (there)
          own = !whole ? static_cast<void*>(p.part_o + part * DH) : static_cast<uint8_t*>(grp.o[member]) + head * DH * (p.io_f32 ? 4 : 2);
        uint8_t* rows[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) rows[j] = of_row(own, j);
        const int h_end = duo && x == 0 ? DH / 64 : DH / 32, n_other = duo ? piece->n_x[x ^ 1] : 0;
        if (duo || n_x > 0) {
          for (int h = duo && x == 1 ? DH / 64 : 0; h < h_end; ++h) {
            uint32_t tmp[32];
            if (n_x > 0) {
              tmem_ld_x32(tm_o + h * 32, tmp);
              tmem_ld_wait();
            }
            if (duo || BITS8) {
#pragma unroll
              for (int j = 0; j < 32; ++j) tmp[j] = n_x > 0 ? __float_as_uint(__uint_as_float(tmp[j]) * mine) : 0;
            }
            if (duo) {
              if (n_other > 0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  uint32_t far[16];
                  if (!apart) {
                    tmem_ld_x16((x == 0 ? tm_o + 128 : tm_o - 128) + h * 32 + e * 16, far);
                    tmem_ld_wait();
                  } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                      const int c = (h - x * (DH / 64)) * 8 + e * 4 + j;
                      const uint4 v = *reinterpret_cast<const uint4*>(shared_row(x ^ 1) + ((c ^ (r & 7)) << 4));
                      far[4 * j] = v.x, far[4 * j + 1] = v.y, far[4 * j + 2] = v.z, far[4 * j + 3] = v.w;
                    }
                  }
#pragma unroll
                  for (int j = 0; j < 16; ++j) tmp[e * 16 + j] = __float_as_uint(fmaf(__uint_as_float(far[j]), others, __uint_as_float(tmp[e * 16 + j])));
                }
              }
            }
            if constexpr (BITS8) {
#pragma unroll
              for (int j = 1; j < 32; j += 4) {
                const uint32_t other = tmp[j];
                tmp[j] = tmp[j + 1];
                tmp[j + 1] = other;
              }
            }
            if (!whole) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                swap_in_quads(&tmp[16 * e], t);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (rows[j] != nullptr)
                    *reinterpret_cast<uint4*>(rows[j] + (h * 32 + e * 16 + t * 4) * 4) = make_uint4(tmp[16 * e + 4 * j], tmp[16 * e + 4 * j + 1], tmp[16 * e + 4 * j + 2], tmp[16 * e + 4 * j + 3]);
              }
            } else {
              uint32_t v[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) v[j] = pack_bf16(__uint_as_float(tmp[2 * j]) * inv_l, __uint_as_float(tmp[2 * j + 1]) * inv_l);
              swap_in_quads(v, t);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (rows[j] == nullptr) continue;
                if (p.io_f32) {
                  uint4* const dst = reinterpret_cast<uint4*>(rows[j] + (h * 32 + t * 8) * 4);
                  dst[0] = make_uint4(v[4 * j] << 16, v[4 * j] & 0xffff0000u, v[4 * j + 1] << 16, v[4 * j + 1] & 0xffff0000u);
                  dst[1] = make_uint4(v[4 * j + 2] << 16, v[4 * j + 2] & 0xffff0000u, v[4 * j + 3] << 16, v[4 * j + 3] & 0xffff0000u);
                } else {
                  *reinterpret_cast<uint4*>(rows[j] + (h * 32 + t * 8) * 2) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                }
              }
            }
            __syncwarp();
          }
        }
      }
      __syncwarp();
      tc_fence_before_sync();
      if (duo) {
        if (lane == 0) mbar_arrive(duo_free);
        if (!warp_wait(duo_free, n_duo & 1, err)) break;
        ++n_duo;
      }
      // (the next piece's first products wait for these warps' P, so O is free by then)
      at += uniform(piece->n);
      done += n_x;
      if (apart) clean = false;
      if (next != nullptr && apart) ask_q(next);
      if (duo && next != nullptr) give_q(next);
      give_back();
      piece = next;
    }
  } else if constexpr (BITS8) {
    // ------------------------------ V's codes to f16 ------------------------------
    // (by eight warps, two groups in turn, which leave the softmax 144 registers a thread, not 192: drafts 240 us instead of 229, prompts 1108 and 1058)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::OTHER_REGS));
    constexpr int CODES = DH / 16;                       // 16-byte pieces of a row of codes
    constexpr int PASSES = STEP * CODES / 128;           // of the four warps; each 128 / CODES rows
    const int tid = threadIdx.x & 127, col = tid % CODES, flip = (col >> 2) & 1;
    while (const Piece* const piece = piece_at(it)) {
      const int n = uniform(piece->n);
      const int2 clear = uniform(piece->clear);
      for (int i = 0; i < n && ok; ++i) {
        const uint32_t j = at + i, s = j % VS, rs = j % RS;
        if (!warp_wait(&raw_full[rs], (j / RS) & 1, err) || !warp_wait(&v_empty[s], ((j / VS) & 1) ^ 1, err)) { ok = false; break; }
        uint4 codes[PASSES];
#pragma unroll
        for (int k = 0; k < PASSES; ++k) {
          // (the half of a column of codes that is stored first; the eight lanes of a phase of stores hit different banks that way)
          const uint8_t* const raw = smem + L::OFF_RAW + rs * L::RAW_BYTES + (k * 128 + tid) / CODES * DH + col * 16;
          const uint2 a = *reinterpret_cast<const uint2*>(raw + flip * 8), b = *reinterpret_cast<const uint2*>(raw + (flip ^ 1) * 8);
          codes[k] = make_uint4(a.x, a.y, b.x, b.y);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&raw_empty[rs]);
        uint8_t* const tile = smem + L::OFF_V + s * L::V_BYTES;
        auto store = [&](int k, const uint4 (&half)[2]) {
          const int row = (k * 128 + tid) / CODES;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int c = col * 2 + (h ^ flip);
            *reinterpret_cast<uint4*>(tile + (c / 8) * KV_HALF + sw128_offset(row, c % 8)) = half[h];
          }
        };
        uint32_t nan = 0;
#pragma unroll
        for (int k = 0; k < PASSES; ++k) nan |= any_nan(codes[k]);
        const bool masked = i < clear.x || i >= clear.y;
        if (!masked && __all_sync(0xffffffffu, nan == 0)) {
#pragma unroll
          for (int k = 0; k < PASSES; ++k) {
            uint4 half[2];
            widen16(codes[k], half);
            store(k, half);
          }
        } else {
          unsigned long long bad = 0;
#pragma unroll 1
          for (int k = 0; k < PASSES; ++k) {
            uint4 some = codes[0];
#pragma unroll
            for (int q = 1; q < PASSES; ++q)
              if (k == q) some = codes[q];
            const int row = (k * 128 + tid) / CODES;
            uint4 half[2];
            widen16(some, half);
            const bool dead = masked && piece->unseen(p, piece->block(i) * STEP + row, 1);
            const bool odd = !dead && any_nan(some) != 0;
            // the lanes of a row
            const uint32_t of_row = __ballot_sync(0xffffffffu, odd) >> (lane / CODES * CODES) & ((1u << CODES) - 1);
            if (dead || (masked && of_row != 0)) {
              half[0] = half[1] = make_uint4(0, 0, 0, 0);
            } else if (odd) {
              put_nan(half);
            }
            const uint32_t firsts = __ballot_sync(0xffffffffu, masked && of_row != 0 && lane % CODES == 0);
            for (int q = 0; q < 32 / CODES; ++q)
              if (firsts >> (q * CODES) & 1) bad |= 1ull << ((k * 128 + tid - lane) / CODES + q);
            store(k, half);
          }
          if (masked && lane == 0) s_bad[s * 4 + (tid >> 5)] = bad;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&v_full[s]);
      }
      at += n;
      give_back();
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
}

// ---------------------------------------------------------------------------------------------
// merge of the pieces of a unit: a warp per row, blockIdx.y a part of the unit's rows
// ---------------------------------------------------------------------------------------------
constexpr int MERGE_THREADS = 256, MERGE_PARTS = 8;
template <int DH, int NG>
__global__ void __launch_bounds__(MERGE_THREADS) chunk_merge_kernel(const __grid_constant__ ChunkParams<NG> p) {
  constexpr int COLS = DH / 32;         // columns of a lane
  grid_dep_launch();
  grid_dep_wait();
  const Merge m = p.merges[blockIdx.x];
  if (m.w0 < 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const ChunkGroup& grp = p.grp[m.g];
  const Span span = span_of(p, m.b);
  const Rows R = p.rows[p.kind[m.g]];
  const int row0 = m.pair * 2 * TILE, n_rows = span.n * R.n;
  for (int row = int(blockIdx.y) + MERGE_PARTS * warp; row < 2 * TILE; row += MERGE_PARTS * (MERGE_THREADS / 32)) {
    if (row0 + row >= n_rows) continue;
    float top = -INFINITY, sum = 0.f, acc[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[c] = 0.f;
    for (int w = m.w0; w <= m.w1; w += 32) {
      // the lane's piece: maximum and sum
      float pm = -INFINITY, pl = 0.f;
      if (w + lane <= m.w1) {
        const size_t part = size_t(2 * (w + lane) + (w + lane == m.w0 ? 1 : 0)) * (2 * TILE) + row;
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + part * 2);
        pm = ml.x;
        pl = ml.y;
      }
      float most = pm;
#pragma unroll
      for (int d = 16; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
      most = fmaxf(top, most);
      const float keep = top == -INFINITY ? 0.f : fast_exp2(top - most);
      top = most;
      sum *= keep;
#pragma unroll
      for (int c = 0; c < COLS; ++c) acc[c] *= keep;
      const float weight = pm == -INFINITY ? 0.f : fast_exp2(pm - most);
      float ws = weight * pl;
#pragma unroll
      for (int d = 16; d > 0; d /= 2) ws += __shfl_xor_sync(0xffffffffu, ws, d);
      sum += ws;
      const int n = min(32, m.w1 - w + 1);
      constexpr int FLY = 4;
      for (int i0 = 0; i0 < n; i0 += FLY) {
        float held[FLY][COLS], f[FLY];
#pragma unroll
        for (int k = 0; k < FLY; ++k) {
          const int i = i0 + k;
          f[k] = __shfl_sync(0xffffffffu, weight, i & 31);
          const float its = __shfl_sync(0xffffffffu, pm, i & 31);
          if (i >= n || its == -INFINITY) {      // (a piece without keys for this tile has left no sums)
            f[k] = 0.f;
#pragma unroll
            for (int c = 0; c < COLS; ++c) held[k][c] = 0.f;
            continue;
          }
          const size_t part = size_t(2 * (w + i) + (w + i == m.w0 ? 1 : 0)) * (2 * TILE) + row;
          const float* const src = p.part_o + part * DH + lane * COLS;
          if constexpr (COLS == 4) {
            const float4 v = *reinterpret_cast<const float4*>(src);
            held[k][0] = v.x, held[k][1] = v.y, held[k][2] = v.z, held[k][3] = v.w;
          } else {
            const float2 v = *reinterpret_cast<const float2*>(src);
            held[k][0] = v.x, held[k][1] = v.y;
          }
        }
#pragma unroll
        for (int k = 0; k < FLY; ++k)
#pragma unroll
          for (int c = 0; c < COLS; ++c) acc[c] = fmaf(held[k][c], f[k], acc[c]);
      }
    }
    const int token = R.token(row0 + row), in = row0 + row - token * R.n, member = p.heads.token(in);
    const size_t head = size_t(span.row0 + token) * p.Hq + m.hk * p.G + in - member * p.G;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint32_t v[COLS / 2];
#pragma unroll
    for (int c = 0; c < COLS / 2; ++c) v[c] = pack_bf16(acc[2 * c] * inv, acc[2 * c + 1] * inv);
    if (p.io_f32) {
      float* const dst = reinterpret_cast<float*>(grp.o[member]) + head * DH + lane * COLS;
#pragma unroll
      for (int c = 0; c < COLS / 2; ++c) *reinterpret_cast<uint2*>(dst + 2 * c) = make_uint2(v[c] << 16, v[c] & 0xffff0000u);
    } else {
      uint32_t* const dst = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(grp.o[member]) + head * DH + lane * COLS);
#pragma unroll
      for (int c = 0; c < COLS / 2; ++c) dst[c] = v[c];
    }
    if (lane == 0) grp.lse[member][head] = sum == 0.f ? -INFINITY : log_sum(top, sum);
  }
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
size_t merge_bytes(int shares) { return align256(size_t(shares) * sizeof(Merge)); }
size_t chunk_bytes(int shares, int dh) {
  return merge_bytes(shares) + align256(size_t(shares) * 2 * (2 * TILE) * dh * 4) + align256(size_t(shares) * 2 * (2 * TILE) * 2 * 4);
}
// Most shares that the call's list can be cut into: no unit of `rows` a token walks more steps than the table is long.
int shares_at_most(const kvp_decode_desc* d, int n_groups, int T) {
  const long long steps = ((long long)d->max_pages * d->page_size + STEP - 1) / STEP + REST;
  const long long units = ((long long)T * (CHUNK_MEMBERS * 16) / (2 * TILE) + std::min(T, d->B)) * d->Hkv * n_groups;
  const long long most = units > (1ll << 40) / steps ? (1ll << 40) : units * steps;
  return int(std::max(1ll, std::min((long long)sm_count(), most / LEAST_SHARE)));
}

int check_chunk(const kvp_decode_desc* d) {
  int rc = d == nullptr ? KVP_ERR_INVALID_ARG : KVP_OK;
  if (rc != KVP_OK) return rc;
  kvp_decode_desc plain = *d;
  plain.num_splits = 0;
  rc = check_desc(&plain);
  if (rc != KVP_OK) return rc;
  // positions, rows of the pool and of the sums in shared memory are counted in 32 bits
  if ((long long)d->max_pages * d->page_size > (1 << 30) || (long long)d->n_pages * d->Hkv * d->page_size > 0x7fffffffLL - STEP ||
      d->Hq > (1 << 16) || d->B > (1 << 14))
    return KVP_ERR_UNSUPPORTED;
  return KVP_OK;
}

// One token a sequence, few query rows: decode's kernels, on a table of the pages that the token sees.  Front pages of first tokens,
// then those from the window's first on; the positions between the two parts are one run, in the last page of the front or the
// first of the window (kvp_host.h).  Those kernels bring in rows of 16 queries where a tile here has 128, and take more rows in passes that
// read K and V again.  So up to 16 rows a group (us, on the tiles -> so; one group, 8 KV heads):
//   rows, bf16, 16 sequences of 4K-16K            8: 134 -> 120   16: 135 -> 119   24: 136 -> 225   32: 136 -> 231
//   the same in 8 bits                            8: 140 -> 67    16: 142 -> 92    24: 143 -> 160   32: 144 -> 165
//   bf16, 32 of 16K-32K under a window of 4096    8: 111 -> 92    16: 112 -> 93    24: 113 -> 181   32: 113 -> 185
//   8 bits, heads of 64, 58 of 1000-3000          8: 107 -> 40    16: 109 -> 59    24: 109 -> 113   32: 110 -> 122
// (4 of 100-200 stay faster so: 16.5 -> 11.5 at 24 and 32 rows.)
struct Ones {
  const int32_t *block_table, *lengths;
  int32_t *table, *shortened;              // [B, columns], [B]; null without a window
  int4* seen;                              // [B]
  int B, page_size, max_pages, columns, window, sinks;
};
constexpr int ONES_THREADS = 128;
__global__ void __launch_bounds__(ONES_THREADS) ones_kernel(const __grid_constant__ Ones p) {
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.x, length = p.lengths[b];
  const bool there = length > 0 && length <= p.max_pages * p.page_size;
  int4 seen = make_int4(0, 0, there, 0);
  if (p.table != nullptr) {
    const int len = there ? length : 0;
    const int from = max(0, len - p.window), front = min((p.sinks + p.page_size - 1) / p.page_size, from / p.page_size), left_out = from / p.page_size - front;
    const int shorter = len - left_out * p.page_size;
    if (p.sinks < from) {
      seen.x = min(p.sinks, len);
      seen.y = from - left_out * p.page_size;
    }
    const int n = (shorter + p.page_size - 1) / p.page_size;
    for (int i = threadIdx.x; i < n; i += ONES_THREADS)
      p.table[size_t(b) * p.columns + i] = p.block_table[size_t(b) * p.max_pages + (i < front ? i : i + left_out)];
    if (n == 0 && threadIdx.x == 0) p.table[size_t(b) * p.columns] = 0;      // (looked at before the length)
    if (threadIdx.x == 0) p.shortened[b] = shorter;
  }
  if (threadIdx.x == 0) p.seen[b] = seen;
}
// Columns of that table; they hold no more than the whole one has.
int ones_columns(const kvp_decode_desc* d, int window, int sinks) {
  return int(std::min((long long)d->max_pages, (long long)(sinks + d->page_size - 1) / d->page_size + ((long long)window + d->page_size - 2) / d->page_size + 1));
}
size_t ones_bytes(const kvp_decode_desc* d, const int32_t* donor, int columns, bool bits8) {
  return align256(size_t(d->B) * sizeof(int4)) + align256(size_t(d->B) * 4) + align256(size_t(d->B) * columns * 4) +
         (bits8 ? kvp_decode8_workspace_bytes(d, donor) : kvp_decode_workspace_bytes(d, donor));
}
// All layers of every donor group fit one pass of decode's.
bool few_rows(const kvp_decode_desc* d, const int32_t* donor, int begin, int end) {
  const int per = std::min(MAX_MEMBERS, 16 / (d->Hq / d->Hkv));
  for (int own = 0; own < end; ++own) {
    int n = 0;
    for (int l = begin; l < end; ++l) n += donor[l] == own;
    if (n > per) return false;
  }
  return true;
}

template <int DH, bool BITS8, int NG>
cudaError_t launch_chunk(const ChunkParams<MANY_CHUNK_GROUPS>& all, int shares, cudaStream_t stream) {
  using L = ChunkSmem<DH, BITS8>;
  static thread_local ChunkParams<NG> p;
  static_cast<ChunkSizes&>(p) = all;
  std::copy(all.grp, all.grp + NG, p.grp);
  cudaError_t e = allow_smem<chunk_kernel<DH, BITS8, NG>>(L::TOTAL);
  if (BITS8 && e == cudaSuccess) {     // the kernel hands registers from warp to warp: without as many at launch it would wait for good
    static const int regs = [] {
      cudaFuncAttributes at;
      return cudaFuncGetAttributes(&at, reinterpret_cast<const void*>(chunk_kernel<DH, BITS8, NG>)) == cudaSuccess ? at.numRegs : 0;
    }();
    if (regs != L::LAUNCH_REGS) return cudaErrorInvalidConfiguration;
  }
  if (e == cudaSuccess) e = launch_kernel(chunk_kernel<DH, BITS8, NG>, shares, L::THREADS, L::TOTAL, stream, 1, p);
  if (e == cudaSuccess && shares > 1) e = launch_kernel(chunk_merge_kernel<DH, NG>, dim3(shares, MERGE_PARTS), MERGE_THREADS, 0, stream, 1, p);
  return e;
}
template <int NG>
cudaError_t launch_chunk(const ChunkParams<MANY_CHUNK_GROUPS>& p, int dh, bool bits8, int shares, cudaStream_t stream) {
  return bits8 ? (dh == 128 ? launch_chunk<128, true, NG>(p, shares, stream) : launch_chunk<64, true, NG>(p, shares, stream))
               : (dh == 128 ? launch_chunk<128, false, NG>(p, shares, stream) : launch_chunk<64, false, NG>(p, shares, stream));
}

}  // namespace

int chunk_read_status() {
  int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_chunk_status, sizeof(int)) != cudaSuccess) return -1;
  if (v != 0) {
    int zero = 0;
    cudaMemcpyToSymbol(g_chunk_status, &zero, sizeof(int));
  }
  return v;
}

}  // namespace kvp

using namespace kvp;

extern "C" size_t kvp_attn_chunk_workspace_bytes(const kvp_decode_desc* d, const int32_t* donor, int32_t T) {
  if (check_chunk(d) != KVP_OK || donor == nullptr || T < 0) return 0;
  size_t bytes = chunk_bytes(shares_at_most(d, std::min(d->L, MANY_CHUNK_GROUPS), T), d->dh);
  if (T >= d->B) {
    kvp_decode_desc plain = *d;
    plain.num_splits = 0;
    bytes = std::max({bytes, ones_bytes(&plain, donor, d->max_pages, false), ones_bytes(&plain, donor, d->max_pages, true)});
  }
  return bytes;
}

extern "C" int kvp_attn_chunk(const kvp_decode_desc* d, const int32_t* donor, int32_t T, const int32_t* first, float scale, int32_t window, int32_t sinks,
                              const void* const* q, const void* const* k_cache, const void* const* v_cache, const uint8_t* const* k_scale,
                              const uint8_t* const* v_scale, const int32_t* block_table, const int32_t* lengths, void* const* o, float* const* lse,
                              int layer_begin, int layer_end, void* ws, size_t ws_bytes, kvp_stream_t stream_) {
  int rc = check_chunk(d);
  if (rc != KVP_OK) return rc;
  if (donor == nullptr || q == nullptr || k_cache == nullptr || v_cache == nullptr || o == nullptr || lse == nullptr || block_table == nullptr ||
      lengths == nullptr || (k_scale == nullptr) != (v_scale == nullptr))
    return KVP_ERR_INVALID_ARG;
  if (layer_begin < 0 || layer_end > d->L || layer_begin >= layer_end || T < 0 || (first == nullptr && T != d->B) || window < 0 || sinks < 0 ||
      (window == 0 && sinks > 0) || !(scale >= 0.f && scale < INFINITY))
    return KVP_ERR_INVALID_ARG;
  for (int l = 0; l < d->L; ++l)
    if (donor[l] < 0 || donor[l] > l || donor[donor[l]] != donor[l]) return KVP_ERR_BAD_DONOR;
  if (T > CHUNK_MOST_TOKENS) return KVP_ERR_UNSUPPORTED;
  if (T == 0) return KVP_OK;           // (tensors without rows have no memory)
  const bool bits8 = k_scale != nullptr;
  for (int l = layer_begin; l < layer_end; ++l) {     // all of them before anything is launched
    const int own = donor[l];
    if (q[l] == nullptr || o[l] == nullptr || lse[l] == nullptr || k_cache[own] == nullptr || v_cache[own] == nullptr ||
        (bits8 && (k_scale[own] == nullptr || v_scale[own] == nullptr)))
      return KVP_ERR_INVALID_ARG;
    if (!aligned16(q[l]) || !aligned16(o[l]) || !aligned16(k_cache[own]) || !aligned16(v_cache[own])) return KVP_ERR_UNSUPPORTED;
  }
  if (ws != nullptr && !aligned16(ws)) return KVP_ERR_UNSUPPORTED;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const int capacity = d->max_pages * d->page_size;
  if (window >= capacity) window = 0;             // (nothing is further back)
  sinks = window > 0 ? std::min(sinks, capacity) : 0;
  if (first == nullptr && few_rows(d, donor, layer_begin, layer_end)) {
    kvp_decode_desc ones = *d;
    ones.num_splits = 0;
    if (window > 0) ones.max_pages = ones_columns(d, window, sinks);
    if (ws == nullptr || ws_bytes < ones_bytes(&ones, donor, ones.max_pages, bits8)) return KVP_ERR_WORKSPACE;
    uint8_t* at = static_cast<uint8_t*>(ws);
    Ones p{block_table, lengths, nullptr, nullptr, reinterpret_cast<int4*>(at), d->B, d->page_size, d->max_pages, ones.max_pages, window, sinks};
    at += align256(size_t(d->B) * sizeof(int4));
    if (window > 0) {
      p.shortened = reinterpret_cast<int32_t*>(at);
      p.table = reinterpret_cast<int32_t*>(at + align256(size_t(d->B) * 4));
    }
    at += align256(size_t(d->B) * 4) + align256(size_t(d->B) * ones.max_pages * 4);
    if (launch_kernel(ones_kernel, d->B, ONES_THREADS, 0, stream, 1, p) != cudaSuccess) return KVP_ERR_CUDA;
    const int32_t* const table = window > 0 ? p.table : block_table;
    const int32_t* const shortened = window > 0 ? p.shortened : lengths;
    const size_t left = ws_bytes - size_t(at - static_cast<uint8_t*>(ws));
    return bits8 ? decode8_seen(&ones, donor, scale, q, k_cache, v_cache, k_scale, v_scale, table, shortened, p.seen, o, lse, layer_begin, layer_end, at, left, stream)
                 : decode_seen(&ones, donor, scale, q, k_cache, v_cache, table, shortened, p.seen, o, lse, layer_begin, layer_end, at, left, stream);
  }
  const int shares = shares_at_most(d, std::min(d->L, MANY_CHUNK_GROUPS), T);
  if (ws == nullptr || ws_bytes < chunk_bytes(shares, d->dh)) return KVP_ERR_WORKSPACE;
  static thread_local ChunkParams<MANY_CHUNK_GROUPS> p;
  p.block_table = block_table;
  p.lengths = lengths;
  p.first = first;
  uint8_t* at = static_cast<uint8_t*>(ws);
  p.merges = reinterpret_cast<Merge*>(at);
  p.part_o = reinterpret_cast<float*>(at += merge_bytes(shares));
  p.part_ml = reinterpret_cast<float*>(at += align256(size_t(shares) * 2 * (2 * TILE) * d->dh * 4));
  p.B = d->B;
  p.T = T;
  p.Hq = d->Hq;
  p.Hkv = d->Hkv;
  p.G = d->Hq / d->Hkv;
  p.heads = rows_of_token(p.G);
  p.page_size = d->page_size;
  p.max_pages = d->max_pages;
  p.n_pages = d->n_pages;
  p.window = window;
  p.sinks = sinks;
  p.box = d->page_size % 64 == 0 ? 64 : d->page_size % 32 == 0 ? 32 : 16;
  p.io_f32 = d->dtype == KVP_F32;
  p.scale = (scale == 0.f ? 1.f / sqrtf(float(d->dh)) : scale) * 1.4426950408889634f;
  int two_to;
  p.scale_rest = 2.f * frexpf(p.scale, &two_to);
  p.scale_power = ldexpf(1.f, two_to - 1);
  // Layers that share a donor, as many as fit a tile's rows for a token.  Those with most layers first.
  const int per = std::min(CHUNK_MEMBERS, TILE / p.G);
  p.n_groups = p.n_kinds = 0;
  int own = 0, l = layer_begin;
  for (;;) {
    // the next group
    ChunkGroup& grp = p.grp[p.n_groups];
    int n = 0;
    for (; own < d->L && n == 0; n == 0 ? (++own, l = layer_begin) : 0) {
      if (donor[own] != own) continue;
      for (; l < layer_end && n < per; ++l) {
        if (donor[l] != own) continue;
        grp.q[n] = q[l];
        grp.o[n] = o[l];
        grp.lse[n] = lse[l];
        ++n;
      }
      if (n > 0) break;
    }
    if (n > 0) {
      for (int i = n; i < CHUNK_MEMBERS; ++i) {
        grp.q[i] = grp.q[0];
        grp.o[i] = grp.o[0];
        grp.lse[i] = grp.lse[0];
      }
      grp.v_pool = v_cache[own];
      grp.k_scale = bits8 ? k_scale[own] : nullptr;
      grp.v_scale = bits8 ? v_scale[own] : nullptr;
      const uint64_t dims[2] = {uint64_t(d->dh), uint64_t(d->n_pages) * d->Hkv * d->page_size};
      const uint64_t strides[1] = {uint64_t(d->dh) * (bits8 ? 1 : 2)};
      const uint32_t box[2] = {bits8 ? uint32_t(d->dh) : 64u, uint32_t(p.box)};
      rc = make_tensor_map(&grp.map_k, k_cache[own], bits8 ? 1 : 2, 2, dims, strides, box, bits8 && d->dh == 64 ? SWIZZLE_64 : SWIZZLE_128);
      if (rc == KVP_OK) rc = make_tensor_map(&grp.map_v, v_cache[own], bits8 ? 1 : 2, 2, dims, strides, box, bits8 ? SWIZZLE_0 : SWIZZLE_128);
      if (rc != KVP_OK) return rc;
      const int g = p.n_groups++;
      int kind = 0;
      while (kind < p.n_kinds && p.rows[kind].n != n * p.G) ++kind;
      if (kind == p.n_kinds) p.rows[p.n_kinds++] = rows_of_token(n * p.G);
      p.kind[g] = kind;
    }
    if (p.n_groups == MANY_CHUNK_GROUPS || (n == 0 && p.n_groups > 0)) {
      for (int g = p.n_groups; g < MANY_CHUNK_GROUPS; ++g) p.grp[g] = p.grp[0];   // no descriptor is left unset
      timing_before(KVP_KERNEL_DECODE, stream);
      const cudaError_t e = p.n_groups <= FEW_CHUNK_GROUPS ? launch_chunk<FEW_CHUNK_GROUPS>(p, d->dh, bits8, shares, stream)
                                                           : launch_chunk<MANY_CHUNK_GROUPS>(p, d->dh, bits8, shares, stream);
      timing_after(KVP_KERNEL_DECODE, stream);
      if (e != cudaSuccess) return KVP_ERR_CUDA;
      p.n_groups = p.n_kinds = 0;
    }
    if (n == 0) return KVP_OK;
  }
}
