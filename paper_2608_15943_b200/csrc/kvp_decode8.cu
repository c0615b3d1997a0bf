// Split-KV decode attention over the shared paged cache held in 8 bits (kvp_cache8.h): half the bytes of the bf16 cache, and the
// same list of K/V rows dealt out to blocks (kvp_decode.cu describes it), the same groups of layers, the same merge.
//
// With half the bytes a warp's step of 32 tokens of one KV head (8 KB at dh 128) has to pass an SM in about 340 cycles to keep HBM
// busy, so the design is about instructions a step and bytes in flight:
//  - K and V are the A operand of mma.sync m16n8k16 (f16 in, fp32 accumulate) and the query rows its N: up to 8 rows cost half the
//    products that they cost as its M, and the scores of a granule are 4 registers a lane.  S^T = K Q^T, O^T += V^T P^T.
//  - e4m3 numbers become f16 exactly, two an instruction.  (mma.sync takes e4m3 as it is, but converts it itself: half
//    as many instructions again, 32 sequences of 16K-32K tokens in six groups 1930 us instead of 1420.)  Which element of a row is which k of a product is free as long as both operands agree, so a lane reads K 16 bytes
//    at a time and its words are its operands; V comes transposed from ldmatrix .b8, four tokens of an element a word, and the
//    rows of S^T are matched to those tokens.
//  - Queries are scaled by a power of two a row into f16's range (the largest to 2^14): exact for all bf16 elements down to 2^-31 of
//    the row's largest, and rounded by at most 2^-39 of it below.  The scale of K joins the factor of the scores.
//  - The scale of V is a power of two: P is multiplied by 2^(e - D) with a reference M + D of the accumulators beside the
//    reference M of the sum (D is of the powers' size, whatever M is).  Both rise only when a value would leave f16's upper range, so that no maximum is exchanged between
//    lanes in nearly all steps: a vote says whether any lane's scores do.  P in f16 has 11 bits, against bf16's 8.
//  - A warp has a ring of tiles, K's and V's apart, each filled again as soon as it has been read: 12 KB in flight of 16.
//  - A length of 0 (an empty place of a padded batch) is one granule without a visible token: output 0, LSE -infinity.
// Measured (us, by the board; in brackets the bytes at the copy rate): 32 sequences of 16K-32K in six groups 1390 to 1500 (1477), 4 of 128K at
// 32 KV heads 583 to 633 (636): memory.  8 of 8K-16K in two groups 68 to 78 (62), of which 75 of 77 are left without the softmax: SMs that end up to 5 us
// apart, 4 of merge and 5 from the merge to the next call's first tiles.  58 of 1 to 700 at dh 64 14 to 16 (6.5): the steps of
// a warp, nearly 1 us each.  16 rows: 32 of 8K-16K in four groups 605 (497), where the same bytes at 8 rows take 483; heads of 64, 16 of 8K-16K in
// two groups 106 at 8 rows, 127 at 16 (63): a step's latencies one behind the other, two or three warps a scheduler.
#include <float.h>

#include <type_traits>

#include "kvp_cache8.cuh"
#include "kvp_decode_list.cuh"

namespace kvp {
namespace {

constexpr int D8_WARPS = 4, D8_THREADS = D8_WARPS * 32;
constexpr int STEP = 2 * GRAN;                    // tokens of a step of a warp: two granules, each with scales of its own
// CTAs per SM, and tiles (32 tokens of K or of V) of a warp in the ring.  (dh 128, two CTAs and six tiles: 32 sequences of 16K-32K in
// six groups 1424 us instead of 1403; dh 64, six tiles: 256 of 100-300 tokens 45.5 instead of 43.9.)
template <int DH, int NB>
constexpr int D8_CTAS = DH == 128 ? (NB == 1 ? 3 : 2) : NB == 1 ? 4 : 3;
template <int DH, int NB>
constexpr int D8_SLOTS = DH == 128 && NB == 2 ? 6 : 4;
constexpr float P_TOP = 14.f, P_NEW = 8.f;        // log2 of the largest weight of V in f16; of the one that raises the reference
// Where whole units are dealt out, four warps take one if there are fewer than blocks that fit.  From there to as many as warps that fit the
// length decides: with a limit on the steps of a warp, the smallest (in parts of the longest unit's) that fits the device, a unit gets
// one, two or four warps.  Above, or with batches larger than LENGTH_WORDS warps look at together, two warps a unit up to
// LONE_UNITS units a block, then one (nothing is merged).
// (us, by the number of units alone -> so: 58 sequences of 1 to 700 tokens, 4 KV heads at dh 64, four groups 17.0 -> 13.7; 80 of 1 to 900, 2
// KV heads 18.6 -> 14.2; at dh 128 25 of 1 to 1000, 8 KV heads, three groups 29.3 -> 23.0; 30 of 600 to 700, 4 KV heads, four groups 21.7 ->
// 20.8; at dh 64 70 of 100 to 200, nearly as many units as warps, 14.3 -> 14.5.  Four -> one: 128 of 50 to 400, 8 KV heads, six groups 116 -> 71.)
constexpr int LONE_UNITS = 2, LENGTH_WORDS = 4, LENGTH_PARTS = 16;
static_assert(D8_WARPS == 4, "teams of 4, 2 and 1 warps");
constexpr float SUM_TOP = 16.f;                   // log2 of the largest term of the sum
// Beyond this |M| a score is rounded before M comes off it, as the one that became M was: equal scores are then equal terms, and the largest is
// 2^0.  (A fused product would be off from M by up to 2^-24 |M|, which has to stay far below the reserve of f16's range; below it is the more exact.)
constexpr float FAR = 65536.f;
// From this power of V (and of how far M lags the largest score) on the results of a unit or a piece are held against a higher M: the sum
// of up to 2^SUM_TOP a term times V would leave fp32 where V is 2^112 and more.  With sums below 2^-16 it stays below the largest of V,
// 2^16 pieces merged.  (Below it 2^64 times the accumulators, at most 2^23 a token, are far from the end.)
constexpr float LARGE_V = 64.f;

// Shares of the list at dh 128.  Rounds: how often the blocks that fit could have shares of long_share places.  Below LARGE_FROM, as many
// shares a block, all alike.  From there on a block gets a large one first, and then come small ones that even out when the blocks end:
// one an eighth of a block's part, or, in long lists, two a sixteenth of it.  Few blocks are started that way, and a table far
// wider than the lengths leaves few without work.
// (us, up to sixteen shares a block, all alike -> so: 64 of 2000 to 20000, 8 KV heads, one group 235 -> 232; the same in five alike 245; 16 rows, 64 of
// 8000 to 16000 344 in one large and four small -> 321.  One eighth -> two sixteenths, medians of five runs in turn: 32 of 16K-32K in six groups 1472 ->
// 1455, 64 of 8K-24K in four 1220 -> 1204, 48 of 4K-32K in twelve 3204 -> 3156; 16 rows, 64 of 8K-32K in four 2094 -> 2111.
// In a table for 32000 tokens: 16 of 2000 to 5000 in two groups 48.1 -> 43.7, 34 of 50 to 60 in six 28.2 -> 18 to 21.)
constexpr int LARGE_FROM = 3, LONG_FROM = 12;
struct LargeFirst {
  Dealt head;                                      // shares ahead of the small ones, or all
  long long in_head;                               // places there
  uint32_t n_head, small;
  static __device__ __forceinline__ int rounds(const DecSizes& p, long long total) {
    return int(max(1LL, min((long long)LONG_FROM, div_places(total, (long long)p.fit * long_share(128)))));
  }
  static __device__ __forceinline__ int small_ones(int rounds) { return rounds < LARGE_FROM ? 0 : rounds < LONG_FROM ? 1 : 2; }
  static __device__ __forceinline__ int shares(const DecSizes& p, long long total) {
    long long n = total / MIN_SHARE;
    if (n > p.fit) {
      const int r = rounds(p, total);
      n = (long long)p.fit * (r < LARGE_FROM ? r : 1 + small_ones(r));
    }
    return int(max(1LL, min(n, (long long)p.max_shares)));
  }
  __device__ __forceinline__ LargeFirst(const DecSizes& p, long long total, int n) : head(total, n), in_head(total), n_head(n), small(0) {
    if (n <= p.fit) return;
    const int s = small_ones(rounds(p, total));
    if (s == 0) return;
    small = uint32_t(div_places(total, 8LL * s * p.fit));
    n_head = p.fit;
    in_head = total - (long long)s * p.fit * small;
    head = Dealt(in_head, n_head);
  }
  __device__ __forceinline__ long long begin(uint32_t i) const { return i < n_head ? head.begin(i) : in_head + (long long)(i - n_head) * small; }
  __device__ __forceinline__ uint32_t size(uint32_t i) const { return i < n_head ? head.size(i) : small; }
  __device__ __forceinline__ int share_of(long long g) const { return g < in_head ? head.share_of(g) : int(n_head + div_places(g - in_head, small)); }
};
template <int DH>
using Deal8 = std::conditional_t<DH == 128, LargeFirst, EvenDeal<DH>>;
constexpr int most_rounds(int dh) { return dh == 128 ? 3 : max_rounds(dh); }

struct Dec8Group {
  const uint8_t *k_cache, *v_cache;               // [n_pages][Hkv][page_size][dh] e4m3
  const uint8_t *k_scale, *v_scale;               // [n_pages][Hkv][page_size / 16]
  const void* q[MAX_MEMBERS];
  void* o[MAX_MEMBERS];
  float* lse[MAX_MEMBERS];
  int n_members;
  int pad;
};
template <int NG>
struct Dec8Params : DecSizes {
  Dec8Group grp[NG];
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two matrices of 16 rows of 16 bytes (row addresses in lanes 0 to 15 and 16 to 31), transposed: register 2m + i of lane (g, t) holds
// columns g + 8i of rows 4t .. 4t + 3 of matrix m.
__device__ __forceinline__ void ldsm_b8_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// 16-byte asynchronous copy
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// Ring stage: 32 rows of DH bytes of K, then of V.  16-byte chunks are permuted inside lines of 128 bytes so that reads are free of
// bank conflicts: K's lanes of a phase want four chunks of rows 4i and 4i + 1, V's eight rows of ldmatrix the same chunk of each.
template <int DH>
__device__ __forceinline__ uint32_t k_off(int row, int chunk) {
  if (DH == 128) return uint32_t(row) * 128 + (uint32_t(chunk ^ ((row & 1) << 2)) << 4);
  return uint32_t(row) * 64 + (uint32_t(chunk) << 4);
}
template <int DH>
__device__ __forceinline__ uint32_t v_off(int row, int chunk) {
  if (DH == 128) return uint32_t(row) * 128 + (uint32_t(chunk ^ (row & 7)) << 4);
  return uint32_t(row >> 1) * 128 + (uint32_t((row & 1) << 2 | (chunk ^ (row >> 1 & 3))) << 4);
}

// WINDOW: some positions of a sequence are not seen (p.seen), and a number outside the pool stands for a page of zeros.
template <int DH, int NB, int NG, bool WINDOW>
__global__ void __launch_bounds__(D8_THREADS, D8_CTAS<DH, NB>) decode8_kernel(const __grid_constant__ Dec8Params<NG> p) {
  constexpr int GRAN_BYTES = GRAN * DH, TILE_BYTES = 2 * GRAN_BYTES, SLOTS = D8_SLOTS<DH, NB>, DEPTH = SLOTS / 2;
  constexpr int CHUNKS = DH / 16;                  // 16-byte chunks of a row
  constexpr int CP_PER_LANE = GRAN_BYTES / 16 / 32;
  constexpr int HALVES = DH / 64;                  // 16-byte words of a K row that a lane takes
  constexpr int KSTEPS = DH / 16;
  constexpr int MB = DH / 16;                      // m-blocks of O^T

  extern __shared__ __align__(128) uint8_t dsmem[];
  __shared__ float2 s_o[D8_WARPS - 1][MB * 32];    // four rows of the results that a team's first warp merges into its own
  __shared__ float2 s_ml[D8_WARPS - 1][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int G = p.Hq / p.Hkv;

  // ---- the block's place in the list ----
  struct Cursor {
    int grp, b, hk, gran, ng, seen;                // seen: tokens of the sequence (0: none, in one granule)
    int id;                                        // the unit's number, where units are dealt out
    int2 hole;                                     // (WINDOW) tokens that are not seen
    __device__ __forceinline__ bool meets(int token, int n) const { return WINDOW && token < hole.y && token + n > hole.x; }
    __device__ __forceinline__ bool skips(int token) const { return WINDOW && token >= hole.x && token < hole.y; }
  };
  Cursor c;
  int todo;                                        // places of the block's share of the list still to do
  const bool caller_splits = p.num_splits > 0;
  const int cap = p.max_pages * p.page_size;
  auto set_length = [&](Cursor& x, int len) {
    x.seen = min(max(len, 0), cap);
    x.ng = granules_of(max(x.seen, 1));
  };
  auto look = [&](Cursor& x) {
    if (WINDOW) {
      const int4 of = p.seen[x.b];
      x.hole = make_int2(of.x, of.y);
    }
  };
  auto set_unit = [&](Cursor& x, int id) {
    x.id = id;
    x.hk = id % p.Hkv;
    x.b = id / p.Hkv % p.B;
    x.grp = id / p.Hkv / p.B;
    x.gran = 0;
  };
  auto go_to_unit = [&](Cursor& x, int id) {
    set_unit(x, id);
    set_length(x, p.lengths[x.b]);
  };
  bool by_units = p.by_units != 0;
  const int units = p.n_groups * p.B * p.Hkv;
  int rest = 0;                                    // places behind the granules of a unit
  // teams of 4, 2 or 1 warps take the steps of a unit or a piece in turn
  const int plain_team = units < p.fit ? 2 : units < LONE_UNITS * p.fit ? 1 : 0;
  int log_team = caller_splits ? 2 : plain_team;
  const bool by_length = units >= p.fit && units < D8_WARPS * p.fit && p.B <= 32 * LENGTH_WORDS;
  const bool read_all = p.by_units != 0 && by_length;                // lengths of the whole batch, not of its first 32 sequences
  const bool read_one = p.by_units != 0 && !by_length && p.B > 32;
  int len[LENGTH_WORDS] = {};                      // of sequence 32 i + lane
  auto find_unit = [&]() -> bool {
    if (by_length && blockIdx.x >= p.fit) return false;   // (no more are needed)
    if (by_length && !read_all) {
#pragma unroll
      for (int i = 1; i < LENGTH_WORDS; ++i) len[i] = 32 * i + lane < p.B ? p.lengths[32 * i + lane] : 0;
    }
    auto begin_unit = [&]() {                      // (lengths may have been read early: none may come through L1 before the wait)
      int mine = 0;
      if (by_length || p.B <= 32) {
#pragma unroll
        for (int i = 0; i < LENGTH_WORDS; ++i) {
          const int v = __shfl_sync(0xffffffffu, len[i], c.b & 31);
          if (c.b >> 5 == i) mine = v;
        }
      } else {
        mine = p.lengths[c.b];
      }
      set_length(c, mine);
      todo = c.ng;
      return true;
    };
    if (by_length) {
      int steps[LENGTH_WORDS], longest = 0;        // of sequence 32 i + lane
#pragma unroll
      for (int i = 0; i < LENGTH_WORDS; ++i) {
        const int b = 32 * i + lane;
        steps[i] = b < p.B ? (granules_of(clamp_length(p, len[i])) + 1) / 2 : 0;
        longest = max(longest, steps[i]);
      }
      longest = __reduce_max_sync(0xffffffffu, longest);
      const int per_seq = p.Hkv * p.n_groups;
      int most = 0, of4 = 0, of2 = 0, of1 = 0;     // steps of a warp, units of each kind of team
      auto fits = [&](int parts) -> bool {
        most = (longest * parts + LENGTH_PARTS - 1) / LENGTH_PARTS;
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < LENGTH_WORDS; ++i) n += (steps[i] > 2 * most ? 1u << 16 : 0u) + (steps[i] > most ? 1u : 0u);
        n = __reduce_add_sync(0xffffffffu, n);
        of1 = (p.B - int(n & 0xffffu)) * per_seq;
        of2 = int((n & 0xffffu) - (n >> 16)) * per_seq;
        of4 = int(n >> 16) * per_seq;
        return of4 + (of2 + 1) / 2 + (of1 + 3) / 4 <= p.fit;
      };
      int parts = LENGTH_PARTS >> (plain_team + 1);
      while (!fits(parts)) ++parts;                // (ends: twice as many parts are the plain teams, which fit)
      int u = blockIdx.x, n = of4;                 // the team's unit among those of its kind, the longest first
      int above = 2 * most, upto = longest;
      log_team = 2;
      if (u >= of4) {
        u = (u - of4) * 2;
        n = of2;
        above = most;
        upto = 2 * most;
        log_team = 1;
        if (u >= of2) {
          u = (u - (of2 + 1) / 2 * 2) * 2;
          n = of1;
          above = 0;
          upto = most;
          log_team = 0;
        }
      }
      u += warp >> log_team;
      if (u >= n) return false;
      int nth = u / per_seq;
      const int r = u - nth * per_seq;
#pragma unroll
      for (int i = 0; i < LENGTH_WORDS; ++i) {
        const bool is_one = steps[i] > above && steps[i] <= upto;
        const uint32_t kind = __ballot_sync(0xffffffffu, is_one);
        const uint32_t hit = __ballot_sync(0xffffffffu, is_one && __popc(kind & ((1u << lane) - 1)) == nth);
        if (hit != 0u) c.b = 32 * i + __ffs(hit) - 1;
        nth -= __popc(kind);
      }
      c.id = units;                                // no other unit comes behind it
      c.hk = r % p.Hkv;
      c.grp = r / p.Hkv;
      c.gran = 0;
      return begin_unit();
    }
    log_team = plain_team;
    const int id = (int(blockIdx.x) * D8_WARPS + warp) >> log_team;
    if (id >= units) return false;
    set_unit(c, id);
    return begin_unit();
  };
  auto find_place = [&]() -> bool {                // from the lengths; false: the block (or the team) has none
    const int len0 = len[0];
    int all = 0;
    long long granules = 0;
    if (!p.by_units) {
      int before, longest;
      sum_granules(p, len0, 0, before, all, longest);
      granules = (long long)all * p.Hkv * p.n_groups;
      by_units = dealt_by_units(DH, granules, units, longest, p.fit);
      rest = by_units ? 0 : unit_rest(DH, granules, p.fit);
    }
    if (by_units) return find_unit();
    log_team = 2;
    const long long per_group = ((long long)all + (long long)p.B * rest) * p.Hkv, total = per_group * p.n_groups;
    const int n_shares = Deal8<DH>::shares(p, total);
    if (blockIdx.x >= n_shares) return false;
    const Deal8<DH> dealt(p, total, n_shares);
    long long at = dealt.begin(blockIdx.x);
    todo = int(dealt.size(blockIdx.x));
    c.id = 0;
    c.grp = int(div_places(at, per_group));
    at -= c.grp * per_group;                       // inside the group: find the sequence, 32 lengths at a time
    for (int b0 = 0;; b0 += 32) {
      const bool is_one = b0 + lane < p.B;
      const int len = !is_one ? 0 : b0 == 0 ? len0 : p.lengths[b0 + lane];
      const int mine = is_one ? granules_of(clamp_length(p, len)) + rest : 0;
      int upto = mine;
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, s);
        if (lane >= s) upto += v;
      }
      const uint32_t hit = __ballot_sync(0xffffffffu, at < (long long)upto * p.Hkv);
      if (hit != 0u) {
        const int src = __ffs(hit) - 1;
        at -= (long long)__shfl_sync(0xffffffffu, upto - mine, src) * p.Hkv;
        c.b = b0 + src;
        set_length(c, __shfl_sync(0xffffffffu, len, src));
        break;
      }
      at -= (long long)__shfl_sync(0xffffffffu, upto, 31) * p.Hkv;
    }
    c.hk = int(at) / (c.ng + rest);                // (a sequence's places of all KV heads fit 32 bits)
    c.gran = int(at) % (c.ng + rest);
    return true;
  };
  bool placed = true;
  if (caller_splits || read_one) {
    grid_dep_wait();
  } else {
    const bool early = (p.B <= 32 || read_all) && blockIdx.x < p.fit;   // (what starts later than that starts behind the wait)
    for (bool behind = !early;; behind = true) {
      if (behind) grid_dep_wait();
      bool same = true;
#pragma unroll
      for (int i = 0; i < LENGTH_WORDS; ++i) {
        const int b = 32 * i + lane, now = b < p.B && (i == 0 || read_all) ? __ldcg(p.lengths + b) : 0;
        same = same && now == len[i];
        len[i] = now;
      }
      if (behind && early && __all_sync(0xffffffffu, same)) break;
      placed = find_place();
      if (behind) break;
    }
  }
  if (!placed) return;
  const int team = 1 << log_team, first_step = warp & (team - 1);
  if (caller_splits) {
    const int split = blockIdx.x % p.num_splits;
    go_to_unit(c, blockIdx.x / p.num_splits);
    const int per = (c.ng + p.num_splits - 1) / p.num_splits;
    c.gran = min(c.ng, split * per);
    todo = min(c.ng - c.gran, per);
  } else if (read_one) {
    const int id = (int(blockIdx.x) * D8_WARPS + warp) >> log_team;
    if (id >= units) return;
    go_to_unit(c, id);
    todo = c.ng;
  }
  const int unit_step = int(gridDim.x) << (2 - log_team);
  auto next_piece = [&](Cursor& x, int& left) {    // past the end: grp >= n_groups
    left -= min(left, x.ng + rest - x.gran);
    if (left > 0) {
      x.gran = 0;
      if (++x.hk == p.Hkv) {
        x.hk = 0;
        if (++x.b == p.B) {
          x.b = 0;
          ++x.grp;
        }
        set_length(x, p.lengths[x.b]);
        look(x);
      }
    } else if (by_units && !caller_splits && x.id + unit_step < units) {
      go_to_unit(x, x.id + unit_step);
      look(x);
      left = x.ng;
    } else {
      x.grp = p.n_groups;
    }
  };
  look(c);
  if (c.gran >= c.ng && !caller_splits) {          // the share begins behind the granules of a unit
    next_piece(c, todo);
    if (c.grp >= p.n_groups) return;
  }

  // ---- copies: a cursor of their own; K_i, V_i, K_i+1, ... of this warp's steps go round a ring of tiles, all but one of them ahead of
  // the arithmetic: V_i+DEPTH-1 is asked for when K_i is there, K_i+DEPTH as soon as K_i has been read ----
  const uint32_t ring = smem_u32(dsmem) + warp * SLOTS * TILE_BYTES;
  Cursor f = c;
  int f_todo = todo;
  int f_left;                                      // steps of the piece from this warp's next one on (<= 0: none)
  const int gran_per_page = p.page_size / GRAN;
  const Dec8Group* f_grp = &p.grp[0];
  const int32_t* bt = nullptr;                     // block-table entry of the page the next step begins in,
  int in_page = 0, f_live = 0;                     // its granule there; tokens of the piece from there on
  int f_at = 0;                                    // (WINDOW) its first token
  int page = 0;                                    // that entry, looked at when its step is asked for: a load ahead of it
  int slot_in = 0, slot_out = 0;                   // in pairs: K's tile and V's behind it
  auto is_page = [&](int page) { return !WINDOW || unsigned(page) < unsigned(p.n_pages); };
  auto block_of = [&](int page) { return (size_t(min(max(page, 0), p.n_pages - 1)) * p.Hkv + f.hk) * gran_per_page; };
  auto enter_piece = [&]() {
    const int n = min(f_todo, f.ng - f.gran);
    f_left = (n + 1) / 2 - first_step;
    if (f_left <= 0) return;
    const int gran = f.gran + 2 * first_step, col = gran / gran_per_page;
    f_grp = &p.grp[f.grp];
    bt = p.block_table + size_t(f.b) * p.max_pages + col;
    in_page = gran - col * gran_per_page;
    f_live = min(f.seen, (f.gran + n) * GRAN) - gran * GRAN;
    f_at = gran * GRAN;
    page = *bt;
  };
  // Scales of the steps in the ring: a lane has the byte of one granule (lane & 3: K's and V's of the first, of the second).
  // (Moved up a step behind the load, or the move would wait for it.)
  uint32_t scales[DEPTH];
#pragma unroll
  for (int s = 0; s < DEPTH; ++s) scales[s] = 0;
  // V's granules of the step whose K was asked for last, and how many tokens of it are to be read (-1: no step)
  const uint8_t *v_src0 = nullptr, *v_src1 = nullptr;
  int v_live = -1;
  int v_at = 0;                                    // (WINDOW) its first token, and the tokens that are not seen
  int2 v_hole = make_int2(0, 0);
  bool v_there0 = true, v_there1 = true;           // (WINDOW) the granules' pages are of the pool
  // the tile of a step: 32 rows in a run from src0, or (split) 16 from either
  auto copy_tile = [&](uint32_t dst, const uint8_t* src0, const uint8_t* src1, int live, bool split, bool is_v, int at, int2 hole, bool there0, bool there1) {
    if (!split) {
#pragma unroll
      for (int i = 0; i < 2 * CP_PER_LANE; ++i) {
        const int idx = i * 32 + lane, row = idx / CHUNKS, chunk = idx % CHUNKS;
        cp_async16(dst + (is_v ? v_off<DH>(row, chunk) : k_off<DH>(row, chunk)), src0 + i * 512);
      }
    } else {                                       // slots never appended may hold anything: zeros instead
#pragma unroll
      for (int i = 0; i < 2 * CP_PER_LANE; ++i) {
        const int idx = i * 32 + lane, row = idx / CHUNKS, chunk = idx % CHUNKS;
        cp_async16(dst + (is_v ? v_off<DH>(row, chunk) : k_off<DH>(row, chunk)), (i < CP_PER_LANE ? src0 : src1) + i % CP_PER_LANE * 512,
                   row < live && (i < CP_PER_LANE ? there0 : there1) && !(WINDOW && at + row >= hole.x && at + row < hole.y) ? 16u : 0u);
      }
    }
  };
  bool v_split = false;
  auto issue_k = [&](uint32_t& scale) {
    while (f_left <= 0 && f.grp < p.n_groups) {
      next_piece(f, f_todo);
      if (f.grp < p.n_groups) enter_piece();
    }
    v_live = -1;
    if (f_left > 0) {
      const size_t block0 = block_of(page) + in_page;
      const bool in_a_row = in_page + 1 < gran_per_page;
      size_t block1 = block0 + 1;
      v_there0 = v_there1 = is_page(page);
      if (!in_a_row || f_live <= GRAN) {
        const int page1 = f_live > GRAN ? bt[1] : page;
        block1 = f_live > GRAN ? block_of(page1) : block0;
        v_there1 = is_page(page1);
      }
      scale = 0;                                   // (no page: the smallest powers, so that a zero of V raises no reference)
      if (lane & 2 ? v_there1 : v_there0) scale = (lane & 1 ? f_grp->v_scale : f_grp->k_scale)[lane & 2 ? block1 : block0];
      const size_t at0 = block0 * GRAN_BYTES + lane * 16, at1 = block1 * GRAN_BYTES + lane * 16;
      v_split = !in_a_row || f_live < STEP || !v_there0 || f.meets(f_at, STEP);
      copy_tile(ring + slot_in * 2 * TILE_BYTES, f_grp->k_cache + at0, f_grp->k_cache + at1, f_live, v_split, false, f_at, f.hole, v_there0, v_there1);
      v_src0 = f_grp->v_cache + at0;
      v_src1 = f_grp->v_cache + at1;
      v_live = max(f_live, 0);
      v_at = f_at;
      v_hole = f.hole;
      f_left -= team;
      f_live -= team * STEP;
      f_at += team * STEP;
      in_page += team * 2;
      if (in_page >= gran_per_page && f_left > 0) {
        do {
          in_page -= gran_per_page;
          ++bt;
        } while (in_page >= gran_per_page);
        page = *bt;
      }
    }
    cp_async_commit();
  };
  auto issue_v = [&]() {
    if (v_live >= 0) {
      copy_tile(ring + (slot_in * 2 + 1) * TILE_BYTES, v_src0, v_src1, v_live, v_split, true, v_at, v_hole, v_there0, v_there1);
      if (++slot_in == DEPTH) slot_in = 0;
    }
    cp_async_commit();
  };
  enter_piece();

  // ---- queries: B operand, row n of the group in lanes g = n mod 8 ----
  uint32_t qb[KSTEPS][NB][2];
  float q_factor[NB][2];                           // of the scores of rows 8 nb + 2 t + h
  auto load_queries = [&]() {
    const Dec8Group& grp = p.grp[c.grp];
    const int R = grp.n_members * G;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int n = nb * 8 + g;
      float v[HALVES * 16];
      if (n < R) {
        const size_t at = (size_t(c.b) * p.Hq + c.hk * G + n % G) * DH;
        const void* const q = grp.q[n / G];
#pragma unroll
        for (int e = 0; e < HALVES * 4; ++e) {
          const size_t four = at + (e >> 2) * 64 + t * 16 + (e & 3) * 4;
          uint2 w;
          if (p.io_f32) {
            const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(q) + four);
            w = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
          } else {
            w = *reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(q) + four);
          }
          v[4 * e] = __uint_as_float(w.x << 16);
          v[4 * e + 1] = __uint_as_float(w.x & 0xffff0000u);
          v[4 * e + 2] = __uint_as_float(w.y << 16);
          v[4 * e + 3] = __uint_as_float(w.y & 0xffff0000u);
        }
      } else {
#pragma unroll
        for (int e = 0; e < HALVES * 16; ++e) v[e] = 0.f;
      }
      float amax = 0.f;
#pragma unroll
      for (int e = 0; e < HALVES * 16; ++e) amax = fmaxf(amax, fabsf(v[e]));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      const int lg = max(int(__float_as_uint(amax) >> 23) - 127, -100);      // (128: infinite, left so)
      const float up = __uint_as_float(power_bits(lg < 128 ? 14 - lg : 0));
      const float down = __uint_as_float(power_bits(lg < 128 ? lg - 14 : 0)) * p.scale_log2;
#pragma unroll
      for (int e = 0; e < KSTEPS; ++e) {
        qb[e][nb][0] = pack_f16(v[4 * e] * up, v[4 * e + 1] * up);
        qb[e][nb][1] = pack_f16(v[4 * e + 2] * up, v[4 * e + 3] * up);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) q_factor[nb][h] = __shfl_sync(0xffffffffu, down, (2 * t + h) * 4);
    }
  };

#pragma unroll
  for (int s = 0; s < DEPTH; ++s) {
    issue_k(scales[s]);
    if (s + 1 < DEPTH) issue_v();
  }
  load_queries();

  const int tok_g = (g >> 1) * 4 + (g & 1);        // token of a granule that row g of its S^T is; row g + 8: two more
  do {
    // ---- one unit, or this block's piece of it ----
    const Dec8Group& grp = p.grp[c.grp];
    const int R = grp.n_members * G;
    const int n_here = min(todo, c.ng - c.gran);
    const bool from_start = c.gran == 0, to_end = c.gran + n_here == c.ng;

    float oacc[MB][NB][4];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) oacc[m][nb][0] = oacc[m][nb][1] = oacc[m][nb][2] = oacc[m][nb][3] = 0.f;
    // of rows 8 nb + 2 t and the next, side by side: sums of this lane's terms; -M, M the reference of the sum; -D, M + D that of oacc
    // (exponents as bytes)
    uint64_t sum2[NB], minus_M[NB], minus_D[NB];
    bool far = false;                              // some |M| is beyond FAR
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      sum2[nb] = 0;
      minus_M[nb] = minus_D[nb] = pack_f2(FLT_MAX, FLT_MAX);   // (no finite score is below M, and no infinity comes off an infinity)
    }

    const int tokens = min(c.seen, (c.gran + n_here) * GRAN) - c.gran * GRAN;   // that the piece sees (0: none)
    for (int i = first_step; 2 * i < n_here; i += team) {
      cp_async_wait<SLOTS - 2>();
      __syncwarp();
      issue_v();                                   // into the place of the previous step's
      const uint32_t sK = ring + slot_out * 2 * TILE_BYTES, sV = sK + TILE_BYTES;
      if (++slot_out == DEPTH) slot_out = 0;

      // ---- S^T[32 tokens, rows] = K Q^T, even and odd k-steps apart ----
      float s2[2][NB][2][4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int u = 0; u < 4; ++u) s2[m][nb][0][u] = s2[m][nb][1][u] = 0.f;
#pragma unroll
        for (int hf = 0; hf < HALVES; ++hf) {
          const uint4 ka = lds16(sK + k_off<DH>(m * GRAN + tok_g, hf * 4 + t)), kb = lds16(sK + k_off<DH>(m * GRAN + tok_g + 2, hf * 4 + t));
          const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t a[4] = {e4m3x2_to_f16x2(uint16_t(wa[w])), e4m3x2_to_f16x2(uint16_t(wb[w])), e4m3x2_to_f16x2(uint16_t(wa[w] >> 16)),
                                   e4m3x2_to_f16x2(uint16_t(wb[w] >> 16))};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma_f16(s2[m][nb][w & 1], a, qb[hf * 4 + w][nb][0], qb[hf * 4 + w][nb][1]);
          }
        }
      }
      __syncwarp();                                // every lane has read K
      const uint32_t scale = scale_byte(scales[0]);
#pragma unroll
      for (int s = 0; s + 1 < DEPTH; ++s) scales[s] = scales[s + 1];
      issue_k(scales[DEPTH - 1]);
      // ---- softmax: terms of the sum 2^(x - M), weights of V 2^(x - M) 2^(e - D) ----
      const int left = tokens - i * STEP;          // visible tokens from this step on
      const int at = c.gran * GRAN + i * STEP;     // its first
      const bool partly = c.meets(at, STEP);
      uint64_t factor[2][NB], x[2][NB][2];         // x - M
      float v_exp[2];
      uint64_t to_v[2][NB];                        // e - D
      bool over = false;
      auto scores = [&]() {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int u = 0; u < 2; ++u) x[m][nb][u] = ffma2(pack_f2(s2[m][nb][0][2 * u], s2[m][nb][0][2 * u + 1]), factor[m][nb], minus_M[nb]);
            to_v[m][nb] = fadd2(pack_f2(v_exp[m], v_exp[m]), minus_D[nb]);
          }
        if (__builtin_expect(far, 0)) {            // (in single operations: the assembler fuses a packed product and sum)
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int u = 0; u < 2; ++u)
                x[m][nb][u] = pack_f2(__fadd_rn(__fmul_rn(s2[m][nb][0][2 * u], f2_lo(factor[m][nb])), f2_lo(minus_M[nb])),
                                      __fadd_rn(__fmul_rn(s2[m][nb][0][2 * u + 1], f2_hi(factor[m][nb])), f2_hi(minus_M[nb])));
        }
        if (left < STEP || partly) {
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (m * GRAN + tok_g + 2 * u >= left || c.skips(at + m * GRAN + tok_g + 2 * u)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) x[m][nb][u] = pack_f2(-INFINITY, -INFINITY);
              }
        }
      };
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float k_scale = __uint_as_float(__shfl_sync(0xffffffffu, scale, 2 * m) << 23);
        v_exp[m] = __uint_as_float(0x4b000000u | __shfl_sync(0xffffffffu, scale, 2 * m + 1)) - 8388608.f;      // (2^23 + byte - 2^23)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          factor[m][nb] = fmul2(pack_f2(q_factor[nb][0], q_factor[nb][1]), pack_f2(k_scale, k_scale));
#pragma unroll
          for (int u = 0; u < 4; ++u) s2[m][nb][0][u] += s2[m][nb][1][u];
        }
      }
      scores();
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          over = over || fmaxf(f2_lo(x[m][nb][0]), f2_lo(x[m][nb][1])) > fminf(SUM_TOP, P_TOP - f2_lo(to_v[m][nb])) ||
                 fmaxf(f2_hi(x[m][nb][0]), f2_hi(x[m][nb][1])) > fminf(SUM_TOP, P_TOP - f2_hi(to_v[m][nb]));
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float M[2] = {-f2_lo(minus_M[nb]), -f2_hi(minus_M[nb])}, D[2] = {-f2_lo(minus_D[nb]), -f2_hi(minus_D[nb])};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float y[2];                            // largest score of each granule
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              y[m] = -INFINITY;
#pragma unroll
              for (int u = 0; u < 2; ++u)
                if (m * GRAN + tok_g + 2 * u < left && !c.skips(at + m * GRAN + tok_g + 2 * u)) y[m] = fmaxf(y[m], s2[m][nb][0][2 * u + h] * (h ? f2_hi(factor[m][nb]) : f2_lo(factor[m][nb])));
            }
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) {
              y[0] = fmaxf(y[0], __shfl_xor_sync(0xffffffffu, y[0], s));
              y[1] = fmaxf(y[1], __shfl_xor_sync(0xffffffffu, y[1], s));
            }
            const float most = fmaxf(y[0], y[1]);
            if (most > M[h] + SUM_TOP) {
              const float rise = most - M[h], factor_s = fast_exp2(-rise);
              sum2[nb] = h ? pack_f2(f2_lo(sum2[nb]), f2_hi(sum2[nb]) * factor_s) : pack_f2(f2_lo(sum2[nb]) * factor_s, f2_hi(sum2[nb]));
              M[h] = most;
              D[h] -= rise;                      // (M + D as it was)
            }
            const float top = fmaxf(y[0] - M[h] + v_exp[0], y[1] - M[h] + v_exp[1]);
            if (top > D[h] + P_TOP) {
              const float to = top - P_NEW, factor_o = fast_exp2(D[h] - to);
              D[h] = to;
#pragma unroll
              for (int m = 0; m < MB; ++m) {
                oacc[m][nb][h] *= factor_o;
                oacc[m][nb][2 + h] *= factor_o;
              }
            }
          }
          minus_M[nb] = pack_f2(-M[0], -M[1]);
          minus_D[nb] = pack_f2(-D[0], -D[1]);
          far = far || fmaxf(fabsf(M[0]), fabsf(M[1])) > FAR;
        }
        far = __any_sync(0xffffffffu, far);
        scores();
      }
      uint32_t pb[2][NB][2];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const uint64_t f = pack_f2(fast_exp2(fminf(f2_lo(to_v[m][nb]), 126.f)), fast_exp2(fminf(f2_hi(to_v[m][nb]), 126.f)));
          uint64_t pr[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            pr[u] = pack_f2(fast_exp2(f2_lo(x[m][nb][u])), fast_exp2(f2_hi(x[m][nb][u])));
            const uint64_t w = fmul2(pr[u], f);
            pb[m][nb][u] = transpose_8x8(pack_f16(f2_lo(w), f2_hi(w)));
          }
          sum2[nb] = fadd2(sum2[nb], fadd2(pr[0], pr[1]));
        }
      // ---- O^T[DH, rows] += V^T P^T ----
      cp_async_wait<SLOTS - 1>();
      __syncwarp();
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        uint32_t v[4];
        ldsm_b8_t(sV + v_off<DH>(lane, m), v);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t a[4] = {e4m3x2_to_f16x2(uint16_t(v[2 * k])), e4m3x2_to_f16x2(uint16_t(v[2 * k + 1])), e4m3x2_to_f16x2(uint16_t(v[2 * k] >> 16)),
                                 e4m3x2_to_f16x2(uint16_t(v[2 * k + 1] >> 16))};
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_f16(oacc[m][nb], a, pb[k][nb][0], pb[k][nb][1]);
        }
      }
      // (every lane is done with V before it is refilled: the barrier at the top)
    }
    const Cursor here = c;
    next_piece(c, todo);
    const bool last = c.grp >= p.n_groups;
    if (last) grid_dep_launch();   // this warp's loads are out, the others' within a granule
    else load_queries();

    // ---- everything against M; no term at all: M = -infinity ----
    float sum[NB][2], M[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        M[nb][h] = h ? -f2_hi(minus_M[nb]) : -f2_lo(minus_M[nb]);
        sum[nb][h] = h ? f2_hi(sum2[nb]) : f2_lo(sum2[nb]);
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) sum[nb][h] += __shfl_xor_sync(0xffffffffu, sum[nb][h], s);
        float up = -127.f - (h ? f2_hi(minus_D[nb]) : f2_lo(minus_D[nb]));
        if (up > LARGE_V) {                        // M rises until the sum is below 2^-16
          const int raise = int(__float_as_uint(sum[nb][h]) >> 23) - (127 - 17);
          sum[nb][h] *= __uint_as_float(power_bits(-raise));
          M[nb][h] += float(raise);
          up -= float(raise);
        }
        const float to_m = fast_exp2(fminf(up, 126.f));
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          oacc[m][nb][h] *= to_m;
          oacc[m][nb][2 + h] *= to_m;
        }
        if (sum[nb][h] == 0.f) M[nb][h] = -INFINITY;
      }
    // ---- the team's first warp merges the results of the others into its own, four rows at a time ----
    auto team_sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + (warp >> log_team)), "r"(32 << log_team) : "memory"); };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (8 * nb + h >= R || team == 1) break;
        team_sync();       // its first warp is done with the previous ones
        if (first_step > 0) {
#pragma unroll
          for (int m = 0; m < MB; ++m) s_o[warp - 1][m * 32 + lane] = make_float2(oacc[m][nb][h], oacc[m][nb][2 + h]);
          s_ml[warp - 1][lane] = make_float2(M[nb][h], sum[nb][h]);
        }
        team_sync();
        if (first_step == 0) {
          float2 om[D8_WARPS - 1];
          float mn = M[nb][h];
#pragma unroll
          for (int w = 0; w < D8_WARPS - 1; ++w) {
            om[w] = w < team - 1 ? s_ml[warp + w][lane] : make_float2(-INFINITY, 0.f);
            mn = fmaxf(mn, om[w].x);
          }
          const float fa = M[nb][h] == -INFINITY ? 0.f : fast_exp2(M[nb][h] - mn);
          M[nb][h] = mn;
          sum[nb][h] *= fa;
#pragma unroll
          for (int m = 0; m < MB; ++m) {
            oacc[m][nb][h] *= fa;
            oacc[m][nb][2 + h] *= fa;
          }
#pragma unroll
          for (int w = 0; w < D8_WARPS - 1; ++w) {
            if (w >= team - 1) break;
            const float fb = om[w].x == -INFINITY ? 0.f : fast_exp2(om[w].x - mn);
            sum[nb][h] += om[w].y * fb;
#pragma unroll
            for (int m = 0; m < MB; ++m) {
              const float2 v = s_o[warp + w][m * 32 + lane];
              oacc[m][nb][h] += v.x * fb;
              oacc[m][nb][2 + h] += v.y * fb;
            }
          }
        }
      }
    if (first_step != 0) {
      // (the piece's first warp alone goes on to store)
    } else if (WINDOW && !caller_splits && from_start && to_end && p.seen[here.b].z == 0) {
      // (the row of no sequence is left as it is)
    } else if (!caller_splits && from_start && to_end) {
      // ---- the whole unit: normalise and store; a lane has elements 16 m + g and 16 m + g + 8, of which lanes g and g ^ 1 make pairs ----
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (8 * nb + h >= R) break;
          const int row = nb * 8 + 2 * t + h;
          const size_t head = size_t(here.b) * p.Hq + here.hk * G + row % G;
          const bool none = sum[nb][h] == 0.f, odd = (g & 1) != 0;
          const float inv = none ? 0.f : 1.f / sum[nb][h];
          void* const o = row < R ? grp.o[row / G] : nullptr;
#pragma unroll
          for (int m = 0; m < MB; ++m) {
            const float lo = oacc[m][nb][h] * inv, hi = oacc[m][nb][2 + h] * inv;
            const float other = __shfl_xor_sync(0xffffffffu, odd ? lo : hi, 4);
            const uint32_t v = odd ? pack_bf16(other, hi) : pack_bf16(lo, other);   // rounded to bf16 either way: one set of results
            const size_t at = head * DH + m * 16 + (odd ? g + 7 : g);
            if (row < R) {
              if (p.io_f32)
                *reinterpret_cast<float2*>(reinterpret_cast<float*>(o) + at) = make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
              else
                *reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(o) + at) = v;
            }
          }
          if (row < R && g == 0) grp.lse[row / G][head] = none ? -INFINITY : log_sum(M[nb][h], sum[nb][h]);
        }
    } else {
      // ---- a piece: the first of a share, or the last one if that starts a unit ----
      const size_t piece = caller_splits ? size_t(blockIdx.x) : size_t(blockIdx.x) * 2 + (from_start ? 1 : 0);
      float* const po = p.part_o + piece * p.rows * DH;
      float* const pml = p.part_ml + piece * p.rows * 2;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = nb * 8 + 2 * t + h;
          if (row < R) {
#pragma unroll
            for (int m = 0; m < MB; ++m) {
              po[row * DH + m * 16 + g] = oacc[m][nb][h];
              po[row * DH + m * 16 + g + 8] = oacc[m][nb][2 + h];
            }
            if (g == 0) *reinterpret_cast<float2*>(pml + row * 2) = make_float2(M[nb][h], sum[nb][h]);
          }
        }
    }
    if (last) break;
  } while (true);
  cp_async_wait<0>();
}

DealBy deal8_by(int dh, int rows) {
  return {sm_count() * (dh == 128 ? (rows <= 8 ? D8_CTAS<128, 1> : D8_CTAS<128, 2>) : rows <= 8 ? D8_CTAS<64, 1> : D8_CTAS<64, 2>), most_rounds(dh)};
}
// Blocks for whole units.  (One too many costs: it has to be started before the next kernel's.  34 sequences of 50 to 60 tokens in six groups 11.7 us instead of 8.3.)
long long blocks_by_units(long long units, int B, int fit) {
  if (units < fit) return units;
  if (units < (long long)D8_WARPS * fit && B <= 32 * LENGTH_WORDS) return fit;
  return units < (long long)LONE_UNITS * fit ? (units + 1) / 2 : (units + D8_WARPS - 1) / D8_WARPS;
}
// query rows of the largest group of a call
int most_rows(const kvp_decode_desc* d, const SubGroup* subs, int n) {
  int rows = 0;
  for (int i = 0; i < n; ++i) rows = std::max(rows, subs[i].n * (d->Hq / d->Hkv));
  return rows;
}

template <int DH, int NB, int NG, bool WINDOW>
cudaError_t launch_decode8(const Dec8Params<MAX_DEC_GROUPS>& all, dim3 grid, dim3 combine_grid, int wpr, cudaStream_t stream) {
  constexpr int smem = D8_WARPS * D8_SLOTS<DH, NB> * STEP * DH;
  cudaError_t e = allow_smem<decode8_kernel<DH, NB, NG, WINDOW>>(smem);
  if (e != cudaSuccess) return e;
  Dec8Params<NG> p;
  static_cast<DecSizes&>(p) = all;
  std::copy(all.grp, all.grp + all.n_groups, p.grp);
  timing_before(KVP_KERNEL_DECODE, stream);
  e = launch_kernel(decode8_kernel<DH, NB, NG, WINDOW>, grid, D8_THREADS, smem, stream, 1, p);
  timing_after(KVP_KERNEL_DECODE, stream);
  if (e == cudaSuccess && (p.num_splits > 0 || p.by_units == 0))   // whole units leave no pieces
    e = launch_kernel(decode_combine_kernel<DH, true, Dec8Params<NG>, Deal8<DH>>, combine_grid, COMBINE_THREADS, 0, stream, 1, p, wpr);
  return e;
}
template <int DH, int NB, int NG>
cudaError_t launch_decode8(const Dec8Params<MAX_DEC_GROUPS>& p, dim3 grid, dim3 combine_grid, int wpr, cudaStream_t stream) {
  return p.seen != nullptr ? launch_decode8<DH, NB, NG, true>(p, grid, combine_grid, wpr, stream) : launch_decode8<DH, NB, NG, false>(p, grid, combine_grid, wpr, stream);
}
template <int DH, int NB>
cudaError_t launch_decode8(const Dec8Params<MAX_DEC_GROUPS>& p, dim3 grid, dim3 combine_grid, int wpr, cudaStream_t stream) {
  return p.n_groups <= FEW_DEC_GROUPS ? launch_decode8<DH, NB, FEW_DEC_GROUPS>(p, grid, combine_grid, wpr, stream)
                                      : launch_decode8<DH, NB, MAX_DEC_GROUPS>(p, grid, combine_grid, wpr, stream);
}

int check_desc8(const kvp_decode_desc* d) {
  const int rc = check_desc(d);
  if (rc != KVP_OK) return rc;
  return (long long)d->max_pages * d->page_size > 0x7fffffffLL - GRAN ? KVP_ERR_UNSUPPORTED : KVP_OK;
}

}  // namespace
}  // namespace kvp

using namespace kvp;

extern "C" size_t kvp_decode8_workspace_bytes(const kvp_decode_desc* d, const int32_t* donor) {
  if (check_desc8(d) != KVP_OK || donor == nullptr) return 0;
  for (int l = 0; l < d->L; ++l)
    if (donor[l] < 0 || donor[l] > l || donor[donor[l]] != donor[l]) return 0;
  // of any layer range: one that leaves out members of the largest groups may have fewer rows, and more blocks that fit
  return std::max(decode_scratch_bytes(d, donor, 0, d->L, deal8_by(d->dh, 8)), decode_scratch_bytes(d, donor, 0, d->L, deal8_by(d->dh, 16)));
}

extern "C" int kvp_decode8(const kvp_decode_desc* d, const int32_t* donor, float scale, const void* const* q, const void* const* k_cache,
                           const void* const* v_cache, const uint8_t* const* k_scale, const uint8_t* const* v_scale, const int32_t* block_table,
                           const int32_t* lengths, void* const* o, float* const* lse, int layer_begin, int layer_end, void* ws, size_t ws_bytes,
                           kvp_stream_t stream) {
  return decode8_seen(d, donor, scale, q, k_cache, v_cache, k_scale, v_scale, block_table, lengths, nullptr, o, lse, layer_begin, layer_end, ws, ws_bytes,
                      reinterpret_cast<cudaStream_t>(stream));
}

int kvp::decode8_seen(const kvp_decode_desc* d, const int32_t* donor, float scale, const void* const* q, const void* const* k_cache, const void* const* v_cache,
                      const uint8_t* const* k_scale, const uint8_t* const* v_scale, const int32_t* block_table, const int32_t* lengths, const int4* seen,
                      void* const* o, float* const* lse, int layer_begin, int layer_end, void* ws, size_t ws_bytes, cudaStream_t stream) {
  const int rc = check_desc8(d);
  if (rc != KVP_OK) return rc;
  if (donor == nullptr || q == nullptr || k_cache == nullptr || v_cache == nullptr || k_scale == nullptr || v_scale == nullptr ||
      block_table == nullptr || lengths == nullptr || o == nullptr || lse == nullptr || !(scale >= 0.f && scale < INFINITY))
    return KVP_ERR_INVALID_ARG;
  if (layer_begin < 0 || layer_end > d->L || layer_begin >= layer_end) return KVP_ERR_INVALID_ARG;
  for (int l = 0; l < d->L; ++l)
    if (donor[l] < 0 || donor[l] > l || donor[donor[l]] != donor[l]) return KVP_ERR_BAD_DONOR;
  static thread_local SubGroup subs[4096];
  const int n_sub = build_groups(d, donor, layer_begin, layer_end, subs, 4096);
  if (n_sub < 0) return KVP_ERR_UNSUPPORTED;
  for (int i = 0; i < n_sub; ++i) {      // all of them before anything is launched
    const int own = subs[i].owner;
    if (k_cache[own] == nullptr || v_cache[own] == nullptr || k_scale[own] == nullptr || v_scale[own] == nullptr) return KVP_ERR_INVALID_ARG;
    if (!aligned16(k_cache[own]) || !aligned16(v_cache[own])) return KVP_ERR_UNSUPPORTED;
    for (int m = 0; m < subs[i].n; ++m) {
      const int l = subs[i].members[m];
      if (q[l] == nullptr || o[l] == nullptr || lse[l] == nullptr) return KVP_ERR_INVALID_ARG;
      if (!aligned16(q[l]) || !aligned16(o[l]) || (reinterpret_cast<uintptr_t>(lse[l]) & 3u) != 0) return KVP_ERR_UNSUPPORTED;
    }
  }
  const DealBy by = deal8_by(d->dh, most_rows(d, subs, n_sub));
  const Scratch plan = plan_scratch(d, subs, n_sub, 0, by);
  if (ws == nullptr || ws_bytes < plan.bytes || !aligned16(ws)) return KVP_ERR_WORKSPACE;

  Dec8Params<MAX_DEC_GROUPS> p;
  p.block_table = block_table;
  p.lengths = lengths;
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(ws) + align256(plan.pieces * plan.rows * d->dh * 4));
  p.B = d->B;
  p.Hq = d->Hq;
  p.Hkv = d->Hkv;
  p.page_size = d->page_size;
  p.max_pages = d->max_pages;
  p.n_pages = d->n_pages;
  p.rows = plan.rows;
  p.fit = by.fit;
  p.max_shares = plan.max_shares;
  p.num_splits = d->num_splits;
  p.io_f32 = d->dtype == KVP_F32;
  p.seen = seen;
  p.scale_log2 = (scale == 0.f ? 1.f / sqrtf(float(d->dh)) : scale) * 1.4426950408889634f;

  for (int s0 = 0; s0 < n_sub; s0 += MAX_DEC_GROUPS) {
    const int n = std::min(n_sub - s0, MAX_DEC_GROUPS);
    for (int i = 0; i < n; ++i) {
      const SubGroup& sg = subs[s0 + i];
      Dec8Group& g = p.grp[i];
      g.k_cache = reinterpret_cast<const uint8_t*>(k_cache[sg.owner]);
      g.v_cache = reinterpret_cast<const uint8_t*>(v_cache[sg.owner]);
      g.k_scale = k_scale[sg.owner];
      g.v_scale = v_scale[sg.owner];
      g.n_members = sg.n;
      g.pad = 0;
      for (int m = 0; m < MAX_MEMBERS; ++m) {
        const int l = sg.members[m < sg.n ? m : 0];
        g.q[m] = q[l];
        g.o[m] = o[l];
        g.lse[m] = lse[l];
      }
    }
    const int rows = most_rows(d, subs + s0, n);
    const long long units = (long long)n * d->B * d->Hkv;
    // a block for every share of the longest list; shares go by the lengths on the device, and so does whether whole units
    // are dealt out instead
    p.n_groups = n;
    p.by_units = dealt_by_units(d->dh, longest_list(d, n), units, longest_unit(d), p.fit);
    const long long most_blocks = (long long)p.fit * by.rounds;
    const long long blocks = d->num_splits > 0 ? units * d->num_splits
                             : p.by_units      ? std::min(blocks_by_units(units, d->B, p.fit), most_blocks)
                                               : std::max((long long)plan.max_shares, std::min(units, most_blocks));
    if (units > 0x3fffffffLL || blocks > 0x3fffffffLL) return KVP_ERR_UNSUPPORTED;
    const long long unit_pieces = d->num_splits > 0 ? d->num_splits : plan.max_shares / units;
    const int wpr = unit_pieces > 8 ? 8 : 1;   // many pieces a unit: eight warps share those of a row
    const int rows_per_block = COMBINE_THREADS / 32 / wpr;
    const dim3 grid(static_cast<unsigned>(blocks)), cgrid(unsigned(units), (rows + rows_per_block - 1) / rows_per_block);
    const cudaError_t e = d->dh == 128 ? (plan.rows <= 8 ? launch_decode8<128, 1>(p, grid, cgrid, wpr, stream) : launch_decode8<128, 2>(p, grid, cgrid, wpr, stream))
                                       : (plan.rows <= 8 ? launch_decode8<64, 1>(p, grid, cgrid, wpr, stream) : launch_decode8<64, 2>(p, grid, cgrid, wpr, stream));
    if (e != cudaSuccess) return KVP_ERR_CUDA;
  }
  return KVP_OK;
}
