// The tokens of a batch by item (longer_sort_ids): a stable radix sort of (id, token), lowest digit first, and the runs of equal ids.
#include "embedding.h"

namespace longer {
namespace srt {

using emb::Divider;

struct Ids {
  const char* data;
  int64_t user, row;
  const int32_t* lens;
  Divider by_L;
  uint32_t n, L, table_rows;
  int wide;
};

constexpr int kMostBits = 11;                        // of a round's digit
constexpr uint32_t kNone = 0xffffffffu;              // of a token that names no row (ids are below 2^31)

__device__ __forceinline__ uint32_t id_of(const Ids& a, uint32_t i) {
  const uint32_t b = a.by_L(i), l = i - b * a.L;
  if (a.lens && (int)l >= a.lens[b]) return kNone;
  const int64_t at = (int64_t)b * a.user + (int64_t)l * a.row;
  const int64_t id = a.wide ? ((const int64_t*)a.data)[at] : ((const int32_t*)a.data)[at];
  return (uint64_t)id < a.table_rows ? (uint32_t)id : kNone;
}

// Places of a wave's items among those with their digit, in the wave's order: item i of lane l comes before item i of lane l + 1, and that
// before item i + 1 of any lane.  `count`: the wave's own, one 16-bit counter a digit, two to a word, zero before.  An item's peers, the lanes with its
// digit, come from one ballot a bit (peers whose bit is as the lane's: not the exclusive or of the ballot and the lane's bit in every
// place); the lowest of them moves the counter on for all, and hands on what it found.  There are `rounds` items (the same for all lanes) of
// ITEMS; an item that is not there has no place.
template <int ITEMS>
__device__ __forceinline__ void rank(const uint32_t* digit, const bool* there, int rounds, int bits, uint32_t* count, uint32_t* at) {
  uint32_t lo[ITEMS], hi[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint64_t all = __ballot(there[i]);
    lo[i] = (uint32_t)all;
    hi[i] = (uint32_t)(all >> 32);
  }
  for (int b = 0; b < bits; ++b) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (i >= rounds) break;
      const uint32_t mine = (uint32_t)__builtin_amdgcn_sbfe(digit[i], b, 1);
      const uint64_t with = __ballot(mine);
      lo[i] = __builtin_amdgcn_bitop3_b32(lo[i], (uint32_t)with, mine, 0x90);
      hi[i] = __builtin_amdgcn_bitop3_b32(hi[i], (uint32_t)(with >> 32), mine, 0x90);
    }
  }
  uint32_t old[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (i >= rounds) break;
    at[i] = __builtin_amdgcn_mbcnt_hi(hi[i], __builtin_amdgcn_mbcnt_lo(lo[i], 0));
    old[i] = 0;
    if (there[i] && at[i] == 0) old[i] = atomicAdd(&count[digit[i] >> 1], (uint32_t)(__popc(lo[i]) + __popc(hi[i])) << 16 * (digit[i] & 1));
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (i >= rounds) break;
    const int first = lo[i] ? __ffs(lo[i]) - 1 : __ffs(hi[i]) + 31;
    at[i] += (uint32_t)__shfl((int)old[i], first & 63) >> 16 * (digit[i] & 1) & 0xffff;
  }
}

// Of the counts of four neighbouring digits, wave by wave, the sums over the waves before, in their place; returns those over all.  (`words`: [waves][digits / 2])
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <int WAVES>
__device__ __forceinline__ u32x4 waves_before(uint32_t* words, uint32_t digits, uint32_t four) {
  u32x2 c[WAVES], sum = {};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) c[w] = *(const u32x2*)(words + w * (digits / 2) + 2 * four);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    *(u32x2*)(words + w * (digits / 2) + 2 * four) = sum;
    sum += c[w];                                     // (no half passes 2^16: a workgroup's items are fewer)
  }
  return u32x4{sum[0] & 0xffff, sum[0] >> 16, sum[1] & 0xffff, sum[1] >> 16};
}

// inclusive sum over a wave
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t w = __shfl_up(v, o);
    if (lane >= o) v += w;
  }
  return v;
}

// exclusive sum over a workgroup, and the sum of all in *sum (lds: a word for each wave); every thread takes part
template <int THREADS>
__device__ __forceinline__ uint32_t group_scan(uint32_t v, uint32_t* lds, uint32_t* sum) {
  const int wave = threadIdx.x >> 6;
  const uint32_t in = wave_scan(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds[wave] = in;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    before += w < wave ? lds[w] : 0;
    all += lds[w];
  }
  *sum = all;
  return before + in - v;
}

// ------------------------------------------------------------------------------------ few tokens: one workgroup
constexpr int kFewThreads = 1024, kFewItems = 4, kFew = kFewThreads * kFewItems, kFewWaves = kFewThreads / 64;

// A wave takes 64 * items neighbours; rounds of up to kMostBits bits, all in LDS.  Bound by the one compute unit that they are on: 256 / 4096 tokens of 1000
// rows in 6.7 / 8.6 us (the launches for many tokens: 9.3 / 9.7), of 1000003 rows 7.4 / 12.9 (15.3 / 17.5); 6144 tokens 11.5 / 18.0 (9.7 / 17.7).
__global__ __launch_bounds__(kFewThreads) void few_kernel(Ids a, int bits, int per_round, longer_order out) {
  __shared__ alignas(16) uint32_t keys[kFew], words[kFewWaves << (kMostBits - 1)], base[1 << kMostBits];
  __shared__ uint32_t lds[kFewWaves];
  __shared__ uint16_t tokens[kFew];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int items = (a.n + kFewThreads - 1) / kFewThreads;
  uint32_t n = a.n, key[kFewItems], token[kFewItems];
#pragma unroll
  for (int i = 0; i < kFewItems; ++i) {
    const uint32_t k = (wave * items + i) * 64 + lane;
    key[i] = i < items && k < n ? id_of(a, k) : kNone;
    token[i] = k;
  }
  for (int shift = 0; shift < bits; shift += per_round) {
    const int round = per_round;                     // (the last one's digits may pass the ids' bits)
    const uint32_t digits = 1u << round;
    if (shift) {
#pragma unroll
      for (int i = 0; i < kFewItems; ++i) {
        const uint32_t k = (wave * items + i) * 64 + lane;
        key[i] = i < items && k < n ? keys[k] : kNone;
        token[i] = i < items && k < n ? tokens[k] : 0;
      }
    }
    for (uint32_t i = threadIdx.x; i < kFewWaves * digits / 2; i += kFewThreads) words[i] = 0;
    __syncthreads();
    uint32_t digit[kFewItems], at[kFewItems];
    bool there[kFewItems];
#pragma unroll
    for (int i = 0; i < kFewItems; ++i) {
      there[i] = key[i] != kNone;
      digit[i] = key[i] >> shift & (digits - 1);
    }
    rank<kFewItems>(digit, there, items, round, words + wave * (digits / 2), at);
    __syncthreads();
    // where each digit begins, and in it each wave
    const uint32_t four = threadIdx.x;
    const u32x4 sums = 4 * four < digits ? waves_before<kFewWaves>(words, digits, four) : u32x4{};
    const uint32_t before = group_scan<kFewThreads>(sums[0] + sums[1] + sums[2] + sums[3], lds, &n);   // (the first round drops the tokens that name no row)
    if (4 * four < digits) *(u32x4*)(base + 4 * four) = u32x4{before, before + sums[0], before + sums[0] + sums[1], before + sums[0] + sums[1] + sums[2]};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewItems; ++i)
      if (i < items && key[i] != kNone) {
        const uint32_t to = base[digit[i]] + ((const uint16_t*)words)[wave * digits + digit[i]] + at[i];
        keys[to] = key[i];
        tokens[to] = (uint16_t)token[i];
      }
    __syncthreads();
  }
  // runs: a wave takes its neighbours 64 at a time
  uint32_t runs = 0, all;
  uint64_t heads[kFewItems];
#pragma unroll
  for (int i = 0; i < kFewItems; ++i) {
    heads[i] = 0;
    const uint32_t k = (wave * items + i) * 64 + lane;
    if (i < items) heads[i] = __ballot(k < n && (k == 0 || keys[k] != keys[k - 1]));
    runs += __popcll(heads[i]);
  }
  if (lane == 0) lds[wave] = runs;
  __syncthreads();
  uint32_t run = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    run += w < wave ? lds[w] : 0;
    all += lds[w];
  }
#pragma unroll
  for (int i = 0; i < kFewItems; ++i) {
    const uint32_t k = (wave * items + i) * 64 + lane;
    if (i < items && k < n) {
      const uint32_t mine = run + __popcll(heads[i] & ((2ull << lane) - 1)) - 1;
      if (heads[i] >> lane & 1) out.rows[mine] = (int)keys[k];
      out.runs[k] = (int)mine;
      out.tokens[k] = tokens[k];
    }
    run += __popcll(heads[i]);
  }
  if (threadIdx.x == 0) {
    out.counts[0] = (int)all;
    out.counts[1] = (int)n;
  }
}

// ------------------------------------------------------------------------------------ many tokens
// A round of the sort takes one digit, in three launches: every workgroup counts the digits of its stretch of the items, the counts are summed
// over the workgroups before it, and it moves its items.  The first round reads the ids themselves and drops the tokens that name no
// row; between rounds an item is a word of eight bytes, id below and token above.  (The sums inside the move, each workgroup reading
// all counts: 30 us a round for 24.)  512000 tokens of 1000003 rows take 40 us, of which each launch's own time is a third: count 5, sums 5, move 12
// and 10, bound by latency and the scattered stores; 14 MB have to move.
//
// The runs' numbers need no pass over the sorted ids where the table has at most 2^22 rows.  One round (up to 2^11 rows): a digit is an id, and its run the
// number of digits before it whose count is not zero.  Two rounds: the first one's move leaves a byte at each id that it meets, the second
// one's count makes of them, for every 32 ids, a mask and how many ids there are before it in its 2048, and the second move looks its ids up.
// Larger tables take three rounds and two launches that number the runs of the sorted ids.
//
// A thread has 4 items of a tile; 2 where that leaves no compute unit a second workgroup, 1 in the smallest (4 / 2 / 1, 1000003 rows: 512000 tokens 40 / 43 / - us,
// 256000 35.6 / 31.5 / 36.6, 64000 28.6 / 26.5 / 25.7, 16384 25.3 / 20.1 / 19.8, 6144 - / 19.7 / 17.7).
constexpr int kThreads = 512, kItems = 4, kWaves = kThreads / 64, kMostGroups = 512;
constexpr int kSumAlone = 64;                        // groups whose counts each workgroup adds up itself, for want of anything to do
constexpr int kMaskRows = 32, kSegment = 2048;       // ids of a mask, and of a segment: a wave's

struct Round {
  Ids ids;
  const uint64_t* in;                                // NULL: the first round
  uint64_t* out;                                     // NULL: the last one
  uint32_t *counts, *totals;                         // [groups][digits], [digits]
  uint8_t* seen;                                     // [2^bits of an id], bytes: whether a token names it (NULL: not asked for)
  uint64_t* masks;                                   // [2^bits / 32]: a mask below, the ids before it in its segment above
  uint32_t* segments;                                // [2^bits / 2048]: ids in each
  uint32_t* keys;                                    // the sorted ids, where the runs are numbered from them
  longer_order order;
  int shift, bits, id_bits;
  uint32_t groups;                                   // workgroups with items; those behind them help with the ids that were seen
  int summed;                                        // summed: counts and totals are sums; else each workgroup adds up the counts itself
};

// Workgroups go to the eight chiplets in turn, each with a second-level cache of its own.  Neighbouring stretches, whose items land side by side,
// go to one chiplet: it has whole lines to write back, not an eighth of each.
__device__ __forceinline__ uint32_t group_number(uint32_t groups) {
  const uint32_t chip = blockIdx.x & 7, each = groups / 8, more = groups % 8;
  return blockIdx.x < groups ? chip * each + min(chip, more) + blockIdx.x / 8 : blockIdx.x;
}

// a workgroup's stretch of n items: whole tiles, as even as they can be dealt (behind the last group: none)
struct Stretch { uint32_t begin, end; };
template <int ITEMS>
__device__ __forceinline__ Stretch stretch(uint32_t n, uint32_t group, uint32_t groups) {
  constexpr uint32_t kTile = kThreads * ITEMS;
  const uint32_t tiles = (n + kTile - 1) / kTile, per = (tiles + groups - 1) / groups;
  const uint32_t begin = min((uint64_t)group * per * kTile, (uint64_t)n);
  return {begin, (uint32_t)min((uint64_t)begin + (uint64_t)per * kTile, (uint64_t)n)};
}

// four bytes that are 0 or 1 as four bits
__device__ __forceinline__ uint32_t four_bits(uint32_t bytes) { return bytes * 0x01020408u >> 24 & 15; }

template <bool FIRST, int ITEMS>
__global__ __launch_bounds__(kThreads) void count_kernel(Round r) {
  __shared__ uint32_t count[1 << kMostBits];
  const uint32_t digits = 1u << r.bits;
  for (uint32_t i = threadIdx.x; i < digits; i += kThreads) count[i] = 0;
  __syncthreads();
  const uint32_t group = group_number(r.groups);
  const Stretch s = stretch<ITEMS>(FIRST ? r.ids.n : (uint32_t)r.order.counts[1], group, r.groups);
  for (uint32_t tile = s.begin; tile < s.end; tile += kThreads * ITEMS) {
    uint32_t key[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const uint32_t i = tile + k * kThreads + threadIdx.x;
      key[k] = i >= s.end ? kNone : FIRST ? id_of(r.ids, i) : (uint32_t)r.in[i];
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
      if (key[k] != kNone) atomicAdd(&count[key[k] >> r.shift & (digits - 1)], 1u);
  }
  if (r.seen) {
    if (FIRST) {
      for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < 1u << (r.id_bits - 4); i += gridDim.x * kThreads) ((u32x4*)r.seen)[i] = u32x4{};
    } else {
      const int lane = threadIdx.x & 63;
      for (uint32_t i = blockIdx.x * kWaves + (threadIdx.x >> 6); i < 1u << r.id_bits >> 11; i += gridDim.x * kWaves) {
        const u32x4* from = (const u32x4*)(r.seen + (size_t)i * kSegment) + 2 * lane;
        const u32x4 lo = from[0], hi = from[1];
        uint32_t mask = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) mask |= four_bits(lo[k]) << 4 * k | four_bits(hi[k]) << (16 + 4 * k);
        const uint32_t ids = __popc(mask), to = wave_scan(ids);
        r.masks[i * 64 + lane] = (uint64_t)(to - ids) << 32 | mask;
        if (lane == 63) r.segments[i] = to;
      }
    }
  }
  __syncthreads();
  if (group < r.groups)
    for (uint32_t i = threadIdx.x; i < digits; i += kThreads) r.counts[(size_t)group * digits + i] = count[i];
}

// counts[g][digit] becomes the sum over the groups before g, totals[digit] that over all: 32 digits a workgroup, 32 shares of SHARE groups at most
template <int SHARE>
__global__ __launch_bounds__(1024) void sum_kernel(uint32_t* counts, uint32_t* totals, int groups, uint32_t digits) {
  __shared__ uint32_t lds[32][33];
  const uint32_t digit = blockIdx.x * 32 + (threadIdx.x & 31);
  const int share = threadIdx.x >> 5, per = (groups + 31) / 32, begin = share * per, mine = max(min(groups - begin, per), 0);
  uint32_t sum = 0, c[SHARE];
#pragma unroll
  for (int k = 0; k < SHARE; ++k) c[k] = k < mine && digit < digits ? counts[(size_t)(begin + k) * digits + digit] : 0;
#pragma unroll
  for (int k = 0; k < SHARE; ++k) sum += c[k];
  lds[share][threadIdx.x & 31] = sum;
  __syncthreads();
  if (digit >= digits) return;
  uint32_t before = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) before += i < share ? lds[i][threadIdx.x & 31] : 0;
  if (share == 31) totals[digit] = before + sum;
#pragma unroll
  for (int k = 0; k < SHARE; ++k) {
    if (k < mine) counts[(size_t)(begin + k) * digits + digit] = before;
    before += c[k];
  }
}

// LAST: 0 items go on to another round, 1 to the order with their runs, 2 to the order and the sorted ids
template <bool FIRST, int LAST, int ITEMS>
__global__ __launch_bounds__(kThreads) void move_kernel(Round r) {
  static_assert((1 << kMostBits) <= 4 * kThreads, "a thread has four digits");
  __shared__ alignas(16) uint32_t words[kWaves << (kMostBits - 1)], base[1 << kMostBits], runs[1 << kMostBits];
  __shared__ uint32_t lds[kWaves];
  const uint32_t digits = 1u << r.bits, group = group_number(r.groups), four = 4 * threadIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  uint32_t key[ITEMS], token[ITEMS], digit[ITEMS], at[ITEMS];
  bool there[ITEMS];
  auto load = [&](uint32_t tile, uint32_t end) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t k = tile + (wave * ITEMS + i) * 64 + lane;
      key[i] = kNone;
      if (k < end) {
        const uint64_t v = FIRST ? 0 : r.in[k];
        key[i] = FIRST ? id_of(r.ids, k) : (uint32_t)v;
        token[i] = FIRST ? k : (uint32_t)(v >> 32);
      }
    }
  };
  Stretch s = stretch<ITEMS>(FIRST ? r.ids.n : (uint32_t)r.order.counts[1], group, r.groups);
  load(s.begin, s.end);                              // (under way while the digits' places are found)
  // where each digit begins, and in it this workgroup
  uint32_t n, named = 0;
  {
    u32x4 all = {}, mine = {};
    if (four < digits) {
      if (r.summed) {
        all = *(const u32x4*)(r.totals + four);
        mine = *(const u32x4*)(r.counts + (size_t)min(group, r.groups - 1) * digits + four);
      } else {
        constexpr uint32_t U = 16;
        for (uint32_t g = 0; g < r.groups; g += U) {
          u32x4 c[U];
#pragma unroll
          for (uint32_t u = 0; u < U; ++u) c[u] = *(const u32x4*)(r.counts + (size_t)min(g + u, r.groups - 1) * digits + four);
#pragma unroll
          for (uint32_t u = 0; u < U; ++u) {
            all += g + u < r.groups ? c[u] : u32x4{};
            mine += g + u < group ? c[u] : u32x4{};
          }
        }
      }
    }
    const uint32_t before = group_scan<kThreads>(all[0] + all[1] + all[2] + all[3], lds, &n);
    if (four < digits) *(u32x4*)(base + four) = mine + u32x4{before, before + all[0], before + all[0] + all[1], before + all[0] + all[1] + all[2]};
    if (FIRST && LAST == 1) {                        // a digit is an id
      const u32x4 one = {all[0] != 0, all[1] != 0, all[2] != 0, all[3] != 0};
      uint32_t run = group_scan<kThreads>(one[0] + one[1] + one[2] + one[3], lds, &named);
      if (four < digits)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          runs[four + k] = run;
          if (group == 0 && one[k]) r.order.rows[run] = (int)(four + k);
          run += one[k];
        }
    }
  }
  if (!FIRST && LAST == 1) {                         // the runs before each segment, and the rows themselves
    const uint32_t segments = 1u << r.id_bits >> 11;
    for (uint32_t d = 0; d < segments; d += kThreads) {
      const uint32_t i = d + threadIdx.x;
      uint32_t sum;
      const uint32_t before = group_scan<kThreads>(i < segments ? r.segments[i] : 0, lds, &sum);
      if (i < segments) runs[i] = named + before;
      named += sum;
    }
    __syncthreads();
    for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < segments * 64; i += gridDim.x * kThreads) {
      const uint64_t v = r.masks[i];
      uint32_t run = runs[i / 64] + (uint32_t)(v >> 32);
      for (uint32_t mask = (uint32_t)v; mask; mask &= mask - 1) r.order.rows[run++] = (int)(i * kMaskRows + __ffs(mask) - 1);
    }
  }
  if (group == 0 && threadIdx.x == 0) {
    if (FIRST) r.order.counts[1] = (int)n;
    if (LAST == 1) r.order.counts[0] = (int)named;
  }
  for (uint32_t tile = s.begin; tile < s.end; tile += kThreads * ITEMS) {
    if (tile != s.begin) load(tile, s.end);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      there[i] = key[i] != kNone;
      digit[i] = key[i] >> r.shift & (digits - 1);
    }
    for (uint32_t i = threadIdx.x; i < kWaves * digits / 2; i += kThreads) words[i] = 0;
    __syncthreads();
    rank<ITEMS>(digit, there, ITEMS, r.bits, words + wave * (digits / 2), at);
    __syncthreads();
    // where each wave begins in a digit
    const u32x4 sums = four < digits ? waves_before<kWaves>(words, digits, four / 4) : u32x4{};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (there[i]) {
        const uint32_t to = base[digit[i]] + ((const uint16_t*)words)[wave * digits + digit[i]] + at[i];
        if (LAST == 0) {
          r.out[to] = (uint64_t)token[i] << 32 | key[i];
          if (FIRST && r.seen) r.seen[key[i]] = 1;
        } else {
          r.order.tokens[to] = (int)token[i];
          if (LAST == 2) {
            r.keys[to] = key[i];
          } else if (FIRST) {
            r.order.runs[to] = (int)runs[digit[i]];
          } else {
            const uint64_t v = r.masks[key[i] / kMaskRows];
            r.order.runs[to] = (int)(runs[key[i] / kSegment] + (uint32_t)(v >> 32) + __popc((uint32_t)v & ((1u << key[i] % kMaskRows) - 1)));
          }
        }
      }
    __syncthreads();
    if (four < digits) *(u32x4*)(base + four) += sums;
  }
}

// how many runs begin in each workgroup's stretch of the sorted ids
__global__ __launch_bounds__(kThreads) void heads_kernel(const uint32_t* keys, const int32_t* n, uint32_t* heads) {
  __shared__ uint32_t lds[kWaves];
  const Stretch s = stretch<kItems>((uint32_t)*n, blockIdx.x, gridDim.x);
  uint32_t mine = 0, all;
  for (uint32_t k = s.begin + threadIdx.x; k < s.end; k += kThreads) mine += k == 0 || keys[k] != keys[k - 1];
  group_scan<kThreads>(mine, lds, &all);
  if (threadIdx.x == 0) heads[blockIdx.x] = all;
}

__global__ __launch_bounds__(kThreads) void runs_kernel(const uint32_t* keys, const uint32_t* heads, longer_order out) {
  static_assert(kMostGroups <= kThreads, "a thread adds up one group's runs");
  __shared__ uint32_t lds[kWaves];
  uint32_t run, all;
  group_scan<kThreads>(threadIdx.x < blockIdx.x ? heads[threadIdx.x] : 0, lds, &run);
  const Stretch s = stretch<kItems>((uint32_t)out.counts[1], blockIdx.x, gridDim.x);
  for (uint32_t tile = s.begin; tile < s.end; tile += kThreads * kItems) {
    const uint32_t first = tile + threadIdx.x * kItems;
    uint32_t key[kItems], before = first && first < s.end ? keys[first - 1] : kNone, mine = 0;
    bool head[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      key[i] = first + i < s.end ? keys[first + i] : kNone;
      head[i] = key[i] != kNone && key[i] != before;
      mine += head[i];
      before = key[i];
    }
    uint32_t at = run + group_scan<kThreads>(mine, lds, &all);
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (key[i] != kNone) {
        if (head[i]) out.rows[at++] = (int)key[i];
        out.runs[first + i] = (int)at - 1;
      }
    run += all;
  }
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) out.counts[0] = (int)run;
}

// ------------------------------------------------------------------------------------ host
static int bits_of(int64_t rows) {
  int bits = 2;                                      // (a thread has four digits)
  while (((int64_t)1 << bits) < rows) ++bits;
  return bits;
}

struct Plan {
  int bits, rounds, per_round, items_each, groups;
  size_t items, keys, counts, totals, seen, masks, segments, heads, bytes;      // places in the workspace: items of two rounds, at its front
};

static Plan plan(int B, int L, int64_t rows) {
  const size_t n = (size_t)B * L;
  Plan p = {};
  p.bits = bits_of(rows);
  p.rounds = (p.bits + kMostBits - 1) / kMostBits;
  p.per_round = (p.bits + p.rounds - 1) / p.rounds;
  if (n <= kFew) {
    p.bytes = 256;
    return p;
  }
  p.items_each = n <= 16384 ? 1 : n <= 256 * 2 * kThreads ? 2 : kItems;
  p.groups = (int)std::min<size_t>((n + kThreads * p.items_each - 1) / (kThreads * p.items_each), kMostGroups);
  size_t at = 0;
  auto place = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  if (p.rounds > 1) place(n * 8);
  if (p.rounds > 2) p.items = place(n * 8);
  if (p.rounds > 2) p.keys = place(n * 4);
  p.counts = place(((size_t)p.groups << p.per_round) * 4);
  p.totals = place((size_t)4 << p.per_round);
  if (p.rounds == 2) {
    p.seen = place((size_t)1 << p.bits);
    p.masks = place((size_t)8 << p.bits >> 5);
    p.segments = place((size_t)4 << p.bits >> 11);
  }
  if (p.rounds > 2) p.heads = place((size_t)p.groups * 4);
  p.bytes = at;
  return p;
}

}  // namespace srt
}  // namespace longer

using namespace longer;

extern "C" {

size_t longer_sort_ids_workspace_bytes(int B, int L, int64_t table_rows) {
  return check_tokens(B, L) || check_table_rows(table_rows) ? 0 : srt::plan(B, L, table_rows).bytes;
}

int longer_sort_ids(const longer_ids* ids, const int32_t* lens, int B, int L, int64_t table_rows, const longer_order* order,
                    void* ws, size_t ws_bytes, void* stream) {
  int rc = check_tokens(B, L);
  if (!rc) rc = check_ids(ids, lens, B, L);
  if (!rc) rc = check_table_rows(table_rows);
  if (!rc) rc = emb::check_order(order);
  if (!rc && (!ws || ((uintptr_t)ws & 255))) rc = api_error(LONGER_ERR_ARG, "ws must be 256-byte aligned and not NULL");
  if (rc) return rc;
  const srt::Plan p = srt::plan(B, L, table_rows);
  if (ws_bytes < p.bytes) return api_error(LONGER_ERR_WS, "workspace too small: %zu < %zu bytes", ws_bytes, p.bytes);
  hipStream_t st = (hipStream_t)stream;
  const srt::Ids a = {(const char*)ids->data, B > 1 ? ids->user_stride : 0, L > 1 ? ids->row_stride : 0, lens, emb::divider(L), (uint32_t)B * L, (uint32_t)L,
                      (uint32_t)table_rows, ids->type == LONGER_I64};
  if (a.n <= srt::kFew) {
    srt::few_kernel<<<1, srt::kFewThreads, 0, st>>>(a, p.bits, p.per_round, *order);
    return launched("sort of ids");
  }
  char* w = (char*)ws;
  uint64_t* items[2] = {(uint64_t*)w, (uint64_t*)(w + p.items)};
  uint32_t* keys = (uint32_t*)(w + p.keys);
  srt::Round r = {a, nullptr, items[0], (uint32_t*)(w + p.counts), (uint32_t*)(w + p.totals), p.rounds == 2 ? (uint8_t*)(w + p.seen) : nullptr, (uint64_t*)(w + p.masks), (uint32_t*)(w + p.segments), keys, *order,
                  0, p.per_round, p.bits, (uint32_t)p.groups, p.groups > srt::kSumAlone};
  // (a wave for each segment of the ids that may have been seen: 9000 tokens of 1000003 rows 37 us with the items' workgroups alone)
  const int grid = p.rounds == 2 ? std::max(p.groups, (1 << p.bits >> 11) / srt::kWaves) : p.groups;
  auto sort = [&](auto items_each) {
    constexpr int ITEMS = decltype(items_each)::value;
    for (int i = 0; i < p.rounds; ++i) {
      r.in = i ? items[(i - 1) & 1] : nullptr;
      r.out = items[i & 1];
      r.shift = i * p.per_round;
      r.bits = p.per_round;                          // (the last round's digits may pass the ids' bits)
      const uint32_t digits = 1u << r.bits;
      if (i == 0) srt::count_kernel<true, ITEMS><<<grid, srt::kThreads, 0, st>>>(r);
      else srt::count_kernel<false, ITEMS><<<grid, srt::kThreads, 0, st>>>(r);
      if (r.summed) {
        auto sum = p.groups > 256 ? srt::sum_kernel<srt::kMostGroups / 32> : srt::sum_kernel<8>;
        sum<<<(digits + 31) / 32, 1024, 0, st>>>(r.counts, r.totals, p.groups, digits);
      }
      const int last = i + 1 < p.rounds ? 0 : p.rounds <= 2 ? 1 : 2;
      if (i == 0 && last) srt::move_kernel<true, 1, ITEMS><<<p.groups, srt::kThreads, 0, st>>>(r);
      else if (i == 0) srt::move_kernel<true, 0, ITEMS><<<p.groups, srt::kThreads, 0, st>>>(r);
      else if (last == 0) srt::move_kernel<false, 0, ITEMS><<<p.groups, srt::kThreads, 0, st>>>(r);
      else if (last == 1) srt::move_kernel<false, 1, ITEMS><<<grid, srt::kThreads, 0, st>>>(r);
      else srt::move_kernel<false, 2, ITEMS><<<p.groups, srt::kThreads, 0, st>>>(r);
    }
  };
  if (p.items_each == 1) sort(std::integral_constant<int, 1>());
  else if (p.items_each == 2) sort(std::integral_constant<int, 2>());
  else sort(std::integral_constant<int, srt::kItems>());
  if (p.rounds > 2) {
    uint32_t* heads = (uint32_t*)(w + p.heads);
    srt::heads_kernel<<<p.groups, srt::kThreads, 0, st>>>(keys, order->counts + 1, heads);
    srt::runs_kernel<<<p.groups, srt::kThreads, 0, st>>>(keys, heads, *order);
  }
  return launched("sort of ids");
}

}  // extern "C"
