// Attention over the paged 8-bit K/V cache (gfx950).
//
// Query row i of a stream (position p = kv_len - q_len + i) of head h sees the keys
// j in [lo, hi) of its stream,
//     end = kv_len without frames, else (floor(p / frame) + 1) * frame,
//     hi = min(end, kv_len), lo = max(0, end - window) with a window, else 0,
//     O = sum_j softmax_j(scale * Q . K_j) V_j,  K_j = code * 2^ke, V_j = code * 2^ve.
//
// Rows are taken per K/V head: the heads / kv_heads query heads that share a K/V head lie
// next to each other, row = token * group + head in the group, in tiles of kRows rows.
// Work item = (tile, chunk of its keys), one workgroup per item and K/V head. The chunk
// length follows from the lengths on the device (work_of), the same in every wave: as many
// items as the chip holds workgroups, where the tiles alone are fewer (of large tiles, as
// many as are estimated to end first). A tile in several chunks leaves unnormalised
// partial results that cache_combine_kernel merges in chunk order (no atomics: the result
// is the same on every run).
//
// Codes enter the products exactly (E4M3 has four significant bits; bf16 holds them times
// the page's power of two, V's times 2^-kValueDown of it); accumulation, statistics and sums
// are fp32. P is rounded to bf16 for its product with V, as the matrix unit takes it: at most
// half a step, 2^-8 of each term, the same as the output's own rounding.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "fva_common.h"
#include "fva_geometry.h"
#include "fva_internal.h"

namespace fva {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;        // query rows of a small tile: one MFMA column each
constexpr int kBigRows = 128;    // query rows of a large tile: 32 for each wave
constexpr int kKeys = 64;        // keys a wave takes at a time
constexpr int kWaves = 4;        // waves of a workgroup (small tiles of few keys: 1 to 8)
constexpr int kCacheSlots = 2048;  // workgroups to split for, small tiles
constexpr int kBigSlots = 512;     // large tiles: two a CU, as many as are resident (a round)
constexpr int kBigRounds = 5;      // that their chunks may take
constexpr int kDeal = 64;          // chunks that are dealt from one end of a head's to the other (32: 82 us for 69.6 below)
constexpr int kXcds = 8;
constexpr int kMostChunks = 128;   // of a tile
constexpr int kMinChunk = kWaves * kKeys;  // a shorter chunk leaves a small tile's waves without keys
// V enters its product on 2^-kValueDown of its scale, and O is scaled back where it is written.
// A page's scale reaches 2^120 (a value above 448 * 2^119, an infinity), on which codes from 256
// on are no finite bf16 numbers: an infinity there would meet the P = 0 of a row that does not
// see its key, and 0 * inf is NaN. Sixteen binades down, the largest value is 1.75 * 2^112, and
// the smallest code of the smallest scale, 2^(-9 - 100 - 16), is still a normal number.
constexpr int kValueDown = 16;
constexpr float kValueUp = 65536.f;
static_assert(kValueUp == (float)(1 << kValueDown) && kCacheExpMin - 9 - kValueDown >= -126);

typedef __attribute__((address_space(4))) const int32_t const_i32;

// n / d for 0 <= n < 2^31 without a division (Divisor).
__device__ __forceinline__ int divide(int n, const Divisor& d) { return (int)(((uint64_t)(uint32_t)n * d.mul) >> d.shift); }

// One stream's share of the work: its rows, keys and tiles.
struct Stream {
  int q0, q_len;  // first token row, tokens (those past Q's rows left out)
  int p0;         // position of the first of them
  int kv_len;
  int tiles;
  int span;       // keys that any of its tiles sees, at most
  int mean;       // about how many they see in the middle, at least span / 2
  int chunks;     // that a tile's keys are cut into, at most (set by work_of)
};

__device__ __forceinline__ Stream stream_of(const CacheAttnArgs& P, int s) {
  Stream r;
  // Lengths and starts come from device memory: clamped, so that no index leaves the
  // tensors whatever they hold.
  const int start = max(P.q_start[s], 0), end = max(P.q_start[s + 1], start);
  r.q0 = min(start, P.tokens);
  r.q_len = min(end, P.tokens) - r.q0;
  r.kv_len = min(max(P.kv_len[s], 0), P.width << P.page_shift);
  r.p0 = r.kv_len - (end - start);
  r.tiles = (int)(((uint32_t)(r.q_len * P.group) + (uint32_t)P.rows - 1) >> P.row_shift);
  r.span = min(r.kv_len, P.most_keys);
  r.mean = P.ramp ? min(r.span, max(r.kv_len - (r.q_len >> 1), (r.kv_len + 1) >> 1)) : r.span;
  r.chunks = 1;
  return r;
}

// The keys of a tile, [begin, end) with begin on a multiple of kKeys: those that its first
// row's window starts with to those that its last row ends with.
struct Span {
  int begin, lo, end;
};

// Chunks that `span` keys are cut into, at least one and at most kMostChunks (their merge
// takes a turn of its own for every few).
__device__ __forceinline__ int chunks_of(int span, int chunk) {
  return (int)min(max(1u, ((uint32_t)span + (uint32_t)chunk - 1u) / (uint32_t)chunk), (uint32_t)kMostChunks);
}

// The largest value of the wave, in every lane.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t b) {
  b = max(b, dpp_move<0xB1>(b));
  b = max(b, dpp_move<0x4E>(b));
  b = max(b, dpp_move<0x141>(b));
  b = max(b, dpp_move<0x140>(b));
  const auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  b = max(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return max(q[0], q[1]);
}

// What a wave knows of the whole call: the streams over its lanes, the first 64 of them
// in registers (the others are looked at again).
struct Work {
  Stream mine;
  int chunk;     // keys of a chunk, at most
  int upto;      // items of the first 64 streams up to and with the lane's
  int items;     // of all, per K/V head
};

__device__ __forceinline__ Stream none() { return Stream{0, 0, 0, 0, 0, 0, 0, 1}; }

__device__ __forceinline__ Stream stream_in(const CacheAttnArgs& P, int s, int chunk) {
  if (s >= P.streams) return none();
  Stream r = stream_of(P, s);
  if (P.slots) r.chunks = chunks_of(r.span, chunk);
  return r;
}

// Chunk length of large tiles. They run in rounds of as many workgroups as are resident, the
// last of which may be nearly empty: 13 tiles of 40 heads, 520 workgroups of 537 steps, took
// 1400 us as they are, 1140 / 1057 / 1023 in two / three / four chunks each (without frames;
// causal by frame 1478 us as they are, 1090 as chosen here). Each lane
// estimates one length: those that fill one round, two, ... and longer ones, and the tiles as
// they are. The end of the rounds is the mean workgroup's steps and its way in for each, what
// the longest has more, and the merge. The workgroups of a length are estimated from the
// tiles' mean keys, whether there is room for its partial results is counted from the widest
// ones': causal chunks have fewer on average, and a length without room is no choice. (One
// stream, causal by frame, 5 heads, 4680 rows, 32,760 keys: 606 us as 185 workgroups, 363
// split; 8 heads, 1560 rows, 61,560 keys 1114 -> 389.) Of more than 64 streams, whose lengths
// even out, the length that fills one round is taken, or, without room for it, the one that
// room is certain for: a tile of more than one chunk has fewer than 2 * span / length. Tiles
// that stay whole need no room, so that a long stream among many short ones is split however
// many there are (100 streams of 32 rows and up to 300 keys, one of 100,000, 8 heads: 1704 us
// whole, 96 split). (Integers but for reciprocals and their products, which round alike
// everywhere: every wave comes to the same length.)
__device__ __forceinline__ int big_chunk(const CacheAttnArgs& P, const Work& w, uint64_t total, int lane) {
  constexpr int kNever = INT32_MAX / 2;
  constexpr int kWayIn = 12;           // steps that a workgroup's start costs
  constexpr int kLengths = 12;         // tried for a number of rounds, by a tenth longer each
  constexpr int kWhole = 1 << 24;      // steps, no less than any tile has: the tiles as they are
  constexpr int kNoRoom = (1 << 26) - 1;  // more than any cost
  auto tiles_by = [&](auto f) {  // the sum of tiles * f(stream)
    uint64_t n = (uint64_t)w.mine.tiles * (uint64_t)f(w.mine);
    for (int s = lane + kWave; s < P.streams; s += kWave) {
      const Stream r = stream_of(P, s);
      n += (uint64_t)r.tiles * (uint64_t)f(r);
    }
    return wave_sum_u64(n);
  };
  const uint64_t steps64 = total / kKeys;
  const int even = (int)min(steps64 * (uint32_t)P.kv_heads / kBigSlots + 1, (uint64_t)kWhole);  // steps of each of a round's places
  if (P.streams <= kWave) {
    const int tiles = (int)wave_sum_u64((uint64_t)w.mine.tiles);
    if (tiles == 0) return kNever;
    const int r = 1 + lane / kLengths, k = lane % kLengths;
    int n = max((even + r - 1) / r, kMinChunk / kKeys);
    n = lane >= kBigRounds * kLengths ? kWhole : n + n * k / 10;
    const float inv = __builtin_amdgcn_rcpf((float)n) * (1.f + 0x1p-20f);
    const int mine = (w.mine.mean + kKeys - 1) / kKeys;
    const int most = (w.mine.span + kKeys - 1) / kKeys;
    const int longest = min((int)wave_max_u32((uint32_t)mine), n);
    // The chunks that all tiles are cut into, of the streams' means, and those with a partial
    // result, of their spans. (No quotient comes out too small: inv is above 1 / n by more than
    // all roundings.)
    int items = 0, room = 0;
    for (int s0 = 0; s0 < P.streams; s0 += 4) {  // (lanes past the streams have no tiles)
#pragma unroll
      for (int s = s0; s < s0 + 4; ++s) {
        const int tiles_s = __builtin_amdgcn_readlane(w.mine.tiles, s);
        auto cut = [&](int steps) { return tiles_s * min(max((int)((float)(steps + n - 1) * inv), 1), kMostChunks); };
        const int widest = cut(__builtin_amdgcn_readlane(most, s));
        room += widest > tiles_s ? widest : 0;
        items += P.ramp ? cut(__builtin_amdgcn_readlane(mine, s)) : widest;
      }
    }
    const int mean = (int)((float)min(steps64, (uint64_t)1 << 30) * __builtin_amdgcn_rcpf((float)items));
    const int rounds = (items * P.kv_heads + kBigSlots - 1) / kBigSlots;
    int cost = rounds * (mean + kWayIn) + max(longest - mean, 0);
    if (items > tiles) cost += 5 + items * P.kv_heads / 64;
    cost = room > P.slots && n < kWhole ? kNoRoom : min(cost, kNoRoom - 1);
    uint32_t key = ~((uint32_t)cost << 6 | (uint32_t)lane);
    key = wave_max_u32(key);
    const int best = 63 - (int)(key & 63);
    n = __builtin_amdgcn_readlane(n, best);
    return n >= kWhole ? kNever : n * kKeys;
  }
  const int one = max(even, kMinChunk / kKeys);
  if (one >= kWhole) return kNever;
  const uint64_t room = tiles_by([&](const Stream& st) {
    const int c = chunks_of(st.span, one * kKeys);
    return c > 1 ? c : 0;
  });
  if (room <= (uint64_t)P.slots) return one * kKeys;
  const double sure = (double)tiles_by([](const Stream& st) { return st.span; }) * P.inv_slots * (2.0 / kKeys) + 1.0;
  return sure < kWhole ? (int)sure * kKeys : kNever;
}

// Places of a stream's partial results: tiles in one chunk leave none.
__device__ __forceinline__ int parts_of(const Stream& st) { return st.chunks > 1 ? st.tiles * st.chunks : 0; }

// Longest chunk: of small tiles, the tiles' keys over the P.slots workgroups there are to
// fill. A stream's keys are then cut into equal chunks of at most that (chunk_keys). Every
// sum is of integers: each wave of the attention and the merge comes to the same numbers.
// The merge has the length from the attention (kFound), which leaves it behind the partial
// results.
enum class Tiles { kSmall, kBig, kFound };
template <Tiles TILES>
__device__ __forceinline__ Work work_of(const CacheAttnArgs& P, int lane) {
  constexpr int kNever = INT32_MAX / 2;
  Work w;
  w.mine = lane < P.streams ? stream_of(P, lane) : none();
  w.chunk = kNever;
  if (P.slots) {
    if constexpr (TILES == Tiles::kFound) {
      w.chunk = *P.chunk;
    } else {
      uint64_t total = (uint64_t)w.mine.tiles * (uint64_t)w.mine.mean;
      for (int s = lane + kWave; s < P.streams; s += kWave) {
        const Stream r = stream_of(P, s);
        total += (uint64_t)r.tiles * (uint64_t)r.mean;
      }
      total = wave_sum_u64(total);
      if constexpr (TILES == Tiles::kBig) {
        w.chunk = big_chunk(P, w, total, lane);
      } else {
        const double units = ceil((double)total * P.inv_slots * (1.0 / kKeys));
        if (units < kNever / kKeys / 8) w.chunk = max((int)units * kKeys, kMinChunk);
      }
      if (blockIdx.x == 0 && threadIdx.x == 0) *P.chunk = w.chunk;
    }
    w.mine.chunks = chunks_of(w.mine.span, w.chunk);
  }
  w.upto = wave_incl_scan_i32(w.mine.tiles * w.mine.chunks, lane);
  w.items = __builtin_amdgcn_readlane(w.upto, 63);
  for (int s0 = kWave; s0 < P.streams; s0 += kWave) {
    const Stream r = stream_in(P, s0 + lane, w.chunk);
    w.items += __builtin_amdgcn_readlane(wave_incl_scan_i32(r.tiles * r.chunks, lane), 63);
  }
  return w;
}

// Keys of a chunk of a stream that is cut into several: equal ones, in whole steps of the
// workgroup's waves (so a tile may need fewer than st.chunks).
__device__ __forceinline__ int chunk_keys(const CacheAttnArgs& P, const Stream& st) {
  const uint32_t unit = P.rows == kBigRows ? kKeys : kMinChunk;  // powers of two
  const uint32_t even = ((uint32_t)st.span + (uint32_t)st.chunks - 1) / (uint32_t)st.chunks;
  return (int)((even + unit - 1) & ~(unit - 1));
}

__device__ __forceinline__ Stream lane_stream(const Stream& r, int l) {
  return Stream{__builtin_amdgcn_readlane(r.q0, l),     __builtin_amdgcn_readlane(r.q_len, l), __builtin_amdgcn_readlane(r.p0, l),
                __builtin_amdgcn_readlane(r.kv_len, l), __builtin_amdgcn_readlane(r.tiles, l), __builtin_amdgcn_readlane(r.span, l),
                __builtin_amdgcn_readlane(r.mean, l),   __builtin_amdgcn_readlane(r.chunks, l)};
}

// Keys [lo, hi) that token i of a stream sees.
__device__ __forceinline__ void visible(const CacheAttnArgs& P, const Stream& st, int i, int& lo, int& hi) {
  const int p = st.p0 + i;
  int64_t end = st.kv_len;
  if (P.frame) end = p < 0 ? 0 : ((int64_t)divide(p, P.by_frame) + 1) * P.frame;
  hi = (int)min(end, (int64_t)st.kv_len);
  lo = P.window ? (int)max(end - P.window, (int64_t)0) : 0;
}

__device__ __forceinline__ Span tile_span(const CacheAttnArgs& P, const Stream& st, int tile) {
  const int row0 = tile << P.row_shift;
  const int row1 = min(row0 + P.rows, st.q_len * P.group) - 1;
  int lo, hi, lo1, hi1;
  visible(P, st, divide(row0, P.by_group), lo, hi);
  visible(P, st, divide(row1, P.by_group), lo1, hi1);
  Span r;
  r.lo = lo;
  r.begin = lo & ~(kKeys - 1);
  r.end = hi1 > lo ? hi1 : r.begin;  // no key at all: an empty span
  return r;
}

// A work item: a tile's chunk, keys [k0, k1).
struct Item {
  int stream;  // -1: no such item
  Stream st;
  int tile, n_chunks, k0, k1;
  int lo;      // first key that any row sees
  int part;    // its partial result's place, where the tile is in several chunks
};
__device__ __forceinline__ Item item_of(const CacheAttnArgs& P, const Work& w, int item, int lane) {
  Item r;
  r.stream = -1;
  int before = 0, parts = 0;  // items, and partial results, of the streams before the one that is found
  for (int s0 = 0; s0 < P.streams; s0 += kWave) {
    const Stream mine = s0 ? stream_in(P, s0 + lane, w.chunk) : w.mine;
    const int upto = s0 ? wave_incl_scan_i32(mine.tiles * mine.chunks, lane) : w.upto;
    const uint64_t past = __ballot(before + upto > item);
    if (past) {
      const int l = __builtin_ctzll(past);
      r.stream = s0 + l;
      r.st = lane_stream(mine, l);
      before += __builtin_amdgcn_readlane(upto, l) - r.st.tiles * r.st.chunks;
      if (r.st.chunks > 1) parts += __builtin_amdgcn_readlane(wave_incl_scan_i32(parts_of(mine), lane), l) - parts_of(r.st);
      break;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
    if (P.slots) parts += __builtin_amdgcn_readlane(wave_incl_scan_i32(parts_of(mine), lane), 63);
  }
  if (r.stream < 0) return r;
  const int at = item - before;
  int chunk = 0;
  r.tile = at;
  r.part = parts + at;
  if (r.st.chunks > 1) {
    r.tile = (int)((uint32_t)at / (uint32_t)r.st.chunks);
    chunk = at - r.tile * r.st.chunks;
  }
  // (sums past 32 bits, from starts that are not ascending)
  if (at < 0 || r.tile >= r.st.tiles || (r.st.chunks > 1 && (uint32_t)r.part >= (uint32_t)P.partials)) {
    r.stream = -1;
    return r;
  }
  const Span span = tile_span(P, r.st, r.tile);
  r.lo = span.lo;
  r.k0 = span.begin;
  r.k1 = span.end;
  r.n_chunks = 1;
  if (r.st.chunks > 1) {
    const int keys = chunk_keys(P, r.st);
    r.n_chunks = chunks_of(span.end - span.begin, keys);
    if (chunk >= r.n_chunks) {  // this tile sees fewer keys than the stream's widest
      r.stream = -1;
      return r;
    }
    r.k0 = (int)min((int64_t)span.begin + (int64_t)chunk * keys, (int64_t)span.end);
    r.k1 = (int)min((int64_t)r.k0 + keys, (int64_t)span.end);
  }
  return r;
}

// Two E4M3 codes (the low or high half of w) times a power of two, as bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t two_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}

__device__ __forceinline__ bf16x8 eight_bf16(uint32_t lo, uint32_t hi, float scale) {
  const uint4 r = make_uint4(two_bf16<false>(lo, scale), two_bf16<true>(lo, scale), two_bf16<false>(hi, scale),
                             two_bf16<true>(hi, scale));
  return __builtin_bit_cast(bf16x8, r);
}

// 2^e of a stored exponent, which lies in [kCacheExpMin, 120].
__device__ __forceinline__ float exp_of(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// The scale of V in its product.
__device__ __forceinline__ float value_exp(int e) { return exp_of(e - kValueDown); }

// What turns a row's sum of P V into O.
__device__ __forceinline__ float out_scale(float sum) { return sum > 0.f ? 1.0f / sum * kValueUp : 0.f; }

// max over lanes l, l^16, l^32, l^48, and the sum of them.
__device__ __forceinline__ float max4(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum4(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <bool STREAM, typename V>
__device__ __forceinline__ V load(const uint8_t* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  return *reinterpret_cast<const V*>(p);
}

// One tile of query rows against one chunk of its keys.
//
// Operand layouts (16x16x32 products; lane = 16 g + l). S^T = K Q^T: lane (g, l) holds key
// l of a 16-key group and channels 64 p + 16 g + 8 f .. + 7 at step 2 p + f, half of one
// 16-byte load; Q has the same order. S^T accumulator r is key 4 g + r, query row l: with
// two groups, the eight keys {4 g + r, 16 + 4 g + r} of a P^T operand. O^T += V^T P^T: lane
// (g, l) needs those eight keys of a channel, so it loads 8 bytes (channels 8 l .. 8 l + 7)
// of each of the eight rows; a byte permute of two rows' words puts two keys of one
// channel side by side, as the conversion takes them. Tile m of O^T holds channel 8 l + m,
// so a lane ends with eight consecutive channels of a query row per accumulator index.
template <int WAVES, bool STREAM>
__global__ __launch_bounds__(WAVES * kWave, 2) void cache_attn_kernel(CacheAttnArgs P) {
  __shared__ __align__(16) float ot[WAVES][kRows][kHeadDim + 4];
  __shared__ float ms[WAVES][kRows], ls[WAVES][kRows];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l = lane & 15;
  const int item = divide(blockIdx.x, P.by_heads);
  const int kh = (int)blockIdx.x - item * P.kv_heads;
  const Work work = work_of<Tiles::kSmall>(P, lane);
  const Item it = item_of(P, work, item, lane);
  if (it.stream < 0) return;
  const Stream& st = it.st;
  const int tile = it.tile, n_chunks = it.n_chunks, k0 = it.k0, k1 = it.k1;

  // This lane's query row.
  const int row = tile * kRows + l;
  const bool real = row < st.q_len * P.group;
  const int tok = real ? divide(row, P.by_group) : 0;
  const int qh = kh * P.group + (real ? row - tok * P.group : 0);
  int lo = 0, hi = 0;
  if (real) visible(P, st, tok, lo, hi);
  const uint16_t* qrow = static_cast<const uint16_t*>(P.Q) + (int64_t)(st.q0 + tok) * P.stride_n + (int64_t)qh * P.stride_h;
  bf16x8 qf[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    qf[s] = bf16x8{};
    if (real) qf[s] = *reinterpret_cast<const bf16x8*>(qrow + 64 * (s >> 1) + 16 * g + 8 * (s & 1));
  }
  // Keys that every real row sees, for which nothing is masked.
  int all_lo = real ? lo : 0, all_hi = real ? hi : INT32_MAX;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    all_lo = max(all_lo, __shfl_xor(all_lo, d));
    all_hi = min(all_hi, __shfl_xor(all_hi, d));
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);

  const int32_t* table = P.table + (int64_t)it.stream * P.width;
  const float c2 = P.scale * 1.44269504088896340736f;
  f32x4 o[8];
#pragma unroll
  for (int m = 0; m < 8; ++m) o[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mref = -1.0e30f, lsum = 0.f;

  // Pages of 16 keys, asked for a turn ahead. Keys outside [lo, k1) repeat the nearest one
  // inside: their pages may be no longer the stream's, and their codes anything.
  const const_i32* tab = (const const_i32*)table;
  int entry[4];
  auto look_up = [&](int base) {
#pragma unroll
    for (int t = 0; t < 4; ++t) entry[t] = tab[min(max(base + 16 * t, it.lo), k1 - 1) >> P.page_shift];
  };
  if (k0 + wave * kKeys < k1) look_up(k0 + wave * kKeys);
  for (int base = k0 + wave * kKeys; base < k1; base += WAVES * kKeys) {
    u32x4 kraw[4][2];
    u32x2 vraw[4][4];
    float ke[4], ve[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t at = (uint32_t)min(max(entry[t], 0), P.pages - 1) * (uint32_t)P.kv_heads + (uint32_t)kh;
      ke[t] = exp_of(((const const_i32*)P.k_exp)[at]);
      ve[t] = value_exp(((const const_i32*)P.v_exp)[at]);
      const uint8_t* kp = P.k8 + (uint64_t)at * (uint32_t)(P.page * kHeadDim);
      const uint8_t* vp = P.v8 + (uint64_t)at * (uint32_t)(P.page * kHeadDim);
      const int kr = min(max(base + 16 * t + l, it.lo), k1 - 1) & (P.page - 1);
      kraw[t][0] = load<STREAM, u32x4>(kp + kr * kHeadDim + 16 * g);
      kraw[t][1] = load<STREAM, u32x4>(kp + kr * kHeadDim + 64 + 16 * g);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int vr = min(max(base + 16 * t + 4 * g + r, it.lo), k1 - 1) & (P.page - 1);
        vraw[t][r] = load<STREAM, u32x2>(vp + vr * kHeadDim + 8 * l);
      }
    }
    look_up(base + WAVES * kKeys);
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_bf16(kraw[t][p].x, kraw[t][p].y, ke[t]), qf[2 * p], s[t], 0, 0, 0);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_bf16(kraw[t][p].z, kraw[t][p].w, ke[t]), qf[2 * p + 1], s[t], 0, 0, 0);
      }
    }
    if (base < all_lo || base + kKeys > min(all_hi, k1)) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = base + 16 * t + 4 * g + r;
          if (key < lo || key >= min(hi, k1)) s[t][r] = -INFINITY;
        }
      }
    }
    float mx = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[t][r]);
    }
    // Running reference in units of exp2's argument; it moves where a row's maximum has
    // passed it.
    mx = max4(mx) * c2;
    const float to = fmaxf(mref, mx);
    if (__ballot(to > mref)) {
      const float alpha = __builtin_amdgcn_exp2f(mref - to);
#pragma unroll
      for (int m = 0; m < 8; ++m) o[m] *= alpha;
      lsum *= alpha;
      mref = to;
    }
    bf16x8 pb[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x8 e;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        e[j] = __builtin_amdgcn_exp2f(fmaf(s[2 * b + (j >> 2)][j & 3], c2, -mref));
        lsum += e[j];
      }
      pb[b] = __builtin_convertvector(e, bf16x8);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        // byte pairs of rows (2 j, 2 j + 1): channels 4 w, 4 w + 1 and 4 w + 2, 4 w + 3
        uint32_t lo2[4], hi2[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x2 ra = vraw[2 * b + (j >> 1)][2 * (j & 1)], rb = vraw[2 * b + (j >> 1)][2 * (j & 1) + 1];
          const uint32_t a = w ? ra.y : ra.x, c = w ? rb.y : rb.x;
          lo2[j] = __builtin_amdgcn_perm(c, a, 0x05010400u);
          hi2[j] = __builtin_amdgcn_perm(c, a, 0x07030602u);
        }
        const float e0 = ve[2 * b], e1 = ve[2 * b + 1];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t(&src)[4] = q < 2 ? lo2 : hi2;
          uint4 f;
          if (q & 1)
            f = make_uint4(two_bf16<true>(src[0], e0), two_bf16<true>(src[1], e0), two_bf16<true>(src[2], e1), two_bf16<true>(src[3], e1));
          else
            f = make_uint4(two_bf16<false>(src[0], e0), two_bf16<false>(src[1], e0), two_bf16<false>(src[2], e1), two_bf16<false>(src[3], e1));
          const int m = 4 * w + q;
          o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), pb[b], o[m], 0, 0, 0);
        }
      }
    }
  }
  lsum = sum4(lsum);
  // The waves' results side by side: accumulator r of tile m is channel 8 (4 g + r) + m of row l.
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    *reinterpret_cast<f32x4*>(&ot[wave][l][32 * g + 8 * r]) = f32x4{o[0][r], o[1][r], o[2][r], o[3][r]};
    *reinterpret_cast<f32x4*>(&ot[wave][l][32 * g + 8 * r + 4]) = f32x4{o[4][r], o[5][r], o[6][r], o[7][r]};
  }
  if (g == 0) {
    ms[wave][l] = mref;
    ls[wave][l] = lsum;
  }
  __syncthreads();
  // Eight channels of a row per thread and turn.
  for (int piece = threadIdx.x; piece < 16 * kRows; piece += WAVES * kWave) {
    const int orow = piece >> 4, oc = 8 * (piece & 15);
    const int out_row = tile * kRows + orow;
    if (out_row >= st.q_len * P.group) break;
    float m = ms[0][orow];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, ms[w][orow]);
    float sum = 0.f;
    f32x8 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ms[w][orow] - m);
      sum += f * ls[w][orow];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += f * ot[w][orow][oc + e];
    }
    if (n_chunks == 1) {
      const float inv = out_scale(sum);
      const int out_tok = divide(out_row, P.by_group);
      const int oh = kh * P.group + out_row - out_tok * P.group;
      uint16_t* dst = static_cast<uint16_t*>(P.O) + (int64_t)(st.q0 + out_tok) * P.stride_n + (int64_t)oh * P.stride_h + oc;
      *reinterpret_cast<bf16x8*>(dst) = __builtin_convertvector(acc * inv, bf16x8);
    } else {
      float* part = P.partial + ((int64_t)it.part * P.kv_heads + kh) * (kRows * (kHeadDim + 2));
      *reinterpret_cast<f32x8*>(part + orow * kHeadDim + oc) = acc;
      if (oc == 0) {
        part[kRows * kHeadDim + orow] = m;
        part[kRows * kHeadDim + kRows + orow] = sum;
      }
    }
  }
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) i32x4 lds_i32x4;

template <int B, int E, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>{});
    static_for<B + 1, E>(f);
  }
}

__device__ __forceinline__ bf16x8 to_bf16x8(f32x4 a, f32x4 b) {
  return __builtin_convertvector(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8);
}

// s * c2 + negm, an exponential's argument, in the score's own register (sharing one
// temporary, each would wait for the exponential before it).
__device__ __forceinline__ float exp2_arg(float s, float c2, float negm) {
  asm("v_fma_f32 %0, %1, %0, %2" : "+v"(s) : "s"(c2), "v"(negm));
  return s;
}

// A large tile: 128 query rows, 32 per wave, against one chunk of its keys, 64 at a time.
//
// The 64 keys' codes are read once for the workgroup (two 16-byte pieces of K and of V per
// thread, two steps ahead) and go to LDS, where all four waves read them: K as it is, V as
// bf16 (a conversion is paid once for 128 rows). LDS holds two such steps. V's rows are 256
// bytes, its 16-byte chunk c of row r at c ^ (2 (r % 8) + r % 2), K's 128 bytes, chunk c at
// c ^ r % 8 ^ 4 (r % 2): reads and writes of both meet no bank twice.
//
// S^T = K Q^T on the E4M3 matrix unit, K's codes as they are: Q, bf16, has eight significant
// bits, which two codes of four hold, q = (high + low / 16) * 2^e with e from the row's
// largest element. high is q rounded, low what that left, times 16: exact down to 2^-13 of
// the row's maximum, and off by at most 2^-21 of it below (half of low's smallest step,
// 2^-14, against a maximum above 224). Two fp8 products take the time of one in bf16 and
// spare K's conversion and half of its LDS traffic: 4680 rows against 32,760 keys (40
// heads) 2713 -> 2499 us.
//
// O^T += V^T P^T in bf16: P would need two codes too, and their making is vector work, of
// which there is no less than of matrix work (36 + 16 products a wave and step of 16 passes
// and more against 32 exponentials, their arguments, maxima and conversions).
template <bool kOnePage>
__global__ __launch_bounds__(kWaves * kWave, 2) void cache_attn_big_kernel(CacheAttnArgs P) {
  constexpr int NT = 2;
  constexpr int NP = kOnePage ? 1 : 2;  // pages of a thread's rows in a step
  constexpr int kRow = 256;             // bytes of a row of V in LDS
  constexpr int kTile = kKeys * kRow;
  constexpr int kKTile = kKeys * kHeadDim;
  __shared__ __align__(16) unsigned char lds[2 * kTile + 2 * kKTile];  // V, V of the next step, K, K
  __shared__ __align__(16) int kscale[2][4];  // E8M0 scales of the 16-key groups of both steps
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l = lane & 15;

  // Work items head by head, in runs of which each is one XCD's (workgroups go to the XCDs in
  // turn): the tiles of a head read its keys out of one L2. Later tiles first: with causal
  // frames they see the most keys. Chunks, of which two of a CU run side by side and a head's
  // may be several XCDs', are dealt besides, every total / 64th of them and then the next, so
  // that neighbours, which are alike, do not all meet in one place: six streams of 558 to
  // 5760 keys (2727 rows, 12 / 4 heads) 93.2 -> 69.6 us, with windows 83.7 -> 67.7, one
  // stream of 14,040 keys causal by frame (5 heads) 134 either way.
  const Work work = work_of<Tiles::kBig>(P, lane);
  const int total = (int)min((int64_t)work.items, P.items_per_head);
  const int64_t all = (int64_t)total * P.kv_heads;
  const int64_t run = (all + kXcds - 1) / kXcds;
  const int64_t index = (blockIdx.x % kXcds) * run + blockIdx.x / kXcds;
  if (total <= 0 || blockIdx.x / kXcds >= run || index >= all) return;
  const int kh = (int)((uint32_t)index / (uint32_t)total);
  const int nth = (int)(index - (int64_t)kh * total);
  const int deal = nth & (kDeal - 1);
  const int dealt = deal * (total / kDeal) + min(deal, total & (kDeal - 1)) + nth / kDeal;
  const int item = total - 1 - (P.slots ? dealt : nth);
  const Item it = item_of(P, work, item, lane);
  if (it.stream < 0) return;
  const Stream& st = it.st;
  const int tile = it.tile, n_chunks = it.n_chunks, k0 = it.k0, k1 = it.k1;

  const int32_t* table = P.table + (int64_t)it.stream * P.width;
  const float c2 = P.scale * 1.44269504088896340736f;

  // This thread's two pieces of a step: 16 channels from 16 pc on of rows 8 wave + pr and
  // 32 more. The eight rows of a wave lie in one page. Eight neighbouring lanes take four
  // pieces of two rows of different parity, so that their writes to LDS meet all banks.
  const int pr = ((lane >> 2) & 1) | ((lane >> 4) << 1), pc = (lane & 3) | ((lane >> 1) & 4);
  uint4 kraw[2], vraw[2];
  int ke[NP];
  float ve[NP];
  // Pages and exponents go through the scalar unit: wave-uniform, and nothing here writes
  // them (kOnePage: pages of 64 tokens or more, a step lies in one; else a wave's eight rows
  // do). The page of a step is asked for three steps before it is multiplied, its exponents
  // and codes two steps. Keys outside [lo, k1) repeat the nearest one inside.
  const const_i32* tab = (const const_i32*)table;
  const const_i32* kexp = (const const_i32*)P.k_exp;
  const const_i32* vexp = (const const_i32*)P.v_exp;
  const uint32_t page_bytes = (uint32_t)P.page * kHeadDim;
  const uint32_t step_pages = (uint32_t)P.kv_heads;
  // Tile (page, head) of the pool that row `at` lies in, from its block table entry.
  auto entry_at = [&](int at) { return tab[min(max(at, it.lo), k1 - 1) >> P.page_shift]; };
  auto tile_of = [&](int entry) { return (uint32_t)min(max(entry, 0), P.pages - 1) * step_pages + (uint32_t)kh; };
  auto row_of = [&](int base, int p) { return base + (kOnePage ? 0 : 32 * p + 8 * wave); };
  const uint32_t lane_off = (uint32_t)((8 * wave + pr) * kHeadDim + 16 * pc);
  uint32_t tiles[NP];
  auto fetch = [&](int base) {
    const bool inside = base >= it.lo && base + kKeys <= k1;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint64_t at = (uint64_t)tiles[u % NP] * page_bytes;
      uint32_t off;
      if (inside)
        off = (uint32_t)(((kOnePage ? base + 32 * u : (base + 32 * u + 8 * wave)) & (P.page - 1)) * kHeadDim) +
              (kOnePage ? lane_off : (uint32_t)(pr * kHeadDim + 16 * pc));
      else
        off = (uint32_t)((min(max(base + 32 * u + 8 * wave + pr, it.lo), k1 - 1) & (P.page - 1)) * kHeadDim + 16 * pc);
      kraw[u] = *reinterpret_cast<const uint4*>(P.k8 + at + off);
      vraw[u] = *reinterpret_cast<const uint4*>(P.v8 + at + off);
    }
  };
  const int kx = pr ^ ((pr & 1) << 2), vx = 2 * pr + (pr & 1);  // swizzles of the thread's rows (32 rows on the same)
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)lds;
  // LDS addresses of a piece: K's 16 codes, the two halves of V's 16 channels.
  uint32_t wk = lds0 + 2 * kTile + (uint32_t)((8 * wave + pr) * kHeadDim) + 16 * (uint32_t)(pc ^ kx);
  uint32_t wv[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) wv[i] = lds0 + (uint32_t)((8 * wave + pr) * kRow) + 16 * (uint32_t)((2 * pc + i) ^ vx);
  // (Opaque: the compiler would move a piece's conversion, which both branches of a step
  // have, up to its load, and wait for it there.)
  auto stage = [&](int buf, int piece) {
    const int u = piece & 1;
    if (piece < 2) {
      *(lds_u32x4*)((lds_u8*)(uintptr_t)wk + buf * kKTile + 32 * u * kHeadDim) = u32x4{kraw[u].x, kraw[u].y, kraw[u].z, kraw[u].w};
      // rows 16 t .. + 15 are those of waves 2 t and 2 t + 1 (mod 4): wave 0 or 2 says their scale
      if (!kOnePage && !(wave & 1) && lane == 0) kscale[buf][2 * u + (wave >> 1)] = 127 + ke[u % NP];
    } else {
      asm volatile("" : "+v"(vraw[u].x), "+v"(vraw[u].y), "+v"(vraw[u].z), "+v"(vraw[u].w));
      *(lds_bf16x8*)((lds_u8*)(uintptr_t)wv[0] + buf * kTile + 32 * u * kRow) = eight_bf16(vraw[u].x, vraw[u].y, ve[u % NP]);
      *(lds_bf16x8*)((lds_u8*)(uintptr_t)wv[1] + buf * kTile + 32 * u * kRow) = eight_bf16(vraw[u].z, vraw[u].w, ve[u % NP]);
    }
  };

  // The first step's page and codes are on their way while the rows of Q are looked at.
  if (k0 < k1) {
#pragma unroll
    for (int p = 0; p < NP; ++p) tiles[p] = tile_of(entry_at(row_of(k0, p)));
    fetch(k0);
  }

  const int rows = st.q_len * P.group;
  const int row0 = tile * kBigRows + 32 * wave;
  int lo[NT], hi[NT];
  int wave_lo = INT32_MAX, wave_hi = 0, all_lo = 0, all_hi = INT32_MAX;
  i32x8 qh[NT], ql[NT];  // Q = (high + low codes) * 2^e
  int sh[NT], sl[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = row0 + 16 * nt + l;
    lo[nt] = hi[nt] = 0;
    bf16x8 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = bf16x8{};
    if (row < rows) {
      const int tok = divide(row, P.by_group);
      const int qh = kh * P.group + row - tok * P.group;
      visible(P, st, tok, lo[nt], hi[nt]);
      hi[nt] = max(min(hi[nt], k1), lo[nt]);
      const uint16_t* q = static_cast<const uint16_t*>(P.Q) + (int64_t)(st.q0 + tok) * P.stride_n + (int64_t)qh * P.stride_h;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const bf16x8*>(q + 64 * (i >> 1) + 16 * g + 8 * (i & 1));
      all_lo = max(all_lo, lo[nt]);
      all_hi = min(all_hi, hi[nt]);
      if (hi[nt] > lo[nt]) {
        wave_lo = min(wave_lo, lo[nt]);
        wave_hi = max(wave_hi, hi[nt]);
      }
    }
    // e as for a page: the smallest with amax <= 448 * 2^e
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf((float)x[i][j]));
    }
    const uint32_t bits = __float_as_uint(max4(amax));
    const int e = bits >> 23 ? max((int)(bits >> 23) - 135 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), kCacheExpMin) : kCacheExpMin;
    const float inv = __uint_as_float((uint32_t)(127 - min(e, 120)) << 23);
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      float f[4], back[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = (float)x[w >> 1][4 * (w & 1) + j] * inv;
      int h = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
      h = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], h, true);
      back[0] = __builtin_amdgcn_cvt_f32_fp8(h, 0);
      back[1] = __builtin_amdgcn_cvt_f32_fp8(h, 1);
      back[2] = __builtin_amdgcn_cvt_f32_fp8(h, 2);
      back[3] = __builtin_amdgcn_cvt_f32_fp8(h, 3);
      int r = __builtin_amdgcn_cvt_pk_fp8_f32(16.f * (f[0] - back[0]), 16.f * (f[1] - back[1]), 0, false);
      r = __builtin_amdgcn_cvt_pk_fp8_f32(16.f * (f[2] - back[2]), 16.f * (f[3] - back[3]), r, true);
      qh[nt][w] = h;
      ql[nt][w] = r;
    }
    sh[nt] = 127 + min(e, 120);
    sl[nt] = sh[nt] - 4;
  }
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    all_lo = max(all_lo, __shfl_xor(all_lo, d));
    all_hi = min(all_hi, __shfl_xor(all_hi, d));
    wave_lo = min(wave_lo, __shfl_xor(wave_lo, d));
    wave_hi = max(wave_hi, __shfl_xor(wave_hi, d));
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = min(__builtin_amdgcn_readfirstlane(all_hi), k1);
  wave_lo = __builtin_amdgcn_readfirstlane(wave_lo);
  wave_hi = min(__builtin_amdgcn_readfirstlane(wave_hi), k1);

  f32x4 o[8][NT], lsum[NT];
  float mrow[NT], thr[NT], negm[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) o[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    lsum[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    mrow[nt] = thr[nt] = -1.0e30f;
    negm[nt] = 0.f;
  }
  // The reference of a row moves when its maximum passes it by 2^8: P stays below 2^8,
  // where its relative rounding is the same, and O is rarely rescaled. The sums of P come
  // from the matrix unit too: a product with ones.
  const float move_ref = 8.0f / c2;
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.0f;

  uint32_t kaddr[2], vaddr[8];
  // K codes: row l of a 16-key group, 16-byte chunks g (channels 16 g ..) and 4 + g
#pragma unroll
  for (int i = 0; i < 2; ++i) kaddr[i] = lds0 + 2 * kTile + l * kHeadDim + 16 * ((4 * i + g) ^ (l & 7) ^ ((l & 1) << 2));
  {
    // transposing reads: lane 4 e + q of group g points at row 16 hf + 4 g + e, 8-byte chunk 4 mt + q
    const int vr = 4 * g + (l >> 2);
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) vaddr[mt] = lds0 + vr * kRow + 16 * ((2 * mt + ((l >> 1) & 1)) ^ (2 * (vr & 7) + (vr & 1))) + 8 * (l & 1);
  }

  int kcur = 0, knext = 0;  // kOnePage: E8M0 scales of the keys of this step and the next

  // (Opaque to the compiler, which would otherwise re-add the lanes' parts at every read.)
  asm volatile("" : "+v"(vaddr[0]), "+v"(vaddr[1]), "+v"(vaddr[2]), "+v"(vaddr[3]), "+v"(vaddr[4]), "+v"(vaddr[5]),
               "+v"(vaddr[6]), "+v"(vaddr[7]));
  asm volatile("" : "+v"(kaddr[0]), "+v"(kaddr[1]), "+v"(wk), "+v"(wv[0]), "+v"(wv[1]));

  // One step: S^T, under it the next step's codes into the other buffer and the loads of the
  // step after that, the softmax, O^T += V^T P^T. (The two buffers are two copies of the
  // code: their offsets are immediate.)
  auto step = [&](auto buf_c, int base) {
    constexpr int BUF = decltype(buf_c)::value;
    auto kfrag = [&](int t) {
      const i32x4 a = *(lds_i32x4*)((lds_u8*)(uintptr_t)kaddr[0] + BUF * kKTile + t * 16 * kHeadDim);
      const i32x4 b = *(lds_i32x4*)((lds_u8*)(uintptr_t)kaddr[1] + BUF * kKTile + t * 16 * kHeadDim);
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto vfrag = [&](int kk, int mt) {
      lds_u8* at = (lds_u8*)(uintptr_t)vaddr[mt] + BUF * kTile + kk * 32 * kRow;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * kRow));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const bool act = base < wave_hi && base + kKeys > wave_lo;  // wave-uniform
    f32x4 s[4][NT];
    if (act) {
      i32x4 ks = {0, 0, 0, 0};
      if constexpr (!kOnePage) ks = *(lds_i32x4*)kscale[BUF];
      i32x8 ka[4];
      ka[0] = kfrag(0);
      ka[1] = kfrag(1);
      __builtin_amdgcn_s_setprio(2);
      // Two key groups against two query tiles, high then low codes of Q: four independent
      // chains alternate.
      static_for<0, 4>([&](auto u_c) {
        constexpr int u = decltype(u_c)::value;
        constexpr int t0 = 2 * (u >> 1);
        if constexpr (u == 0) {
          ka[2] = kfrag(2);
          ka[3] = kfrag(3);
        }
#pragma unroll
        for (int t = t0; t < t0 + 2; ++t) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const int sa = kOnePage ? kcur : ks[t];
            if (u % 2 == 0)
              s[t][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka[t], qh[nt], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, sa, 0, sh[nt]);
            else
              s[t][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka[t], ql[nt], s[t][nt], 0, 0, 0, sa, 0, sl[nt]);
          }
        }
        stage(BUF ^ 1, u);
        __builtin_amdgcn_sched_barrier(0);
      });
      __builtin_amdgcn_s_setprio(0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) stage(BUF ^ 1, i);
    }
    fetch(base + 2 * kKeys);  // (behind the last step: the last key again)
    int k_exp[NP], v_exp[NP], entry[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      k_exp[p] = kexp[tiles[p]];
      v_exp[p] = vexp[tiles[p]];
      entry[p] = entry_at(row_of(base + 3 * kKeys, p));
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 pb[2][NT];
    if (act) {
      if (base < all_lo || base + kKeys > all_hi) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint32_t past = (uint32_t)(base + 4 * g - lo[nt]) + (16 * t + r);
              if (past >= (uint32_t)(hi[nt] - lo[nt])) s[t][nt][r] = -INFINITY;
            }
          }
        }
      }
      float mx[NT];
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mx[nt] = s[0][nt][0];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
          for (int r = 0; r < 4; ++r) mx[nt] = fmaxf(mx[nt], s[t][nt][r]);
        }
        over |= mx[nt] > thr[nt];
      }
      if (__ballot(over)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float rmx = max4(mx[nt]);
          const bool grow = rmx > thr[nt];
          const float to = grow ? rmx : mrow[nt];
          const float alpha = grow ? __builtin_amdgcn_exp2f((mrow[nt] - to) * c2) : 1.0f;
          mrow[nt] = to;
          if (__ballot(grow)) {
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) o[mt][nt] *= alpha;
            lsum[nt] *= alpha;
            thr[nt] = mrow[nt] + move_ref;
            negm[nt] = -mrow[nt] * c2;
          }
        }
      }
      // The exponentials of the first 32 keys; those of the second come under the products
      // of the first.
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[t][nt][r] = __builtin_amdgcn_exp2f(exp2_arg(s[t][nt][r], c2, negm[nt]));
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) pb[0][nt] = to_bf16x8(s[0][nt], s[1][nt]);
    }
    // The scalars have come; no LDS read is in flight that this wait would hold up.
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      if (kOnePage) {
        kcur = knext;
        knext = 127 + k_exp[p];
      }
      ke[p] = k_exp[p];
      ve[p] = value_exp(v_exp[p]);
      tiles[p] = tile_of(entry[p]);
    }
    if (act) {
      // O^T += V^T P^T
      bf16x8 vq[3];
      vq[0] = vfrag(0, 0);
      vq[1] = vfrag(0, 1);
      __builtin_amdgcn_s_setprio(1);
      static_for<0, 16>([&](auto u_c) {
        constexpr int u = decltype(u_c)::value;
        constexpr int kk = u >> 3, mt = u & 7;
        if constexpr (u + 2 < 16) vq[(u + 2) % 3] = vfrag((u + 2) >> 3, (u + 2) & 7);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          o[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vq[u % 3], pb[kk][nt], o[mt][nt], 0, 0, 0);
        if constexpr (mt == 7) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            lsum[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[kk][nt], lsum[nt], 0, 0, 0);
        }
        if constexpr (u < 8) {
          constexpr int t = 2 + (u >> 2), r = u & 3;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[t][nt][r] = __builtin_amdgcn_exp2f(exp2_arg(s[t][nt][r], c2, negm[nt]));
          if constexpr (u == 7) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) pb[1][nt] = to_bf16x8(s[2][nt], s[3][nt]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      __builtin_amdgcn_s_setprio(0);
    }
    __syncthreads();
  };

  if (k0 < k1) {
    uint32_t next[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      ke[p] = kexp[tiles[p]];
      if (kOnePage) kcur = 127 + ke[p];
      ve[p] = value_exp(vexp[tiles[p]]);
      tiles[p] = tile_of(entry_at(row_of(k0 + kKeys, p)));
      next[p] = tile_of(entry_at(row_of(k0 + 2 * kKeys, p)));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) stage(0, i);
    fetch(k0 + kKeys);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      ke[p] = kexp[tiles[p]];
      if (kOnePage) knext = 127 + ke[p];
      ve[p] = value_exp(vexp[tiles[p]]);
      tiles[p] = next[p];
    }
    __syncthreads();
    for (int base = k0;;) {
      step(std::integral_constant<int, 0>{}, base);
      if ((base += kKeys) >= k1) break;
      step(std::integral_constant<int, 1>{}, base);
      if ((base += kKeys) >= k1) break;
    }
  }

  // Accumulator r of (mt, nt): channel 16 mt + 4 g + r of row 16 nt + l.
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = row0 + 16 * nt + l;
    if (row >= rows) continue;
    if (n_chunks == 1) {
      const float inv = out_scale(lsum[nt][0]);
      const int tok = divide(row, P.by_group);
      const int qh = kh * P.group + row - tok * P.group;
      uint16_t* out = static_cast<uint16_t*>(P.O) + (int64_t)(st.q0 + tok) * P.stride_n + (int64_t)qh * P.stride_h + 4 * g;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
        *reinterpret_cast<bf16x4*>(out + 16 * mt) = __builtin_convertvector(o[mt][nt] * inv, bf16x4);
    } else {
      float* part = P.partial + ((int64_t)it.part * P.kv_heads + kh) * (kBigRows * (kHeadDim + 2));
      const int r = row - tile * kBigRows;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) *reinterpret_cast<f32x4*>(part + r * kHeadDim + 16 * mt + 4 * g) = o[mt][nt];
      if (g == 0) {
        part[kBigRows * kHeadDim + r] = mrow[nt] * c2;
        part[kBigRows * kHeadDim + kBigRows + r] = lsum[nt][0];
      }
    }
  }
}

// All-lane reduction by a commutative operation, the same bits in every lane.
template <typename Op>
__device__ __forceinline__ float wave_reduce(float v, Op op) {
  auto with = [&](uint32_t x) { v = op(v, __uint_as_float(x)); };
  with(dpp_move<0xB1>(__float_as_uint(v)));
  with(dpp_move<0x4E>(__float_as_uint(v)));
  with(dpp_move<0x141>(__float_as_uint(v)));
  with(dpp_move<0x140>(__float_as_uint(v)));
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// ROWS rows of a tile from row r on: the partial results of its chunks [c_begin, c_end), in
// chunk order. Lane c has the reference and sum of chunk c (64 chunks at a time), then the
// chunks' rows are loaded DEPTH chunks at a time for all ROWS rows, all loads independent;
// lane i has channels 2 i and 2 i + 1. out(i, reference, sum, value) is called for every row.
template <int ROWS, int DEPTH, typename F>
__device__ __forceinline__ void merge_rows(const float* base, int64_t step, int tile_rows, int c_begin, int c_end, int r, int lane, F&& out) {
  float m[ROWS], sum[ROWS];
  float2 acc[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    m[i] = -1.0e30f;
    sum[i] = 0.f;
    acc[i] = make_float2(0.f, 0.f);
  }
  for (int c0 = c_begin; c0 < c_end; c0 += kWave) {
    const int n = min(c_end - c0, kWave);
    const float* at = base + (int64_t)(c0 + min(lane, n - 1)) * step + tile_rows * kHeadDim + r;
    float w[ROWS], pl[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      w[i] = at[i];
      pl[i] = at[tile_rows + i];
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float to = fmaxf(wave_reduce(w[i], [](float a, float b) { return fmaxf(a, b); }), m[i]);
      const float keep = __builtin_amdgcn_exp2f(m[i] - to);
      w[i] = lane < n ? __builtin_amdgcn_exp2f(w[i] - to) : 0.f;
      sum[i] = sum[i] * keep + wave_reduce(w[i] * pl[i], [](float a, float b) { return a + b; });
      acc[i].x *= keep;
      acc[i].y *= keep;
      m[i] = to;
    }
    const float* row = base + (int64_t)c0 * step + (int64_t)r * kHeadDim + 2 * lane;
    for (int c = 0; c < n; c += DEPTH) {
      float2 v[DEPTH][ROWS];
#pragma unroll
      for (int j = 0; j < DEPTH; ++j) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
          v[j][i] = *reinterpret_cast<const float2*>(row + (int64_t)min(c + j, n - 1) * step + i * kHeadDim);
      }
#pragma unroll
      for (int j = 0; j < DEPTH; ++j) {
        if (c + j < n) {
#pragma unroll
          for (int i = 0; i < ROWS; ++i) {
            const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w[i]), c + j));
            acc[i].x = fmaf(f, v[j][i].x, acc[i].x);
            acc[i].y = fmaf(f, v[j][i].y, acc[i].y);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) out(i, m[i], sum[i], acc[i]);
}

// 16 rows of a tile per workgroup, four per wave at once. Where there are few rows and many
// chunks (single tokens), the waves share the chunks instead and meet in LDS: 71,900 keys
// of one K/V head, four query heads: 66 us with each wave on rows of its own, 29 so.
__global__ __launch_bounds__(256) void cache_combine_kernel(CacheAttnArgs P) {
  __shared__ float2 acc_s[4][4][kWave];
  __shared__ float m_s[4][4], sum_s[4][4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part_shift = P.row_shift - 4;
  const int part = blockIdx.x & ((1 << part_shift) - 1);
  const int tile_id = divide(blockIdx.x >> part_shift, P.by_heads);
  const int kh = (int)(blockIdx.x >> part_shift) - tile_id * P.kv_heads;
  const Work work = work_of<Tiles::kFound>(P, lane);
  // the stream that holds tile tile_id, its first tile and its first partial result
  int tiles = 0, part0 = 0, stream = -1;
  Stream st;
  for (int s0 = 0; s0 < P.streams; s0 += kWave) {
    const Stream mine = s0 ? stream_in(P, s0 + lane, work.chunk) : work.mine;
    const int upto = wave_incl_scan_i32(parts_of(mine), lane);
    const int tiles_upto = wave_incl_scan_i32(mine.tiles, lane);
    const uint64_t past = __ballot(tiles + tiles_upto > tile_id);
    if (past) {
      const int l = __builtin_ctzll(past);
      stream = s0 + l;
      st = lane_stream(mine, l);
      tiles += __builtin_amdgcn_readlane(tiles_upto, l) - st.tiles;
      part0 += __builtin_amdgcn_readlane(upto, l) - parts_of(st);
      break;
    }
    tiles += __builtin_amdgcn_readlane(tiles_upto, 63);
    part0 += __builtin_amdgcn_readlane(upto, 63);
  }
  if (stream < 0 || st.chunks == 1) return;
  const int tile = tile_id - tiles;
  const Span span = tile_span(P, st, tile);
  const int n_chunks = chunks_of(span.end - span.begin, chunk_keys(P, st));
  if (n_chunks == 1) return;
  const int64_t first = (int64_t)part0 + (int64_t)tile * st.chunks;
  // (sums past 32 bits, from starts that are not ascending)
  if (tile < 0 || tile >= st.tiles || part0 < 0 || first + n_chunks > P.partials) return;
  const int64_t size = P.rows * (kHeadDim + 2);
  const float* base = P.partial + (first * P.kv_heads + kh) * size;
  const int64_t step = P.kv_heads * size;
  const int rows = st.q_len * P.group;
  auto put = [&](int r, float sum, float2 o) {
    const int row = tile * P.rows + r;
    if (row >= rows) return;
    const float inv = out_scale(sum);
    const int tok = divide(row, P.by_group);
    const int qh = kh * P.group + row - tok * P.group;
    bf16x2 v;
    v[0] = (__bf16)(o.x * inv);
    v[1] = (__bf16)(o.y * inv);
    *reinterpret_cast<bf16x2*>(static_cast<uint16_t*>(P.O) + (int64_t)(st.q0 + tok) * P.stride_n + (int64_t)qh * P.stride_h + 2 * lane) = v;
  };
  const int r0 = 16 * part;
  const int left = rows - (tile * P.rows + r0);  // real rows from the part's first on
  if (left > 8 || n_chunks <= 8) {
    const int r = r0 + 4 * wave;
    if (left > 4 * wave)
      merge_rows<4, 4>(base, step, P.rows, 0, n_chunks, r, lane, [&](int i, float, float sum, float2 o) { put(r + i, sum, o); });
    return;
  }
  const int share = (n_chunks + 3) / 4;
  for (int g0 = 0; g0 < left; g0 += 4) {
    merge_rows<4, 4>(base, step, P.rows, min(wave * share, n_chunks), min((wave + 1) * share, n_chunks), r0 + g0, lane,
                     [&](int i, float m, float sum, float2 o) {
                       acc_s[wave][i][lane] = o;
                       if (lane == 0) {
                         m_s[wave][i] = m;
                         sum_s[wave][i] = sum;
                       }
                     });
    __syncthreads();
    float m = m_s[0][wave];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, m_s[w][wave]);
    float sum = 0.f;
    float2 o = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(m_s[w][wave] - m);
      sum = fmaf(f, sum_s[w][wave], sum);
      o.x = fmaf(f, acc_s[w][wave][lane].x, o.x);
      o.y = fmaf(f, acc_s[w][wave][lane].y, o.y);
    }
    put(r0 + g0 + wave, sum, o);
    __syncthreads();
  }
}

// Workgroups per K/V head to split for (large tiles: at most; 0: not split), and the items
// there can be.
struct Sizes {
  bool big;
  int rows, slots;
  int64_t tiles, items;
  int64_t partials;  // partial results that there are at most (below 2^31, as the items)
  int64_t keys;  // that any tile sees, at most
};
// Streams of few keys stay in one workgroup a tile: up to four turns of eight waves.
bool few_keys(int64_t most_keys) { return most_keys <= 2048; }

int64_t tiles_of(int64_t tokens, int group, int rows, int streams) {
  return tokens * group / rows + streams;  // at most one partly filled tile a stream
}

// window, frame: 0 where they are not known.
Sizes sizes_of(bool big, int tokens, int heads, int kv_heads, int streams, int64_t most_keys, int window, int frame) {
  const int group = heads / kv_heads;
  Sizes r;
  r.big = big;
  r.rows = big ? kBigRows : kRows;
  r.tiles = tiles_of(tokens, group, r.rows, streams);
  r.keys = most_keys;
  if (window) r.keys = std::min(most_keys, (int64_t)window + 2 * (int64_t)frame + r.rows + kKeys);
  // Chunks do not pay for a second launch that merges them where keys are few (large tiles:
  // ten steps), nor where the tiles, not split, fill two rounds.
  const int64_t full = ((int64_t)tokens * group + r.rows - 1) / r.rows;  // tiles if the rows fill them
  if (big) {
    const int64_t places = std::max(1, (full * kv_heads > kBigSlots ? kBigRounds : 2) * kBigSlots / kv_heads);
    const int64_t most = r.tiles * std::min<int64_t>(kMostChunks, (r.keys + kMinChunk - 1) / kMinChunk);
    r.slots = r.keys <= 10 * kKeys || 2 * full > places ? 0 : (int)std::min(places, most);
    // big_chunk splits into no more than r.slots; tiles of one stream are split all or not at all
    r.items = streams > 1 ? r.tiles + r.slots : std::max(r.tiles, (int64_t)r.slots);
    r.partials = r.slots;
  } else {
    const int round = std::max(1, kCacheSlots / kv_heads);
    r.slots = few_keys(r.keys) || full >= 2 * (int64_t)round ? 0 : (full > round ? 2 : 1) * round;
    r.items = r.tiles + r.slots;  // the sum of chunks_of(span)
    r.partials = r.items;
  }
  return r;
}

// One small tile per stream reads the keys once, straight into registers. More rows share
// the keys' conversion through LDS in large tiles, unless there is so little to do that a
// large tile's longer way in (some 13 us against 5 on an idle device) decides. In turns of
// 16 rows x 64 keys: streams of up to 2048 keys 1170 / 3800 / 10240 / 12250 turns 10.5 /
// 11.3 / 23.5 / 23.0 us in small tiles, 13.2 / 13.4 / 29.8 / 32.7 in large ones; longer
// streams, whose merge small tiles make longer, 441 / 3384 / 8192 / 12384 turns 14.9 / 25.2
// / 34.1 / 55.8 against 19.8 / 27.6 / 29.5 / 38.1. (Keys are those that the table's width and
// the window allow: the lengths are not known here.)
constexpr int kFewTurns = 16384, kManyTurns = 4096;
bool is_big(int tokens, int heads, int kv_heads, int streams, int max_q, int64_t most_keys, int window, int frame) {
  const int group = heads / kv_heads;
  if ((int64_t)max_q * group <= kRows) return false;
  const int64_t keys = sizes_of(false, tokens, heads, kv_heads, streams, most_keys, window, frame).keys;
  const double turns = (double)tiles_of(tokens, group, kRows, streams) * kv_heads * (double)((keys + kKeys - 1) / kKeys);
  return turns > (few_keys(keys) ? kFewTurns : kManyTurns);
}

}  // namespace

// Both queries hold for either kernel, as a window, which they are not told, may change the
// choice (but for small tiles past kFewTurns, which none makes).
bool cache_attn_fits(int tokens, int heads, int kv_heads, int streams, int max_q, int64_t most_keys) {
  const bool may_be_big = (int64_t)max_q * (heads / kv_heads) > kRows;
  for (int big = 0; big <= (may_be_big ? 1 : 0); ++big) {
    const Sizes z = sizes_of(big, tokens, heads, kv_heads, streams, most_keys, 0, 0);
    if (!big && may_be_big && z.tiles * kv_heads > kFewTurns) continue;
    const int64_t merges = z.slots ? z.tiles * (z.rows / 16) : 0;
    if (std::max(z.items, merges) * kv_heads + kXcds > kCacheWorkgroups) return false;
  }
  return true;
}

static size_t partial_floats(const Sizes& z, int kv_heads) { return (size_t)z.partials * kv_heads * z.rows * (kHeadDim + 2); }

size_t cache_attn_workspace_bytes(int tokens, int heads, int kv_heads, int streams, int max_q, int64_t most_keys) {
  size_t most = 0;
  for (int big = 0; big <= ((int64_t)max_q * (heads / kv_heads) > kRows ? 1 : 0); ++big) {
    const Sizes z = sizes_of(big, tokens, heads, kv_heads, streams, most_keys, 0, 0);
    if (z.slots) most = std::max(most, (partial_floats(z, kv_heads) + 1) * sizeof(float));
  }
  return most;
}

namespace {
// n / d = n * mul >> shift for 0 <= n < 2^31: mul = ceil(2^shift / d), shift = 31 + ceil(log2 d)
// (its error, below n / 2^shift, cannot reach the next multiple of 1 / d).
Divisor divisor_of(int d) {
  int up = 0;
  while (((int64_t)1 << up) < d) ++up;
  const int shift = 31 + up;
  return {(uint32_t)((((uint64_t)1 << shift) + (uint32_t)d - 1) / (uint32_t)d), shift};
}

template <int WAVES, bool STREAM>
void launch_small(const CacheAttnArgs& a) {
  cache_attn_kernel<WAVES, STREAM><<<(unsigned)a.items, WAVES * kWave, 0, a.stream>>>(a);
}
}  // namespace

hipError_t launch_cache_attn(CacheAttnArgs a) {
  (void)hipGetLastError();
  if (a.tokens == 0 || a.heads == 0 || a.streams == 0) return hipSuccess;
  a.group = a.heads / a.kv_heads;
  const int64_t most_keys = (int64_t)a.width * a.page;
  const bool big = is_big(a.tokens, a.heads, a.kv_heads, a.streams, a.max_q, most_keys, a.window, a.frame);
  const Sizes z = sizes_of(big, a.tokens, a.heads, a.kv_heads, a.streams, most_keys, a.window, a.frame);
  a.rows = z.rows;
  a.row_shift = z.big ? 7 : 4;
  a.ramp = z.big && a.frame;
  a.most_keys = (int)std::min<int64_t>(z.keys, INT32_MAX);
  a.by_group = divisor_of(a.group);
  a.by_heads = divisor_of(a.kv_heads);
  a.by_frame = divisor_of(std::max(a.frame, 1));
  a.items_per_head = z.items;
  a.partials = (int)z.partials;
  a.slots = z.slots;
  a.inv_slots = z.slots ? 1.0 / z.slots : 0.0;
  a.items = z.items * a.kv_heads;
  a.chunk = z.slots ? reinterpret_cast<int32_t*>(a.partial + partial_floats(z, a.kv_heads)) : nullptr;
  // Small tiles of few keys: as many waves a tile as the chip has room for (twelve a CU) when
  // all tiles run at once. Of many keys: four, and codes that no other workgroup of
  // the call reads go past the caches (64 ragged streams of up to 16000 keys, 8 heads: 165 ->
  // 154 us; 111,600 keys of 40 heads: 207 -> 190, 6.0 TB/s).
  const unsigned grid = (unsigned)((a.items + kXcds - 1) / kXcds * kXcds);
  if (z.big && a.page >= kKeys)
    cache_attn_big_kernel<true><<<grid, kWaves * kWave, 0, a.stream>>>(a);
  else if (z.big)
    cache_attn_big_kernel<false><<<grid, kWaves * kWave, 0, a.stream>>>(a);
  else if (few_keys(z.keys) && a.items <= 384)
    launch_small<8, false>(a);
  else if (few_keys(z.keys) && a.items > 1536)
    launch_small<1, false>(a);
  else if (few_keys(z.keys) && a.items > 768)
    launch_small<2, false>(a);
  else if (few_keys(z.keys))
    launch_small<4, false>(a);
  else if ((int64_t)a.max_q * a.group > kRows)  // several tiles read the same keys
    launch_small<4, false>(a);
  else
    launch_small<4, true>(a);
  if (z.slots) cache_combine_kernel<<<(unsigned)(z.tiles * a.kv_heads * (z.rows / 16)), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

}  // namespace fva
