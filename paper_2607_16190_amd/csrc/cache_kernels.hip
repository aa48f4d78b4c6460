// The paged 8-bit K/V cache (gfx950): pages from request lengths, and the store.
//
// A page holds `page` tokens of every K/V head: codes uint8 [pages, heads, page, 128]
// (OCP E4M3) for K and for V, and one power-of-two scale 2^e per (page, head), e int32
// [pages, heads]. A stream's tokens lie in the pages its block table row names.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "fva_common.h"
#include "fva_geometry.h"
#include "fva_internal.h"

namespace fva {
namespace {

constexpr int kPlanThreads = 256;

// Exclusive prefix sums over the workgroup of three values a thread holds, and the totals.
// (64 bits: lengths come from device memory, and no sum of them may turn negative.)
struct Three {
  uint64_t a, b, c;
};
__device__ __forceinline__ Three block_exclusive(Three v, Three& total, uint64_t (&part)[3][kPlanThreads / kWave]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Three in = {wave_incl_scan_u64(v.a, lane), wave_incl_scan_u64(v.b, lane), wave_incl_scan_u64(v.c, lane)};
  if (lane == 63) {
    part[0][wave] = in.a;
    part[1][wave] = in.b;
    part[2][wave] = in.c;
  }
  __syncthreads();
  Three below = {0, 0, 0};
  total = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    if (w < wave) below = {below.a + part[0][w], below.b + part[1][w], below.c + part[2][w]};
    total = {total.a + part[0][w], total.b + part[1][w], total.c + part[2][w]};
  }
  return {below.a + in.a - v.a, below.b + in.b - v.b, below.c + in.c - v.c};
}

__device__ __forceinline__ int to_int(uint64_t v) { return (int)min(v, (uint64_t)INT32_MAX); }

// Largest s in [0, n) with start[s] <= x, of ascending start with start[0] = 0 (streams
// of no width share a start; the last of them is found, which is the one that holds x).
__device__ __forceinline__ int find_stream(const int* start, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Block tables, slots and positions. Every workgroup forms the prefix sums over the
// streams by itself (a few loads per thread: cheaper than a second launch) and writes its
// share of the table entries and token rows; nothing that one workgroup writes is read
// by another: popped ring entries lie in [head, head + count), pushed ones behind, new
// table entries behind a row's old ones, and the lengths and the ring state go to buffers
// of their own.
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(PlanArgs P) {
  __shared__ int q_start[kPlanStreams + 1];   // first token row of each stream
  __shared__ int first[kPlanStreams + 1];     // pages popped before it
  __shared__ int behind[kPlanStreams + 1];    // pages pushed before it
  __shared__ int held_s[kPlanStreams];        // tokens held, or -1 - tokens held where the stream is refused
  __shared__ uint64_t part[3][kPlanThreads / kWave];
  __shared__ int refused_s;
  const int S = P.streams;
  const int cap = P.ring_size;
  const int per = (S + kPlanThreads - 1) / kPlanThreads;
  const int s0 = min((int)threadIdx.x * per, S), s1 = min(s0 + per, S);
  int count = min(max(P.state[1], 0), cap);
  int head = P.state[0] % cap;
  head += head < 0 ? cap : 0;
  if (threadIdx.x == 0) refused_s = 0;

  const int most = (int)min((int64_t)P.width * P.page, (int64_t)INT32_MAX);  // tokens a table row can hold
  auto pages_of = [&](int tokens) { return (tokens + P.page - 1) / P.page; };
  // (tokens added, pages popped, pages pushed) of stream s; wide: the row has room
  auto wants = [&](int s, int& held, bool& wide) {
    held = min(max(P.held[s], 0), most);
    const int add = P.fresh[s];
    const int now = pages_of(held);
    if (add < 0) {
      wide = true;
      return Three{0, 0, (uint64_t)now};
    }
    wide = add <= most - held;
    return Three{(uint64_t)add, wide ? (uint64_t)(pages_of(held + add) - now) : 0, 0};
  };
  Three mine = {0, 0, 0}, total;
  for (int s = s0; s < s1; ++s) {
    int held;
    bool wide;
    const Three w = wants(s, held, wide);
    mine = {mine.a + w.a, mine.b + w.b, mine.c + w.c};
  }
  Three at = block_exclusive(mine, total, part);
  int refused = 0;
  for (int s = s0; s < s1; ++s) {
    int held;
    bool wide;
    const Three w = wants(s, held, wide);
    const bool fits = wide && (w.b == 0 || at.b + w.b <= (uint64_t)count);
    q_start[s] = to_int(at.a);
    // refused pops lie behind the granted ones: the search below never reaches them
    first[s] = (int)min(at.b, (uint64_t)count);
    behind[s] = to_int(at.c);
    held_s[s] = fits ? held : -1 - held;
    refused += fits ? 0 : 1;
    if (blockIdx.x == 0) {
      P.q_start[s] = to_int(at.a);
      P.kv_len[s] = P.fresh[s] < 0 ? 0 : (fits ? held + (int)w.a : held);
    }
    at = {at.a + w.a, at.b + w.b, at.c + w.c};
  }
  if (refused) atomicAdd(&refused_s, refused);
  if (threadIdx.x == 0) {
    q_start[S] = to_int(total.a);
    behind[S] = to_int(total.c);
  }
  __syncthreads();
  // Pages granted: the pops of streams up to the first that did not fit.
  int taken = 0;
  {
    uint64_t t = 0;
    for (int s = s0; s < s1; ++s) {
      int held;
      bool wide;
      const Three w = wants(s, held, wide);
      if (held_s[s] >= 0) t += w.b;
    }
    Three sum;
    __syncthreads();
    (void)block_exclusive({t, 0, 0}, sum, part);
    taken = (int)sum.a;  // at most count
  }
  const int pushed = (int)min(total.c, (uint64_t)(cap - count));
  const int rows = to_int(total.a);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    P.q_start[S] = rows;
    P.state_out[0] = (int)(((int64_t)head + taken) % cap);
    P.state_out[1] = count - taken + pushed;
    P.state_out[2] = refused_s;
  }
  // (Unsigned: the step past the last of up to 2^31 - 1 rows or pages is no negative index.)
  const uint32_t step = gridDim.x * kPlanThreads;
  const uint32_t i0 = blockIdx.x * kPlanThreads + threadIdx.x;
  for (uint32_t i = i0; i < (uint32_t)taken; i += step) {
    const int s = find_stream(first, S, (int)i);
    const int col = pages_of(held_s[s]) + (int)i - first[s];
    P.table[(int64_t)s * P.width + col] = P.ring[((int64_t)head + i) % cap];
  }
  for (uint32_t i = i0; i < (uint32_t)pushed; i += step) {
    const int s = find_stream(behind, S, (int)i);
    P.ring[((int64_t)head + count + i) % cap] = P.table[(int64_t)s * P.width + (int)i - behind[s]];
  }
  for (uint32_t r = i0; r < (uint32_t)P.tokens; r += step) {
    int slot = -1, id = -1;
    if (r < (uint32_t)rows) {
      const int s = find_stream(q_start, S, (int)r);
      const int held = held_s[s];
      if (held >= 0) {
        id = held + (int)r - q_start[s];
        const int col = id / P.page, now = pages_of(held);
        const int page = col < now ? P.table[(int64_t)s * P.width + col] : P.ring[((int64_t)head + first[s] + col - now) % cap];
        slot = page < 0 ? -1 : page * P.page + id % P.page;
      }
    }
    P.slots[r] = slot;
    P.ids[r] = id;
  }
}

// ---- store ------------------------------------------------------------------

// Smallest e >= kCacheExpMin with amax <= 448 * 2^e: amax = 1.f * 2^(E - 127), and
// 448 = 1.75 * 2^8, so e = E - 135 where 1.f <= 1.75, else E - 134.
__device__ __forceinline__ int cache_exponent(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int E = (int)(bits >> 23);
  const int e = E - 135 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return E == 0 ? kCacheExpMin : max(e, kCacheExpMin);
}

// The largest of the wave's non-negative values.
__device__ __forceinline__ float wave_max_abs(float v) {
  uint32_t b = __float_as_uint(v);
  b = max(b, dpp_move<0xB1>(b));
  b = max(b, dpp_move<0x4E>(b));
  b = max(b, dpp_move<0x141>(b));
  b = max(b, dpp_move<0x140>(b));
  const auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  b = max(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float(max(q[0], q[1]));
}

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  // Inputs are at most 448 in magnitude except infinities, which become 448 (the cache
  // holds no NaN: a masked key's V is multiplied by zero).
  constexpr float kTop = 448.f;
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(a, -kTop, kTop), __builtin_amdgcn_fmed3f(b, -kTop, kTop), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(c, -kTop, kTop), __builtin_amdgcn_fmed3f(d, -kTop, kTop), w, true);
  return (uint32_t)w;
}

// One wave takes the runs that begin in a window of token rows, for one head and one of
// K and V. A run is a stretch of rows with consecutive slots in one page. Its rows go
// through registers HOLD at a time (16 lanes a row): a run of up to HOLD rows is read once;
// of a longer one all but the last HOLD a second time behind the maximum, from the L2.
// PAGE: the page's tokens.
template <int PAGE, int HOLD>
__global__ __launch_bounds__(256) void cache_store_kernel(StoreArgs P) {
  constexpr int kGroups = HOLD / 4;  // four rows per load
  constexpr bool kOnce = PAGE <= HOLD;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t unit = blockIdx.x * 4 + wave;
  const uint32_t hv = unit % (uint32_t)(2 * P.heads);
  const int w0 = (int)(unit / (uint32_t)(2 * P.heads)) * P.window;
  const int rows = P.batch * P.tokens;
  if (w0 >= rows) return;
  const int head = (int)(hv >> 1);
  const bool is_v = hv & 1;
  const uint16_t* src = static_cast<const uint16_t*>(is_v ? P.V : P.K) + (int64_t)head * P.stride_h;
  uint8_t* codes = is_v ? P.v8 : P.k8;
  int32_t* exps = is_v ? P.v_exp : P.k_exp;
  const int top = P.pages * PAGE;
  const int lr = lane >> 4, lc = lane & 15;
  auto slot_of = [&](int64_t r) { return r >= 0 && r < rows ? P.slots[r] : -1; };
  const int64_t wr = (int64_t)w0 + lane;
  const int mine = slot_of(wr), prev = slot_of(wr - 1);
  const bool starts = lane < P.window && mine >= 0 && mine < top && !(prev == mine - 1 && mine % PAGE != 0);
  for (uint64_t todo = __ballot(starts); todo; todo &= todo - 1) {
    const int at = __builtin_ctzll(todo);
    const int64_t r0 = (int64_t)w0 + at;
    const int slot = __builtin_amdgcn_readlane(mine, at);
    const int page = slot / PAGE, off = slot % PAGE;
    int n;
    {
      const bool in = off + lane < PAGE && slot_of(r0 + lane) == slot + lane;
      const uint64_t out = ~__ballot(in);
      n = out ? __builtin_ctzll(out) : 64;
      if (PAGE > 64 && n == 64) {
        const bool more = off + 64 + lane < PAGE && slot_of(r0 + 64 + lane) == slot + 64 + lane;
        const uint64_t end = ~__ballot(more);
        n += end ? __builtin_ctzll(end) : 64;
      }
    }
    uint4 x[kGroups];
    auto load = [&](int row) {  // rows row .. row + HOLD - 1 of the run
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        x[i] = make_uint4(0, 0, 0, 0);
        if (row + 4 * i < n) {  // wave-uniform
          const uint32_t r = (uint32_t)(r0 + min(row + 4 * i + lr, n - 1));
          const uint32_t b = P.batch == 1 ? 0u : r / (uint32_t)P.tokens;
          x[i] = *reinterpret_cast<const uint4*>(src + (int64_t)b * P.stride_b + (int64_t)(r - b * (uint32_t)P.tokens) * P.stride_n + 8 * lc);
        }
      }
    };
    const int64_t tile = (int64_t)page * P.heads + head;
    const int before = off > 0 ? exps[tile] : kCacheExpMin;
    float amax = 0.f;
    for (int row = 0; row < (kOnce ? 1 : n); row += HOLD) {
      load(row);
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fmaxf(fabsf(bf16_lo(w[e])), fabsf(bf16_hi(w[e]))));
      }
    }
    int e = cache_exponent(wave_max_abs(amax));
    uint8_t* out = codes + tile * (PAGE * kHeadDim);
    if (before >= e) {
      e = before;
    } else if (off > 0) {
      // the tokens already there, on the new scale: one rounding more
      const float by = ldexpf(1.f, max(before - e, -60));
      for (int r = lr; r < off; r += 4) {
        uint2* p = reinterpret_cast<uint2*>(out + r * kHeadDim + 8 * lc);
        const uint2 v = *p;
        float f[8];
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const int w = (int)(d ? v.y : v.x);
          f[4 * d] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * by;
          f[4 * d + 1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * by;
          f[4 * d + 2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * by;
          f[4 * d + 3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * by;
        }
        *p = make_uint2(four_codes(f[0], f[1], f[2], f[3]), four_codes(f[4], f[5], f[6], f[7]));
      }
    }
    const float inv = __uint_as_float((uint32_t)(127 - min(max(e, kCacheExpMin), 120)) << 23);
    // the rows that are still held first, the ones before them once more
    const int last = kOnce ? 0 : (n - 1) / HOLD * HOLD;
    for (int row = last; row >= 0; row -= HOLD) {
      if (!kOnce && row < last) load(row);
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int r = row + 4 * i + lr;
        if (r < n) {
          const uint2 c = make_uint2(
              four_codes(bf16_lo(x[i].x) * inv, bf16_hi(x[i].x) * inv, bf16_lo(x[i].y) * inv, bf16_hi(x[i].y) * inv),
              four_codes(bf16_lo(x[i].z) * inv, bf16_hi(x[i].z) * inv, bf16_lo(x[i].w) * inv, bf16_hi(x[i].w) * inv));
          *reinterpret_cast<uint2*>(out + (off + r) * kHeadDim + 8 * lc) = c;
        }
      }
      if (kOnce) break;
    }
    if (lane == 0) exps[tile] = e;
  }
}

template <int HOLD>
void launch_store(const StoreArgs& a, dim3 grid) {
  switch (a.page) {
    case 16: cache_store_kernel<16, 16><<<grid, 256, 0, a.stream>>>(a); break;
    case 32: cache_store_kernel<32, HOLD < 32 ? HOLD : 32><<<grid, 256, 0, a.stream>>>(a); break;
    case 64: cache_store_kernel<64, HOLD><<<grid, 256, 0, a.stream>>>(a); break;
    default: cache_store_kernel<128, HOLD == 64 ? 128 : HOLD><<<grid, 256, 0, a.stream>>>(a); break;
  }
}

}  // namespace

hipError_t launch_cache_plan(const PlanArgs& a) {
  (void)hipGetLastError();
  // Four rows a thread. The pages that ended streams give back go through the same grid, so that
  // a call of few rows that ends many long streams takes longer: 64 streams of 30,000 tokens (30,016
  // pages) 68 us in one workgroup, 6.5 in the 30 of 30,000 rows.
  const int grid = (int)std::min<int64_t>(256, std::max<int64_t>(1, ((int64_t)a.tokens + 4 * kPlanThreads - 1) / (4 * kPlanThreads)));
  cache_plan_kernel<<<grid, kPlanThreads, 0, a.stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_store(StoreArgs a) {
  (void)hipGetLastError();
  const int64_t rows = (int64_t)a.batch * a.tokens;
  if (rows == 0 || a.heads == 0) return hipSuccess;
  // Windows of up to 64 rows; smaller while that leaves fewer than 4096 waves (16 a CU),
  // since a window of single tokens goes through its runs one after the other.
  a.window = 64;
  while (a.window > 1 && (rows + a.window - 1) / a.window * 2 * a.heads < 4096) a.window >>= 1;
  const int64_t units = (rows + a.window - 1) / a.window * 2 * a.heads;
  const dim3 grid((unsigned)((units + 3) / 4));
  // Rows held: small windows go with calls of many single tokens, whose waves should all be
  // resident (16 rows: eight waves a SIMD); where windows hold whole runs, reading a run
  // once counts (the page: two waves, one with 128). 3041 rows of 40 heads in pages of
  // 64 / 128: 20.2 / 29.9 us held whole, 29.2 in 16 rows / 34.5 in 64; 256 single tokens of
  // 40 heads: 11.2 with 16 rows held, 14.9 with 32, 26.6 with 64; 3041 rows of 5 heads
  // (short windows, whole runs): 12.3, 10.3, 9.9.
  if (a.window < 16)
    launch_store<16>(a, grid);
  else
    launch_store<64>(a, grid);
  return hipGetLastError();
}

}  // namespace fva
