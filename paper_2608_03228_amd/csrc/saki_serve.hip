// The operators that serving runs around the index, for gfx950 (CDNA4, wave64):
//
//   rope_kernel           rotary positions of queries and keys, one to three axes
//   block_tables_kernel   block tables, slots and positions from request lengths
//   cache_write_kernel    keys and values to the 8-bit cache (E4M3 codes, one
//                         power-of-two scale per block of 64 tokens and head)
//   cache_attend_kernel   attention over every cached key of a request, split
//                         evenly over the GPU; cache_join_kernel joins the parts
//   cache_lists_kernel    attention over the keys that a list names

#include "saki_cache.h"

namespace {

constexpr int kBlockBytes = kTile * kHeadDim;  // codes of one (block, head), keys or values

// ---------------------------------------------------------------- rotary positions

struct Turns {
  double f[kHeadDim / 2];  // turns of pair m per position: theta^(-2m/d) / (2 pi)
};

// sine and cosine of `turns` full turns: float64 to within an eighth of a turn
// of a quarter, then the Taylor series (errors below 2e-9 and 2e-10).
__device__ __forceinline__ void sin_cos_turns(double turns, float* s, float* c) {
  const double q = 4.0 * (turns - floor(turns));
  const double n = rint(q);
  const float x = (float)((q - n) * 1.5707963267948966192);
  const float y = x * x;
  const float ps = fmaf(fmaf(fmaf(fmaf(1.f / 362880, y, -1.f / 5040), y, 1.f / 120), y, -1.f / 6) * y, x, x);
  const float pc =
      fmaf(fmaf(fmaf(fmaf(fmaf(-1.f / 3628800, y, 1.f / 40320), y, -1.f / 720), y, 1.f / 24), y, -0.5f), y, 1.f);
  const int k = (int)n;
  const float a = (k & 1) ? pc : ps, b = (k & 1) ? ps : pc;
  *s = (k & 2) ? -a : a;
  *c = ((k + 1) & 2) ? -b : b;
}

// The pair (x_m, x_{m+d/2}) of every head of token t turned by
// pos[axis(m)][t] * theta^(-2m/d).  One wave per token and share of its heads;
// a lane holds the same pairs of every head it visits, so that a token's sines
// and cosines are formed once per wave.  Each lane reads both halves of its
// pairs before it writes them: the outputs may be the inputs.  HBM bound: 16,384
// float32 tokens of 28 + 4 heads in 100 us, 5.4 TB/s; 64 bf16 tokens of 32 + 8
// heads, a few loads deep, in 4.0.
constexpr int kRopeWaves = 4;
constexpr int kRopeAhead = 4;  // heads a lane has in flight
template <typename T>
__global__ __launch_bounds__(kRopeWaves* kWave) void rope_kernel(
    const T* q, const T* k, size_t ld_q, size_t ld_k, T* q_out, T* k_out, size_t ld_qo, size_t ld_ko, int n_tokens,
    int H_q, int H_kv, const int* __restrict__ pos, int s0, int s1, Turns turns, float sign) {
  constexpr int V = 16 / sizeof(T);            // pairs a lane turns
  constexpr int kLanes = kHeadDim / 2 / V;     // lanes a head
  constexpr int kHeads = kWave / kLanes;       // heads a wave visits at once
  const int lane = threadIdx.x % kWave;
  const int t = blockIdx.x * kRopeWaves + threadIdx.x / kWave;
  if (t >= n_tokens) return;
  const int m0 = lane % kLanes * V;
  float sn[V], cs[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int m = m0 + e;
    const int axis = m < s0 ? 0 : m < s0 + s1 ? 1 : 2;
    sin_cos_turns((double)pos[(size_t)axis * n_tokens + t] * turns.f[m], &sn[e], &cs[e]);
    sn[e] *= sign;
  }
  const int H = H_q + H_kv, step = kHeads * gridDim.y;
  for (int h0 = blockIdx.y * kHeads + lane / kLanes; h0 < H; h0 += step * kRopeAhead) {
    float x[kRopeAhead][2][V];
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) {
      const int h = h0 + u * step;
      if (h < H) {
        const T* p = (h < H_q ? q + (size_t)t * ld_q + (size_t)h * kHeadDim
                              : k + (size_t)t * ld_k + (size_t)(h - H_q) * kHeadDim) + m0;
        load_elems<T, V>(p, x[u][0]);
        load_elems<T, V>(p + kHeadDim / 2, x[u][1]);
      }
    }
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) {
      const int h = h0 + u * step;
      if (h < H) {
        T* p = (h < H_q ? q_out + (size_t)t * ld_qo + (size_t)h * kHeadDim
                        : k_out + (size_t)t * ld_ko + (size_t)(h - H_q) * kHeadDim) + m0;
        float a[V], b[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          a[e] = x[u][0][e] * cs[e] - x[u][1][e] * sn[e];
          b[e] = x[u][0][e] * sn[e] + x[u][1][e] * cs[e];
        }
        store_elems<T, V>(p, a);
        store_elems<T, V>(p + kHeadDim / 2, b);
      }
    }
  }
}

// ---------------------------------------------------------------- block tables

// The last i in [0, n) with at[i] <= x (at ascending, at[0] <= x).
__device__ __forceinline__ int find_last(const long long* at, int n, long long x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Request b holds ceil(ctx / 64) blocks and gets new tokens; the blocks that it
// lacks come from the free list, in the order of the requests.  Every
// work-group forms the running sums of all requests (1,024 at a time, in LDS)
// and fills its share of the tokens and of the new table entries, so that one
// launch does and nothing waits for another group: an entry of the tables is
// read only where it was there before, and written only where it was not.
// Latency bound: 5.0 us for 64 requests of one token, 6.2 for 512 with 131,000.
constexpr int kTableChunk = 1024;
__global__ __launch_bounds__(256) void block_tables_kernel(
    const int* __restrict__ ctx, const int* __restrict__ fresh, int B, const int* __restrict__ free_blocks,
    int n_free, int* tables, int max_blocks, int* __restrict__ slots, int* __restrict__ pos, int T,
    int* __restrict__ cu, int* __restrict__ lens, int* __restrict__ counts) {
  __shared__ long long s_tok[kTableChunk], s_want[kTableChunk], part[4];
  __shared__ int s_ctx[kTableChunk], s_got[kTableChunk];
  constexpr int kPer = kTableChunk / 256;
  const int tid = threadIdx.x, stride = gridDim.x * 256;
  long long tok0 = 0, want0 = 0, lack = 0;  // of the requests before this chunk
  long long t = blockIdx.x * 256 + tid, f = t;  // this thread's next token and new entry
  for (int b0 = 0, c = 0; b0 < B; b0 += kTableChunk, ++c) {
    const int n = min(kTableChunk, B - b0);
    long long tok[kPer], want[kPer], tok_sum = 0, want_sum = 0;
    int held[kPer], cx[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid * kPer + j;
      const bool in = i < n;
      cx[j] = in ? min(max(ctx[b0 + i], 0), max_blocks * kTile) : 0;
      tok[j] = in ? max(fresh[b0 + i], 0) : 0;
      held[j] = (cx[j] + kTile - 1) / kTile;
      const long long need = (cx[j] + tok[j] + kTile - 1) / kTile;
      want[j] = min(need, (long long)max_blocks) - held[j];
      lack += need - held[j] - want[j];
      tok_sum += tok[j];
      want_sum += want[j];
    }
    long long tok_all, want_all;
    long long at = tok0 + group_scan(tok_sum, part, &tok_all) - tok_sum;
    long long wat = want0 + group_scan(want_sum, part, &want_all) - want_sum;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid * kPer + j;
      if (i < n) {
        const int got = (int)min(max((long long)n_free - wat, 0LL), want[j]);
        s_tok[i] = at;
        s_want[i] = wat;
        s_ctx[i] = cx[j];
        s_got[i] = got;
        if (c % gridDim.x == blockIdx.x) {
          const long long end = at + tok[j];
          lens[b0 + i] = (int)min(cx[j] + tok[j], (long long)(held[j] + got) * kTile);
          cu[b0 + i + 1] = (int)min(end, (long long)INT_MAX);
          if (b0 + i == 0) cu[0] = 0;
        }
      }
      at += tok[j];
      wat += want[j];
    }
    __syncthreads();
    const long long tok1 = tok0 + tok_all, want1 = want0 + want_all;
    for (; t < T && t < tok1; t += stride) {
      const int i = find_last(s_tok, n, t);
      const int cxt = s_ctx[i], h = (cxt + kTile - 1) / kTile;
      const long long p = cxt + (t - s_tok[i]), blk = p / kTile;
      int id = -1;
      if (blk < h)
        id = tables[(size_t)(b0 + i) * max_blocks + blk];
      else if (blk - h < s_got[i])
        id = free_blocks[s_want[i] + (blk - h)];
      slots[t] = id < 0 || id > INT_MAX / kTile - 1 ? -1 : id * kTile + (int)(p % kTile);
      pos[t] = (int)min(p, (long long)INT_MAX);
    }
    for (; f < n_free && f < want1; f += stride) {
      const int i = find_last(s_want, n, f);
      const int h = (s_ctx[i] + kTile - 1) / kTile;
      tables[(size_t)(b0 + i) * max_blocks + h + (f - s_want[i])] = free_blocks[f];
    }
    tok0 = tok1;
    want0 = want1;
    __syncthreads();  // the chunk's arrays are read
  }
  for (; t < T; t += stride) slots[t] = -1, pos[t] = 0;  // no token of any request
  if (blockIdx.x == 0) {
    long long lacking;
    group_scan(lack, part, &lacking);
    if (tid == 0) {
      const long long taken = min(want0, (long long)n_free);
      counts[0] = (int)taken;
      counts[1] = (int)min(lacking + want0 - taken, (long long)INT_MAX);
    }
  }
}

// ---------------------------------------------------------------- writing the cache

// Four floats times inv as E4M3 codes: nearest, ties to the even code.
__device__ __forceinline__ uint32_t encode4(const float* x, float inv) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, lo, true);
}

__device__ __forceinline__ void decode16(uint4 v, float* x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
    x[4 * j] = lo[0], x[4 * j + 1] = lo[1], x[4 * j + 2] = hi[0], x[4 * j + 3] = hi[1];
  }
}

// Exponent e of the least scale 2^e with top <= 448 * 2^e (448 = 0.875 * 2^9):
// with top = m 2^x, m in [0.5, 1), it is x - 9 for m <= 0.875 and x - 8 else.
// At least -100, so that 2^-e is finite; top = +infinity gets the largest.
__device__ __forceinline__ int scale_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 126 - ((u & 0x7fffffu) <= 0x600000u ? 9 : 8);
  return min(max(e, -100), 120);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// A run is a stretch of tokens whose slots ascend within one block; it belongs
// to the window of tokens in which it begins.  One work-group takes the runs of
// one window for one head's keys or values; each of its four waves holds 16 rows
// of a run in registers between the search for the largest element and the
// rounding, all its loads in flight at once (a wave with all 64 rows, 253
// registers, reached 3.1 TB/s on prompts of float32 tokens).  The block's scale
// is the least power of two that covers the run, and, where the block holds
// tokens before the run, no less than it was; if it grew, the codes before the
// run are moved to it.  Powers of two make that exact but for codes that become
// subnormal, and codes times scale exact in bf16.  HBM bound on prompts: 30,400
// float32 tokens of 4 heads in 37 us, 4.3 TB/s (repeated on the same arrays 5.5);
// latency on single tokens: 64 of 8 heads in 3.6.
template <typename T>
__global__ __launch_bounds__(256) void cache_write_kernel(const T* __restrict__ k, const T* __restrict__ v,
                                                          size_t ld_k, size_t ld_v, int n_tokens, int window,
                                                          const int* __restrict__ slots, int n_blocks, int H,
                                                          uint8_t* k_cache, uint8_t* v_cache, float* scales) {
  constexpr int V = 16 / sizeof(T);      // elements a lane loads at once
  constexpr int kLanes = kHeadDim / V;   // lanes a row
  constexpr int kStep = kWave / kLanes;  // rows a wave loads at once
  constexpr int kRows = kTile / 4, kLoads = kRows / kStep;
  __shared__ float part[2][4];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int h = blockIdx.y >> 1, which = blockIdx.y & 1;
  const T* src = (which ? v : k) + (size_t)h * kHeadDim;
  const size_t ld = which ? ld_v : ld_k;
  uint8_t* const cache = which ? v_cache : k_cache;
  const int n_slots = n_blocks * kTile;
  const int t0 = blockIdx.x * window;
  // tokens t0 - 1 .. t0 + 127: where runs begin and where they go on
  const int s0 = t0 + lane < n_tokens ? slots[t0 + lane] : -1;
  const int s1 = t0 + kWave + lane < n_tokens ? slots[t0 + kWave + lane] : -1;
  int p0 = __shfl_up(s0, 1), p1 = __shfl_up(s1, 1);
  if (lane == 0) p0 = t0 > 0 ? slots[t0 - 1] : -1;
  const int last0 = __builtin_amdgcn_readlane(s0, kWave - 1);
  if (lane == 0) p1 = last0;
  auto goes_on = [&](int s, int p) { return p >= 0 && p < s && s < n_slots && s / kTile == p / kTile; };
  const bool on0 = goes_on(s0, p0);
  const uint64_t on_a = __ballot(on0), on_b = __ballot(goes_on(s1, p1));
  uint64_t begins = __ballot(lane < window && s0 >= 0 && s0 < n_slots && !on0);
  const uint64_t ones = begins & ~((on_a >> 1) | (on_b << (kWave - 1)));
  const int row = lane / kLanes, col = lane % kLanes * V;
  // moves the codes before slot `first` of a block to a grown scale
  auto move = [&](uint8_t* block, int first, float ratio, int from, int step) {
    for (int i = from + lane / 8; i < first; i += step) {
      uint4* o = reinterpret_cast<uint4*>(block + i * kHeadDim + lane % 8 * 16);
      float y[16];
      decode16(*o, y);
      *o = make_uint4(encode4(y, ratio), encode4(y + 4, ratio), encode4(y + 8, ratio), encode4(y + 12, ratio));
    }
  };

  // runs of one token (decode steps): a row of lanes each, a quarter of the window a wave
  const int b = wave * kRows;
  if (const uint32_t mine = (uint32_t)(ones >> b) & ((1u << kRows) - 1)) {
    uint4 x[kLoads];
    int slot[kLoads];
    float old[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      slot[u] = -1;
      x[u] = make_uint4(0u, 0u, 0u, 0u);
      if (mine >> (u * kStep) & ((1u << kStep) - 1)) {
        const int at = u * kStep + row, sl = __shfl(s0, b + at);
        if (mine >> at & 1) {
          slot[u] = sl;
          x[u] = *reinterpret_cast<const uint4*>(src + (size_t)(t0 + b + at) * ld + col);
          old[u] = scales[((size_t)(sl / kTile) * H + h) * 2 + which];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      if (mine >> (u * kStep) & ((1u << kStep) - 1)) {
        float y[V], top = 0.f, ratio = 0.f;
        unpack16<T>(x[u], y);
#pragma unroll
        for (int e = 0; e < V; ++e) top = fmaxf(top, fabsf(y[e]));
#pragma unroll
        for (int m = 1; m < kLanes; m <<= 1) top = fmaxf(top, xor_f32(top, m));
        const int blk = slot[u] / kTile, first = slot[u] % kTile;
        bool grew = false;
        if (slot[u] >= 0) {
          const int e = scale_exponent(top);
          grew = first && !(old[u] >= pow2(e));
          const bool keeps = first && !grew;
          const float inv = keeps ? 1.f / old[u] : pow2(-e);
          ratio = old[u] * inv;
          uint32_t w[V / 4];
#pragma unroll
          for (int j = 0; j < V / 4; ++j) w[j] = encode4(y + 4 * j, inv);
          __builtin_memcpy(cache + ((size_t)blk * H + h) * kBlockBytes + first * kHeadDim + col, w, V);
          if (col == 0 && !keeps) scales[((size_t)blk * H + h) * 2 + which] = pow2(e);
        }
        for (uint64_t g = __ballot(grew && col == 0); g; g &= g - 1) {
          const int l = __builtin_ctzll(g);
          move(cache + ((size_t)__builtin_amdgcn_readlane(blk, l) * H + h) * kBlockBytes,
               __builtin_amdgcn_readlane(first, l),
               __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(ratio), l)), 0, 8);
        }
      }
  }

  // The run of n tokens from t0 + at on, all waves together or one wave alone
  int turn = 0;
  auto take = [&](int at, int n, auto together) __attribute__((always_inline)) {
    const int t = t0 + at, b = together ? wave * kRows : 0;
    const int slot = __builtin_amdgcn_readlane(s0, at);
    const int blk = slot / kTile, first = slot % kTile;
    uint8_t* out = cache + ((size_t)blk * H + h) * kBlockBytes;
    float* scale = scales + ((size_t)blk * H + h) * 2 + which;
    uint4 x[kLoads];
    int to[kLoads];
    float top = 0.f;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = b + u * kStep + row;
      x[u] = make_uint4(0u, 0u, 0u, 0u);
      if (i < n) {
        x[u] = *reinterpret_cast<const uint4*>(src + (size_t)(t + i) * ld + col);
        to[u] = slots[t + i] % kTile;
      }
    }
    const float old = first ? *scale : 0.f;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      float y[V];
      unpack16<T>(x[u], y);
#pragma unroll
      for (int e = 0; e < V; ++e) top = fmaxf(top, fabsf(y[e]));
    }
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) top = fmaxf(top, xor_f32(top, m));
    if constexpr (together) {
      if (lane == 0) part[turn][wave] = top;
      __syncthreads();  // (the next run has the other half of `part`)
      top = fmaxf(fmaxf(part[turn][0], part[turn][1]), fmaxf(part[turn][2], part[turn][3]));
      turn ^= 1;
    }
    const int e = scale_exponent(top);
    const bool grew = first && !(old >= pow2(e));
    const float now = first && !grew ? old : pow2(e);
    const float inv = first && !grew ? 1.f / now : pow2(-e);
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      if (b + u * kStep + row < n) {
        float y[V];
        unpack16<T>(x[u], y);
        uint32_t w[V / 4];
#pragma unroll
        for (int j = 0; j < V / 4; ++j) w[j] = encode4(y + 4 * j, inv);
        __builtin_memcpy(out + to[u] * kHeadDim + col, w, V);
      }
    if (grew) move(out, first, old * inv, together ? 8 * wave : 0, together ? 32 : 8);
    // (all waves that take part have read the scale, before the barrier above)
    if (b == 0 && lane == 0 && (!first || grew)) *scale = now;
  };
  int alone = 0;
  for (begins &= ~ones; begins; begins &= begins - 1) {
    const int at = __builtin_ctzll(begins);
    // the tokens after `at` that go on: at most 63, as a block's slots ascend
    const uint64_t on = at == kWave - 1 ? on_b : (on_a >> (at + 1)) | (on_b << (kWave - 1 - at));
    const int n = ~on ? 1 + __builtin_ctzll(~on) : kTile;
    if (n > kRows)
      take(at, n, std::true_type());
    else if (alone++ % 4 == wave)  // (2,000 requests of 3 tokens: 43 us with all waves at each)
      take(at, n, std::false_type());
  }
}

// ---------------------------------------------------------------- attention over the cache

constexpr int kAttendGroups = 512;  // two a CU

__device__ __forceinline__ Share share_of(long long total, int groups) {
  Share s;
  s.total = total;
  s.piece = (total + groups - 1) / groups;
  if (s.piece < kMinPiece) s.piece = kMinPiece;
  return s;
}

// Eight E4M3 codes as bf16 (exact: a code has at most 4 significant bits).
__device__ __forceinline__ bf16x8_t widen8(uint32_t lo, uint32_t hi) {
  uint32_t w[4];
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  __builtin_memcpy(&w[0], &a, 4);
  __builtin_memcpy(&w[1], &b, 4);
  __builtin_memcpy(&w[2], &c, 4);
  __builtin_memcpy(&w[3], &d, 4);
  bf16x8_t r;
  __builtin_memcpy(&r, w, sizeof(r));
  return r;
}

// s_k = (q . code_k) scale_k / sqrt(d) over a request's keys, softmax, sum of
// values.  A work-group takes a share of the tiles (a tile is a cache block of
// one head); its four waves take every fourth tile of each stretch of one pair
// and keep their own running maximum, weight and sums, joined in LDS at the
// stretch's end.  A stretch that is not the whole pair goes to the workspace.
//
// One tile: S^T = K Q^T on the 16x16x32 MFMA, keys as rows, the 16 query rows
// of a KV group as columns.  Key rows are taken in the order that leaves lane
// group g (16 lanes) with the scores of keys 16 g .. 16 g + 15 of one query, so
// that these are at once its operand of O^T = V^T P^T, with no exchange.  A
// lane reads 8 dims of each of its 16 keys' values and transposes bytes in
// registers; dims 8 m .. 8 m + 7 of lane m are the rows m of eight products.
// The codes are exact in bf16; queries (float32: three terms) and weights (two
// terms, three for float32 output) are split so that nothing but the output is
// rounded to bf16.  HBM bound, 16 KB a tile: 8 requests of up to 131,072 keys in
// 4 heads in 108 us, 5.5 TB/s of 590 MB fetched.  A request of 4,001 keys in 8
// heads takes 9.5-10.2 us, and the join 4.2-4.8 (in a kernel trace; 13.4 as calls
// in a row): a chain of reads (lengths, table, codes) with a tile a
// wave behind it.  Holding the next tile's codes in registers (241 of them) did
// not shorten either, 14.2 us against 13.4 for the step.
//
// Without SPLIT a work-group takes one whole pair: no share to find, no
// workspace and no join (see whole_better).
template <bool F32, bool SPLIT>
__global__ __launch_bounds__(256, 2) void cache_attend_kernel(CacheArgs a, const void* __restrict__ q, void* out,
                                                              float* __restrict__ ws) {
  constexpr int kQT = F32 ? 3 : 1, kPT = F32 ? 3 : 2;
  __shared__ float s_m[4][16], s_l[4][16], s_o[4][16][kHeadDim + 4];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int n = lane % 16, g = lane / 16;
  const int G = a.H_q / a.H_kv, R = G * a.Q, RB = (R + 15) / 16, pairs = a.H_kv * RB;

  long long cur = 0, end = 1, base = 0;  // the tiles to take, the tiles before request b
  int b = blockIdx.x / pairs, lens = 0;  // (lens: of request `lane` of up to 64)
  if constexpr (SPLIT) {
    __shared__ long long part[4], found[2];
    if (a.B <= kWave) {  // every wave for itself
      const Sums all = wave_sums(a);
      const Share sh = share_of((long long)all.total * pairs, gridDim.x);
      cur = sh.piece * blockIdx.x;
      end = min(sh.total, cur + sh.piece);
      if (cur >= end) return;
      b = __builtin_ctzll(__ballot(cur < (long long)all.upto * pairs));
      base = (long long)__builtin_amdgcn_readlane(all.upto - all.mine, b) * pairs;
      lens = all.len;
    } else {
      long long total = 0;
      for (int b0 = 0; b0 < a.B; b0 += 256) {
        const int t = b0 + tid < a.B ? tiles_of(a.lens[b0 + tid], a.max_blocks) : 0;
        long long sum;
        group_scan((long long)t * pairs, part, &sum);
        total += sum;
      }
      const Share sh = share_of(total, gridDim.x);
      cur = sh.piece * blockIdx.x;
      end = min(total, cur + sh.piece);
      if (cur >= end) return;
      for (int b0 = 0; b0 < a.B; b0 += 256) {
        const long long t = b0 + tid < a.B ? (long long)tiles_of(a.lens[b0 + tid], a.max_blocks) * pairs : 0;
        long long sum;
        const long long upto = base + group_scan(t, part, &sum);
        if (cur < upto && cur >= upto - t) found[0] = b0 + tid, found[1] = upto - t;
        base += sum;
        if (cur < base) break;
      }
      __syncthreads();
      b = (int)found[0];
      base = found[1];
    }
  }

  while (cur < end) {
    const int len = SPLIT && a.B <= kWave ? __builtin_amdgcn_readlane(lens, b) : a.lens[b];
    const int nt = tiles_of(len, a.max_blocks);
    if (SPLIT && cur >= base + (long long)nt * pairs) {
      base += (long long)nt * pairs;
      if (++b >= a.B) return;  // (a later request has the tiles that are left)
      continue;
    }
    const int pair = SPLIT ? (int)((cur - base) / nt) : blockIdx.x % pairs, t0 = SPLIT ? (int)((cur - base) % nt) : 0;
    const int t1 = SPLIT ? (int)min((long long)nt, t0 + (end - cur)) : nt;
    const int hk = pair / RB, r0 = pair % RB * 16;
    const size_t row0 = ((size_t)b * a.H_q + (size_t)hk * G) * a.Q + r0;

    // a tile's block is asked for a tile ahead, the first one's before the queries
    const int* table = a.tables + (size_t)b * a.max_blocks;
    int next = t0 + wave < t1 ? table[t0 + wave] : -1;

    // queries: dims 64 (s / 2) + 16 g + 8 (s % 2) .. + 7 for step s
    bf16x8_t qf[4][kQT];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      const size_t at = (row0 + n) * kHeadDim + 64 * (s / 2) + 16 * g + 8 * (s % 2);
      if (r0 + n < R) {
        if constexpr (F32)
          load_elems<float, 8>((const float*)q + at, x);
        else
          load_elems<__bf16, 8>((const __bf16*)q + at, x);
      }
      split_bf16<kQT>(x, qf[s]);
    }
    const int seen = len - a.Q + (r0 + n) % a.Q + 1;  // keys that this lane's query sees
    const int least = len - a.Q + 1;

    f32x4_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    for (int t = t0 + wave; t < t1; t += 4) {
      const int blk = next;
      next = t + 4 < t1 ? table[t + 4] : -1;
      if (blk < 0 || blk >= a.n_blocks) continue;
      const size_t at = ((size_t)blk * a.H_kv + hk) * kBlockBytes;
      const float2 sc = *reinterpret_cast<const float2*>((const float*)a.scales + ((size_t)blk * a.H_kv + hk) * 2);
      uint4 kx[4][2];
      uint2 vx[16];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const uint8_t* p = a.k + at + (16 * (n / 4) + 4 * s + n % 4) * kHeadDim + 16 * g;
        kx[s][0] = *reinterpret_cast<const uint4*>(p);
        kx[s][1] = *reinterpret_cast<const uint4*>(p + 64);
      }
#pragma unroll
      for (int j = 0; j < 16; ++j)
        vx[j] = *reinterpret_cast<const uint2*>(a.v + at + (16 * g + j) * kHeadDim + 8 * n);

      float p[16];
      const float f = sc.x * (0.08838834764831845f * kLog2e);
      float top = -INFINITY;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const bf16x8_t k0 = widen8(kx[s][w].x, kx[s][w].y), k1 = widen8(kx[s][w].z, kx[s][w].w);
#pragma unroll
          for (int x = kQT - 1; x >= 0; --x) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[2 * w][x], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[2 * w + 1][x], acc, 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) p[4 * s + i] = acc[i] * f;
      }
      if ((t + 1) * kTile > least) {  // keys that a query does not see, or that were never written
        const int left = seen - t * kTile - 16 * g, whole = len - t * kTile - 16 * g;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (j >= left) p[j] = -INFINITY;
          if (j >= whole) vx[j] = make_uint2(0u, 0u);
        }
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, p[j]);
      top = fmaxf(top, xor_f32(top, 16));
      top = fmaxf(top, xor_f32(top, 32));
      const float m1 = fmaxf(m, top), ref = m1 == -INFINITY ? 0.f : m1;
      const float keep = __builtin_amdgcn_exp2f(m - ref);
      m = m1;
      l *= keep;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        p[j] = __builtin_amdgcn_exp2f(p[j] - ref);
        l += p[j];
        p[j] *= sc.y;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] *= keep;
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // 8 keys a lane
        bf16x8_t pt[kPT];
        split_bf16<kPT>(p + 8 * half, pt);
        // bytes of dim 4 w + c of keys 0..3 and 4..7
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint32_t tr[2][4];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            uint32_t r[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const uint2 e = vx[8 * half + 4 * x + y];
              r[y] = w ? e.y : e.x;
            }
            // v_perm_b32(hi, lo, sel): selector bytes 0-3 pick from lo, 4-7 from hi
            const uint32_t a0 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u);  // r0.0 r1.0 r0.1 r1.1
            const uint32_t a1 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);  // r0.2 r1.2 r0.3 r1.3
            const uint32_t b0 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u);
            const uint32_t b1 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
            tr[x][0] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
            tr[x][1] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
            tr[x][2] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
            tr[x][3] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const bf16x8_t vv = widen8(tr[0][c], tr[1][c]);
#pragma unroll
            for (int x = kPT - 1; x >= 0; --x)
              o[4 * w + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pt[x], o[4 * w + c], 0, 0, 0);
          }
        }
      }
    }

    // the waves' parts: lane (n, g) holds dims 8 (4 g + i) + j of row n in o[j][i]
    l += xor_f32(l, 16);
    l += xor_f32(l, 32);
    __syncthreads();  // the last stretch's parts are read
    if (g == 0) s_m[wave][n] = m, s_l[wave][n] = l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* p = &s_o[wave][n][8 * (4 * g + i)];
      *reinterpret_cast<float4*>(p) = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
      *reinterpret_cast<float4*>(p + 4) = make_float4(o[4][i], o[5][i], o[6][i], o[7][i]);
    }
    __syncthreads();
    constexpr int kDims = 8;  // of a thread
    const int row = tid / 16, d0 = tid % 16 * kDims;
    float M = -INFINITY, L = 0.f, y[kDims];
#pragma unroll
    for (int j = 0; j < kDims; ++j) y[j] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, s_m[w][row]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float e = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][row] - M);
      L += s_l[w][row] * e;
#pragma unroll
      for (int j = 0; j < kDims; ++j) y[j] += s_o[w][row][d0 + j] * e;
    }
    if (r0 + row < R) {
      if (!SPLIT || (t0 == 0 && t1 == nt)) {
        const float inv = L > 0.f ? 1.f / L : 0.f;
        const size_t to = (row0 + row) * kHeadDim + d0;
#pragma unroll
        for (int j = 0; j < kDims; ++j) y[j] *= inv;
        if constexpr (F32)
          store_elems<float, kDims>((float*)out + to, y);
        else
          store_elems<__bf16, kDims>((__bf16*)out + to, y);
      } else if constexpr (SPLIT) {
        // a share has two such stretches at most: one that began before it, one that ends after it
        float* p = ws + ((size_t)blockIdx.x * 2 + (t0 == 0)) * kPartFloats;
        store_elems<float, kDims>(p + row * kHeadDim + d0, y);
        if (d0 == 0) p[kPartRows * kHeadDim + row] = M, p[kPartRows * kHeadDim + kPartRows + row] = L;
      }
    }
    if (!SPLIT) break;
    cur += t1 - t0;
  }
}

// Joins the parts of the pairs that several work-groups shared, and writes
// zeros for requests without a key.  A work-group takes 16 dims of a pair (all
// dims, 16 at a time, above 256 pairs); its four waves take every fourth part.
// us of attention and join, a group a pair / eight (bf16, 32 / 8 heads, tables of
// 40 and 80 tiles): 128 pairs 26.1 / 19.3, 256 34.0 / 30.3, 320 50.4 / 47.2, 512
// 89.1 / 88.3, 1,024 148 / 153, 4,096 524 / 562.
template <bool F32>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheArgs a, int groups, const float* __restrict__ ws,
                                                         void* out) {
  __shared__ long long part[4], s_base;
  __shared__ float s_m[4][16], s_l[4][16], s_y[4][16][16];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int G = a.H_q / a.H_kv, R = G * a.Q, RB = (R + 15) / 16, pairs = a.H_kv * RB;
  const int b = blockIdx.x / pairs, pair = blockIdx.x % pairs;
  long long total = 0, base;
  int nt;
  if (a.B <= kWave) {
    const Sums all = wave_sums(a);
    total = (long long)all.total * pairs;
    nt = __builtin_amdgcn_readlane(all.mine, b);
    base = (long long)(__builtin_amdgcn_readlane(all.upto, b) - nt) * pairs;
  } else {
    for (int b0 = 0; b0 < a.B; b0 += 256) {
      const int t = b0 + tid < a.B ? tiles_of(a.lens[b0 + tid], a.max_blocks) : 0;
      long long sum;
      const long long upto = group_scan((long long)t * pairs, part, &sum);
      if (b0 + tid == b) s_base = total + upto - (long long)t * pairs;
      total += sum;
    }
    __syncthreads();
    nt = tiles_of(a.lens[b], a.max_blocks);
    base = s_base;
  }
  const Share sh = share_of(total, groups);
  const long long from = base + (long long)nt * pair;
  const int w0 = (int)(from / sh.piece), w1 = nt ? (int)((from + nt - 1) / sh.piece) : w0;
  if (nt && w0 == w1) return;
  const int row = lane / 4;
  const int hk = pair / RB, r0 = pair % RB * 16;
  const bool in = r0 + row < R;
  for (int part16 = blockIdx.y; part16 < kHeadDim / 16; part16 += gridDim.y) {
    const int d0 = part16 * 16 + lane % 4 * 4;
    float M = -INFINITY, L = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    if (nt && in)
      for (int w = w0 + wave; w <= w1; w += 4) {
        const float* p = ws + ((size_t)w * 2 + (w == w0)) * kPartFloats;
        const float m = p[kPartRows * kHeadDim + row], l = p[kPartRows * kHeadDim + kPartRows + row];
        const float4 x = *reinterpret_cast<const float4*>(p + row * kHeadDim + d0);
        const float m1 = fmaxf(M, m), ref = m1 == -INFINITY ? 0.f : m1;
        const float e0 = __builtin_amdgcn_exp2f(M - ref), e1 = __builtin_amdgcn_exp2f(m - ref);
        M = m1;
        L = L * e0 + l * e1;
        y[0] = y[0] * e0 + x.x * e1, y[1] = y[1] * e0 + x.y * e1;
        y[2] = y[2] * e0 + x.z * e1, y[3] = y[3] * e0 + x.w * e1;
      }
    __syncthreads();  // the last dims are read
    s_m[wave][row] = M, s_l[wave][row] = L;  // equal from a row's four lanes
#pragma unroll
    for (int j = 0; j < 4; ++j) s_y[wave][row][lane % 4 * 4 + j] = y[j];
    __syncthreads();
    const int r = tid / 16, d = tid % 16;
    if (r0 + r >= R) continue;
    M = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
    float sum = 0.f;
    L = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float e = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][r] - M);
      L += s_l[w][r] * e;
      sum += s_y[w][r][d] * e;
    }
    sum = L == 0.f ? 0.f : sum / L;  // (a NaN stays one)
    const size_t to = (((size_t)b * a.H_q + (size_t)hk * G) * a.Q + r0 + r) * kHeadDim + part16 * 16 + d;
    if constexpr (F32)
      ((float*)out)[to] = sum;
    else
      ((__bf16*)out)[to] = (__bf16)sum;
  }
}

// Attention over listed keys: one wave per (request, head, query) row.  Lane e
// looks up entry e; eight lanes then read one key's or value's 128 bytes, eight
// entries at a time, all in flight together.  Few rows are latency bound (list,
// table, codes): 256 over 131,072 keys take 7.2-7.7 us as calls in a row (8.4-8.6
// in a kernel trace), 8.4 with four of the waves a work-group, on a quarter
// of the CUs; 32,768 rows read 5.4 TB/s.
template <bool F32>
__global__ __launch_bounds__(64) void cache_lists_kernel(CacheArgs a, const void* __restrict__ q,
                                                          const int* __restrict__ top_idx, int k,
                                                          void* __restrict__ out) {
  using T = std::conditional_t<F32, float, __bf16>;
  const int lane = threadIdx.x % kWave;
  const size_t r = blockIdx.x;
  const int i = (int)(r % a.Q), h = (int)(r / a.Q % a.H_q), b = (int)(r / a.Q / a.H_q);
  const int hk = h / (a.H_q / a.H_kv);
  const long long seen = (long long)a.lens[b] - a.Q + i + 1;
  int at = -1;  // the entry's row of the cache
  float2 sc = make_float2(0.f, 0.f);
  const int j = lane < k ? top_idx[r * k + lane] : -1;
  if (j >= 0 && j < seen && j / kTile < a.max_blocks) {
    const int blk = a.tables[(size_t)b * a.max_blocks + j / kTile];
    if (blk >= 0 && blk < a.n_blocks) {
      at = (blk * a.H_kv + hk) * kTile + j % kTile;
      sc = *reinterpret_cast<const float2*>((const float*)a.scales + ((size_t)blk * a.H_kv + hk) * 2);
    }
  }
  const int c = lane % 8, e0 = lane / 8;
  float qx[16];
  load_elems<T, 16>((const T*)q + r * kHeadDim + 16 * c, qx);
  uint4 kx[8], vx[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int row = __shfl(at, 8 * u + e0);
    kx[u] = vx[u] = make_uint4(0u, 0u, 0u, 0u);
    if (row >= 0) {
      kx[u] = *reinterpret_cast<const uint4*>(a.k + (size_t)row * kHeadDim + 16 * c);
      vx[u] = *reinterpret_cast<const uint4*>(a.v + (size_t)row * kHeadDim + 16 * c);
    }
  }
  float p[8], top = -INFINITY;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    float x[16], s = 0.f;
    decode16(kx[u], x);
#pragma unroll
    for (int e = 0; e < 16; ++e) s = fmaf(x[e], qx[e], s);
    s += xor_f32(s, 1);
    s += xor_f32(s, 2);
    s += xor_f32(s, 4);
    const int row = __shfl(at, 8 * u + e0);  // (every lane takes part in both)
    const float f = __shfl(sc.x, 8 * u + e0) * (0.08838834764831845f * kLog2e);
    p[u] = row < 0 ? -INFINITY : s * f;
    top = fmaxf(top, p[u]);
  }
#pragma unroll
  for (int m = 8; m < kWave; m <<= 1) top = fmaxf(top, xor_f32(top, m));
  if (top == -INFINITY) top = 0.f;
  float l = 0.f, o[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) o[e] = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float w = __builtin_amdgcn_exp2f(p[u] - top);
    const float ws = w * __shfl(sc.y, 8 * u + e0);
    float x[16];
    l += w;
    decode16(vx[u], x);
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = fmaf(ws, x[e], o[e]);
  }
  // sums over the eight lanes of equal c, each step halving the dims a lane keeps
#pragma unroll
  for (int m = 8; m < kWave; m <<= 1) l += xor_f32(l, m);
  int d0 = 16 * c;
#pragma unroll
  for (int m = 32, w = 8; m >= 8; m >>= 1, w >>= 1) {
    const bool up = lane & m;
#pragma unroll
    for (int e = 0; e < w; ++e) {
      const float give = up ? o[e] : o[e + w], mine = up ? o[e + w] : o[e];
      o[e] = mine + xor_f32(give, m);
    }
    d0 += up ? w : 0;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if constexpr (F32)
    *reinterpret_cast<float2*>((float*)out + r * kHeadDim + d0) = make_float2(o[0] * inv, o[1] * inv);
  else
    *reinterpret_cast<uint32_t*>((__bf16*)out + r * kHeadDim + d0) = pack_bf16(o[0] * inv, o[1] * inv);
}

// ---------------------------------------------------------------- argument checks

constexpr int kMaxRopeTokens = kMaxTokens - kRopeWaves;  // 256 threads for kRopeWaves tokens: fewer than 2^32

// Blocks and heads of a cache: row numbers (64 tokens a block) fit an int.
int check_cache(const void* k, const void* v, const void* scales, int n_blocks, int H_kv) {
  if (n_blocks < 0 || H_kv <= 0) return SAKI_ERR_ARG;
  if ((long long)n_blocks * H_kv > INT_MAX / kTile || H_kv > 32767) return SAKI_ERR_UNSUPPORTED;
  if (n_blocks > 0 && (!k || !v || !scales || !aligned(k, 16) || !aligned(v, 16) || !aligned(scales, 8)))
    return SAKI_ERR_ARG;
  return SAKI_OK;
}

int attend_groups(long long tiles) {
  const long long g = (tiles + kMinPiece - 1) / kMinPiece;
  return (int)(g < 1 ? 1 : g > kAttendGroups ? kAttendGroups : g);
}

}  // namespace

extern "C" {

int saki_rope(const void* q, const void* k, int dtype, int T, int H_q, int H_kv, int d, size_t ld_q, size_t ld_k,
              const int* pos, int axes, const int* sections, float rope_theta, int inverse, void* q_out,
              void* k_out, size_t ld_q_out, size_t ld_k_out, void* stream) {
  if (T < 0 || H_q < 0 || H_kv < 0 || H_q > 65535 || H_kv > 65535 || d <= 0 || !(rope_theta > 0.f) ||
      !std::isfinite(rope_theta) || !sections)
    return SAKI_ERR_ARG;
  if (d != kHeadDim || !type_ok(dtype) || axes < 1 || axes > 3 || T > kMaxRopeTokens)
    return SAKI_ERR_UNSUPPORTED;
  int s[3] = {0, 0, 0}, sum = 0;
  for (int i = 0; i < axes; ++i) {
    if (sections[i] < 0 || sections[i] > d / 2) return SAKI_ERR_ARG;
    sum += s[i] = sections[i];
  }
  if (sum != d / 2) return SAKI_ERR_ARG;
  if (T == 0 || H_q + H_kv == 0) return SAKI_OK;
  if (!pos) return SAKI_ERR_ARG;
  if (H_q && (!rows_ok(q, ld_q, H_q, dtype) || !rows_ok(q_out, ld_q_out, H_q, dtype))) return SAKI_ERR_ARG;
  if (H_kv && (!rows_ok(k, ld_k, H_kv, dtype) || !rows_ok(k_out, ld_k_out, H_kv, dtype))) return SAKI_ERR_ARG;
  Turns turns;
  // powers by products, within 2^-51 (3.5e-16 at theta = 500,000; 64 or 16 calls
  // of pow are 0.3 us and more of a call of 5)
  const double r = std::pow((double)rope_theta, -2.0 / d), r8 = std::pow((double)rope_theta, -16.0 / d);
  double lo[8] = {1.0}, hi[8] = {0.15915494309189533577};
  for (int i = 1; i < 8; ++i) lo[i] = lo[i - 1] * r, hi[i] = hi[i - 1] * r8;
  for (int m = 0; m < d / 2; ++m) turns.f[m] = hi[m / 8] * lo[m % 8];
  // heads that a wave visits at once; a token's heads are split over up to that
  // many waves while there are few tokens
  const int at_once = dtype == SAKI_F32 ? 4 : 8;
  const int most = (H_q + H_kv + at_once - 1) / at_once;
  int split = 4096 / T;
  split = split < 1 ? 1 : split > most ? most : split;
  const dim3 grid((T + kRopeWaves - 1) / kRopeWaves, split), block(kRopeWaves * kWave);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const float sign = inverse ? -1.f : 1.f;
  if (dtype == SAKI_F32)
    hipLaunchKernelGGL((rope_kernel<float>), grid, block, 0, st, (const float*)q, (const float*)k, ld_q, ld_k,
                       (float*)q_out, (float*)k_out, ld_q_out, ld_k_out, T, H_q, H_kv, pos, s[0], s[1], turns, sign);
  else
    hipLaunchKernelGGL((rope_kernel<__bf16>), grid, block, 0, st, (const __bf16*)q, (const __bf16*)k, ld_q, ld_k,
                       (__bf16*)q_out, (__bf16*)k_out, ld_q_out, ld_k_out, T, H_q, H_kv, pos, s[0], s[1], turns,
                       sign);
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

int saki_block_tables(const int* ctx_lens, const int* new_lens, int B, const int* free_blocks, int n_free,
                      int* tables, int max_blocks, int* slots, int* pos, int T, int* cu, int* lens, int* counts,
                      void* stream) {
  if (B <= 0 || n_free < 0 || max_blocks <= 0 || T < 0) return SAKI_ERR_ARG;
  if (max_blocks > INT_MAX / kTile - 1) return SAKI_ERR_UNSUPPORTED;
  if (!ctx_lens || !new_lens || !tables || !cu || !lens || !counts || (n_free && !free_blocks) ||
      (T && (!slots || !pos)))
    return SAKI_ERR_ARG;
  const int* in[3] = {ctx_lens, new_lens, free_blocks};
  const size_t in_n[3] = {(size_t)B, (size_t)B, (size_t)n_free};
  const int* const to[6] = {tables, slots, pos, cu, lens, counts};
  const size_t to_n[6] = {(size_t)B * max_blocks, (size_t)T, (size_t)T, (size_t)B + 1, (size_t)B, 2};
  for (int i = 0; i < 3; ++i)  // (a group may write before another has read)
    for (int j = 0; j < 6; ++j)
      if (overlap(in[i], in_n[i] * sizeof(int), to[j], to_n[j] * sizeof(int))) return SAKI_ERR_ARG;
  int groups = (T + 255) / 256;  // a token a thread: 512 x 256 tokens in 6.0 us, two 6.8, four 8.5
  groups = groups < 1 ? 1 : groups > 1024 ? 1024 : groups;
  hipLaunchKernelGGL(block_tables_kernel, dim3(groups), dim3(256), 0, reinterpret_cast<hipStream_t>(stream),
                     ctx_lens, new_lens, B, free_blocks, n_free, tables, max_blocks, slots, pos, T, cu, lens, counts);
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

int saki_cache_write(const void* k, const void* v, int dtype, int T, int H_kv, int d, size_t ld_k, size_t ld_v,
                     const int* slots, void* k_cache, void* v_cache, float* scales, int n_blocks, void* stream) {
  if (T < 0 || d <= 0) return SAKI_ERR_ARG;
  const int st = check_cache(k_cache, v_cache, scales, n_blocks, H_kv);
  if (st != SAKI_OK) return st;
  if (d != kHeadDim || !type_ok(dtype) || T > kMaxTokens) return SAKI_ERR_UNSUPPORTED;
  if (T == 0) return SAKI_OK;
  if (!slots || !rows_ok(k, ld_k, H_kv, dtype) || !rows_ok(v, ld_v, H_kv, dtype)) return SAKI_ERR_ARG;
  if (n_blocks == 0) return SAKI_OK;  // no slot is within it
  const size_t codes = (size_t)n_blocks * H_kv * kBlockBytes, n_scales = (size_t)n_blocks * H_kv * 2 * sizeof(float);
  if (overlap(k_cache, codes, v_cache, codes) || overlap(k_cache, codes, scales, n_scales) ||
      overlap(v_cache, codes, scales, n_scales))
    return SAKI_ERR_ARG;
  // some 2,000 work-groups (twice as many: 4,000 tokens of 8 heads 10.1 us in place of 7.1)
  int window = 1;
  while (window < kWave && (long long)T * 2 * H_kv > 2048LL * window) window *= 2;
  const dim3 grid((T + window - 1) / window, 2 * H_kv);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == SAKI_F32)
    hipLaunchKernelGGL((cache_write_kernel<float>), grid, dim3(256), 0, s, (const float*)k, (const float*)v, ld_k,
                       ld_v, T, window, slots, n_blocks, H_kv, (uint8_t*)k_cache, (uint8_t*)v_cache, scales);
  else
    hipLaunchKernelGGL((cache_write_kernel<__bf16>), grid, dim3(256), 0, s, (const __bf16*)k, (const __bf16*)v,
                       ld_k, ld_v, T, window, slots, n_blocks, H_kv, (uint8_t*)k_cache, (uint8_t*)v_cache, scales);
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

}  // extern "C"

namespace {

// Whether a work-group takes a whole pair: the lengths are read on the device,
// so the tables' width has to bound a group's time.  us (bf16, 32 / 8 heads, calls
// in a row in a graph), split and joined / whole pairs, for requests of the full
// width:
//                4 tiles       8            12           16           32           64
//    1 request   8.1 / 5.7    9.4 / 7.6    9.3 / 9.2    9.5 / 10.8  10.0 / 17.2  10.8 / 29.6
//    8           8.4 / 5.8    9.7 / 7.7    9.8 / 9.3   10.0 / 10.9  13.2 / 18.8
//   16                                                 13.5 / 12.2
//   32                       14.2 / 8.5                20.8 / 14.7  30.6 / 23.3
//   64          12.7 / 8.2   18.7 / 14.3               29.1 / 24.7  49.3 / 44.0   106 / 99
//  256          34.1 / 26.2                             108 / 100    193 / 192
// float32, later, with lengths of the full width, and with any up to it:
//    1 request   9.2 / 6.4   10.2 / 8.5   10.3 / 10.5  10.3 / 12.4  10.8 / 20.8
//    8                       10.8 / 8.6   11.4 / 10.6  12.0 / 14.3  15.4 / 24.1
//    8, any                  13.8 / 8.6   13.8 / 10.5  21.1 / 12.5  17.3 / 23.2
//   16                                                 15.3 / 15.1  20.1 / 24.5
//   32                                                 21.0 / 16.0  31.0 / 27.1  61.8 / 63.9
//   32, any                                            29.7 / 14.9  43.9 / 24.4  55.0 / 54.4
//   64                                                 28.2 / 24.7  57.1 / 53.1   104 / 100
//   64, any                                            50.4 / 20.5  63.0 / 37.8  97.0 / 73.5
//  256          40.4 / 34.3                             114 / 105    209 / 200
// (many pairs fill the GPU without being split, up to the width where one long
// request among short ones would keep its groups at work alone for long).
bool whole_better(long long pairs, int max_blocks) {
  return max_blocks <= (pairs >= 512 ? 64 : pairs >= 256 ? 32 : pairs >= 128 ? 16 : 12);
}

}  // namespace

extern "C" {

size_t saki_cache_attend_workspace_bytes(int B, int H_q, int H_kv, int Q, int max_blocks, int k) {
  if (B <= 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || Q < 0 || Q > SAKI_CACHE_MAX_Q || max_blocks <= 0 || k < 0 ||
      k > saki::kMaxK)
    return 0;
  const long long row_blocks = ((long long)(H_q / H_kv) * Q + 15) / 16;
  if (k > 0 || Q == 0 || whole_better((long long)B * H_kv * row_blocks, max_blocks)) return 256;
  const double tiles = (double)B * H_kv * row_blocks * max_blocks;
  const int groups = attend_groups(tiles > 1e9 ? 1000000000LL : (long long)tiles);
  return (size_t)groups * 2 * kPartFloats * sizeof(float);
}

int saki_cache_attend(const void* q, int dtype, int B, int H_q, int H_kv, int Q, int d, const void* k_cache,
                      const void* v_cache, const float* scales, int n_blocks, const int* tables, int max_blocks,
                      const int* lens, const int* top_idx, int k, void* out, void* ws, size_t ws_bytes,
                      void* stream) {
  if (B <= 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || Q < 0 || d <= 0 || max_blocks <= 0 || k < 0 ||
      (top_idx != nullptr) != (k > 0))
    return SAKI_ERR_ARG;
  const int st = check_cache(k_cache, v_cache, scales, n_blocks, H_kv);
  if (st != SAKI_OK) return st;
  const long long row_blocks = ((long long)(H_q / H_kv) * Q + 15) / 16;
  if (d != kHeadDim || !type_ok(dtype) || k > saki::kMaxK || Q > SAKI_CACHE_MAX_Q || max_blocks > INT_MAX / kTile - 1 ||
      (long long)B * H_kv * row_blocks > (1 << 22) || (long long)B * H_q * Q > (1 << 25))
    return SAKI_ERR_UNSUPPORTED;
  if (Q == 0) return SAKI_OK;
  if (!q || !out || !tables || !lens || !aligned(q, 16) || !aligned(out, 16)) return SAKI_ERR_ARG;
  const CacheArgs a{(const uint8_t*)k_cache, (const uint8_t*)v_cache, scales, n_blocks, tables, max_blocks, lens,
                    B, H_q, H_kv, Q};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (k > 0) {
    const dim3 grid((unsigned)((size_t)B * H_q * Q));
    if (dtype == SAKI_F32)
      hipLaunchKernelGGL((cache_lists_kernel<true>), grid, dim3(64), 0, s, a, q, top_idx, k, out);
    else
      hipLaunchKernelGGL((cache_lists_kernel<false>), grid, dim3(64), 0, s, a, q, top_idx, k, out);
    return launched() ? SAKI_OK : SAKI_ERR_HIP;
  }
  const long long pairs = (long long)B * H_kv * row_blocks;
  if (whole_better(pairs, max_blocks)) {
    const dim3 grid((unsigned)pairs);
    if (dtype == SAKI_F32)
      hipLaunchKernelGGL((cache_attend_kernel<true, false>), grid, dim3(256), 0, s, a, q, out, nullptr);
    else
      hipLaunchKernelGGL((cache_attend_kernel<false, false>), grid, dim3(256), 0, s, a, q, out, nullptr);
    return launched() ? SAKI_OK : SAKI_ERR_HIP;
  }
  const size_t need = saki_cache_attend_workspace_bytes(B, H_q, H_kv, Q, max_blocks, 0);
  if (!ws || ws_bytes < need || !aligned(ws, 16)) return SAKI_ERR_WORKSPACE;
  const int groups = (int)(need / (2 * kPartFloats * sizeof(float)));
  const dim3 join((unsigned)pairs, pairs > 256 ? 1 : kHeadDim / 16);
  if (dtype == SAKI_F32) {
    hipLaunchKernelGGL((cache_attend_kernel<true, true>), dim3(groups), dim3(256), 0, s, a, q, out, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    hipLaunchKernelGGL((cache_join_kernel<true>), join, dim3(256), 0, s, a, groups, (const float*)ws, out);
  } else {
    hipLaunchKernelGGL((cache_attend_kernel<false, true>), dim3(groups), dim3(256), 0, s, a, q, out, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    hipLaunchKernelGGL((cache_join_kernel<false>), join, dim3(256), 0, s, a, groups, (const float*)ws, out);
  }
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

}  // extern "C"
