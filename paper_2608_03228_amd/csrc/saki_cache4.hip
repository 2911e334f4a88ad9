// A paged cache held in 4 bits, for gfx950 (CDNA4, wave64):
//
//   cache4_write_kernel   keys and values to their slots (E2M1 codes, one power-of-two
//                         scale per token and 32 dims)
//   cache4_read_kernel    ranges of the requests' tokens back as float32 or bf16 rows
//   cache4_attend_kernel  attention over every cached key of a request, split evenly
//                         over the GPU; cache4_join_kernel joins the parts
//   cache4_lists_kernel   attention over the keys that a list names

#include "saki_cache4.h"

namespace {

// ---------------------------------------------------------------- writing

// A wave takes eight tokens of one head's keys or values, four at a time, 16 lanes
// a token and 8 dims a lane; four lanes hold a group and find its largest element.
// Four tokens whose slots stand together fill 256 contiguous bytes of codes, in
// either layout.  Groups have their own scales, so that nothing there before is
// read.  HBM bound on prompts: 39,000 float32 tokens of 4 heads (187 MB) in 36 us,
// 5.2 TB/s; bf16 in 21 (a fifth more with four tokens a wave and their loads behind
// the slots').
constexpr int kWriteTokens = 8;  // of a wave
template <typename T>
__global__ __launch_bounds__(256) void cache4_write_kernel(const T* __restrict__ k, const T* __restrict__ v,
                                                           size_t ld_k, size_t ld_v, int n_tokens,
                                                           const int* __restrict__ slots, int n_blocks, int H,
                                                           uint8_t* k_cache, uint8_t* v_cache, uint8_t* scales) {
  constexpr int U = kWriteTokens / 4;
  const int lane = threadIdx.x % kWave;
  const uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
  const uint32_t quad = item / (2 * H) * U, hw = item % (2 * H);
  const int which = hw >= (uint32_t)H, h = which ? hw - H : hw;
  const int m = lane % 16;
  int slot[U];
  float x[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t t = (quad + u) * 4 + lane / 16;
    slot[u] = t < (uint32_t)n_tokens ? slots[t] : -1;
    if (slot[u] >= n_blocks * kTile) slot[u] = -1;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
    if (t < (uint32_t)n_tokens)
      load_elems<T, 8>((which ? v + t * ld_v : k + t * ld_k) + (size_t)h * kHeadDim + 8 * m, x[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[u][e]) & 0x7fffffffu);
    top = max(top, xor_shfl_u32(top, 1));
    top = max(top, xor_shfl_u32(top, 2));
    const uint32_t byte = scale_byte(top);
    const uint32_t codes = encode8(x[u], scale_of(byte));
    if (slot[u] < 0) continue;
    const size_t at = (size_t)(slot[u] / kTile) * H + h;
    const int token = slot[u] % kTile;
    *reinterpret_cast<uint32_t*>((which ? v_cache : k_cache) + at * kCodes4 + code_at(which, token, m)) = codes;
    if (m % 4 == 0) scales[at * kScales4 + (which * kTile + token) * kGroups4 + m / 4] = (uint8_t)byte;
  }
}

// ---------------------------------------------------------------- reading back

// The eight dies' L2s: outputs of that size and more are stored past them.  us, bf16 of
// 8 heads, stores that stay / that do not: 16 MB 6.7 / 6.3, 32 MB 10.0 / 8.4, 64 MB
// 15.9 / 13.4, 128 MB 28.7 / 28.8, 256 MB 66.9 / 53.6; float32 6.5 / 6.3, 9.4 / 7.8,
// 14.8 / 15.0, 26.1 / 27.1, 67.9 / 55.6.
constexpr size_t kL2Bytes = 32u << 20;

struct Read4Args {
  const uint8_t *k, *v, *scales;
  int n_blocks, H;
  const int* tables;
  int max_blocks;
  const int *starts, *cu;
  int B, T;
  void *k_out, *v_out;
  size_t ld_k, ld_v;
};

// Output rows cu[b] .. cu[b + 1] - 1 are request b's tokens from starts[b] on.  A
// work-group takes 16 rows (float32: 8): every wave finds their requests (of up to
// 64 in its lanes; of more 64 told apart at once, then the next 64 one after
// another) and slots, and the waves share the heads' keys and values, 16 bytes of
// output a lane.
//
// Bound by its stores: a wave's fill whole lines, and past what the L2s hold (NT)
// they do not stay there: 472 MB (nine tenths written) in 70 us, 6.7 TB/s (106 with
// stores that stay); 361 MB as bf16 in 55 (75).
template <typename T>
constexpr int read_rows() {
  return 4 * kWave / (kHeadDim * (int)sizeof(T) / 16);
}
template <typename T, bool NT>
__global__ __launch_bounds__(256) void cache4_read_kernel(Read4Args a) {
  constexpr int kReadRows = read_rows<T>();
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int t0 = blockIdx.x * kReadRows, t = t0 + lane % kReadRows;
  auto at = [&](int b) { return min(max(a.cu[b], 0), a.T); };
  // this row's request: its first row and the one behind its last, its first token
  int mine = 0, first, begin, end, start;
  if (a.B <= kWave) {  // all offsets and starts in a wave's lanes, one read deep
    const int c = at(min(lane, a.B)), last = at(a.B), s = a.starts && lane < a.B ? a.starts[lane] : 0;
#pragma unroll
    for (int half = kWave / 2; half; half >>= 1) {
      const int x = __shfl(c, (mine + half) % kWave);
      if (mine + half < a.B && x <= t) mine += half;
    }
    first = __shfl(c, 0);
    begin = __shfl(c, mine), start = __shfl(s, mine);
    end = __shfl(c, (mine + 1) % kWave);
    if (mine + 1 == a.B) end = last;
  } else {
    int b = 0, n = a.B;  // the last request that starts at or before t0 is one of b .. b + n - 1
    while (n > 1) {
      const int step = (n + kWave - 1) / kWave, i = lane * step;
      const uint64_t which = __ballot(i < n && at(b + i) <= t0);
      const int part = which ? (63 - __builtin_clzll(which)) * step : 0;
      n = min(n - part, step);
      b += part;
    }
    mine = b;
    for (int more = b + 1; more < a.B; more += kWave) {  // requests that start within the rows
      const int c = more + lane < a.B ? at(more + lane) : a.T;
      int j = 0;
      for (; j < kWave; ++j) {
        const int s = __builtin_amdgcn_readlane(c, j);
        if (s >= t0 + kReadRows || more + j >= a.B) break;
        if (s <= t) mine = more + j;
      }
      if (j < kWave) break;
    }
    first = at(0), begin = at(mine), end = at(mine + 1), start = a.starts ? a.starts[mine] : 0;
  }
  // (block * H) and token, or where there is no such token: its row is zero
  int blk = -1, token = 0;
  const bool row = t >= first && t < a.T && t < end;
  if (row) {
    const long long p = (long long)start + (t - begin);
    if (p >= 0 && p / kTile < a.max_blocks) {
      const int x = a.tables[(size_t)mine * a.max_blocks + p / kTile];
      if (x >= 0 && x < a.n_blocks) blk = x * a.H, token = (int)(p % kTile);
    }
  }
  const uint64_t rows = __ballot(row);
  if (!rows) return;
  // a lane stores 16 bytes: kDims elements of one row
  constexpr int kDims = 16 / sizeof(T), kLanes = kHeadDim / kDims, kAtOnce = kWave / kLanes;
  constexpr int kLoads = kReadRows / kAtOnce;
  const int c = lane % kLanes, m = c * kDims / 8, q = lane / kLanes;
  int blks[kLoads], tokens[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) blks[u] = __shfl(blk, kAtOnce * u + q), tokens[u] = __shfl(token, kAtOnce * u + q);
  const int from = a.k_out ? 0 : a.H, to = a.v_out ? 2 * a.H : a.H;
  for (int hw = from + blockIdx.y * 4 + wave; hw < to; hw += gridDim.y * 4) {
    const int which = hw >= a.H, h = which ? hw - a.H : hw;
    uint32_t codes[kLoads], s[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      codes[u] = 0, s[u] = 0;
      if (blks[u] >= 0) {
        const size_t x = (size_t)blks[u] + h;
        codes[u] = *reinterpret_cast<const uint32_t*>((which ? a.v : a.k) + x * kCodes4 + code_at(which, tokens[u], m));
        s[u] = a.scales[x * kScales4 + (which * kTile + tokens[u]) * kGroups4 + m / 4];
      }
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = kAtOnce * u + q;
      if (!(rows >> i & 1)) continue;
      T* out = (which ? (T*)a.v_out + (size_t)(t0 + i) * a.ld_v : (T*)a.k_out + (size_t)(t0 + i) * a.ld_k) +
               (size_t)h * kHeadDim + kDims * c;
      uint32_t x[4];
      if constexpr (std::is_same_v<T, float>) {
        const uint32_t four = codes[u] >> (c % 2 * 16);
        const f32x2_t y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(four, scale_of(s[u]), 0);
        const f32x2_t z = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(four, scale_of(s[u]), 1);
        x[0] = __float_as_uint(y[0]), x[1] = __float_as_uint(y[1]);
        x[2] = __float_as_uint(z[0]), x[3] = __float_as_uint(z[1]);
      } else {
        decode8(codes[u], scale_of(s[u]), x);
      }
      typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
      const u32x4_t v = {x[0], x[1], x[2], x[3]};
      if constexpr (NT)
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(out));
      else
        *reinterpret_cast<u32x4_t*>(out) = v;
    }
  }
}

// ---------------------------------------------------------------- attention

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ long long uniform(long long x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (long long)((uint64_t)hi << 32 | lo);
}

constexpr int kTile4 = 2 * kCodes4 + kScales4;  // bytes of a tile: keys, values, scales
constexpr int kAttendGroups4 = 512;             // two a CU

// A sum is scaled down only once a score passes the maximum that it goes by by
// this many powers of two: most tiles that bring a new maximum cost no pass over
// the sums.
constexpr float kSlack = 8.f;

// The value of lane n + N (mod 16) of each 16 lanes.
template <int N>
__device__ __forceinline__ float turned(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + N, 0xf, 0xf, true));
}

// The upper halves of two words as a pair: bf16 of floats, the rest cut off.
__device__ __forceinline__ uint32_t upper(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float cut(float x, uint32_t mask) { return __uint_as_float(__float_as_uint(x) & mask); }

// The three bf16 terms whose sum a float32 is (8 bits each, cut off, not rounded)
// for lanes whose column holds term `term`: RP = 16, one after another; 8, the
// first or second, then the third or none; 4, one of the three or none.
template <int RP>
__device__ __forceinline__ void side_by_side(const float* x, int term, bf16x8_t* to) {
  constexpr uint32_t kUpper = 0xffff0000u;
  constexpr int N = RP == 16 ? 3 : RP / 4;
  uint32_t w[3][4];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float y[3][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float v = x[e + i];
      if constexpr (RP == 4) {
        // (a mask of ones takes all of it away: no term)
        const float r = fmaf(cut(v, term == 3 ? ~0u : kUpper), term == 0 ? 0.f : -1.f, v);
        y[0][i] = fmaf(cut(r, kUpper), term < 2 ? 0.f : -1.f, r);
      } else {
        const float r = v - cut(v, kUpper), z = r - cut(r, kUpper);
        y[0][i] = RP == 16 || term == 0 ? v : r;
        y[1][i] = RP == 16 ? r : cut(z, term == 0 ? ~0u : 0u);
        y[2][i] = z;
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) w[n][e / 2] = upper(y[n][0], y[n][1]);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) __builtin_memcpy(&to[n], w[n], 16);
}
// The upper bits of eight floats (term 0), or what these leave, rounded to bf16.
__device__ __forceinline__ bf16x8_t one_of_two(const float* x, int term) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float y[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float h = cut(x[e + i], 0xffff0000u), r = x[e + i] - h;
      y[i] = term == 0 ? h : r;
    }
    w[e / 2] = pack_bf16(y[0], y[1]);
  }
  bf16x8_t t;
  __builtin_memcpy(&t, w, 16);
  return t;
}

// Scales (four groups' bytes a token, of tokens 16 u + 4 g ..) that must not
// reach a product: those of tokens from `whole` on, and NaN of tokens from `some` on.
__device__ __forceinline__ void hide_values(uint4* e, int g, int whole, int some) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    uint32_t x[4] = {e[u].x, e[u].y, e[u].z, e[u].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 16 * u + 4 * g + i;
      if (t >= some) {
        uint32_t odd = ~x[i];  // bytes of zero: NaN
        odd = ~(((odd & 0x7f7f7f7fu) + 0x7f7f7f7fu) | odd | 0x7f7f7f7fu);  // 0x80 in these
        x[i] = t >= whole ? 0u : x[i] & ~((odd >> 7) * 255u);
      }
    }
    e[u] = make_uint4(x[0], x[1], x[2], x[3]);
  }
}

// As many tiles for each group, divided in 32 bits where they do (in 64 it takes 0.2 us
// of a step's 13), 4 at least, and 8 at least where pairs have more than 256: of one pair's
// 1,563 tiles 391 parts take longer to join (21.0 us in all) than 196 (15.6); of
// 141 tiles it is 10.3 us for 36 parts and 11.2 for 18.
__device__ __forceinline__ Share share4_of(long long total, int groups, long long pairs) {
  Share s;
  s.total = total;
  const long long up = total + groups - 1;
  s.piece = up >> 32 ? up / groups : (uint32_t)up / (uint32_t)groups;
  const int least = total > 256 * pairs ? 2 * kMinPiece : kMinPiece;
  if (s.piece < least) s.piece = least;
  return s;
}
__device__ __forceinline__ long long share4_at(long long tile, const Share& s) {
  return (tile | s.piece) >> 32 ? tile / s.piece : (uint32_t)tile / (uint32_t)s.piece;
}

// s_k = q . key_k / sqrt(d) over a request's keys, softmax, sum of values; shares,
// stretches and parts as in cache_attend_kernel, whose products these are too: S^T
// = K Q^T leaves lane group g (16 lanes) with four scores of one query per 16
// keys, which are at once its operand of O^T = V^T P^T.  Elements are converted to
// bf16 with their scale, exactly; queries (float32: three terms) and weights (two
// terms, three for float32 output) are split, so that nothing but the output is
// rounded to bf16.
//
// A KV group rarely has 16 rows, so that columns are free: with RP rows of 16
// columns the terms stand side by side in one product, column n holding term n /
// RP of row n % RP, and meet as sums over the columns (scores: in the softmax's
// registers; outputs: once at the end).
//
// Each wave brings its tiles (8.7 KB) to LDS by direct loads, one at a time, and has
// them in registers only while they are multiplied: with the next one on its way in
// registers too a wave held 200 of them, and two groups a CU gave 79 us for 8 requests
// of up to 131,072 keys (float32, 28 / 4 heads) and 37.8 for 16 of up to 9,000 and four
// queries (bf16, 32 / 8), where this gives 75.9 and 33.6; 89 and 39.7 with a tile's
// values still on their way while its keys are multiplied, each wait then in the
// middle of the products.  (Both with the join.)  Bound by HBM and by the conversions:
// the 353 MB of the first in 73-74 us, 4.8 TB/s (its loads alone reach 5.4), 706 MB of
// bf16 and 32 / 8 heads in 132 with the join, 5.3; about 400 vector instructions a tile
// and wave, 0.9 us of a SIMD.  A short call is a chain of reads (lengths, table, tile)
// and one tile's products.
//
// Tried: products of the fp4 codes themselves with queries in E4M3 terms (16x16x128,
// scales in the operands) save a sixth of the instructions and 1% of the time, but
// their sums keep about 18 bits: 1.4e-5 off in float32.  Four groups of 128
// registers a CU: 88 us; shares of 640, 768 and 1,024 groups: 86, 80 and 88.
template <bool F32, bool SPLIT, int RP, int W>
__global__ __launch_bounds__(64 * W, W == 8 ? 2 : 3) void cache4_attend_kernel(CacheArgs a, const void* __restrict__ q,
                                                                        void* out, float* __restrict__ ws) {
  // products per step: queries, weights
  constexpr int kQT = F32 ? (RP == 16 ? 3 : RP / 4) : 1, kPT = F32 ? kQT : RP / 8;
  constexpr float kScores = 0.08838834764831845f * kLog2e;  // of a product, in powers of two
  constexpr int kThreads = 64 * W;
  __shared__ alignas(1024) uint8_t lds[W][kTile4];  // a tile of each wave; after the loop:
  float(*const s_o)[16][kHeadDim + 4] = reinterpret_cast<float(*)[16][kHeadDim + 4]>(lds);
  constexpr int kSums = sizeof(float) * W * 16 * (kHeadDim + 4);
  float(*const s_m)[16] = reinterpret_cast<float(*)[16]>(&lds[0][0] + kSums), (*const s_l)[16] = s_m + W;
  static_assert(kSums + 2 * sizeof(float) * W * 16 <= sizeof(lds));
  __shared__ uint4 s_q[4 * kQT][kWave];  // the queries, as the lanes take them
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane % 16, g = lane / 16;
  const int rn = n % RP, term = n / RP;  // this lane's row and term
  const int G = a.H_q / a.H_kv, R = G * a.Q, RB = (R + 15) / 16, pairs = a.H_kv * RB;

  long long cur = 0, end = 1, base = 0;  // the tiles to take, the tiles before request b
  int b = blockIdx.x / pairs, lens = 0;  // (lens: of request `lane` of up to 64)
  if constexpr (SPLIT) {
    long long *const part = reinterpret_cast<long long*>(lds), *const found = part + W;  // (before the loop)
    if (a.B <= kWave) {  // every wave for itself
      const Sums all = wave_sums(a);
      const Share sh = share4_of((long long)all.total * pairs, gridDim.x, (long long)a.B * pairs);
      cur = sh.piece * blockIdx.x;
      end = min(sh.total, cur + sh.piece);
      if (cur >= end) return;
      b = __builtin_ctzll(__ballot(cur < (long long)all.upto * pairs));
      base = (long long)__builtin_amdgcn_readlane(all.upto - all.mine, b) * pairs;
      lens = all.len;
    } else {
      long long total = 0;
      for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int t = b0 + tid < a.B ? tiles_of(a.lens[b0 + tid], a.max_blocks) : 0;
        long long sum;
        group_scan<W>((long long)t * pairs, part, &sum);
        total += sum;
      }
      const Share sh = share4_of(total, gridDim.x, (long long)a.B * pairs);
      cur = sh.piece * blockIdx.x;
      end = min(total, cur + sh.piece);
      if (cur >= end) return;
      for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const long long t = b0 + tid < a.B ? (long long)tiles_of(a.lens[b0 + tid], a.max_blocks) * pairs : 0;
        long long sum;
        const long long upto = base + group_scan<W>(t, part, &sum);
        if (cur < upto && cur >= upto - t) found[0] = b0 + tid, found[1] = upto - t;
        base += sum;
        if (cur < base) break;
      }
      __syncthreads();
      b = (int)found[0];
      base = found[1];
      __syncthreads();  // it is read, before the tiles come
    }
  }

  b = __builtin_amdgcn_readfirstlane(b);  // (these are the same in all lanes)
  cur = uniform(cur), end = uniform(end), base = uniform(base);
  while (cur < end) {
    const int len =
        __builtin_amdgcn_readfirstlane(SPLIT && a.B <= kWave ? __builtin_amdgcn_readlane(lens, b) : a.lens[b]);
    const int nt = tiles_of(len, a.max_blocks);
    if (SPLIT && cur >= base + (long long)nt * pairs) {
      base += (long long)nt * pairs;
      if (++b >= a.B) return;  // (a later request has the tiles that are left)
      continue;
    }
    int pair = blockIdx.x % pairs, t0 = 0;
    if constexpr (SPLIT) {  // (32 bits where they do)
      const long long from = cur - base;
      pair = __builtin_amdgcn_readfirstlane(from >> 32 ? (int)(from / nt) : (int)((uint32_t)from / (uint32_t)nt));
      t0 = __builtin_amdgcn_readfirstlane((int)(from - (long long)pair * nt));
    }
    const int t1 = SPLIT ? __builtin_amdgcn_readfirstlane((int)min((long long)nt, t0 + (end - cur))) : nt;
    const int hk = pair / RB, r0 = pair % RB * 16;
    const size_t row0 = ((size_t)b * a.H_q + (size_t)hk * G) * a.Q + r0;

    // a wave's first tile is asked for before the queries
    const const_int* table = (const const_int*)(uintptr_t)(a.tables + (size_t)b * a.max_blocks);
    auto block_of = [&](int t) __attribute__((always_inline)) {
      const int x = t < t1 ? table[t] : -1;
      return x < a.n_blocks ? x : -1;  // (below 0: none)
    };
    // (block, head)'s bytes to LDS: each lane's 16 where it reads them again
    auto stage = [&](int blk, uint8_t* to) __attribute__((always_inline)) {
      // (the same in all lanes: addresses are a scalar and 32 bits a lane)
      const size_t at = (size_t)blk * a.H_kv + hk;
      const uint8_t *kp = a.k + at * kCodes4, *vp = a.v + at * kCodes4, *sp = (const uint8_t*)a.scales + at * kScales4;
      const uint32_t k_off = n * 64 + g * 16, v_off = lane * 16, s_off = lane * 4;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        __builtin_amdgcn_global_load_lds((global_void*)(kp + u * 1024 + k_off), (lds_void*)(to + u * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_void*)(vp + u * 1024 + v_off), (lds_void*)(to + kCodes4 + u * 1024),
                                         16, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
        __builtin_amdgcn_global_load_lds((global_void*)(sp + u * 256 + s_off),
                                         (lds_void*)(to + 2 * kCodes4 + u * 256), 4, 0, 0);
    };
    uint8_t* const tile = lds[wave];
    int blk = block_of(t0 + wave), next = block_of(t0 + wave + W);
    if (blk >= 0) stage(blk, tile);

    // queries: dims 32 g + 8 s .. + 7 for step s, one of the waves each
    if (wave < 4) {
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      const size_t at = (row0 + rn) * kHeadDim + 32 * g + 8 * wave;
      if (r0 + rn < R) {
        if constexpr (F32)
          load_elems<float, 8>((const float*)q + at, x);
        else
          load_elems<__bf16, 8>((const __bf16*)q + at, x);
      }
      bf16x8_t qf[kQT];
      if constexpr (F32) {
        side_by_side<RP>(x, term, qf);
      } else {
        // an infinite element is taken as NaN, as the row is by the formula: the products may give one infinity
        // for all its scores, which are a row without a key then (the terms of float32 are NaN by themselves)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e], 0.f, x[e]);
        split_bf16<1>(x, qf);
      }
#pragma unroll
      for (int x = 0; x < kQT; ++x) __builtin_memcpy(&s_q[kQT * wave + x][lane], &qf[x], 16);
    }
    __syncthreads();
    const int seen = len - a.Q + (r0 + rn) % a.Q + 1;  // keys that this lane's query sees
    const int least = len - a.Q + 1;

    f32x4_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;  // (m: of the products)
    bool nan = false;              // whether the row sees a NaN value that not all rows see

    // A wave's next tile is asked for as soon as this one's bytes are in registers,
    // and is on its way while the weights are formed and the values multiplied.
    for (int t = t0 + wave; t < t1; t += W) {
      const int after = block_of(t + 2 * W);
      if (blk >= 0) {
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the tile is there
        float p[16];
        f32x4_t acc[4];
        uint32_t c[4][4];
        float f[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // keys 16 u + lane % 16
          acc[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          __builtin_memcpy(c[u], tile + u * 1024 + lane * 16, 16);
          f[u] = scale_of(tile[2 * kCodes4 + (16 * u + n) * kGroups4 + g]);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          bf16x8_t qf[kQT], kf[4];
#pragma unroll
          for (int x = 0; x < kQT; ++x) __builtin_memcpy(&qf[x], &s_q[kQT * s + x][lane], 16);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            uint32_t w[4];
            decode8(c[u][s], f[u], w);
            __builtin_memcpy(&kf[u], w, 16);
          }
#pragma unroll
          for (int x = kQT - 1; x >= 0; --x)
#pragma unroll
            for (int u = 0; u < 4; ++u)
              acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u], qf[x], acc[u], 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[4 * u + i] = acc[u][i];
            if constexpr (F32 && RP <= 8) p[4 * u + i] += turned<8>(p[4 * u + i]);
            if constexpr (F32 && RP == 4) p[4 * u + i] += turned<4>(p[4 * u + i]);
          }
        uint4 vx[4], ve[4];  // values of tokens 16 u + 4 g .., and these tokens' scales
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          vx[u] = *reinterpret_cast<const uint4*>(tile + kCodes4 + u * 1024 + lane * 16);
          ve[u] = *reinterpret_cast<const uint4*>(tile + 2 * kCodes4 + (kTile + 16 * u + 4 * g) * kGroups4);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the tile is read
        __builtin_amdgcn_sched_barrier(0);
        if (next >= 0) stage(next, tile);
        __builtin_amdgcn_sched_barrier(0);
        if ((t + 1) * kTile > least) {  // keys that a query does not see, or that were never written
          const int left = seen - t * kTile, whole = len - t * kTile, some = least - t * kTile;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (16 * (j / 4) + 4 * g + j % 4 >= left) p[j] = -INFINITY;
          // a value times a weight of zero has to be zero: no scale for tokens behind the last, nor NaN where
          // a row may not see it
          hide_values(ve, g, whole, some);
          // that is for the rows that see such a token, in its group's dims (this lane's sums are of dims 32 g ..)
          const uint8_t* vs = (const uint8_t*)a.scales + ((size_t)blk * a.H_kv + hk) * kScales4 + kTile * kGroups4;
          for (int j = max(some, 0); j < min(whole, kTile); ++j) nan |= vs[j * kGroups4 + g] == 255 && j < left;
        }
        float top = p[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) top = fmaxf(top, p[j]);
        top = fmaxf(top, xor_f32(top, 16));
        top = fmaxf(top, xor_f32(top, 32));
        if (__any(top > m + kSlack / kScores)) {
          const float m1 = fmaxf(m, top);
          float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m1) * kScores);
          asm volatile("" : "+v"(keep));  // (the products below stay in the branch)
          m = m1;
          l *= keep;
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] *= keep;
        }
        const float shift = m == -INFINITY ? 0.f : -m * kScores;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          p[j] = __builtin_amdgcn_exp2f(fmaf(p[j], kScores, shift));
          sum += p[j];
        }
        l += sum;
        // brings the group's byte of a token's scales to the exponent's place (the rest is ignored)
        const int turn = (n / 4 * 8 + 9) % 32;
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // tokens 32 half + 4 g .. + 3 and + 16 .. + 19 of the lane
          bf16x8_t pt[kPT];
          if constexpr (F32) {
            side_by_side<RP>(p + 8 * half, term, pt);
          } else if constexpr (RP == 8) {
            pt[0] = one_of_two(p + 8 * half, term);
          } else {
            split_bf16<kPT>(p + 8 * half, pt);
          }
          uint32_t c[8];
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint4 x = vx[2 * half + i / 4], e = ve[2 * half + i / 4];
            const uint32_t s = i % 4 == 0 ? e.x : i % 4 == 1 ? e.y : i % 4 == 2 ? e.z : e.w;
            c[i] = i % 4 == 0 ? x.x : i % 4 == 1 ? x.y : i % 4 == 2 ? x.z : x.w;
            f[i] = __uint_as_float(__builtin_amdgcn_alignbit(s, s, turn));
          }
#pragma unroll
          for (int y = 0; y < 4; ++y) {  // dims 8 m + 2 y, + 1
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = y == 0   ? decode2<0>(c[i], f[i])
                                               : y == 1 ? decode2<1>(c[i], f[i])
                                               : y == 2 ? decode2<2>(c[i], f[i])
                                                        : decode2<3>(c[i], f[i]);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              uint32_t r[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)  // v_perm_b32(hi, lo, sel): the low or high halves of two tokens
                r[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], x ? 0x07060302u : 0x05040100u);
              bf16x8_t vv;
              __builtin_memcpy(&vv, r, 16);
#pragma unroll
              for (int z = kPT - 1; z >= 0; --z)
                o[2 * y + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pt[z], o[2 * y + x], 0, 0, 0);
            }
          }
        }
      } else if (next >= 0) {
        stage(next, tile);
      }
      blk = next;
      next = after;
    }

    // the waves' parts: lane (n, g) holds dims 8 (4 g + i) + j of row n in o[j][i]
    l += xor_f32(l, 16);
    l += xor_f32(l, 32);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (nan) o[j][i] = NAN;
        if constexpr (RP <= 8) o[j][i] += turned<8>(o[j][i]);
        if constexpr (RP == 4) o[j][i] += turned<4>(o[j][i]);
      }
    __syncthreads();  // all waves' tiles are read
    if (g == 0) s_m[wave][n] = m * kScores, s_l[wave][n] = l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* p = &s_o[wave][n][8 * (4 * g + i)];
      *reinterpret_cast<float4*>(p) = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
      *reinterpret_cast<float4*>(p + 4) = make_float4(o[4][i], o[5][i], o[6][i], o[7][i]);
    }
    __syncthreads();
    constexpr int kDims = 16 * kHeadDim / kThreads;  // of a thread
    const int row = tid / (kHeadDim / kDims), d0 = tid % (kHeadDim / kDims) * kDims;
    float M = -INFINITY, L = 0.f, y[kDims];
#pragma unroll
    for (int j = 0; j < kDims; ++j) y[j] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, s_m[w][row]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float e = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][row] - M);
      L += s_l[w][row] * e;
#pragma unroll
      for (int j = 0; j < kDims; ++j) y[j] += s_o[w][row][d0 + j] * e;
    }
    if (r0 + row < R) {
      if (!SPLIT || (t0 == 0 && t1 == nt)) {
        const float inv = L == 0.f ? 0.f : 1.f / L;  // (a NaN stays one)
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
    __syncthreads();  // the parts are read, before the next stretch's tiles come
  }
}

// Joins the parts of the pairs that several work-groups shared, and writes zeros
// for requests without a key.  A work-group takes 16 dims of a pair (all dims, 16
// at a time, above 256 pairs); each of its waves takes every kJoinWaves-th part, four
// parts' loads at once: a part after another, one request of one head (391 parts of
// 100,000 keys) took 40 us.
constexpr int kJoinParts = 4;
template <bool F32, int kJoinWaves>
__global__ __launch_bounds__(64 * kJoinWaves) void cache4_join_kernel(CacheArgs a, int groups,
                                                                     const float* __restrict__ ws, void* out) {
  __shared__ long long part[kJoinWaves], s_base;
  __shared__ float s_m[kJoinWaves][16], s_l[kJoinWaves][16], s_y[kJoinWaves][16][16];
  constexpr int kThreads = 64 * kJoinWaves;
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
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
      const int t = b0 + tid < a.B ? tiles_of(a.lens[b0 + tid], a.max_blocks) : 0;
      long long sum;
      const long long upto = group_scan<kJoinWaves>((long long)t * pairs, part, &sum);
      if (b0 + tid == b) s_base = total + upto - (long long)t * pairs;
      total += sum;
    }
    __syncthreads();
    nt = tiles_of(a.lens[b], a.max_blocks);
    base = s_base;
  }
  const Share sh = share4_of(total, groups, (long long)a.B * pairs);
  const long long from = base + (long long)nt * pair;
  const int w0 = (int)share4_at(from, sh), w1 = nt ? (int)share4_at(from + nt - 1, sh) : w0;
  if (nt && w0 == w1) return;
  const int row = lane / 4;
  const int hk = pair / RB, r0 = pair % RB * 16;
  const bool in = r0 + row < R;
  for (int part16 = blockIdx.y; part16 < kHeadDim / 16; part16 += gridDim.y) {
    const int d0 = part16 * 16 + lane % 4 * 4;
    float M = -INFINITY, L = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    if (nt && in)
      for (int w = w0 + wave; w <= w1; w += kJoinWaves * kJoinParts) {
        float m[kJoinParts], l[kJoinParts];
        float4 x[kJoinParts];
#pragma unroll
        for (int i = 0; i < kJoinParts; ++i) {
          const int u = w + i * kJoinWaves;
          m[i] = -INFINITY, l[i] = 0.f, x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (u <= w1) {
            const float* p = ws + ((size_t)u * 2 + (u == w0)) * kPartFloats;
            m[i] = p[kPartRows * kHeadDim + row], l[i] = p[kPartRows * kHeadDim + kPartRows + row];
            x[i] = *reinterpret_cast<const float4*>(p + row * kHeadDim + d0);
          }
        }
        float m1 = M;
#pragma unroll
        for (int i = 0; i < kJoinParts; ++i) m1 = fmaxf(m1, m[i]);
        const float ref = m1 == -INFINITY ? 0.f : m1, e0 = __builtin_amdgcn_exp2f(M - ref);
        M = m1;
        L *= e0;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] *= e0;
#pragma unroll
        for (int i = 0; i < kJoinParts; ++i) {
          const float e = __builtin_amdgcn_exp2f(m[i] - ref);
          L += l[i] * e;
          y[0] += x[i].x * e, y[1] += x[i].y * e, y[2] += x[i].z * e, y[3] += x[i].w * e;
        }
      }
    __syncthreads();  // the last dims are read
    s_m[wave][row] = M, s_l[wave][row] = L;  // equal from a row's four lanes
#pragma unroll
    for (int j = 0; j < 4; ++j) s_y[wave][row][lane % 4 * 4 + j] = y[j];
    __syncthreads();
    const int r = tid / 16, d = tid % 16;
    if (r >= 16 || r0 + r >= R) continue;  // (256 threads write)
    M = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) M = fmaxf(M, s_m[w][r]);
    float sum = 0.f;
    L = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) {
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
// looks up entry e.  Few rows are latency bound, by the addresses that a load
// has to translate: a page an entry and array.  So a key's 64 bytes are read by
// four lanes, 16 entries a load; a value's 256 (with the three tokens between) by
// 16 lanes, four entries a load; and both scales of 32 entries by one load: 256
// rows over 131,072 keys in 6.4 us as calls in a row, 16.2 with four lanes a value
// and scales of their own.
template <bool F32>
__global__ __launch_bounds__(64) void cache4_lists_kernel(CacheArgs a, const void* __restrict__ q,
                                                           const int* __restrict__ top_idx, int k,
                                                           void* __restrict__ out) {
  using T = std::conditional_t<F32, float, __bf16>;
  const int lane = threadIdx.x % kWave;
  const size_t r = blockIdx.x;
  const int i = (int)(r % a.Q), h = (int)(r / a.Q % a.H_q), b = (int)(r / a.Q / a.H_q);
  const int hk = h / (a.H_q / a.H_kv);
  const long long seen = (long long)a.lens[b] - a.Q + i + 1;
  int at = -1;  // the entry's row of the cache
  const int j = lane < k ? top_idx[r * k + lane] : -1;
  if (j >= 0 && j < seen && j / kTile < a.max_blocks) {
    const int blk = a.tables[(size_t)b * a.max_blocks + j / kTile];
    if (blk >= 0 && blk < a.n_blocks) at = (blk * a.H_kv + hk) * kTile + j % kTile;
  }
  // keys: group c of entry 16 u + e0; values: dims 8 m .. of entry 4 u + g
  const int c = lane % 4, e0 = lane / 4, m = lane % 16, g = lane / 16;
  float qx[32];
  load_elems<T, 32>((const T*)q + r * kHeadDim + 32 * c, qx);
  float odd = 0.f;  // NaN where an element is not finite: the row is, also where all its scores are -infinity
#pragma unroll
  for (int e = 0; e < 32; ++e) odd = fmaf(qx[e], 0.f, odd);
  uint4 kx[4];
  uint32_t vx[16], se[2];  // se: the keys' scales of entries 32 u + lane (lanes 0 .. 31), the values' (32 .. 63)
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int row = __shfl(at, 16 * u + e0);
    kx[u] = make_uint4(0u, 0u, 0u, 0u);
    if (row >= 0)
      kx[u] = *reinterpret_cast<const uint4*>(a.k + (size_t)(row / kTile) * kCodes4 + code_at(0, row % kTile, 4 * c));
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int row = __shfl(at, 32 * u + lane % 32);
    se[u] = 0;
    if (row >= 0)
      se[u] = *reinterpret_cast<const uint32_t*>((const uint8_t*)a.scales + (size_t)(row / kTile) * kScales4 +
                                                 (lane / 32 * kTile + row % kTile) * kGroups4);
  }
#pragma unroll
  for (int u = 0; u < 16; ++u) {
    const int row = __shfl(at, 4 * u + g);
    vx[u] = 0;
    if (row >= 0)
      vx[u] = *reinterpret_cast<const uint32_t*>(a.v + (size_t)(row / kTile) * kCodes4 + code_at(1, row % kTile, m));
  }
  float p[4], top = -INFINITY;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t w[4] = {kx[u].x, kx[u].y, kx[u].z, kx[u].w};
    const float f = scale_of((uint32_t)__shfl((int)se[u / 2], 16 * (u % 2) + e0) >> (8 * c) & 255);
    float s = odd;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float y[8];
      decode8(w[x], f, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(y[e], qx[8 * x + e], s);
    }
    s += xor_f32(s, 1);
    s += xor_f32(s, 2);
    p[u] = __shfl(at, 16 * u + e0) >= 0 ? s * (0.08838834764831845f * kLog2e) : -INFINITY;
    top = fmaxf(top, p[u]);
  }
#pragma unroll
  for (int x = 4; x < kWave; x <<= 1) top = fmaxf(top, xor_f32(top, x));
  if (top == -INFINITY) top = 0.f;
  float l = 0.f, o[8];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    p[u] = __builtin_amdgcn_exp2f(p[u] - top);
    l += p[u];
  }
#pragma unroll
  for (int x = 4; x < kWave; x <<= 1) l += xor_f32(l, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
  for (int u = 0; u < 16; ++u) {
    const float w = __shfl(p[u / 4], 16 * (u % 4) + 4 * g);
    const float f = scale_of((uint32_t)__shfl((int)se[u / 8], 32 + 4 * (u % 8) + g) >> (8 * (m / 4)) & 255);
    float y[8];
    decode8(vx[u], f, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(w, y[e], o[e]);
  }
  // sums over the four lanes of equal m, each step halving the dims a lane keeps
  int d0 = 8 * m;
#pragma unroll
  for (int x = 32, w = 4; x >= 16; x >>= 1, w >>= 1) {
    const bool up = lane & x;
#pragma unroll
    for (int e = 0; e < w; ++e) {
      const float give = up ? o[e] : o[e + w], mine = up ? o[e + w] : o[e];
      o[e] = mine + xor_f32(give, x);
    }
    d0 += up ? w : 0;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (F32)
    *reinterpret_cast<float2*>((float*)out + r * kHeadDim + d0) = make_float2(o[0] * inv, o[1] * inv);
  else
    *reinterpret_cast<uint32_t*>((__bf16*)out + r * kHeadDim + d0) = pack_bf16(o[0] * inv, o[1] * inv);
}

// ---------------------------------------------------------------- argument checks

int attend4_groups(long long tiles) {
  const long long g = (tiles + kMinPiece - 1) / kMinPiece;
  return (int)(g < 1 ? 1 : g > kAttendGroups4 ? kAttendGroups4 : g);
}

// R rows of a KV group: as many terms side by side as their columns leave room for.
// W waves a work-group.
template <bool F32, bool SPLIT, int W>
void launch_attend4(int R, dim3 grid, hipStream_t s, const CacheArgs& a, const void* q, void* out, float* ws) {
  if (F32 && R <= 4)
    hipLaunchKernelGGL((cache4_attend_kernel<F32, SPLIT, F32 ? 4 : 8, W>), grid, dim3(64 * W), 0, s, a, q, out, ws);
  else if (R <= 8)
    hipLaunchKernelGGL((cache4_attend_kernel<F32, SPLIT, 8, W>), grid, dim3(64 * W), 0, s, a, q, out, ws);
  else
    hipLaunchKernelGGL((cache4_attend_kernel<F32, SPLIT, 16, W>), grid, dim3(64 * W), 0, s, a, q, out, ws);
}

// Eight waves a pair for less than 64 pairs.  us in all (bf16, 32 / 8 heads, lengths of
// a quarter to the whole of the width), eight waves / four: 8 pairs of 600 tiles 18.0 /
// 18.9, 32 24.6 / 24.9, 64 40.9 / 40.2; of 200 tiles 12.2 / 12.6, 16.7 / 16.9, 23.5 /
// 22.9, 128 pairs 31.8 / 30.3, 256 56.0 / 53.2.
template <bool F32>
void launch_join4(unsigned pairs, hipStream_t s, const CacheArgs& a, int groups, const float* ws, void* out) {
  const dim3 grid(pairs, pairs > 256 ? 1 : kHeadDim / 16);
  if (pairs < 64)
    hipLaunchKernelGGL((cache4_join_kernel<F32, 8>), grid, dim3(512), 0, s, a, groups, ws, out);
  else
    hipLaunchKernelGGL((cache4_join_kernel<F32, 4>), grid, dim3(256), 0, s, a, groups, ws, out);
}

// Whether a work-group takes a whole pair, with no join, and whether with eight
// waves in place of four (at most one pair a CU, and enough tiles for them).  The
// lengths are read on the device, so the tables' width has to bound a group's
// time.  us (bf16, 32 / 8 heads, lengths of a quarter to the whole of the width, calls
// in a row), four waves / eight / split and joined:
//                 8 tiles              16                   32                   64
//    8 pairs   5.9 /  5.9 /  9.3    8.2 /  7.7 /  9.4   12.8 / 11.2 /  9.7   22.1 / 18.4 / 10.1
//   32         6.4 /  6.5 / 12.7    8.6 /  8.2 / 12.7   13.3 / 11.8 / 13.4   23.9 / 20.0 / 15.7
//   64         6.5 /  6.7 / 12.9    8.9 /  8.5 / 13.4   14.4 / 12.7 / 16.1   24.2 / 20.2 / 18.9
//  128         6.7 /  6.7 / 14.2    9.6 /  9.4 / 16.3   14.6 / 13.2 / 18.4   24.2 / 20.7 / 21.6
//  256         7.6 /  7.8 / 18.0   10.4 / 10.6 / 19.9   15.4 / 14.8 / 25.0   25.6 / 23.0 / 29.1
//  512        10.5 / 13.3 / 25.4   14.0 / 17.4 / 28.2   21.6 / 24.3 / 35.0   41.3 / 42.7 / 51.5
// 1024        16.3 / 23.4 / 35.8   22.8 / 31.5 / 44.8   40.7 / 47.6 / 62.3
// float32, 28 / 4 heads: 4 pairs of 16 and 24 tiles 9.4 / 8.9 / 9.9 and 12.4 / 11.3 /
// 10.3; 32 of 32 and 48 16.3 / 14.5 / 14.7 and 21.7 / 19.0 / 15.0; 256 of 48 23.8 /
// 21.6 / 28.2.  512 pairs of 96 tiles 49.8 / 48.4 / 55.5, 1,024 of 64 and 96 76.2 /
// 76.0 / 84.9 and 114 / 108 / 118: many pairs would gain further still, but one long
// request among short ones keeps its groups at work alone (512 pairs, one request of
// 48, 64 and 96 tiles and the others of 5: 18.1 / 23.0, 22.7 / 23.1 and 32.5 / 26.5
// with four waves and split).
bool whole4_better(long long pairs, int max_blocks) {
  return max_blocks <= (pairs >= 512 ? 96 : pairs >= 128 ? 64 : pairs >= 64 ? 48 : pairs >= 16 ? 32 : 20);
}
bool eight4_better(long long pairs, int max_blocks) {
  return pairs <= 256 && max_blocks > (pairs > 128 ? 16 : 8);
}

template <typename T>
int launch_read4(const Read4Args& a, hipStream_t s) {
  const int sides = a.k_out && a.v_out ? 2 : 1;
  // some 2,000 work-groups while the heads allow it (us for 512, 1,024, 2,048 and 4,096 of them: 2,000 bf16 tokens
  // of 32 heads 11.2, 10.3, 10.0, 10.0; 8,000 of 8 10.5, 9.9, 9.8, 9.8; few tokens alike)
  const int blocks = (a.T + read_rows<T>() - 1) / read_rows<T>(), most = (sides * a.H + 3) / 4;
  int split = 2048 / blocks;
  split = split < 1 ? 1 : split > most ? most : split;
  const dim3 grid(blocks, split);
  if ((size_t)a.T * sides * a.H * kHeadDim * sizeof(T) >= kL2Bytes)
    hipLaunchKernelGGL((cache4_read_kernel<T, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((cache4_read_kernel<T, false>), grid, dim3(256), 0, s, a);
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

}  // namespace

extern "C" {

int saki_cache4_write(const void* k, const void* v, int dtype, int T, int H_kv, int d, size_t ld_k, size_t ld_v,
                      const int* slots, void* k_cache, void* v_cache, void* scales, int n_blocks, void* stream) {
  if (T < 0 || d <= 0) return SAKI_ERR_ARG;
  const int st = check_cache4(k_cache, v_cache, scales, n_blocks, H_kv);
  if (st != SAKI_OK) return st;
  if (d != kHeadDim || !type_ok(dtype) || T > kMaxTokens) return SAKI_ERR_UNSUPPORTED;
  if (T == 0) return SAKI_OK;
  if (!slots || !rows_ok(k, ld_k, H_kv, dtype) || !rows_ok(v, ld_v, H_kv, dtype)) return SAKI_ERR_ARG;
  if (n_blocks == 0) return SAKI_OK;  // no slot is within it
  const size_t codes = (size_t)n_blocks * H_kv * kCodes4, n_scales = (size_t)n_blocks * H_kv * kScales4;
  if (overlap(k_cache, codes, v_cache, codes) || overlap(k_cache, codes, scales, n_scales) ||
      overlap(v_cache, codes, scales, n_scales))
    return SAKI_ERR_ARG;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // tokens a launch: its waves in 2^23 work-groups at most
  const int most = (int)((1LL << 25) / (2 * H_kv)) * kWriteTokens;
  for (int t = 0; t < T; t += most) {
    const int n = T - t < most ? T - t : most;
    const long long items = (long long)((n + kWriteTokens - 1) / kWriteTokens) * 2 * H_kv;
    const dim3 grid((unsigned)((items + 3) / 4));
    if (dtype == SAKI_F32)
      hipLaunchKernelGGL((cache4_write_kernel<float>), grid, dim3(256), 0, s, (const float*)k + t * ld_k,
                         (const float*)v + t * ld_v, ld_k, ld_v, n, slots + t, n_blocks, H_kv, (uint8_t*)k_cache,
                         (uint8_t*)v_cache, (uint8_t*)scales);
    else
      hipLaunchKernelGGL((cache4_write_kernel<__bf16>), grid, dim3(256), 0, s, (const __bf16*)k + t * ld_k,
                         (const __bf16*)v + t * ld_v, ld_k, ld_v, n, slots + t, n_blocks, H_kv, (uint8_t*)k_cache,
                         (uint8_t*)v_cache, (uint8_t*)scales);
    if (!launched()) return SAKI_ERR_HIP;
  }
  return SAKI_OK;
}

int saki_cache4_read(const void* k_cache, const void* v_cache, const void* scales, int n_blocks, const int* tables,
                     int max_blocks, const int* starts, const int* cu, int B, int T, int H_kv, int d, int dtype,
                     void* k_out, void* v_out, size_t ld_k, size_t ld_v, void* stream) {
  if (T < 0 || B < 0 || d <= 0 || max_blocks <= 0) return SAKI_ERR_ARG;
  const int st = check_cache4(k_cache, v_cache, scales, n_blocks, H_kv);
  if (st != SAKI_OK) return st;
  if (d != kHeadDim || !type_ok(dtype) || T > kMaxTokens || max_blocks > INT_MAX / kTile - 1)
    return SAKI_ERR_UNSUPPORTED;
  if (T == 0 || B == 0 || (!k_out && !v_out)) return SAKI_OK;
  if (!tables || !cu || (k_out && !rows_ok(k_out, ld_k, H_kv, dtype)) ||
      (v_out && !rows_ok(v_out, ld_v, H_kv, dtype)))
    return SAKI_ERR_ARG;
  const Read4Args a{(const uint8_t*)k_cache, (const uint8_t*)v_cache, (const uint8_t*)scales, n_blocks, H_kv, tables,
                    max_blocks, starts, cu, B, T, k_out, v_out, ld_k, ld_v};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return dtype == SAKI_F32 ? launch_read4<float>(a, s) : launch_read4<__bf16>(a, s);
}

size_t saki_cache4_attend_workspace_bytes(int B, int H_q, int H_kv, int Q, int max_blocks, int k) {
  if (B <= 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || Q < 0 || Q > SAKI_CACHE_MAX_Q || max_blocks <= 0 || k < 0 ||
      k > saki::kMaxK)
    return 0;
  const long long row_blocks = ((long long)(H_q / H_kv) * Q + 15) / 16;
  if (k > 0 || Q == 0 || whole4_better((long long)B * H_kv * row_blocks, max_blocks)) return 256;
  const double tiles = (double)B * H_kv * row_blocks * max_blocks;
  const int groups = attend4_groups(tiles > 1e9 ? 1000000000LL : (long long)tiles);
  return (size_t)groups * 2 * kPartFloats * sizeof(float);
}

int saki_cache4_attend(const void* q, int dtype, int B, int H_q, int H_kv, int Q, int d, const void* k_cache,
                       const void* v_cache, const void* scales, int n_blocks, const int* tables, int max_blocks,
                       const int* lens, const int* top_idx, int k, void* out, void* ws, size_t ws_bytes,
                       void* stream) {
  if (B <= 0 || H_q <= 0 || H_kv <= 0 || H_q % H_kv != 0 || Q < 0 || d <= 0 || max_blocks <= 0 || k < 0 ||
      (top_idx != nullptr) != (k > 0))
    return SAKI_ERR_ARG;
  const int st = check_cache4(k_cache, v_cache, scales, n_blocks, H_kv);
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
      hipLaunchKernelGGL((cache4_lists_kernel<true>), grid, dim3(64), 0, s, a, q, top_idx, k, out);
    else
      hipLaunchKernelGGL((cache4_lists_kernel<false>), grid, dim3(64), 0, s, a, q, top_idx, k, out);
    return launched() ? SAKI_OK : SAKI_ERR_HIP;
  }
  const long long pairs = (long long)B * H_kv * row_blocks;
  const int R = H_q / H_kv * Q;
  if (whole4_better(pairs, max_blocks)) {
    const dim3 grid((unsigned)pairs);
    const bool eight = eight4_better(pairs, max_blocks);
    if (dtype == SAKI_F32) {
      if (eight)
        launch_attend4<true, false, 8>(R, grid, s, a, q, out, nullptr);
      else
        launch_attend4<true, false, 4>(R, grid, s, a, q, out, nullptr);
    } else {
      if (eight)
        launch_attend4<false, false, 8>(R, grid, s, a, q, out, nullptr);
      else
        launch_attend4<false, false, 4>(R, grid, s, a, q, out, nullptr);
    }
    return launched() ? SAKI_OK : SAKI_ERR_HIP;
  }
  const size_t need = saki_cache4_attend_workspace_bytes(B, H_q, H_kv, Q, max_blocks, 0);
  if (!ws || ws_bytes < need || !aligned(ws, 16)) return SAKI_ERR_WORKSPACE;
  const int groups = (int)(need / (2 * kPartFloats * sizeof(float)));
  if (dtype == SAKI_F32) {
    launch_attend4<true, true, 4>(R, dim3(groups), s, a, q, out, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    launch_join4<true>((unsigned)pairs, s, a, groups, (const float*)ws, out);
  } else {
    launch_attend4<false, true, 4>(R, dim3(groups), s, a, q, out, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    launch_join4<false>((unsigned)pairs, s, a, groups, (const float*)ws, out);
  }
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

}  // extern "C"
