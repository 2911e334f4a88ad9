// A paged cache held in 4 bits, for gfx950 (CDNA4, wave64):
//
//   cache4_write_kernel   keys and values to their slots (E2M1 codes, one power-of-two
//                         scale per token and 32 dims)
//   cache4_read_kernel    ranges of the requests' tokens back as float32 or bf16 rows
//   cache4_attend_kernel  attention over every cached key of a request, split evenly
//                         over the GPU; cache_join_kernel joins the parts
//   cache4_lists_kernel   attention over the keys that a list names

#include "saki_cache4.h"

namespace {

// ---------------------------------------------------------------- writing

// A wave takes four tokens of one head's keys or values, 16 lanes a token and 8
// dims a lane; four lanes hold a group and find its largest element.  Four tokens
// whose slots stand together fill 256 contiguous bytes of codes, in either
// layout.  Groups have their own scales, so that nothing there before is read.
template <typename T>
__global__ __launch_bounds__(256) void cache4_write_kernel(const T* __restrict__ k, const T* __restrict__ v,
                                                           size_t ld_k, size_t ld_v, int n_tokens,
                                                           const int* __restrict__ slots, int n_blocks, int H,
                                                           uint8_t* k_cache, uint8_t* v_cache, uint8_t* scales) {
  const int lane = threadIdx.x % kWave;
  const uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
  const uint32_t quad = item / (2 * H), hw = item % (2 * H);
  const int which = hw >= (uint32_t)H, h = which ? hw - H : hw;
  const uint32_t t = quad * 4 + lane / 16;
  const int m = lane % 16;
  const int slot = t < (uint32_t)n_tokens ? slots[t] : -1;
  const bool in = slot >= 0 && slot < n_blocks * kTile;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (in) load_elems<T, 8>((which ? v + t * ld_v : k + t * ld_k) + (size_t)h * kHeadDim + 8 * m, x);
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, xor_shfl_u32(top, 1));
  top = max(top, xor_shfl_u32(top, 2));
  const uint32_t byte = scale_byte(top);
  const uint32_t codes = encode8(x, scale_of(byte));
  if (!in) return;
  const size_t at = (size_t)(slot / kTile) * H + h;
  const int token = slot % kTile;
  *reinterpret_cast<uint32_t*>((which ? v_cache : k_cache) + at * kCodes4 + code_at(which, token, m)) = codes;
  if (m % 4 == 0) scales[at * kScales4 + (which * kTile + token) * kGroups4 + m / 4] = (uint8_t)byte;
}

// ---------------------------------------------------------------- reading back

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
// work-group takes 16 rows: every wave finds their requests (64 offsets told
// apart at once, then the next 64 one after another) and slots, and the waves
// share the heads' keys and values, four tokens of one head a load.
constexpr int kReadRows = 16;
template <typename T>
__global__ __launch_bounds__(256) void cache4_read_kernel(Read4Args a) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int t0 = blockIdx.x * kReadRows, t = t0 + lane % kReadRows;
  auto at = [&](int b) { return min(max(a.cu[b], 0), a.T); };
  int b = 0, n = a.B;  // the last request that starts at or before t0 is one of b .. b + n - 1
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave, i = lane * step;
    const uint64_t which = __ballot(i < n && at(b + i) <= t0);
    const int part = which ? (63 - __builtin_clzll(which)) * step : 0;
    n = min(n - part, step);
    b += part;
  }
  const int first = at(0);
  int mine = b;
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
  // (block * H) and token, or where there is no such token: its row is zero
  int blk = -1, token = 0;
  const bool row = t >= first && t < a.T && t < at(mine + 1);
  if (row) {
    const long long p = (long long)(a.starts ? a.starts[mine] : 0) + (t - at(mine));
    if (p >= 0 && p / kTile < a.max_blocks) {
      const int x = a.tables[(size_t)mine * a.max_blocks + p / kTile];
      if (x >= 0 && x < a.n_blocks) blk = x * a.H, token = (int)(p % kTile);
    }
  }
  const uint64_t rows = __ballot(row);
  if (!rows) return;
  const int m = lane % 16, q = lane / 16;
  constexpr int kQuads = kReadRows / 4;
  int blks[kQuads], tokens[kQuads];
#pragma unroll
  for (int u = 0; u < kQuads; ++u) blks[u] = __shfl(blk, 4 * u + q), tokens[u] = __shfl(token, 4 * u + q);
  const int from = a.k_out ? 0 : a.H, to = a.v_out ? 2 * a.H : a.H;
  for (int hw = from + blockIdx.y * 4 + wave; hw < to; hw += gridDim.y * 4) {
    const int which = hw >= a.H, h = which ? hw - a.H : hw;
    uint32_t codes[kQuads], s[kQuads];
#pragma unroll
    for (int u = 0; u < kQuads; ++u) {
      codes[u] = 0, s[u] = 0;
      if (blks[u] >= 0) {
        const size_t x = (size_t)blks[u] + h;
        codes[u] = *reinterpret_cast<const uint32_t*>((which ? a.v : a.k) + x * kCodes4 + code_at(which, tokens[u], m));
        s[u] = a.scales[x * kScales4 + (which * kTile + tokens[u]) * kGroups4 + m / 4];
      }
    }
#pragma unroll
    for (int u = 0; u < kQuads; ++u) {
      const int i = 4 * u + q;
      if (!(rows >> i & 1)) continue;
      T* out = (which ? (T*)a.v_out + (size_t)(t0 + i) * a.ld_v : (T*)a.k_out + (size_t)(t0 + i) * a.ld_k) +
               (size_t)h * kHeadDim + 8 * m;
      if constexpr (std::is_same_v<T, float>) {
        float x[8];
        decode8(codes[u], scale_of(s[u]), x);
        store_elems<float, 8>(out, x);
      } else {
        uint32_t x[4];
        decode8(codes[u], scale_of(s[u]), x);
        *reinterpret_cast<uint4*>(out) = make_uint4(x[0], x[1], x[2], x[3]);
      }
    }
  }
}

// ---------------------------------------------------------------- attention

// s_k = q . key_k / sqrt(d) over a request's keys, softmax, sum of values; shares,
// stretches and parts as in cache_attend_kernel, whose products these are too: S^T
// = K Q^T leaves lane group g (16 lanes) with four scores of one query per 16
// keys, which are at once its operand of O^T = V^T P^T.  Elements are converted to
// bf16 with their scale, exactly; queries (float32: three terms) and weights (two
// terms, three for float32 output) are split, so that nothing but the output is
// rounded to bf16.
template <bool F32, bool SPLIT>
__global__ __launch_bounds__(256, 2) void cache4_attend_kernel(CacheArgs a, const void* __restrict__ q, void* out,
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

    // queries: dims 32 g + 8 s .. + 7 for step s
    bf16x8_t qf[4][kQT];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      const size_t at = (row0 + n) * kHeadDim + 32 * g + 8 * s;
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
      const size_t at = (size_t)blk * a.H_kv + hk;
      const uint8_t* kp = a.k + at * kCodes4 + lane % 16 * 64 + g * 16;
      const uint8_t* vp = a.v + at * kCodes4 + lane * 16;
      const uint8_t* ks = (const uint8_t*)a.scales + at * kScales4;
      const uint8_t* vs = ks + kTile * kGroups4;
      uint4 kx[4], vx[4], ve[4];
      uint32_t ke[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {  // keys 16 u + lane % 16, values of tokens 16 u + 4 g ..
        kx[u] = *reinterpret_cast<const uint4*>(kp + u * 1024);
        ke[u] = ks[(16 * u + n) * kGroups4 + g];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        vx[u] = *reinterpret_cast<const uint4*>(vp + u * 1024);
        ve[u] = *reinterpret_cast<const uint4*>(vs + (16 * u + 4 * g) * kGroups4);
      }

      float p[16];
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
        const float f = scale_of(ke[u]);
        const uint32_t c[4] = {kx[u].x, kx[u].y, kx[u].z, kx[u].w};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          uint32_t w[4];
          decode8(c[s], f, w);
          bf16x8_t kf;
          __builtin_memcpy(&kf, w, 16);
#pragma unroll
          for (int x = kQT - 1; x >= 0; --x) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[s][x], acc, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) p[4 * u + i] = acc[i] * (0.08838834764831845f * kLog2e);
      }
      // scales of values 4 u + c of the lane: byte m / 4 of a token's four, to the exponent's place
      float vf[16];
      const int turn = (n / 4 * 8 + 9) % 32;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t c[4] = {ve[u].x, ve[u].y, ve[u].z, ve[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vf[4 * u + i] = __uint_as_float(__builtin_amdgcn_alignbit(c[i], c[i], turn) & 0x7f800000u);
      }
      bool nan = false;
      if ((t + 1) * kTile > least) {  // keys that a query does not see, or that were never written
        const int left = seen - t * kTile - 4 * g, some = least - t * kTile - 4 * g, whole = len - t * kTile - 4 * g;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int at16 = 16 * (j / 4) + j % 4;
          if (at16 >= left) p[j] = -INFINITY;
          // (a value times a weight of zero has to be zero)
          if (at16 >= whole || (at16 >= some && __float_as_uint(vf[j]) == 0x7f800000u)) vf[j] = 0.f;
        }
        // NaN for the rows that see such a token, in its group's dims (this lane's sums are of dims 32 g ..)
        for (int j = max(least - t * kTile, 0); j < min(len - t * kTile, kTile); ++j)
          nan |= vs[j * kGroups4 + g] == 255 && j < seen - t * kTile;
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
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] *= keep;
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // tokens 32 half + 4 g .. + 3 and + 16 .. + 19 of the lane
        bf16x8_t pt[kPT];
        split_bf16<kPT>(p + 8 * half, pt);
        uint32_t w[8][4];  // dims 8 m + 2 y, + 1 of each token
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint4 x = vx[2 * half + i / 4];
          decode8(i % 4 == 0 ? x.x : i % 4 == 1 ? x.y : i % 4 == 2 ? x.z : x.w, vf[8 * half + i], w[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t r[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)  // v_perm_b32(hi, lo, sel): the low or high halves of two tokens
            r[i] = __builtin_amdgcn_perm(w[2 * i + 1][j / 2], w[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
          bf16x8_t vv;
          __builtin_memcpy(&vv, r, 16);
#pragma unroll
          for (int x = kPT - 1; x >= 0; --x)
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pt[x], o[j], 0, 0, 0);
        }
      }
      if (nan) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[j][i] = NAN;
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
  }
}

// Attention over listed keys: one wave per (request, head, query) row.  Lane e
// looks up entry e; four lanes then read one key's or value's codes, a group of
// 32 dims each, 16 entries at a time, all in flight together.
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
  const int c = lane % 4, e0 = lane / 4;
  float qx[32];
  load_elems<T, 32>((const T*)q + r * kHeadDim + 32 * c, qx);
  uint4 kx[4];
  uint32_t vx[4][4], ke[4], ve[4];
  bool in[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int row = __shfl(at, 16 * u + e0);
    in[u] = row >= 0;
    kx[u] = make_uint4(0u, 0u, 0u, 0u);
    ke[u] = ve[u] = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) vx[u][x] = 0;
    if (in[u]) {
      const size_t block = (size_t)(row / kTile);
      const int token = row % kTile;
      const uint8_t* s = (const uint8_t*)a.scales + block * kScales4 + token * kGroups4 + c;
      kx[u] = *reinterpret_cast<const uint4*>(a.k + block * kCodes4 + code_at(0, token, 4 * c));
      ke[u] = s[0];
#pragma unroll
      for (int x = 0; x < 4; ++x)
        vx[u][x] = *reinterpret_cast<const uint32_t*>(a.v + block * kCodes4 + code_at(1, token, 4 * c + x));
      ve[u] = s[kTile * kGroups4];
    }
  }
  float p[4], top = -INFINITY;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t w[4] = {kx[u].x, kx[u].y, kx[u].z, kx[u].w};
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float y[8];
      decode8(w[x], scale_of(ke[u]), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(y[e], qx[8 * x + e], s);
    }
    s += xor_f32(s, 1);
    s += xor_f32(s, 2);
    p[u] = in[u] ? s * (0.08838834764831845f * kLog2e) : -INFINITY;
    top = fmaxf(top, p[u]);
  }
#pragma unroll
  for (int x = 4; x < kWave; x <<= 1) top = fmaxf(top, xor_f32(top, x));
  if (top == -INFINITY) top = 0.f;
  float l = 0.f, o[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) o[e] = 0.f;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float w = __builtin_amdgcn_exp2f(p[u] - top);
    l += w;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float y[8];
      decode8(vx[u][x], scale_of(ve[u]), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[8 * x + e] = fmaf(w, y[e], o[8 * x + e]);
    }
  }
  // sums over the 16 lanes of equal c, each step halving the dims a lane keeps
#pragma unroll
  for (int x = 4; x < kWave; x <<= 1) l += xor_f32(l, x);
  int d0 = 32 * c;
#pragma unroll
  for (int x = 32, w = 16; x >= 4; x >>= 1, w >>= 1) {
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
  return (int)(g < 1 ? 1 : g > kAttendGroups ? kAttendGroups : g);
}

// Whether a work-group takes a whole pair (see cache_attend_kernel's launch).
bool whole4_better(long long pairs, int max_blocks) {
  return max_blocks <= (pairs >= 512 ? 64 : pairs >= 256 ? 32 : pairs >= 128 ? 16 : 12);
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
  // tokens a launch: its waves, one per four tokens of a head, in 2^23 work-groups at most
  const int most = (int)((1LL << 25) / (2 * H_kv)) * 4;
  for (int t = 0; t < T; t += most) {
    const int n = T - t < most ? T - t : most;
    const long long items = (long long)((n + 3) / 4) * 2 * H_kv;
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
  // some 2,000 work-groups while the heads allow it
  const int blocks = (T + kReadRows - 1) / kReadRows, most = ((k_out && v_out ? 2 : 1) * H_kv + 3) / 4;
  int split = 2048 / blocks;
  split = split < 1 ? 1 : split > most ? most : split;
  const dim3 grid(blocks, split);
  if (dtype == SAKI_F32)
    hipLaunchKernelGGL((cache4_read_kernel<float>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
  else
    hipLaunchKernelGGL((cache4_read_kernel<__bf16>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
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
  if (whole4_better(pairs, max_blocks)) {
    const dim3 grid((unsigned)pairs);
    if (dtype == SAKI_F32)
      hipLaunchKernelGGL((cache4_attend_kernel<true, false>), grid, dim3(256), 0, s, a, q, out, nullptr);
    else
      hipLaunchKernelGGL((cache4_attend_kernel<false, false>), grid, dim3(256), 0, s, a, q, out, nullptr);
    return launched() ? SAKI_OK : SAKI_ERR_HIP;
  }
  const size_t need = saki_cache4_attend_workspace_bytes(B, H_q, H_kv, Q, max_blocks, 0);
  if (!ws || ws_bytes < need || !aligned(ws, 16)) return SAKI_ERR_WORKSPACE;
  const int groups = (int)(need / (2 * kPartFloats * sizeof(float)));
  const dim3 join((unsigned)pairs, pairs > 256 ? 1 : kHeadDim / 16);
  if (dtype == SAKI_F32) {
    hipLaunchKernelGGL((cache4_attend_kernel<true, true>), dim3(groups), dim3(256), 0, s, a, q, out, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    hipLaunchKernelGGL((cache_join_kernel<true>), join, dim3(256), 0, s, a, groups, (const float*)ws, out);
  } else {
    hipLaunchKernelGGL((cache4_attend_kernel<false, true>), dim3(groups), dim3(256), 0, s, a, q, out, (float*)ws);
    if (!launched()) return SAKI_ERR_HIP;
    hipLaunchKernelGGL((cache_join_kernel<false>), join, dim3(256), 0, s, a, groups, (const float*)ws, out);
  }
  return launched() ? SAKI_OK : SAKI_ERR_HIP;
}

}  // extern "C"
