// What the kernels over a paged cache (8 bits in saki_serve.hip, 4 bits in
// saki_cache4.hip) share: element loads and stores, how a call's tiles are
// divided among work-groups, the join of their parts, and argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "saki.h"
#include "saki_internal.h"
#include "saki_topk.h"

namespace {

using saki::kHeadDim;
using saki::kTile;
using saki_dev::kWave;
using saki_dev::xor_shfl_u32;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float xor_f32(float v, int m) {
  return __uint_as_float(xor_shfl_u32(__float_as_uint(v), m));
}

// The 4 float32 or 8 bf16 elements of 16 bytes as floats.
template <typename T>
__device__ __forceinline__ void unpack16(uint4 v, float* out) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (std::is_same_v<T, float>) {
      out[e] = __uint_as_float(w[e]);
    } else {
      out[2 * e] = __uint_as_float(w[e] << 16);
      out[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}

// N elements at p, a 16-byte boundary, as floats.
template <typename T, int N>
__device__ __forceinline__ void load_elems(const T* p, float* out) {
#pragma unroll
  for (int j = 0; j < N; j += 16 / (int)sizeof(T)) unpack16<T>(*reinterpret_cast<const uint4*>(p + j), out + j);
}

// Two floats as a pair of bf16, round to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  bf16x2_t v = {(__bf16)a, (__bf16)b};
  uint32_t r;
  __builtin_memcpy(&r, &v, sizeof(r));
  return r;
}

template <typename T, int N>
__device__ __forceinline__ void store_elems(T* p, const float* v) {
  if constexpr (std::is_same_v<T, float>) {
#pragma unroll
    for (int j = 0; j < N; j += 4)
      *reinterpret_cast<float4*>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 8)
      *reinterpret_cast<uint4*>(p + j) =
          make_uint4(pack_bf16(v[j], v[j + 1]), pack_bf16(v[j + 2], v[j + 3]),
                     pack_bf16(v[j + 4], v[j + 5]), pack_bf16(v[j + 6], v[j + 7]));
  }
}

// Inclusive scan of one value a thread over a work-group of 256; *total gets
// the sum.  `part` holds 4 values.
__device__ __forceinline__ long long group_scan(long long v, long long* part, long long* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const long long up = __shfl_up(v, d);
    if (lane >= d) v += up;
  }
  __syncthreads();  // readers of the last call are done with `part`
  if (lane == kWave - 1) part[wave] = v;
  __syncthreads();
  long long before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const long long p = part[w];
    if (w < wave) before += p;
    sum += p;
  }
  *total = sum;
  return v + before;
}

// ---------------------------------------------------------------- attention over a cache

struct CacheArgs {
  const uint8_t *k, *v;
  const void* scales;  // float [n_blocks, H_kv, 2] (8 bits), E8M0 bytes [n_blocks, H_kv, 2, 64, 4] (4 bits)
  int n_blocks;
  const int* tables;
  int max_blocks;
  const int* lens;
  int B, H_q, H_kv, Q;
};

// A float as the sum of bf16 terms, each the nearest to what is left: two
// terms leave 2^-17 of it, three 2^-25.
template <int N>
__device__ __forceinline__ void split_bf16(const float* x, bf16x8_t* terms) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const __bf16 b = (__bf16)r[e];
      terms[n][e] = b;
      r[e] -= (float)b;
    }
}

__device__ __forceinline__ int tiles_of(int len, int max_blocks) {
  return len <= 0 ? 0 : min((len - 1) / kTile + 1, max_blocks);
}

constexpr int kPartRows = 16;
constexpr int kPartFloats = kPartRows * kHeadDim + 2 * kPartRows;  // sums, maxima, weights
constexpr int kMinPiece = 4;                                       // tiles a work-group takes at least
constexpr int kAttendGroups = 512;                                 // two a CU

// Tiles of up to 64 requests, one a lane: its own, the sum up to it, and all
// (below 2^31, as a table has fewer than 2^25 - 1 blocks).
struct Sums {
  int len, mine, upto, total;
};
__device__ __forceinline__ Sums wave_sums(const CacheArgs& a) {
  const int lane = threadIdx.x % kWave;
  Sums s;
  s.len = lane < a.B ? a.lens[lane] : 0;
  s.mine = tiles_of(s.len, a.max_blocks);
  s.upto = s.mine;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int up = __shfl_up(s.upto, d);
    if (lane >= d) s.upto += up;
  }
  s.total = __builtin_amdgcn_readlane(s.upto, kWave - 1);
  return s;
}

// Where a work-group's share of the tiles begins.  All tiles of all (request,
// KV head, 16-row block) pairs stand in one line, a request's pairs one after
// another; group w takes [w * piece, (w + 1) * piece).
struct Share {
  long long total, piece;
};
__device__ __forceinline__ Share share_of(long long total, int groups) {
  Share s;
  s.total = total;
  s.piece = (total + groups - 1) / groups;
  if (s.piece < kMinPiece) s.piece = kMinPiece;
  return s;
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

// ---------------------------------------------------------------- argument checks

bool type_ok(int t) { return t == SAKI_F32 || t == SAKI_BF16; }
size_t type_bytes(int t) { return t == SAKI_F32 ? 4 : 2; }

// Token rows of H heads at `p`, ld elements apart: what the 16-byte accesses need.
bool rows_ok(const void* p, size_t ld, int H, int dtype) {
  return p && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld >= (size_t)H * kHeadDim &&
         ld * type_bytes(dtype) % 16 == 0 && ld <= ((size_t)1 << 40);
}
bool overlap(const void* p, size_t n, const void* q, size_t m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + m && b < a + n;
}
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

constexpr int kMaxTokens = 1 << 26;
bool launched() { return hipGetLastError() == hipSuccess; }

}  // namespace
