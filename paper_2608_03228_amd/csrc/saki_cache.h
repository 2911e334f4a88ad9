// What the kernels over a paged cache (8 bits in saki_serve.hip, 4 bits in
// saki_cache4.hip) share: element loads and stores, how a call's tiles are
// divided among work-groups, and argument checks.
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
  } else if constexpr (N == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 8)
      *reinterpret_cast<uint4*>(p + j) =
          make_uint4(pack_bf16(v[j], v[j + 1]), pack_bf16(v[j + 2], v[j + 3]),
                     pack_bf16(v[j + 4], v[j + 5]), pack_bf16(v[j + 6], v[j + 7]));
  }
}

// Inclusive scan of one value a thread over a work-group of W waves; *total gets
// the sum.  `part` holds W values.
template <int W = 4>
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
  for (int w = 0; w < W; ++w) {
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
