// Row operations of the norm kernels (vnm_norm.hip, vnm_norm_backward.hip).
#pragma once
#include "vnm_i8.h"

namespace vnm {

// 8 consecutive elements as they are stored: one 16-byte load for 16-bit types, two for fp32
template <typename T> struct alignas(16) Octet { T v[8]; };

// Says that the octets may change here: values that stay the same from row to row are then widened where they are used and
// occupy half of the registers between.
template <typename T, int NCH>
__device__ __forceinline__ void keep_stored(Octet<T> (&r)[NCH]) {
  typedef unsigned words __attribute__((ext_vector_type(sizeof(T) * 2)));
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    words w = __builtin_bit_cast(words, r[c]);
    asm volatile("" : "+v"(w));
    r[c] = __builtin_bit_cast(Octet<T>, w);
  }
}

// The share of a row that a thread of TPR holds: octets tid, tid + TPR, ...  VEC: rows are 16-byte aligned and n % 8 == 0, so
// that an octet is inside the row or outside as a whole; otherwise its elements are fetched and stored one by one.
template <typename T, int TPR, int NCH>
__device__ __forceinline__ void load_row(const T* p, int n, int tid, bool vec, Octet<T> (&r)[NCH]) {
  if (vec) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int at = (c * TPR + tid) * 8;
      if (at < n) r[c] = *(const Octet<T>*)(p + at);
      else r[c] = Octet<T>{};
    }
  } else {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = (c * TPR + tid) * 8 + e;
        r[c].v[e] = at < n ? p[at] : (T)0.f;
      }
  }
}
// A row of parameters, or of `other` where there is none (the elements past n do not matter)
template <typename T, int TPR, int NCH>
__device__ __forceinline__ void load_parameters(const void* p, float other, int n, int tid, bool vec, Octet<T> (&r)[NCH]) {
  if (p) { load_row<T, TPR, NCH>((const T*)p, n, tid, vec, r); return; }
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) r[c].v[e] = (T)other;
}
// Zeros for the elements past n: a branch that all but the last of the row's waves skip
template <int TPR, int NCH>
__device__ __forceinline__ void clear_past(float (&x)[NCH][8], int n, int tid) {
#pragma unroll
  for (int c = 0; c < NCH; ++c)
    if ((c * TPR + tid) * 8 + 8 > n) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = (c * TPR + tid) * 8 + e < n ? x[c][e] : 0.f;
    }
}
template <typename T, int TPR, int NCH>
__device__ __forceinline__ void store_row(T* p, int n, int tid, bool vec, const float (&x)[NCH][8]) {
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int at = (c * TPR + tid) * 8;
    Octet<T> o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[e] = (T)x[c][e];
    if (vec) { if (at < n) *(Octet<T>*)(p + at) = o; }
    else {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (at + e < n) p[at + e] = o.v[e];
    }
  }
}

// Over a wave by the data-parallel shifts of its rows of 16 lanes and two broadcasts, which need no LDS; the result, taken from
// the last lane, is uniform.  Lanes without a source add 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ float wave_sum(float v) {
  auto add = [&](unsigned o) { v += __builtin_bit_cast(float, o); };
  const auto bits = [&] { return __builtin_bit_cast(unsigned, v); };
  add(dpp<0x111, 0xf>(bits())); add(dpp<0x112, 0xf>(bits())); add(dpp<0x114, 0xf>(bits())); add(dpp<0x118, 0xf>(bits()));
  add(dpp<0x142, 0xa>(bits())); add(dpp<0x143, 0xc>(bits()));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)bits(), 63));
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
  auto top = [&](unsigned o) { v = o > v ? o : v; };
  top(dpp<0x111, 0xf>(v)); top(dpp<0x112, 0xf>(v)); top(dpp<0x114, 0xf>(v)); top(dpp<0x118, 0xf>(v));
  top(dpp<0x142, 0xa>(v)); top(dpp<0x143, 0xc>(v));
  return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}
// Over the TPR threads that share a row.  `lds`: two halves of TPR / 64 pairs, used in turn (`turn`), so that one barrier per
// reduction is enough: a wave reaches the use after next of a half only past the barrier of the next.
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* lds, int& turn) {
  a = wave_sum(a); b = wave_sum(b);
  if (TPR == 64) return make_float2(a, b);
  constexpr int W = TPR / 64;
  float2* half = lds + (turn & 1) * W;
  ++turn;
  if ((threadIdx.x & 63) == 0) half[threadIdx.x >> 6] = make_float2(a, b);
  __syncthreads();
  float2 s = half[0];
#pragma unroll
  for (int w = 1; w < W; ++w) { s.x += half[w].x; s.y += half[w].y; }
  return s;
}
template <int TPR>
__device__ __forceinline__ unsigned row_max(unsigned v, float2* lds, int& turn) {
  v = wave_max(v);
  if (TPR == 64) return v;
  constexpr int W = TPR / 64;
  unsigned* half = (unsigned*)(lds + (turn & 1) * W);
  ++turn;
  if ((threadIdx.x & 63) == 0) half[threadIdx.x >> 6] = v;
  __syncthreads();
  unsigned m = half[0];
#pragma unroll
  for (int w = 1; w < W; ++w) m = half[w] > m ? half[w] : m;
  return m;
}

}  // namespace vnm
