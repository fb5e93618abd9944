// Between two blocks: the norm after a block, its gate, the residual addition and the norm in front of the next block, in one
// pass (vnm_residual_norm); int8 activations from such a row or from a matrix as it is (vnm_quantize_x).
//
// Bound by memory: a token's row of the residual stream and of the block's output is read once and held in registers in fp32,
// the sums of both norms and the largest magnitude are reductions over the threads that share the row, and every result is
// rounded once, when it is stored.  12608 x 768 fp16, layer norm and gate, 19.9 us (3.9 TB/s; 96 of 128 lanes have channels);
// 2048 x 4096 with an fp32 stream, two rms norms and an int8 result 20.9 (4.4); one token of 4096 channels 3.4.  Mean and variance are taken one after the other from registers, so the variance is a sum
// of squared deviations and cannot cancel.
#include "vnm_norm.h"

namespace vnm {

// 8 values of a row as int8
template <typename F>
__device__ __forceinline__ void store_i8(unsigned char* q, int n, int at, bool vec, float factor, F value) {
  unsigned b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = i8_round(value(e), factor);
  uint2 o = make_uint2(i8_pack4(b[0], b[1], b[2], b[3]), i8_pack4(b[4], b[5], b[6], b[7]));
  if (!(factor > 0.f)) o = make_uint2(0, 0);               // (no value of such a row counts; an infinity times 0 is none)
  if (vec) {
    if (at < n) *(uint2*)(q + at) = o;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) if (at + e < n) q[at + e] = (unsigned char)((e < 4 ? o.x : o.y) >> (8 * (e & 3)));
  }
}

template <typename HT, typename XT, int TPR, int NCH>
__global__ void __launch_bounds__(TPR == 64 ? 256 : TPR)
residual_norm_kernel(const vnm_residual_norm_args a, const int vec) {
  constexpr int RPB = TPR == 64 ? 4 : 1;         // rows that a workgroup has at a time
  __shared__ float2 lds[TPR == 64 ? 1 : 2 * (TPR / 64)];
  int turn = 0;
  const int tid = TPR == 64 ? (threadIdx.x & 63) : threadIdx.x;
  const int n = (int)a.n;
  const float fn = (float)n;
  Octet<XT> ow[NCH], ob[NCH], pw[NCH], pb[NCH], gt[NCH];
  if (a.post != VNM_NORM_NONE) {
    load_parameters<XT, TPR, NCH>(a.post_weight, 1.f, n, tid, vec, ow);
    load_parameters<XT, TPR, NCH>(a.post_bias, 0.f, n, tid, vec, ob);
  }
  if (a.pre != VNM_NORM_NONE) {
    load_parameters<XT, TPR, NCH>(a.pre_weight, 1.f, n, tid, vec, pw);
    load_parameters<XT, TPR, NCH>(a.pre_bias, 0.f, n, tid, vec, pb);
  }
  int64_t gate_at = -1;

  // mean and reciprocal deviation of the row in v (zeros past its end, before and after), and v normalised
  auto norm = [&](float (&v)[NCH][8], int kind, float eps, const Octet<XT> (&w)[NCH], const Octet<XT> (&b)[NCH], float& mean, float& r) {
    mean = 0.f; r = 1.f;
    if (kind == VNM_NORM_NONE) return;
    if (kind == VNM_NORM_LAYER) {
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[c][e];
      mean = row_sum2<TPR>(s, 0.f, lds, turn).x / fn;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] -= mean;
      clear_past<TPR, NCH>(v, n, tid);
    }
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) q += v[c][e] * v[c][e];
    r = 1.f / sqrtf(row_sum2<TPR>(q, 0.f, lds, turn).x / fn + eps);
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = v[c][e] * r * (float)w[c].v[e] + (float)b[c].v[e];
    clear_past<TPR, NCH>(v, n, tid);
  };

  // The next row is requested when this one's has been taken over into fp32: its way from memory overlaps the reductions.
  Octet<HT> hr[NCH];
  Octet<XT> yr[NCH];
  auto request = [&](int64_t t) {
    load_row<HT, TPR, NCH>((const HT*)a.h + t * a.ldh, n, tid, vec, hr);
    if (a.y) load_row<XT, TPR, NCH>((const XT*)a.y + t * a.ldy, n, tid, vec, yr);
  };
  const int64_t first = (int64_t)blockIdx.x * RPB + (TPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  const int64_t stride = (int64_t)gridDim.x * RPB;
  if (first < a.T) request(first);
  for (int64_t t = first; t < a.T; t += stride) {
    if (a.gate) {
      const int64_t g = a.gate_tokens ? t / a.gate_tokens : 0;
      if (g != gate_at) load_row<XT, TPR, NCH>((const XT*)a.gate + g * a.ldg, n, tid, vec, gt);
      gate_at = g;
    }
    keep_stored(pw); keep_stored(pb); keep_stored(ow); keep_stored(ob); keep_stored(gt);
    float v[NCH][8], hv[NCH][8], mean_post = 0.f, r_post = 1.f, mean_pre, r_pre;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) hv[c][e] = a.residual_scale * (float)hr[c].v[e];
    if (a.y) {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = (float)yr[c].v[e];
    }
    if (t + stride < a.T) request(t + stride);
    if (a.y) {
      norm(v, a.post, a.post_eps, ow, ob, mean_post, r_post);
      if (a.gate) {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[c][e] = v[c][e] * (float)gt[c].v[e] + hv[c][e];
      } else {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[c][e] += hv[c][e];
      }
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = hv[c][e];
    }
    if (a.h_out) store_row<HT, TPR, NCH>((HT*)a.h_out + t * a.ldho, n, tid, vec, v);
    if (!a.x && !a.q && !a.stats) continue;
    norm(v, a.pre, a.pre_eps, pw, pb, mean_pre, r_pre);
    if (a.stats && tid == 0) ((float4*)a.stats)[t] = make_float4(mean_post, r_post, mean_pre, r_pre);
    if (a.x) store_row<XT, TPR, NCH>((XT*)a.x + t * a.ldx, n, tid, vec, v);
    if (a.q) {
      unsigned top = 0;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned m = magnitude_bits(v[c][e]);
          top = m > top ? m : top;
        }
      float factor, scale;
      i8_factor(__builtin_bit_cast(float, row_max<TPR>(top, lds, turn)), &factor, &scale);
      if (tid == 0) ((float*)a.q_scale)[t] = scale;
      unsigned char* q = (unsigned char*)a.q + t * a.ldq;
#pragma unroll
      for (int c = 0; c < NCH; ++c) store_i8(q, n, (c * TPR + tid) * 8, vec, factor, [&](int e) { return v[c][e]; });
    }
  }
}

// vnm_quantize_x: the largest magnitude of a row and then its int8 values, from registers.  4096 x 4096 bf16 in 11 us (4.5 TB/s),
// 24 x 11008 in 3.3 (a launch and one row's latency).  Bound by memory (the reductions leave it
// idle, so the next row is requested before them).
template <typename XT, int TPR, int NCH>
__global__ void __launch_bounds__(TPR == 64 ? 256 : TPR)
quantize_rows_kernel(const XT* __restrict__ X, int64_t T, int n, int64_t ldx, unsigned char* __restrict__ Q, int64_t ldq,
                     float* __restrict__ scales, int64_t scale_rows, const int vec) {
  constexpr int RPB = TPR == 64 ? 4 : 1;
  __shared__ float2 lds[TPR == 64 ? 1 : 2 * (TPR / 64)];
  int turn = 0;
  const int tid = TPR == 64 ? (threadIdx.x & 63) : threadIdx.x;
  const int64_t first = (int64_t)blockIdx.x * RPB + (TPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  const int64_t stride = (int64_t)gridDim.x * RPB;
  Octet<XT> next[NCH], x[NCH];
  if (first < T) load_row<XT, TPR, NCH>(X + first * ldx, n, tid, vec, next);
  for (int64_t t = first; t < T; t += stride) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) x[c] = next[c];
    if (t + stride < T) load_row<XT, TPR, NCH>(X + (t + stride) * ldx, n, tid, vec, next);
    unsigned top = 0;                                      // (zeros past the row's end)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned m = magnitude_bits((float)x[c].v[e]);
        top = m > top ? m : top;
      }
    float factor, scale;
    i8_factor(__builtin_bit_cast(float, row_max<TPR>(top, lds, turn)), &factor, &scale);
    if (tid == 0 && t < scale_rows) scales[t] = scale;
    unsigned char* q = Q + t * ldq;
#pragma unroll
    for (int c = 0; c < NCH; ++c) store_i8(q, n, (c * TPR + tid) * 8, vec, factor, [&](int e) { return (float)x[c].v[e]; });
  }
}

// Rows that no kernel above holds in registers: two passes over memory.
template <typename XT>
__global__ void __launch_bounds__(1024)
quantize_long_kernel(const XT* __restrict__ X, int64_t T, int64_t n, int64_t ldx, unsigned char* __restrict__ Q, int64_t ldq,
                     float* __restrict__ scales, int64_t scale_rows) {
  __shared__ float2 lds[32];
  int turn = 0;
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const XT* x = X + t * ldx;
    unsigned top = 0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) { const unsigned m = magnitude_bits((float)x[i]); top = m > top ? m : top; }
    float factor, scale;
    i8_factor(__builtin_bit_cast(float, row_max<1024>(top, lds, turn)), &factor, &scale);
    if (threadIdx.x == 0 && t < scale_rows) scales[t] = scale;
    for (int64_t i = threadIdx.x; i < n; i += 1024) Q[t * ldq + i] = (unsigned char)(factor > 0.f ? i8_round((float)x[i], factor) : 0u);
  }
}

template <typename HT, typename XT, int TPR, int NCH>
static int launch_norm_cfg(const vnm_residual_norm_args& a, bool vec, hipStream_t st) {
  constexpr int RPB = TPR == 64 ? 4 : 1, THREADS = TPR == 64 ? 256 : TPR;
  int64_t blocks = (a.T + RPB - 1) / RPB;
  const int64_t most = 256 * (16 * 64 / THREADS);         // 16 waves per compute unit: what the registers of all-fp32 rows allow
  if (blocks > most) blocks = most;
  hipLaunchKernelGGL((residual_norm_kernel<HT, XT, TPR, NCH>), dim3((unsigned)blocks), dim3(THREADS), 0, st, a, (int)vec);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "residual_norm_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}
// An octet per thread where a row has at most 8192 channels: with the next row requested ahead a thread needs 75 to 105 registers
// for each, and fewer waves per SIMD cost more than the barriers of rows that are spread over several.  (Two octets in 1024 threads
// do not fit 128 registers: 148 to 316 bytes of scratch memory per thread.)
template <typename HT, typename XT>
static int launch_norm(const vnm_residual_norm_args& a, bool vec, hipStream_t st) {
  if (a.n <= 512) return launch_norm_cfg<HT, XT, 64, 1>(a, vec, st);
  if (a.n <= 1024) return launch_norm_cfg<HT, XT, 128, 1>(a, vec, st);
  if (a.n <= 2048) return launch_norm_cfg<HT, XT, 256, 1>(a, vec, st);
  if (a.n <= 4096) return launch_norm_cfg<HT, XT, 512, 1>(a, vec, st);
  if (a.n <= 8192) return launch_norm_cfg<HT, XT, 1024, 1>(a, vec, st);
  return launch_norm_cfg<HT, XT, 1024, 2>(a, vec, st);
}
static int launch_norm_types(const vnm_residual_norm_args& a, bool vec, hipStream_t st) {
  if (a.x_dtype == VNM_F32) return launch_norm<float, float>(a, vec, st);
  if (a.h_dtype == VNM_F32)
    return a.x_dtype == VNM_F16 ? launch_norm<float, _Float16>(a, vec, st) : launch_norm<float, __bf16>(a, vec, st);
  return a.x_dtype == VNM_F16 ? launch_norm<_Float16, _Float16>(a, vec, st) : launch_norm<__bf16, __bf16>(a, vec, st);
}

template <typename XT>
static int launch_quantize_long(const void* X, int64_t T, int64_t n, int64_t ldx, void* Q, int64_t ldq, void* scale,
                                int64_t scale_rows, hipStream_t st) {
  hipLaunchKernelGGL(quantize_long_kernel<XT>, dim3((unsigned)(T < 2048 ? T : 2048)), dim3(1024), 0, st, (const XT*)X, T, n, ldx,
                     (unsigned char*)Q, ldq, (float*)scale, scale_rows);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "quantize_long_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}

template <typename XT, int TPR, int NCH>
static int launch_quantize_cfg(const void* X, int64_t T, int64_t n, int64_t ldx, void* Q, int64_t ldq, void* scale, int64_t scale_rows,
                               bool vec, hipStream_t st) {
  constexpr int RPB = TPR == 64 ? 4 : 1, THREADS = TPR == 64 ? 256 : TPR;
  int64_t blocks = (T + RPB - 1) / RPB;
  const int64_t most = 256 * (32 * 64 / THREADS);         // 32 waves per compute unit
  if (blocks > most) blocks = most;
  hipLaunchKernelGGL((quantize_rows_kernel<XT, TPR, NCH>), dim3((unsigned)blocks), dim3(THREADS), 0, st, (const XT*)X, T, (int)n, ldx,
                     (unsigned char*)Q, ldq, (float*)scale, scale_rows, (int)vec);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "quantize_rows_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}
template <typename XT>
static int launch_quantize(const void* X, int64_t T, int64_t n, int64_t ldx, void* Q, int64_t ldq, void* scale, int64_t scale_rows, hipStream_t st) {
  const bool vec = n % 8 == 0 && ldx % 8 == 0 && ldq % 8 == 0 && ((uintptr_t)X & 15) == 0 && ((uintptr_t)Q & 7) == 0;
  if (n > VNM_NORM_MAX_CHANNELS) return launch_quantize_long<XT>(X, T, n, ldx, Q, ldq, scale, scale_rows, st);
  if (n <= 512) return launch_quantize_cfg<XT, 64, 1>(X, T, n, ldx, Q, ldq, scale, scale_rows, vec, st);
  if (n <= 1024) return launch_quantize_cfg<XT, 64, 2>(X, T, n, ldx, Q, ldq, scale, scale_rows, vec, st);
  if (n <= 2048) return launch_quantize_cfg<XT, 256, 1>(X, T, n, ldx, Q, ldq, scale, scale_rows, vec, st);
  if (n <= 4096) return launch_quantize_cfg<XT, 256, 2>(X, T, n, ldx, Q, ldq, scale, scale_rows, vec, st);
  if (n <= 8192) return launch_quantize_cfg<XT, 512, 2>(X, T, n, ldx, Q, ldq, scale, scale_rows, vec, st);
  return launch_quantize_cfg<XT, 1024, 2>(X, T, n, ldx, Q, ldq, scale, scale_rows, vec, st);
}

// rows from scale_rows on have no scale to store
int launch_quantize_rows(const void* X, int64_t T, int64_t n, int64_t ldx, int x_dtype, void* Q, int64_t ldq, void* scale,
                         int64_t scale_rows, hipStream_t st) {
  return x_dtype == VNM_F32   ? launch_quantize<float>(X, T, n, ldx, Q, ldq, scale, scale_rows, st)
         : x_dtype == VNM_F16 ? launch_quantize<_Float16>(X, T, n, ldx, Q, ldq, scale, scale_rows, st)
                              : launch_quantize<__bf16>(X, T, n, ldx, Q, ldq, scale, scale_rows, st);
}

}  // namespace vnm

using namespace vnm;

static bool dtype_ok(int t) { return t == VNM_F16 || t == VNM_F32 || t == VNM_BF16; }
static uintptr_t dtype_bytes(int t) { return t == VNM_F32 ? 4 : 2; }

extern "C" int vnm_quantize_x(const void* X, int64_t T, int64_t n, int64_t ldx, int x_dtype, void* Q, int64_t ldq, void* scale,
                              void* stream) {
  if (T != 0 && (!X || !Q || !scale)) return VNM_ERR_NULL;
  if (T < 0 || n <= 0 || ldx < n || ldq < n) return VNM_ERR_SHAPE;
  if (!dtype_ok(x_dtype)) return VNM_ERR_UNSUPPORTED;
  if (((uintptr_t)X & (dtype_bytes(x_dtype) - 1)) || ((uintptr_t)scale & 3)) return VNM_ERR_ALIGN;
  if (T == 0) return VNM_OK;
  return launch_quantize_rows(X, T, n, ldx, x_dtype, Q, ldq, scale, T, (hipStream_t)stream);
}

extern "C" int vnm_residual_norm(const vnm_residual_norm_args* args, void* stream) {
  if (!args) return VNM_ERR_NULL;
  const vnm_residual_norm_args& a = *args;
  if (a.T < 0 || a.n <= 0 || a.gate_tokens < 0) return VNM_ERR_SHAPE;
  if (a.n > VNM_NORM_MAX_CHANNELS) return VNM_ERR_UNSUPPORTED;
  if (!dtype_ok(a.x_dtype) || !(a.h_dtype == a.x_dtype || a.h_dtype == VNM_F32)) return VNM_ERR_UNSUPPORTED;
  if (a.post < VNM_NORM_NONE || a.post > VNM_NORM_LAYER || a.pre < VNM_NORM_NONE || a.pre > VNM_NORM_LAYER) return VNM_ERR_UNSUPPORTED;
  if ((a.post != VNM_NORM_NONE && !(a.post_eps > 0.f)) || (a.pre != VNM_NORM_NONE && !(a.pre_eps > 0.f))) return VNM_ERR_UNSUPPORTED;
  // what belongs to a norm that is not there, or to a block's output that is not there
  if (a.post == VNM_NORM_NONE && (a.post_weight || a.post_bias)) return VNM_ERR_UNSUPPORTED;
  if (a.pre == VNM_NORM_NONE && (a.pre_weight || a.pre_bias)) return VNM_ERR_UNSUPPORTED;
  if (a.T != 0 && !a.y && (a.gate || a.post != VNM_NORM_NONE)) return VNM_ERR_NULL;
  if (a.x && a.q) return VNM_ERR_UNSUPPORTED;
  if (a.T != 0 && (!a.h || (!a.x && !a.q && !a.h_out) || (a.q && !a.q_scale))) return VNM_ERR_NULL;
  if (a.T == 0) return VNM_OK;
  if (a.ldh < a.n || (a.y && a.ldy < a.n) || (a.gate && a.gate_tokens && a.ldg < a.n) || (a.h_out && a.ldho < a.n) ||
      (a.x && a.ldx < a.n) || (a.q && a.ldq < a.n) || (a.h_out == a.h && a.ldho != a.ldh))
    return VNM_ERR_SHAPE;
  const uintptr_t hp = (uintptr_t)a.h | (uintptr_t)a.h_out;
  const uintptr_t xp = (uintptr_t)a.y | (uintptr_t)a.gate | (uintptr_t)a.post_weight | (uintptr_t)a.post_bias |
                       (uintptr_t)a.pre_weight | (uintptr_t)a.pre_bias | (uintptr_t)a.x;
  if ((hp & (dtype_bytes(a.h_dtype) - 1)) || (xp & (dtype_bytes(a.x_dtype) - 1)) || ((uintptr_t)a.q_scale & 3) || ((uintptr_t)a.stats & 15))
    return VNM_ERR_ALIGN;
  const int64_t lds = a.ldh | (a.y ? a.ldy : 0) | (a.gate && a.gate_tokens ? a.ldg : 0) | (a.h_out ? a.ldho : 0) | (a.x ? a.ldx : 0) |
                      (a.q ? a.ldq : 0);
  const bool vec = a.n % 8 == 0 && lds % 8 == 0 && ((hp | xp) & 15) == 0 && ((uintptr_t)a.q & 7) == 0;
  return launch_norm_types(a, vec, (hipStream_t)stream);
}
