// Gradients of vnm_residual_norm.
//
// With xhat = (h' - mean) r, g = dx * weight, a row's gradient through a norm is r (g - mean(g) - xhat mean(g xhat)) (without
// the mean of g for VNM_NORM_RMS), so a row needs two sums per norm; the gradients of weights, biases and gates are sums over
// the tokens.  One pass over the tokens does both: a worker (the threads that share a row) owns a run of consecutive tokens of
// one gate row, keeps its share of the column sums in registers, and leaves them at the end as one row of partial sums in the
// workspace; a second kernel adds the workers' rows in a fixed order.  Bound by memory, and by the waves that fit beside the column
// sums in registers: 4096 x 4096 bf16 with rms norms on both sides 52 us (3.9 TB/s) and 7 in the second kernel; 1576 x 384, fp32
// stream, a gate per 197 tokens 11.5 and 3.9.
#include "vnm_norm.h"

namespace vnm {

enum { kPreWeight, kPreBias, kPostWeight, kPostBias, kGate, kSums };

// How the tokens are cut: `groups` gate rows (1 without) of `tokens` tokens each, `pieces` runs of `per` tokens per group.
struct Cut { int64_t groups, tokens, pieces, per; };

// What the call has, kBiases | kGated | kPosted; a kernel for fewer keeps fewer sums and fits more waves.
enum { kBiases = 1, kGated = 2, kPosted = 4, kAllParts = 7 };
// Waves per SIMD that the registers are held down for: four, also where that takes a little scratch memory (a post norm: 12 to 28
// bytes per thread from 2049 channels on, 56 to 88 in rows that are all fp32; 4096 x 4096 bf16 61 us with four waves, 78 with three
// and no scratch; without a post norm, where four need none, 45 and 80); three with a gate and biases (1576 x 384: 16.3 us, with
// four and scratch 20.7); two with everything.  1024 threads are four waves per SIMD whatever that takes: up to 176 bytes, and 684 to
// 864 above 8192 channels.
constexpr int back_waves(int TPR, int NCH, int PARTS) {
  return TPR == 1024 ? 4 : NCH > 1 || PARTS == kAllParts ? 2 : (PARTS & kGated) || (TPR == 64 && PARTS) ? 3 : 4;
}

static Cut make_cut(int64_t T, int64_t n, int64_t gate_tokens, bool four_waves) {
  Cut c;
  c.tokens = gate_tokens > 0 && gate_tokens < T ? gate_tokens : T > 0 ? T : 1;
  c.groups = T > 0 ? (T + c.tokens - 1) / c.tokens : 0;
  // Few tokens: up to 256 workers.  Many: as many as run at once with four or three waves per SIMD (one more than that and the
  // call takes two rounds: 12608 x 768 with a gate 61 us in 1802 workers), as every one leaves a row of partial sums.  Up to 512
  // channels, where a worker is one wave, half of that: 12608 x 384 and 16384 x 512 take the same time with 8 and 16 per unit.
  const int64_t per_cu = n <= 512 ? 8 : n <= 1024 ? (four_waves ? 8 : 6) : n <= 2048 ? (four_waves ? 4 : 3) : n <= 4096 ? (four_waves ? 2 : 1) : 1;
  const int64_t workers = T <= 1024 ? 256 : 256 * per_cu;
  c.per = (T + workers - 1) / workers;
  if (T > 1024 && c.per < 4) c.per = 4;
  if (c.per < 1) c.per = 1;
  if (c.per > c.tokens) c.per = c.tokens;
  c.pieces = (c.tokens + c.per - 1) / c.per;
  return c;
}

struct BackArgs {
  vnm_residual_norm_backward_args a;
  Cut cut;
  float* part;            // [kSums][workers][n]; a sum that is not asked for has no room of its own
  int64_t part_at[kSums];
  int vec;
};

template <typename HT, typename XT, int TPR, int NCH, int PARTS>
__global__ void __launch_bounds__(TPR == 64 ? 256 : TPR, back_waves(TPR, NCH, PARTS))
residual_norm_backward_kernel(const BackArgs b) {
  constexpr bool BIASES = PARTS & kBiases, GATED = PARTS & kGated, POSTED = PARTS & kPosted;
  constexpr int RPB = TPR == 64 ? 4 : 1;
  __shared__ float2 lds[TPR == 64 ? 1 : 2 * (TPR / 64)];
  int turn = 0;
  const vnm_residual_norm_backward_args& a = b.a;
  const int tid = TPR == 64 ? (threadIdx.x & 63) : threadIdx.x;
  const int64_t worker = (int64_t)blockIdx.x * RPB + (TPR == 64 ? threadIdx.x >> 6 : 0);
  if (worker >= b.cut.groups * b.cut.pieces) return;     // a whole worker: those of one wave share no barrier
  const int64_t group = worker / b.cut.pieces, first = group * b.cut.tokens + (worker - group * b.cut.pieces) * b.cut.per;
  int64_t end = first + b.cut.per;
  const int64_t group_end = (group + 1) * b.cut.tokens < a.T ? (group + 1) * b.cut.tokens : a.T;
  end = end < group_end ? end : group_end;
  const int n = (int)a.n;
  const float fn = (float)n;
  const bool vec = b.vec;
  Octet<XT> pw[NCH], ow[NCH], ob[NCH], gt[NCH];
  load_parameters<XT, TPR, NCH>(a.pre_weight, 1.f, n, tid, vec, pw);
  if (POSTED) load_parameters<XT, TPR, NCH>(a.post_weight, 1.f, n, tid, vec, ow);
  if (BIASES) load_parameters<XT, TPR, NCH>(a.post_bias, 0.f, n, tid, vec, ob);
  if (GATED) load_parameters<XT, TPR, NCH>(a.gate ? (const XT*)a.gate + group * a.ldg : nullptr, 1.f, n, tid, vec, gt);
  float sum[kSums][NCH][8];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[k][c][e] = 0.f;
  const bool through_pre = a.dx && a.pre != VNM_NORM_NONE;
  Octet<XT> xr[NCH], yr[NCH];                            // (zeros for a gradient or an output that is not there)
  Octet<HT> hr[NCH], gr[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) { xr[c] = yr[c] = Octet<XT>{}; hr[c] = gr[c] = Octet<HT>{}; }
  float4 next_stats = make_float4(0.f, 1.f, 0.f, 1.f);
  auto request = [&](int64_t t) {
    if (a.stats) next_stats = ((const float4*)a.stats)[t];
    if (a.dx) load_row<XT, TPR, NCH>((const XT*)a.dx + t * a.lddx, n, tid, vec, xr);
    if (through_pre) load_row<HT, TPR, NCH>((const HT*)a.h_new + t * a.ldh, n, tid, vec, hr);
    if (a.dh_out) load_row<HT, TPR, NCH>((const HT*)a.dh_out + t * a.lddho, n, tid, vec, gr);
    if (a.y) load_row<XT, TPR, NCH>((const XT*)a.y + t * a.ldy, n, tid, vec, yr);
  };
  if (first < end) request(first);                       // (the last group may have fewer tokens than pieces)
  for (int64_t t = first; t < end; ++t) {
    const float4 st = next_stats;
    keep_stored(pw); keep_stored(ow); keep_stored(ob); keep_stored(gt);
    // d = gradient of h'; the next row is requested when this one's has been taken over into fp32
    float d[NCH][8], yv[NCH][8], gv[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        yv[c][e] = (float)yr[c].v[e];
        gv[c][e] = (float)gr[c].v[e];
      }
    if (through_pre) {
      float xhat[NCH][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float dx = (float)xr[c].v[e];
          xhat[c][e] = ((float)hr[c].v[e] - st.z) * st.w;
          sum[kPreWeight][c][e] += dx * xhat[c][e];
          if (BIASES) sum[kPreBias][c][e] += dx;
          d[c][e] = dx * (float)pw[c].v[e];
          s1 += d[c][e] * xhat[c][e];                    // (dx is 0 outside the row)
          s2 += d[c][e];
        }
      if (t + 1 < end) request(t + 1);
      const float2 s = row_sum2<TPR>(s1, s2, lds, turn);
      const float m1 = s.x / fn, m2 = a.pre == VNM_NORM_LAYER ? s.y / fn : 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[c][e] = st.w * (d[c][e] - m2 - xhat[c][e] * m1);
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[c][e] = (float)xr[c].v[e];
      if (t + 1 < end) request(t + 1);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) d[c][e] += gv[c][e];
    if (a.dh) {
      float o[NCH][8];
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[c][e] = a.residual_scale * d[c][e];
      store_row<HT, TPR, NCH>((HT*)a.dh + t * a.lddh, n, tid, vec, o);
    }
    if (!a.dy && !a.d_gate && !a.d_post_weight && !a.d_post_bias) continue;
    // through the gate and the post norm
    float yhat[NCH][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) yhat[c][e] = (yv[c][e] - st.x) * st.y;
    clear_past<TPR, NCH>(yhat, n, tid);
    clear_past<TPR, NCH>(d, n, tid);                     // (means were taken away past the row's end too)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (GATED) {
          float p = yhat[c][e];
          if (POSTED) p *= (float)ow[c].v[e];
          if (BIASES) p += (float)ob[c].v[e];
          sum[kGate][c][e] += d[c][e] * p;
          d[c][e] *= (float)gt[c].v[e];
        }
        if (POSTED) {
          sum[kPostWeight][c][e] += d[c][e] * yhat[c][e];
          if (BIASES) sum[kPostBias][c][e] += d[c][e];
          d[c][e] *= (float)ow[c].v[e];
          s1 += d[c][e] * yhat[c][e];
          s2 += d[c][e];
        }
      }
    if (!a.dy) continue;
    if (POSTED && a.post != VNM_NORM_NONE) {               // (rows past 8192 channels have the kernel of all parts)
      const float2 s = row_sum2<TPR>(s1, s2, lds, turn);
      const float m1 = s.x / fn, m2 = a.post == VNM_NORM_LAYER ? s.y / fn : 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[c][e] = st.y * (d[c][e] - m2 - yhat[c][e] * m1);
    }
    store_row<XT, TPR, NCH>((XT*)a.dy + t * a.lddy, n, tid, vec, d);
  }
  // the worker's row of every sum that is asked for
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    if (b.part_at[k] < 0) continue;                      // (the parts that the kernel lacks are not asked for)
    float* p = b.part + b.part_at[k] + worker * n;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int at = (c * TPR + tid) * 8;
      if (n % 8 == 0) {
        if (at < n) {
          *(float4*)(p + at) = make_float4(sum[k][c][0], sum[k][c][1], sum[k][c][2], sum[k][c][3]);
          *(float4*)(p + at + 4) = make_float4(sum[k][c][4], sum[k][c][5], sum[k][c][6], sum[k][c][7]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (at + e < n) p[at + e] = sum[k][c][e];
      }
    }
  }
}

// out[row][i] = sum over the `count` rows of part from row * count on: 16 columns per workgroup, 64 threads per column that
// request eight rows at a time
struct ReduceArgs { const float* part[kSums]; float* out[kSums]; int64_t rows[kSums], count[kSums]; int64_t n; };
__global__ void __launch_bounds__(1024) column_reduce_kernel(const ReduceArgs r) {
  __shared__ float lds[64][17];
  const int col = threadIdx.x & 15, slice = threadIdx.x >> 4;
  const int64_t i = (int64_t)blockIdx.x * 16 + col;
  const int k = blockIdx.z;
  for (int64_t row = blockIdx.y; row < r.rows[k]; row += gridDim.y) {
    const int64_t count = r.count[k];
    const float* p = r.part[k] + row * count * r.n;
    float s = 0.f;
    if (i < r.n)
      for (int64_t w = slice; w < count; w += 512) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = w + 64 * q < count ? p[(w + 64 * q) * r.n + i] : 0.f;
        s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
      }
    lds[slice][col] = s;
    __syncthreads();
    if (slice < 4) {
#pragma unroll
      for (int q = 1; q < 16; ++q) s += lds[slice + 4 * q][col];
      lds[slice][col] = s;                                // (only its own thread has read this entry)
    }
    __syncthreads();
    if (slice == 0 && i < r.n) r.out[k][row * r.n + i] = (lds[0][col] + lds[1][col]) + (lds[2][col] + lds[3][col]);
    __syncthreads();
  }
}

template <typename HT, typename XT, int TPR, int NCH, int PARTS>
static int launch_back_cfg(const BackArgs& b, hipStream_t st) {
  constexpr int RPB = TPR == 64 ? 4 : 1, THREADS = TPR == 64 ? 256 : TPR;
  const int64_t blocks = (b.cut.groups * b.cut.pieces + RPB - 1) / RPB;
  if (blocks > 0x7FFFFFFF) return VNM_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((residual_norm_backward_kernel<HT, XT, TPR, NCH, PARTS>), dim3((unsigned)blocks), dim3(THREADS), 0, st, b);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "residual_norm_backward_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}
template <typename HT, typename XT, int PARTS>
static int launch_back_parts(const BackArgs& b, hipStream_t st) {
  if (b.a.n <= 512) return launch_back_cfg<HT, XT, 64, 1, PARTS>(b, st);
  if (b.a.n <= 1024) return launch_back_cfg<HT, XT, 128, 1, PARTS>(b, st);
  if (b.a.n <= 2048) return launch_back_cfg<HT, XT, 256, 1, PARTS>(b, st);
  if (b.a.n <= 4096) return launch_back_cfg<HT, XT, 512, 1, PARTS>(b, st);
  if (b.a.n <= 8192) return launch_back_cfg<HT, XT, 1024, 1, PARTS>(b, st);
  return launch_back_cfg<HT, XT, 1024, 2, kAllParts>(b, st);
}
static int parts_of(const vnm_residual_norm_backward_args& a) {
  const bool biases = a.post_bias || a.d_post_bias || a.d_pre_bias, gated = a.gate || a.d_gate;
  if (a.post != VNM_NORM_NONE) return biases || gated ? kAllParts : kPosted;
  return gated ? kBiases | kGated : biases ? kBiases : 0;
}
template <typename HT, typename XT>
static int launch_back(const BackArgs& b, hipStream_t st) {
  switch (parts_of(b.a)) {
    case kAllParts: return launch_back_parts<HT, XT, kAllParts>(b, st);
    case kPosted: return launch_back_parts<HT, XT, kPosted>(b, st);
    case kBiases | kGated: return launch_back_parts<HT, XT, kBiases | kGated>(b, st);
    case kBiases: return launch_back_parts<HT, XT, kBiases>(b, st);
  }
  return launch_back_parts<HT, XT, 0>(b, st);
}

static int64_t gate_rows(int64_t T, int64_t gate_tokens) { return gate_tokens > 0 ? (T + gate_tokens - 1) / gate_tokens : 1; }

}  // namespace vnm

using namespace vnm;

static bool dtype_ok(int t) { return t == VNM_F16 || t == VNM_F32 || t == VNM_BF16; }
static uintptr_t dtype_bytes(int t) { return t == VNM_F32 ? 4 : 2; }

extern "C" int vnm_residual_norm_backward_workspace_bytes(int64_t T, int64_t n, int64_t gate_tokens, int64_t* bytes) {
  if (!bytes) return VNM_ERR_NULL;
  if (T < 0 || n <= 0 || gate_tokens < 0) return VNM_ERR_SHAPE;
  if (n > VNM_NORM_MAX_CHANNELS) return VNM_ERR_UNSUPPORTED;
  const Cut c = make_cut(T, n, gate_tokens, true);       // (the most workers)
  const int64_t each = (c.groups * c.pieces * n * 4 + 255) / 256 * 256;
  *bytes = kSums * each + 256;
  return VNM_OK;
}

extern "C" int vnm_residual_norm_backward(const vnm_residual_norm_backward_args* args, void* workspace, int64_t workspace_bytes,
                                          void* stream) {
  if (!args) return VNM_ERR_NULL;
  const vnm_residual_norm_backward_args& a = *args;
  if (a.T < 0 || a.n <= 0 || a.gate_tokens < 0) return VNM_ERR_SHAPE;
  if (a.n > VNM_NORM_MAX_CHANNELS) return VNM_ERR_UNSUPPORTED;
  if (!dtype_ok(a.x_dtype) || !(a.h_dtype == a.x_dtype || a.h_dtype == VNM_F32)) return VNM_ERR_UNSUPPORTED;
  if (a.post < VNM_NORM_NONE || a.post > VNM_NORM_LAYER || a.pre < VNM_NORM_NONE || a.pre > VNM_NORM_LAYER) return VNM_ERR_UNSUPPORTED;
  const bool has_post = a.post != VNM_NORM_NONE, has_pre = a.pre != VNM_NORM_NONE;
  if (!has_post && (a.post_weight || a.post_bias || a.d_post_weight || a.d_post_bias)) return VNM_ERR_UNSUPPORTED;
  if (!has_pre && (a.pre_weight || a.d_pre_weight || a.d_pre_bias)) return VNM_ERR_UNSUPPORTED;
  if (workspace_bytes < 0) return VNM_ERR_WORKSPACE;
  const bool past_gate = a.dy || a.d_post_weight || a.d_post_bias || a.d_gate;
  const bool any_sum = a.d_pre_weight || a.d_pre_bias || a.d_post_weight || a.d_post_bias || a.d_gate;
  if (!a.dh && !a.dy && !any_sum) return VNM_ERR_NULL;
  if (a.T != 0) {
    if (!a.dx && !a.dh_out) return VNM_ERR_NULL;
    if ((a.dx && has_pre && (!a.h_new || !a.stats)) || (past_gate && has_post && (!a.y || !a.stats)) || (a.d_gate && !a.y))
      return VNM_ERR_NULL;
    if ((a.dx && a.lddx < a.n) || (a.dh_out && a.lddho < a.n) || (a.h_new && a.ldh < a.n) || (a.y && a.ldy < a.n) ||
        (a.gate && a.gate_tokens && a.ldg < a.n) || (a.dh && a.lddh < a.n) || (a.dy && a.lddy < a.n) ||
        (a.dh && a.dh == a.dh_out && a.lddh != a.lddho))
      return VNM_ERR_SHAPE;
  }
  const uintptr_t hp = (uintptr_t)a.dh_out | (uintptr_t)a.h_new | (uintptr_t)a.dh;
  const uintptr_t xp = (uintptr_t)a.dx | (uintptr_t)a.y | (uintptr_t)a.gate | (uintptr_t)a.post_weight | (uintptr_t)a.post_bias |
                       (uintptr_t)a.pre_weight | (uintptr_t)a.dy;
  const uintptr_t sp = (uintptr_t)a.d_post_weight | (uintptr_t)a.d_post_bias | (uintptr_t)a.d_pre_weight | (uintptr_t)a.d_pre_bias |
                       (uintptr_t)a.d_gate;
  if ((hp & (dtype_bytes(a.h_dtype) - 1)) || (xp & (dtype_bytes(a.x_dtype) - 1)) || (sp & 3) || ((uintptr_t)a.stats & 15) ||
      ((uintptr_t)workspace & 15))
    return VNM_ERR_ALIGN;
  if (a.T != 0 && any_sum && !workspace) return VNM_ERR_WORKSPACE;
  BackArgs b;
  b.a = a;
  const int parts = parts_of(a);
  b.cut = make_cut(a.T, a.n, a.gate_tokens, parts != kAllParts && !(parts & kGated));
  const int64_t workers = b.cut.groups * b.cut.pieces, each = (workers * a.n * 4 + 255) / 256 * 256;
  void* const outs[kSums] = {a.d_pre_weight, a.d_pre_bias, a.d_post_weight, a.d_post_bias, a.d_gate};
  ReduceArgs r{};
  r.n = a.n;
  int asked = 0;
  b.part = (float*)workspace;
  for (int k = 0; k < kSums; ++k) {
    b.part_at[k] = -1;
    if (!outs[k]) continue;
    b.part_at[k] = asked * (each / 4);
    r.part[asked] = b.part + b.part_at[k];
    r.out[asked] = (float*)outs[k];
    r.rows[asked] = k == kGate ? gate_rows(a.T, a.gate_tokens) : 1;
    r.count[asked] = k == kGate ? b.cut.pieces : workers;
    ++asked;
  }
  if (a.T != 0 && asked && workspace_bytes < asked * each) return VNM_ERR_WORKSPACE;
  if (a.T == 0) for (int k = 0; k < asked; ++k) r.count[k] = 0;       // the sums of no tokens
  hipStream_t st = (hipStream_t)stream;
  if (a.T != 0) {
    const int64_t lds = (a.dx ? a.lddx : 0) | (a.dh_out ? a.lddho : 0) | (a.h_new ? a.ldh : 0) | (a.y ? a.ldy : 0) |
                        (a.gate && a.gate_tokens ? a.ldg : 0) | (a.dh ? a.lddh : 0) | (a.dy ? a.lddy : 0);
    b.vec = a.n % 8 == 0 && lds % 8 == 0 && ((hp | xp) & 15) == 0;
    if (!a.gate_tokens) b.a.ldg = 0;
    int rc;
    if (a.x_dtype == VNM_F32) rc = launch_back<float, float>(b, st);
    else if (a.h_dtype == VNM_F32) rc = a.x_dtype == VNM_F16 ? launch_back<float, _Float16>(b, st) : launch_back<float, __bf16>(b, st);
    else rc = a.x_dtype == VNM_F16 ? launch_back<_Float16, _Float16>(b, st) : launch_back<__bf16, __bf16>(b, st);
    if (rc) return rc;
  }
  if (!asked) return VNM_OK;
  const int64_t rows = gate_rows(a.T, a.gate_tokens);
  const unsigned gy = (unsigned)(a.d_gate && rows > 1 ? (rows < 65535 ? rows : 65535) : 1);
  hipLaunchKernelGGL(column_reduce_kernel, dim3((unsigned)((a.n + 15) / 16), gy, (unsigned)asked), dim3(1024), 0, st, r);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "column_reduce_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}
