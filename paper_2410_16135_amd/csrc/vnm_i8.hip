// The V:N:M layer in 8-bit integers: C entry points, the packed copy of an int8 weight, and the product on the canonical triple.
#include "vnm_i8.h"
#include "vnm_i8_rules.h"

namespace vnm {

// ---------------------------------------------------------------- pack
// One thread per (64-row block, step, tile, lane) for the A operand, and one per dword of the two column tables.
__global__ void __launch_bounds__(256)
pack_i8_kernel(const unsigned char* __restrict__ qvalues, const unsigned char* __restrict__ meta,
               const unsigned char* __restrict__ colidx, int64_t in, int V, int M, int64_t R, int64_t B, int64_t RS, int64_t S,
               int nsel, unsigned char* __restrict__ pa, unsigned* __restrict__ pidx, unsigned* __restrict__ pcol,
               unsigned* __restrict__ psel) {
  const int NT = V == 32 ? 2 : 1;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (gid < RS * 128) {
    const int lane = (int)(gid & 63), at = (int)((gid >> 6) & 1);
    const int64_t rs = gid >> 7, s = rs % S, rp = rs / S;
    const int i = lane & 31, h = lane >> 5;
    const int64_t row = rp * 64 + at * 32 + i;
    unsigned char v[16];
    unsigned idx = 0;
#pragma unroll
    for (int g = 0; g < 8; ++g) {                          // bytes 2 g, 2 g + 1: block 8 (g / 4) + 4 h + g mod 4
      const int64_t b = s * 16 + 8 * (g >> 2) + 4 * h + (g & 3);
      unsigned nib = 4, v0 = 0, v1 = 0;                    // (0, 1)
      if (b < B && row < R * V) {
        const unsigned byte = meta[row * ((B + 1) / 2) + (b >> 1)];
        nib = (b & 1) ? byte >> 4 : byte & 15u;
        const unsigned char* c = colidx + ((row / V) * B + b) * 4;
        if (b * M + c[nib & 3] < in) v0 = qvalues[row * 2 * B + 2 * b];
        if (b * M + c[nib >> 2] < in) v1 = qvalues[row * 2 * B + 2 * b + 1];
      }
      v[2 * g] = (unsigned char)v0;
      v[2 * g + 1] = (unsigned char)v1;
      idx |= nib << (4 * g);
    }
    uint4 q;
    q.x = v[0] | v[1] << 8 | v[2] << 16 | (unsigned)v[3] << 24;
    q.y = v[4] | v[5] << 8 | v[6] << 16 | (unsigned)v[7] << 24;
    q.z = v[8] | v[9] << 8 | v[10] << 16 | (unsigned)v[11] << 24;
    q.w = v[12] | v[13] << 8 | v[14] << 16 | (unsigned)v[15] << 24;
    *(uint4*)(pa + gid * 16) = q;
    pidx[rs * 128 + lane * 2 + at] = idx;
  }
  if (gid < RS * 16 * NT) {
    const int t = (int)(gid % NT), role = (int)(gid / NT % 16), h = role >> 3, r = role & 7;
    const int64_t rs = gid / NT / 16, s = rs % S, rb = ((rs / S) * 64 + t * 32) / V;
    unsigned o = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int blk = 8 * h + 2 * i + (r >> 2);
      const int64_t b = s * 16 + blk;
      const unsigned c = b < B && rb < R ? colidx[(rb * B + b) * 4 + (r & 3)] : (unsigned)(r & 3);
      o |= (unsigned)(blk * M + (int)c) << (8 * i);
    }
    pcol[gid] = o;
  }
  if (gid < RS * 8 * NT) {                                 // two blocks of a lane half's run
    const int i = (int)(gid & 3), h = (int)(gid >> 2) & 1, t = (int)(gid / 8 % NT);
    const int64_t rs = gid / 8 / NT, s = rs % S, rb = ((rs / S) * 64 + t * 32) / V;
    for (int w = 0; w < nsel; ++w) {
      unsigned sel = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = 2 * i + e, first = (M * d) & 3;      // byte of the block's first column in its first dword
        const int64_t b = s * 16 + 8 * h + d;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int at = first + (b < B && rb < R ? (int)colidx[(rb * B + b) * 4 + k] : k) - 8 * w;
          sel |= (unsigned)(at >= 0 && at < 8 ? at : 12) << (8 * k + 4 * e);
        }
      }
      psel[(((rs * NT + t) * nsel + w) * 2 + h) * 4 + i] = sel;
    }
  }
}

int launch_pack_i8(const void* qvalues, const void* meta, const void* colidx, const Dims& d, void* packed, hipStream_t st) {
  const I8Layout l = i8_layout(d);
  if (l.total == 0) return VNM_ERR_UNSUPPORTED;
  const int64_t S = i8_steps(d), RS = packed_row_blocks(d) * S;
  if ((RS * 128 + 255) / 256 > 0x7FFFFFFF) return VNM_ERR_UNSUPPORTED;
  unsigned char* p = (unsigned char*)packed;
  hipLaunchKernelGGL(pack_i8_kernel, dim3((unsigned)((RS * 128 + 255) / 256)), dim3(256), 0, st, (const unsigned char*)qvalues,
                     (const unsigned char*)meta, (const unsigned char*)colidx, d.in, d.V, d.M, d.R, d.B, RS, S, i8_selectors(d.M), p,
                     (unsigned*)(p + l.pidx_off), (unsigned*)(p + l.pcol_off), (unsigned*)(p + l.psel_off));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "pack_i8_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}

// ---------------------------------------------------------------- product on the canonical triple
// One thread per output, written straight from the formula: any V, M, width and alignment.
__global__ void __launch_bounds__(256)
spmm_i8_triple_kernel(const signed char* __restrict__ Q, int64_t ldq, const signed char* __restrict__ qvalues,
                      const unsigned char* __restrict__ meta, const unsigned char* __restrict__ colidx, int64_t out, int64_t in,
                      int V, int M, int64_t B, int64_t t0, const I8Epilogue e) {
  const int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x, t = t0 + blockIdx.y;
  if (o >= out) return;
  const signed char* x = Q + t * ldq;
  const signed char* v = qvalues + o * 2 * B;
  const unsigned char* mrow = meta + o * ((B + 1) / 2);
  const unsigned char* crow = colidx + o / V * B * 4;
  int acc = 0;
  for (int64_t b = 0; b < B; ++b) {
    const unsigned byte = mrow[b >> 1], nib = (b & 1) ? byte >> 4 : byte & 15u;
    const int64_t c0 = b * M + crow[b * 4 + (nib & 3)], c1 = b * M + crow[b * 4 + (nib >> 2)];
    if (c0 < in) acc += (int)v[2 * b] * x[c0];
    if (c1 < in) acc += (int)v[2 * b + 1] * x[c1];
  }
  i8_store(e, t, o, i8_result(acc, e.scale_w[o], e.scale_x[t], e.bias, e.bias ? (float)e.bias[o] : 0.f));
}

int launch_spmm_i8_triple(const void* Q, int64_t T, int64_t ldq, const void* qvalues, const void* meta, const void* colidx,
                          const Dims& d, const I8Epilogue& e, hipStream_t st) {
  if ((d.out + 255) / 256 > 0x7FFFFFFF) return VNM_ERR_UNSUPPORTED;
  for (int64_t t0 = 0; t0 < T; t0 += 65535) {                     // grid.y limit
    const int64_t nt = T - t0 < 65535 ? T - t0 : 65535;
    hipLaunchKernelGGL(spmm_i8_triple_kernel, dim3((unsigned)((d.out + 255) / 256), (unsigned)nt), dim3(256), 0, st,
                       (const signed char*)Q, ldq, (const signed char*)qvalues, (const unsigned char*)meta,
                       (const unsigned char*)colidx, d.out, d.in, d.V, d.M, d.B, t0, e);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) { set_hip_error(err, "spmm_i8_triple_kernel"); return VNM_ERR_HIP; }
  }
  return VNM_OK;
}

}  // namespace vnm

using namespace vnm;

extern "C" int vnm_i8_packed_bytes(int64_t out, int64_t in, int V, int N, int M, int64_t* bytes) {
  if (!bytes) return VNM_ERR_NULL;
  if (int rc = check_pattern(out, in, V, N, M)) return rc;
  *bytes = i8_layout(make_dims(out, in, V, M)).total;
  return VNM_OK;
}

extern "C" int vnm_quantize_compressed(const void* values, const void* meta, const void* colidx, int64_t out, int64_t in, int V,
                                       int N, int M, void* qvalues, void* scale, void* packed, void* stream) {
  if (!values || !meta || !colidx || !qvalues || !scale) return VNM_ERR_NULL;
  if (int rc = check_pattern(out, in, V, N, M)) return rc;
  if (((uintptr_t)values & 1) || ((uintptr_t)scale & 3) || ((uintptr_t)packed & 255)) return VNM_ERR_ALIGN;
  if (packed && !has_packed(V, M)) return VNM_ERR_UNSUPPORTED;
  const Dims d = make_dims(out, in, V, M);
  // (the rows past `out` hold zeros: their int8 values become zeros and their scales are not stored)
  if (int rc = launch_quantize_rows(values, d.out_pad, 2 * d.B, 2 * d.B, VNM_F16, qvalues, 2 * d.B, scale, out, (hipStream_t)stream))
    return rc;
  return packed ? launch_pack_i8(qvalues, meta, colidx, d, packed, (hipStream_t)stream) : VNM_OK;
}

extern "C" int vnm_pack_i8(const void* qvalues, const void* meta, const void* colidx, int64_t out, int64_t in, int V, int N, int M,
                           void* packed, void* stream) {
  if (!qvalues || !meta || !colidx || !packed) return VNM_ERR_NULL;
  if (int rc = check_pattern(out, in, V, N, M)) return rc;
  if (!has_packed(V, M)) return VNM_ERR_UNSUPPORTED;
  if ((uintptr_t)packed & 255) return VNM_ERR_ALIGN;
  return launch_pack_i8(qvalues, meta, colidx, make_dims(out, in, V, M), packed, (hipStream_t)stream);
}

extern "C" int vnm_spmm_i8_workspace_bytes(int64_t T, int64_t out, int64_t in, int V, int N, int M, int64_t* bytes) {
  if (!bytes) return VNM_ERR_NULL;
  if (int rc = check_pattern(out, in, V, N, M)) return rc;
  if (T < 0) return VNM_ERR_SHAPE;
  const Dims d = make_dims(out, in, V, M);
  *bytes = has_packed(V, M) && T > 0 && !i8_takes_few(T, packed_row_blocks(d), in, i8_steps(d), M) ? staged_q_bytes(T, d) : 0;
  return VNM_OK;
}

static bool dtype_ok(int t) { return t == VNM_F16 || t == VNM_F32 || t == VNM_BF16; }
static uintptr_t dtype_mask(int t) { return t == VNM_F32 ? 3 : 1; }

extern "C" int vnm_spmm_i8(const void* Q, int64_t T, int64_t ldq, const void* scale_x, const void* qvalues, const void* meta,
                           const void* colidx, const void* packed, const void* scale_w, int64_t out, int64_t in, int V, int N, int M,
                           const void* bias, void* Y, int64_t ldy, int y_dtype, int path, void* workspace, int64_t workspace_bytes,
                           void* stream) {
  if (!qvalues || !meta || !colidx || !scale_w) return VNM_ERR_NULL;
  if (T != 0 && (!Q || !scale_x || !Y)) return VNM_ERR_NULL;      // an empty batch may come with null tensors
  if (int rc = check_pattern(out, in, V, N, M)) return rc;
  if (T < 0 || ldq < in || ldy < out) return VNM_ERR_SHAPE;
  if (!dtype_ok(y_dtype)) return VNM_ERR_UNSUPPORTED;
  if (path != VNM_PATH_AUTO && path != VNM_PATH_GENERIC && path != VNM_PATH_SMFMAC) return VNM_ERR_UNSUPPORTED;
  if (workspace_bytes < 0) return VNM_ERR_WORKSPACE;
  if (((uintptr_t)Y & dtype_mask(y_dtype)) || ((uintptr_t)scale_x & 3) || ((uintptr_t)scale_w & 3) || ((uintptr_t)bias & 1) ||
      ((uintptr_t)packed & 255))
    return VNM_ERR_ALIGN;
  const Dims d = make_dims(out, in, V, M);
  if (!i8_sums_fit(d)) return VNM_ERR_UNSUPPORTED;
  if (T == 0) return VNM_OK;
  // (rows so far apart that 64 of them leave 31 bits are the kernel on the triple's business)
  const bool matrix = packed && has_packed(V, M) && ldq % 16 == 0 && ((uintptr_t)Q & 15) == 0 && ldq <= kI8MaxRowPitch;
  if (path == VNM_PATH_SMFMAC && !matrix) return VNM_ERR_UNSUPPORTED;
  const I8Epilogue e{(const float*)scale_x, (const float*)scale_w, (const _Float16*)bias, Y, ldy, y_dtype};
  if (path != VNM_PATH_GENERIC && matrix) {
    if (i8_takes_few(T, packed_row_blocks(d), in, i8_steps(d), M)) return launch_spmm_i8_few(Q, T, ldq, packed, d, e, (hipStream_t)stream);
    if (!workspace || workspace_bytes < staged_q_bytes(T, d)) return VNM_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255) return VNM_ERR_ALIGN;
    if (int rc = launch_stage_q(Q, T, ldq, d, workspace, (hipStream_t)stream)) return rc;
    return launch_spmm_i8_staged(workspace, T, packed, d, e, (hipStream_t)stream);
  }
  return launch_spmm_i8_triple(Q, T, ldq, qvalues, meta, colidx, d, e, (hipStream_t)stream);
}

extern "C" int vnm_stage_q_bytes(int64_t T, int64_t in, int M, int64_t* bytes) {
  if (!bytes) return VNM_ERR_NULL;
  if (in <= 0 || T < 0) return VNM_ERR_SHAPE;
  if (M < 4 || M > 16) return VNM_ERR_UNSUPPORTED;
  *bytes = staged_q_bytes(T, make_dims(64, in, 64, M));            // (the layout depends on in and M only)
  return VNM_OK;
}

extern "C" int vnm_stage_q(const void* Q, int64_t T, int64_t ldq, int64_t in, int M, void* staged, int64_t staged_bytes, void* stream) {
  if (T != 0 && (!Q || !staged)) return VNM_ERR_NULL;
  if (in <= 0 || T < 0 || ldq < in) return VNM_ERR_SHAPE;
  if (M < 4 || M > 16 || ldq % 16 != 0 || ((uintptr_t)Q & 15) || in > 0x7FFFFFFF) return VNM_ERR_UNSUPPORTED;
  if (T == 0) return VNM_OK;
  const Dims d = make_dims(64, in, 64, M);
  if (staged_bytes < staged_q_bytes(T, d)) return VNM_ERR_WORKSPACE;
  if ((uintptr_t)staged & 255) return VNM_ERR_ALIGN;
  return launch_stage_q(Q, T, ldq, d, staged, (hipStream_t)stream);
}

extern "C" int vnm_spmm_i8_staged(const void* staged, int64_t staged_bytes, int64_t T, const void* scale_x, const void* packed,
                                  const void* scale_w, int64_t out, int64_t in, int V, int N, int M, const void* bias, void* Y,
                                  int64_t ldy, int y_dtype, void* stream) {
  if (!packed || !scale_w || (T != 0 && (!staged || !scale_x || !Y))) return VNM_ERR_NULL;
  if (int rc = check_pattern(out, in, V, N, M)) return rc;
  if (T < 0 || ldy < out) return VNM_ERR_SHAPE;
  if (!dtype_ok(y_dtype) || !has_packed(V, M)) return VNM_ERR_UNSUPPORTED;
  if (((uintptr_t)staged & 255) || ((uintptr_t)packed & 255) || ((uintptr_t)Y & dtype_mask(y_dtype)) || ((uintptr_t)scale_x & 3) ||
      ((uintptr_t)scale_w & 3) || ((uintptr_t)bias & 1))
    return VNM_ERR_ALIGN;
  const Dims d = make_dims(out, in, V, M);
  if (!i8_sums_fit(d)) return VNM_ERR_UNSUPPORTED;
  if (T == 0) return VNM_OK;
  if (staged_bytes < staged_q_bytes(T, d)) return VNM_ERR_WORKSPACE;
  const I8Epilogue e{(const float*)scale_x, (const float*)scale_w, (const _Float16*)bias, Y, ldy, y_dtype};
  return launch_spmm_i8_staged(staged, T, packed, d, e, (hipStream_t)stream);
}
