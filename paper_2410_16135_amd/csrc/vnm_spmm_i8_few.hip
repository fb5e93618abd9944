// Few tokens: the int8 product as a stream of the packed weight (vnm_spmm_i8).
#include "vnm_i8.h"

namespace vnm {

typedef int i4v __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));
typedef int i16v __attribute__((ext_vector_type(16)));

struct I8FewArgs {
  const unsigned char* Q; int64_t T, ldq; int in;
  const unsigned char* pa; const unsigned char* pidx; const unsigned char* psel;
  int64_t out; unsigned S;
  I8Epilogue e;
};

// The 4 kept columns of the 8 blocks of a lane's run, from its raw dwords: a byte permutation per 8 bytes that a block can reach
// into (selectors of bytes elsewhere give zero).
template <int M>
__device__ __forceinline__ i8v i8_gather(const unsigned (&x)[2 * M], const uint4* sel) {
  constexpr int NSEL = i8_selectors(M);
  i8v b;
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    const int first = (M * d) >> 2;
    unsigned v = 0;
#pragma unroll
    for (int w = 0; w < NSEL; ++w) {
      const unsigned s = ((const unsigned*)(sel + 2 * w))[d];
      const int lo = first + 2 * w, hi = lo + 1;
      if (lo < 2 * M) {
        const unsigned p = __builtin_amdgcn_perm(hi < 2 * M ? x[hi] : 0u, x[lo], s);
        v = w == 0 ? p : v | p;
      }
    }
    b[d] = (int)v;
  }
  return b;
}

template <int M, int NT, int WAVES, int RING>
__global__ void __launch_bounds__(64 * WAVES)
spmm_i8_few_kernel(const I8FewArgs a, const int tp) {
  extern __shared__ __attribute__((aligned(16))) int red[];       // [wave][row][tp tokens]
  constexpr int NSEL = i8_selectors(M);
  const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
  const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned n = blockIdx.x;
  // both tiles of a row block on one XCD (workgroup n runs on XCD n mod 8): they share the positions' and selectors' lines
  const bool by_xcd = n < (gridDim.x & ~15u);
  const unsigned at = by_xcd ? (n >> 3) & 1 : n & 1, rp = by_xcd ? (n >> 4) * 8 + (n & 7) : n >> 1;
  const int64_t t0 = (int64_t)blockIdx.y * 32;
  const int nt = a.T - t0 < 32 ? (int)(a.T - t0) : 32;
  const unsigned char* xrow = a.Q + (t0 + (j < nt ? j : nt - 1)) * a.ldq;
  const unsigned S = a.S;
  const size_t rs0 = (size_t)rp * S;

  struct Slot { uint4 w; unsigned idx; uint4 sel[2 * NSEL]; unsigned x[2 * M]; };
  auto load = [&](Slot& o, unsigned s) {
    s = s < S ? s : S - 1;                         // (beyond the range: not used)
    const size_t rs = rs0 + s;
    o.w = *(const uint4*)(a.pa + (rs * 2 + at) * 1024 + lane * 16);
    o.idx = *(const unsigned*)(a.pidx + rs * 512 + lane * 8 + at * 4);
#pragma unroll
    for (int k = 0; k < NSEL; ++k)
#pragma unroll
      for (int q = 0; q < 2; ++q)
        o.sel[2 * k + q] = *(const uint4*)(a.psel + ((rs * NT + (NT == 2 ? at : 0)) * NSEL + k) * 64 + h * 32 + q * 16);
    const int col = (int)(s * 16 * M) + 8 * M * h;
    // A piece that begins inside the row is read whole: it is aligned, so what it holds past the row's end stands in the same
    // 16 bytes as the row's last channel.  A piece past the end meets weights that are zero.
    if constexpr (M % 2 == 0) {
#pragma unroll
      for (int k = 0; k < M / 2; ++k) {
        const int c = col + 16 * k;
        const uint4 v = *(const uint4*)(xrow + (c < a.in ? c : 0));
        o.x[4 * k] = v.x; o.x[4 * k + 1] = v.y; o.x[4 * k + 2] = v.z; o.x[4 * k + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < M; ++k) {
        const int c = col + 8 * k;
        const uint2 v = *(const uint2*)(xrow + (c < a.in ? c : 0));
        o.x[2 * k] = v.x; o.x[2 * k + 1] = v.y;
      }
    }
  };
  Slot ring[RING];
  i16v acc = {};
  auto multiply = [&](const Slot& o) {
    const i8v b = i8_gather<M>(o.x, o.sel);
    acc = __builtin_amdgcn_smfmac_i32_32x32x64_i8(__builtin_bit_cast(i4v, o.w), b, acc, (int)o.idx, 0, 0);
  };
#pragma unroll
  for (int i = 0; i < RING; ++i) load(ring[i], wave + i * WAVES);
  for (unsigned sb = wave; sb < S; sb += RING * WAVES) {
    if (sb + RING * WAVES < S) {
#pragma unroll
      for (int i = 0; i < RING; ++i) {
        multiply(ring[i]);                         // (sb + i * WAVES < S, as the round after this one exists)
        load(ring[i], sb + (RING + i) * WAVES);
      }
    } else {
#pragma unroll
      for (int i = 0; i < RING; ++i)
        if (sb + i * WAVES < S) multiply(ring[i]);
    }
  }
  if (j < nt) {
#pragma unroll
    for (int r = 0; r < 16; ++r) red[(wave * 32 + 8 * (r >> 2) + 4 * h + (r & 3)) * tp + j] = acc[r];
  }
  __syncthreads();
  for (int k = threadIdx.x; k < 32 * nt; k += 64 * WAVES) {
    const int row = k & 31, tok = k >> 5;
    const int64_t o = (int64_t)rp * 64 + at * 32 + row, t = t0 + tok;
    if (o >= a.out) continue;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += red[(w * 32 + row) * tp + tok];
    float y = i8_result(sum, a.e.scale_w[o], a.e.scale_x[t]);
    if (a.e.bias) y = __fadd_rn(y, (float)a.e.bias[o]);
    i8_store(a.e, t, o, y);
  }
}

template <int M, int NT, int WAVES>
static int launch_few_cfg(const I8FewArgs& a, int64_t R64, hipStream_t st) {
  constexpr int RING = M <= 5 ? 4 : M <= 8 ? 3 : 2;
  auto kern = spmm_i8_few_kernel<M, NT, WAVES, RING>;
  if (int rc = allow_big_lds((const void*)kern, "hipFuncSetAttribute(spmm_i8_few)")) return rc;
  const int tp = (int)(a.T < 32 ? a.T : 32) | 1;
  hipLaunchKernelGGL(kern, dim3((unsigned)(2 * R64), (unsigned)((a.T + 31) / 32)), dim3(64 * WAVES), (size_t)WAVES * 32 * tp * 4, st, a, tp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "spmm_i8_few_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}
template <int M>
static int launch_few_m(const I8FewArgs& a, const Dims& d, hipStream_t st) {
  const int64_t R64 = packed_row_blocks(d);
  if (packed_tables(d.V) == 2) return a.S > 8 ? launch_few_cfg<M, 2, 16>(a, R64, st) : launch_few_cfg<M, 2, 4>(a, R64, st);
  return a.S > 8 ? launch_few_cfg<M, 1, 16>(a, R64, st) : launch_few_cfg<M, 1, 4>(a, R64, st);
}

int launch_spmm_i8_few(const void* Q, int64_t T, int64_t ldq, const void* packed, const Dims& d, const I8Epilogue& e, hipStream_t st) {
  const I8Layout l = i8_layout(d);
  const unsigned char* p = (const unsigned char*)packed;
  if (2 * packed_row_blocks(d) > 0x7FFFFFFF || (T + 31) / 32 > 65535 || i8_steps(d) * 16 * d.M > 0x7FFFFFFF) return VNM_ERR_UNSUPPORTED;
  const I8FewArgs a{(const unsigned char*)Q, T, ldq, (int)d.in, p, p + l.pidx_off, p + l.psel_off, d.out, (unsigned)i8_steps(d), e};
  switch (d.M) {
    case 4: return launch_few_m<4>(a, d, st);
    case 5: return launch_few_m<5>(a, d, st);
    case 6: return launch_few_m<6>(a, d, st);
    case 7: return launch_few_m<7>(a, d, st);
    case 8: return launch_few_m<8>(a, d, st);
    case 9: return launch_few_m<9>(a, d, st);
    case 10: return launch_few_m<10>(a, d, st);
    case 11: return launch_few_m<11>(a, d, st);
    case 12: return launch_few_m<12>(a, d, st);
    case 13: return launch_few_m<13>(a, d, st);
    case 14: return launch_few_m<14>(a, d, st);
    case 15: return launch_few_m<15>(a, d, st);
    case 16: return launch_few_m<16>(a, d, st);
  }
  return VNM_ERR_UNSUPPORTED;
}

}  // namespace vnm
