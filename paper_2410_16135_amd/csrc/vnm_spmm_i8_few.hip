// Few tokens: the int8 product as a stream of the packed weight (vnm_spmm_i8).
//
// Y^T = W' . Q^T on V_SMFMAC_I32_32X32X64_I8, the compressed weight being the sparse A operand and up to 32 tokens the B operand.
// A workgroup owns 32 or 64 rows; its waves cut K between them and add their sums through LDS at the end, which is exact in
// int32, so any cut gives the same bits.  The kept columns of a column block are picked from a token's raw bytes by byte
// permutations, whose selectors are laid out with the weight: activations are not re-laid, no second kernel, no workspace.
//
// Bound by the latency of one wave's chain (weights and activations of the next steps requested while this step's are picked),
// then by the bytes of the packed weight (1.27 per kept value).  Call after call from a graph, the next weight each time out of the
// last-level cache (so all times of this kernel here and in vnm_i8_rules.h), 64:2:5 unless said: 4096 x 4096 at 1 / 16 / 64 tokens
// 5.4 / 7.1 / 7.6 us, 11008 x 4096 7.3 / 8.3 / 14.6, 4096 x 11008 7.4 / 8.8 / 12.3, 11008 x 4096 at M = 8 5.7 / 6.5 / 11.2; at one
// token 1.6, 3.2, 3.1 and 2.5 TB/s.
#include "vnm_i8.h"
#include "vnm_i8_rules.h"

namespace vnm {

typedef unsigned u2v __attribute__((ext_vector_type(2)));
typedef unsigned u4v __attribute__((ext_vector_type(4)));
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
// into (selectors of bytes elsewhere give zero).  Selectors come 4 bits each, two blocks to a dword: 16 bytes per lane instead
// of 32 are a load less per step for one and a half instructions more per block.
template <int M>
__device__ __forceinline__ i8v i8_gather(const unsigned (&x)[2 * M], const u4v* sel) {
  constexpr int NSEL = i8_selectors(M);
  i8v b;
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    const int first = (M * d) >> 2;
    unsigned v = 0;
#pragma unroll
    for (int w = 0; w < NSEL; ++w) {
      const unsigned two = sel[w][d >> 1], s = (d & 1 ? two >> 4 : two) & 0x0f0f0f0fu;
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

// K steps of a chunk of activations: the next chunk is requested when this one goes to LDS, so it has that long to arrive.  Four
// steps for groups of four tokens, where they are a load or two per lane (4096 x 4096, M = 5: two steps 6.2 us, four 5.4, eight 5.3;
// 11008 x 4096 7.5, 7.3, 7.3; but 4096 x 11008 7.8, 7.4, 7.9 and 1000 x 1030, M = 7 3.4, 3.2, 3.7).
constexpr int i8_few_chunk(int M, int TT) { return TT == 4 && M <= 8 ? 4 : 2; }

// M: columns per block.  NT: column tables per 64-row block.  AT: 32-row tiles per workgroup (a row block's, or one of them).
// TT: tokens per workgroup.  WAVES: they cut the K steps between them, a contiguous run each.
template <int M, int NT, int AT, int TT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
spmm_i8_few_kernel(const I8FewArgs a, const int tp) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int NSEL = i8_selectors(M), G = (TT + 31) / 32, TABLES = AT == 2 ? NT : 1;
  constexpr int CS = i8_few_chunk(M, TT);          // K steps of a chunk of activations
  constexpr int PIECES = CS * M;                   // its 16-byte pieces per token
  constexpr int PITCH = PIECES * 16 + (M % 2 ? 8 : 16);   // 2 or 4 times an odd number of dwords: the lanes' reads below cover all banks
  constexpr int NX = (TT * PIECES + 63) / 64;      // pieces per lane
  // Fewer registers and with them more waves beat a longer reach from 16 tokens on: 11008 x 4096, M = 5 at 16 tokens 8.8 us with
  // four, 8.3 with two, 4096 x 11008 9.7 and 8.8 (but 4096 x 4096, a workgroup on every other compute unit, 6.7 and 7.1)
  constexpr int RW = TT == 4 ? 4 : 2;               // K steps whose weights are in flight
  const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
  const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned n = blockIdx.x;
  unsigned at = 0, rp = n;
  if (AT == 1) {
    // both tiles of a row block on one XCD (workgroup n runs on XCD n mod 8): they share the positions' and selectors' lines
    const bool by_xcd = n < (gridDim.x & ~15u);
    at = by_xcd ? (n >> 3) & 1 : n & 1;
    rp = by_xcd ? (n >> 4) * 8 + (n & 7) : n >> 1;
  }
  const int64_t t0 = (int64_t)blockIdx.y * TT;
  const int nt = a.T - t0 < TT ? (int)(a.T - t0) : TT;
  const unsigned S = a.S, per = (S + WAVES - 1) / WAVES;
  const unsigned s0 = wave * per < S ? wave * per : S, s1 = s0 + per < S ? s0 + per : S;
  const size_t rs0 = (size_t)rp * S;
  unsigned char* const xs = smem + wave * (TT * PITCH);        // this wave's activations: [token][a chunk's raw columns]

  // addresses as a uniform base and a 32-bit offset of the lane
  const unsigned char* const xbase = a.Q + t0 * a.ldq;
  unsigned xrow[NX], xcol[NX], xdst[NX];
#pragma unroll
  for (int i = 0; i < NX; ++i) {
    int q = i * 64 + lane;
    if (q >= TT * PIECES) q = TT * PIECES - 1;
    const int tok = q / PIECES, piece = q - tok * PIECES;
    xrow[i] = (unsigned)(tok < nt ? tok : nt - 1) * (unsigned)a.ldq;
    xcol[i] = piece * 16;
    xdst[i] = tok * PITCH + piece * 16;
  }
  u4v xr[NX];                                      // (passed to what follows: captured, it costs up to 9 % at 32 tokens)
  // A piece that begins inside the row is read whole: it is aligned, so what it holds past the row's end stands in the same
  // 16 bytes as the row's last channel.  Columns past the end meet weights that are zero.
  auto load_x = [&](u4v (&xr)[NX], unsigned s) {
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const unsigned c = s * (16 * M) + xcol[i];
      xr[i] = *(const u4v*)(xbase + (xrow[i] + (c < (unsigned)a.in ? c : 0u)));
    }
  };
  auto store_x = [&](const u4v (&xr)[NX]) {
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      if constexpr (M % 2 == 0) *(u4v*)(xs + xdst[i]) = xr[i];
      else {
        *(u2v*)(xs + xdst[i]) = xr[i].xy;
        *(u2v*)(xs + xdst[i] + 8) = xr[i].zw;
      }
    }
  };
  struct Slot { u4v w[AT]; unsigned idx[AT]; u4v sel[TABLES * NSEL]; };
  auto load_w = [&](Slot& o, unsigned s) {
    s = s < S ? s : S - 1;                         // (beyond the wave's range: not used)
    const size_t rs = rs0 + s;
#pragma unroll
    for (int i = 0; i < AT; ++i) o.w[i] = *(const u4v*)(a.pa + (rs * 2 + (AT == 2 ? i : at)) * 1024 + (unsigned)(lane * 16));
    if constexpr (AT == 2) {
      const u2v v = *(const u2v*)(a.pidx + rs * 512 + (unsigned)(lane * 8));
      o.idx[0] = v.x; o.idx[1] = v.y;
    } else o.idx[0] = *(const unsigned*)(a.pidx + rs * 512 + at * 4 + (unsigned)(lane * 8));
#pragma unroll
    for (int t = 0; t < TABLES; ++t)
#pragma unroll
      for (int k = 0; k < NSEL; ++k)
        o.sel[t * NSEL + k] = *(const u4v*)(a.psel + ((rs * NT + (AT == 2 ? t : NT == 2 ? at : 0)) * NSEL + k) * 32 + (unsigned)(h * 16));
  };
  i16v acc[AT][G];
#pragma unroll
  for (int i = 0; i < AT; ++i)
#pragma unroll
    for (int g = 0; g < G; ++g) acc[i][g] = (i16v)0;
  auto multiply = [&](const Slot& o, int sl) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int tok = g * 32 + j < TT ? g * 32 + j : TT - 1;
      const unsigned char* p = xs + tok * PITCH + sl * (16 * M) + h * (8 * M);
      unsigned x[2 * M];
      if constexpr (M % 2 == 0) {
#pragma unroll
        for (int k = 0; k < M / 2; ++k) {
          const u4v v = *(const u4v*)(p + 16 * k);
          x[4 * k] = v.x; x[4 * k + 1] = v.y; x[4 * k + 2] = v.z; x[4 * k + 3] = v.w;
        }
      } else {
#pragma unroll
        for (int k = 0; k < M; ++k) {
          const u2v v = *(const u2v*)(p + 8 * k);
          x[2 * k] = v.x; x[2 * k + 1] = v.y;
        }
      }
      i8v b = i8_gather<M>(x, o.sel);
#pragma unroll
      for (int i = 0; i < AT; ++i) {
        if (TABLES == 2 && i == 1) b = i8_gather<M>(x, o.sel + NSEL);
        acc[i][g] = __builtin_amdgcn_smfmac_i32_32x32x64_i8(__builtin_bit_cast(i4v, o.w[i]), b, acc[i][g], (int)o.idx[i], 0, 0);
      }
    }
  };
  constexpr int BODY = CS > RW ? CS : RW;          // steps after which chunks and slots are back in place
  static_assert(BODY % CS == 0 && BODY % RW == 0, "whole chunks and rounds of slots");
  Slot ring[RW];
  load_x(xr, s0);
#pragma unroll
  for (int k = 0; k < RW; ++k) load_w(ring[k], s0 + k);
  for (unsigned sb = s0; sb < s1; sb += BODY) {
#pragma unroll
    for (int c = 0; c < BODY; c += CS) {
      const unsigned sc = sb + c;
      if (sc >= s1) break;
      // The chunk's activations go through LDS, where each lane finds the run of its token.  The region is the wave's own and
      // LDS executes a wave's accesses in order; the fences keep the compiler from moving reads and writes past each other.
      __builtin_amdgcn_wave_barrier();
      store_x(xr);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      load_x(xr, sc + CS);
#pragma unroll
      for (int k = 0; k < CS; ++k) {
        if (sc + k < s1) multiply(ring[(c + k) % RW], k);
        load_w(ring[(c + k) % RW], sc + k + RW);
      }
    }
  }
  __syncthreads();                                 // the sums take the place of the activations
  int* red = (int*)smem;                           // [wave][row][tp]
#pragma unroll
  for (int g = 0; g < G; ++g)
    if (g * 32 + j < nt) {
#pragma unroll
      for (int i = 0; i < AT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          red[(wave * (32 * AT) + i * 32 + 8 * (r >> 2) + 4 * h + (r & 3)) * tp + g * 32 + j] = acc[i][g][r];
    }
  __syncthreads();
  for (int k = threadIdx.x; k < 32 * AT * nt; k += 64 * WAVES) {
    const int row = k % (32 * AT), tok = k / (32 * AT);
    const int64_t o = (int64_t)rp * 64 + at * 32 + row, t = t0 + tok;
    if (o >= a.out) continue;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += red[(w * (32 * AT) + row) * tp + tok];
    i8_store(a.e, t, o, i8_result(sum, a.e.scale_w[o], a.e.scale_x[t], a.e.bias, a.e.bias ? (float)a.e.bias[o] : 0.f));
  }
}

template <int M, int NT, int AT, int TT, int WAVES>
static int launch_few_cfg(const I8FewArgs& a, int64_t R64, hipStream_t st) {
  constexpr int CS = i8_few_chunk(M, TT), PITCH = CS * M * 16 + (M % 2 ? 8 : 16);
  auto kern = spmm_i8_few_kernel<M, NT, AT, TT, WAVES>;
  const int tp = (int)(a.T < TT ? a.T : TT) | 1;
  const size_t xs = (size_t)WAVES * TT * PITCH, sums = (size_t)WAVES * 32 * AT * tp * 4, lds = xs > sums ? xs : sums;
  if (lds > 64 * 1024)
    if (int rc = allow_big_lds((const void*)kern, "hipFuncSetAttribute(spmm_i8_few)")) return rc;
  static_assert((size_t)WAVES * TT * PITCH <= 160 * 1024 && (size_t)WAVES * 32 * AT * (TT | 1) * 4 <= 160 * 1024, "LDS of a compute unit");
  hipLaunchKernelGGL(kern, dim3((unsigned)(AT == 1 ? 2 * R64 : R64), (unsigned)((a.T + TT - 1) / TT)), dim3(64 * WAVES), lds, st, a, tp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "spmm_i8_few_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}
template <int M, int NT>
static int launch_few_m(const I8FewArgs& a, const Dims& d, hipStream_t st) {
  const int64_t R64 = packed_row_blocks(d);
  const I8FewShape s = i8_few_shape(a.T, R64, a.S, M);
  if (s.tiles == 2) return launch_few_cfg<M, NT, 2, 32, 4>(a, R64, st);
  if (s.waves == 8)
    return s.tokens == 4 ? launch_few_cfg<M, NT, 1, 4, 8>(a, R64, st) : s.tokens == 16 ? launch_few_cfg<M, NT, 1, 16, 8>(a, R64, st)
                                                                       : launch_few_cfg<M, NT, 1, 32, 8>(a, R64, st);
  return s.tokens == 4 ? launch_few_cfg<M, NT, 1, 4, 4>(a, R64, st) : s.tokens == 16 ? launch_few_cfg<M, NT, 1, 16, 4>(a, R64, st)
                                                                     : launch_few_cfg<M, NT, 1, 32, 4>(a, R64, st);
}
template <int M>
static int launch_few_m(const I8FewArgs& a, const Dims& d, hipStream_t st) {
  return packed_tables(d.V) == 2 ? launch_few_m<M, 2>(a, d, st) : launch_few_m<M, 1>(a, d, st);
}

int launch_spmm_i8_few(const void* Q, int64_t T, int64_t ldq, const void* packed, const Dims& d, const I8Epilogue& e, hipStream_t st) {
  const I8Layout l = i8_layout(d);
  const unsigned char* p = (const unsigned char*)packed;
  // (ldq <= kI8MaxRowPitch, and i8_sums_fit bounds a row at 2^20 channels: 64 rows and a step stay in 31 bits)
  if (2 * packed_row_blocks(d) > 0x7FFFFFFF || (T + 3) / 4 > 65535 || ldq > kI8MaxRowPitch) return VNM_ERR_UNSUPPORTED;
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
