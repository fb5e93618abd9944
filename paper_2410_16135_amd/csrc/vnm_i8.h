// Declarations shared by the sources of the 8-bit layers (not part of the C ABI).
#pragma once
#include "vnm_internal.h"

namespace vnm {

// ---- the packed copy of an int8 weight ------------------------------------------------------------
// A K step is one V_SMFMAC_I32_32X32X64_I8: 64 compacted K = 16 column blocks = 16 M raw input columns.  Its K order is
// free as long as both operands follow it; here lane half h of the B operand (the activations) holds the kept columns of
// blocks 8 h .. 8 h + 7 of the step, dword d of its 8 registers block 8 h + d, so that a lane's raw columns are one run of
// 8 M bytes of its token.  (Instruction: B lane (j, h) byte e is k = 32 (e / 16) + 16 h + e mod 16; A lane (i, h) byte e is
// kept value 16 h + e of row i, i.e. of 4-group 8 h + e / 2 in k order.  So A byte e belongs to block 8 (e / 8) + 4 h + (e / 2) mod 4.)
// Rows are grouped in blocks of 64 (two 32-row tiles) as in the fp16 copy, with NT = 1 column table per block or 2 (V = 32).
//   pa    int8 [R64][S][2 tiles][64 lanes][16]   A operand
//   pidx  u32  [R64][S][64 lanes][2 tiles]       2-bit position of value e at bits 2 e
//   pcol  u32  [R64][S][16 roles][NT]            raw column within the step (0 .. 16 M - 1) of the row that lane role
//                                                (h, r) = 8 h + r addresses in transposing read i, at bits 8 i: kept
//                                                column r mod 4 of block 8 h + 2 i + r / 4
//   psel  u32  [R64][S][NT][NSEL][2 h][4]        byte selectors: the 4 kept columns of a block as bytes of the dwords that
//                                                hold its M raw columns (8 bytes per selector; 12 selects zero), 4 bits
//                                                each: dword i has block 8 h + 2 i in the low halves of its bytes, the
//                                                next block in the high ones
inline int64_t i8_steps(const Dims& d) { return (d.B + 15) / 16; }
constexpr int i8_selectors(int M) {            // 8-byte pairs of dwords that a block of a lane's run can reach into
  int most = 0;
  for (int b = 0; b < 8; ++b) { const int end = ((M * b) & 3) + M; most = end > most ? end : most; }
  return (most + 7) / 8;
}
struct I8Layout { int64_t pidx_off, pcol_off, psel_off, total; };
constexpr int64_t kI8Slack = 16384;            // look-ahead loads may read (never use) this far past a section
inline I8Layout i8_layout(const Dims& d) {
  I8Layout l{0, 0, 0, 0};
  if (!has_packed(d.V, d.M)) return l;
  auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
  const int64_t rs = packed_row_blocks(d) * i8_steps(d), nt = packed_tables(d.V);
  l.pidx_off = up(rs * 2048);
  l.pcol_off = l.pidx_off + up(rs * 512);
  l.psel_off = l.pcol_off + up(rs * 64 * nt);
  l.total = l.psel_off + up(rs * 32 * nt * i8_selectors(d.M)) + kI8Slack;
  return l;
}
// Staged activations: an image per (tile of kTokTile tokens, K step), 16 M rows [raw column][token], padded to a multiple of 1 KiB.
// Rows lie 144 bytes apart, 16 more than they hold: a transposing read takes 16 bytes of each of its rows, and rows that differ
// modulo 16 then start in different banks (160 bytes, modulo 8: 1 to 4 % slower, and an eighth more to copy).
constexpr int kImagePitchI8 = kTokTile + 16;
inline int64_t i8_image_bytes(int M) { return ((int64_t)16 * M * kImagePitchI8 + 1023) / 1024 * 1024; }
int64_t staged_q_bytes(int64_t T, const Dims& d);

constexpr int64_t kI8MaxRowPitch = 1 << 24;    // of activations: the few-token kernel's offsets within 64 rows have 31 bits

// No sum may leave 32 bits, whatever the int8 values (-128 included)
inline bool i8_sums_fit(const Dims& d) { return 2 * d.B <= (0x7FFFFFFFll >> 14); }

// One product: y = ((float)sum * scale_w[o]) * scale_x[t] + bias[o], each operation rounded by itself, so that every kernel
// gives the same bits.
struct I8Epilogue {
  const float* scale_x; const float* scale_w; const _Float16* bias;
  void* Y; int64_t ldy; int y_dtype;
};
__device__ __forceinline__ float i8_result(int sum, float scale_w, float scale_x, bool has_bias, float bias) {
#pragma clang fp contract(off)
  const float y = ((float)sum * scale_w) * scale_x;
  return has_bias ? y + bias : y;
}
__device__ __forceinline__ unsigned short bf16_bits(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }
__device__ __forceinline__ void i8_store(const I8Epilogue& e, int64_t t, int64_t o, float v) {
  if (e.y_dtype == VNM_F16) ((_Float16*)e.Y)[t * e.ldy + o] = (_Float16)v;
  else if (e.y_dtype == VNM_BF16) ((__bf16*)e.Y)[t * e.ldy + o] = (__bf16)v;
  else ((float*)e.Y)[t * e.ldy + o] = v;
}

// Quantization of a row to int8 (vnm_quantize_x): factor and scale from the largest magnitude.
__device__ __forceinline__ void i8_factor(float top, float* factor, float* scale) {
  const bool bad = !(top < __builtin_inff());                       // an infinity, or a NaN
  const bool none = top < 0x1p-100f;                                // the quotient could leave fp32
  *factor = bad || none ? 0.f : (1.f / top) * 127.f;
  *scale = bad ? __builtin_nanf("") : none ? 0.f : top * (1.f / 127.f);
}
// x * factor rounded once to the integer: the addend's unit in the last place is 1 (fused, so the product is not rounded
// before); the low byte of the sum's bits is the int8.  (factor 0: x may be infinite, the result is set to zero by the caller.)
__device__ __forceinline__ unsigned i8_round(float x, float factor) {
  return __builtin_bit_cast(unsigned, __builtin_fmaf(x, factor, 12582912.f));
}
__device__ __forceinline__ unsigned i8_pack4(unsigned a, unsigned b, unsigned c, unsigned d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// The largest magnitude of a row, by its bits: orders like the value, and an infinity or NaN is above everything else.
__device__ __forceinline__ unsigned magnitude_bits(float x) { return __builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu; }

int launch_quantize_rows(const void* X, int64_t T, int64_t n, int64_t ldx, int x_dtype, void* Q, int64_t ldq, void* scale,
                         int64_t scale_rows, hipStream_t st);
int launch_pack_i8(const void* qvalues, const void* meta, const void* colidx, const Dims& d, void* packed, hipStream_t st);
int launch_spmm_i8_triple(const void* Q, int64_t T, int64_t ldq, const void* qvalues, const void* meta, const void* colidx,
                          const Dims& d, const I8Epilogue& e, hipStream_t st);
int launch_stage_q(const void* Q, int64_t T, int64_t ldq, const Dims& d, void* staged, hipStream_t st);
int launch_spmm_i8_staged(const void* staged, int64_t T, const void* packed, const Dims& d, const I8Epilogue& e, hipStream_t st);
int launch_spmm_i8_few(const void* Q, int64_t T, int64_t ldq, const void* packed, const Dims& d, const I8Epilogue& e, hipStream_t st);

}  // namespace vnm
