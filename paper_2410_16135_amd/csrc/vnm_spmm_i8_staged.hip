// Many tokens: the int8 product on the 2:4 sparse matrix cores (V_SMFMAC_I32_32X32X64_I8) with activations that are first
// re-laid as [raw column][token] (vnm_spmm_i8).
//
// Y^T = W' . Q^T, the compressed weight being the sparse A operand.  The activations of a K step (16 column blocks) and a tile
// of 128 tokens are one image of 16 M rows, which a workgroup streams through a ring of LDS buffers by asynchronous copies and
// all its row blocks share; the columns that a row block keeps are picked when a wave reads its B operand.
// ds_read_b64_tr_b8 takes 8 rows x 16 tokens -- rows chosen per lane from the packed column table, two column blocks' kept
// columns -- and hands every lane the 8 K-consecutive values of its token: LDS is read once per multiplied value, and no
// vector instruction touches it.  A wave owns a block of 64 rows x 128 tokens (128 accumulators); its weights come straight
// from the packed copy, 16 bytes per lane and tile.
//
// Per step a wave issues 8 matrix instructions of 32 cycles, 16 transposing reads (512 bytes each), 2 to 9 image copies and 4
// loads of weights; of a compute unit with 8 such waves that is 512 cycles of its matrix cores, 512 of LDS and 480 of the
// 64 bytes per cycle that reach it (M = 5): balanced, so the loop is written in assembly with explicit waits, in which
// younger requests stay in flight (compiled code drains all of them at each use).
//
// Measured: 4096 tokens x 4096 x 4096 at 64:2:5 40 us after 8.9 us of staging (3.4 P dense-equivalent operations per second), by time
// stamps in a copy of the kernel 0.7 in the prologue, 0.55 per step of the loop and 6.3 for writing Y; 4096 x 11008 85 and 20.  Counters
// of these two: the matrix cores work 33 and 39 % of the cycles in which the compute units do, LDS 37 and 40 (nearly half of that
// for bank conflicts), so neither bounds it alone.  At 256 tokens (64 workgroups of two wave groups) 19.5 and 5.1.
#include <type_traits>
#include "vnm_i8.h"
#include "vnm_i8_rules.h"

namespace vnm {

typedef int i4v __attribute__((ext_vector_type(4)));
typedef int i16v __attribute__((ext_vector_type(16)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef unsigned u2v __attribute__((ext_vector_type(2)));
typedef unsigned u4v __attribute__((ext_vector_type(4)));
#define VNM_LDS(T) __attribute__((address_space(3))) T*
#define VNM_GLB(T) __attribute__((address_space(1))) T*

// ---------------------------------------------------------------- staging
// One workgroup: one token tile x KC K steps.  Bound by memory: 4096 x 4096 in 8.9 us (3.8 TB/s), 4096 x 11008 in 20.3 (4.4).
// Rows are read 16 bytes per lane, parked in LDS as [token][column], and read back
// by transposing reads of 8 tokens x 16 columns, after which a lane holds 16 tokens of one column: an aligned piece of an image row.
template <int KC>
__global__ void __launch_bounds__(256)
stage_q_kernel(const unsigned char* __restrict__ Q, int64_t T, int64_t ldq, int in, int M, int64_t S, int64_t image,
               unsigned char* __restrict__ staged) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int64_t tile = blockIdx.y, s0 = (int64_t)blockIdx.x * KC, t0 = tile * kTokTile;
  const int pieces = KC * M, pitch = pieces * 16 + 16;             // (an odd number of 16-byte pieces)
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int NI = pieces / 2;                                       // 128 tokens x pieces over 256 threads
  const int dtok = 256 / pieces, dpc = 256 - dtok * pieces;
  const int64_t col0 = s0 * 16 * M;
  {
    u4v w[16];
    int tok = tid / pieces, pc = tid - tok * pieces;
    const int tok_first = tok, pc_first = pc;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < NI) {
        // a piece that begins inside the row is read whole (it is aligned); columns past the end meet weights that are zero
        const int64_t t = t0 + tok < T ? t0 + tok : T - 1, c = col0 + pc * 16;
        w[i] = *(const u4v*)(Q + t * ldq + (c < in ? c : 0));
        pc += dpc; tok += dtok;
        if (pc >= pieces) { pc -= pieces; ++tok; }
      }
    tok = tok_first; pc = pc_first;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < NI) {
        *(u4v*)(smem + tok * pitch + pc * 16) = w[i];
        pc += dpc; tok += dtok;
        if (pc >= pieces) { pc -= pieces; ++tok; }
      }
  }
  __syncthreads();
  const int g = lane >> 4, i16 = lane & 15, r = i16 >> 1;          // 16 lanes: 8 tokens x 16 columns per read
  for (int k = wave; k < 2 * pieces; k += 4) {
    const int cg = k >> 1, tg = (k & 1) * 4 + g;                   // 16 columns, 16 tokens
    const int64_t s = s0 + cg / M;
    if (s >= S) break;
    const unsigned char* p = smem + (tg * 16 + r) * pitch + cg * 16 + (i16 & 1) * 8;
    typedef int i2v __attribute__((ext_vector_type(2)));
    const i2v lo = __builtin_amdgcn_ds_read_tr8_b64_v2i32((VNM_LDS(i2v))p);
    const i2v hi = __builtin_amdgcn_ds_read_tr8_b64_v2i32((VNM_LDS(i2v))(p + 8 * pitch));
    *(i4v*)(staged + (tile * S + s) * image + ((cg % M) * 16 + i16) * kImagePitchI8 + tg * 16) = (i4v){lo[0], lo[1], hi[0], hi[1]};
  }
}

int64_t staged_q_bytes(int64_t T, const Dims& d) {
  // + 5 images that the product kernel's look-ahead copies may read (never use) past the last tile
  return ((T + kTokTile - 1) / kTokTile * i8_steps(d) + 5) * i8_image_bytes(d.M);
}

template <int KC>
static int launch_stage_q_cfg(const void* Q, int64_t T, int64_t ldq, const Dims& d, void* staged, hipStream_t st) {
  const int64_t tiles = (T + kTokTile - 1) / kTokTile, S = i8_steps(d), subs = (S + KC - 1) / KC;
  auto kern = stage_q_kernel<KC>;
  if (int rc = allow_big_lds((const void*)kern, "hipFuncSetAttribute(stage_q)")) return rc;
  for (int64_t tile = 0; tile < tiles; tile += kI8GridY) {         // grid.y limit
    const int64_t nt = tiles - tile < kI8GridY ? tiles - tile : kI8GridY, t0 = tile * kTokTile;
    hipLaunchKernelGGL(kern, dim3((unsigned)subs, (unsigned)nt), dim3(256), (size_t)kTokTile * (KC * d.M * 16 + 16), st,
                       (const unsigned char*)Q + t0 * ldq, T - t0, ldq, (int)d.in, d.M, S, i8_image_bytes(d.M),
                       (unsigned char*)staged + tile * S * i8_image_bytes(d.M));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error(e, "stage_q_kernel"); return VNM_ERR_HIP; }
  }
  return VNM_OK;
}
int launch_stage_q(const void* Q, int64_t T, int64_t ldq, const Dims& d, void* staged, hipStream_t st) {
  return d.M <= 5 ? launch_stage_q_cfg<4>(Q, T, ldq, d, staged, st) : launch_stage_q_cfg<2>(Q, T, ldq, d, staged, st);
}

// ---------------------------------------------------------------- product: the K loop
// Registers that the loops name: s[80:81] weights, s[82:83] positions, s[84:85] column table, s[86:87] image, s[88:89] copy source.
// One column table (V = 64, 128): v[150:153] B row addresses, v154 v155 scratch, v[156:187] B tiles 0..3, six weight sets {tile 0,
// tile 1, positions of both, column table} from v188, 22 registers for two of them.
// Two tables (V = 32): v152 v153 scratch, v[154:157] v[158:161] row addresses, slots v[162:193], five sets of 12 from v194.
// The compiler does not see the matrix instructions inside, so the loop ends with idle states of its own before compiled code
// reads the accumulators.
#define VNM_I8_DRAIN "s_nop 15\n s_nop 7\n"
#define VNM_I8_COPY(OFF)                                      \
  "s_add_u32 %[tci], %[woff], " #OFF "\n"                     \
  "s_min_u32 %[tci], %[tci], %[clamp]\n"                      \
  "s_add_u32 s88, s86, %[tci]\n"                              \
  "s_addc_u32 s89, s87, 0\n"                                  \
  "s_add_u32 m0, %[wr], %[tci]\n"                             \
  "s_nop 0\n"                                                 \
  "global_load_lds_dwordx4 %[voff16], s[88:89]\n"
// The copies per wave and image (1 KiB each, 4 or 8 waves), in two groups that are issued under two different matrix instructions
#define VNM_I8_C4_3A VNM_I8_COPY(0) VNM_I8_COPY(4096)
#define VNM_I8_C4_3B VNM_I8_COPY(8192)
#define VNM_I8_C4_4A VNM_I8_C4_3A
#define VNM_I8_C4_4B VNM_I8_C4_3B VNM_I8_COPY(12288)
#define VNM_I8_C4_5A VNM_I8_C4_3A VNM_I8_COPY(8192)
#define VNM_I8_C4_5B VNM_I8_COPY(12288) VNM_I8_COPY(16384)
#define VNM_I8_C4_6A VNM_I8_C4_5A
#define VNM_I8_C4_6B VNM_I8_C4_5B VNM_I8_COPY(20480)
#define VNM_I8_C4_7A VNM_I8_C4_5A VNM_I8_COPY(12288)
#define VNM_I8_C4_7B VNM_I8_COPY(16384) VNM_I8_COPY(20480) VNM_I8_COPY(24576)
#define VNM_I8_C4_8A VNM_I8_C4_7A
#define VNM_I8_C4_8B VNM_I8_C4_7B VNM_I8_COPY(28672)
#define VNM_I8_C4_9A VNM_I8_C4_7A VNM_I8_COPY(16384)
#define VNM_I8_C4_9B VNM_I8_COPY(20480) VNM_I8_COPY(24576) VNM_I8_COPY(28672) VNM_I8_COPY(32768)
#define VNM_I8_C8_2A VNM_I8_COPY(0)
#define VNM_I8_C8_2B VNM_I8_COPY(8192)
#define VNM_I8_C8_3A VNM_I8_COPY(0) VNM_I8_COPY(8192)
#define VNM_I8_C8_3B VNM_I8_COPY(16384)
#define VNM_I8_C8_4A VNM_I8_C8_3A
#define VNM_I8_C8_4B VNM_I8_C8_3B VNM_I8_COPY(24576)
#define VNM_I8_C8_5A VNM_I8_C8_3A VNM_I8_COPY(16384)
#define VNM_I8_C8_5B VNM_I8_COPY(24576) VNM_I8_COPY(32768)

#define VNM_I8_READ2(OFF, R0, A0, R1, A1)                                     \
  "ds_read_b64_tr_b8 v[" #R0 ":" #R0 "+1], v" #A0 " offset:" #OFF "\n"        \
  "ds_read_b64_tr_b8 v[" #R1 ":" #R1 "+1], v" #A1 " offset:" #OFF "\n"
#define VNM_I8_READ4(OFF, R0, R1, R2, R3) VNM_I8_READ2(OFF, R0, 150, R1, 151) VNM_I8_READ2(OFF, R2, 152, R3, 153)
#define VNM_I8_MFMA(ACC, W, B, IDX) "v_smfmac_i32_32x32x64_i8 %[" ACC "], v[" W "], v[" B "], v" IDX "\n"
#define VNM_I8_LOAD_A(W0, W1, IDX, PC, PCW, PCB)                               \
  "global_load_dwordx4 v[" W0 "], %[voff16], s[80:81]\n"                       \
  "global_load_dwordx4 v[" W1 "], %[voff16], s[80:81] offset:1024\n"           \
  "global_load_dwordx2 v[" IDX "], %[voffi], s[82:83]\n"                       \
  "global_load_dword" PCW " v" PC ", %[voffp], s[84:85]\n"                     \
  VNM_I8_ADVANCE(PCB)
#define VNM_I8_ADVANCE(PCB)                                                    \
  "s_add_u32 s80, s80, 2048\n s_addc_u32 s81, s81, 0\n"                        \
  "s_add_u32 s82, s82, 512\n s_addc_u32 s83, s83, 0\n"                         \
  "s_add_u32 s84, s84, " PCB "\n s_addc_u32 s85, s85, 0\n"
// row addresses from a column table register (4 x 8-bit rows of the image) and the ring slot
#define VNM_I8_ADDR4(PC, BASE, TMP, A0, A1, A2, A3)                            \
  "v_and_b32 v" #TMP ", 0xff, v" PC "\n"                                       \
  "v_mad_u32_u24 v" #A0 ", v" #TMP ", %[pitch], v" #BASE "\n"                  \
  "v_bfe_u32 v" #TMP ", v" PC ", 8, 8\n"                                       \
  "v_mad_u32_u24 v" #A1 ", v" #TMP ", %[pitch], v" #BASE "\n"                  \
  "v_bfe_u32 v" #TMP ", v" PC ", 16, 8\n"                                      \
  "v_mad_u32_u24 v" #A2 ", v" #TMP ", %[pitch], v" #BASE "\n"                  \
  "v_lshrrev_b32 v" #TMP ", 24, v" PC "\n"                                     \
  "v_mad_u32_u24 v" #A3 ", v" #TMP ", %[pitch], v" #BASE "\n"
#define VNM_I8_ADDR(PC) "v_add_u32 v154, %[rd], %[vtok]\n" VNM_I8_ADDR4(PC, 154, 155, 150, 151, 152, 153)
#define VNM_I8_W4 "s_waitcnt lgkmcnt(4)\n s_nop 0\n"
#define VNM_I8_NEXT_RD "s_add_u32 %[rd], %[rd], %[img]\n s_cmp_eq_u32 %[rd], %[lend]\n s_cselect_b32 %[rd], %[lbeg], %[rd]\n"
#define VNM_I8_NEXT_WR "s_add_u32 %[wr], %[wr], %[img]\n s_cmp_eq_u32 %[wr], %[lend]\n s_cselect_b32 %[wr], %[lbeg], %[wr]\n" \
                       "s_add_u32 s86, s86, %[img]\n s_addc_u32 s87, s87, 0\n"
#define VNM_I8_LAST "s_sub_u32 %[n], %[n], 1\n s_cmp_eq_u32 %[n], 0\n s_cbranch_scc1 9f\n"

// One K step.  CW0 CW1 CI0 CI1: weights and positions of both tiles; NPC: column table of the next step; LW0 LW1 LIDX LPC: the
// set that receives the weights of a later step.  B tiles are requested two tiles (four matrix instructions) ahead of their
// use, across the step boundary; at each use the four reads of the following tile may still be in flight.
//   tiles 0, 1 multiplied | under them: weights requested, tiles 2, 3 of this step requested
//   wait for the next step's weights and image, barrier: every wave has left the previous step, its ring slot is free
//   tiles 2, 3 multiplied | under them: next step's row addresses, copies of the image NBUF - 1 ahead, next step's tiles 0, 1
// Between the two waits at the barrier and the next matrix instruction stands nothing else: the barrier brings the two waves
// of a SIMD to the same point, and what both issued there would leave the matrix cores idle.
#define VNM_I8_STEP(CW0, CW1, CI0, CI1, NPC, LW0, LW1, LIDX, LPC, COPY_A, COPY_B)               \
      VNM_I8_W4 VNM_I8_MFMA("a00", CW0, "156:163", CI0)                                             \
      "global_load_dwordx4 v[" LW0 "], %[voff16], s[80:81]\n" VNM_I8_READ2(64, 172, 150, 174, 151)  \
      VNM_I8_MFMA("a10", CW1, "156:163", CI1)                                                       \
      "global_load_dwordx4 v[" LW1 "], %[voff16], s[80:81] offset:1024\n" VNM_I8_READ2(64, 176, 152, 178, 153) \
      VNM_I8_W4 VNM_I8_MFMA("a01", CW0, "164:171", CI0)                                             \
      "global_load_dwordx2 v[" LIDX "], %[voffi], s[82:83]\n" VNM_I8_READ2(96, 180, 150, 182, 151)  \
      VNM_I8_NEXT_RD                                                                                \
      VNM_I8_MFMA("a11", CW1, "164:171", CI1)                                                       \
      "global_load_dword v" LPC ", %[voffp], s[84:85]\n" VNM_I8_READ2(96, 184, 152, 186, 153)       \
      VNM_I8_ADVANCE("64")                                                                          \
      "s_waitcnt vmcnt(%[vm])\n s_barrier\n"                                                       \
      VNM_I8_W4 VNM_I8_MFMA("a02", CW0, "172:179", CI0)                                             \
      VNM_I8_ADDR(NPC) VNM_I8_READ2(0, 156, 150, 158, 151) COPY_A                                   \
      VNM_I8_MFMA("a12", CW1, "172:179", CI1)                                                       \
      VNM_I8_READ2(0, 160, 152, 162, 153) COPY_B VNM_I8_NEXT_WR                                     \
      VNM_I8_W4 VNM_I8_MFMA("a03", CW0, "180:187", CI0)                                             \
      VNM_I8_READ2(32, 164, 150, 166, 151)                                                          \
      VNM_I8_MFMA("a13", CW1, "180:187", CI1)                                                       \
      VNM_I8_READ2(32, 168, 152, 170, 153) VNM_I8_LAST

// Two column tables: every matrix instruction has a B operand of its own, kept in a ring of four slots; operand i + 3 is
// requested after instruction i into the slot that i - 1 has used, so at each use 8 reads may still be in flight.
#define VNM_I8_D_READ4(OFF, X, A0)                                                                  \
  "ds_read_b64_tr_b8 v[" #X ":" #X "+1], v[" #A0 "] offset:" #OFF "\n"                              \
  "ds_read_b64_tr_b8 v[" #X "+2:" #X "+3], v[" #A0 "+1] offset:" #OFF "\n"                          \
  "ds_read_b64_tr_b8 v[" #X "+4:" #X "+5], v[" #A0 "+2] offset:" #OFF "\n"                          \
  "ds_read_b64_tr_b8 v[" #X "+6:" #X "+7], v[" #A0 "+3] offset:" #OFF "\n"
#define VNM_I8_D_ADDR(PC0, PC1) "v_add_u32 v152, %[rd], %[vtok]\n"                                  \
  VNM_I8_ADDR4(PC0, 152, 153, 154, 155, 156, 157) VNM_I8_ADDR4(PC1, 152, 153, 158, 159, 160, 161)
#define VNM_I8_W8 "s_waitcnt lgkmcnt(8)\n s_nop 0\n"
#define VNM_I8_D_STEP(CW0, CW1, CI0, CI1, NPC0, NPC1, LW0, LW1, LIDX, LPC, COPY_A, COPY_B)      \
      VNM_I8_W8 VNM_I8_MFMA("a00", CW0, "162:169", CI0)                                             \
      "global_load_dwordx4 v[" LW0 "], %[voff16], s[80:81]\n" VNM_I8_D_READ4(32, 186, 158)          \
      VNM_I8_W8 VNM_I8_MFMA("a10", CW1, "170:177", CI1)                                             \
      "global_load_dwordx4 v[" LW1 "], %[voff16], s[80:81] offset:1024\n" VNM_I8_D_READ4(64, 162, 154) \
      VNM_I8_W8 VNM_I8_MFMA("a01", CW0, "178:185", CI0)                                             \
      "global_load_dwordx2 v[" LIDX "], %[voffi], s[82:83]\n" VNM_I8_D_READ4(64, 170, 158)          \
      VNM_I8_W8 VNM_I8_MFMA("a11", CW1, "186:193", CI1)                                             \
      "global_load_dwordx2 v[" LPC "], %[voffp], s[84:85]\n" VNM_I8_D_READ4(96, 178, 154)           \
      VNM_I8_ADVANCE("128") VNM_I8_NEXT_RD                                                          \
      "s_waitcnt vmcnt(%[vm])\n s_barrier\n"                                                       \
      VNM_I8_W8 VNM_I8_MFMA("a02", CW0, "162:169", CI0)                                             \
      VNM_I8_D_READ4(96, 186, 158) COPY_A VNM_I8_D_ADDR(NPC0, NPC1)                                 \
      VNM_I8_W8 VNM_I8_MFMA("a12", CW1, "170:177", CI1)                                             \
      VNM_I8_D_READ4(0, 162, 154) COPY_B VNM_I8_NEXT_WR                                             \
      VNM_I8_W8 VNM_I8_MFMA("a03", CW0, "178:185", CI0)                                             \
      VNM_I8_D_READ4(0, 170, 158)                                                                   \
      VNM_I8_W8 VNM_I8_MFMA("a13", CW1, "186:193", CI1)                                             \
      VNM_I8_D_READ4(32, 178, 154) VNM_I8_LAST

#define VNM_I8_LOOP(FIRST_LOADS, FIRST_READS, STEPS)                                                \
  asm volatile(                                                                                     \
      "s_mov_b32 s80, %[pa_lo]\n s_mov_b32 s81, %[pa_hi]\n"                                         \
      "s_mov_b32 s82, %[pi_lo]\n s_mov_b32 s83, %[pi_hi]\n"                                         \
      "s_mov_b32 s84, %[pc_lo]\n s_mov_b32 s85, %[pc_hi]\n"                                         \
      "s_mov_b32 s86, %[xs_lo]\n s_mov_b32 s87, %[xs_hi]\n"                                         \
      FIRST_LOADS                                                                                   \
      "s_waitcnt vmcnt(0) lgkmcnt(0)\n s_barrier\n"                                                 \
      FIRST_READS                                                                                   \
      "1:\n" STEPS "s_branch 1b\n"                                                                  \
      "9:\n"                                                                                        \
      "s_waitcnt vmcnt(0) lgkmcnt(0)\n s_barrier\n" VNM_I8_DRAIN                                    \
      : [a00] "+v"(acc[0][0]), [a01] "+v"(acc[0][1]), [a02] "+v"(acc[0][2]), [a03] "+v"(acc[0][3]), \
        [a10] "+v"(acc[1][0]), [a11] "+v"(acc[1][1]), [a12] "+v"(acc[1][2]), [a13] "+v"(acc[1][3]), \
        [rd] "+&s"(l_rd), [wr] "+&s"(l_wr), [n] "+&s"(l_n), [tci] "=&s"(l_tci)                      \
      : [pa_lo] "s"(l_pa_lo), [pa_hi] "s"(l_pa_hi), [pi_lo] "s"(l_pi_lo), [pi_hi] "s"(l_pi_hi),     \
        [pc_lo] "s"(l_pc_lo), [pc_hi] "s"(l_pc_hi), [xs_lo] "s"(l_xs_lo), [xs_hi] "s"(l_xs_hi),     \
        [voff16] "v"(l_voff16), [voffi] "v"(l_voffi), [voffp] "v"(l_voffp), [vtok] "v"(l_vtok),     \
        [woff] "s"(l_woff), [clamp] "s"(l_clamp), [pitch] "s"(l_pitch), [img] "s"(l_img),           \
        [lbeg] "s"(l_lbeg), [lend] "s"(l_lend), [vm] "n"(VM)                                        \
      : "memory", "scc", "m0", VNM_I8_CLOBBERS)
#define VNM_I8_CLOBBERS \
        "v150", "v151", "v152", "v153", "v154", "v155", "v156", "v157", "v158", "v159", "v160", "v161", "v162", \
        "v163", "v164", "v165", "v166", "v167", "v168", "v169", "v170", "v171", "v172", "v173", "v174", "v175", \
        "v176", "v177", "v178", "v179", "v180", "v181", "v182", "v183", "v184", "v185", "v186", "v187", "v188", \
        "v189", "v190", "v191", "v192", "v193", "v194", "v195", "v196", "v197", "v198", "v199", "v200", "v201", \
        "v202", "v203", "v204", "v205", "v206", "v207", "v208", "v209", "v210", "v211", "v212", "v213", "v214", \
        "v215", "v216", "v217", "v218", "v219", "v220", "v221", "v222", "v223", "v224", "v225", "v226", "v227", \
        "v228", "v229", "v230", "v231", "v232", "v233", "v234", "v235", "v236", "v237", "v238", "v239", "v240", \
        "v241", "v242", "v243", "v244", "v245", "v246", "v247", "v248", "v249", "v250", "v251", "v252", "v253", \
        "v254", "v255", "s80", "s81", "s82", "s83", "s84", "s85", "s86", "s87", "s88", "s89"
// (sets in turn: six that are loaded five steps ahead, or five that are loaded four)
#define VNM_I8_LOOP_1(CA, CB) VNM_I8_LOOP( \
      VNM_I8_LOAD_A("188:191", "192:195", "196:197", "198", "", "64") \
      VNM_I8_LOAD_A("200:203", "204:207", "208:209", "199", "", "64") \
      VNM_I8_LOAD_A("210:213", "214:217", "218:219", "220", "", "64") \
      VNM_I8_LOAD_A("222:225", "226:229", "230:231", "221", "", "64") \
      VNM_I8_LOAD_A("232:235", "236:239", "240:241", "242", "", "64"), \
      VNM_I8_ADDR("198") VNM_I8_READ4(0, 156, 158, 160, 162) VNM_I8_READ4(32, 164, 166, 168, 170), \
      VNM_I8_STEP("188:191", "192:195", "196", "197", "199", "244:247", "248:251", "252:253", "243", CA, CB) \
      VNM_I8_STEP("200:203", "204:207", "208", "209", "220", "188:191", "192:195", "196:197", "198", CA, CB) \
      VNM_I8_STEP("210:213", "214:217", "218", "219", "221", "200:203", "204:207", "208:209", "199", CA, CB) \
      VNM_I8_STEP("222:225", "226:229", "230", "231", "242", "210:213", "214:217", "218:219", "220", CA, CB) \
      VNM_I8_STEP("232:235", "236:239", "240", "241", "243", "222:225", "226:229", "230:231", "221", CA, CB) \
      VNM_I8_STEP("244:247", "248:251", "252", "253", "198", "232:235", "236:239", "240:241", "242", CA, CB))
#define VNM_I8_LOOP_2(CA, CB) VNM_I8_LOOP( \
      VNM_I8_LOAD_A("194:197", "198:201", "202:203", "[204:205]", "x2", "128") \
      VNM_I8_LOAD_A("206:209", "210:213", "214:215", "[216:217]", "x2", "128") \
      VNM_I8_LOAD_A("218:221", "222:225", "226:227", "[228:229]", "x2", "128") \
      VNM_I8_LOAD_A("230:233", "234:237", "238:239", "[240:241]", "x2", "128"), \
      VNM_I8_D_ADDR("204", "205") VNM_I8_D_READ4(0, 162, 154) VNM_I8_D_READ4(0, 170, 158) VNM_I8_D_READ4(32, 178, 154), \
      VNM_I8_D_STEP("194:197", "198:201", "202", "203", "216", "217", "242:245", "246:249", "250:251", "252:253", CA, CB) \
      VNM_I8_D_STEP("206:209", "210:213", "214", "215", "228", "229", "194:197", "198:201", "202:203", "204:205", CA, CB) \
      VNM_I8_D_STEP("218:221", "222:225", "226", "227", "240", "241", "206:209", "210:213", "214:215", "216:217", CA, CB) \
      VNM_I8_D_STEP("230:233", "234:237", "238", "239", "252", "253", "218:221", "222:225", "226:227", "228:229", CA, CB) \
      VNM_I8_D_STEP("242:245", "246:249", "250", "251", "204", "205", "230:233", "234:237", "238:239", "240:241", CA, CB))

struct I8StagedArgs {
  const unsigned char* staged; int64_t T;
  const unsigned char* pa; const unsigned char* pidx; const unsigned char* pcol;
  int64_t out, R, S;
  int image;                       // bytes, a multiple of 1024
  int run;                         // results that a lane stores at once: 16 bytes where Y's rows are aligned to them
  I8Epilogue e;
};

// WR: row blocks (waves) per K group.  KG: groups that share rows and tokens and cut the K steps in halves, each with a ring of
// images of its own; at the end each takes the sums of its half of the tokens over through LDS.  NCW: image copies per wave.
// NBUF: images in the ring.  DUAL: two column tables per row block.
template <int WR, int KG, int NCW, int NBUF, bool DUAL>
__global__ void __launch_bounds__(64 * WR * KG)
spmm_i8_staged_kernel(const I8StagedArgs a) {
  constexpr int AT = 2, BT = 4, NW = WR, P = kImagePitchI8;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_id = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = KG == 1 ? 0 : wave_id / WR, wave = KG == 1 ? wave_id : wave_id % WR;
  const int64_t r = (int64_t)blockIdx.y * WR + wave;
  const bool r_valid = r < a.R;
  const int64_t rr = r_valid ? r : a.R - 1;      // waves past the last row block compute it again and store nothing
  const int64_t t0 = (int64_t)blockIdx.x * kTokTile;
  const int64_t SG = (a.S + KG - 1) / KG;        // steps of the first group
  const int64_t s0 = kg * SG, S = KG == 1 || kg == 0 ? SG : a.S - SG;
  const int64_t rs0 = rr * a.S + s0;
  const int img = a.image, n_ci = img / 1024;
  unsigned char* const ring = smem + kg * NBUF * img;

  i16v acc[AT][BT];
#pragma unroll
  for (int i = 0; i < AT; ++i)
#pragma unroll
    for (int j = 0; j < BT; ++j) acc[i][j] = (i16v)0;

  // Scales and bias of this wave's channels and tokens, one or two per lane: requested here, so that nothing is waited for
  // when the loop has ended (clamped: what lies beyond is not stored)
  constexpr int TE = kTokTile / KG;                      // tokens this wave has the results of
  const int64_t t_wave = t0 + kg * TE;
  auto clamped = [](int64_t i, int64_t n) { return i < n ? i : n - 1; };
  const float sw_lane = a.e.scale_w[clamped(rr * 64 + lane, a.out)];
  const float bias_lane = a.e.bias ? (float)a.e.bias[clamped(rr * 64 + lane, a.out)] : 0.f;
  float sx_lane[TE / 64];
#pragma unroll
  for (int k = 0; k < TE / 64; ++k) sx_lane[k] = a.e.scale_x[clamped(t_wave + k * 64 + lane, a.T)];

  const unsigned char* xs_tile = a.staged + ((int64_t)blockIdx.x * a.S + s0) * img;
  // a wave's share of an image; pieces past the image are its last one again, so that every wave issues the same number
  auto copy_image = [&](int64_t s, int slot) {
    const unsigned char* src = xs_tile + s * img + lane * 16;
    for (int k = 0; k < NCW; ++k) {
      int ci = wave + k * NW;
      ci = ci < n_ci ? ci : n_ci - 1;
      __builtin_amdgcn_global_load_lds((VNM_GLB(void))(src + ci * 1024), (VNM_LDS(void))(ring + slot * img + ci * 1024), 16, 0, 0);
    }
  };
  for (int k = 0; k < NBUF - 1 && k < S; ++k) copy_image(k, k);
  {
    // Every step requests the image NBUF - 1 steps ahead and the weights up to five ahead without looking at S: near the end these
    // are the next tile's and row block's, or the slack behind the staged buffer (5 images) and the packed copy; never used.
    auto lo = [](uint64_t p) { return (unsigned)__builtin_amdgcn_readfirstlane((unsigned)p); };
    auto hi = [](uint64_t p) { return (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(p >> 32)); };
    const uint64_t pa_p = (uint64_t)(a.pa + rs0 * 2048), pi_p = (uint64_t)(a.pidx + rs0 * 512);
    const uint64_t pc_p = (uint64_t)(a.pcol + rs0 * (DUAL ? 128 : 64)), xs_p = (uint64_t)(xs_tile + (int64_t)(NBUF - 1) * img);
    const unsigned l_pa_lo = lo(pa_p), l_pa_hi = hi(pa_p), l_pi_lo = lo(pi_p), l_pi_hi = hi(pi_p);
    const unsigned l_pc_lo = lo(pc_p), l_pc_hi = hi(pc_p), l_xs_lo = lo(xs_p), l_xs_hi = hi(xs_p);
    const int role = (lane >> 5) * 8 + ((lane & 15) >> 1);         // the row this lane addresses in a transposing read
    const unsigned l_voff16 = lane * 16, l_voffi = lane * 8, l_voffp = role * (DUAL ? 8 : 4);
    const unsigned l_vtok = ((lane >> 4) & 1) * 16 + (lane & 1) * 8;
    const unsigned l_woff = wave * 1024, l_clamp = (n_ci - 1) * 1024, l_pitch = P, l_img = img;
    const unsigned l_lbeg = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(VNM_LDS(unsigned char))ring), l_lend = l_lbeg + NBUF * img;
    unsigned l_rd = l_lbeg, l_wr = l_lbeg + (NBUF - 1) * img, l_tci, l_n = (unsigned)S;
    // What may stay in flight at a step's wait, when the next step's image (requested NBUF - 1 steps before it) and weights (AHEAD
    // steps before it) must have landed: requests return in order, a step makes 4 for weights, then NCW copies.
    constexpr int AHEAD = DUAL ? 4 : 5;
    constexpr int AFTER_IMAGE = (NBUF - 3) * (4 + NCW) + 4, AFTER_WEIGHTS = (AHEAD - 2) * (4 + NCW) + NCW + 4;
    constexpr int VM = AFTER_IMAGE < AFTER_WEIGHTS ? AFTER_IMAGE : AFTER_WEIGHTS;
    static_assert(NBUF >= 3 && VM < 64, "counted in 6 bits");
#define VNM_I8_GO(W, N)                                                                             \
    if constexpr (NW == W && NCW == N) {                                                            \
      if constexpr (DUAL) VNM_I8_LOOP_2(VNM_I8_C##W##_##N##A, VNM_I8_C##W##_##N##B);                \
      else VNM_I8_LOOP_1(VNM_I8_C##W##_##N##A, VNM_I8_C##W##_##N##B);                               \
    }
    VNM_I8_GO(4, 3) VNM_I8_GO(4, 4) VNM_I8_GO(4, 5) VNM_I8_GO(4, 6) VNM_I8_GO(4, 7) VNM_I8_GO(4, 8) VNM_I8_GO(4, 9)
    VNM_I8_GO(8, 2) VNM_I8_GO(8, 3) VNM_I8_GO(8, 4) VNM_I8_GO(8, 5)
#undef VNM_I8_GO
  }

  constexpr int BE = BT / KG;                            // its token tiles
  // What is derived from the lane is computed again: kept from before the loop it would leave no room beside the accumulators.
  int le = lane;
  asm volatile("" : "+v"(le));
  constexpr int EP = 64 * 2 + 8, EPB = TE * EP + 1024;   // bytes of LDS per token, and per wave
  unsigned char* ep = smem + (size_t)wave_id * EPB;
  if constexpr (KG == 2) {
    // A step has one barrier, so a group with a step less has one to add; what follows may not pass it, as the other group
    // still reads its ring.
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    if (S < SG) __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    constexpr int XB = AT * BE * 16 * 64 * 4;
    unsigned char* mine = smem + (size_t)wave_id * XB;
    unsigned char* theirs = smem + (size_t)(wave_id ^ WR) * XB;
#pragma unroll
    for (int i = 0; i < AT; ++i)
#pragma unroll
      for (int j = 0; j < BE; ++j) {
        const i16v send = kg ? acc[i][j] : acc[i][j + BE];
        acc[i][j] = kg ? acc[i][j + BE] : acc[i][j];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          *(i4v*)(mine + (((i * BE + j) * 4 + k) * 64 + le) * 16) = (i4v){send[4 * k], send[4 * k + 1], send[4 * k + 2], send[4 * k + 3]};
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < AT; ++i)
#pragma unroll
      for (int j = 0; j < BE; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const i4v v = *(const i4v*)(theirs + (((i * BE + j) * 4 + k) * 64 + le) * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][4 * k + e] += v[e];
        }
    ep = theirs;                                         // nobody else reads it
    static_assert(EPB <= XB, "the turned-around tile fits there");
  }
  if (!r_valid) return;
  const int tokl = le & 31, hB = le >> 5;
  float* const scales = (float*)(ep + TE * EP);          // [64 channels][64 biases][TE tokens], this wave's own
  scales[le] = sw_lane;
  scales[64 + le] = bias_lane;
#pragma unroll
  for (int k = 0; k < TE / 64; ++k) scales[128 + k * 64 + le] = sx_lane[k];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  float sx[BE];
#pragma unroll
  for (int j = 0; j < BE; ++j) sx[j] = scales[128 + j * 32 + tokl];
  // (type and bias are decided once: decided at each of the 128 values of a lane they cost a third of this part's time)
  auto each = [&](auto has_bias, int j0, int j1, auto&& take) {
#pragma unroll
    for (int i = 0; i < AT; ++i)
#pragma unroll
      for (int jq = 0; jq < 4; ++jq) {
        const int row = i * 32 + 8 * jq + 4 * hB;        // of the lane's four channels
        const f4v sw = *(const f4v*)(scales + row), bias = *(const f4v*)(scales + 64 + row);
#pragma unroll
        for (int j = j0; j < j1; ++j) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = i8_result(acc[i][j][4 * jq + e], sw[e], sx[j], decltype(has_bias)::value, bias[e]);
          take(row, j, v);
        }
      }
  };
  auto either = [&](int j0, int j1, auto&& take) {
    if (a.e.bias) each(std::true_type{}, j0, j1, take); else each(std::false_type{}, j0, j1, take);
  };
  auto turned = [&] {                                    // this wave's own region of LDS: in order, only the compiler is held
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  // Results are turned around in LDS, from 4 channels of a token per lane to whole runs of a token's row, whatever their
  // alignment: stored from where they are, fp32 and unaligned rows took as long as the rest of the call (2122 tokens, 3496 x 208,
  // M = 4, fp32 40.1 us, now 17.7; 1844, 5824 x 3904 86.9 and 43.2; 389, 10654 x 1584, fp16 33.9 and 22.2).  Y is not read again
  // here: non-temporal stores keep it from displacing what others stream through L2.
  // fp32: 32 tokens at a time, PER channels per lane
  auto rows32 = [&](auto per_lane) {
    constexpr int PER = decltype(per_lane)::value, P32 = 64 * 4 + 16;
    static_assert(32 * P32 <= TE * EP, "a tile of fp32 results");
    const int ch = le % (64 / PER) * PER, tl = le / (64 / PER);
#pragma unroll
    for (int j = 0; j < BE; ++j) {
      either(j, j + 1, [&](int row, int, const float (&v)[4]) { *(f4v*)(ep + tokl * P32 + row * 4) = (f4v){v[0], v[1], v[2], v[3]}; });
      turned();
#pragma unroll 4
      for (int it = 0; it < 32 / PER; ++it) {
        const int tk = it * PER + tl;
        const int64_t t = t_wave + j * 32 + tk, o = r * 64 + ch;
        float* const y = (float*)a.e.Y + t * a.e.ldy + o;
        const float* const from = (const float*)(ep + tk * P32) + ch;
        if (t < a.T && o + PER <= a.out) {
          if constexpr (PER == 4) __builtin_nontemporal_store(*(const f4v*)from, (f4v*)y);
          else __builtin_nontemporal_store(*from, y);
        } else if (PER > 1 && t < a.T)
          for (int e = 0; e < PER; ++e) if (o + e < a.out) y[e] = from[e];
      }
      turned();
    }
  };
  if (a.e.y_dtype == VNM_F32) {
    if (a.run == 4) rows32(std::integral_constant<int, 4>{}); else rows32(std::integral_constant<int, 1>{});
    return;
  }
  auto turn = [&](int row, int j, u2v pk) { *(u2v*)(ep + (size_t)(j * 32 + tokl) * EP + row * 2) = pk; };
  if (a.e.y_dtype == VNM_F16)
    either(0, BE, [&](int row, int j, const float (&v)[4]) {
      typedef _Float16 h4 __attribute__((ext_vector_type(4)));
      turn(row, j, __builtin_bit_cast(u2v, (h4){(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]}));
    });
  else
    either(0, BE, [&](int row, int j, const float (&v)[4]) {
      turn(row, j, (u2v){bf16_bits(v[0]) | (unsigned)bf16_bits(v[1]) << 16, bf16_bits(v[2]) | (unsigned)bf16_bits(v[3]) << 16});
    });
  turned();
  auto rows16 = [&](auto per_lane) {
    constexpr int PER = decltype(per_lane)::value;
    const int ch = le % (64 / PER) * PER, tl = le / (64 / PER);
#pragma unroll 8
    for (int it = 0; it < TE / PER; ++it) {
      const int tk = it * PER + tl;
      const int64_t t = t_wave + tk, o = r * 64 + ch;
      unsigned short* const y = (unsigned short*)a.e.Y + t * a.e.ldy + o;
      const unsigned short* const from = (const unsigned short*)(ep + (size_t)tk * EP) + ch;
      if (t < a.T && o + PER <= a.out) {
        if constexpr (PER == 8) {
          const u2v v0 = *(const u2v*)from, v1 = *(const u2v*)(from + 4);
          __builtin_nontemporal_store((u4v){v0.x, v0.y, v1.x, v1.y}, (u4v*)y);
        } else if constexpr (PER == 2) __builtin_nontemporal_store(*(const unsigned*)from, (unsigned*)y);
        else __builtin_nontemporal_store(*from, y);
      } else if (PER > 1 && t < a.T)
        for (int e = 0; e < PER; ++e) if (o + e < a.out) y[e] = from[e];
    }
  };
  if (a.run == 8) rows16(std::integral_constant<int, 8>{});
  else if (a.run == 2) rows16(std::integral_constant<int, 2>{});
  else rows16(std::integral_constant<int, 1>{});
}

template <int WR, int KG, int NCW, int NBUF, bool DUAL>
static int launch_staged_cfg(const I8StagedArgs& a, hipStream_t st) {
  size_t lds = (size_t)KG * NBUF * a.image;
  const size_t ep = KG == 1 ? (size_t)WR * (kTokTile * (64 * 2 + 8) + 1024) : (size_t)2 * WR * 2 * 2 * 16 * 64 * 4;
  if (ep > lds) lds = ep;
  auto kern = spmm_i8_staged_kernel<WR, KG, NCW, NBUF, DUAL>;
  if (int rc = allow_big_lds((const void*)kern, "hipFuncSetAttribute(spmm_i8_staged)")) return rc;
  const int64_t tiles = (a.T + kTokTile - 1) / kTokTile, groups = (a.R + WR - 1) / WR;
  hipLaunchKernelGGL(kern, dim3((unsigned)tiles, (unsigned)groups), dim3(64 * WR * KG), lds, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_hip_error(e, "spmm_i8_staged_kernel"); return VNM_ERR_HIP; }
  return VNM_OK;
}
// The longest ring of images that LDS holds, 6 at most, by the columns per block
constexpr int i8_ring(int M, int rings) {
  const int kib = (16 * M * kImagePitchI8 + 1023) / 1024, n = 160 / (kib * rings);
  return n > 6 ? 6 : n;
}
constexpr int i8_copies(int M, int waves) { return ((16 * M * kImagePitchI8 + 1023) / 1024 + waves - 1) / waves; }
// wide: 8 row blocks per workgroup; otherwise 4, in two groups of waves on halves of K where LDS holds two rings and there are
// steps for both
template <bool DUAL, int M>
static int launch_staged_m(const I8StagedArgs& a, bool wide, hipStream_t st) {
  if (wide) return launch_staged_cfg<8, 1, i8_copies(M, 8), i8_ring(M, 1), DUAL>(a, st);
  if constexpr (i8_ring(M, 2) >= 3)
    if (a.S >= 8) return launch_staged_cfg<4, 2, i8_copies(M, 4), i8_ring(M, 2), DUAL>(a, st);
  return launch_staged_cfg<4, 1, i8_copies(M, 4), i8_ring(M, 1), DUAL>(a, st);
}
template <bool DUAL>
static int launch_staged(const I8StagedArgs& a, int M, bool wide, hipStream_t st) {
  switch (M) {
    case 4: return launch_staged_m<DUAL, 4>(a, wide, st);
    case 5: return launch_staged_m<DUAL, 5>(a, wide, st);
    case 6: return launch_staged_m<DUAL, 6>(a, wide, st);
    case 7: return launch_staged_m<DUAL, 7>(a, wide, st);
    case 8: return launch_staged_m<DUAL, 8>(a, wide, st);
    case 9: return launch_staged_m<DUAL, 9>(a, wide, st);
    case 10: return launch_staged_m<DUAL, 10>(a, wide, st);
    case 11: return launch_staged_m<DUAL, 11>(a, wide, st);
    case 12: return launch_staged_m<DUAL, 12>(a, wide, st);
    case 13: return launch_staged_m<DUAL, 13>(a, wide, st);
    case 14: return launch_staged_m<DUAL, 14>(a, wide, st);
    case 15: return launch_staged_m<DUAL, 15>(a, wide, st);
    case 16: return launch_staged_m<DUAL, 16>(a, wide, st);
  }
  return VNM_ERR_UNSUPPORTED;
}

int launch_spmm_i8_staged(const void* staged, int64_t T, const void* packed, const Dims& d, const I8Epilogue& e, hipStream_t st) {
  const I8Layout l = i8_layout(d);
  const unsigned char* p = (const unsigned char*)packed;
  I8StagedArgs a{(const unsigned char*)staged, T, p, p + l.pidx_off, p + l.pcol_off, d.out, packed_row_blocks(d), i8_steps(d),
                 (int)i8_image_bytes(d.M), 1, e};
  auto aligned = [&](int elements, int bytes) { return e.ldy % elements == 0 && ((uintptr_t)e.Y & (bytes - 1)) == 0; };
  if (e.y_dtype == VNM_F32) a.run = aligned(4, 16) ? 4 : 1;
  else a.run = aligned(8, 16) ? 8 : aligned(2, 4) ? 2 : 1;
  const int64_t tiles = (T + kTokTile - 1) / kTokTile;
  const bool dual = packed_tables(d.V) == 2;
  const bool wide = i8_staged_wide(tiles, a.R);
  const int64_t S = a.S, R = a.R, y_bytes = e.y_dtype == VNM_F32 ? 4 : 2;
  // more tiles or row blocks than a grid has room for: one launch per range of them
  for (int64_t tile = 0; tile < tiles; tile += kI8GridTiles)
    for (int64_t r = 0; r < R; r += kI8GridRows) {
      const int64_t t0 = tile * kTokTile, o0 = r * kPackedRows;
      I8StagedArgs b = a;
      b.staged += tile * S * a.image;
      b.T = T - t0 < kI8GridTiles * kTokTile ? T - t0 : kI8GridTiles * kTokTile;
      b.pa += r * S * 2048; b.pidx += r * S * 512; b.pcol += r * S * 64 * (dual ? 2 : 1);
      b.R = R - r < kI8GridRows ? R - r : kI8GridRows;
      b.out = d.out - o0 < kI8GridRows * kPackedRows ? d.out - o0 : kI8GridRows * kPackedRows;
      b.e.Y = (unsigned char*)e.Y + (t0 * e.ldy + o0) * y_bytes;
      b.e.scale_x += t0; b.e.scale_w += o0;
      if (e.bias) b.e.bias += o0;
      if (int rc = dual ? launch_staged<true>(b, d.M, wide, st) : launch_staged<false>(b, d.M, wide, st)) return rc;
    }
  return VNM_OK;
}

}  // namespace vnm
