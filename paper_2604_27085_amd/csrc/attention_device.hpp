// Device code that the attention kernels share: tiles on their way from memory through registers to LDS, the fragments that the matrix
// instructions read from them, and accumulators on their way out.  attention.hip says how the kernels are built from these.
#pragma once
#include "common.hpp"

namespace {

typedef __amdgpu_buffer_rsrc_t rsrc_t;

// Consecutive workgroups go to consecutive XCDs (eight, each with an L2 of its own).  The i-th of the nhb workgroups of a
// query tile therefore takes head (i mod 8) * nhb/8 + i/8 instead of head i: an XCD then works on nhb/8 neighbouring query
// heads, i.e. on one or two K/V heads with grouped queries, and its L2 fetches their K/V tiles once for all the workgroups
// that stream them side by side -- instead of every XCD fetching every K/V head.
RP_DEV int xcd_head(int i, int nhb) { return (nhb & 7) ? i : (i & 7) * (nhb >> 3) + (i >> 3); }

RP_DEV uint4 buf_load16(rsrc_t r, uint32_t voff) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)voff, 0, 0);
  return make_uint4(v.x, v.y, v.z, v.w);
}

// Row stride of a tile in LDS (elements): 8 banks past a multiple of 64, so that neither the 16-byte reads of 16 rows by four lane groups nor
// the transposing ones (32 lanes a phase: eight rows of 32 bytes) meet on a bank.
constexpr int tile_ld(int d) { return d + 16; }

// ---- 64 x D tile: global -> registers -> LDS -----------------------------------------------------------------
template <int D, int NT>
struct Tile64 {
  static constexpr int CH = D / 8, NREG = 64 * CH / NT;
  static_assert((64 * CH) % NT == 0, "tile does not divide over the threads");
  // rows row0..row0+63 of a [seq, D] view with row stride ld (elements)
  static RP_DEV void load(uint4 (&r)[NREG], rsrc_t rs, long ld, int row0, int tid) {
#pragma unroll
    for (int it = 0; it < NREG; ++it) {
      const int c = it * NT + tid;
      r[it] = buf_load16(rs, (uint32_t)(((long)(row0 + c / CH) * ld + (c % CH) * 8) * 2));
    }
  }
  template <int LDS_LD>
  static RP_DEV void store(const uint4 (&r)[NREG], bf16* S, int tid) {
#pragma unroll
    for (int it = 0; it < NREG; ++it) {
      const int c = it * NT + tid;
      *reinterpret_cast<uint4*>(S + (c / CH) * LDS_LD + (c % CH) * 8) = r[it];
    }
  }
};

// A-operand fragment from a [64][LD] tile whose rows are the reduction index (keys or queries) and whose columns are
// the MFMA rows: the 8 values of lane group g = lane / 16 are tile rows {4g + e, 16 + 4g + e}, e = 0..3, at column lane % 16 -- the
// order in which two 16-row tiles of scores hold them.  base = S + tr_base(lane) + first row * LD + first column.
template <int LD>
RP_DEV uint4 read_frag_tr(const bf16* base) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* lds_ptr;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(base));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(base + 16 * LD));
  const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
  return make_uint4(l2.x, l2.y, h2.x, h2.y);
}
template <int LD>
RP_DEV int tr_base(int lane) {
  return (4 * (lane >> 4) + ((lane & 15) >> 2)) * LD + 4 * (lane & 3);
}

// Two 16-row score tiles, one above the other, as the B operand of the next product: 32 reduction indices in the order of read_frag_tr.
RP_DEV uint4 pack_frag(const f32x4& a, const f32x4& b) {
  return make_uint4(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3]));
}

// Sum over the four lanes that hold a column.
RP_DEV float column_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
RP_DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Two waves share a SIMD in the forward kernel.  Left alone they fall into step: both issue their matrix products at
// the same time (each at half rate) and then both do their exponentials, so the matrix pipeline idles while the vector
// pipeline works and the other way round.  A wave raises its issue priority for its runs of MFMAs: whichever wave gets
// there first keeps the matrix pipeline to itself, the other one falls behind by a phase, and from then on one wave's
// exponentials run under the other wave's products (forward kernel +6 % at 8192 to 31744 tokens; the dQ kernel, whose
// vector phase is short against its three products, does not change).
#define MFMA_PHASE_BEGIN() __builtin_amdgcn_s_setprio(1)
#define MFMA_PHASE_END() __builtin_amdgcn_s_setprio(0)

// A wave's staged 32 x D block to global.
template <int D>
RP_DEV void store_staged(const bf16* stage, bf16* __restrict__ out, long ld, int row0, int nrows, int lane) {
  __syncthreads();
#pragma unroll
  for (int it = 0; it < (32 * (D / 8)) / 64; ++it) {
    const int idx = it * 64 + lane;
    const int row = idx / (D / 8), ch = idx % (D / 8);
    if (row0 + row < nrows)
      *reinterpret_cast<uint4*>(out + (long)(row0 + row) * ld + ch * 8) =
          *reinterpret_cast<const uint4*>(stage + row * (D + 8) + ch * 8);
  }
  __syncthreads();
}

// Writes a wave's 32 x D transposed accumulator (16x16 tiles; columns = the wave's 32 rows of the output) through LDS to global.
template <int D>
RP_DEV void store_acc_T(const f32x4 (&acc)[D / 16][2], float mul, bf16* stage /* [32][D+8] */, bf16* __restrict__ out,
                        long ld, int row0, int nrows, int lane) {
  const int lr = lane & 15, lg = lane >> 4;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
    for (int c = 0; c < 2; ++c)
      *reinterpret_cast<uint2*>(stage + (16 * c + lr) * (D + 8) + 16 * dt + 4 * lg) =
          make_uint2(pack_bf16x2(acc[dt][c][0] * mul, acc[dt][c][1] * mul),
                     pack_bf16x2(acc[dt][c][2] * mul, acc[dt][c][3] * mul));
  store_staged<D>(stage, out, ld, row0, nrows, lane);
}

// Same for an fp32 destination; stage is [32][D + 4] floats per wave.
template <int D>
RP_DEV void store_acc_T_f32(const f32x4 (&acc)[D / 16][2], float mul, float* stage, float* __restrict__ out, long ld,
                            int row0, int nrows, int lane) {
  const int lr = lane & 15, lg = lane >> 4;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
    for (int c = 0; c < 2; ++c)
      *reinterpret_cast<float4*>(stage + (16 * c + lr) * (D + 4) + 16 * dt + 4 * lg) =
          make_float4(acc[dt][c][0] * mul, acc[dt][c][1] * mul, acc[dt][c][2] * mul, acc[dt][c][3] * mul);
  __syncthreads();
#pragma unroll
  for (int it = 0; it < (32 * (D / 4)) / 64; ++it) {
    const int idx = it * 64 + lane;
    const int row = idx / (D / 4), ch = idx % (D / 4);
    if (row0 + row < nrows)
      *reinterpret_cast<float4*>(out + (long)(row0 + row) * ld + ch * 4) =
          *reinterpret_cast<const float4*>(stage + row * (D + 4) + ch * 4);
  }
  __syncthreads();
}

// The fragments of the forward kernel's 32x32 tiles.  The lane half h = lane / 32 holds, of 16 rows, {4h..4h+3, 8+4h..8+4h+3}: what read_frag_tr is
// to the 16x16 tiles; the 8 values of the A operand are tile rows 16 g + those, at column lane % 32 from x_off on.
template <int LD>
RP_DEV uint4 read_frag_tr32(const bf16* base, int g, int x_off) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* lds_ptr;
  const bf16* q = base + 16 * g * LD + x_off;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(q));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(q + 8 * LD));
  const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
  return make_uint4(l2.x, l2.y, h2.x, h2.y);
}
template <int LD>
RP_DEV int tr_base32(int lane) {
  const int lk = lane >> 5, l16 = lane & 15, g16 = lane >> 4;
  return (4 * lk + (l16 >> 2)) * LD + 16 * (g16 & 1) + 4 * (l16 & 3);
}
RP_DEV uint4 pack_frag32(const f32x16& s, int off) {
  return make_uint4(pack_bf16x2(s[off + 0], s[off + 1]), pack_bf16x2(s[off + 2], s[off + 3]),
                    pack_bf16x2(s[off + 4], s[off + 5]), pack_bf16x2(s[off + 6], s[off + 7]));
}
// max over lanes l and l ^ 32, in the vector unit: the exchange through LDS is a round trip of the wave in every key tile.  Forward of
// 8192 tokens, 64 heads of 64: 702 -> 673 us (with the mask test on one limit per lane); the eight-wave kernel, whose waves pair up
// around that wait, is 4 % slower with it (521 -> 542) and keeps the exchange
RP_DEV float half_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// store_acc_T for 32x32 tiles.
template <int D>
RP_DEV void store_acc_T32(const f32x16 (&acc)[D / 32], float mul, bf16* stage /* [32][D+8] */, bf16* __restrict__ out, long ld, int row0, int nrows, int lane) {
  const int lr = lane & 31, lk = lane >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int vg = 0; vg < 4; ++vg) {
      const int dd = 32 * dt + 8 * vg + 4 * lk;
      *reinterpret_cast<uint2*>(stage + lr * (D + 8) + dd) =
          make_uint2(pack_bf16x2(acc[dt][4 * vg] * mul, acc[dt][4 * vg + 1] * mul),
                     pack_bf16x2(acc[dt][4 * vg + 2] * mul, acc[dt][4 * vg + 3] * mul));
    }
  store_staged<D>(stage, out, ld, row0, nrows, lane);
}

}  // namespace
