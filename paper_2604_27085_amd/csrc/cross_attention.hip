// Attention of one sequence's queries to another sequence's keys (a decoder attending to an encoder's states), forward and backward:
// no causal mask, lengths of their own for queries and keys, padded batches.
//
//   S = scale q k^T over the keys before kv_len;  lse = log sum exp S;  P = exp(S - lse);  o = P v
//   dV = P^T dO;  dP = dO V^T;  delta = rowsum(P dP) (= rowsum(dO o));  dS = P (dP - delta);  dQ = scale dS K;  dK = scale dS^T Q
//
// Without a causal mask nothing tells the query heads of a key head's group apart: the grp query heads times q_len queries of one key head
// are simply grp q_len ROWS against the same keys (row r is query r % q_len of head r / q_len; the padded queries come behind them all).
// Tiles are cut from the rows, so short sequences of many heads fill them, one workgroup's keys serve all heads of the group, and dK, dV of a
// group need no partials per head.  The tiles, fragments and instructions are those of attention.hip.
//
//   forward: workgroup = four waves x 32 rows, loop over 64-key tiles (eight waves, one workgroup per CU, which pays in attention.hip, are 0 to 3 %
//            slower here, where no workgroup has fewer tiles than another)
//   dQ     : the same; delta on the way (with the loop in slices, in a launch before)
//   dK, dV : workgroup = 128 keys, loop over 64-row tiles (d = 128: eight waves, pairs of which share 32 keys; d = 64: four waves)
// Where there are too few workgroups for the chip, the loop is cut into `splits` slices, whose results another kernel joins in slice
// order (fp32 partials in the caller's scratch; no atomics, so the result does not depend on timing).
// Keys behind kv_len are never read (they may hold anything); rows behind q_len get zeros, and lse -inf.
//
// What bounds them, at 4096 queries of 32 heads of 128 against 8192 keys of 8 heads (kernels alone, medians of 60 passes): forward 536 us (1.03 PFLOP/s), dQ 940 (1.17
// with the product's second part, see cross_dq_kernel), dK/dV 988 (1.11); matrix pipe busy 58, 58 and 50 %, vector issue 48, 52 and 41 %, memory nothing to speak of: the
// exponentials and conversions beside the products, and the clock that the power allows, as in attention.hip.  At d = 64 (64 heads, 4 x 512 queries against 1536 keys)
// 71, 140 and 124 us: the
// vector instructions of a tile are the same for half the products.  A padded batch adds what its longest sequence's workgroups last longer.
// P, and dS for dK, are rounded to bf16, as the matrix instruction takes them (2^-8 a term at most); dS for dQ is taken in two parts; scores, statistics,
// dP - delta and every sum are fp32.
#include "attention_device.hpp"
#include "layer_ops.hpp"

namespace {

// Lengths and places of one sequence and key head.  Lengths that the caller got wrong count as the nearest possible one.
struct Rows {
  int b, g, grp, qlen, kvlen, valid, total, seq_q;   // valid = grp * qlen rows hold queries, total = grp * seq_q
  RP_DEV Rows(const CrossArgs& p, int hb) {
    b = hb / p.kh;
    g = hb - b * p.kh;
    grp = p.a / p.kh;
    seq_q = p.seq_q;
    qlen = p.q_len ? min(max(p.q_len[b], 0), p.seq_q) : p.seq_q;
    kvlen = p.kv_len ? min(max(p.kv_len[b], 0), p.seq_kv) : p.seq_kv;
    valid = grp * qlen;
    total = grp * seq_q;
  }
  // head within the group and query of row r < total
  RP_DEV void at(int r, int& h, int& q) const {
    if (r < valid) {
      h = r / qlen;
      q = r - h * qlen;
    } else {
      const int j = r - valid, pad = seq_q - qlen;
      h = j / pad;
      q = qlen + j - h * pad;
    }
  }
  // offset of row r in a [T, heads, d] tensor of row stride ld, from its first element
  RP_DEV long offset(int r, long ld, int d) const {
    int h, q;
    at(r, h, q);
    return ((long)b * seq_q + q) * ld + (long)(g * grp + h) * d;
  }
  RP_DEV long stat(int r, int a) const {   // in a [batch, a, seq_q] array
    int h, q;
    at(r, h, q);
    return ((long)b * a + g * grp + h) * seq_q + q;
  }
};

// Slice `s` of `n` steps cut into `splits`: [first, last).  The number of slices that have any is used again where they are joined.
RP_DEV void slice_of(int n, int splits, int s, int& first, int& last) {
  const int per = (n + splits - 1) / splits;
  first = min(s * per, n);
  last = min(first + per, n);
}
RP_DEV int slices_used(int n, int splits) {
  if (n == 0) return 0;
  const int per = (n + splits - 1) / splits;
  return (n + per - 1) / per;
}

// Launch order: the key heads of all sequences change fastest, so that (workgroups go round the eight XCDs) one XCD's L2 keeps to the key heads of
// its residue, and the sequences of a padded batch spread over all XCDs.  From one round of 256 workgroups to the next the heads move on by eight: a CU
// that had a workgroup of the longest sequence gets one of another then.  (Training 4 x 509 queries of 64 heads of 64 against up to 1500 keys:
// forward 68.6 us with neighbouring key heads per XCD as in attention.hip, where two XCDs have the longest sequence to themselves.)
RP_DEV int head_at(int pos, int rest, int nhb) { return (pos - rest * nhb + 8 * (int)(((long)rest * nhb) >> 8)) % nhb; }

// Between a wave's stores to LDS and its lanes' reads of one another's (and the other way round): LDS works in order for a wave, so this is for the compiler.
RP_DEV void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A 64-key tile, through a descriptor of its own that ends with the sequence: rows past the end read as zero, and no offset outgrows 32
// bits however long the sequence is.
template <int D, int NT>
struct KeyTile {
  using T64 = Tile64<D, NT>;
  const bf16* base;
  long ld;
  int len;
  RP_DEV KeyTile(const bf16* b, long l, int n) : base(b), ld(l), len(n) {}
  RP_DEV void load(uint4 (&r)[T64::NREG], int key0, int tid) const {
    const int left = min(64, len - key0);      // >= 1
    const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(base + (long)key0 * ld), 0, (int)(((long)(left - 1) * ld + D) * 2), 0x00020000);
    T64::load(r, rs, ld, 0, tid);
  }
};

// Zeros for the rows of [r0, r0 + n) that are behind the queries, all threads of the block.
template <int D, int NT>
RP_DEV void zero_rows(const CrossArgs& p, const Rows& s, bf16* out, long ld, float* lse, int r0, int n, int tid) {
  constexpr int CH = D / 8;
  for (int i = tid; i < n * CH; i += NT) {
    const int r = r0 + i / CH;
    if (r < s.valid || r >= s.total) continue;
    *reinterpret_cast<uint4*>(out + s.offset(r, ld, D) + (i % CH) * 8) = make_uint4(0u, 0u, 0u, 0u);
    if (lse && i % CH == 0) lse[s.stat(r, p.a)] = -INFINITY;
  }
}

// ================================================================================================ forward
template <int D, bool SPLIT>
__global__ void __launch_bounds__(256, 2) cross_fwd_kernel(const CrossArgs p) {
  constexpr int LDK = D + 8, LDV = D + 32, KS = D / 16, DT = D / 32, NT = 256, BQ = 128;
  using T64 = Tile64<D, NT>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];   // fwd_smem_bytes(D)
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);
  bf16* const Ks = smem;
  bf16* const Vs = smem + 64 * LDK;

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lk = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nhb = p.kh * p.batch;
  const int rest = (int)blockIdx.x / nhb;
  const int hb = head_at((int)blockIdx.x, rest, nhb);
  const int split = SPLIT ? rest % p.splits : 0;
  const int r0 = (SPLIT ? rest / p.splits : rest) * BQ;
  const Rows s(p, hb);
  if (r0 >= s.valid) {      // uniform over the workgroup, before any barrier
    if (!SPLIT) zero_rows<D, NT>(p, s, p.o, p.ldo, p.lse, r0, BQ, tid);
    return;
  }
  int j0 = 0, j1 = (s.kvlen + 63) / 64;
  if (SPLIT) {
    slice_of(j1, p.splits, split, j0, j1);
    if (j0 >= j1) return;
  }
  const KeyTile<D, NT> kt_(p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D, p.ldk, s.kvlen), vt_(p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D, p.ldv, s.kvlen);

  const int row = r0 + 32 * w + lr;     // the lane's row
  const bool live = row < s.valid;
  uint4 qf[KS];
  {
    const bf16* const qr = live ? p.q + s.offset(row, p.ldq, D) : p.q;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = make_uint4(0u, 0u, 0u, 0u);
      if (live) qf[ks] = *reinterpret_cast<const uint4*>(qr + 16 * ks + 8 * lk);
    }
  }

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) oacc[dt][v] = 0.f;

  const bf16* const kfrag = Ks + lr * LDK + 8 * lk;
  const bf16* const vfrag = Vs + tr_base32<LDV>(lane);
  uint4 kreg[T64::NREG], vreg[T64::NREG];
  auto load_tiles = [&](int j) {
    kt_.load(kreg, j * 64, tid);
    vt_.load(vreg, j * 64, tid);
  };
  if (j0 < j1) load_tiles(j0);
  for (int j = j0; j < j1; ++j) {
    __syncthreads();
    T64::template store<LDK>(kreg, Ks, tid);
    T64::template store<LDV>(vreg, Vs, tid);
    __syncthreads();
    if (j + 1 < j1) load_tiles(j + 1);
    const int kv0 = j * 64;
    f32x16 sT[2];
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = 3;      // LDS fragments are requested that many products early
    {
      constexpr int NS = 2 * KS;
      auto sfrag_at = [&](int n) { return *reinterpret_cast<const uint4*>(kfrag + 32 * (n & 1) * LDK + 16 * (n >> 1)); };
      uint4 ring[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) ring[n] = sfrag_at(n);
      MFMA_PHASE_BEGIN();
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const uint4 a = ring[n % AHEAD];
        if (n + AHEAD < NS) ring[n % AHEAD] = sfrag_at(n + AHEAD);
        sT[n & 1] = mfma32(a, qf[n >> 1], n < 2 ? zero16 : sT[n & 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
      MFMA_PHASE_END();
    }
    constexpr int NU = 4 * DT;
    auto ufrag_at = [&](int n) { return read_frag_tr32<LDV>(vfrag, n / DT, 32 * (n % DT)); };
    uint4 uring[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) uring[n] = ufrag_at(n);
    __builtin_amdgcn_sched_barrier(0);
    if (kv0 + 64 > s.kvlen) {      // uniform: the last tile
      const int klim = s.kvlen - 1 - (kv0 + 4 * lk);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v) sT[kt][v] = (32 * kt + 8 * (v >> 2) + (v & 3) > klim) ? -INFINITY : sT[kt][v];
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sT[kt][v]);
    mx = half_max(mx) * p.scale_log2e;
    // m_run is a reference exponent that moves only when a row's maximum outgrows it by 2^8 (see attention.hip); every tile has a key,
    // so it is finite from the first one on
    const bool grow = mx > m_run + 8.f;
    if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
      const float m_new = grow ? mx : m_run;
      float alpha = fast_exp2(m_run - m_new);
      asm volatile("" : "+v"(alpha));
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
    }
    float psum = 0.f;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float e = fast_exp2(__builtin_fmaf(sT[kt][v], p.scale_log2e, -m_run));
        sT[kt][v] = e;
        psum += e;
      }
    l_run += psum;
    {
      uint4 pf[4];      // P in bf16, as the matrix instruction takes it: relative 2^-8 a term, on sums held in fp32
#pragma unroll
      for (int gk = 0; gk < 4; ++gk) pf[gk] = pack_frag32(sT[gk >> 1], 8 * (gk & 1));
      MFMA_PHASE_BEGIN();
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        const uint4 a = uring[n % AHEAD];
        if (n + AHEAD < NU) uring[n % AHEAD] = ufrag_at(n + AHEAD);
        oacc[n % DT] = mfma32(a, pf[n / DT], oacc[n % DT]);
        __builtin_amdgcn_sched_barrier(0);
      }
      MFMA_PHASE_END();
    }
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if constexpr (SPLIT) {
    const long at = ((long)split * nhb + hb) * s.total + row;
    if (live) {
      if (lk == 0) p.part_ml[at] = make_float2(m_run, l_tot);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int vg = 0; vg < 4; ++vg)
          *reinterpret_cast<float4*>(p.part + at * D + 32 * dt + 8 * vg + 4 * lk) =
              make_float4(oacc[dt][4 * vg], oacc[dt][4 * vg + 1], oacc[dt][4 * vg + 2], oacc[dt][4 * vg + 3]);
    }
  } else {
    const bool some = live && j0 < j1;      // a row without keys: o = 0, lse = -inf
    const float mul = some ? 1.f / l_tot : 0.f;
    if (p.lse && lk == 0 && row < s.total) p.lse[s.stat(row, p.a)] = some ? m_run * 0.6931471805599453f + logf(l_tot) : -INFINITY;
    __syncthreads();
    bf16* const stage = smem + w * 32 * LDK;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int vg = 0; vg < 4; ++vg) {
        const uint2 u = make_uint2(pack_bf16x2(oacc[dt][4 * vg] * mul, oacc[dt][4 * vg + 1] * mul), pack_bf16x2(oacc[dt][4 * vg + 2] * mul, oacc[dt][4 * vg + 3] * mul));
        *reinterpret_cast<uint2*>(stage + lr * LDK + 32 * dt + 8 * vg + 4 * lk) = some ? u : make_uint2(0u, 0u);
      }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < (32 * (D / 8)) / 64; ++it) {
      const int idx = it * 64 + lane, rr = idx / (D / 8), ch = idx % (D / 8), r = r0 + 32 * w + rr;
      if (r < s.total) *reinterpret_cast<uint4*>(p.o + s.offset(r, p.ldo, D) + ch * 8) = *reinterpret_cast<const uint4*>(stage + rr * LDK + ch * 8);
    }
  }
}

// ---- few rows: the step of a generation -----------------------------------------------------------------------
// At most 16 NC rows per key head (the queries of a step times the heads of the group).  Bound by reading K and V once, so a wave works alone, without
// barriers: the waves of a workgroup take its 32-key steps in turn, K goes from memory straight into the fragments of the matrix
// instruction (16 rows x 64 bytes a load: a whole row is used by one wave), V through a piece of LDS of the wave's own, since its
// reduction runs over the keys.  The next step's K and V are on their way during a step.  At the end the waves join in LDS.
// One token of 2 sequences with 64 heads against 32768 keys: 57 us with the join, 52 of them for 268 MB, the rate of a large copy.
template <int D, int NC, int NW, bool SPLIT>
__global__ void __launch_bounds__(64 * NW) cross_step_kernel(const CrossArgs p) {
  constexpr int LD = tile_ld(D), KS = D / 32, DT = D / 16, CH = D / 8, NV = 32 * CH / 64;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];   // step_smem_bytes(D, NC, NW)
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  bf16* const Vs = reinterpret_cast<bf16*>(dyn_smem) + w * 32 * LD;
  const int nhb = p.kh * p.batch;
  const int hb = (int)blockIdx.x % nhb, split = (int)blockIdx.x / nhb;
  const Rows s(p, hb);
  int j0 = 0, j1 = (s.kvlen + 31) / 32;
  if (SPLIT) {
    slice_of(j1, p.splits, split, j0, j1);
    if (j0 >= j1) return;      // uniform, before any barrier
  }
  const bf16* const kb = p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D;
  const bf16* const vb = p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D;

  uint4 qf[NC][KS];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int row = 16 * c + lr;
    const bool live = row < s.valid;
    const bf16* const qr = live ? p.q + s.offset(row, p.ldq, D) + 8 * lg : p.q;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      if (live) qf[c][ks] = *reinterpret_cast<const uint4*>(qr + 32 * ks);
    }
  }
  float m_run[NC], l_run[NC];
  f32x4 oacc[DT][NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m_run[c] = -INFINITY;
    l_run[c] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  u32x4 kreg[2][KS], vreg[NV];
  auto load_step = [&](int j) {      // rows past the end read as zero
    const int left = min(32, s.kvlen - 32 * j);
    const rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(kb + (long)(32 * j) * p.ldk), 0, (int)(((long)(left - 1) * p.ldk + D) * 2), 0x00020000);
    const rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(vb + (long)(32 * j) * p.ldv), 0, (int)(((long)(left - 1) * p.ldv + D) * 2), 0x00020000);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        kreg[kt][ks] = __builtin_amdgcn_raw_buffer_load_b128(rk, (int)(((16 * kt + lr) * (int)p.ldk + 32 * ks + 8 * lg) * 2), 0, 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 64 * i + lane;
      vreg[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, (int)(((c / CH) * (int)p.ldv + (c % CH) * 8) * 2), 0, 0);
    }
  };
  if (j0 + w < j1) load_step(j0 + w);
  const bf16* const vfrag = Vs + tr_base<LD>(lane);
  for (int j = j0 + w; j < j1; j += NW) {
    f32x4 sT[2][NC];      // [16 keys][16 rows]
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          sT[kt][c] = mfma16(__builtin_bit_cast(uint4, kreg[kt][ks]), qf[c][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sT[kt][c]);
    wave_lds_order();      // the last step's V has been read
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 64 * i + lane;
      *reinterpret_cast<u32x4*>(Vs + (c / CH) * LD + (c % CH) * 8) = vreg[i];
    }
    wave_lds_order();
    if (j + NW < j1) load_step(j + NW);
    if (32 * j + 32 > s.kvlen) {      // uniform: the last step
      const int klim = s.kvlen - 1 - (32 * j + 4 * lg);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) sT[kt][c][e] = 16 * kt + e > klim ? -INFINITY : sT[kt][c][e];
    }
    uint4 pf[NC];
    bool grow = false;
    float mx[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      mx[c] = fmaxf(fmaxf(fmaxf(sT[0][c][0], sT[0][c][1]), fmaxf(sT[0][c][2], sT[0][c][3])), fmaxf(fmaxf(sT[1][c][0], sT[1][c][1]), fmaxf(sT[1][c][2], sT[1][c][3])));
      grow = grow || mx[c] * p.scale_log2e > m_run[c] + 8.f;
    }
    // the reference exponent is the same in the four lanes of a column, and moves only when one of them outgrows it by 2^8
    if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float m = fmaxf(mx[c], __shfl_xor(mx[c], 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64)) * p.scale_log2e;
        const float m_new = m > m_run[c] + 8.f ? m : m_run[c];
        const float alpha = fast_exp2(m_run[c] - m_new);
        l_run[c] *= alpha;
        m_run[c] = m_new;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) oacc[dt][c] *= alpha;
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sT[kt][c][e] = fast_exp2(__builtin_fmaf(sT[kt][c][e], p.scale_log2e, -m_run[c]));
          l_run[c] += sT[kt][c][e];
        }
      pf[c] = pack_frag(sT[0][c], sT[1][c]);
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const uint4 a = read_frag_tr<LD>(vfrag + 16 * dt);
#pragma unroll
      for (int c = 0; c < NC; ++c) oacc[dt][c] = mfma16(a, pf[c], oacc[dt][c]);
    }
  }

  // the waves join: wave w's reference exponent and sum of every row, then its rows of O^T
  float* const ml = reinterpret_cast<float*>(dyn_smem);      // [NW][2][16 NC]
  float* const os = ml + 2 * NW * 16 * NC;                   // [NW][16 NC][D + 4]
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const float l = column_sum(l_run[c]);
    if (lg == 0) {
      ml[(2 * w) * 16 * NC + 16 * c + lr] = m_run[c];
      ml[(2 * w + 1) * 16 * NC + 16 * c + lr] = l;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<f32x4*>(os + (w * 16 * NC + 16 * c + lr) * (D + 4) + 16 * dt + 4 * lg) = oacc[dt][c];
  }
  __syncthreads();
  for (int i = tid; i < 16 * NC * CH; i += 64 * NW) {
    const int row = i / CH, ch = i % CH;
    if (row >= s.total) break;
    const bool live = row < s.valid && j0 < j1;
    if (SPLIT && !live) continue;
    float m = -INFINITY, l = 0.f, acc[8];
#pragma unroll
    for (int u = 0; u < NW; ++u) m = fmaxf(m, ml[2 * u * 16 * NC + row]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int u = 0; u < NW; ++u) {
      const float mu = ml[2 * u * 16 * NC + row];
      const float wgt = mu == -INFINITY ? 0.f : fast_exp2(mu - m);      // (a wave without a step)
      l += wgt * ml[(2 * u + 1) * 16 * NC + row];
      const float* const src = os + (u * 16 * NC + row) * (D + 4) + 8 * ch;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += wgt * src[e];
    }
    if constexpr (SPLIT) {
      const long at = ((long)split * nhb + hb) * s.total + row;
      if (ch == 0) p.part_ml[at] = make_float2(m, l);
      *reinterpret_cast<float4*>(p.part + at * D + 8 * ch) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      *reinterpret_cast<float4*>(p.part + at * D + 8 * ch + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
    } else {
      const float mul = live ? 1.f / l : 0.f;
      if (p.lse && ch == 0) p.lse[s.stat(row, p.a)] = live ? m * 0.6931471805599453f + logf(l) : -INFINITY;
      const uint4 u = make_uint4(pack_bf16x2(acc[0] * mul, acc[1] * mul), pack_bf16x2(acc[2] * mul, acc[3] * mul), pack_bf16x2(acc[4] * mul, acc[5] * mul),
                                 pack_bf16x2(acc[6] * mul, acc[7] * mul));
      *reinterpret_cast<uint4*>(p.o + s.offset(row, p.ldo, D) + 8 * ch) = live ? u : make_uint4(0u, 0u, 0u, 0u);
    }
  }
}

// ---- joining slices.  A thread has eight elements of one row and every G-th slice; the G threads that share them are added up in a fixed order, by
// lane exchanges and, where they are in several waves, through LDS.  G grows with the number of slices: few slices of many rows are a matter
// of bandwidth, many slices of few rows one of the latency of the loads that follow one another.
template <int CH, int G, int N>
RP_DEV bool add_groups(float (&acc)[N], float* red /* [256 / 64][CH * N] */) {
  const int tid = threadIdx.x, lane = tid & 63;
  constexpr int IN_WAVE = CH * G < 64 ? CH * G : 64, WAVES = CH * G / IN_WAVE;
#pragma unroll
  for (int e = 0; e < N; ++e)
#pragma unroll
    for (int o = CH; o < IN_WAVE; o <<= 1) acc[e] += __shfl_xor(acc[e], o, 64);
  if constexpr (WAVES > 1) {
    const int ch = tid % CH, w = tid >> 6, first = w / WAVES * WAVES;
    if (lane < CH)
#pragma unroll
      for (int e = 0; e < N; ++e) red[w * CH * N + ch * N + e] = acc[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < N; ++e) {
      acc[e] = red[first * CH * N + ch * N + e];
#pragma unroll
      for (int u = 1; u < WAVES; ++u) acc[e] += red[(first + u) * CH * N + ch * N + e];
    }
  }
  return tid % (CH * G) < CH;      // the thread that stores
}
RP_DEV uint4 pack_times(const float* acc, float mul) {
  return make_uint4(pack_bf16x2(acc[0] * mul, acc[1] * mul), pack_bf16x2(acc[2] * mul, acc[3] * mul), pack_bf16x2(acc[4] * mul, acc[5] * mul),
                    pack_bf16x2(acc[6] * mul, acc[7] * mul));
}
RP_DEV void add_times(float* acc, const float* src, float wgt) {
  const float4 x0 = *reinterpret_cast<const float4*>(src), x1 = *reinterpret_cast<const float4*>(src + 4);
  acc[0] += wgt * x0.x; acc[1] += wgt * x0.y; acc[2] += wgt * x0.z; acc[3] += wgt * x0.w;
  acc[4] += wgt * x1.x; acc[5] += wgt * x1.y; acc[6] += wgt * x1.z; acc[7] += wgt * x1.w;
}

// Rows of the forward (weights exp2(m_i - max m)) or, with DQ, of dq (sums, times scale).  unit: keys a step of the kernel that cut the slices.
template <int D, int G, bool DQ>
__global__ void __launch_bounds__(256) cross_row_join_kernel(const CrossArgs p, int unit) {
  constexpr int CH = D / 8, RPB = 256 / (CH * G);
  __shared__ float red[CH * G > 64 ? 4 * CH * 9 : 1];
  const int total = (p.a / p.kh) * p.seq_q, nhb = p.kh * p.batch;
  const int tid = threadIdx.x, ch = tid % CH, grp = tid / CH % G;
  const long item = (long)blockIdx.x * RPB + tid / (CH * G);
  const bool in = item < (long)nhb * total;
  const int hb = in ? (int)(item / total) : 0, r = in ? (int)(item - (long)hb * total) : 0;
  const Rows s(p, hb);
  const int n = in && r < s.valid ? slices_used((s.kvlen + unit - 1) / unit, p.splits) : 0;
  const long row = (long)hb * total + r, step = (long)nhb * total;
  constexpr int N = DQ ? 8 : 9;      // eight elements, and the forward's sum of exponentials
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  float m = -INFINITY;
  if constexpr (!DQ) {
    constexpr int L = CH * G < 64 ? CH * G : 64;      // lanes of a wave that work on the row
#pragma unroll 2
    for (int i = tid % L; i < n; i += L) m = fmaxf(m, p.part_ml[i * step + row].x);
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  }
#pragma unroll 4
  for (int i = grp; i < n; i += G) {
    float wgt = 1.f;
    if constexpr (!DQ) {
      const float2 ml = p.part_ml[i * step + row];
      wgt = fast_exp2(ml.x - m);
      acc[8] += wgt * ml.y;
    }
    add_times(acc, p.part + (i * step + row) * D + ch * 8, wgt);
  }
  const bool mine = add_groups<CH, G, N>(acc, red);
  if (!in || !mine) return;
  if constexpr (DQ) {
    *reinterpret_cast<uint4*>(p.dq + s.offset(r, p.lddq, D) + ch * 8) = pack_times(acc, p.scale);
  } else {
    if (p.lse && ch == 0) p.lse[s.stat(r, p.a)] = n ? m * 0.6931471805599453f + logf(acc[8]) : -INFINITY;
    *reinterpret_cast<uint4*>(p.o + s.offset(r, p.ldo, D) + ch * 8) = pack_times(acc, n ? 1.f / acc[8] : 0.f);
  }
}

// ================================================================================================ dQ
// dP - delta cancels where a row puts nearly all of its weight on one key, and a delta from the stored output, dO.o, carries that one's rounding (2^-8 at most):
// rows on one of 129 keys had dq off by 0.06 to 0.16 of its norm.  So delta has to be as exact as the scores where it matters:
//   up to EXACT_DELTA keys, unless cut into slices, the scores are made twice, the first time for delta = sum P dP / sum P;
//   with the key loop in slices a launch of its own (DELTA) makes those two sums of every slice;
//   else delta starts as dO.o, and the rows of dS, which sum up to zero, tell at the end what it was off by.  Rows where that is more than FAR sum |dS|, more
//   than a rounding of every dS to bf16 could do, get dq - off sum P K (mean_keys; of rows whose scores have standard deviation 2
//   one in 10000 against 8192 keys, one in 1500 against 1500 and one in 240 against 300), the others dq - off times the mean of 64 keys: that takes out what a
//   part that all keys share would add (three times their spread: dq off by 1.9e-3 instead of 8e-3).  dK, dV take the corrected delta in any case.
// dS goes into its product in two parts, its bf16 and the bf16 of what that left over: K^T's fragments serve both, and dq is off by little more than its
// own rounding (relative 2-norm 1.7e-3 with delta from the scores; in one part 2.4e-3).
constexpr int EXACT_DELTA = 256;
constexpr float FAR = 1.f / 256.f;
// WHOLE: a workgroup's rows against all keys; EXACT: the same where no sequence has more than EXACT_DELTA keys; SLICE, DELTA: a slice of them
enum DqPass { WHOLE, EXACT, SLICE, DELTA };

// Two score tiles as pack_frag gives them, and what that rounding left over.  (a, b are used up.)
RP_DEV void two_parts(f32x4& a, f32x4& b, uint4& high, uint4& low) {
  high = pack_frag(a, b);
  a -= f32x4{bf16_lo(high.x), bf16_hi(high.x), bf16_lo(high.y), bf16_hi(high.y)};
  b -= f32x4{bf16_lo(high.z), bf16_hi(high.z), bf16_lo(high.w), bf16_hi(high.w)};
  low = pack_frag(a, b);
}

constexpr int dq_tile_bytes(int d) { return 2 * 64 * tile_ld(d) * 2; }

// sum[i][..] = sum_k P K of rows list[i], i < n <= 16, of a workgroup's 128.  There are few of them, so the waves share their keys: a wave takes every fourth
// step of 32 keys by itself, K from memory straight into fragments for the scores, three steps ahead, and through a piece of LDS of its own for the product
// whose reduction runs over the keys; in the end the waves' parts are added in order.  All threads; smem is free before and holds the sums, rows D + 4
// apart, behind.  Training step of 2 x 1024 queries of 16 heads against 1024 keys, where each workgroup is alone on its CU and half of them have such
// a row: 118 us without, 131 with (32 rows at a time, one step ahead: 134).
template <int D>
RP_DEV void mean_keys(const CrossArgs& p, const Rows& s, int r0, const int* list, int n, bf16* smem, int tid) {
  constexpr int LD = tile_ld(D), KS = D / 32, DT = D / 16, AHEAD = 3;
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const int lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  bf16* const Ks = smem + w * 32 * LD;
  const bf16* const kb = p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D;
  u32x4 kreg[AHEAD][2][KS];
  auto load_step = [&](u32x4 (&r)[2][KS], int k0) {      // rows past the end read as zero
    const int left = min(32, s.kvlen - k0);
    const rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(kb + (long)k0 * p.ldk), 0, (int)(((long)(left - 1) * p.ldk + D) * 2), 0x00020000);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        r[kt][ks] = __builtin_amdgcn_raw_buffer_load_b128(rk, (int)(((16 * kt + lr) * (int)p.ldk + 32 * ks + 8 * lg) * 2), 0, 0);
  };
  const int k_first = 32 * w;
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (k_first + 128 * i < s.kvlen) load_step(kreg[i], k_first + 128 * i);
  const bool ok = lr < n;
  const int row = r0 + list[ok ? lr : 0];
  const bf16* const qr = p.q + s.offset(row, p.ldq, D) + 8 * lg;
  uint4 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const uint4*>(qr + 32 * ks);
  const float lse2 = ok ? p.lse_in[s.stat(row, p.a)] * 1.4426950408889634f : INFINITY;      // P = 0
  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = k_first; k0 < s.kvlen; k0 += 128 * AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int k = k0 + 128 * i;
      if (k >= s.kvlen) break;
      f32x4 sT[2];      // [16 keys][16 rows]
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) sT[kt] = mfma16(__builtin_bit_cast(uint4, kreg[i][kt][ks]), qf[ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sT[kt]);
      wave_lds_order();      // the last step's K has been read
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) *reinterpret_cast<u32x4*>(Ks + (16 * kt + lr) * LD + 32 * ks + 8 * lg) = kreg[i][kt][ks];
      wave_lds_order();
      if (k + 128 * AHEAD < s.kvlen) load_step(kreg[i], k + 128 * AHEAD);
      const int klim = s.kvlen - 1 - (k + 4 * lg);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) sT[kt][e] = 16 * kt + e > klim ? 0.f : fast_exp2(__builtin_fmaf(sT[kt][e], p.scale_log2e, -lse2));
      uint4 high, low;
      two_parts(sT[0], sT[1], high, low);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint4 a = read_frag_tr<LD>(Ks + tr_base<LD>(lane) + 16 * dt);
        acc[dt] = mfma16(a, high, acc[dt]);
        acc[dt] = mfma16(a, low, acc[dt]);
      }
    }
  }
  float* const sum = reinterpret_cast<float*>(smem) + lr * (D + 4) + 4 * lg;
  for (int u = 0; u < 4; ++u) {
    __syncthreads();
    if (w == u) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x4* const at = reinterpret_cast<f32x4*>(sum + 16 * dt);
        *at = u ? *at + acc[dt] : acc[dt];
      }
    }
  }
  __syncthreads();
}

template <int D, DqPass PASS>
__global__ void __launch_bounds__(256, 2) cross_dq_kernel(const CrossArgs p) {
  constexpr bool SPLIT = PASS == SLICE || PASS == DELTA;
  constexpr int LD = tile_ld(D), KS = D / 32, DT = D / 16, NT = 256, BQ = 128;
  using T64 = Tile64<D, NT>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];   // dq_smem_bytes(D)
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);
  bf16* const Ks = smem;
  bf16* const Vs = smem + 64 * LD;

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nhb = p.kh * p.batch;
  const int rest = (int)blockIdx.x / nhb;
  const int hb = head_at((int)blockIdx.x, rest, nhb);
  const int split = SPLIT ? rest % p.splits : 0;
  const int r0 = (SPLIT ? rest / p.splits : rest) * BQ;
  const Rows s(p, hb);
  if (r0 >= s.valid) {
    if (!SPLIT) zero_rows<D, NT>(p, s, p.dq, p.lddq, nullptr, r0, BQ, tid);
    return;
  }
  const int tiles = (s.kvlen + 63) / 64;
  int j0 = 0, j1 = tiles;
  if (SPLIT) {
    slice_of(tiles, p.splits, split, j0, j1);
    if (j0 >= j1 && split > 0) return;
  }
  if (PASS == DELTA && j0 >= j1) return;      // uniform, before any barrier
  const bool exact_delta = PASS == EXACT || (PASS == WHOLE && s.kvlen <= EXACT_DELTA);
  const KeyTile<D, NT> kt_(p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D, p.ldk, s.kvlen), vt_(p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D, p.ldv, s.kvlen);

  uint4 qf[2][KS], dof[2][KS];     // a lane's rows: column tiles c = 0, 1
  float lse2[2], dl[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int row = r0 + 32 * w + 16 * c + lr;
    const bool ok = row < s.valid;
    const int rc = ok ? row : 0;
    const bf16* const qr = p.q + s.offset(rc, p.ldq, D) + 8 * lg;
    const bf16* const dor = p.dout + s.offset(rc, p.lddo, D) + 8 * lg;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      dof[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      if (ok) {
        qf[c][ks] = *reinterpret_cast<const uint4*>(qr + 32 * ks);
        dof[c][ks] = *reinterpret_cast<const uint4*>(dor + 32 * ks);
      }
    }
    lse2[c] = ok ? p.lse_in[s.stat(rc, p.a)] * 1.4426950408889634f : INFINITY;   // rows past the end get P = 0
    dl[c] = 0.f;
    if (PASS == SLICE) {      // the slices' sums, every fourth by one of the four lanes of a row
      float sum = 0.f, mass = 0.f;
      const int n = slices_used(tiles, p.splits);
#pragma unroll 8
      for (int i = lg; i < n; i += 4) {
        const float2 v = ok ? p.part_ml[((long)i * nhb + hb) * s.total + row] : make_float2(0.f, 0.f);
        sum += v.x;
        mass += v.y;
      }
      sum = column_sum(sum);
      mass = column_sum(mass);
      dl[c] = ok && n ? sum / mass : 0.f;
    }
    if (PASS == WHOLE && !exact_delta) {
      float sum = 0.f;
      if (ok) {
        const bf16* const orow = p.o_in + s.offset(rc, p.ldo, D) + 8 * lg;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint4 u = *reinterpret_cast<const uint4*>(orow + 32 * ks), d = dof[c][ks];
          sum += bf16_lo(u.x) * bf16_lo(d.x) + bf16_hi(u.x) * bf16_hi(d.x) + bf16_lo(u.y) * bf16_lo(d.y) + bf16_hi(u.y) * bf16_hi(d.y) +
                 bf16_lo(u.z) * bf16_lo(d.z) + bf16_hi(u.z) * bf16_hi(d.z) + bf16_lo(u.w) * bf16_lo(d.w) + bf16_hi(u.w) * bf16_hi(d.w);
        }
      }
      dl[c] = column_sum(sum);
    }
  }

  const bf16* const kfrag = Ks + lr * LD + 8 * lg;      // (V lies 64 rows further on)
  const bf16* const ktfrag = Ks + tr_base<LD>(lane);
  uint4 kreg[T64::NREG], vreg[T64::NREG];
  auto load_tiles = [&](int j) {
    kt_.load(kreg, j * 64, tid);
    vt_.load(vreg, j * 64, tid);
  };
  auto store_tiles = [&]() {
    T64::template store<LD>(kreg, Ks, tid);
    T64::template store<LD>(vreg, Vs, tid);
  };
  // scores and dP of 32 keys, transposed: [16 keys][16 rows]
  auto scores = [&](int k2, f32x4 (&sT)[2][2], f32x4 (&dpT)[2][2]) {
    const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
    constexpr int NS = 4 * KS, AHEAD = 4;     // n = (ks * 2 + kt) * 2 + which
    auto sfrag_at = [&](int n) { return *reinterpret_cast<const uint4*>(kfrag + (32 * k2 + 16 * ((n >> 1) & 1) + 64 * (n & 1)) * LD + 32 * (n >> 2)); };
    uint4 ring[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) ring[n] = sfrag_at(n);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const uint4 a = ring[n % AHEAD];
      if (n + AHEAD < NS) ring[n % AHEAD] = sfrag_at(n + AHEAD);
      const int ks = n >> 2, kt = (n >> 1) & 1;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (n & 1) dpT[kt][c] = mfma16(a, dof[c][ks], ks == 0 ? zero4 : dpT[kt][c]);
        else sT[kt][c] = mfma16(a, qf[c][ks], ks == 0 ? zero4 : sT[kt][c]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (PASS == DELTA || exact_delta) {      // uniform over the workgroup
    const int first = PASS == DELTA ? j0 : 0, last = PASS == DELTA ? j1 : tiles;
    float mass[2] = {0.f, 0.f};
    if (first < last) load_tiles(first);
    for (int j = first; j < last; ++j) {
      __syncthreads();
      store_tiles();
      __syncthreads();
      if (j + 1 < last) load_tiles(j + 1);
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        f32x4 sT[2][2], dpT[2][2];
        scores(k2, sT, dpT);
        const int klim = s.kvlen - 1 - (j * 64 + 32 * k2 + 4 * lg);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool in = 16 * kt + e <= klim;
              const float pr = in ? fast_exp2(__builtin_fmaf(sT[kt][c][e], p.scale_log2e, -lse2[c])) : 0.f;
              mass[c] += pr;
              dl[c] += in ? pr * dpT[kt][c][e] : 0.f;
            }
      }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = r0 + 32 * w + 16 * c + lr;
      dl[c] = column_sum(dl[c]);
      mass[c] = column_sum(mass[c]);
      if constexpr (PASS == DELTA) {
        if (lg == 0 && row < s.valid) p.part_ml[((long)split * nhb + hb) * s.total + row] = make_float2(dl[c], mass[c]);
      } else {
        dl[c] = row < s.valid && tiles > 0 ? dl[c] / mass[c] : 0.f;
      }
    }
    if (PASS == DELTA) return;
    __syncthreads();      // the tiles are stored anew below
  }
  f32x4 dqacc[DT][2];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dqacc[dt][0] = dqacc[dt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  float row_sum[2] = {0.f, 0.f}, row_size[2] = {0.f, 0.f};      // of dS: its sum, and that of its absolute values
  if (j0 < j1) load_tiles(j1 - 1);
  for (int j = j1 - 1; j >= j0; --j) {      // the first tile last: it is full, and its keys are averaged below
    __syncthreads();
    store_tiles();
    __syncthreads();
    if (j > j0) load_tiles(j - 1);
    const bool need_mask = j * 64 + 64 > s.kvlen;
    // the two 32-key halves of the tile one after the other: half as many score registers live at a time
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      f32x4 sT[2][2], dpT[2][2];
      scores(k2, sT, dpT);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sT[kt][c][e] = fast_exp2(__builtin_fmaf(sT[kt][c][e], p.scale_log2e, -lse2[c])) * (dpT[kt][c][e] - dl[c]);   // dS^T
      if (need_mask) {
        const int klim = s.kvlen - 1 - (j * 64 + 32 * k2 + 4 * lg);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) sT[kt][c][e] = 16 * kt + e > klim ? 0.f : sT[kt][c][e];
      }
      if (PASS == WHOLE) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              row_sum[c] += sT[kt][c][e];
              row_size[c] += fabsf(sT[kt][c][e]);
            }
      }
      constexpr int AHEAD = 2;      // K^T fragments requested that many pairs of products early
      uint4 df[2], low[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) two_parts(sT[0][c], sT[1][c], df[c], low[c]);
      auto ufrag_at = [&](int n) { return read_frag_tr<LD>(ktfrag + 32 * k2 * LD + 16 * n); };
      uint4 uring[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) uring[n] = ufrag_at(n);
#pragma unroll
      for (int n = 0; n < DT; ++n) {
        const uint4 a = uring[n % AHEAD];
        if (n + AHEAD < DT) uring[n % AHEAD] = ufrag_at(n + AHEAD);
#pragma unroll
        for (int c = 0; c < 2; ++c) dqacc[n][c] = mfma16(a, df[c], dqacc[n][c]);
#pragma unroll
        for (int c = 0; c < 2; ++c) dqacc[n][c] = mfma16(a, low[c], dqacc[n][c]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // the rows of dS sum up to zero: what they do sum up to is what delta was off by, and dq by that times sum P K
  if constexpr (PASS == WHOLE) {
    float off[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      off[c] = column_sum(row_sum[c]);
      dl[c] += off[c];
    }
    if (!exact_delta) {
      int* const marks = reinterpret_cast<int*>(dyn_smem + dq_tile_bytes(D));      // the four waves' column tiles: a bit a row
      int* const list = marks + 8;                                                 // the rows that are off, in order
      bool far[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        far[c] = fabsf(off[c]) > FAR * column_sum(row_size[c]);
        const int mark = (int)(__builtin_amdgcn_ballot_w64(far[c]) & 0xffffull);      // (the four lanes of a row agree)
        if (lane == 0) marks[2 * w + c] = mark;
      }
      __syncthreads();      // (the last tile has been read as well)
      // the other rows: the mean of 64 keys in the place of sum P K, which is what all keys share of it
      float* const mean = reinterpret_cast<float*>(Vs);      // [NT / D][D]
      {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 64 * D / NT; ++i) sum += (float)Ks[((tid / D) * (64 * D / NT) + i) * LD + tid % D];
        mean[tid] = sum * (1.f / 64.f);
      }
      __syncthreads();
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x4 m = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NT / D; ++i) m += *reinterpret_cast<const f32x4*>(mean + i * D + 16 * dt + 4 * lg);
#pragma unroll
        for (int c = 0; c < 2; ++c) dqacc[dt][c] -= (far[c] ? 0.f : off[c]) * m;
      }
      int count = 0, at[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = __popc(marks[i]);
        at[0] += i < 2 * w ? n : 0;
        at[1] += i < 2 * w + 1 ? n : 0;
        count += n;
      }
      count = __builtin_amdgcn_readfirstlane(count);
      if (count) {      // uniform over the workgroup
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          at[c] += __popc(marks[2 * w + c] & ((1 << lr) - 1));
          if (lg == 0 && far[c]) list[at[c]] = 32 * w + 16 * c + lr;
        }
        __syncthreads();
        for (int first = 0; first < count; first += 16) {
          mean_keys<D>(p, s, r0, list + first, min(16, count - first), smem, tid);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int i = at[c] - first;
            if (far[c] && i >= 0 && i < 16) {
              const float* const sum = reinterpret_cast<const float*>(smem) + i * (D + 4) + 4 * lg;
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) dqacc[dt][c] -= off[c] * *reinterpret_cast<const f32x4*>(sum + 16 * dt);
            }
          }
          __syncthreads();
        }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int row = r0 + 32 * w + 16 * c + lr;
    if (lg == 0 && row < s.valid && (!SPLIT || split == 0)) p.delta[s.stat(row, p.a)] = dl[c];
  }
  if constexpr (SPLIT) {
    if (j0 >= j1) return;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = r0 + 32 * w + 16 * c + lr;
      if (row < s.valid) {
        float* const out = p.part + (((long)split * nhb + hb) * s.total + row) * D + 4 * lg;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          *reinterpret_cast<float4*>(out + 16 * dt) = make_float4(dqacc[dt][c][0], dqacc[dt][c][1], dqacc[dt][c][2], dqacc[dt][c][3]);
      }
    }
  } else {
    __syncthreads();
    bf16* const stage = smem + w * 32 * (D + 8);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        *reinterpret_cast<uint2*>(stage + (16 * c + lr) * (D + 8) + 16 * dt + 4 * lg) =
            make_uint2(pack_bf16x2(dqacc[dt][c][0] * p.scale, dqacc[dt][c][1] * p.scale), pack_bf16x2(dqacc[dt][c][2] * p.scale, dqacc[dt][c][3] * p.scale));
    __syncthreads();
#pragma unroll
    for (int it = 0; it < (32 * (D / 8)) / 64; ++it) {
      const int idx = it * 64 + lane, rr = idx / (D / 8), ch = idx % (D / 8), r = r0 + 32 * w + rr;
      if (r < s.total)
        *reinterpret_cast<uint4*>(p.dq + s.offset(r, p.lddq, D) + ch * 8) =
            r < s.valid ? *reinterpret_cast<const uint4*>(stage + rr * (D + 8) + ch * 8) : make_uint4(0u, 0u, 0u, 0u);
    }
  }
}

// ================================================================================================ dK, dV
// A thread's share of the 64-row tiles of q and dO: which head and query each of its 16-byte pieces belongs to.  Rows past the last query
// read row 0 again (their P is made zero, see row_start).
template <int D, int NT>
struct RowTile {
  static constexpr int CH = D / 8, NREG = 64 * CH / NT;
  int h[NREG], q[NREG];
  int qlen, grp, step_h, step_q;
  RP_DEV void start(const Rows& s, int row0, int tid) {
    qlen = max(s.qlen, 1);
    grp = s.grp;
    step_h = 64 / qlen;
    step_q = 64 - step_h * qlen;
#pragma unroll
    for (int it = 0; it < NREG; ++it) {
      const int r = row0 + (it * NT + tid) / CH;
      h[it] = r / qlen;
      q[it] = r - h[it] * qlen;
    }
  }
  // base: the group's first head of the sequence's first query
  RP_DEV void load(uint4 (&r)[NREG], const bf16* base, long ld, int tid) const {
#pragma unroll
    for (int it = 0; it < NREG; ++it) {
      const bool in = h[it] < grp;
      typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));      // (copied as a struct, the pieces would live in scratch memory)
      const u32x4 v = *reinterpret_cast<const u32x4*>(base + (long)(in ? q[it] : 0) * ld + (in ? h[it] : 0) * D + ((it * NT + tid) % CH) * 8);
      r[it] = make_uint4(v.x, v.y, v.z, v.w);
    }
  }
  RP_DEV void next() {
#pragma unroll
    for (int it = 0; it < NREG; ++it) {
      h[it] += step_h;
      q[it] += step_q;
      if (q[it] >= qlen) { q[it] -= qlen; ++h[it]; }
    }
  }
};

// What the products start from for a row (wave 0: -lse / scale, wave 1: -delta), so that they come out as q.k - lse / scale and
// dO.v - delta; rows past the end get P = exp(-inf) = 0.
RP_DEV float row_start(float raw, int wave, bool in, float inv_scale) { return wave == 0 ? (in ? -raw * inv_scale : -INFINITY) : (in ? -raw : 0.f); }

// lse and delta of a 64-row tile, a row per lane of waves 0 and 1.  The load is only issued here; row_start comes a tile later.
struct RowStat {
  int h, q, qlen, grp, step_h, step_q, seq_q;
  const float* base;
  RP_DEV void start(const CrossArgs& p, const Rows& s, int row0, int lane, int wave) {
    qlen = max(s.qlen, 1);
    grp = s.grp;
    seq_q = s.seq_q;
    step_h = 64 / qlen;
    step_q = 64 - step_h * qlen;
    const int r = row0 + lane;
    h = r / qlen;
    q = r - h * qlen;
    base = (wave == 0 ? p.lse_in : p.delta) + ((long)s.b * p.a + s.g * grp) * seq_q;
  }
  RP_DEV float load() {      // and on to the next tile
    const bool in = h < grp;
    const float v = base[in ? (long)h * seq_q + q : 0];
    h += step_h;
    q += step_q;
    if (q >= qlen) { q -= qlen; ++h; }
    return v;
  }
};

// P = exp(s) and dS = P dP in place.
RP_DEV void probabilities(f32x4 (&s)[2][2], f32x4 (&dp)[2][2], float scale_log2e) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int qt = 0; qt < 2; ++qt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float pr = fast_exp2(s[qt][c][e] * scale_log2e);
        s[qt][c][e] = pr;
        dp[qt][c][e] = pr * dp[qt][c][e];
      }
}

// Zeros for the keys of a 128-key tile that are behind the sequence.
template <int D, int NT>
RP_DEV void zero_keys(const CrossArgs& p, const Rows& s, int kv0, int tid) {
  constexpr int CH = D / 8;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  for (int i = tid; i < 128 * CH; i += NT) {
    const int key = kv0 + i / CH;
    if (key < s.kvlen || key >= p.seq_kv) continue;
    const long t = (long)s.b * p.seq_kv + key;
    *reinterpret_cast<uint4*>(p.dk + t * p.lddk + s.g * D + (i % CH) * 8) = zero;
    *reinterpret_cast<uint4*>(p.dv + t * p.lddv + s.g * D + (i % CH) * 8) = zero;
  }
}

// The keys of a workgroup do not mix: a column of the score tiles is a key's own, so keys behind the sequence need no mask here; what comes out for
// them is not stored.
template <int D>
__global__ void __launch_bounds__(256) cross_dkv_kernel(const CrossArgs p) {
  constexpr int LD = tile_ld(D), KS = D / 32, DT = D / 16;
  using T64 = Tile64<D, 256>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);             // Q | dO | what the rows start from
  bf16* const Qs = smem;
  bf16* const dOs = smem + 64 * LD;
  float* const stat = reinterpret_cast<float*>(smem + 2 * 64 * LD);     // [2][64]

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nhb = p.kh * p.batch;
  const int rest = (int)blockIdx.x / nhb;
  const int hb = head_at((int)blockIdx.x, rest, nhb);
  const int split = rest % p.splits, kv0 = (rest / p.splits) * 128, kw0 = kv0 + 32 * w;
  const Rows s(p, hb);
  if (p.splits == 1) zero_keys<D, 256>(p, s, kv0, tid);
  if (kv0 >= s.kvlen) return;      // uniform, before any barrier
  int u0, u1;
  slice_of((s.valid + 63) / 64, p.splits, split, u0, u1);
  if (p.splits > 1 && u0 >= u1) return;
  const int kpos[2] = {kw0 + lr, kw0 + 16 + lr};
  const bf16* const kb = p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D;
  const bf16* const vb = p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D;

  uint4 kf[2][KS], vf[2][KS];
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      vf[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      if (kpos[c] < s.kvlen) {
        kf[c][ks] = *reinterpret_cast<const uint4*>(kb + (long)kpos[c] * p.ldk + 32 * ks + 8 * lg);
        vf[c][ks] = *reinterpret_cast<const uint4*>(vb + (long)kpos[c] * p.ldv + 32 * ks + 8 * lg);
      }
    }
  f32x4 dkacc[DT][2], dvacc[DT][2];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dkacc[dt][0] = dkacc[dt][1] = dvacc[dt][0] = dvacc[dt][1] = f32x4{0.f, 0.f, 0.f, 0.f};

  const bf16* qfrag = Qs + lr * LD + 8 * lg;
  const bf16* dofrag = dOs + lr * LD + 8 * lg;
  const bf16* qtfrag = Qs + tr_base<LD>(lane);
  const bf16* dotfrag = dOs + tr_base<LD>(lane);

  const bf16* const qb = p.q + (long)s.b * p.seq_q * p.ldq + (long)s.g * s.grp * D;
  const bf16* const dob = p.dout + (long)s.b * p.seq_q * p.lddo + (long)s.g * s.grp * D;
  uint4 qreg[T64::NREG], doreg[T64::NREG];
  float st_reg = 0.f;
  RowTile<D, 256> rows;
  RowStat rstat;
  rows.start(s, u0 * 64, tid);
  rstat.start(p, s, u0 * 64, lane, w);
  auto prefetch = [&]() {
    rows.load(qreg, qb, p.ldq, tid);
    rows.load(doreg, dob, p.lddo, tid);
    rows.next();
    if (w < 2) st_reg = rstat.load();
  };
  if (u0 < u1) prefetch();
  for (int u = u0; u < u1; ++u) {
    __syncthreads();
    T64::template store<LD>(qreg, Qs, tid);
    T64::template store<LD>(doreg, dOs, tid);
    if (w < 2) stat[64 * w + lane] = row_start(st_reg, w, u * 64 + lane < s.valid, p.inv_scale);
    __syncthreads();
    if (u + 1 < u1) prefetch();
    // the two 32-row halves of the tile one after the other: half as many score registers live at a time
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      f32x4 sc[2][2], dp[2][2], s0[2], dp0[2];     // [16 rows][16 keys]; what they start from
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        s0[qt] = *reinterpret_cast<const f32x4*>(stat + 32 * t2 + 16 * qt + 4 * lg);
        dp0[qt] = *reinterpret_cast<const f32x4*>(stat + 64 + 32 * t2 + 16 * qt + 4 * lg);
      }
      constexpr int AHEAD = 4;
      {
        constexpr int NS = 4 * KS;     // n = (ks * 2 + qt) * 2 + which
        auto sfrag_at = [&](int n) { return *reinterpret_cast<const uint4*>(((n & 1) ? dofrag : qfrag) + (32 * t2 + 16 * ((n >> 1) & 1)) * LD + 32 * (n >> 2)); };
        uint4 ring[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) ring[n] = sfrag_at(n);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          const uint4 a = ring[n % AHEAD];
          if (n + AHEAD < NS) ring[n % AHEAD] = sfrag_at(n + AHEAD);
          const int ks = n >> 2, qt = (n >> 1) & 1;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            if (n & 1) dp[qt][c] = mfma16(a, vf[c][ks], ks == 0 ? dp0[qt] : dp[qt][c]);
            else sc[qt][c] = mfma16(a, kf[c][ks], ks == 0 ? s0[qt] : sc[qt][c]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      constexpr int NU = 2 * DT;
      auto ufrag_at = [&](int n) { return read_frag_tr<LD>(((n & 1) ? qtfrag : dotfrag) + 32 * t2 * LD + 16 * (n >> 1)); };
      uint4 uring[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) uring[n] = ufrag_at(n);
      __builtin_amdgcn_sched_barrier(0);
      probabilities(sc, dp, p.scale_log2e);
      {
        const uint4 pfg[2] = {pack_frag(sc[0][0], sc[1][0]), pack_frag(sc[0][1], sc[1][1])};
        const uint4 dfg[2] = {pack_frag(dp[0][0], dp[1][0]), pack_frag(dp[0][1], dp[1][1])};
#pragma unroll
        for (int n = 0; n < NU; ++n) {
          const uint4 a = uring[n % AHEAD];
          if (n + AHEAD < NU) uring[n % AHEAD] = ufrag_at(n + AHEAD);
          const int dt = n >> 1;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            if (n & 1) dkacc[dt][c] = mfma16(a, dfg[c], dkacc[dt][c]);
            else dvacc[dt][c] = mfma16(a, pfg[c], dvacc[dt][c]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  __syncthreads();
  const long tok0 = (long)s.b * p.seq_kv;
  if (p.splits == 1) {
    store_acc_T<D>(dkacc, p.scale, smem + w * 32 * (D + 8), p.dk + tok0 * p.lddk + s.g * D, p.lddk, kw0, s.kvlen, lane);
    store_acc_T<D>(dvacc, 1.f, smem + w * 32 * (D + 8), p.dv + tok0 * p.lddv + s.g * D, p.lddv, kw0, s.kvlen, lane);
  } else {
    float* const stage = reinterpret_cast<float*>(smem) + w * 32 * (D + 4);
    const long ldp = (long)p.kh * D, each = (long)p.batch * p.seq_kv * ldp;
    float* const out = p.part + split * each + tok0 * ldp + s.g * D;
    store_acc_T_f32<D>(dkacc, p.scale, stage, out, ldp, kw0, s.kvlen, lane);
    store_acc_T_f32<D>(dvacc, 1.f, stage, out + p.splits * each, ldp, kw0, s.kvlen, lane);
  }
}

// Two waves per SIMD at d = 128 (see attn_bwd_dkv_pair_kernel in attention.hip): the 32 keys of a pair of waves are shared, wave h of it keeps
// the accumulators of half h of the head dimension, makes the scores of rows 32 h .. of each tile and hands P and dS to its partner through LDS.
template <int D>
__global__ void __launch_bounds__(512) cross_dkv_pair_kernel(const CrossArgs p) {
  constexpr int LD = tile_ld(D), KS = D / 32, DH = D / 32;
  using T64 = Tile64<D, 512>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);             // two sets (tile parity) of Q | dO, then the exchange
  constexpr int TSET = 2 * 64 * LD;
  uint4* const exch = reinterpret_cast<uint4*>(smem + 2 * TSET);    // [8 waves][4 fragments][64 lanes]
  float* const stat = reinterpret_cast<float*>(exch + 8 * 4 * 64);  // [2 sets][2][64]

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w8 = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = w8 >> 1, h = w8 & 1;
  const int nhb = p.kh * p.batch;
  const int rest = (int)blockIdx.x / nhb;
  const int hb = head_at((int)blockIdx.x, rest, nhb);
  const int split = rest % p.splits, kv0 = (rest / p.splits) * 128, kw0 = kv0 + 32 * w;
  const Rows s(p, hb);
  if (p.splits == 1) zero_keys<D, 512>(p, s, kv0, tid);
  if (kv0 >= s.kvlen) return;      // uniform, before any barrier
  int u0, u1;
  slice_of((s.valid + 63) / 64, p.splits, split, u0, u1);
  if (p.splits > 1 && u0 >= u1) return;
  const int kpos[2] = {kw0 + lr, kw0 + 16 + lr};
  const bf16* const kb = p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D;
  const bf16* const vb = p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D;

  uint4 kf[2][KS], vf[2][KS];
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      vf[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      if (kpos[c] < s.kvlen) {
        kf[c][ks] = *reinterpret_cast<const uint4*>(kb + (long)kpos[c] * p.ldk + 32 * ks + 8 * lg);
        vf[c][ks] = *reinterpret_cast<const uint4*>(vb + (long)kpos[c] * p.ldv + 32 * ks + 8 * lg);
      }
    }
  f32x4 dkacc[DH][2], dvacc[DH][2];
#pragma unroll
  for (int dt = 0; dt < DH; ++dt) dkacc[dt][0] = dkacc[dt][1] = dvacc[dt][0] = dvacc[dt][1] = f32x4{0.f, 0.f, 0.f, 0.f};

  const bf16* qfrag = smem + (32 * h + lr) * LD + 8 * lg;           // this wave's 32 rows of a tile
  const bf16* dofrag = qfrag + 64 * LD;
  const bf16* qtfrag = smem + tr_base<LD>(lane) + 16 * DH * h;      // its half of the head dimension
  const bf16* dotfrag = qtfrag + 64 * LD;
  uint4* const ex_mine = exch + (w8 * 4) * 64 + lane;
  const uint4* const ex_theirs = exch + ((w8 ^ 1) * 4) * 64 + lane;

  const bf16* const qb = p.q + (long)s.b * p.seq_q * p.ldq + (long)s.g * s.grp * D;
  const bf16* const dob = p.dout + (long)s.b * p.seq_q * p.lddo + (long)s.g * s.grp * D;
  uint4 qreg[T64::NREG], doreg[T64::NREG];
  float st_reg = 0.f;
  RowTile<D, 512> rows;
  RowStat rstat;
  rows.start(s, u0 * 64, tid);
  rstat.start(p, s, u0 * 64, lane, w8);
  auto prefetch = [&]() {
    rows.load(qreg, qb, p.ldq, tid);
    rows.load(doreg, dob, p.lddo, tid);
    rows.next();
    if (w8 < 2) st_reg = rstat.load();
  };
  if (u0 < u1) prefetch();

  constexpr int AHEAD = 2;     // two waves per SIMD cover each other's LDS latency: a short ring is enough
  auto update_half = [&](int set, int t2, const uint4 (&pf)[2], const uint4 (&df)[2]) {
    constexpr int NU = 2 * DH;     // n = dt * 2 + which
    auto ufrag_at = [&](int n) { return read_frag_tr<LD>(((n & 1) ? qtfrag : dotfrag) + set * TSET + 32 * t2 * LD + 16 * (n >> 1)); };
    uint4 uring[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) uring[n] = ufrag_at(n);
    MFMA_PHASE_BEGIN();
#pragma unroll
    for (int n = 0; n < NU; ++n) {
      const uint4 a = uring[n % AHEAD];
      if (n + AHEAD < NU) uring[n % AHEAD] = ufrag_at(n + AHEAD);
      const int dt = n >> 1;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (n & 1) dkacc[dt][c] = mfma16(a, df[c], dkacc[dt][c]);
        else dvacc[dt][c] = mfma16(a, pf[c], dvacc[dt][c]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    MFMA_PHASE_END();
  };
  // Two barriers per tile.  After the first one every wave is done with the previous tile's scores and has published its fragments: the
  // new tile is stored (into the other set) while the accumulators take the partner's half of the PREVIOUS tile.
  auto partner_update = [&](int prev) {
    const uint4 ppf[2] = {ex_theirs[0], ex_theirs[64]};
    const uint4 pdf[2] = {ex_theirs[128], ex_theirs[192]};
    update_half(prev & 1, h ^ 1, ppf, pdf);
  };
  const int n_tiles = u1 - u0;
  for (int i = 0; i < n_tiles; ++i) {
    __syncthreads();
    bf16* const q_set = smem + (i & 1) * TSET;
    T64::template store<LD>(qreg, q_set, tid);
    T64::template store<LD>(doreg, q_set + 64 * LD, tid);
    if (w8 < 2) stat[128 * (i & 1) + 64 * w8 + lane] = row_start(st_reg, w8, (u0 + i) * 64 + lane < s.valid, p.inv_scale);
    if (i > 0) partner_update(i - 1);
    __syncthreads();
    if (i + 1 < n_tiles) prefetch();
    f32x4 sc[2][2], dp[2][2], s0[2], dp0[2];      // [16 rows][16 keys]; what they start from
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      s0[qt] = *reinterpret_cast<const f32x4*>(stat + 128 * (i & 1) + 32 * h + 16 * qt + 4 * lg);
      dp0[qt] = *reinterpret_cast<const f32x4*>(stat + 128 * (i & 1) + 64 + 32 * h + 16 * qt + 4 * lg);
    }
    {
      constexpr int NS = 4 * KS;     // n = (ks * 2 + qt) * 2 + which
      auto sfrag_at = [&](int n) { return *reinterpret_cast<const uint4*>(((n & 1) ? dofrag : qfrag) + (i & 1) * TSET + 16 * ((n >> 1) & 1) * LD + 32 * (n >> 2)); };
      uint4 ring[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) ring[n] = sfrag_at(n);
      MFMA_PHASE_BEGIN();
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const uint4 a = ring[n % AHEAD];
        if (n + AHEAD < NS) ring[n % AHEAD] = sfrag_at(n + AHEAD);
        const int ks = n >> 2, qt = (n >> 1) & 1;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if (n & 1) dp[qt][c] = mfma16(a, vf[c][ks], ks == 0 ? dp0[qt] : dp[qt][c]);
          else sc[qt][c] = mfma16(a, kf[c][ks], ks == 0 ? s0[qt] : sc[qt][c]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      MFMA_PHASE_END();
    }
    probabilities(sc, dp, p.scale_log2e);
    const uint4 pfg[2] = {pack_frag(sc[0][0], sc[1][0]), pack_frag(sc[0][1], sc[1][1])};
    const uint4 dfg[2] = {pack_frag(dp[0][0], dp[1][0]), pack_frag(dp[0][1], dp[1][1])};
    // the partner read last tile's fragments before the barrier above: the slots are free
    ex_mine[0] = pfg[0]; ex_mine[64] = pfg[1]; ex_mine[128] = dfg[0]; ex_mine[192] = dfg[1];
    update_half(i & 1, h, pfg, dfg);
  }
  __syncthreads();
  if (n_tiles > 0) partner_update(n_tiles - 1);
  __syncthreads();
  const long tok0 = (long)s.b * p.seq_kv;
  const int d0 = s.g * D + h * (D / 2);
  if (p.splits == 1) {
    bf16* const stage = smem + w8 * 32 * (D / 2 + 8);
    store_acc_T<D / 2>(dkacc, p.scale, stage, p.dk + tok0 * p.lddk + d0, p.lddk, kw0, s.kvlen, lane);
    store_acc_T<D / 2>(dvacc, 1.f, stage, p.dv + tok0 * p.lddv + d0, p.lddv, kw0, s.kvlen, lane);
  } else {
    float* const stage = reinterpret_cast<float*>(smem) + w8 * 32 * (D / 2 + 4);
    const long ldp = (long)p.kh * D, each = (long)p.batch * p.seq_kv * ldp;
    float* const out = p.part + split * each + tok0 * ldp + d0;
    store_acc_T_f32<D / 2>(dkacc, p.scale, stage, out, ldp, kw0, s.kvlen, lane);
    store_acc_T_f32<D / 2>(dvacc, 1.f, stage, out + p.splits * each, ldp, kw0, s.kvlen, lane);
  }
}

// dk, dv = the sum of a key's slices; zero behind the sequence.  A "row" is a key head of dk or dv.
template <int D, int G>
__global__ void __launch_bounds__(256) cross_key_join_kernel(const CrossArgs p) {
  constexpr int CH = D / 8, RPB = 256 / (CH * G);
  __shared__ float red[CH * G > 64 ? 4 * CH * 8 : 1];
  const int tid = threadIdx.x, ch = tid % CH, grp = tid / CH % G;
  const long T = (long)p.batch * p.seq_kv, rows = T * p.kh;
  const long item = (long)blockIdx.x * RPB + tid / (CH * G);
  const bool in = item < 2 * rows, is_v = item >= rows;
  const long kv = !in ? 0 : is_v ? item - rows : item;
  const long t = kv / p.kh;
  const int g = (int)(kv - t * p.kh), b = (int)(t / p.seq_kv), key = (int)(t - (long)b * p.seq_kv);
  const Rows s(p, b * p.kh);
  const int n = in && key < s.kvlen ? slices_used((s.valid + 63) / 64, p.splits) : 0;
  const float* const src = p.part + (is_v ? p.splits * rows * D : 0) + kv * D + ch * 8;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll 4
  for (int i = grp; i < n; i += G) add_times(acc, src + i * rows * D, 1.f);
  const bool mine = add_groups<CH, G, 8>(acc, red);
  if (in && mine) *reinterpret_cast<uint4*>((is_v ? p.dv + t * p.lddv : p.dk + t * p.lddk) + g * D + ch * 8) = pack_times(acc, 1.f);
}

// operand tiles, or the epilogue's staging of every wave's 32 x d block, whichever is larger
constexpr int max_i(int a, int b) { return a > b ? a : b; }
constexpr int fwd_smem_bytes(int d) { return max_i(64 * (d + 8) + 64 * (d + 32), 128 * (d + 8)) * 2; }
constexpr int step_smem_bytes(int d, int nc, int nw) { return nw * max_i(32 * tile_ld(d) * 2, 16 * nc * (2 + d + 4) * 4); }
constexpr int dq_smem_bytes(int d) { return max_i(dq_tile_bytes(d), 128 * (d + 8) * 2) + (8 + 128) * 4; }
constexpr int dkv_smem_bytes(int d) { return max_i(2 * 64 * tile_ld(d) * 2 + 512, 4 * 32 * (d + 4) * 4); }
constexpr int dkv_pair_smem_bytes(int d) { return 2 * (2 * 64 * tile_ld(d)) * 2 + 8 * 4 * 64 * 16 + 1024; }

template <typename K, typename... More>
hipError_t launch(K kern, int grid, int threads, int smem, hipStream_t st, const CrossArgs& p, More... more) {
  // (a host-side table entry, not a stream operation: allowed while a graph is captured)
  if (smem > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
  }
  RP_LAUNCH(kern, dim3(grid), dim3(threads), smem, st, p, more...);
  return hipGetLastError();
}

// Slices of a loop over `steps` tiles that would run in `groups` workgroups, at most so many that they make `want`, and as the scratch holds: the
// number that saves most, if any.  A tile of a workgroup that has few others beside it takes `tile_us` (its chain of loads, products and
// exponentials); joining costs a launch, about 5 us, and the slices' way to memory and back at 5 TB/s.  Measured with a slice of at least two |
// four | eight tiles (forward and backward of a training step, us): 102 queries x 16 heads against 1711 keys 48.3 | 52.0 | 58.8; 8 x 15 x 4 heads against
// 352 32.5 | 36.1 | 36.1; 8 x 47 x 64 heads of 64 against up to 538 60.3 | 60.3 | 47.7; this rule takes the best of each.
int splits_for(long groups, long want, int steps, double tile_us, size_t bytes_each, size_t scratch_bytes) {
  if (groups < 1) return 1;
  long most = want / groups;
  if (most > steps) most = steps;
  if (bytes_each && most > (long)(scratch_bytes / bytes_each)) most = (long)(scratch_bytes / bytes_each);
  int best = 1;
  double saved = 0.0;
  for (int n = 2; n <= most; ++n) {
    const double s = (steps - (steps + n - 1) / n) * tile_us - 5.0 - 2.0 * n * (double)bytes_each / 5.0e6;
    if (s > saved) { saved = s; best = n; }
  }
  return best;
}
int ceil_div(long a, int b) { return (int)((a + b - 1) / b); }
long row_count(const CrossArgs& p) { return (long)(p.a / p.kh) * p.seq_q; }
size_t row_part_bytes(const CrossArgs& p, int d) { return (size_t)p.kh * p.batch * row_count(p) * (d + 2) * 4; }      // o or dq, and (m, l)
size_t key_part_bytes(const CrossArgs& p, int d) { return (size_t)2 * p.batch * p.seq_kv * p.kh * d * 4; }
// Forward and dQ: two workgroups of 128 rows per CU.
int row_splits(const CrossArgs& p, int d, size_t bytes) {
  return splits_for((long)ceil_div(row_count(p), 128) * p.kh * p.batch, 512, ceil_div(p.seq_kv, 64), 1.4, row_part_bytes(p, d), bytes);
}
// Few rows: slices for two workgroups of four waves per CU, with a 32-key step for each wave at least -- or one workgroup of eight waves, without slices,
// where its waves are through with their steps (2.1 us each, one after the other: a CU fetches 60 GB/s) before the slices would have been joined (a
// second launch, 3 us).  One token against d = 128, us, slices | eight waves: 8 sequences of 1500 keys, 8 key heads 14.6 | 17.2, 1 of 700 9.0 | 10.0,
// 32 of 1000 30.1 | 25.6; 2 of 300, 16 key heads of 64 8.1 | 5.7.
bool few_rows(const CrossArgs& p) { return row_count(p) <= 32; }
int step_splits(const CrossArgs& p, int d, size_t bytes) {
  const long nhb = (long)p.kh * p.batch;
  const size_t each = row_part_bytes(p, d);
  const int steps = ceil_div(p.seq_kv, 32);
  long n = nhb ? 512 / nhb : 1;
  if (n > ceil_div(steps, 4)) n = ceil_div(steps, 4);
  if (each && n > (long)(bytes / each)) n = (long)(bytes / each);
  if (n < 2 || ceil_div(steps, 8) * 2.1 <= ceil_div(ceil_div(steps, (int)n), 4) * 2.1 + 3.0) return 1;
  return (int)n;
}
template <int D, int NC>
hipError_t launch_step(hipStream_t st, const CrossArgs& p) {
  const int nhb = p.kh * p.batch;
  if (p.splits > 1) return launch(cross_step_kernel<D, NC, 4, true>, nhb * p.splits, 256, step_smem_bytes(D, NC, 4), st, p);
  if (p.seq_kv > 128 && nhb < 512) return launch(cross_step_kernel<D, NC, 8, false>, nhb, 512, step_smem_bytes(D, NC, 8), st, p);
  return launch(cross_step_kernel<D, NC, 4, false>, nhb, 256, step_smem_bytes(D, NC, 4), st, p);
}
// dK, dV: the kernel at d = 128 has a CU to itself; at d = 64 two share one, and a third takes the place of those that end early
int key_splits(const CrossArgs& p, int d, size_t bytes) {
  return splits_for((long)ceil_div(p.seq_kv, 128) * p.kh * p.batch, d == 128 ? 256 : 768, ceil_div(row_count(p), 64), d == 128 ? 2.2 : 1.6, key_part_bytes(p, d), bytes);
}

// Threads that share a row of n slices.
int join_groups(int n) { return n < 6 ? 1 : n < 24 ? 4 : 16; }
template <int D, bool DQ>
hipError_t join_rows(hipStream_t st, const CrossArgs& p, int unit) {
  const int g = join_groups(p.splits), grid = ceil_div(row_count(p) * p.kh * p.batch, 256 / (D / 8 * g));
  if (g == 1) return launch(cross_row_join_kernel<D, 1, DQ>, grid, 256, 0, st, p, unit);
  if (g == 4) return launch(cross_row_join_kernel<D, 4, DQ>, grid, 256, 0, st, p, unit);
  return launch(cross_row_join_kernel<D, 16, DQ>, grid, 256, 0, st, p, unit);
}
template <int D>
hipError_t join_keys(hipStream_t st, const CrossArgs& p) {
  const int g = join_groups(p.splits), grid = ceil_div((long)2 * p.batch * p.seq_kv * p.kh, 256 / (D / 8 * g));
  if (g == 1) return launch(cross_key_join_kernel<D, 1>, grid, 256, 0, st, p);
  if (g == 4) return launch(cross_key_join_kernel<D, 4>, grid, 256, 0, st, p);
  return launch(cross_key_join_kernel<D, 16>, grid, 256, 0, st, p);
}

template <int D>
hipError_t fwd(hipStream_t st, CrossArgs p, void* scratch, size_t bytes) {
  const int nhb = p.kh * p.batch;
  const long rows = row_count(p);
  const bool few = few_rows(p);
  p.splits = few ? step_splits(p, D, bytes) : row_splits(p, D, bytes);
  p.part = static_cast<float*>(scratch);
  p.part_ml = reinterpret_cast<float2*>(p.part + (size_t)p.splits * nhb * rows * D);
  hipError_t e = hipSuccess;
  if (few) {
    e = rows <= 16 ? launch_step<D, 1>(st, p) : launch_step<D, 2>(st, p);
  } else if (p.splits > 1) {
    e = launch(cross_fwd_kernel<D, true>, ceil_div(rows, 128) * nhb * p.splits, 256, fwd_smem_bytes(D), st, p);
  }
  if (p.splits > 1 && e == hipSuccess) e = join_rows<D, false>(st, p, few ? 32 : 64);
  if (few || p.splits > 1) return e;
  return launch(cross_fwd_kernel<D, false>, ceil_div(rows, 128) * nhb, 256, fwd_smem_bytes(D), st, p);
}

template <int D>
hipError_t bwd(hipStream_t st, CrossArgs p, void* scratch, size_t bytes) {
  const int nhb = p.kh * p.batch;
  const long rows = row_count(p);
  p.part = static_cast<float*>(scratch);
  // dQ first: it works out delta, which dK/dV reads
  p.splits = row_splits(p, D, bytes);
  p.part_ml = reinterpret_cast<float2*>(p.part + (size_t)p.splits * nhb * rows * D);
  hipError_t e = hipSuccess;
  if (rows == 0) {
    // no queries: dk and dv are zero
  } else if (p.splits > 1) {
    const int grid = ceil_div(rows, 128) * nhb * p.splits;
    e = launch(cross_dq_kernel<D, DELTA>, grid, 256, dq_smem_bytes(D), st, p);
    if (e == hipSuccess) e = launch(cross_dq_kernel<D, SLICE>, grid, 256, dq_smem_bytes(D), st, p);
    if (e == hipSuccess) e = join_rows<D, true>(st, p, 64);
  } else {
    const int grid = ceil_div(rows, 128) * nhb;
    e = p.seq_kv <= EXACT_DELTA ? launch(cross_dq_kernel<D, EXACT>, grid, 256, dq_smem_bytes(D), st, p)
                                : launch(cross_dq_kernel<D, WHOLE>, grid, 256, dq_smem_bytes(D), st, p);
  }
  if (e != hipSuccess || p.seq_kv == 0) return e;
  p.splits = key_splits(p, D, bytes);
  const int grid = ceil_div(p.seq_kv, 128) * nhb * p.splits;
  if constexpr (D == 128) e = launch(cross_dkv_pair_kernel<D>, grid, 512, dkv_pair_smem_bytes(D), st, p);
  else e = launch(cross_dkv_kernel<D>, grid, 256, dkv_smem_bytes(D), st, p);
  if (e != hipSuccess || p.splits == 1) return e;
  return join_keys<D>(st, p);
}

}  // namespace

// ------------------------------------------------------------------------------------------------ launchers
void k_cross_attn_scratch(const CrossArgs& p, int d, size_t* fwd_bytes, size_t* bwd_bytes) {
  const size_t all = ~(size_t)0;
  const int fs = few_rows(p) ? step_splits(p, d, all) : row_splits(p, d, all), rs = row_splits(p, d, all), ks = key_splits(p, d, all);
  const size_t r = rs > 1 ? rs * row_part_bytes(p, d) : 0, k = ks > 1 ? ks * key_part_bytes(p, d) : 0;
  *fwd_bytes = fs > 1 ? fs * row_part_bytes(p, d) : 0;
  *bwd_bytes = r > k ? r : k;
}

hipError_t k_cross_attn_fwd(hipStream_t st, const CrossArgs& p, int d, void* scratch, size_t bytes) {
  if (p.batch == 0 || p.seq_q == 0) return hipSuccess;
  return d == 128 ? fwd<128>(st, p, scratch, bytes) : fwd<64>(st, p, scratch, bytes);
}

hipError_t k_cross_attn_bwd(hipStream_t st, const CrossArgs& p, int d, void* scratch, size_t bytes) {
  if (p.batch == 0 || (p.seq_q == 0 && p.seq_kv == 0)) return hipSuccess;
  return d == 128 ? bwd<128>(st, p, scratch, bytes) : bwd<64>(st, p, scratch, bytes);
}
