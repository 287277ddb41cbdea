// Attention in which every query sees a span of the keys, lo_t <= j < hi_t: documents of a packed row, windows, prefixes, padding, caches of different lengths.
//
//   z = scale q k^T;  c = cap tanh(z / cap) (or z);  S = c - slope |p_t - j| (or c);  lse = log sum exp S;  P = exp(S - lse);  o = P v
//   dV = P^T dO;  dP = dO V^T;  delta = rowsum(P dP) = rowsum(dO o);  dS = P (dP - delta) (1 - (c / cap)^2);  dQ = scale dS K;  dK = scale dS^T Q
//
// The span belongs to the query, so the query heads of a key head's group share it: row r of a key head is query r / grp of head r % grp, and a tile of 128 rows holds 128 / grp
// neighbouring queries with all their heads.  Their spans nearly agree: the keys that a tile needs are those that any of its queries sees, tiles of keys that every
// query sees take no mask, and dK, dV of a group need no partials per head.
//
//   forward, dQ: workgroup = four waves x 32 rows, loop over the 64-key tiles that any row sees, the last rows first (causal rows at the end see most)
//   dK, dV     : workgroup = 128 keys, loop over the 64-row tiles that see any of them (d = 128: eight waves, pairs of which share 32 keys; d = 64: four); what each row
//                tile sees in all is left behind by dQ, which runs before
// Where there are too few workgroups for the chip, the loop is cut into `splits` slices, whose results another kernel joins in slice order (fp32 partials in the caller's
// scratch; no atomics, so the result does not depend on timing).
//
// In a tile that some rows do not see, scores are replaced, and what the products sum over (V; K of dQ; Q and dO) has its infinities and NaN taken out, since 0 times those would
// reach the rows beside them: a document is not touched by what is in another.  What does see such a value is made NaN as a whole: the row of o that sees it in v, the row of dQ that sees it in
// k (both marked key by key in LDS), and dK, dV of the keys that a row with it in q or dO sees (by a delta of its own: lse need not show it, and dV does not know of delta).
//
// P (for P v and dV) and dS are rounded to bf16, as the matrix instruction takes them (2^-8 a term at most; P of few rows, and dS in small calls, in two parts, 2^-16); scores, statistics, dP - delta and every sum are
// fp32.  The forward divides by the sum of the rounded P: what all terms of a row were rounded by alike drops out, and where a row lies on one key o is that key's v.  o goes out in two
// parts, its bf16 and that of what the rounding left over, so that delta = dO.(o + rest) does not carry o's rounding, which would be as large as dP - delta in such rows.
//
// What bounds it (rocprofv3; docs: 16384 tokens of 4 documents, 32 heads of 128 in groups of 4; window: 4096 tokens, 16 heads of 128 in groups of 2, 1024 keys, capped; prefix: 2 x 1021 tokens of 3
// documents, 64 heads of 64 in groups of 8, biased; matrix pipe and vector issue busy, waves waiting):
//   forward  docs 1030 us 48 %, 50 %, 17 %;  window 70 us 26 %, 57 %, 18 %;  prefix 37 us 17 %, 73 %, 27 %
//   dQ       docs 1265 us 56 %, 43 %, 16 %;  window 82 us 30 %, 49 %, 19 %;  prefix 39 us 22 %, 57 %, 26 %
//   dK, dV   docs 1995 us 45 %, 32 %, 25 %;  window 116 us 29 %, 39 %, 29 %;  prefix 57 us 25 %, 45 %, 32 %
// docs: the exponentials and conversions beside the products, and the clock that the matrix pipe's power leaves (2.0 to 2.3 GHz; 8192 causal tokens take 570, 705 and 1015 us, 960,
// 1170 and 1080 TFLOP/s of their products);
// window: the same with the tangent's exponential and quotient, and masks in an eighth of the tiles; prefix: 5 to 9 tiles a workgroup, most of them masked, between launches of a round or two.
#include <type_traits>

#include "attention_slices.hpp"
#include "pack_ops.hpp"

namespace {

// operand tiles, or the epilogue's staging of every wave's 32 x d block, whichever is larger
constexpr int fwd_tile_bytes(int d) { return max_i(64 * (d + 8) + 64 * (d + 32), 128 * (d + 8)) * 2; }
constexpr int dq_tile_bytes(int d) { return max_i(2 * 64 * tile_ld(d), 128 * (d + 8)) * 2; }

constexpr int step_smem_bytes(int d, int nc, int nw) { return nw * max_i(32 * tile_ld(d) * 2, 16 * nc * (3 + d + 4) * 4); }
constexpr int dkv_smem_bytes(int d) { return max_i(2 * 64 * tile_ld(d) * 2 + 6 * 64 * 4, 4 * 32 * (d + 4) * 4); }
constexpr int dkv_pair_smem_bytes(int d, bool two) { return 2 * (2 * 64 * tile_ld(d)) * 2 + 8 * (two ? 6 : 4) * 64 * 16 + 2 * 6 * 64 * 4; }
constexpr float LOG2E = 1.4426950408889634f;

// Sizes of one sequence and key head.
struct Rows {
  int b, g, grp, total, seq_q;
  unsigned inv;      // 2^32 / grp, rounded up
  RP_DEV Rows(const SpanArgs& p, int hb) {
    b = hb / p.kh;
    g = hb - b * p.kh;
    grp = p.a / p.kh;
    seq_q = p.seq_q;
    total = grp * seq_q;
    inv = grp > 1 ? 0xffffffffu / (unsigned)grp + 1u : 0u;
  }
  // query and head within the group of row r: r inv / 2^32 is at most one too large
  RP_DEV void at(int r, int& q, int& h) const {
    q = grp > 1 ? (int)__umulhi((unsigned)r, inv) : r;
    h = r - q * grp;
    if (h < 0) { --q; h += grp; }
  }
  // offset of row r in a [T, heads, d] tensor of row stride ld, from its first element
  RP_DEV long offset(int r, long ld, int d) const {
    int q, h;
    at(r, q, h);
    return ((long)b * seq_q + q) * ld + (long)(g * grp + h) * d;
  }
  RP_DEV long stat(int r, int a) const {   // in a [batch, a, seq_q] array
    int q, h;
    at(r, q, h);
    return ((long)b * a + g * grp + h) * seq_q + q;
  }
};

// What a row sees; nothing: 0, 0.  Rows behind the last one see nothing either.
RP_DEV int2 span_of(const SpanArgs& p, const Rows& s, int r) {
  int q, h;
  s.at(r < s.total ? r : 0, q, h);
  const int2 v = p.span[(long)s.b * p.seq_q + q];
  const int lo = max(v.x, 0), hi = min(v.y, p.seq_kv);
  return r < s.total && hi > lo ? make_int2(lo, hi) : make_int2(0, 0);
}

// Of several rows: the keys that any of them sees, [lo, hi), and those that all of them see, [all_lo, all_hi).
struct Seen {
  int lo, hi, all_lo, all_hi;
  RP_DEV void start(const int2& v, bool row) {
    lo = v.y > v.x ? v.x : 0x7fffffff;
    hi = v.y;
    all_lo = row ? v.x : 0;
    all_hi = row ? v.y : 0x7fffffff;
  }
  RP_DEV void add(int a, int b, int c, int d) {
    lo = min(lo, a);
    hi = max(hi, b);
    all_lo = max(all_lo, c);
    all_hi = min(all_hi, d);
  }
  // over the lanes l ^ from, l ^ 2 from, .. below `to`; then the same in all lanes
  RP_DEV void lanes(int from, int to) {
    for (int o = from; o < to; o <<= 1) add(__shfl_xor(lo, o, 64), __shfl_xor(hi, o, 64), __shfl_xor(all_lo, o, 64), __shfl_xor(all_hi, o, 64));
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  }
  RP_DEV bool any(int k0, int k1) const { return k0 < hi && k1 > lo; }
  RP_DEV bool all(int k0, int k1) const { return all_lo <= k0 && all_hi >= k1; }
};
// The four waves' rows together, through LDS [4]; all threads.
RP_DEV Seen seen_by_all(const Seen& mine, int4* lds, int w, int lane) {
  if (lane == 0) lds[w] = make_int4(mine.lo, mine.hi, mine.all_lo, mine.all_hi);
  __syncthreads();
  Seen s = mine;
  for (int u = 0; u < 4; ++u) {
    const int4 v = lds[u];
    s.add(v.x, v.y, v.z, v.w);
  }
  s.lanes(64, 64);
  return s;
}

// Scores as exponents of two: k1 z' for plain ones, z' = q.k; capped ones from e = 2^(k1 z') = exp(2 z / cap): tanh = 1 - 2 r, r = 1 / (1 + e).
struct Score {
  float k1, k2;      // plain: scale log2(e);  capped: 2 scale log2(e) / cap, cap log2(e)
  float grad;        // what dS k and dS^T q are multiplied with: scale, and the 4 of 1 - tanh^2 = 4 (r - r^2)
  RP_DEV explicit Score(const SpanArgs& p) {
    grad = p.cap > 0.f ? 4.f * p.scale : p.scale;
    k1 = p.cap > 0.f ? 2.f * p.scale * LOG2E / p.cap : p.scale * LOG2E;
    k2 = p.cap * LOG2E;
  }
};
// (absolute error cap 2^-23 or so, from 1 + e)
RP_DEV float cap_r(float z, const Score& c) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(z * c.k1)); }
template <bool CAP>
RP_DEV float score2(float z, const Score& c) { return CAP ? __builtin_fmaf(-2.f * c.k2, cap_r(z, c), c.k2) : z * c.k1; }
// The same to 2^-22 of itself, for lse of a few keys, which may be small: tanh(u) of small u by its series (the next term is below 2^-26 there).  Where vector instructions do not count.
RP_DEV float fine_capped2(float z, const Score& c) {
  const float u = z * (c.k1 * 0.34657359027997264f), v = u * u;
  float t = __builtin_fmaf(v, -1382.f / 155925.f, 62.f / 2835.f);
  t = __builtin_fmaf(v, t, -17.f / 315.f);
  t = __builtin_fmaf(v, t, 2.f / 15.f);
  t = __builtin_fmaf(v, t, -1.f / 3.f);
  t = __builtin_fmaf(v * u, t, u);
  return fabsf(u) < 0.35f ? c.k2 * t : score2<true>(z, c);
}

// 16 bytes with infinities and NaN made zero.
RP_DEV uint32_t finite2(uint32_t u) {
  return ((u & 0x7f80u) == 0x7f80u ? 0u : u & 0xffffu) | ((u & 0x7f800000u) == 0x7f800000u ? 0u : u & 0xffff0000u);
}
RP_DEV uint4 finite8(const uint4& u) { return make_uint4(finite2(u.x), finite2(u.y), finite2(u.z), finite2(u.w)); }
// Whether there are any: three instructions for two values.  (An exponent of all ones carries into the bit above.)
RP_DEV uint32_t carries(uint32_t u) { return (u & 0x7f807f80u) + 0x00800080u; }
RP_DEV uint32_t carries(const uint4& u) { return carries(u.x) | carries(u.y) | carries(u.z) | carries(u.w); }
RP_DEV bool not_finite(uint32_t carried) { return (carried & 0x80008000u) != 0u; }
// In any lane of the wave.
template <int N>
RP_DEV bool any_not_finite(const uint4 (&r)[N]) {
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) c |= carries(r[i]);
  return __any(not_finite(c));
}
// What is made of x in a branch that is hardly ever taken is made there, not before a loop and kept in registers.
RP_DEV int found_here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
template <int N>
RP_DEV void make_finite(uint4 (&r)[N]) {
  if (!any_not_finite(r)) return;
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = finite8(r[i]);
}
// Which keys of a 64-key tile held an infinity or NaN, in LDS: key by key the number of the last tile where that was so, and the number of the last tile with any.  Nothing is cleared
// from tile to tile, and a tile without any costs one read, asked for before the next tile's loads.  (Asked for where the masks are applied: dQ of 2 x 1021 tokens, 64 heads of 64, prefixes 39.8 us
// instead of 38.9; 38.1 without marks.)
struct BadKeys {
  int* lds;      // [64], then one for all
  static constexpr int BYTES = 272;
  RP_DEV void start(int tid) const {      // before a barrier
    if (tid < 65) lds[tid] = -1;
  }
  // a thread's pieces (NT threads, CH a key) of tile j, made finite, in the barriers between which they are stored
  template <int CH, int NT, int N>
  RP_DEV void make_finite(uint4 (&r)[N], int j, int tid) const {
    if (!any_not_finite(r)) return;
    const int t = found_here(tid);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (not_finite(carries(r[i]))) lds[(i * NT + t) / CH] = lds[64] = j;      // (the same from all lanes)
      r[i] = finite8(r[i]);
    }
  }
  RP_DEV int last() const { return lds[64]; }      // of the tiles stored
  RP_DEV unsigned long long of(int j, int lane) const { return __ballot(lds[lane] == j); }      // a bit a key; all lanes
};

RP_DEV float sum2(uint32_t pair, float acc) {      // the two bf16 of a register, added up in fp32
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2, pair), __builtin_bit_cast(v2, 0x3f803f80u), acc, false);
}

// dS of up to FEW_KEYS keys, in calls of up to FEW_ROWS rows of all heads, goes to the products in two parts, its bf16 and that of what the rounding left over: dQ and dK are
// then off by their own rounding alone.  In one part the two are 1.45 times as far from the exact result as that rounding is, and where few rows see few keys, chance makes it up to
// 1.56 (relative 2-norm, 10^-3: 2.4 to 2.5 | 2.6, in two 1.7).  The products more cost little there (200 tokens, 16 heads of 128: dQ 13.8 -> 14.3 us, dK, dV 19.0 -> 19.3; 512
// tokens, 32 heads: 22 -> 25 and 29 -> 32); beyond, both would take a fifth longer (8192 causal tokens, 32 heads of 128: 718 -> 882 and 1087 -> 1306).
constexpr int FEW_KEYS = 512, FEW_ROWS = 16384;
RP_DEV uint32_t left_over(float a, float b, uint32_t rounded) { return pack_bf16x2(a - bf16_lo(rounded), b - bf16_hi(rounded)); }
RP_DEV uint4 left_over(const f32x4& a, const f32x4& b, const uint4& rounded) {      // rounded: pack_frag(a, b)
  return make_uint4(left_over(a[0], a[1], rounded.x), left_over(a[2], a[3], rounded.y), left_over(b[0], b[1], rounded.z), left_over(b[2], b[3], rounded.w));
}
template <bool TWO>
struct Parts {
  uint4 hi[2], lo[2];      // of the column tiles
  RP_DEV Parts() {}
  RP_DEV Parts(const f32x4 (&x)[2][2]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      hi[c] = pack_frag(x[0][c], x[1][c]);
      if (TWO) lo[c] = left_over(x[0][c], x[1][c], hi[c]);
    }
  }
  RP_DEV f32x4 times(const uint4& a, int c, f32x4 acc) const {
    if (TWO) acc = mfma16(a, lo[c], acc);
    return mfma16(a, hi[c], acc);
  }
};

// In a branch that is taken for the few tiles at the edge of a span: keeps the compiler from doing the work for every tile and selecting.
RP_DEV void stay_in_branch() { asm volatile("" ::: "memory"); }

// delta of a row whose q or dO is not finite: a NaN that dK, dV know it by, in place of a score and a sum that are made from zeros there.
constexpr uint32_t SPOILT = 0x7fc0bad0u;

constexpr float FLOOR = -1.0e37f;      // the reference exponent of rows that have seen nothing yet: finite, so that exp2(-inf - FLOOR) = 0

// ================================================================================================ forward
template <int D, bool SPLIT, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) span_fwd_kernel(const SpanArgs p) {
  constexpr int LDK = D + 8, LDV = D + 32, KS = D / 16, DT = D / 32, NT = 256, BQ = 128, CH = D / 8;
  using T64 = Tile64<D, NT>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];   // fwd_smem_bytes(D)
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);
  bf16* const Ks = smem;
  bf16* const Vs = smem + 64 * LDK;
  int4* const seen_lds = reinterpret_cast<int4*>(dyn_smem + fwd_tile_bytes(D));       // [4]
  const BadKeys bad_keys{reinterpret_cast<int*>(seen_lds + 4)};

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lk = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nhb = p.kh * p.batch;
  const int rest = (int)blockIdx.x / nhb;
  const int hb = head_at((int)blockIdx.x, rest, nhb);
  const int split = SPLIT ? rest % p.splits : 0;
  const Rows s(p, hb);
  const int blocks = (s.total + BQ - 1) / BQ;
  const int r0 = (blocks - 1 - (SPLIT ? rest / p.splits : rest)) * BQ;
  const Score sc(p);

  const int row = r0 + 32 * w + lr;     // the lane's row
  const bool live = row < s.total;
  const int2 span = span_of(p, s, row);
  Seen mine;
  mine.start(span, live);
  mine.lanes(1, 32);
  bad_keys.start(tid);
  const Seen block = seen_by_all(mine, seen_lds, w, lane);
  int j0 = 0, j1 = 0;
  if (block.hi > block.lo) {
    j0 = block.lo / 64;
    j1 = (block.hi + 63) / 64;
  }
  if (SPLIT) {
    int first, last;
    slice_of(j1 - j0, p.splits, split, first, last);
    j1 = j0 + last;
    j0 += first;
  }
  const KeyTile<D, NT> kt_(p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D, p.ldk, p.seq_kv), vt_(p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D, p.ldv, p.seq_kv);

  uint4 qf[KS];
  float slope2 = 0.f;
  int pos = 0;
  {
    int q, h;
    s.at(live ? row : 0, q, h);
    const bf16* const qr = p.q + ((long)s.b * p.seq_q + q) * p.ldq + (long)(s.g * s.grp + h) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = make_uint4(0u, 0u, 0u, 0u);
      if (live) qf[ks] = *reinterpret_cast<const uint4*>(qr + 16 * ks + 8 * lk);
    }
    if (BIAS && live) {
      slope2 = p.slopes[s.g * s.grp + h] * LOG2E;
      pos = p.q_pos ? p.q_pos[(long)s.b * p.seq_q + q] : q + p.seq_kv - p.seq_q;
    }
  }

  float m_run = FLOOR, l_run = 0.f, lt_run = 0.f;      // lt: the sum of the rounded P
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
    const int kv0 = j * 64;
    const bool whole = block.all(kv0, kv0 + 64);      // uniform over the workgroup
    __syncthreads();
    if (!whole) bad_keys.make_finite<CH, NT>(vreg, j, tid);
    T64::template store<LDK>(kreg, Ks, tid);
    T64::template store<LDV>(vreg, Vs, tid);
    __syncthreads();
    if (j + 1 < j1) load_tiles(j + 1);
    const int last_bad = whole ? -1 : bad_keys.last();
    if (!mine.any(kv0, kv0 + 64)) continue;                   // uniform over the wave
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
    if constexpr (CAP) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v) sT[kt][v] = score2<true>(sT[kt][v], sc);
    }
    if constexpr (BIAS) {
      const float from = (float)(pos - (kv0 + 4 * lk));
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          sT[kt][v] = __builtin_fmaf(-slope2, fabsf(from - (float)(32 * kt + 8 * (v >> 2) + (v & 3))), CAP ? sT[kt][v] : sT[kt][v] * sc.k1);
    }
    constexpr bool DONE = CAP || BIAS;      // scores are exponents already
    if (!whole) {
      const int lo = span.x - (kv0 + 4 * lk);
      const unsigned n = (unsigned)(span.y - span.x);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v) sT[kt][v] = (unsigned)(32 * kt + 8 * (v >> 2) + (v & 3) - lo) < n ? sT[kt][v] : -INFINITY;
      if (__builtin_amdgcn_readfirstlane(last_bad) == j) {      // does the row see one of the keys whose v was not finite?
        const unsigned long long bad = bad_keys.of(j, lane);
        const int from = max(span.x - kv0, 0), to = min(span.y - kv0, 64);
        if (to > from && (bad >> from & (to - from == 64 ? ~0ull : (1ull << (to - from)) - 1ull))) lt_run = NAN;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sT[kt][v]);
    mx = DONE ? half_max(mx) : half_max(mx) * sc.k1;
    // m_run is a reference exponent that moves only when a row's maximum outgrows it by 2^8 (see attention.hip)
    const bool grow = mx > m_run + 8.f;
    if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
      const float m_new = grow ? mx : m_run;
      float alpha = fast_exp2(m_run - m_new);
      asm volatile("" : "+v"(alpha));
      l_run *= alpha;
      lt_run *= alpha;
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
        const float e = fast_exp2(DONE ? sT[kt][v] - m_run : __builtin_fmaf(sT[kt][v], sc.k1, -m_run));
        sT[kt][v] = e;
        psum += e;
      }
    l_run += psum;
    {
      uint4 pf[4];
      float rsum = 0.f;
#pragma unroll
      for (int gk = 0; gk < 4; ++gk) {
        pf[gk] = pack_frag32(sT[gk >> 1], 8 * (gk & 1));
        rsum = sum2(pf[gk].x, sum2(pf[gk].y, sum2(pf[gk].z, sum2(pf[gk].w, rsum))));
      }
      lt_run += rsum;
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

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64), lt_tot = lt_run + __shfl_xor(lt_run, 32, 64);
  if constexpr (SPLIT) {
    const long at = ((long)split * nhb + hb) * s.total + row;
    if (live) {
      if (lk == 0) p.part_ml[at] = make_float4(m_run, l_tot, lt_tot, j0 < j1 ? 1.f : 0.f);
      if (j0 < j1)      // (else the slice has no keys, and its part is not read)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int vg = 0; vg < 4; ++vg)
            *reinterpret_cast<float4*>(p.part + at * D + 32 * dt + 8 * vg + 4 * lk) =
                make_float4(oacc[dt][4 * vg], oacc[dt][4 * vg + 1], oacc[dt][4 * vg + 2], oacc[dt][4 * vg + 3]);
    }
  } else {
    const bool some = live && span.y > span.x;      // a row that sees nothing: o = 0, lse = -inf
    const float mul = some ? 1.f / lt_tot : 0.f;
    if (p.lse && lk == 0 && live) p.lse[s.stat(row, p.a)] = some ? m_run * 0.6931471805599453f + logf(l_tot) : -INFINITY;
    bf16* const stage = smem + w * 32 * LDK;
#pragma unroll
    for (int part = 0; part < 2; ++part) {      // o, then what its rounding left over
      bf16* const dst = part ? p.rest : p.o;
      if (!dst) continue;
      __syncthreads();
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int vg = 0; vg < 4; ++vg) {
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[e] = some ? oacc[dt][4 * vg + e] * mul : 0.f;
            if (part) y[e] -= (float)(bf16)y[e];
          }
          *reinterpret_cast<uint2*>(stage + lr * LDK + 32 * dt + 8 * vg + 4 * lk) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
        }
      __syncthreads();
#pragma unroll
      for (int it = 0; it < (32 * CH) / 64; ++it) {
        const int idx = it * 64 + lane, rr = idx / CH, ch = idx % CH, r = r0 + 32 * w + rr;
        if (r < s.total) *reinterpret_cast<uint4*>(dst + s.offset(r, p.ldo, D) + ch * 8) = *reinterpret_cast<const uint4*>(stage + rr * LDK + ch * 8);
      }
    }
  }
}

// ---- few rows: the step of a generation -----------------------------------------------------------------------
// At most 16 NC rows per key head (the queries of a step times the heads of the group).  Bound by reading K and V once, so a wave works alone, without
// barriers: the waves of a workgroup take the 32-key steps in turn, K goes from memory straight into the fragments of the matrix
// instruction (16 rows x 64 bytes a load: a whole row is used by one wave), V through a piece of LDS of the wave's own, since its
// reduction runs over the keys.  The next step's K and V are on their way during a step.  At the end the waves join in LDS.  P goes to the product in two parts, its bf16 and that of what
// the rounding left over, since the matrix pipe has little to do: o is then off by its own rounding alone (relative 2-norm from 64 bits 1.6e-3, in one part 1.9e-3; one query of 8 sequences against
// 4096 keys, 32 heads of 128 in groups of 4: 35.0 -> 35.1 us, of one sequence 11.57 -> 11.66).
template <int D, int NC, int NW, bool SPLIT, bool CAP, bool BIAS>
__global__ void __launch_bounds__(64 * NW) span_step_kernel(const SpanArgs p) {
  constexpr int LD = tile_ld(D), KS = D / 32, DT = D / 16, CH = D / 8, NV = 32 * CH / 64;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];   // step_smem_bytes(D, NC, NW)
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  bf16* const Vs = reinterpret_cast<bf16*>(dyn_smem) + w * 32 * LD;
  const int nhb = p.kh * p.batch;
  const int hb = (int)blockIdx.x % nhb, split = (int)blockIdx.x / nhb;
  const Rows s(p, hb);
  const Score sc(p);

  uint4 qf[NC][KS];
  int2 span[NC];
  float slope2[NC];
  int pos[NC];
  Seen seen;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int row = 16 * c + lr;
    const bool live = row < s.total;
    span[c] = span_of(p, s, row);
    Seen v;
    v.start(span[c], live);
    if (c == 0) seen = v;
    else seen.add(v.lo, v.hi, v.all_lo, v.all_hi);
    int q, h;
    s.at(live ? row : 0, q, h);
    const bf16* const qr = p.q + ((long)s.b * p.seq_q + q) * p.ldq + (long)(s.g * s.grp + h) * D + 8 * lg;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[c][ks] = make_uint4(0u, 0u, 0u, 0u);
      if (live) qf[c][ks] = *reinterpret_cast<const uint4*>(qr + 32 * ks);
    }
    slope2[c] = 0.f;
    pos[c] = 0;
    if (BIAS && live) {
      slope2[c] = p.slopes[s.g * s.grp + h] * LOG2E;
      pos[c] = p.q_pos ? p.q_pos[(long)s.b * p.seq_q + q] : q + p.seq_kv - p.seq_q;
    }
  }
  seen.lanes(1, 16);      // all the rows there are: the same in all waves
  int j0 = 0, j1 = 0;
  if (seen.hi > seen.lo) {
    j0 = seen.lo / 32;
    j1 = (seen.hi + 31) / 32;
  }
  if (SPLIT) {
    int first, last;
    slice_of(j1 - j0, p.splits, split, first, last);
    j1 = j0 + last;
    j0 += first;
  }
  const bf16* const kb = p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D;
  const bf16* const vb = p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D;

  float m_run[NC], l_run[NC], lt_run[NC];
  f32x4 oacc[DT][NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m_run[c] = FLOOR;
    l_run[c] = lt_run[c] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  u32x4 kreg[2][KS];
  uint4 vreg[NV];
  auto load_step = [&](int j) {      // rows past the end read as zero
    const int left = min(32, p.seq_kv - 32 * j);
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
      vreg[i] = buf_load16(rv, (uint32_t)(((c / CH) * (int)p.ldv + (c % CH) * 8) * 2));
    }
  };
  if (j0 + w < j1) load_step(j0 + w);
  const bf16* const vfrag = Vs + tr_base<LD>(lane);
  for (int j = j0 + w; j < j1; j += NW) {
    const bool whole = seen.all(32 * j, 32 * j + 32);      // uniform
    f32x4 sT[2][NC];      // [16 keys][16 rows]
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          sT[kt][c] = mfma16(__builtin_bit_cast(uint4, kreg[kt][ks]), qf[c][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sT[kt][c]);
    unsigned bad_keys = 0u;      // whose v is not finite, of a step that some rows do not see
    if (!whole && any_not_finite(vreg)) {
      stay_in_branch();
      unsigned mine = 0u;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        mine |= not_finite(carries(vreg[i])) ? 1u << i : 0u;
        vreg[i] = finite8(vreg[i]);
      }
#pragma unroll 1
      for (int i = 0; i < 32; ++i)      // key i is in the CH lanes from CH i % 64 on, their piece CH i / 64
        bad_keys |= __any((mine >> (CH * i / 64) & 1u) && lane / CH == i % (64 / CH)) ? 1u << i : 0u;
    }
    wave_lds_order();      // the last step's V has been read
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 64 * i + lane;
      *reinterpret_cast<uint4*>(Vs + (c / CH) * LD + (c % CH) * 8) = vreg[i];
    }
    wave_lds_order();
    if (j + NW < j1) load_step(j + NW);
    // exponents
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float from = BIAS ? (float)(pos[c] - (32 * j + 4 * lg)) : 0.f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = CAP ? fine_capped2(sT[kt][c][e], sc) : score2<false>(sT[kt][c][e], sc);
          if (BIAS) x = __builtin_fmaf(-slope2[c], fabsf(from - (float)(16 * kt + e)), x);
          sT[kt][c][e] = x;
        }
    }
    if (!whole) {
      stay_in_branch();
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int lo = span[c].x - (32 * j + 4 * lg);
        const unsigned n = (unsigned)(span[c].y - span[c].x);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) sT[kt][c][e] = (unsigned)(16 * kt + e - lo) < n ? sT[kt][c][e] : -INFINITY;
        if (bad_keys) {      // uniform
          const int first = max(span[c].x - 32 * j, 0), last = min(span[c].y - 32 * j, 32);
          if (last > first && (bad_keys >> first & (last - first == 32 ? ~0u : (1u << (last - first)) - 1u))) lt_run[c] = NAN;
        }
      }
    }
    bool grow = false;
    float mx[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      mx[c] = fmaxf(fmaxf(fmaxf(sT[0][c][0], sT[0][c][1]), fmaxf(sT[0][c][2], sT[0][c][3])), fmaxf(fmaxf(sT[1][c][0], sT[1][c][1]), fmaxf(sT[1][c][2], sT[1][c][3])));
      grow = grow || mx[c] > m_run[c] + 8.f;
    }
    // the reference exponent is the same in the four lanes of a column, and moves only when one of them outgrows it by 2^8
    if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float m = fmaxf(mx[c], __shfl_xor(mx[c], 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const float m_new = m > m_run[c] + 8.f ? m : m_run[c];
        const float alpha = fast_exp2(m_run[c] - m_new);
        l_run[c] *= alpha;
        lt_run[c] *= alpha;
        m_run[c] = m_new;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) oacc[dt][c] *= alpha;
      }
    }
    uint4 pf[NC], pf_left[NC];      // P, and what its rounding left over
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sT[kt][c][e] = fast_exp2(sT[kt][c][e] - m_run[c]);
          l_run[c] += sT[kt][c][e];
        }
      pf[c] = pack_frag(sT[0][c], sT[1][c]);
      pf_left[c] = left_over(sT[0][c], sT[1][c], pf[c]);
      lt_run[c] += sum2(pf[c].x, sum2(pf[c].y, sum2(pf[c].z, sum2(pf[c].w, sum2(pf_left[c].x, sum2(pf_left[c].y, sum2(pf_left[c].z, sum2(pf_left[c].w, 0.f))))))));
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const uint4 a = read_frag_tr<LD>(vfrag + 16 * dt);
#pragma unroll
      for (int c = 0; c < NC; ++c) oacc[dt][c] = mfma16(a, pf[c], mfma16(a, pf_left[c], oacc[dt][c]));
    }
  }

  // the waves join: wave w's reference exponent and sums of every row, then its rows of O^T
  float* const ml = reinterpret_cast<float*>(dyn_smem);      // [NW][3][16 NC]
  float* const os = ml + 3 * NW * 16 * NC;                   // [NW][16 NC][D + 4]
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const float l = column_sum(l_run[c]), lt = column_sum(lt_run[c]);
    if (lg == 0) {
      ml[(3 * w) * 16 * NC + 16 * c + lr] = m_run[c];
      ml[(3 * w + 1) * 16 * NC + 16 * c + lr] = l;
      ml[(3 * w + 2) * 16 * NC + 16 * c + lr] = lt;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<f32x4*>(os + (w * 16 * NC + 16 * c + lr) * (D + 4) + 16 * dt + 4 * lg) = oacc[dt][c];
  }
  __syncthreads();
  for (int i = tid; i < 16 * NC * CH; i += 64 * NW) {
    const int row = i / CH, ch = i % CH;
    if (row >= s.total) break;
    float m = FLOOR, l = 0.f, lt = 0.f, acc[8];
#pragma unroll
    for (int u = 0; u < NW; ++u) m = fmaxf(m, ml[3 * u * 16 * NC + row]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int u = 0; u < NW; ++u) {
      const float wgt = fast_exp2(ml[3 * u * 16 * NC + row] - m);      // (a wave without keys has sums of zero)
      l += wgt * ml[(3 * u + 1) * 16 * NC + row];
      lt += wgt * ml[(3 * u + 2) * 16 * NC + row];
      const float* const src = os + (u * 16 * NC + row) * (D + 4) + 8 * ch;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += wgt * src[e];
    }
    if constexpr (SPLIT) {
      const long at = ((long)split * nhb + hb) * s.total + row;
      if (ch == 0) p.part_ml[at] = make_float4(m, l, lt, j0 < j1 ? 1.f : 0.f);
      if (j0 < j1) {      // (else the slice has no keys, and its part is not read)
        *reinterpret_cast<float4*>(p.part + at * D + 8 * ch) = make_float4(acc[0], acc[1], acc[2], acc[3]);
        *reinterpret_cast<float4*>(p.part + at * D + 8 * ch + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
      }
    } else {
      const int2 v = span_of(p, s, row);
      const bool some = v.y > v.x;
      const float mul = some ? 1.f / lt : 0.f;
      if (p.lse && ch == 0) p.lse[s.stat(row, p.a)] = some ? m * 0.6931471805599453f + logf(l) : -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = some ? acc[e] * mul : 0.f;
      const long at = s.offset(row, p.ldo, D) + 8 * ch;
      *reinterpret_cast<uint4*>(p.o + at) = pack_times(acc, 1.f);
      if (p.rest) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] -= (float)(bf16)acc[e];
        *reinterpret_cast<uint4*>(p.rest + at) = pack_times(acc, 1.f);
      }
    }
  }
}

// Rows of the forward (weights exp2(m_i - max m)) or, with DQ, of dq (sums).
template <int D, int G, bool DQ>
__global__ void __launch_bounds__(256) span_row_join_kernel(const SpanArgs p) {
  constexpr int CH = D / 8, RPB = 256 / (CH * G), N = DQ ? 8 : 10;      // eight elements, and the forward's two sums
  __shared__ float red[CH * G > 64 ? 4 * CH * N : 1];
  const int total = (p.a / p.kh) * p.seq_q, nhb = p.kh * p.batch;
  const int tid = threadIdx.x, ch = tid % CH, grp = tid / CH % G;
  const long item = (long)blockIdx.x * RPB + tid / (CH * G);
  const bool in = item < (long)nhb * total;
  const int hb = in ? (int)(item / total) : 0, r = in ? (int)(item - (long)hb * total) : 0;
  const Rows s(p, hb);
  const int n = in ? p.splits : 0;
  const long row = (long)hb * total + r, step = (long)nhb * total;
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
    if constexpr (DQ) {
      add_times(acc, p.part + (i * step + row) * D + ch * 8, 1.f);
    } else {
      const float4 ml = p.part_ml[i * step + row];
      if (ml.w != 0.f) {      // the slice has keys.  (Its weights may all be 0 and its part NaN all the same, of a v that is not finite.)
        const float wgt = fast_exp2(ml.x - m);
        acc[8] += wgt * ml.y;
        acc[9] += wgt * ml.z;
        add_times(acc, p.part + (i * step + row) * D + ch * 8, wgt);
      }
    }
  }
  const bool store = add_groups<CH, G, N>(acc, red);
  if (!in || !store) return;
  if constexpr (DQ) {
    *reinterpret_cast<uint4*>(p.dq + s.offset(r, p.lddq, D) + ch * 8) = pack_times(acc, Score(p).grad);
  } else {
    const int2 span = span_of(p, s, r);
    const bool some = span.y > span.x;
    if (p.lse && ch == 0) p.lse[s.stat(r, p.a)] = some ? m * 0.6931471805599453f + logf(acc[8]) : -INFINITY;
    const float mul = some ? 1.f / acc[9] : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = some ? acc[e] * mul : 0.f;
    const long at = s.offset(r, p.ldo, D) + ch * 8;
    *reinterpret_cast<uint4*>(p.o + at) = pack_times(acc, 1.f);
    if (p.rest) {
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] -= (float)(bf16)acc[e];
      *reinterpret_cast<uint4*>(p.rest + at) = pack_times(acc, 1.f);
    }
  }
}

// ================================================================================================ dQ
template <int D, bool SPLIT, bool CAP, bool BIAS, bool TWO>
__global__ void __launch_bounds__(256, D == 64 && !TWO && !(CAP && BIAS) ? 3 : 2) span_dq_kernel(const SpanArgs p) {
  constexpr int LD = tile_ld(D), KS = D / 32, DT = D / 16, NT = 256, BQ = 128;
  using T64 = Tile64<D, NT>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];   // dq_smem_bytes(D)
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);
  bf16* const Ks = smem;
  bf16* const Vs = smem + 64 * LD;
  int4* const seen_lds = reinterpret_cast<int4*>(dyn_smem + dq_tile_bytes(D));       // [4]
  const BadKeys bad_keys{reinterpret_cast<int*>(seen_lds + 4)};

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nhb = p.kh * p.batch;
  const int rest = (int)blockIdx.x / nhb;
  const int hb = head_at((int)blockIdx.x, rest, nhb);
  const int split = SPLIT ? rest % p.splits : 0;
  const Rows s(p, hb);
  const int blocks = (s.total + BQ - 1) / BQ;
  const int r0 = (blocks - 1 - (SPLIT ? rest / p.splits : rest)) * BQ;
  const Score sc(p);

  int2 span[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) span[c] = span_of(p, s, r0 + 32 * w + 16 * c + lr);
  // A lane's rows, all on their way at once and while the spans are put together (a row behind the last one takes row 0's: nothing of it leaves the kernel).
  uint4 qf[2][KS], dof[2][KS], of[2][2][KS];     // column tiles c = 0, 1; o, and what its rounding left over
  float lse2[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int row = r0 + 32 * w + 16 * c + lr, rc = row < s.total ? row : 0;
    const bf16* const qr = p.q + s.offset(rc, p.ldq, D) + 8 * lg;
    const bf16* const dor = p.dout + s.offset(rc, p.lddo, D) + 8 * lg;
    const long at_o = s.offset(rc, p.ldo, D) + 8 * lg;
    lse2[c] = p.lse_in[s.stat(rc, p.a)];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[c][ks] = *reinterpret_cast<const uint4*>(qr + 32 * ks);
      dof[c][ks] = *reinterpret_cast<const uint4*>(dor + 32 * ks);
      of[0][c][ks] = *reinterpret_cast<const uint4*>(p.o_in + at_o + 32 * ks);
      of[1][c][ks] = make_uint4(0u, 0u, 0u, 0u);
      if (p.rest_in) of[1][c][ks] = *reinterpret_cast<const uint4*>(p.rest_in + at_o + 32 * ks);
    }
  }
  Seen mine;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    Seen v;
    v.start(span[c], r0 + 32 * w + 16 * c + lr < s.total);
    if (c == 0) mine = v;
    else mine.add(v.lo, v.hi, v.all_lo, v.all_hi);
  }
  mine.lanes(1, 16);
  bad_keys.start(tid);
  const Seen block = seen_by_all(mine, seen_lds, w, lane);
  // what dK, dV have to know of the two tiles of 64 rows
  if (s.g == 0 && split == 0 && (tid & 127) == 0 && r0 + 32 * w < s.total) {
    const int4 x = seen_lds[w], y = seen_lds[w + 1];
    p.tiles[(long)s.b * ((s.total + 63) / 64) + r0 / 64 + w / 2] = make_int4(min(x.x, y.x), max(x.y, y.y), max(x.z, y.z), min(x.w, y.w));
  }
  int j0 = 0, j1 = 0;
  if (block.hi > block.lo) {
    j0 = block.lo / 64;
    j1 = (block.hi + 63) / 64;
  }
  if (SPLIT) {
    int first, last;
    slice_of(j1 - j0, p.splits, split, first, last);
    j1 = j0 + last;
    j0 += first;
  }
  const KeyTile<D, NT> kt_(p.k + (long)s.b * p.seq_kv * p.ldk + s.g * D, p.ldk, p.seq_kv), vt_(p.v + (long)s.b * p.seq_kv * p.ldv + s.g * D, p.ldv, p.seq_kv);

  uint4 kreg[T64::NREG], vreg[T64::NREG];
  auto load_tiles = [&](int j) {
    kt_.load(kreg, j * 64, tid);
    vt_.load(vreg, j * 64, tid);
  };
  if (j0 < j1) load_tiles(j0);
  float dl[2], slope2[2] = {0.f, 0.f};
  int pos[2] = {0, 0};
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int row = r0 + 32 * w + 16 * c + lr;
    const bool ok = row < s.total;
    const int rc = ok ? row : 0;
    float sum = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint4 d = dof[c][ks];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 o = of[i][c][ks];
        sum += bf16_lo(o.x) * bf16_lo(d.x) + bf16_hi(o.x) * bf16_hi(d.x) + bf16_lo(o.y) * bf16_lo(d.y) + bf16_hi(o.y) * bf16_hi(d.y) +
               bf16_lo(o.z) * bf16_lo(d.z) + bf16_hi(o.z) * bf16_hi(d.z) + bf16_lo(o.w) * bf16_lo(d.w) + bf16_hi(o.w) * bf16_hi(d.w);
      }
    }
    const bool some = span[c].y > span[c].x;
    lse2[c] = some ? lse2[c] * LOG2E : INFINITY;      // rows that see nothing get P = 0
    sum = column_sum(sum);
    dl[c] = some ? sum : 0.f;
    // (a dO that is not finite has a delta that is not, whatever o is; a q that is not, scores and an lse that are not, unless capped)
    uint32_t carried = 0u;
    if (CAP)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) carried |= carries(qf[c][ks]);
    if (__any(!__builtin_isfinite(sum) || not_finite(carried))) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) carried |= carries(dof[c][ks]);
      carried |= __shfl_xor(carried, 16, 64);
      carried |= __shfl_xor(carried, 32, 64);
    }
    if (BIAS) {
      int q, h;
      s.at(rc, q, h);
      slope2[c] = p.slopes[s.g * s.grp + h] * LOG2E;
      pos[c] = p.q_pos ? p.q_pos[(long)s.b * p.seq_q + q] : q + p.seq_kv - p.seq_q;
    }
    if (lg == 0 && ok && split == 0) p.delta[s.stat(row, p.a)] = some && not_finite(carried) ? __uint_as_float(SPOILT) : dl[c];
  }

  const bf16* const kfrag = Ks + lr * LD + 8 * lg;      // (V lies 64 rows further on)
  const bf16* const ktfrag = Ks + tr_base<LD>(lane);
  f32x4 dqacc[DT][2];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dqacc[dt][0] = dqacc[dt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int j = j0; j < j1; ++j) {
    const bool whole = block.all(j * 64, j * 64 + 64);      // uniform over the workgroup
    __syncthreads();
    if (!whole) bad_keys.make_finite<D / 8, NT>(kreg, j, tid);
    T64::template store<LD>(kreg, Ks, tid);
    T64::template store<LD>(vreg, Vs, tid);
    __syncthreads();
    const int asked = whole ? -1 : bad_keys.last();
    if (j + 1 < j1) load_tiles(j + 1);
    const int last_bad = __builtin_amdgcn_readfirstlane(asked);
    // the two 32-key halves of the tile one after the other: half as many score registers live at a time
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      const int k0 = j * 64 + 32 * k2;
      if (!mine.any(k0, k0 + 32)) continue;      // uniform over the wave
      f32x4 sT[2][2], dpT[2][2];      // [16 keys][16 rows]
      const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
      {
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
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float from = BIAS ? (float)(pos[c] - (k0 + 4 * lg)) : 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float z = sT[kt][c][e], r = CAP ? cap_r(z, sc) : 0.f;
            float x = CAP ? __builtin_fmaf(-2.f * sc.k2, r, sc.k2 - lse2[c]) : __builtin_fmaf(z, sc.k1, -lse2[c]);      // exponent of P
            if (BIAS) x = __builtin_fmaf(-slope2[c], fabsf(from - (float)(16 * kt + e)), x);
            float ds = fast_exp2(x) * (dpT[kt][c][e] - dl[c]);
            if (CAP) ds *= __builtin_fmaf(-r, r, r);      // (1 - tanh^2) / 4
            sT[kt][c][e] = ds;   // dS^T
          }
      }
      if (!whole) {
        stay_in_branch();
        if (last_bad == j) {
          const unsigned mine4 = (unsigned)(bad_keys.of(j, lane) >> 32 * k2) >> found_here(4 * lg);
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
              for (int e = 0; e < 4; ++e) sT[kt][c][e] = mine4 >> (16 * kt + e) & 1u ? NAN : sT[kt][c][e];
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int lo = span[c].x - (k0 + 4 * lg);
          const unsigned n = (unsigned)(span[c].y - span[c].x);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) sT[kt][c][e] = (unsigned)(16 * kt + e - lo) < n ? sT[kt][c][e] : 0.f;
        }
      }
      constexpr int AHEAD = 4;      // K^T fragments requested that many pairs of products early
      const Parts<TWO> df(sT);
      auto ufrag_at = [&](int n) { return read_frag_tr<LD>(ktfrag + 32 * k2 * LD + 16 * n); };
      uint4 uring[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) uring[n] = ufrag_at(n);
#pragma unroll
      for (int n = 0; n < DT; ++n) {
        const uint4 a = uring[n % AHEAD];
        if (n + AHEAD < DT) uring[n % AHEAD] = ufrag_at(n + AHEAD);
#pragma unroll
        for (int c = 0; c < 2; ++c) dqacc[n][c] = df.times(a, c, dqacc[n][c]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if constexpr (SPLIT) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = r0 + 32 * w + 16 * c + lr;
      if (row < s.total) {
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
            make_uint2(pack_bf16x2(dqacc[dt][c][0] * sc.grad, dqacc[dt][c][1] * sc.grad), pack_bf16x2(dqacc[dt][c][2] * sc.grad, dqacc[dt][c][3] * sc.grad));
    __syncthreads();
#pragma unroll
    for (int it = 0; it < (32 * (D / 8)) / 64; ++it) {
      const int idx = it * 64 + lane, rr = idx / (D / 8), ch = idx % (D / 8), r = r0 + 32 * w + rr;
      if (r < s.total) *reinterpret_cast<uint4*>(p.dq + s.offset(r, p.lddq, D) + ch * 8) = *reinterpret_cast<const uint4*>(stage + rr * (D + 8) + ch * 8);
    }
  }
}

// ================================================================================================ dK, dV
// A thread's share of the 64-row tiles of q and dO, zero behind the last row: through descriptors that begin at the tile's first query and end behind the last one.  Where 64
// divides by the heads of a group (EVEN) a tile begins with a query, and a thread's pieces are at the same places from there in every tile.  (Worked out for every piece: 16 heads in
// groups of 2, a window of 1024 in 4096, 138 us for dK, dV instead of 118.)
template <int D, int NT, bool EVEN>
struct RowTile {
  static constexpr int CH = D / 8, NREG = 64 * CH / NT;
  const bf16 *qb, *dob;      // the group's first head of the sequence's first query
  long ldq, lddo;
  int q_off[NREG], do_off[NREG], queries;
  RP_DEV void place(int it, const Rows& s, int row0, int q0, int tid, int& q_at, int& do_at) const {
    int q, h;
    s.at(row0 + (it * NT + tid) / CH, q, h);
    const int in_row = h * D + ((it * NT + tid) % CH) * 8;
    q_at = (int)(((q - q0) * ldq + in_row) * 2);
    do_at = (int)(((q - q0) * lddo + in_row) * 2);
  }
  RP_DEV void start(const SpanArgs& p, const Rows& s, int tid) {
    ldq = p.ldq;
    lddo = p.lddo;
    queries = 64 / s.grp;
    qb = p.q + (long)s.b * p.seq_q * ldq + (long)s.g * s.grp * D;
    dob = p.dout + (long)s.b * p.seq_q * lddo + (long)s.g * s.grp * D;
#pragma unroll
    for (int it = 0; it < NREG; ++it) place(it, s, 0, 0, tid, q_off[it], do_off[it]);
  }
  RP_DEV rsrc_t from(const bf16* base, long ld, const Rows& s, int q0) const {
    const int left = min(queries + 2, s.seq_q - q0);      // >= 1
    // (all of this is the same in all lanes; where the compiler does not see it, it loops over the lanes around every load)
    const uint64_t at = reinterpret_cast<uint64_t>(base + (long)q0 * ld);
    const uint64_t same = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(same), 0, __builtin_amdgcn_readfirstlane((int)(((left - 1) * ld + (long)s.grp * D) * 2)), 0x00020000);
  }
  RP_DEV void load(uint4 (&q_reg)[NREG], uint4 (&do_reg)[NREG], const Rows& s, int u, int tid) const {
    int q0 = u * queries, h0;
    if (!EVEN) s.at(u * 64, q0, h0);
    const rsrc_t rq = from(qb, ldq, s, q0), rdo = from(dob, lddo, s, q0);
#pragma unroll
    for (int it = 0; it < NREG; ++it) {
      int q_at = q_off[it], do_at = do_off[it];
      if (!EVEN) place(it, s, u * 64, q0, tid, q_at, do_at);
      q_reg[it] = buf_load16(rq, (uint32_t)q_at);
      do_reg[it] = buf_load16(rdo, (uint32_t)do_at);
    }
  }
};

// Waits for all loads, before a loop that reads what they loaded.  Without it the compiler has to take them as on their way at every pass of the loop, and waits there for all that
// is: for the next tile's rows too, right after their loads were issued (4096 queries, 8192 keys, 32 heads of 128: dK, dV 1150 us instead of 1000).
RP_DEV void wait_for_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }      // vmcnt(0)

// The lane's number, found anew where registers are short: kept over a loop it is what the compiler puts in scratch memory.
RP_DEV int lane_now() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(l));
  return l;
}

// What there is to know of the rows of a 64-row tile, a row per lane of waves 0 to 3, in LDS as six arrays of 64: what the score starts from, -delta, first key,
// key behind the last, position from the tile's first key, slope.  Rows behind the last one: P = exp(-inf) = 0.  Rows that see nothing are masked.  Rows whose q or dO is not finite: P is NaN.
// load() only issues loads, and store(), a tile later, works on what came: whatever it did to them at once would have these waves, and at the next barrier all others, wait for
// the tile's rows too, whose loads are in flight before them (8192 causal tokens, 32 heads of 128: dK, dV 1250 us instead of 1170).
template <bool CAP, bool BIAS>
struct RowStat {
  static constexpr int FLOATS = 64 * 6;
  const int* src;      // wave 0: lse, 1: delta, 2: first key seen, 3: key behind the last; of the group's first head
  const int* src2;     // wave 0: positions, or NULL, 1: slopes
  long per_q, per_h;   // their strides
  int left;            // rows of the sequence from the tile's first one on
  float start_mul;     // the same in all lanes
  int x, y, z;
  RP_DEV void start(const SpanArgs& p, const Rows& s, int w) {
    // plain scores: the product starts from -lse / scale, so that it comes out as z - lse; a capped or biased one is taken off after
    start_mul = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(CAP || BIAS ? -LOG2E : -1.f / p.scale)));
    const long q = (long)s.b * p.seq_q, stat = ((long)s.b * p.a + s.g * s.grp) * p.seq_q;
    src = w == 0 ? (const int*)(p.lse_in + stat) : w == 1 ? (const int*)(p.delta + stat) : (const int*)(p.span + q) + (w & 1);
    per_q = w < 2 ? 1 : 2;
    per_h = w < 2 ? p.seq_q : 0;
    if (BIAS) src2 = w == 0 ? (p.q_pos ? p.q_pos + q : nullptr) : (const int*)(p.slopes + s.g * s.grp);
  }
  RP_DEV void load(const SpanArgs& p, const Rows& s, int row0, int lane, int w) {
    left = s.total - row0;
    if (w >= 4) return;
    int q, h;
    s.at(lane < left ? row0 + lane : 0, q, h);
    x = src[q * per_q + h * per_h];
    if (w == 0) z = __float_as_int(p.delta[((long)s.b * p.a + s.g * s.grp + h) * s.seq_q + q]);
    if (BIAS && w == 0) {
      y = q + p.seq_kv - s.seq_q;
      if (src2) y = src2[q];
    }
    if (BIAS && w == 1) y = src2[h];
  }
  RP_DEV void store(float* lds, const SpanArgs& p, int kv0, int lane, int w) const {
    const float f = w == 0 && z == (int)SPOILT ? NAN : __int_as_float(x);
    if (w == 0) lds[lane] = lane >= left ? -INFINITY : CAP ? __builtin_fmaf(f, start_mul, p.cap * LOG2E) : f * start_mul;
    if (w == 1) lds[64 + lane] = lane < left ? -f : 0.f;
    if (w == 2) lds[128 + lane] = __int_as_float(max(x, 0));
    if (w == 3) lds[192 + lane] = __int_as_float(lane < left ? min(x, p.seq_kv) : 0);
    if (BIAS && w == 0) lds[256 + lane] = (float)(y - kv0);
    if (BIAS && w == 1) lds[320 + lane] = __int_as_float(y) * LOG2E;
  }
};

// P and dS of 2 x 16 rows by 2 x 16 keys, in place of the scores and dP - delta.  lds: RowStat's, from the first of the rows on; key: the lane's first key, from kv0.
template <bool CAP, bool BIAS>
RP_DEV void probabilities(f32x4 (&s)[2][2], f32x4 (&dp)[2][2], const Score& c, const float* lds, int lg, int key, int kv0, bool whole) {
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const float* const at = lds + 16 * qt + 4 * lg;
    f32x4 start, pos, slope;
    if (CAP || BIAS) start = *reinterpret_cast<const f32x4*>(at);
    if (BIAS) {
      pos = *reinterpret_cast<const f32x4*>(at + 256);
      slope = *reinterpret_cast<const f32x4*>(at + 320);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float z = s[qt][t][e], r = CAP ? cap_r(z, c) : 0.f;
        float x = CAP ? __builtin_fmaf(-2.f * c.k2, r, start[e]) : BIAS ? __builtin_fmaf(z, c.k1, start[e]) : z * c.k1;
        if (BIAS) x = __builtin_fmaf(-slope[e], fabsf(pos[e] - (float)(key + 16 * t)), x);
        const float pr = fast_exp2(x);
        s[qt][t][e] = pr;
        dp[qt][t][e] = pr * dp[qt][t][e];
        if (CAP) dp[qt][t][e] *= __builtin_fmaf(-r, r, r);      // (1 - tanh^2) / 4
      }
  }
  if (!whole) {
    stay_in_branch();
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      const int4 lo = *reinterpret_cast<const int4*>(lds + 128 + 16 * qt + 4 * lg), hi = *reinterpret_cast<const int4*>(lds + 192 + 16 * qt + 4 * lg);
      const int first[4] = {lo.x, lo.y, lo.z, lo.w};
      const int behind[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int at = kv0 + key + 16 * t;
          const bool seen = at >= first[e] && at < behind[e];
          s[qt][t][e] = seen ? s[qt][t][e] : 0.f;
          dp[qt][t][e] = seen ? dp[qt][t][e] : 0.f;
        }
    }
  }
}

// Of the row tiles: x: the first one that sees any of the keys k0 .. k1 - 1, y: the one behind the last, z: how many see some of them, but not all rows all.  (Tiles in between may see none.)
// Over the tiles first, first + step, ..
RP_DEV int4 look_through(const int4* tiles, int n, int k0, int k1, int first, int step) {
  int lo = 0x7fffffff, hi = 0, part = 0;
#pragma unroll 4
  for (int t = first; t < n; t += step) {
    const int4 v = tiles[t];
    if (k0 < v.y && k1 > v.x) {
      lo = min(lo, t);
      hi = t + 1;
      part += v.z > k0 || v.w < k1;
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {      // of the wave
    lo = min(lo, __shfl_xor(lo, o, 64));
    hi = max(hi, __shfl_xor(hi, o, 64));
    part += __shfl_xor(part, o, 64);
  }
  return make_int4(lo, hi, part, 0);
}

// A walk over the row tiles [from, to) that see any of the keys, the last one first (the other way round takes as long).  What 64 neighbouring tiles see is asked for at once, a tile a lane, and kept as two masks: a
// load on the way to every tile would be waited for.
struct RowWalk {
  const int4* tiles;
  int k0, k1;
  int base, u, from;            // the masks' first tile; the present tile
  unsigned long long any, all;
  RP_DEV void look(int lane) {      // u and the 63 before it
    base = u - 63;
    const int t = base + lane;
    const int4 v = tiles[max(t, from)];
    any = __ballot(t >= from && k0 < v.y && k1 > v.x);
    all = __ballot(v.z <= k0 && v.w >= k1);
  }
  RP_DEV void settle(int lane) {      // to the present tile or the next one that sees any key; u < from: no more
    while (u >= from) {
      if (u < base) look(lane);
      const unsigned long long m = any << (63 - (u - base));
      if (m) {
        u -= __builtin_clzll(m);
        return;
      }
      u = base - 1;
    }
  }
  // (the last tile is taken in any case, so that its rows are on their way before anything is known of it: where it sees none of the keys the mask says so)
  RP_DEV void start(const int4* t, int key0, int key1, int first, int end) {
    tiles = t;
    k0 = key0;
    k1 = key1;
    from = first;
    u = end - 1;
    base = end;
    any = all = 0;
  }
  RP_DEV bool more() const { return u >= from; }
  RP_DEV bool whole() const { return all >> (u - base) & 1; }      // every row of the present tile sees all of the keys
  RP_DEV void next(int lane) {
    --u;
    settle(lane);
  }
};

// ---- who does what.  The key tiles of a causal row differ by as much as there are row tiles: where a launch has only a few rounds of them, the chip waits for the longest.  So the
// (key tile, row tile) pairs of a key head, in order, are cut into `parts` pieces of one length, and a workgroup does a piece: the end of one key tile, some whole
// ones, the beginning of another.  What it has of a key tile that others share goes to scratch, at most two of them a workgroup, and another kernel adds those up
// in order.  (8192 causal tokens, 64 heads of 64: a key tile a workgroup 1880 us.)  With more than MOST_TILES key tiles, or without scratch for the parts (parts 0), a
// workgroup does a key tile.
constexpr int MOST_TILES = 2048;
// A key tile counts for more pairs than its row tiles: beginning and ending with it costs about as much as FRONT of them, before its first, and the mask of a row tile that sees a part
// of it 3/8 of one, spread over them all (16384 tokens, 32 heads of 128: a key tile of 32 to 256 row tiles costs 4.3 of them more, a causal one 0.34 to 0.39 more for each of the eight
// at its edge).  A key tile with the end of one document and the beginning of a long one is masked all along: without counting that, the piece with it lasted 14 % longer than the others.
constexpr int FRONT = 4;
RP_DEV int edge_pairs(int part) { return FRONT + (3 * part + 4) / 8; }
// The row tiles of a key tile, of `rows` in `pairs`, that come before pair `pair` of it.  At most one a pair: the last pair has the last row tile, and four behind the front have two or more.
RP_DEV int rows_before(int pair, int rows, int pairs) {
  return pair <= FRONT ? 0 : pair >= pairs ? rows : (int)((unsigned long long)(pair - FRONT) * rows / (pairs - FRONT));
}
// The first pair that has a row tile (rows > 0).
RP_DEV int first_pair(int rows, int pairs) { return FRONT + (pairs - FRONT - 1) / rows; }
// (No shorter than what a piece costs by itself; it may hold nothing but a part of a front.  788 tokens, 6 heads of 128 in groups of 3, a window of 43: with eight pairs at least 26 us, with
// four 20.)
RP_DEV int piece_length(int pairs, int parts) { return max((pairs + parts - 1) / parts, FRONT); }

// ranges[i]: of key tile i % KT of sequence i / KT
__global__ void __launch_bounds__(256) span_range_kernel(const SpanArgs p) {
  __shared__ int4 lds[4];
  const int kt = (p.seq_kv + 127) / 128, b = (int)blockIdx.x / kt, k0 = ((int)blockIdx.x - b * kt) * 128;
  const int n = ((p.a / p.kh) * p.seq_q + 63) / 64;
  const int4 v = look_through(p.tiles + (long)b * n, n, k0, min(k0 + 128, p.seq_kv), threadIdx.x, 256);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x > 0) return;
  const int lo = min(min(lds[0].x, lds[1].x), min(lds[2].x, lds[3].x)), hi = max(max(lds[0].y, lds[1].y), max(lds[2].y, lds[3].y));
  p.ranges[blockIdx.x] = make_int2(hi > 0 ? lo : 0, hi);
  if (p.parts > 0) p.sums[blockIdx.x] = edge_pairs(lds[0].z + lds[1].z + lds[2].z + lds[3].z);      // (for the plan, which writes them anew)
}

// sums[i]: pairs before key tile i, edges included; pieces[i]: first key tile, first pair, pair behind the last.  One block, which with FIND finds the ranges too (where there
// is little to look through: one launch instead of two; 64 key tiles x 512 row tiles 20 us, 5 and 5 in two).
constexpr long FEW_LOOKS = 8192;
template <bool FIND>
__global__ void __launch_bounds__(1024) span_plan_kernel(const SpanArgs p) {
  __shared__ int sum[MOST_TILES + 1], wave[16];
  const int tid = threadIdx.x, kt = (p.seq_kv + 127) / 128, n = p.batch * kt;
  if (FIND) {
    const int lane = tid & 63, rows = ((p.a / p.kh) * p.seq_q + 63) / 64;
    for (int t = tid >> 6; t < n; t += 16) {      // a wave takes a key tile
      const int b = t / kt, k0 = (t - b * kt) * 128, k1 = min(k0 + 128, p.seq_kv);
      const int4 v = look_through(p.tiles + (long)b * rows, rows, k0, k1, lane, 64);
      if (lane == 0) {
        p.ranges[t] = make_int2(v.y > 0 ? v.x : 0, v.y);
        sum[t] = v.y > 0 ? v.y - v.x + edge_pairs(v.z) : 0;
      }
    }
    __syncthreads();
  }
  int c[2], s = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = 2 * tid + i;
    c[i] = 0;
    if (t < n) {
      if (FIND) {
        c[i] = sum[t];
      } else {
        const int2 r = p.ranges[t];
        c[i] = r.y > r.x ? r.y - r.x + p.sums[t] : 0;
      }
    }
    s += c[i];
  }
  __syncthreads();      // the counts have been read
  const int own = s;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(s, o, 64);
    if ((tid & 63) >= o) s += v;
  }
  if ((tid & 63) == 63) wave[tid >> 6] = s;
  __syncthreads();
  int at = s - own, all = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < tid >> 6) at += wave[w];
    all += wave[w];
  }
  if (2 * tid <= n) p.sums[2 * tid] = sum[2 * tid] = at;
  if (2 * tid + 1 <= n) p.sums[2 * tid + 1] = sum[2 * tid + 1] = at + c[0];
  if (n == MOST_TILES && tid == 0) p.sums[n] = sum[n] = all;
  __syncthreads();
  const int each = piece_length(all, p.parts);
  for (int i = tid; i < p.parts; i += 1024) {
    const int from = i * each, to = min(from + each, all);
    int lo = 0, hi = n;      // the last key tile that begins at or before the first pair
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (sum[mid] <= from) lo = mid;
      else hi = mid;
    }
    p.pieces[i] = make_int4(lo, from, to, 0);
  }
}

// The kernel's only argument, read anew: what is needed once for a key tile would otherwise sit in (spilled) scalar registers through the loop over its rows.
template <typename T>
RP_DEV void in_global(T*& p) { p = (T*)(__attribute__((address_space(1))) T*)reinterpret_cast<uint64_t>(p); }      // (else its loads would be flat ones)
RP_DEV SpanArgs read_again() {
  static_assert(sizeof(SpanArgs) % 8 == 0, "read by eight bytes");
  typedef const __attribute__((address_space(4))) uint64_t* args_t;      // (the constant address space: scalar loads)
  args_t at = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  uint64_t raw[sizeof(SpanArgs) / 8];
#pragma unroll
  for (int i = 0; i < (int)(sizeof(SpanArgs) / 8); ++i) raw[i] = at[i];
  SpanArgs p;
  __builtin_memcpy(&p, raw, sizeof p);
  in_global(p.q); in_global(p.k); in_global(p.v); in_global(p.dout); in_global(p.dk); in_global(p.dv); in_global(p.lse_in); in_global(p.delta);
  in_global(p.span); in_global(p.q_pos); in_global(p.slopes); in_global(p.tiles); in_global(p.part); in_global(p.ranges); in_global(p.sums);
  return p;
}

// The row tiles of a key tile; all waves.  Where no launch before has found them (ranges NULL: OWN_LOOKS row tiles at most, and a key tile a workgroup), every wave does.
constexpr int OWN_LOOKS = 256;
RP_DEV int2 tiles_of(const SpanArgs& p, const Rows& s, int tile, int k0, int lane) {
  if (p.ranges) return p.ranges[tile];
  const int n = (s.total + 63) / 64;
  const int4 v = look_through(p.tiles + (long)s.b * n, n, k0, min(k0 + 128, p.seq_kv), lane, 64);
  return make_int2(__builtin_amdgcn_readfirstlane(v.y > 0 ? v.x : 0), __builtin_amdgcn_readfirstlane(v.y));
}

// The keys of a workgroup do not mix: a column of the score tiles is a key's own.
template <int D, bool CAP, bool BIAS, bool EVEN, bool TWO>
__global__ void __launch_bounds__(256, 2) span_dkv_kernel(const SpanArgs args) {
  constexpr int LD = tile_ld(D), KS = D / 32, DT = D / 16, NT = 256;
  using T64 = Tile64<D, NT>;
  using Stat = RowStat<CAP, BIAS>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);             // Q | dO | the rows' numbers
  bf16* const Qs = smem;
  bf16* const dOs = smem + 64 * LD;
  float* const stat = reinterpret_cast<float*>(smem + 2 * 64 * LD);

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Score sc(args);
  const int tiles_kv = (args.seq_kv + 127) / 128;
  int tile, pair = 0, last_pair = 1, g;      // the present key tile and, in pieces, (key tile, row tile) pair of the head
  if (args.parts > 0) {
    g = (int)blockIdx.x % args.kh;
    const int4 piece = args.pieces[(int)blockIdx.x / args.kh];
    tile = piece.x;
    pair = piece.y;
    last_pair = piece.z;
    if (pair >= last_pair) return;      // uniform over the workgroup
  } else {
    const int nhb = args.kh * args.batch, rest = (int)blockIdx.x / nhb, hb = head_at((int)blockIdx.x, rest, nhb);
    g = hb % args.kh;
    tile = hb / args.kh * tiles_kv + rest;
  }
  for (int slot = 0;; slot = 1) {      // slot: of the parts that go to scratch, the piece begins with it, or not
  const SpanArgs p = read_again();
  const int b = tile / tiles_kv, kv0 = (tile - b * tiles_kv) * 128, kw0 = kv0 + 32 * w;
  const Rows s(p, b * p.kh + g);
  const int2 r = tiles_of(p, s, tile, kv0, lane);
  int u0 = r.x, u1 = r.y, end = 0;
  if (p.parts > 0) {
    end = p.sums[tile + 1];
    const int begin = p.sums[tile];
    u0 = r.x + rows_before(pair - begin, r.y - r.x, end - begin);
    u1 = r.x + rows_before(last_pair - begin, r.y - r.x, end - begin);
    if (u0 >= u1) return;      // nothing but the front of the last key tile is left (uniform over the workgroup)
  }
  const bool mine = u0 == r.x && u1 == r.y;      // the whole key tile is done here
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
      if (kpos[c] < p.seq_kv) {
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

  uint4 qreg[T64::NREG], doreg[T64::NREG];
  RowTile<D, NT, EVEN> rows;
  rows.start(p, s, tid);
  Stat rstat;
  rstat.start(p, s, w);
  auto prefetch = [&](int u) {
    rows.load(qreg, doreg, s, u, tid);
    rstat.load(p, s, u * 64, lane, w);
  };
  RowWalk range;
  range.start(p.tiles + (long)s.b * ((s.total + 63) / 64), kv0, min(kv0 + 128, p.seq_kv), u0, u1);
  if (range.more()) {
    prefetch(range.u);
    range.look(lane);
  }
  wait_for_loads();
  while (range.more()) {
    const bool whole = range.whole();
    __syncthreads();
    if (!whole) {
      make_finite(qreg);
      make_finite(doreg);
    }
    T64::template store<LD>(qreg, Qs, tid);
    T64::template store<LD>(doreg, dOs, tid);
    rstat.store(stat, p, kv0, lane, w);
    __syncthreads();
    range.next(lane);
    if (range.more()) prefetch(range.u);
    // the two 32-row halves of the tile one after the other: half as many score registers live at a time
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      f32x4 z[2][2], dp[2][2], z0[2], dp0[2];     // [16 rows][16 keys]; what they start from
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        z0[qt] = CAP || BIAS ? f32x4{0.f, 0.f, 0.f, 0.f} : *reinterpret_cast<const f32x4*>(stat + 32 * t2 + 16 * qt + 4 * lg);
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
            else z[qt][c] = mfma16(a, kf[c][ks], ks == 0 ? z0[qt] : z[qt][c]);
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
      probabilities<CAP, BIAS>(z, dp, sc, stat + 32 * t2, lg, 32 * w + lr, kv0, whole);
      {
        const uint4 pfg[2] = {pack_frag(z[0][0], z[1][0]), pack_frag(z[0][1], z[1][1])};
        const Parts<TWO> dfg(dp);
#pragma unroll
        for (int n = 0; n < NU; ++n) {
          const uint4 a = uring[n % AHEAD];
          if (n + AHEAD < NU) uring[n % AHEAD] = ufrag_at(n + AHEAD);
          const int dt = n >> 1;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            if (n & 1) dkacc[dt][c] = dfg.times(a, c, dkacc[dt][c]);
            else dvacc[dt][c] = mfma16(a, pfg[c], dvacc[dt][c]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  __syncthreads();
  const SpanArgs out = read_again();
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {      // dk, then dv in its place: the code once
    const float mul = which ? 1.f : sc.grad;
    const long ld = which ? out.lddv : out.lddk;
    if (mine) store_acc_T<D>(dkacc, mul, smem + w * 32 * (D + 8), (which ? out.dv : out.dk) + (long)s.b * out.seq_kv * ld + s.g * D, ld, kw0, out.seq_kv, lane);
    else store_acc_T_f32<D>(dkacc, mul, reinterpret_cast<float*>(smem) + w * 32 * (D + 4), out.part + (((long)blockIdx.x * 2 + slot) * 2 + which) * (128 * D), D, 32 * w, 128, lane);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) { dkacc[dt][0] = dvacc[dt][0]; dkacc[dt][1] = dvacc[dt][1]; }
  }
  if (out.parts == 0 || end >= last_pair) return;
  pair = end;
  do ++tile;
  while (out.sums[tile + 1] == pair);      // over key tiles that nothing sees (there is a pair left, so this ends)
  }
}

// Two waves per SIMD at d = 128 (see attn_bwd_dkv_pair_kernel in attention.hip): the 32 keys of a pair of waves are shared, wave h of it keeps
// the accumulators of half h of the head dimension, makes the scores of rows 32 h .. of each tile and hands P and dS to its partner through LDS.
template <int D, bool CAP, bool BIAS, bool EVEN, bool TWO>
__global__ void __launch_bounds__(512, 2) span_dkv_pair_kernel(const SpanArgs args) {
  constexpr int LD = tile_ld(D), KS = D / 32, DH = D / 32, NT = 512, NX = TWO ? 6 : 4;
  using T64 = Tile64<D, NT>;
  using Stat = RowStat<CAP, BIAS>;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];
  bf16* const smem = reinterpret_cast<bf16*>(dyn_smem);             // two sets (tile parity) of Q | dO, then the exchange
  constexpr int TSET = 2 * 64 * LD;
  uint4* const exch = reinterpret_cast<uint4*>(smem + 2 * TSET);    // [8 waves][NX fragments][64 lanes]
  float* const stat = reinterpret_cast<float*>(exch + 8 * NX * 64); // [2 sets]

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w8 = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = w8 >> 1, h = w8 & 1;
  const Score sc(args);
  const int tiles_kv = (args.seq_kv + 127) / 128;
  int tile, pair = 0, last_pair = 1, g;      // the present key tile and, in pieces, (key tile, row tile) pair of the head
  if (args.parts > 0) {
    g = (int)blockIdx.x % args.kh;
    const int4 piece = args.pieces[(int)blockIdx.x / args.kh];
    tile = piece.x;
    pair = piece.y;
    last_pair = piece.z;
    if (pair >= last_pair) return;      // uniform over the workgroup
  } else {
    const int nhb = args.kh * args.batch, rest = (int)blockIdx.x / nhb, hb = head_at((int)blockIdx.x, rest, nhb);
    g = hb % args.kh;
    tile = hb / args.kh * tiles_kv + rest;
  }
  for (int slot = 0;; slot = 1) {      // slot: of the parts that go to scratch, the piece begins with it, or not
  const SpanArgs p = read_again();
  const int b = tile / tiles_kv, kv0 = (tile - b * tiles_kv) * 128, kw0 = kv0 + 32 * w;
  const Rows s(p, b * p.kh + g);
  const int2 r = tiles_of(p, s, tile, kv0, lane);
  int u0 = r.x, u1 = r.y, end = 0;
  if (p.parts > 0) {
    end = p.sums[tile + 1];
    const int begin = p.sums[tile];
    u0 = r.x + rows_before(pair - begin, r.y - r.x, end - begin);
    u1 = r.x + rows_before(last_pair - begin, r.y - r.x, end - begin);
    if (u0 >= u1) return;      // nothing but the front of the last key tile is left (uniform over the workgroup)
  }
  const bool mine = u0 == r.x && u1 == r.y;      // the whole key tile is done here
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
      if (kpos[c] < p.seq_kv) {
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
  uint4* const ex_mine = exch + (w8 * NX) * 64 + lane;
  const uint4* const ex_theirs = exch + ((w8 ^ 1) * NX) * 64 + lane;

  uint4 qreg[T64::NREG], doreg[T64::NREG];
  RowTile<D, NT, EVEN> rows;
  rows.start(p, s, tid);
  Stat rstat;
  rstat.start(p, s, w8);
  auto prefetch = [&](int u) {
    rows.load(qreg, doreg, s, u, tid);
    rstat.load(p, s, u * 64, lane_now(), w8);
  };
  RowWalk range;
  range.start(p.tiles + (long)s.b * ((s.total + 63) / 64), kv0, min(kv0 + 128, p.seq_kv), u0, u1);

  constexpr int AHEAD = 2;     // two waves per SIMD cover each other's LDS latency: a short ring is enough
  auto update_half = [&](int set, int t2, const uint4 (&pf)[2], const Parts<TWO>& df) {
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
        if (n & 1) dkacc[dt][c] = df.times(a, c, dkacc[dt][c]);
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
    Parts<TWO> pdf;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      pdf.hi[c] = ex_theirs[128 + 64 * c];
      if (TWO) pdf.lo[c] = ex_theirs[256 + 64 * c];
    }
    update_half(prev & 1, h ^ 1, ppf, pdf);
  };
  if (range.more()) {
    prefetch(range.u);
    range.look(lane_now());
  }
  wait_for_loads();
  int i = 0;
  for (; range.more(); ++i) {
    const bool whole = range.whole();
    __syncthreads();
    bf16* const q_set = smem + (i & 1) * TSET;
    float* const st_set = stat + (i & 1) * Stat::FLOATS;
    if (!whole) {
      make_finite(qreg);
      make_finite(doreg);
    }
    T64::template store<LD>(qreg, q_set, tid);
    T64::template store<LD>(doreg, q_set + 64 * LD, tid);
    rstat.store(st_set, p, kv0, lane_now(), w8);
    if (i > 0) partner_update(i - 1);
    __syncthreads();
    range.next(lane_now());
    if (range.more()) prefetch(range.u);
    f32x4 z[2][2], dp[2][2], z0[2], dp0[2];      // [16 rows][16 keys]; what they start from
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      z0[qt] = CAP || BIAS ? f32x4{0.f, 0.f, 0.f, 0.f} : *reinterpret_cast<const f32x4*>(st_set + 32 * h + 16 * qt + 4 * lg);
      dp0[qt] = *reinterpret_cast<const f32x4*>(st_set + 64 + 32 * h + 16 * qt + 4 * lg);
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
          else z[qt][c] = mfma16(a, kf[c][ks], ks == 0 ? z0[qt] : z[qt][c]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      MFMA_PHASE_END();
    }
    probabilities<CAP, BIAS>(z, dp, sc, st_set + 32 * h, lg, 32 * w + lr, kv0, whole);
    const uint4 pfg[2] = {pack_frag(z[0][0], z[1][0]), pack_frag(z[0][1], z[1][1])};
    const Parts<TWO> dfg(dp);
    // the partner read last tile's fragments before the barrier above: the slots are free
    ex_mine[0] = pfg[0]; ex_mine[64] = pfg[1]; ex_mine[128] = dfg.hi[0]; ex_mine[192] = dfg.hi[1];
    if (TWO) { ex_mine[256] = dfg.lo[0]; ex_mine[320] = dfg.lo[1]; }
    update_half(i & 1, h, pfg, dfg);
  }
  __syncthreads();
  if (i > 0) partner_update(i - 1);
  __syncthreads();
  const SpanArgs out = read_again();
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {      // dk, then dv in its place: the code once
    const float mul = which ? 1.f : sc.grad;
    const int d0 = s.g * D + h * (D / 2);
    const long ld = which ? out.lddv : out.lddk;
    if (mine) store_acc_T<D / 2>(dkacc, mul, smem + w8 * 32 * (D / 2 + 8), (which ? out.dv : out.dk) + (long)s.b * out.seq_kv * ld + d0, ld, kw0, out.seq_kv, lane);
    else store_acc_T_f32<D / 2>(dkacc, mul, reinterpret_cast<float*>(smem) + w8 * 32 * (D / 2 + 4), out.part + (((long)blockIdx.x * 2 + slot) * 2 + which) * (128 * D) + h * (D / 2), D, 32 * w, 128, lane);
#pragma unroll
    for (int dt = 0; dt < DH; ++dt) { dkacc[dt][0] = dvacc[dt][0]; dkacc[dt][1] = dvacc[dt][1]; }
  }
  if (out.parts == 0 || end >= last_pair) return;
  pair = end;
  do ++tile;
  while (out.sums[tile + 1] == pair);      // over key tiles that nothing sees (there is a pair left, so this ends)
  }
}

// dk, dv of the key tiles that several workgroups share: the sum of their parts, in order; zero where nothing sees a key.  A block takes 32 keys of a key tile, of dk or of dv.
template <int D>
__global__ void __launch_bounds__(256) span_key_join_kernel(const SpanArgs p) {
  constexpr int CH = D / 8;
  const int tiles_kv = (p.seq_kv + 127) / 128, all_kv = p.batch * tiles_kv;
  const int i = (int)blockIdx.x >> 3, rows = ((int)blockIdx.x & 3) * 32, is_v = (int)blockIdx.x >> 2 & 1;
  const int tile = i / p.kh, g = i - tile * p.kh;
  const int2 r = p.ranges[tile];
  const int begin = p.sums[tile], end = p.sums[tile + 1], each = piece_length(p.sums[all_kv], p.parts);
  const int from = end > begin ? (begin + first_pair(r.y - r.x, end - begin)) / each : 0, to = (end - 1) / each;      // the pieces of its first and of its last row tile
  if (end > begin && from == to) return;      // one workgroup had it all
  const int b = tile / tiles_kv, kv0 = (tile - b * tiles_kv) * 128;
  for (int e = threadIdx.x; e < 32 * CH; e += 256) {
    const int row = rows + e / CH, ch = e % CH, key = kv0 + row;
    if (key >= p.seq_kv) continue;
    float acc[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) acc[x] = 0.f;
    if (end > begin) {
      // the first of them began its piece with another key tile, unless it begins in this one's front; the others begin with this key tile
      const float* const src = p.part + (long)is_v * 128 * D + row * D + ch * 8;
      add_times(acc, src + ((long)(from * p.kh + g) * 2 + (from * each >= begin ? 0 : 1)) * (2 * 128 * D), 1.f);
#pragma unroll 4
      for (int w = from + 1; w <= to; ++w) add_times(acc, src + (long)(w * p.kh + g) * 2 * (2 * 128 * D), 1.f);
    }
    const long t = (long)b * p.seq_kv + key;
    *reinterpret_cast<uint4*>((is_v ? p.dv + t * p.lddv : p.dk + t * p.lddk) + g * D + ch * 8) = pack_times(acc, 1.f);
  }
}

constexpr int fwd_smem_bytes(int d) { return fwd_tile_bytes(d) + 64 + BadKeys::BYTES; }
constexpr int dq_smem_bytes(int d) { return dq_tile_bytes(d) + 64 + BadKeys::BYTES; }

long row_count(const SpanArgs& p) { return (long)(p.a / p.kh) * p.seq_q; }
size_t row_part_bytes(const SpanArgs& p, int d) { return (size_t)p.kh * p.batch * row_count(p) * (d + 4) * 4; }      // o or dq, and (m, l, lt)
// Forward and dQ: two workgroups of 128 rows per CU.
int row_splits(const SpanArgs& p, int d, size_t bytes) {
  return splits_for((long)ceil_div(row_count(p), 128) * p.kh * p.batch, 512, ceil_div(p.seq_kv, 64), 1.4, row_part_bytes(p, d), bytes);
}
long key_tiles(const SpanArgs& p) { return (long)p.batch * ceil_div(p.seq_kv, 128); }
// Pieces of a key head for dK, dV: as many as the chip works on at a time (at d = 128 a workgroup has a CU to itself, at d = 64 two share one), unless there are
// rounds enough for the key tiles to even out by themselves.
int parts_of(const SpanArgs& p, int d) {
  const long groups = key_tiles(p) * p.kh, slots = d == 128 ? 256 : 512;
  if (key_tiles(p) > MOST_TILES || groups == 0 || groups >= 8 * slots) return 0;
  if (key_tiles(p) * (ceil_div(row_count(p), 64) * 3l / 2 + 20) >= 1l << 31) return 0;      // (pairs are counted in 31 bits)
  long n = slots / p.kh;
  const long most = key_tiles(p) * ceil_div(row_count(p), 64) / 4;      // (of four row tiles or more)
  if (most <= key_tiles(p)) return 0;      // no more of them than key tiles: a launch to join them for nothing (27 tokens of 6 heads of 64: backward 25 us instead of 19)
  if (n > most) n = most;
  return n < 1 ? 1 : (int)n;
}
size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }
// What the backward call cannot do without: what the row tiles see, and the row tiles of every key tile.
size_t tiles_bytes(const SpanArgs& p) { return round256((size_t)p.batch * ceil_div(row_count(p), 64) * 16); }
size_t least_bytes(const SpanArgs& p) { return tiles_bytes(p) + round256((size_t)key_tiles(p) * 8); }
struct KeyPlaces {      // in the scratch behind that
  size_t sums, pieces, part, end;
  KeyPlaces(const SpanArgs& p, int d, int parts) {
    sums = 0;
    pieces = round256((key_tiles(p) + 1) * 4);
    part = pieces + round256((size_t)parts * 16);
    end = parts ? part + (size_t)parts * p.kh * 2 * (2 * 128 * d * 4) : 0;
  }
};

template <int D, bool DQ>
hipError_t join_rows(hipStream_t st, const SpanArgs& p) {
  const int g = join_groups(p.splits), grid = ceil_div(row_count(p) * p.kh * p.batch, 256 / (D / 8 * g));
  if (g == 1) return launch(span_row_join_kernel<D, 1, DQ>, grid, 256, 0, st, p);
  if (g == 4) return launch(span_row_join_kernel<D, 4, DQ>, grid, 256, 0, st, p);
  return launch(span_row_join_kernel<D, 16, DQ>, grid, 256, 0, st, p);
}
// Few rows: slices for two workgroups of four waves per CU, with a 32-key step for each wave at least -- or one workgroup of eight waves, without slices, where
// its waves are through with their steps before the slices would have been joined, a second launch of 3 us.  (A step takes 2.1 us at d = 128, 1.1 at d = 64, one after the other: one
// query of 8 key heads against 512, 1024, 4096 keys of 128 8.3, 12.5, 38.5 us without slices, 8.4 and 9.3 with them from 1024 on; of 64 5.7, 7.8, 20.8 and 7.3, 8.6.)
bool few_rows(const SpanArgs& p) { return row_count(p) <= 32; }
int step_splits(const SpanArgs& p, int d, size_t bytes) {
  const long nhb = (long)p.kh * p.batch;
  const size_t each = row_part_bytes(p, d);
  const int steps = ceil_div(p.seq_kv, 32);
  long n = nhb ? 512 / nhb : 1;
  if (n > ceil_div(steps, 4)) n = ceil_div(steps, 4);
  if (each && n > (long)(bytes / each)) n = (long)(bytes / each);
  if (n < 2 || ceil_div(steps, 8) * 2.1 <= ceil_div(ceil_div(steps, (int)n), 4) * 2.1 + 3.0) return 1;
  return (int)n;
}
template <int D, int NC, bool CAP, bool BIAS>
hipError_t launch_step(hipStream_t st, const SpanArgs& p) {
  const int nhb = p.kh * p.batch;
  if (p.splits > 1) return launch(span_step_kernel<D, NC, 4, true, CAP, BIAS>, nhb * p.splits, 256, step_smem_bytes(D, NC, 4), st, p);
  if (p.seq_kv > 128 && nhb < 512) return launch(span_step_kernel<D, NC, 8, false, CAP, BIAS>, nhb, 512, step_smem_bytes(D, NC, 8), st, p);
  return launch(span_step_kernel<D, NC, 4, false, CAP, BIAS>, nhb, 256, step_smem_bytes(D, NC, 4), st, p);
}

template <int D, bool CAP, bool BIAS>
hipError_t fwd(hipStream_t st, SpanArgs p, void* scratch, size_t bytes) {
  const int nhb = p.kh * p.batch;
  const long rows = row_count(p);
  const bool few = few_rows(p);
  p.splits = few ? step_splits(p, D, bytes) : row_splits(p, D, bytes);
  p.part = static_cast<float*>(scratch);
  p.part_ml = reinterpret_cast<float4*>(p.part + (size_t)p.splits * nhb * rows * D);
  if (few) {
    const hipError_t e = rows <= 16 ? launch_step<D, 1, CAP, BIAS>(st, p) : launch_step<D, 2, CAP, BIAS>(st, p);
    return p.splits > 1 && e == hipSuccess ? join_rows<D, false>(st, p) : e;
  }
  const int grid = ceil_div(rows, 128) * nhb * p.splits;
  if (p.splits == 1) return launch(span_fwd_kernel<D, false, CAP, BIAS>, grid, 256, fwd_smem_bytes(D), st, p);
  const hipError_t e = launch(span_fwd_kernel<D, true, CAP, BIAS>, grid, 256, fwd_smem_bytes(D), st, p);
  return e == hipSuccess ? join_rows<D, false>(st, p) : e;
}

template <int D, bool CAP, bool BIAS, bool TWO>
hipError_t bwd_parts(hipStream_t st, SpanArgs p, void* scratch, size_t bytes) {
  const int nhb = p.kh * p.batch;
  const long rows = row_count(p);
  const size_t head = least_bytes(p);
  p.tiles = static_cast<int4*>(scratch);
  p.ranges = reinterpret_cast<int2*>(static_cast<char*>(scratch) + tiles_bytes(p));
  p.part = reinterpret_cast<float*>(static_cast<char*>(scratch) + head);
  bytes -= head;
  hipError_t e = hipSuccess;
  // dQ first: it works out delta, and what the row tiles see, which dK/dV read
  if (rows > 0) {
    p.splits = row_splits(p, D, bytes);
    const int grid = ceil_div(rows, 128) * nhb * p.splits;
    if (p.splits > 1) {
      e = launch(span_dq_kernel<D, true, CAP, BIAS, TWO>, grid, 256, dq_smem_bytes(D), st, p);
      if (e == hipSuccess) e = join_rows<D, true>(st, p);
    } else {
      e = launch(span_dq_kernel<D, false, CAP, BIAS, TWO>, grid, 256, dq_smem_bytes(D), st, p);
    }
  }
  if (e != hipSuccess || p.seq_kv == 0) return e;
  p.parts = rows > 0 ? parts_of(p, D) : 0;
  const KeyPlaces at(p, D, p.parts);
  if (bytes < at.end) p.parts = 0;
  const bool find = p.parts > 0 && key_tiles(p) * ceil_div(rows, 64) <= FEW_LOOKS;
  if (p.parts > 0) {
    char* const mem = static_cast<char*>(scratch) + head;
    p.sums = reinterpret_cast<int*>(mem + at.sums);
    p.pieces = reinterpret_cast<int4*>(mem + at.pieces);
    p.part = reinterpret_cast<float*>(mem + at.part);
  }
  if (p.parts == 0 && ceil_div(rows, 64) <= OWN_LOOKS) p.ranges = nullptr;
  else if (!find) e = launch(span_range_kernel, (int)key_tiles(p), 256, 0, st, p);
  if (e != hipSuccess) return e;
  if (p.parts > 0) {
    e = launch(find ? span_plan_kernel<true> : span_plan_kernel<false>, 1, 1024, 0, st, p);
    if (e != hipSuccess) return e;
  }
  const int grid = p.parts > 0 ? p.parts * p.kh : (int)key_tiles(p) * p.kh;
  constexpr bool E = !TWO;      // (few keys: one kernel for all groups)
  const bool even = E && 64 % (p.a / p.kh) == 0;
  if constexpr (D == 128) e = launch(even ? span_dkv_pair_kernel<D, CAP, BIAS, E, TWO> : span_dkv_pair_kernel<D, CAP, BIAS, false, TWO>, grid, 512, dkv_pair_smem_bytes(D, TWO), st, p);
  else e = launch(even ? span_dkv_kernel<D, CAP, BIAS, E, TWO> : span_dkv_kernel<D, CAP, BIAS, false, TWO>, grid, 256, dkv_smem_bytes(D), st, p);
  if (e != hipSuccess || p.parts == 0) return e;
  return launch(span_key_join_kernel<D>, (int)key_tiles(p) * p.kh * 8, 256, 0, st, p);
}

template <int D, bool CAP, bool BIAS>
hipError_t bwd(hipStream_t st, const SpanArgs& p, void* scratch, size_t bytes) {
  return p.seq_kv <= FEW_KEYS && (long)p.batch * p.a * p.seq_q <= FEW_ROWS ? bwd_parts<D, CAP, BIAS, true>(st, p, scratch, bytes) : bwd_parts<D, CAP, BIAS, false>(st, p, scratch, bytes);
}

// One of eight: d, cap, bias.
template <typename F>
hipError_t with_kind(const SpanArgs& p, int d, F&& f) {
  typedef std::integral_constant<int, 64> d64;
  typedef std::integral_constant<int, 128> d128;
  const auto kind = [&](auto dd) {
    if (p.cap > 0.f) return p.slopes ? f(dd, std::true_type{}, std::true_type{}) : f(dd, std::true_type{}, std::false_type{});
    return p.slopes ? f(dd, std::false_type{}, std::true_type{}) : f(dd, std::false_type{}, std::false_type{});
  };
  return d == 128 ? kind(d128{}) : kind(d64{});
}

}  // namespace

// ------------------------------------------------------------------------------------------------ launchers
void k_span_attn_scratch(const SpanArgs& p, int d, size_t* fwd_bytes, size_t* bwd_bytes) {
  const size_t all = ~(size_t)0;
  const int rs = row_splits(p, d, all), parts = row_count(p) > 0 ? parts_of(p, d) : 0;
  const size_t r = rs > 1 ? rs * row_part_bytes(p, d) : 0, k = KeyPlaces(p, d, parts).end;
  const int fs = few_rows(p) ? step_splits(p, d, all) : rs;
  *fwd_bytes = fs > 1 ? fs * row_part_bytes(p, d) : 0;
  *bwd_bytes = least_bytes(p) + (r > k ? r : k);
}
size_t k_span_attn_least(const SpanArgs& p) { return least_bytes(p); }

hipError_t k_span_attn_fwd(hipStream_t st, const SpanArgs& p, int d, void* scratch, size_t bytes) {
  if (p.batch == 0 || p.seq_q == 0) return hipSuccess;
  return with_kind(p, d, [&](auto dd, auto cap, auto bias) { return fwd<decltype(dd)::value, decltype(cap)::value, decltype(bias)::value>(st, p, scratch, bytes); });
}

hipError_t k_span_attn_bwd(hipStream_t st, const SpanArgs& p, int d, void* scratch, size_t bytes) {
  if (p.batch == 0 || (p.seq_q == 0 && p.seq_kv == 0)) return hipSuccess;
  return with_kind(p, d, [&](auto dd, auto cap, auto bias) { return bwd<decltype(dd)::value, decltype(cap)::value, decltype(bias)::value>(st, p, scratch, bytes); });
}
