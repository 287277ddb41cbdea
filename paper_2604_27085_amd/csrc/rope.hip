// Rotary positions beyond the stage's own (elementwise.hip: half-split pairs over the whole head, one base): both pair layouts, a
// rotated part of the head, positions given per token, and the tables of contexts longer than the trained one.
//
// A pair (x, y) of a head at position p turns by the angle p theta_i:  (x c - y s, x s + y c) with (c, s) = A (cos, sin)(p theta_i).
// The rotation is linear, so its backward is the transpose: the same with -s, on the gradients.
#include "layer_ops.hpp"

namespace {

// ------------------------------------------------------------------------------------------------ table
// cs[p][i] = A (cos, sin)(p theta_i).  Angles are kept as turns, p theta_i / 2 pi, in 64 bits: only then does a position of 2^20 leave the
// 30 bits of a turn that an fp32 cosine needs.  The whole turns and the quarter turns come off exactly, which leaves |x| <= pi / 4, where
// the Taylor polynomials of sine (to x^11) and cosine (to x^12) are off by less than 1e-11.
RP_DEV double frequency(const RopeScale& r, int i) {      // turns a position
  const double theta = exp2(-(double)i * r.log2_base_step);
  double f = 1.0;
  if (r.by_parts) {
    const double turns = r.trained_len * theta * 0.15915494309189535;
    const double keep = fmin(fmax((turns - r.slow) * r.inv_span, 0.0), 1.0);
    f = keep + (1.0 - keep) * r.inv_factor;
  } else {
    f = r.inv_factor;
  }
  return theta * f * 0.15915494309189535;
}

RP_DEV void cos_sin_turns(double turns, double& co, double& si) {
  double t = turns - rint(turns);          // [-1/2, 1/2]: exact
  const double quarter = rint(4.0 * t);
  const double x = fma(quarter, -0.25, t) * 6.283185307179586;
  const double z = x * x;
  double s = -1.0 / 39916800.0, c = 1.0 / 479001600.0;
  s = fma(s, z, 1.0 / 362880.0);
  c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, -1.0 / 5040.0);
  c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, 1.0 / 120.0);
  c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, -1.0 / 6.0);
  c = fma(c, z, 1.0 / 24.0);
  s = fma(s * z, x, x);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int q = (int)quarter & 3;          // -2 and 2 are the same half turn
  co = (q & 1) ? s : c;
  si = (q & 1) ? c : s;
  co = (q == 1 || q == 2) ? -co : co;
  si = (q & 2) ? -si : si;
}

// Thread = one pair index and every `rows`-th of the block's positions.  Only the first of them and the step between them are worked out
// from their angles; from there on the pair is turned by the step, in 64 bits (4 products a position where the polynomials and the angle take
// 30, which would bound the kernel: 131072 x 64 pairs 20.9 us).  32 steps at most: they multiply the polynomials' error to 3e-10.
// Now bound by its writes: 131072 x 64 pairs 11.7 us, 5.7 TB/s (a fill reaches 6.9).
__global__ void __launch_bounds__(256) rope_table_scaled_kernel(float2* __restrict__ cs, int n_pos, int half, int rows, int per_block, const RopeScale r) {
  const int i0 = (int)threadIdx.x % half, lane_row = (int)threadIdx.x / half;      // (half <= 256)
  if (lane_row >= rows) return;
  const long p0 = (long)blockIdx.x * per_block + lane_row;
  if (p0 >= n_pos) return;
  const long end = min((long)(blockIdx.x + 1) * per_block, (long)n_pos);
  const double f = frequency(r, i0);
  double c, s, dc, ds;
  cos_sin_turns((double)p0 * f, c, s);
  cos_sin_turns((double)rows * f, dc, ds);
  c *= r.amplitude;
  s *= r.amplitude;
  for (long p = p0; p < end; p += rows) {
    cs[p * half + i0] = make_float2((float)c, (float)s);
    const double t = c * dc - s * ds;
    s = s * dc + c * ds;
    c = t;
  }
}

// ------------------------------------------------------------------------------------------------ rotation
template <int V> struct Piece;      // V elements on a boundary of their own size
template <> struct Piece<8> { typedef uint4 type; };
template <> struct Piece<4> { typedef uint2 type; };
template <> struct Piece<2> { typedef uint32_t type; };
template <> struct Piece<1> { typedef unsigned short type; };
template <int V>
RP_DEV void unpack(const typename Piece<V>::type& w, float (&f)[V]) {
  if constexpr (V == 1) {
    f[0] = bf16_bits_to_f32(w);
  } else {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(&w);
#pragma unroll
    for (int e = 0; e < V / 2; ++e) { f[2 * e] = bf16_lo(u[e]); f[2 * e + 1] = bf16_hi(u[e]); }
  }
}
template <int V>
RP_DEV typename Piece<V>::type pack(const float (&f)[V]) {
  typename Piece<V>::type w;
  if constexpr (V == 1) {
    w = (unsigned short)f32_to_bf16_bits(f[0]);
  } else {
    uint32_t* u = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
    for (int e = 0; e < V / 2; ++e) u[e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
  }
  return w;
}

// Eight elements at any even address: an access that crosses a line costs a second one, far less than two bytes at a time would.
struct __attribute__((packed, aligned(2))) Any8 { uint32_t x, y, z, w; };
template <int V, bool ANY>
RP_DEV typename Piece<V>::type load(const bf16* p) {
  if constexpr (ANY) {
    const Any8 v = *reinterpret_cast<const Any8*>(p);
    return make_uint4(v.x, v.y, v.z, v.w);
  } else {
    return *reinterpret_cast<const typename Piece<V>::type*>(p);
  }
}
template <int V, bool ANY>
RP_DEV void store(bf16* p, const typename Piece<V>::type& v) {
  if constexpr (ANY) *reinterpret_cast<Any8*>(p) = Any8{v.x, v.y, v.z, v.w};
  else *reinterpret_cast<typename Piece<V>::type*>(p) = v;
}

// How the units of a head are cut.  HALVES: V pairs, elements u V .. of both halves of the rotated part, V the largest power of two that divides
// rot / 2, and V elements to carry over.  WINDOWS: the same with eight elements at any even address, the last window of the pairs and of what is
// carried over pushed back to where it ends, so that some elements are written twice, with the same value: not for calls in place.  PAIRS: 16-byte
// pieces of four neighbouring pairs.  PAIRS_CUT: the same where the rotated part ends inside a piece.
enum Cut { HALVES, WINDOWS, PAIRS, PAIRS_CUT };

// A thread owns the same unit of NH heads of one token, so that what it reads of the table serves all of them, and has their loads in flight
// together.  In place, what is only carried over is left out.  Each thread reads all it changes before it writes, and (but for WINDOWS) no two share
// an element.  All units go one way through the code: a path of their own for the carried pieces doubles the time where a wave has both.
// Bound by memory: 16384 tokens of 72 heads of 128 in 114 us, 5.37 TB/s, where a large copy reaches 5.16.
template <int V, Cut CUT, int NH>
__global__ void __launch_bounds__(256) rope_kernel(const RotateArgs p) {
  constexpr bool ANY = CUT == WINDOWS, NEAR = CUT == PAIRS || CUT == PAIRS_CUT;
  constexpr int NCS = NEAR ? V / 2 : V;
  typedef typename Piece<V>::type piece;
  const int heads = p.a + p.k, nhg = (heads + NH - 1) / NH;
  const int per = nhg * p.nunits, half = p.rot / 2, nrot = p.nrot;
  const int tl = (int)threadIdx.x / per;
  const int t = p.first + (int)blockIdx.x * p.tokens_per_block + (p.tokens_per_block > 1 ? tl : 0);
  if (t >= p.T || (p.tokens_per_block > 1 && tl >= p.tokens_per_block)) return;
  const int pos = p.pos ? p.pos[t] : t % p.seq;
  const bool in_table = pos >= 0 && pos < p.n_pos;
  for (int it = p.tokens_per_block > 1 ? (int)threadIdx.x - tl * per : (int)threadIdx.x; it < per; it += 256) {
    const int u = it % p.nunits, h0 = it / p.nunits;
    const bool turn = u < nrot;
    int x0 = turn || NEAR ? u * V : p.rot + (u - nrot) * V;
    if (ANY) x0 = turn ? min(x0, half - V) : min(x0, p.d - V);
    float co[NCS], si[NCS];
    if (turn) {
      const int i0 = NEAR ? u * NCS : x0;
      const float2* const row = p.cs + (long)pos * half + i0;
#pragma unroll
      for (int e = 0; e < NCS; ++e) {
        const float2 v = in_table && (CUT != PAIRS_CUT || i0 + e < half) ? row[e] : make_float2(NAN, NAN);
        co[e] = v.x;
        si[e] = p.bwd ? -v.y : v.y;
      }
    }
    piece w0[NH], w1[NH];
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      const int head = h0 + i * nhg;
      if (head >= heads) break;
      const bf16* src = head < p.a ? p.in_q + (long)t * p.ld_in_q + (long)head * p.d : p.in_k + (long)t * p.ld_in_k + (long)(head - p.a) * p.d;
      w0[i] = load<V, ANY>(src + x0);
      if (!NEAR && turn) w1[i] = load<V, ANY>(src + x0 + half);
    }
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      const int head = h0 + i * nhg;
      if (head >= heads) break;
      bf16* dst = head < p.a ? p.out_q + (long)t * p.ld_out_q + (long)head * p.d : p.out_k + (long)t * p.ld_out_k + (long)(head - p.a) * p.d;
      if (turn) {
        float x[V];
        unpack<V>(w0[i], x);
        if constexpr (NEAR) {
#pragma unroll
          for (int e = 0; e < V / 2; ++e) {
            const float a = x[2 * e], b = x[2 * e + 1];
            const bool on = CUT != PAIRS_CUT || u * NCS + e < half;
            x[2 * e] = on ? a * co[e] - b * si[e] : a;
            x[2 * e + 1] = on ? b * co[e] + a * si[e] : b;
          }
        } else {
          float y[V], z[V];
          unpack<V>(w1[i], y);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            z[e] = y[e] * co[e] + x[e] * si[e];
            x[e] = x[e] * co[e] - y[e] * si[e];
          }
          store<V, ANY>(dst + x0 + half, pack<V>(z));
        }
        w0[i] = pack<V>(x);
      }
      store<V, ANY>(dst + x0, w0[i]);
    }
  }
}

template <int V, Cut CUT>
hipError_t launch_rope(hipStream_t st, RotateArgs p, bool in_place) {
  constexpr int NH = 4;
  const int heads = p.a + p.k;
  if (CUT == PAIRS || CUT == PAIRS_CUT) {
    p.nrot = (p.rot + 7) / 8;
    p.nunits = in_place ? p.nrot : p.d / 8;
  } else {
    p.nrot = (p.rot / 2 + V - 1) / V;
    p.nunits = p.nrot + (in_place ? 0 : (p.d - p.rot + V - 1) / V);
  }
  const int per = ((heads + NH - 1) / NH) * p.nunits;
  p.tokens_per_block = per < 256 ? 256 / per : 1;
  // a launch has fewer than 2^32 threads: 2^31 in one, and as many launches as it takes
  const long blocks = ((long)p.T + p.tokens_per_block - 1) / p.tokens_per_block, most = 1l << 23;
  for (long b = 0; b < blocks; b += most) {
    p.first = (int)(b * p.tokens_per_block);
    RP_LAUNCH((rope_kernel<V, CUT, NH>), dim3((unsigned)(blocks - b < most ? blocks - b : most)), dim3(256), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

// ------------------------------------------------------------------------------------------------ launchers
hipError_t k_rope_table_scaled(hipStream_t st, float2* cs, int n_pos, int rot, const RopeScale& r) {
  if (n_pos == 0) return hipSuccess;
  const int half = rot / 2;
  const int rows = 256 / half;
  // enough blocks to fill the chip; then positions share what a frequency costs, 32 a thread at most
  int each = (int)((long)n_pos / ((long)rows * 1024));
  each = each < 1 ? 1 : each > 32 ? 32 : each;
  const int per_block = rows * each;
  RP_LAUNCH(rope_table_scaled_kernel, dim3((unsigned)(((long)n_pos + per_block - 1) / per_block)), dim3(256), 0, st, cs, n_pos, half, rows, per_block, r);
  return hipGetLastError();
}

hipError_t k_rope(hipStream_t st, int layout, const RotateArgs& p) {
  if (p.T == 0 || p.a + p.k == 0) return hipSuccess;
  const bool in_place = (p.a == 0 || p.in_q == p.out_q) && (p.k == 0 || p.in_k == p.out_k);
  if (layout) return p.rot % 8 == 0 ? launch_rope<8, PAIRS>(st, p, in_place) : launch_rope<8, PAIRS_CUT>(st, p, in_place);
  const int half = p.rot / 2, rest = p.d - p.rot;
  if (half % 8 == 0) return launch_rope<8, HALVES>(st, p, in_place);
  if (half % 4 == 0) return launch_rope<4, HALVES>(st, p, in_place);
  // Windows touch elements twice: no part of a call may be in place.  84166 tokens of 6 heads of 256, rot 234: one element an access 224 us, windows
  // 127;  where four elements an access do, either is ahead by some per cent (rot 24 of 96: 63 | 58, 60 of 128: 42 | 44).
  const bool apart = (p.a == 0 || p.in_q != p.out_q) && (p.k == 0 || p.in_k != p.out_k);
  if (apart && half >= 8 && (rest == 0 || rest >= 8)) return launch_rope<8, WINDOWS>(st, p, in_place);
  if (half % 2 == 0) return launch_rope<2, HALVES>(st, p, in_place);
  return launch_rope<1, HALVES>(st, p, in_place);
}
