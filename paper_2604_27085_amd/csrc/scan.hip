// Gated linear recurrence over the tokens of a sequence, every channel by itself, forward and backward.
//
//   f_t = sigmoid(g_t);  h_t = f_t h_(t-1) + w_t x_t,  w_t = 1 | 1 - f_t | sqrt(1 - f_t^2);  y_t = h_t
//   lam_t = dy_t + mu_(t+1),  mu_t = f_t lam_t;  dx_t = w_t lam_t;  dg_t = lam_t (h_(t-1) f_t (1 - f_t) + x_t dw_t/dg_t);  dh_0 = mu_0
//
// Where a document starts, f_t of the recurrence is 0 (the state before counts for nothing, and gets no gradient).  Behind a sequence's length the state is kept as it is.
// 1 - f is taken as sigmoid(-g): a gate near one keeps its distance from it.
//
// h_t = a_t h_(t-1) + b_t is a scan over the maps (a, b), which compose as (a2, b2) after (a1, b1) = (a2 a1, a2 b1 + b2).  Chunks of 64 tokens by 256 channels; a wave
// has eight tokens, a lane four channels, all in registers.  One launch makes every chunk's map, one the state that each starts from, one the outputs.  The backward
// pass is the same from behind; h_(t-1) is made again from the states that the forward pass left, in fp32 (4 bytes for 64 tokens), not from y, which is rounded.
// States, sums and products are fp32 throughout.
#include "pack_ops.hpp"

namespace {

constexpr int NW = 8, TOK = 8, CHUNK = NW * TOK, LANES = 4, BLOCK_CH = 64 * LANES;

typedef float f4 __attribute__((ext_vector_type(4)));

RP_DEV f4 unpack(const uint2& u) { return f4{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)}; }
RP_DEV uint2 pack(const f4& v) { return make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])); }

// sigmoid(g) and sigmoid(-g): the smaller one from an exponential that is at most 1, so that it keeps its relative precision (the exponential's argument is
// rounded: 2^-22 or so), the larger one as 1 less it, which is then one rounding off.  Errors of f add up over as many tokens as a gate remembers.
RP_DEV void gates(float g, float& f, float& r) {
  const float e = __expf(-fabsf(g)), t = e * __builtin_amdgcn_rcpf(1.f + e), s = 1.f - t;      // (NaN stays NaN)
  f = g >= 0.f ? s : t;
  r = g >= 0.f ? t : s;
}
template <int W>
RP_DEV float weight(float f, float r) { return W == 0 ? 1.f : W == 1 ? r : __builtin_amdgcn_sqrtf(r * (1.f + f)); }
// dw / dg: 0, -f r, -f^2 r / w = -f^2 sqrt(r / (1 + f))
template <int W>
RP_DEV float weight_slope(float f, float r) { return W == 0 ? 0.f : W == 1 ? -f * r : -f * f * __builtin_amdgcn_sqrtf(r * __builtin_amdgcn_rcpf(1.f + f)); }

// A workgroup's place: the channels change fastest, so that workgroups side by side read neighbouring pieces of the same rows.
struct Place {
  int b, chunk, ch, tid, lane, w, t0, len;      // t0: the wave's first token
  bool in;
  RP_DEV Place(const ScanArgs& p) {
    tid = threadIdx.x;
    lane = tid & 63;
    w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rest = (int)(blockIdx.x / (unsigned)p.blocks), cb = (int)blockIdx.x - rest * p.blocks;
    b = rest / p.chunks;
    chunk = rest - b * p.chunks;
    ch = cb * BLOCK_CH + LANES * lane;
    in = ch < p.c;
    t0 = chunk * CHUNK + w * TOK;
    len = p.len ? min(max(p.len[b], 0), p.seq) : p.seq;
  }
  RP_DEV long at(const ScanArgs& p) const { return ((long)b * p.chunks + chunk) * p.c + ch; }      // in [batch, chunks, c]
};
// Tokens t0 .. t0 + 7 of a tensor, zero behind the length.
RP_DEV void load_rows(const bf16* base, long ld, const Place& s, int seq, uint2 (&r)[TOK]) {
  const bf16* const src = base + ((long)s.b * seq + s.t0) * ld + s.ch;
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    r[i] = make_uint2(0u, 0u);
    if (s.in && s.t0 + i < s.len) r[i] = *reinterpret_cast<const uint2*>(src + i * ld);
  }
}
// The gates are made again from g for every use: kept from one to the next they would be the registers of half of the waves (244 instead of 110 for the backward kernel).
RP_DEV void forget(uint2 (&r)[TOK]) {
#pragma unroll
  for (int i = 0; i < TOK; ++i) asm volatile("" : "+v"(r[i].x), "+v"(r[i].y));
}
// bit i: token t0 + i begins a document
RP_DEV uint32_t load_first(const ScanArgs& p, const Place& s) {
  uint32_t m = 0;
  if (p.first) {
    const unsigned char* const src = p.first + (long)s.b * p.seq + s.t0;
#pragma unroll
    for (int i = 0; i < TOK; ++i)
      if (s.t0 + i < s.len) m |= (src[i] != 0 ? 1u : 0u) << i;
  }
  return m;
}

// The map of a wave's eight tokens, forwards (state) or backwards (mu).  A token behind the length has the map (1, 0); what decides is the same in all lanes, so the
// selects cost less than branches around the registers that the tokens are in.
template <int W>
RP_DEV void wave_map(const uint2 (&gr)[TOK], const uint2 (&xr)[TOK], uint32_t first, const Place& s, f4& A, f4& B) {
  A = f4{1.f, 1.f, 1.f, 1.f};
  B = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const bool live = s.t0 + i < s.len, begins = first >> i & 1;
    const f4 g = unpack(gr[i]), x = unpack(xr[i]);
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      float f, r;
      gates(g[e], f, r);
      const float u = weight<W>(f, r) * x[e];
      const float a = begins ? 0.f : A[e] * f, b = begins ? u : __builtin_fmaf(f, B[e], u);
      A[e] = live ? a : A[e];
      B[e] = live ? b : B[e];
    }
  }
}
RP_DEV void wave_map_back(const uint2 (&gr)[TOK], const uint2 (&dyr)[TOK], uint32_t first, const Place& s, f4& A, f4& B) {
  A = f4{1.f, 1.f, 1.f, 1.f};
  B = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < TOK; ++j) {
    const int i = TOK - 1 - j;
    const bool live = s.t0 + i < s.len, begins = first >> i & 1;
    const f4 g = unpack(gr[i]), dy = unpack(dyr[i]);
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      float f, r;
      gates(g[e], f, r);
      const float a = begins ? 0.f : A[e] * f, b = begins ? 0.f : f * (dy[e] + B[e]);
      A[e] = live ? a : A[e];
      B[e] = live ? b : B[e];
    }
  }
}

// What comes out of the map (a, b), and (a, b) after (A, B).  a = 0 where a document begins: what was before is not multiplied by it, or an infinity there would
// reach every document behind it.
RP_DEV float through(float a, float b, float h) { return a == 0.f ? b : __builtin_fmaf(a, h, b); }

// ------------------------------------------------------------------------------------------------ the chunks' maps
template <int W, bool BACK>
__global__ void __launch_bounds__(64 * NW) scan_map_kernel(const ScanArgs p) {
  __shared__ f4 As[NW][64], Bs[NW][64];
  const Place s(p);
  uint2 gr[TOK], xr[TOK];
  load_rows(p.g, p.ldg, s, p.seq, gr);
  if (BACK) load_rows(p.dy, p.lddy, s, p.seq, xr);
  else load_rows(p.x, p.ldx, s, p.seq, xr);
  const uint32_t first = load_first(p, s);
  f4 A, B;
  if (BACK) wave_map_back(gr, xr, first, s, A, B);
  else wave_map<W>(gr, xr, first, s, A, B);
  As[s.w][s.lane] = A;
  Bs[s.w][s.lane] = B;
  __syncthreads();
  if (s.w != 0 || !s.in) return;
#pragma unroll
  for (int i = 1; i < NW; ++i) {
    const int u = BACK ? NW - 1 - i : i;
    if (i == 1) {
      A = As[BACK ? NW - 1 : 0][s.lane];
      B = Bs[BACK ? NW - 1 : 0][s.lane];
    }
    const f4 a = As[u][s.lane], b = Bs[u][s.lane];
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      A[e] = a[e] == 0.f ? 0.f : A[e] * a[e];
      B[e] = through(a[e], b[e], B[e]);
    }
  }
  float4* const out = reinterpret_cast<float4*>(p.agg + s.at(p));
  out[0] = make_float4(A[0], B[0], A[1], B[1]);
  out[1] = make_float4(A[2], B[2], A[3], B[3]);
}

// What every chunk starts from: a thread takes a channel, chunk by chunk.
template <bool BACK>
__global__ void __launch_bounds__(64) scan_carry_kernel(const ScanArgs p, float* carry) {
  constexpr int AHEAD = 16;
  const long i = (long)blockIdx.x * 64 + threadIdx.x;
  if (i >= (long)p.batch * p.c) return;
  const int b = (int)(i / p.c), ch = (int)(i - (long)b * p.c);
  const float* const start = BACK ? p.dlast : p.h0;
  float h = start ? start[i] : 0.f;
  const long base = (long)b * p.chunks * p.c + ch;
  for (int k0 = 0; k0 < p.chunks; k0 += AHEAD) {
    float2 m[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int k = min(k0 + j, p.chunks - 1);
      m[j] = p.agg[base + (long)(BACK ? p.chunks - 1 - k : k) * p.c];
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int k = k0 + j;
      if (k < p.chunks) {
        carry[base + (long)(BACK ? p.chunks - 1 - k : k) * p.c] = h;
        h = through(m[j].x, m[j].y, h);
      }
    }
  }
  float* const end = BACK ? p.dh0 : p.last;
  if (end) end[i] = h;
}

// ------------------------------------------------------------------------------------------------ outputs
// The maps of the waves before (behind) this one on what the chunk starts from.
template <bool BACK>
RP_DEV f4 enter(const f4 (&As)[NW][64], const f4 (&Bs)[NW][64], const Place& s, f4 h) {
  for (int i = 0; i < (BACK ? NW - 1 - s.w : s.w); ++i) {
    const int u = BACK ? NW - 1 - i : i;
    const f4 a = As[u][s.lane], b = Bs[u][s.lane];
#pragma unroll
    for (int e = 0; e < LANES; ++e) h[e] = through(a[e], b[e], h[e]);
  }
  return h;
}
// ONE: a sequence is one chunk, which starts from the call's own state
template <bool ONE>
RP_DEV f4 chunk_start(const ScanArgs& p, const Place& s, const float* carry, const float* given) {
  const float* const src = ONE ? given : carry;
  if (!src || !s.in) return f4{0.f, 0.f, 0.f, 0.f};
  return *reinterpret_cast<const f4*>(src + (ONE ? (long)s.b * p.c + s.ch : s.at(p)));
}

template <int W, bool ONE>
__global__ void __launch_bounds__(64 * NW) scan_fwd_kernel(const ScanArgs p, const float* carry) {
  __shared__ f4 As[NW][64], Bs[NW][64];
  const Place s(p);
  uint2 gr[TOK], xr[TOK];
  load_rows(p.g, p.ldg, s, p.seq, gr);
  load_rows(p.x, p.ldx, s, p.seq, xr);
  const uint32_t first = load_first(p, s);
  const f4 start = chunk_start<ONE>(p, s, carry, p.h0);
  f4 A, B;
  wave_map<W>(gr, xr, first, s, A, B);
  As[s.w][s.lane] = A;
  Bs[s.w][s.lane] = B;
  __syncthreads();
  f4 h = enter<false>(As, Bs, s, start);
  if (ONE && s.in && s.w == 0 && p.states && p.seq > 0) *reinterpret_cast<f4*>(p.states + s.at(p)) = start;
  bf16* const out = p.y + ((long)s.b * p.seq + s.t0) * p.ldy + s.ch;
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const bool live = s.t0 + i < s.len, begins = first >> i & 1;
    const f4 g = unpack(gr[i]), x = unpack(xr[i]);
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      float f, r;
      gates(g[e], f, r);
      const float u = weight<W>(f, r) * x[e];
      const float next = begins ? u : __builtin_fmaf(f, h[e], u);
      h[e] = live ? next : h[e];
    }
    if (s.in && s.t0 + i < p.seq) *reinterpret_cast<uint2*>(out + i * p.ldy) = live ? pack(h) : make_uint2(0u, 0u);
  }
  if (ONE && p.last && s.w == NW - 1 && s.in) *reinterpret_cast<f4*>(p.last + (long)s.b * p.c + s.ch) = h;      // (waves without tokens pass the state on)
}

template <int W, bool ONE>
__global__ void __launch_bounds__(64 * NW, 4) scan_bwd_kernel(const ScanArgs p, const float* carry) {
  __shared__ f4 As[NW][64], Bs[NW][64], Ab[NW][64], Bb[NW][64];
  const Place s(p);
  uint2 gr[TOK], xr[TOK], dyr[TOK];
  load_rows(p.g, p.ldg, s, p.seq, gr);
  load_rows(p.x, p.ldx, s, p.seq, xr);
  load_rows(p.dy, p.lddy, s, p.seq, dyr);
  const uint32_t first = load_first(p, s);
  f4 h = s.in && p.seq > 0 ? *reinterpret_cast<const f4*>(p.states + s.at(p)) : f4{0.f, 0.f, 0.f, 0.f};
  f4 mu = chunk_start<ONE>(p, s, carry, p.dlast);
  f4 A, B;
  wave_map<W>(gr, xr, first, s, A, B);
  As[s.w][s.lane] = A;
  Bs[s.w][s.lane] = B;
  forget(gr);
  wave_map_back(gr, dyr, first, s, A, B);
  Ab[s.w][s.lane] = A;
  Bb[s.w][s.lane] = B;
  __syncthreads();
  h = enter<false>(As, Bs, s, h);
  mu = enter<true>(Ab, Bb, s, mu);
  forget(gr);
  f4 before[TOK];      // h_(t-1), 0 where a document begins
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const bool live = s.t0 + i < s.len, begins = first >> i & 1;
    const f4 g = unpack(gr[i]), x = unpack(xr[i]);
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      float f, r;
      gates(g[e], f, r);
      const float u = weight<W>(f, r) * x[e];
      before[i][e] = begins ? 0.f : h[e];
      const float next = begins ? u : __builtin_fmaf(f, h[e], u);
      h[e] = live ? next : h[e];
    }
  }
  forget(gr);
  bf16* const dx = p.dx + ((long)s.b * p.seq + s.t0) * p.lddx + s.ch;
  bf16* const dg = p.dg + ((long)s.b * p.seq + s.t0) * p.lddg + s.ch;
#pragma unroll
  for (int j = 0; j < TOK; ++j) {
    const int i = TOK - 1 - j;
    const bool live = s.t0 + i < s.len, begins = first >> i & 1;
    const f4 g = unpack(gr[i]), x = unpack(xr[i]), dy = unpack(dyr[i]);
    f4 gx, gg;
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      float f, r;
      gates(g[e], f, r);
      const float lam = dy[e] + mu[e];
      gx[e] = live ? weight<W>(f, r) * lam : 0.f;
      gg[e] = live ? lam * (before[i][e] * (f * r) + x[e] * weight_slope<W>(f, r)) : 0.f;
      const float next = begins ? 0.f : f * lam;
      mu[e] = live ? next : mu[e];
    }
    if (s.in && s.t0 + i < p.seq) {
      *reinterpret_cast<uint2*>(dx + i * p.lddx) = pack(gx);
      *reinterpret_cast<uint2*>(dg + i * p.lddg) = pack(gg);
    }
  }
  if (ONE && p.dh0 && s.w == 0 && s.in) *reinterpret_cast<f4*>(p.dh0 + (long)s.b * p.c + s.ch) = mu;
}

int chunks_of(int seq) { return (seq + CHUNK - 1) / CHUNK; }

template <int W>
hipError_t fwd(hipStream_t st, const ScanArgs& p, float* carry) {
  const dim3 grid((unsigned)p.batch * p.chunks * p.blocks), block(64 * NW);
  if (p.chunks == 1) {
    RP_LAUNCH((scan_fwd_kernel<W, true>), grid, block, 0, st, p, carry);
    return hipGetLastError();
  }
  RP_LAUNCH((scan_map_kernel<W, false>), grid, block, 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  RP_LAUNCH((scan_carry_kernel<false>), dim3((unsigned)(((long)p.batch * p.c + 63) / 64)), dim3(64), 0, st, p, carry);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  RP_LAUNCH((scan_fwd_kernel<W, false>), grid, block, 0, st, p, carry);
  return hipGetLastError();
}
template <int W>
hipError_t bwd(hipStream_t st, const ScanArgs& p, float* carry) {
  const dim3 grid((unsigned)p.batch * p.chunks * p.blocks), block(64 * NW);
  if (p.chunks == 1) {
    RP_LAUNCH((scan_bwd_kernel<W, true>), grid, block, 0, st, p, carry);
    return hipGetLastError();
  }
  RP_LAUNCH((scan_map_kernel<W, true>), grid, block, 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  RP_LAUNCH((scan_carry_kernel<true>), dim3((unsigned)(((long)p.batch * p.c + 63) / 64)), dim3(64), 0, st, p, carry);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  RP_LAUNCH((scan_bwd_kernel<W, false>), grid, block, 0, st, p, carry);
  return hipGetLastError();
}

}  // namespace

void k_scan_sizes(int batch, int seq, int c, size_t* states, size_t* scratch) {
  const size_t n = (size_t)batch * chunks_of(seq) * c;
  *states = 4 * n;
  *scratch = chunks_of(seq) > 1 ? 12 * n : 0;
}

hipError_t k_scan_fwd(hipStream_t st, int weight, const ScanArgs& args, void* scratch) {
  ScanArgs p = args;
  p.chunks = p.seq ? chunks_of(p.seq) : 1;      // without tokens the state is passed on
  p.blocks = (p.c + BLOCK_CH - 1) / BLOCK_CH;
  if (p.batch == 0 || p.c == 0) return hipSuccess;
  const size_t n = (size_t)p.batch * p.chunks * p.c;
  p.agg = static_cast<float2*>(scratch);
  float* const carry = p.states ? p.states : reinterpret_cast<float*>(p.agg + n);
  return weight == 0 ? fwd<0>(st, p, carry) : weight == 1 ? fwd<1>(st, p, carry) : fwd<2>(st, p, carry);
}

hipError_t k_scan_bwd(hipStream_t st, int weight, const ScanArgs& args, void* scratch) {
  ScanArgs p = args;
  p.chunks = p.seq ? chunks_of(p.seq) : 1;
  p.blocks = (p.c + BLOCK_CH - 1) / BLOCK_CH;
  if (p.batch == 0 || p.c == 0) return hipSuccess;
  const size_t n = (size_t)p.batch * p.chunks * p.c;
  p.agg = static_cast<float2*>(scratch);
  float* const carry = reinterpret_cast<float*>(p.agg + n);
  return weight == 0 ? bwd<0>(st, p, carry) : weight == 1 ? bwd<1>(st, p, carry) : bwd<2>(st, p, carry);
}
