// Gated linear recurrence over the tokens of a sequence, every channel by itself, forward and backward.
//
//   f_t = sigmoid(g_t);  h_t = f_t h_(t-1) + w_t x_t,  w_t = 1 | 1 - f_t | sqrt(1 - f_t^2);  y_t = h_t
//   lam_t = dy_t + mu_(t+1),  mu_t = f_t lam_t;  dx_t = w_t lam_t;  dg_t = lam_t (h_(t-1) f_t (1 - f_t) + x_t dw_t/dg_t);  dh_0 = mu_0
//
// Where a document starts, f_t of the recurrence is 0 (the state before counts for nothing, and gets no gradient).  Behind a sequence's length the state is kept as it is.
// 1 - f is taken as sigmoid(-g): a gate near one keeps its distance from it.
//
// h_t = a_t h_(t-1) + b_t is a scan over the maps (a, b), which compose as (a2, b2) after (a1, b1) = (a2 a1, a2 b1 + b2).  Chunks of 128 tokens by 128 channels; a wave
// has 16 tokens, a lane two channels, all in registers, so every input is read once: a workgroup makes its chunk's map, publishes it, finds out what its chunk starts from, and writes
// the outputs.  That it finds by looking back over the chunks before (the decoupled look-back of Merrill and Garland, Single-pass parallel prefix scan, 2016): from the nearest one whose
// end state is there, through the maps of those in between.  Workgroups take their
// chunks in order of time by a counter, so whoever waits waits for workgroups that have started and that wait only for earlier ones; the first waits for none.  A
// chunk's end state is the same sequence of operations wherever the looking ended: the results do not depend on timing.
// The backward pass is the same from behind; h_(t-1) is made again from the states that the forward pass left, in fp32 (4 bytes for 128 tokens), not from y, which is
// rounded.  States, sums and products are fp32 throughout.
//
// What bounds it (w = 1 - f; forward and backward in turn, three sets of inputs): memory where the chunks need not wait for one another (128 sequences of 128 tokens, 4096 channels: forward 84 us,
// backward 131, 4.8 and 5.1 TB/s).  One sequence of 16384 tokens takes 103 and 139 us, 3.9 and 4.8 TB/s: a workgroup holds its registers while it waits for the ones before it, and two of them share a
// CU; with documents that begin in it every 1000 tokens, whose waves go by selects and read a byte a token besides, 120 and 166.  4 x 1021 tokens of 2880 channels, 736 workgroups for 512 places
// (those behind a length too), 29 and 40 us.  When the 16384 tokens took 106 and 148 us: chunks of 64 tokens (half the tokens a wave, or half the waves) 150 to 175 and 180, 16 waves of 8 tokens or of 16
// behind, too; three workgroups a CU spill (119), a backward pass without its few spills has room for one (169).
#include <type_traits>

#include "pack_ops.hpp"

namespace {

constexpr int NW = 8, TOK = 16, CHUNK = NW * TOK, LANES = 2, BLOCK_CH = 64 * LANES;

typedef float fch __attribute__((ext_vector_type(LANES)));      // a lane's channels
typedef uint32_t raw_t;                                          // as they are in memory

RP_DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
RP_DEV fch unpack(raw_t u) { return fch{bf16_lo(u), bf16_hi(u)}; }
RP_DEV raw_t pack(const fch& v) { return pack_bf16x2(v[0], v[1]); }

// sigmoid(g) and sigmoid(-g): the smaller one, t, from an exponential that is at most 1, so that it keeps its relative precision (the exponential's argument is
// rounded: 2^-22 or so), the larger one as 1 - t, which is then one rounding off.  Errors of f add up over as many tokens as a gate remembers.  Kept between uses: t
// with g's sign.
RP_DEV float smaller_gate(float g) {
  const float e = fast_exp2(fabsf(g) * -1.4426950408889634f);
  return __builtin_copysignf(e * __builtin_amdgcn_rcpf(1.f + e), g);      // (NaN stays NaN)
}
RP_DEV void gates(float ts, float& f, float& r) {
  const float t = fabsf(ts), s = 1.f - t;
  const bool below = __float_as_int(ts) < 0;      // (t may be 0)
  f = below ? t : s;
  r = below ? s : t;
}
template <int W>
RP_DEV float weight(float f, float r) { return W == 0 ? 1.f : W == 1 ? r : __builtin_amdgcn_sqrtf(r * (1.f + f)); }
// dw / dg: 0, -f r, -f^2 r / w = -f^2 sqrt(r / (1 + f))
template <int W>
RP_DEV float weight_slope(float f, float r) { return W == 0 ? 0.f : W == 1 ? -f * r : -f * f * __builtin_amdgcn_sqrtf(r * __builtin_amdgcn_rcpf(1.f + f)); }

// A workgroup's place: the channels change fastest, so that workgroups side by side read neighbouring pieces of the same rows, and time slowest.
struct Place {
  int b, chunk, ch, tid, lane, w, t0, len;      // t0: the wave's first token
  bool in, full;      // full: all of the wave's tokens are in use
  RP_DEV Place(const ScanArgs& p, int id, bool back) {
    tid = threadIdx.x;
    lane = tid & 63;
    w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rest = __builtin_amdgcn_readfirstlane(id / p.blocks), cb = id - rest * p.blocks;
    chunk = __builtin_amdgcn_readfirstlane(rest / p.batch);
    b = rest - chunk * p.batch;
    if (back) chunk = p.chunks - 1 - chunk;
    ch = cb * BLOCK_CH + LANES * lane;
    in = ch < p.c;
    t0 = chunk * CHUNK + w * TOK;
    len = __builtin_amdgcn_readfirstlane(p.len ? min(max(p.len[b], 0), p.seq) : p.seq);
    full = t0 + TOK <= len;
  }
  RP_DEV long at(const ScanArgs& p) const { return ((long)b * p.chunks + chunk) * p.c + ch; }      // in [batch, chunks, c]
};
// A wave's tokens of a tensor, through a descriptor that begins at the first of them and ends behind the last one in use: the others read as zero, and are not written.
struct TokenRows {
  __amdgpu_buffer_rsrc_t rsrc;
  int lane, step;      // byte offsets of the lane's channels (a lane without channels: out of range), and from token to token
  RP_DEV TokenRows(const bf16* base, long ld, const Place& s, const ScanArgs& p, int end /* of the sequence's tokens in use */) {
    const int n = min(max(end - s.t0, 0), TOK);
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(base + ((long)s.b * p.seq + s.t0) * ld), 0, n ? (int)(((n - 1) * ld + p.c) * 2) : 0, 0x00020000);
    lane = s.in ? s.ch * 2 : (int)0x80000000;
    step = (int)(ld * 2);
  }
  RP_DEV void load(raw_t (&r)[TOK]) const {
#pragma unroll
    for (int i = 0; i < TOK; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, lane, i * step, 0);
  }
  RP_DEV void store(int i, raw_t v) const { __builtin_amdgcn_raw_buffer_store_b32(v, rsrc, lane, i * step, 0); }
};
// The compiler is not to keep what it has made of these for a later use: it is made again for less than the registers would cost.
RP_DEV void forget(raw_t (&r)[TOK]) {
#pragma unroll
  for (int i = 0; i < TOK; ++i) asm volatile("" : "+v"(r[i]));
}
RP_DEV void forget(fch (&r)[TOK]) {
#pragma unroll
  for (int i = 0; i < TOK; ++i) asm volatile("" : "+v"(r[i]));
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

// PLAIN: the wave is full and no token begins a document; else selects, by what is the same in all lanes.
template <int W, bool PLAIN>
RP_DEV float step(float ts, float x, bool live, bool begins, float h) {      // h_t from h_(t-1)
  float f, r;
  gates(ts, f, r);
  const float u = weight<W>(f, r) * x;
  const float next = !PLAIN && begins ? u : __builtin_fmaf(f, h, u);
  return PLAIN || live ? next : h;
}

// What comes out of the map (a, b), and (a, b) after (A, B).  a = ANEW, -0, where a document begins on the way: what was before is not multiplied by it, or an infinity there would reach every
// document behind it.  A product of gates that is too small for fp32 (128 of g = -2) is +0, and NaN and infinities come through that as they do token by token.
constexpr float ANEW = -0.f;
RP_DEV bool is_anew(float a) { return __float_as_uint(a) == 0x80000000u; }      // (gates are no less than +0: -0 times one stays)
template <bool EXACT>
RP_DEV fch through(const fch& a, const fch& b, const fch& h) {
  fch to;
#pragma unroll
  for (int e = 0; e < LANES; ++e) {
    to[e] = is_anew(a[e]) ? b[e] : __builtin_fmaf(a[e], h[e], b[e]);
    if (EXACT && a[e] == 0.f && !is_anew(a[e]) && __builtin_isinf(h[e])) to[e] = h[e] + b[e];
  }
  return to;
}
// A walk through maps: without asking for infinities first, which then come out as 0 times them, NaN.  (Asked for in every map: 16384 tokens of 4096 2 % more.)
template <typename F>
RP_DEV fch walk(F&& f) {
  const fch h = f(std::false_type{});
  return __any(h[0] != h[0] || h[1] != h[1]) ? f(std::true_type{}) : h;
}
RP_DEV float both(float a, float A) { return is_anew(a) ? ANEW : a * A; }

// The map of a wave's tokens, forwards (state), with the gates on the way, or backwards (mu).  A token behind the length has the map (1, 0).
template <int W, bool PLAIN>
RP_DEV void wave_map(const raw_t (&gr)[TOK], const raw_t (&xr)[TOK], fch (&ts)[TOK], uint32_t first, const Place& s, fch& A, fch& B) {
  A = fch{1.f, 1.f};
  B = fch{0.f, 0.f};
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const bool live = s.t0 + i < s.len, begins = first >> i & 1;
    const fch g = unpack(gr[i]), x = unpack(xr[i]);
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      ts[i][e] = smaller_gate(g[e]);
      float f, r;
      gates(ts[i][e], f, r);
      const float a = !PLAIN && begins ? ANEW : A[e] * f;
      A[e] = PLAIN || live ? a : A[e];
      B[e] = step<W, PLAIN>(ts[i][e], x[e], live, begins, B[e]);
    }
  }
}
template <bool PLAIN>
RP_DEV void wave_map_back(const raw_t (&dyr)[TOK], const fch (&ts)[TOK], uint32_t first, const Place& s, fch& A, fch& B) {
  A = fch{1.f, 1.f};
  B = fch{0.f, 0.f};
#pragma unroll
  for (int j = 0; j < TOK; ++j) {
    const int i = TOK - 1 - j;
    const bool live = s.t0 + i < s.len, begins = first >> i & 1;
    const fch dy = unpack(dyr[i]);
#pragma unroll
    for (int e = 0; e < LANES; ++e) {
      float f, r;
      gates(ts[i][e], f, r);
      const float a = !PLAIN && begins ? ANEW : A[e] * f, b = !PLAIN && begins ? 0.f : f * (dy[e] + B[e]);
      A[e] = PLAIN || live ? a : A[e];
      B[e] = PLAIN || live ? b : B[e];
    }
  }
}
template <typename F>
RP_DEV void plain_or_not(const Place& s, uint32_t first, F&& f) {
  if (s.full && first == 0u) f(std::true_type{});      // uniform
  else f(std::false_type{});
}

// ------------------------------------------------------------------------------------------------ between chunks
// What a chunk tells the ones behind it of a channel, 64 bits that are written and read at once: nothing yet (0); its map: b, and a (0 .. 1, or NaN) with the sign bit
// set, or -2 for ANEW; or its end state, with all bits set above it, which is what comes out of a map of ANEW.
typedef unsigned long long word_t;
constexpr uint32_t STATE = 0xffffffffu, MAP_ANEW = 0xc0000000u;
RP_DEV word_t map_word(float a, float b) {
  return (word_t)(is_anew(a) ? MAP_ANEW : (a != a ? 0x7fc00000u : __float_as_uint(a)) | 0x80000000u) << 32 | __float_as_uint(b);
}
RP_DEV float map_factor(uint32_t hi) { return hi >= MAP_ANEW && hi != 0xffc00000u ? ANEW : __uint_as_float(hi & 0x7fffffffu); }
RP_DEV word_t state_word(float h) { return (word_t)STATE << 32 | __float_as_uint(h); }
RP_DEV void publish(word_t* at, word_t w) { __hip_atomic_store(at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
RP_DEV word_t look(const word_t* at) { return __hip_atomic_load(const_cast<word_t*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// What a chunk starts from, for all waves of its workgroup.  Wave 0 publishes the chunk's map; every wave then waits for EACH of the 8 EACH chunks before and puts what they say into
// LDS, and all of them go from the nearest end state through the maps behind it.  Where none of those chunks has its end state yet, they look again.  EACH is 4 where all of a launch's
// workgroups are on the chip at once, and the chain of looks is what takes the time (18467 tokens of 72 channels: forward 34.5 -> 22 us, backward 36.7 -> 23), else 1 (16384 tokens of 4096:
// 103 and 139 us, with 4 112 and 149).
// `given`: the state before the first chunk (behind the last one, BACK), in LDS; end: wave 0's, the chunk's own end state.
template <int EACH>
struct Looks {
  fch a[EACH * NW][64], b[EACH * NW][64];
  int state[EACH * NW];
};
template <int EACH, bool BACK>
RP_DEV fch start_of(const ScanArgs& p, const Place& s, const fch (&As)[NW][64], const fch (&Bs)[NW][64], Looks<EACH>& looks, const fch (&given)[64], fch& end) {
  const int before = BACK ? p.chunks - 1 - s.chunk : s.chunk;
  word_t* const mine = p.words + (s.in ? s.at(p) : 0);
  fch A = As[BACK ? NW - 1 : 0][s.lane], B = Bs[BACK ? NW - 1 : 0][s.lane];
  if (s.w == 0) {
    const fch B0 = B;
    B = walk([&](auto exact) {
      fch x = B0;
#pragma unroll
      for (int i = 1; i < NW; ++i) {
        const int u = BACK ? NW - 1 - i : i;
        x = through<decltype(exact)::value>(As[u][s.lane], Bs[u][s.lane], x);
      }
      return x;
    });
#pragma unroll
    for (int i = 1; i < NW; ++i) {
      const fch a = As[BACK ? NW - 1 - i : i][s.lane];
#pragma unroll
      for (int e = 0; e < LANES; ++e) A[e] = both(a[e], A[e]);
    }
    if (before > 0 && s.in)
#pragma unroll
      for (int e = 0; e < LANES; ++e) publish(mine + e, map_word(A[e], B[e]));
  }
  fch h = given[s.lane];
  if (before > 0) {      // uniform over the workgroup
    int from;
    for (;;) {
      bool there[EACH], state[EACH];
      word_t w[EACH][LANES];
      for (;;) {      // ends: those chunks' workgroups took their places before this one
        bool all = true;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
          const int n = s.w + k * NW;      // that many chunks between
          const word_t* const theirs = mine + (BACK ? 1 : -1) * (long)(n + 1) * p.c;
#pragma unroll
          for (int e = 0; e < LANES; ++e) w[k][e] = s.in && n < before ? look(theirs + e) : state_word(0.f);
        }
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
          there[k] = state[k] = true;
#pragma unroll
          for (int e = 0; e < LANES; ++e) {
            there[k] = there[k] && (uint32_t)(w[k][e] >> 32) != 0u;
            state[k] = state[k] && (uint32_t)(w[k][e] >> 32) == STATE;
          }
          all = all && there[k];
        }
        if (__all(all)) break;
        __builtin_amdgcn_s_sleep(1);
      }
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        const int n = s.w + k * NW;
        fch a, b;
#pragma unroll
        for (int e = 0; e < LANES; ++e) {
          a[e] = map_factor((uint32_t)(w[k][e] >> 32));
          b[e] = __uint_as_float((uint32_t)w[k][e]);
        }
        looks.a[n][s.lane] = a;
        looks.b[n][s.lane] = b;
        const bool is = __all(state[k]) && n < before;
        if (s.lane == 0) looks.state[n] = is;
      }
      __syncthreads();
      from = -1;
#pragma unroll
      for (int i = EACH * NW - 1; i >= 0; --i)
        if (looks.state[i]) from = i;
      if (__builtin_amdgcn_readfirstlane(from) >= 0) break;
      __syncthreads();      // all have seen that there is none
    }
    from = __builtin_amdgcn_readfirstlane(from);
    h = walk([&](auto exact) {
      fch x = looks.b[from][s.lane];
      for (int i = from - 1; i >= 0; --i) x = through<decltype(exact)::value>(looks.a[i][s.lane], looks.b[i][s.lane], x);
      return x;
    });
  }
  if (s.w == 0) {
    end = walk([&](auto exact) { return through<decltype(exact)::value>(A, B, h); });
    if (s.in)
#pragma unroll
      for (int e = 0; e < LANES; ++e) publish(mine + e, state_word(end[e]));
  }
  return h;
}

__global__ void __launch_bounds__(256) scan_clear_kernel(uint4* to, long n) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) to[i] = make_uint4(0u, 0u, 0u, 0u);
}

// ------------------------------------------------------------------------------------------------ outputs
// The maps of the waves before (behind) this one on what the chunk starts from.
template <bool BACK>
RP_DEV fch enter(const fch (&As)[NW][64], const fch (&Bs)[NW][64], const Place& s, fch h) {
  return walk([&](auto exact) {
    fch x = h;
    for (int i = 0; i < (BACK ? NW - 1 - s.w : s.w); ++i) {
      const int u = BACK ? NW - 1 - i : i;
      x = through<decltype(exact)::value>(As[u][s.lane], Bs[u][s.lane], x);
    }
    return x;
  });
}
// EACH 0: a sequence is one chunk, which starts from the call's own state
template <int EACH>
RP_DEV int take_place(const ScanArgs& p, int* lds) {
  if (EACH == 0) {
    int id = (int)blockIdx.x;
    asm volatile("" : "+s"(id)::"memory");      // (with its number known the backward pass spills inside its loops: 128 sequences of 128 tokens 181 us instead of 139, plain weights)
    return id;
  }
  if (threadIdx.x == 0) *lds = (int)atomicAdd(p.counter, 1u);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(*lds);
}
RP_DEV fch given_state(const float* src, const ScanArgs& p, const Place& s) {
  return src && s.in ? *reinterpret_cast<const fch*>(src + (long)s.b * p.c + s.ch) : fch{0.f, 0.f};
}
// The call's own state goes to LDS, before the barrier behind the waves' maps: it is read by the first chunk's wave 0 alone (the last chunk's, BACK), and once that barrier is passed it
// is not read again, so that whoever is told of this chunk's end may write the state in its place (`last` may be h0, dh0 dlast).
template <bool BACK>
RP_DEV void keep_given(const float* src, const ScanArgs& p, const Place& s, fch (&given)[64]) {
  if (s.w == 0) given[s.lane] = given_state(s.chunk == (BACK ? p.chunks - 1 : 0) ? src : nullptr, p, s);      // uniform
}
// What the chunk starts from; the waves have put their maps into LDS, wave 0 the call's own state.  The state behind the last chunk goes to `last`.
template <int EACH, bool BACK>
RP_DEV fch chunk_start(const ScanArgs& p, const Place& s, const fch (&As)[NW][64], const fch (&Bs)[NW][64], Looks<EACH ? EACH : 1>* looks, const fch (&given)[64], float* last) {
  fch h = given[s.lane];
  if constexpr (EACH > 0) {
    fch end;
    h = start_of<EACH, BACK>(p, s, As, Bs, *looks, given, end);
    if (last && s.w == 0 && s.in && s.chunk == (BACK ? 0 : p.chunks - 1)) *reinterpret_cast<fch*>(last + (long)s.b * p.c + s.ch) = end;
  }
  return h;
}

template <int W, int EACH>
__global__ void __launch_bounds__(64 * NW) scan_fwd_kernel(const ScanArgs p) {
  __shared__ fch As[NW][64], Bs[NW][64], given[64];
  __shared__ Looks<EACH ? EACH : 1> looks;
  __shared__ int place;
  const Place s(p, take_place<EACH>(p, &place), false);
  raw_t gr[TOK], xr[TOK];
  TokenRows(p.g, p.ldg, s, p, s.len).load(gr);
  TokenRows(p.x, p.ldx, s, p, s.len).load(xr);
  const uint32_t first = load_first(p, s);
  fch ts[TOK];
  {
    fch A, B;
    plain_or_not(s, first, [&](auto plain) { wave_map<W, decltype(plain)::value>(gr, xr, ts, first, s, A, B); });
    As[s.w][s.lane] = A;
    Bs[s.w][s.lane] = B;
  }
  keep_given<false>(p.h0, p, s, given);
  __syncthreads();
  const fch start = chunk_start<EACH, false>(p, s, As, Bs, &looks, given, p.last);
  fch h = enter<false>(As, Bs, s, start);
  if (s.in && s.w == 0 && p.states && p.seq > 0) *reinterpret_cast<fch*>(p.states + s.at(p)) = start;
  const TokenRows out(p.y, p.ldy, s, p, p.seq);
  forget(xr);
  forget(ts);
  plain_or_not(s, first, [&](auto plain) {
    constexpr bool PLAIN = decltype(plain)::value;
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
      const bool live = s.t0 + i < s.len, begins = first >> i & 1;
      const fch x = unpack(xr[i]);
#pragma unroll
      for (int e = 0; e < LANES; ++e) h[e] = step<W, PLAIN>(ts[i][e], x[e], live, begins, h[e]);
      out.store(i, PLAIN || live ? pack(h) : 0u);
      }
  });
  if (EACH == 0 && p.last && s.w == NW - 1 && s.in) *reinterpret_cast<fch*>(p.last + (long)s.b * p.c + s.ch) = h;      // (waves without tokens pass the state on)
}

template <int W, int EACH>
__global__ void __launch_bounds__(64 * NW, 4) scan_bwd_kernel(const ScanArgs p) {
  __shared__ fch As[NW][64], Bs[NW][64], Ab[NW][64], Bb[NW][64], given[64];
  __shared__ Looks<EACH ? EACH : 1> looks;
  __shared__ int place;
  const Place s(p, take_place<EACH>(p, &place), true);
  raw_t xr[TOK], dyr[TOK];
  uint32_t first;
  fch ts[TOK];
  fch h = s.in && p.seq > 0 ? *reinterpret_cast<const fch*>(p.states + s.at(p)) : fch{0.f, 0.f};
  {
    raw_t gr[TOK];
    TokenRows(p.g, p.ldg, s, p, s.len).load(gr);
    TokenRows(p.x, p.ldx, s, p, s.len).load(xr);
    TokenRows(p.dy, p.lddy, s, p, s.len).load(dyr);
    first = load_first(p, s);
    plain_or_not(s, first, [&](auto plain) {
      constexpr bool PLAIN = decltype(plain)::value;
      fch A, B;
      wave_map<W, PLAIN>(gr, xr, ts, first, s, A, B);
      As[s.w][s.lane] = A;
      Bs[s.w][s.lane] = B;
      forget(ts);
      wave_map_back<PLAIN>(dyr, ts, first, s, A, B);
      Ab[s.w][s.lane] = A;
      Bb[s.w][s.lane] = B;
    });
  }
  if (EACH > 0) keep_given<true>(p.dlast, p, s, given);
  __syncthreads();
  // (one chunk: every wave reads the state for itself, and dh0 waits for all of them; through LDS the compiler spills in other places, 128 sequences of 128 tokens 143 us instead of 130)
  fch mu;
  if constexpr (EACH == 0) mu = given_state(p.dlast, p, s);
  else mu = chunk_start<EACH, true>(p, s, Ab, Bb, &looks, given, p.dh0);
  h = enter<false>(As, Bs, s, h);
  mu = enter<true>(Ab, Bb, s, mu);
  forget(xr);
  forget(dyr);
  forget(ts);
  const TokenRows dx(p.dx, p.lddx, s, p, p.seq), dg(p.dg, p.lddg, s, p, p.seq);
  // back through the tokens for lam and dx, then forward for h and dg: dy's registers become lam's
  plain_or_not(s, first, [&](auto plain) {
    constexpr bool PLAIN = decltype(plain)::value;
    fch lam[TOK];
#pragma unroll
    for (int j = 0; j < TOK; ++j) {
      const int i = TOK - 1 - j;
      const bool live = s.t0 + i < s.len, begins = first >> i & 1;
      const fch dy = unpack(dyr[i]);
      fch gx;
#pragma unroll
      for (int e = 0; e < LANES; ++e) {
        float f, r;
        gates(ts[i][e], f, r);
        lam[i][e] = dy[e] + mu[e];
        gx[e] = weight<W>(f, r) * lam[i][e];
        const float next = !PLAIN && begins ? 0.f : f * lam[i][e];
        mu[e] = PLAIN || live ? next : mu[e];
      }
      dx.store(i, PLAIN || live ? pack(gx) : 0u);
      }
    forget(ts);
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
      const bool live = s.t0 + i < s.len, begins = first >> i & 1;
      const fch x = unpack(xr[i]);
      fch gg;
#pragma unroll
      for (int e = 0; e < LANES; ++e) {
        float f, r;
        gates(ts[i][e], f, r);
        const float before = !PLAIN && begins ? 0.f : h[e];
        // (w = 1 - f: the two terms share f (1 - f))
        gg[e] = lam[i][e] * (W == 1 ? f * r * (before - x[e]) : before * (f * r) + x[e] * weight_slope<W>(f, r));
        h[e] = step<W, PLAIN>(ts[i][e], x[e], live, begins, h[e]);
      }
      dg.store(i, PLAIN || live ? pack(gg) : 0u);
      }
  });
  if (EACH == 0 && p.dh0) {
    __syncthreads();
    if (s.w == 0 && s.in) *reinterpret_cast<fch*>(p.dh0 + (long)s.b * p.c + s.ch) = mu;
  }
}

int chunks_of(int seq) { return (seq + CHUNK - 1) / CHUNK; }
// The counter, and a word for every channel of every chunk.
size_t scratch_bytes(int batch, int chunks, int c) { return chunks > 1 ? 16 + 8 * (size_t)batch * chunks * c : 0; }

template <int W, int EACH>
void enqueue(hipStream_t st, const ScanArgs& p, bool back) {
  const dim3 grid((unsigned)p.batch * p.chunks * p.blocks), block(64 * NW);
  if (back) RP_LAUNCH((scan_bwd_kernel<W, EACH>), grid, block, 0, st, p);
  else RP_LAUNCH((scan_fwd_kernel<W, EACH>), grid, block, 0, st, p);
}
template <int W>
void enqueue(hipStream_t st, const ScanArgs& p, bool back) {
  if (p.chunks == 1) enqueue<W, 0>(st, p, back);
  else if (p.chunks > NW && (long)p.batch * p.chunks * p.blocks <= 512) enqueue<W, 4>(st, p, back);      // (two workgroups a CU)
  else enqueue<W, 1>(st, p, back);
}

hipError_t run(hipStream_t st, int weight, ScanArgs p, void* scratch, bool back) {
  p.chunks = p.seq ? chunks_of(p.seq) : 1;      // without tokens the state is passed on
  p.blocks = (p.c + BLOCK_CH - 1) / BLOCK_CH;
  if (p.batch == 0 || p.c == 0) return hipSuccess;
  if (p.chunks > 1) {
    p.counter = static_cast<unsigned*>(scratch);
    p.words = reinterpret_cast<unsigned long long*>(static_cast<char*>(scratch) + 16);
    const long n = (long)(scratch_bytes(p.batch, p.chunks, p.c) / 16);      // (c is even)
    const long blocks = (n + 1023) / 1024;
    RP_LAUNCH(scan_clear_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, st, static_cast<uint4*>(scratch), n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  weight == 0 ? enqueue<0>(st, p, back) : weight == 1 ? enqueue<1>(st, p, back) : enqueue<2>(st, p, back);
  return hipGetLastError();
}

}  // namespace

void k_scan_sizes(int batch, int seq, int c, size_t* states, size_t* scratch) {
  *states = 4 * (size_t)batch * chunks_of(seq) * c;
  *scratch = scratch_bytes(batch, chunks_of(seq), c);
}

hipError_t k_scan_fwd(hipStream_t st, int weight, const ScanArgs& p, void* scratch) { return run(st, weight, p, scratch, false); }
hipError_t k_scan_bwd(hipStream_t st, int weight, const ScanArgs& p, void* scratch) { return run(st, weight, p, scratch, true); }
