// The plan of packed rows, and dropout.
#include "pack_ops.hpp"

namespace {

// A thread takes a token: its document by bisection of the starts (as many loads that follow one another as their number has bits, 31 at most, all of them in the caches after the first wave).
__global__ void __launch_bounds__(256) pack_plan_kernel(const PackArgs p) {
  const long t = (long)blockIdx.x * 256 + threadIdx.x;
  if (t >= p.T) return;
  int lo = 0, hi = p.n_docs + 1;      // starts[lo - 1] <= t < starts[hi]
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.starts[mid] <= t) lo = mid + 1;
    else hi = mid;
  }
  const int doc = lo - 1;
  const bool in = doc >= 0 && doc < p.n_docs;
  const int row0 = (int)(t / p.seq) * p.seq;      // first token of the row
  int2 span = make_int2(0, 0);
  int pos = 0, first = 1;
  if (in) {
    const int start = p.starts[doc], end = (int)min((long)p.starts[doc + 1], (long)row0 + p.seq);
    pos = (int)t - start;
    first = pos == 0;
    int from = max(start, row0), to = (int)t + 1;
    if (p.window > 0 && (long)t + 1 - p.window > from) from = (int)t + 1 - p.window;
    if (p.prefix) {
      const long pre = min((long)start + max(p.prefix[doc], 0), (long)end);
      if (pre > to) to = (int)pre;
    }
    span = make_int2(from - row0, to - row0);
  }
  if (p.span) p.span[t] = span;
  if (p.pos) p.pos[t] = pos;
  if (p.first) p.first[t] = (unsigned char)first;
}

// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011): a bijection of the 128-bit counter under a
// 64-bit key, from products of 32 x 32 bits.
RP_DEV void philox(uint32_t (&x)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)x[0] * 0xD2511F53u, b = (uint64_t)x[2] * 0xCD9E8D57u;
    x[0] = (uint32_t)(b >> 32) ^ x[1] ^ k0;
    x[1] = (uint32_t)b;
    x[2] = (uint32_t)(a >> 32) ^ x[3] ^ k1;
    x[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

RP_DEV uint32_t drop2(uint32_t x, uint32_t res, uint32_t bits, uint32_t keep, float scale) {
  const float lo = (bits & 0xffffu) < keep ? bf16_lo(x) * scale : 0.f;      // (a select: what is dropped may be infinite)
  const float hi = (bits >> 16) < keep ? bf16_hi(x) * scale : 0.f;
  return pack_bf16x2(lo + bf16_lo(res), hi + bf16_hi(res));
}

// Eight elements share a counter: 16 bits decide on one, so that ten rounds of products, at a quarter of the vector rate, stay below the time that the
// memory takes (vector issue 41 % busy).  A thread takes UNROLL groups 256 apart, all of its loads before the first product.  Bound by memory: 16384 x 5120 with a residual in 91 us, 5.5 TB/s.
constexpr int DROP_UNROLL = 4;
template <bool RES, bool WHOLE>      // WHOLE: rows without gaps
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutArgs p) {
  const long first = (long)blockIdx.x * (256 * DROP_UNROLL) + threadIdx.x;
  const unsigned long long offset = p.offset + (p.step ? *p.step : 0ull);
  long row = 0;
  uint32_t col = 0;
  if (!WHOLE) {
    row = first / p.n8;
    col = (uint32_t)(first - row * p.n8);
  }
  uint4 x[DROP_UNROLL], r[DROP_UNROLL];
  long out[DROP_UNROLL];
#pragma unroll
  for (int i = 0; i < DROP_UNROLL; ++i) {
    const long g = first + 256 * i;
    r[i] = make_uint4(0u, 0u, 0u, 0u);
    if (g < p.groups) {
      x[i] = *reinterpret_cast<const uint4*>(p.x + (WHOLE ? 8 * g : row * p.ldx + 8 * col));
      if (RES) r[i] = *reinterpret_cast<const uint4*>(p.res + (WHOLE ? 8 * g : row * p.ldr + 8 * col));
    }
    out[i] = WHOLE ? 8 * g : row * p.ldy + 8 * col;
    if (!WHOLE) {
      col += 256;
      const uint32_t more = col / p.n8;
      row += more;
      col -= more * p.n8;
    }
  }
#pragma unroll
  for (int i = 0; i < DROP_UNROLL; ++i) {
    const long g = first + 256 * i;
    uint32_t w[4] = {(uint32_t)g, (uint32_t)(g >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
    philox(w, (uint32_t)p.seed, (uint32_t)(p.seed >> 32));
    if (g < p.groups)
      *reinterpret_cast<uint4*>(p.y + out[i]) = make_uint4(drop2(x[i].x, r[i].x, w[0], p.keep, p.scale), drop2(x[i].y, r[i].y, w[1], p.keep, p.scale),
                                                           drop2(x[i].z, r[i].z, w[2], p.keep, p.scale), drop2(x[i].w, r[i].w, w[3], p.keep, p.scale));
  }
}

}  // namespace

hipError_t k_pack_plan(hipStream_t st, const PackArgs& p) {
  if (p.T == 0) return hipSuccess;
  RP_LAUNCH(pack_plan_kernel, dim3((unsigned)(((long)p.T + 255) / 256)), dim3(256), 0, st, p);
  return hipGetLastError();
}

hipError_t k_dropout(hipStream_t st, const DropoutArgs& p) {
  if (p.groups == 0) return hipSuccess;
  const dim3 grid((unsigned)((p.groups + 256 * DROP_UNROLL - 1) / (256 * DROP_UNROLL))), block(256);
  const long n = 8l * p.n8;
  const bool whole = p.ldx == n && p.ldy == n && (!p.res || p.ldr == n);
  if (p.res) {
    if (whole) RP_LAUNCH((dropout_kernel<true, true>), grid, block, 0, st, p);
    else RP_LAUNCH((dropout_kernel<true, false>), grid, block, 0, st, p);
  } else {
    if (whole) RP_LAUNCH((dropout_kernel<false, true>), grid, block, 0, st, p);
    else RP_LAUNCH((dropout_kernel<false, false>), grid, block, 0, st, p);
  }
  return hipGetLastError();
}
