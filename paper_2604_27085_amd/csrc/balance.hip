// Balance loss of a top-k mixture's router, with its gradient, in one pass over the logits.
//
//   p_t   = softmax(logits_t) over all experts;  f_ge = (choices of expert e among the valid tokens of group g) / (n_g top_k)
//   L_b   = E / N sum_t sum_e f_ge p_te   = sum_g n_g / N  E sum_e f_ge P_ge, with P_ge the group's mean probability
//   L_z   = 1 / N sum_t lse_t^2, lse_t = log sum_e exp(logits_te)
//   d logits_te = scale (c_b E / N p_te (f_ge - sum_e' f_ge' p_te') + c_z 2 / N lse_t p_te)          (f is a count: no gradient)
//
// sum_e f_ge p_te is what the gradient needs of its row and, summed over the rows, what the loss is: once the choices are counted, one
// pass gives both, and no mean probability is ever formed.
//
//   count : choices and valid tokens of a slice of a group, in LDS (integers: any order gives the same), a row of counts per slice
//   rows  : a few lanes hold a token's logits; every block first adds the slices' counts of its group up; loss terms leave one pair of fp32 sums
//           per block
//   total : one block adds the pairs in a fixed order
#include "kernels.hpp"
#include "layer_ops.hpp"

namespace {

// Sum over the lanes of a block, in 64 bits where it counts: thread 0 has it.  red: one entry per wave.
template <typename T>
RP_DEV T block_sum(T v, T* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T s = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += red[w];
  return s;
}

// hist[g][slice][e], tok[g][slice].  Choices outside 0 .. E-1 are not counted.
__global__ void __launch_bounds__(256) balance_count_kernel(const BalanceArgs p) {
  __shared__ int s_hist[1024];
  __shared__ int red[4];
  const int tid = threadIdx.x, slice = (int)blockIdx.x % p.slices;
  const long g = (int)blockIdx.x / p.slices;
  for (int e = tid; e < p.E; e += 256) s_hist[e] = 0;
  __syncthreads();
  const int per = (p.seq + p.slices - 1) / p.slices;
  const int t0 = slice * per, t1 = t0 + per < p.seq ? t0 + per : p.seq;
  const long base = g * p.seq;
  int valid = 0;
  if (p.mask) {
    for (int t = t0 + tid; t < t1; t += 256) valid += p.mask[base + t] != 0;
  } else if (tid == 0) {
    valid = t1 > t0 ? t1 - t0 : 0;
  }
  const long n = t1 > t0 ? (long)(t1 - t0) * p.top_k : 0;
  const int* const idx = p.idx + (base + t0) * p.top_k;
  for (long i = tid; i < n; i += 256) {
    const int e = idx[i];
    if (e >= 0 && e < p.E && (!p.mask || p.mask[base + t0 + i / p.top_k])) atomicAdd(&s_hist[e], 1);
  }
  const int all = block_sum(valid, red);      // (its barriers order the counts as well)
  int* const out = p.hist + (g * p.slices + slice) * p.E;
  for (int e = tid; e < p.E; e += 256) out[e] = s_hist[e];
  if (tid == 0) p.tok[g * p.slices + slice] = all;
}

// Tokens of all groups, for masked batches of many groups (else the rows' blocks add them up themselves).
__global__ void __launch_bounds__(1024) balance_tokens_kernel(const BalanceArgs p) {
  __shared__ int red[16];
  int n = 0;
  for (long i = threadIdx.x; i < (long)p.groups * p.slices; i += 1024) n += p.tok[i];
  n = block_sum(n, red);
  if (threadIdx.x == 0) p.tokens[p.groups] = n;
}

// L lanes per token, C accesses of VEC logits a lane: element (lane + L i) VEC + v.
template <int L, int C, int VEC>
__global__ void __launch_bounds__(256) balance_rows_kernel(const BalanceArgs p) {
  __shared__ float s_f[1024];
  __shared__ int red[4];
  __shared__ float redf[4];
  typedef float fvec __attribute__((ext_vector_type(VEC)));
  const int tid = threadIdx.x, chunk = (int)blockIdx.x % p.chunks;
  const long g = (int)blockIdx.x / p.chunks;
  int part = 0;
  for (int i = tid; i < p.slices; i += 256) part += p.tok[g * p.slices + i];
  const int n_g = block_sum(part, red);
  int total = n_g;
  if (p.groups > 1) {
    if (!p.mask) {
      total = p.groups * p.seq;
    } else if (p.total_given) {
      total = p.tokens[p.groups];
    } else {
      part = 0;
      for (int i = tid; i < p.groups * p.slices; i += 256) part += p.tok[i];
      total = block_sum(part, red);
    }
  }
  const float inv_choices = n_g ? 1.f / ((float)n_g * (float)p.top_k) : 0.f;
  for (int e = tid; e < p.E; e += 256) {
    int n = 0;
    for (int s = 0; s < p.slices; ++s) n += p.hist[(g * p.slices + s) * p.E + e];
    s_f[e] = (float)n * inv_choices;
    if (chunk == 0) p.counts[g * p.E + e] = n;
  }
  if (chunk == 0 && tid == 0) {
    p.tokens[g] = n_g;
    if (g == 0 && !(p.groups > 1 && p.mask && p.total_given)) p.tokens[p.groups] = total;
  }
  __syncthreads();
  const int sub = tid % L, row_in = tid / L;
  constexpr int ROWS = 256 / L;
  fvec f[C];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const int e = (sub + L * c) * VEC + v;
      f[c][v] = e < p.E ? s_f[e] : 0.f;
    }
  const float inv_n = total ? 1.f / (float)total : 0.f;
  const float kb = p.grad_scale * p.coef * (float)p.E * inv_n, kz = p.grad_scale * 2.f * p.z_coef * inv_n;
  float sum_b = 0.f, sum_z = 0.f;
  const int t1 = min(p.seq, (chunk + 1) * p.rows_per_block);
  for (int t0 = chunk * p.rows_per_block; t0 < t1; t0 += ROWS) {
    const int t = t0 + row_in;
    const bool in = t < t1;
    const long row = g * p.seq + t;
    const bool on = in && (!p.mask || p.mask[row]);
    fvec x[C], given[C];
    float m = -INFINITY;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e0 = (sub + L * c) * VEC;
#pragma unroll
      for (int v = 0; v < VEC; ++v) { x[c][v] = -INFINITY; given[c][v] = 0.f; }
      if (on && e0 < p.E) x[c] = *reinterpret_cast<const fvec*>(p.logits + row * p.E + e0);
      if (in && p.dlogits_in && e0 < p.E) given[c] = *reinterpret_cast<const fvec*>(p.dlogits_in + row * p.E + e0);
#pragma unroll
      for (int v = 0; v < VEC; ++v) m = fmaxf(m, x[c][v]);
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    float l = 0.f, dot = 0.f;
    const float ref = m == -INFINITY ? 0.f : m;      // a row of -inf has no probabilities
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        x[c][v] = __expf(x[c][v] - ref);
        l += x[c][v];
        dot += f[c][v] * x[c][v];
      }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) { l += __shfl_xor(l, o, 64); dot += __shfl_xor(dot, o, 64); }
    const bool some = m != -INFINITY;
    const float inv_l = some ? 1.f / l : 0.f, lse = some ? m + logf(l) : 0.f;
    dot *= inv_l;
    if (sub == 0) { sum_b += dot; sum_z += lse * lse; }
    if (in && p.dlogits) {
      const float shift = kz * lse - kb * dot;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e0 = (sub + L * c) * VEC;
        if (e0 < p.E) {
          fvec d;
#pragma unroll
          for (int v = 0; v < VEC; ++v) d[v] = given[c][v] + (on ? x[c][v] * inv_l * (kb * f[c][v] + shift) : 0.f);
          *reinterpret_cast<fvec*>(p.dlogits + row * p.E + e0) = d;
        }
      }
    }
  }
  const float tb = block_sum(sum_b, redf), tz = block_sum(sum_z, redf);
  if (tid == 0) p.part[blockIdx.x] = make_float2(tb, tz);
}

// loss = {coef L_b + z_coef L_z, L_b, L_z}
__global__ void __launch_bounds__(1024) balance_total_kernel(const BalanceArgs p, long n) {
  __shared__ double red[16];
  double b = 0.0, z = 0.0;
  for (long i = threadIdx.x; i < n; i += 1024) {
    const float2 v = p.part[i];
    b += v.x;
    z += v.y;
  }
  b = block_sum(b, red);
  z = block_sum(z, red);
  if (threadIdx.x == 0) {
    const int N = p.tokens[p.groups];
    const double inv = N ? 1.0 / N : 0.0;
    b *= inv * p.E;
    z *= inv;
    p.loss[0] = (float)(p.coef * b + p.z_coef * z);
    p.loss[1] = (float)b;
    p.loss[2] = (float)z;
  }
}

struct Shape { int slices, rows_per_block, chunks; };

// Slices of a group for counting and blocks of its rows.  A slice is worth about 4096 tokens' choices at one a token; rows go out in at
// most 2048 blocks altogether, of 32 rows at least.
Shape shape_of(long T, int seq) {
  const int groups = (int)(T / seq);
  Shape s;
  s.slices = (seq + 1023) / 1024;
  s.slices = s.slices < 1 ? 1 : s.slices > 32 ? 32 : s.slices;
  const int most = groups < 2048 ? 2048 / groups : 1;
  int rows = (seq + most - 1) / most;
  rows = rows < 32 ? 32 : (rows + 31) / 32 * 32;
  s.rows_per_block = rows;
  s.chunks = (seq + rows - 1) / rows;
  return s;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// ------------------------------------------------------------------------------------------------ launchers
size_t k_moe_balance_scratch(int T, int seq, int E) {
  if (T == 0) return 0;
  const Shape s = shape_of(T, seq);
  const size_t groups = (size_t)(T / seq);
  return up256(groups * s.slices * E * 4) + up256(groups * s.slices * 4) + up256(groups * s.chunks * 8);
}

hipError_t k_moe_balance(hipStream_t st, BalanceArgs p, int T, void* scratch) {
  if (T == 0) {
    const hipError_t e = k_fill_u32(st, p.loss, 3, 0u);
    return e == hipSuccess ? k_fill_u32(st, p.tokens, 1, 0u) : e;
  }
  const Shape s = shape_of(T, p.seq);
  p.groups = T / p.seq;
  p.slices = s.slices;
  p.rows_per_block = s.rows_per_block;
  p.chunks = s.chunks;
  char* at = static_cast<char*>(scratch);
  p.hist = reinterpret_cast<int*>(at);
  at += up256((size_t)p.groups * s.slices * p.E * 4);
  p.tok = reinterpret_cast<int*>(at);
  at += up256((size_t)p.groups * s.slices * 4);
  p.part = reinterpret_cast<float2*>(at);
  p.total_given = p.groups > 1 && p.mask && (long)p.groups * s.slices > 1024;
  RP_LAUNCH(balance_count_kernel, dim3(p.groups * s.slices), dim3(256), 0, st, p);
  if (p.total_given) RP_LAUNCH(balance_tokens_kernel, dim3(1), dim3(1024), 0, st, p);
#define RP_LAUNCH_BR(L, C, VEC) RP_LAUNCH((balance_rows_kernel<L, C, VEC>), dim3(p.groups * s.chunks), dim3(256), 0, st, p)
  const uintptr_t at16 = reinterpret_cast<uintptr_t>(p.logits) | reinterpret_cast<uintptr_t>(p.dlogits) | reinterpret_cast<uintptr_t>(p.dlogits_in);
  if (p.E % 4 == 0 && at16 % 16 == 0) {      // rows on 16-byte boundaries: 16-byte accesses
    if (p.E <= 16) RP_LAUNCH_BR(4, 1, 4);
    else if (p.E <= 32) RP_LAUNCH_BR(8, 1, 4);
    else if (p.E <= 64) RP_LAUNCH_BR(16, 1, 4);
    else if (p.E <= 128) RP_LAUNCH_BR(32, 1, 4);
    else if (p.E <= 256) RP_LAUNCH_BR(64, 1, 4);
    else if (p.E <= 512) RP_LAUNCH_BR(64, 2, 4);
    else RP_LAUNCH_BR(64, 4, 4);
  } else {
    if (p.E <= 16) RP_LAUNCH_BR(16, 1, 1);
    else if (p.E <= 64) RP_LAUNCH_BR(64, 1, 1);
    else if (p.E <= 256) RP_LAUNCH_BR(64, 4, 1);
    else RP_LAUNCH_BR(64, 16, 1);
  }
#undef RP_LAUNCH_BR
  RP_LAUNCH(balance_total_kernel, dim3(1), dim3(1024), 0, st, p, (long)p.groups * s.chunks);
  return hipGetLastError();
}
