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
//   rows  : a few lanes hold a token's logits, the next token's on their way; every block first adds the slices' counts of its group up; loss
//           terms leave one pair of fp32 sums per block
//   total : one block adds the pairs in a fixed order
//   small : a group in one block, for groups that one block is through with before the other launches would have started
//
// Bound by launches that wait for one another: 31744 tokens, eight of 128 experts, with a gradient to add to 19.6 us (count 5, rows 12, total 3) where its 50 MB
// take 9.6; 4 x 1001 x 256 13.7.
#include "kernels.hpp"
#include "layer_ops.hpp"

namespace {

// Reductions over L neighbouring lanes, in all of them, without LDS: exchanges inside a row of 16 lanes (neighbours, pairs, mirrored halves:
// every step joins two halves that hold one value each), then of rows and of half waves.
template <int CTRL>
RP_DEV float dpp(float x) { return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xf, 0xf, true)); }
template <int L, typename F>
RP_DEV float over_lanes(float x, F f) {
  if constexpr (L > 1) x = f(x, dpp<0xB1>(x));        // lanes 1 0 3 2
  if constexpr (L > 2) x = f(x, dpp<0x4E>(x));        // lanes 2 3 0 1
  if constexpr (L > 4) x = f(x, dpp<0x141>(x));       // 7 .. 0
  if constexpr (L > 8) x = f(x, dpp<0x140>(x));       // 15 .. 0
  if constexpr (L > 16) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (L > 32) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return x;
}
struct Max { RP_DEV float operator()(float a, float b) const { return fmaxf(a, b); } };
struct Add { RP_DEV float operator()(float a, float b) const { return a + b; } };

// Sum over the threads of a block, in all of them.  red: one entry per wave.
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

// Counts the choices of tokens t0 .. t1 - 1 of a group into s_hist [E] (zeroed here); returns the number of valid ones, in all threads.
// Choices outside 0 .. E-1 are not counted.
template <int NT>
RP_DEV int count_choices(const BalanceArgs& p, long base, int t0, int t1, int* s_hist, int* red) {
  const int tid = threadIdx.x;
  for (int e = tid; e < p.E; e += NT) s_hist[e] = 0;
  __syncthreads();
  int valid = 0;
  if (p.mask) {
    for (int t = t0 + tid; t < t1; t += NT) valid += p.mask[base + t] != 0;
  } else if (tid == 0) {
    valid = t1 - t0;
  }
  const int* const idx = p.idx + (base + t0) * p.top_k;
  const unsigned n = (unsigned)(t1 - t0) * (unsigned)p.top_k;
#pragma unroll 8
  for (unsigned i = tid; i < n; i += NT) {
    const int e = idx[i];
    if (e >= 0 && e < p.E && (!p.mask || p.mask[base + t0 + (int)(i / (unsigned)p.top_k)])) atomicAdd(&s_hist[e], 1);
  }
  return block_sum(valid, red);      // (its barriers order the counts as well)
}

// hist[g][slice][e], tok[g][slice]
__global__ void __launch_bounds__(1024) balance_count_kernel(const BalanceArgs p) {
  __shared__ int s_hist[1024];
  __shared__ int red[16];
  const int tid = threadIdx.x, slice = (int)blockIdx.x % p.slices;
  const long g = p.first + (int)blockIdx.x / p.slices, out_at = g * p.slices + slice;
  const int per = (p.seq + p.slices - 1) / p.slices;
  const int t0 = min(slice * per, p.seq), t1 = min(t0 + per, p.seq);
  const int valid = count_choices<1024>(p, g * p.seq, t0, t1, s_hist, red);
  int* const out = p.hist + out_at * p.E;
  for (int e = tid; e < p.E; e += 1024) out[e] = s_hist[e];
  if (tid == 0) p.tok[out_at] = valid;
}

// Tokens of all groups, for masked batches of many groups (else the rows' blocks add them up themselves).
__global__ void __launch_bounds__(1024) balance_tokens_kernel(const BalanceArgs p) {
  __shared__ int red[16];
  int n = 0;
  for (long i = threadIdx.x; i < (long)p.groups * p.slices; i += 1024) n += p.tok[i];
  n = block_sum(n, red);
  if (threadIdx.x == 0) p.tokens[p.groups] = n;
}

// A block's share of the rows: L lanes per token, C accesses of VEC logits a lane, element (lane + L i) VEC + v.  FULL: E = L C VEC, no lane is left over.
template <int L, int C, int VEC, bool FULL, int NT>
struct RowPass {
  typedef float fvec __attribute__((ext_vector_type(VEC)));
  static constexpr int ROWS = NT / L;
  fvec x[C], given[C];
  bool on;

  // the logits of token t of the group, and what is there of the gradient; -inf where there is no token, or a padded one
  RP_DEV void load(const BalanceArgs& p, long base, int t, int t1, int sub) {
    const bool in = t < t1;
    const long row = base + t;
    on = in && (!p.mask || p.mask[row]);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e0 = (sub + L * c) * VEC;
#pragma unroll
      for (int v = 0; v < VEC; ++v) { x[c][v] = -INFINITY; given[c][v] = 0.f; }
      if (in && (FULL || e0 < p.E)) {
        x[c] = *reinterpret_cast<const fvec*>(p.logits + row * p.E + e0);
        if (p.dlogits_in) given[c] = *reinterpret_cast<const fvec*>(p.dlogits_in + row * p.E + e0);
      }
    }
  }

  // rows t0 .. t1 - 1, the first of them loaded already; kb, kz: what the gradient's two terms are multiplied with
  RP_DEV void run(const BalanceArgs& p, long base, int t0, int t1, const float* s_f, float kb, float kz, float& sum_b, float& sum_z) {
    const int sub = (int)threadIdx.x % L, row_in = (int)threadIdx.x / L;
    fvec f[C];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const int e = (sub + L * c) * VEC + v;
        f[c][v] = FULL || e < p.E ? s_f[e] : 0.f;
      }
    for (int t = t0 + row_in; t - row_in < t1; t += ROWS) {
      fvec y[C], was[C];
      const bool live = on;
      float m = -INFINITY;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        was[c] = given[c];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          y[c][v] = live ? x[c][v] : -INFINITY;
          m = fmaxf(m, y[c][v]);
        }
      }
      if (t - row_in + ROWS < t1) load(p, base, t + ROWS, t1, sub);
      m = over_lanes<L>(m, Max());
      const float ref = m != -INFINITY ? m : 0.f;
      float l = 0.f, dot = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          y[c][v] = __expf(y[c][v] - ref);
          l += y[c][v];
          dot += f[c][v] * y[c][v];
        }
      l = over_lanes<L>(l, Add());
      dot = over_lanes<L>(dot, Add());
      const bool some = l != 0.f;      // a row of -inf has no probabilities; one of NaN, which the maximum passes over, has NaN here
      const float inv_l = some ? 1.f / l : 0.f, lse = some ? ref + logf(l) : 0.f;
      dot *= inv_l;
      if (sub == 0) { sum_b += dot; sum_z += lse * lse; }
      if (t < t1 && p.dlogits) {
        const float shift = kz * lse - kb * dot;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int e0 = (sub + L * c) * VEC;
          if (FULL || e0 < p.E) {
            fvec d;
#pragma unroll
            for (int v = 0; v < VEC; ++v) d[v] = was[c][v] + (live ? y[c][v] * inv_l * (kb * f[c][v] + shift) : 0.f);
            *reinterpret_cast<fvec*>(p.dlogits + (base + t) * p.E + e0) = d;
          }
        }
      }
    }
  }
};

template <int L, int C, int VEC, bool FULL>
__global__ void __launch_bounds__(256) balance_rows_kernel(const BalanceArgs p) {
  __shared__ int s_cnt[1024];
  __shared__ float s_f[1024];
  __shared__ int red[4];
  __shared__ float redf[4];
  const int tid = threadIdx.x, chunk = (int)blockIdx.x % p.chunks;
  const long g = p.first + (int)blockIdx.x / p.chunks, base = g * p.seq;
  const int t0 = chunk * p.rows_per_block, t1 = min(p.seq, t0 + p.rows_per_block);
  RowPass<L, C, VEC, FULL, 256> rows;
  rows.load(p, base, t0 + tid / L, t1, tid % L);
  for (int e = tid; e < p.E; e += 256) s_cnt[e] = 0;
  __syncthreads();
  int part = 0;
  for (int i = tid; i < p.slices; i += 256) part += p.tok[g * p.slices + i];
  // the slices' counts of an expert: several threads share it where there are more threads than experts
  const int lanes = p.E < 256 ? 256 / p.E : 1, mine = p.E < 256 ? tid / p.E : 0;
  if (mine < lanes) {
    for (int e = tid - mine * p.E; e < p.E; e += 256) {
      int n = 0;
#pragma unroll 16
      for (int s = mine; s < p.slices; s += lanes) n += p.hist[(g * p.slices + s) * p.E + e];
      atomicAdd(&s_cnt[e], n);
    }
  }
  const int n_g = block_sum(part, red);      // (its barriers order the counts as well)
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
    s_f[e] = (float)s_cnt[e] * inv_choices;
    if (chunk == 0) p.counts[g * p.E + e] = s_cnt[e];
  }
  if (chunk == 0 && tid == 0) {
    p.tokens[g] = n_g;
    if (g == 0 && !(p.groups > 1 && p.mask && p.total_given)) p.tokens[p.groups] = total;
  }
  __syncthreads();
  const float inv_n = total ? 1.f / (float)total : 0.f;
  float sum_b = 0.f, sum_z = 0.f;
  rows.run(p, base, t0, t1, s_f, p.grad_scale * p.coef * (float)p.E * inv_n, p.grad_scale * 2.f * p.z_coef * inv_n, sum_b, sum_z);
  const float tb = block_sum(sum_b, redf), tz = block_sum(sum_z, redf);
  if (tid == 0) p.part[g * p.chunks + chunk] = make_float2(tb, tz);
}

RP_DEV void write_loss(const BalanceArgs& p, double b, double z, int N) {
  const double inv = N ? 1.0 / N : 0.0;
  b *= inv * p.E;
  z *= inv;
  p.loss[0] = (float)(p.coef * b + p.z_coef * z);
  p.loss[1] = (float)b;
  p.loss[2] = (float)z;
}

// A group in one block; a single group's block writes the loss as well.
template <int L, int C, int VEC, bool FULL>
__global__ void __launch_bounds__(1024) balance_small_kernel(const BalanceArgs p) {
  __shared__ int s_hist[1024];
  __shared__ float s_f[1024];
  __shared__ int red[16];
  __shared__ float redf[16];
  const int tid = threadIdx.x;
  const long g = p.first + (int)blockIdx.x, base = g * p.seq;
  RowPass<L, C, VEC, FULL, 1024> rows;
  rows.load(p, base, tid / L, p.seq, tid % L);
  const int n = count_choices<1024>(p, base, 0, p.seq, s_hist, red);
  int total = n;
  if (p.groups > 1) {
    total = p.groups * p.seq;
    if (p.mask) {      // every block counts all tokens: a byte each
      int valid = 0;
      for (int t = tid; t < total; t += 1024) valid += p.mask[t] != 0;
      total = block_sum(valid, red);
    }
  }
  const float inv_choices = n ? 1.f / ((float)n * (float)p.top_k) : 0.f;
  for (int e = tid; e < p.E; e += 1024) {
    s_f[e] = (float)s_hist[e] * inv_choices;
    p.counts[g * p.E + e] = s_hist[e];
  }
  __syncthreads();
  const float inv_n = total ? 1.f / (float)total : 0.f;
  float sum_b = 0.f, sum_z = 0.f;
  rows.run(p, base, 0, p.seq, s_f, p.grad_scale * p.coef * (float)p.E * inv_n, p.grad_scale * 2.f * p.z_coef * inv_n, sum_b, sum_z);
  sum_b = block_sum(sum_b, redf);
  sum_z = block_sum(sum_z, redf);
  if (tid == 0) {
    p.tokens[g] = n;
    if (g == 0) p.tokens[p.groups] = total;
    if (p.groups == 1) write_loss(p, sum_b, sum_z, n);
    else p.part[g] = make_float2(sum_b, sum_z);
  }
}

// loss = {coef L_b + z_coef L_z, L_b, L_z}
__global__ void __launch_bounds__(256) balance_total_kernel(const BalanceArgs p, int n) {
  __shared__ double red[2][4];
  double b = 0.0, z = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 256) {
    const float2 v = p.part[i];
    b += v.x;
    z += v.y;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { b += __shfl_xor(b, o, 64); z += __shfl_xor(z, o, 64); }
  if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = b; red[1][threadIdx.x >> 6] = z; }
  __syncthreads();
  if (threadIdx.x == 0) write_loss(p, (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]), (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]), p.tokens[p.groups]);
}

struct Shape { int slices, rows_per_block, chunks; };

// Lanes per token where the rows lie on 16-byte boundaries: two accesses a lane and more, so that a reduction has few steps (31744 x 128: 16 lanes 21.0
// us, 32 lanes 21.2; 6468 x 8: two lanes 9.9, four 11.6).
int lanes_of(int E) { return E <= 8 ? 2 : E <= 32 ? 4 : E <= 64 ? 8 : E <= 128 ? 16 : E <= 256 ? 32 : 64; }

// Slices of a group for counting, of 2048 choices (two a thread) up to 32 of them; blocks of its rows, each going over its 256 threads' worth of
// rows once or, where that would make more than 1024 blocks, several times.  31744 x 128, eight choices, us: slices of 8192 | 4096, up to 64 | 2048,
// up to 64 | 2048: 24.9 | 24.4 | 26.0 | 22.1;  512 | 1024 | 2048 blocks: 25.8 | 24.9 | 29.3.
Shape shape_of(int T, int seq, int E, int top_k) {
  const int groups = T / seq;
  Shape s;
  const long slices = ((long)seq * top_k + 2047) / 2048;
  s.slices = slices > 32 ? 32 : (int)slices;
  const int rows = 256 / lanes_of(E);
  const int passes = (seq + rows - 1) / rows, most = groups < 1024 ? 1024 / groups : 1;
  int each = (passes + most - 1) / most;
  // a block of four rows spends as long on the counts of more than 512 experts as on them: twice as many where 256 blocks and more are left
  // (1024 experts, 3968 tokens 26.3 -> 21.5 us, 353 tokens 12.8 -> 14.1)
  if (E > 512 && each < 2 && (long)groups * passes >= 512) each = 2;
  s.rows_per_block = rows * each;
  s.chunks = (seq + s.rows_per_block - 1) / s.rows_per_block;
  return s;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// ------------------------------------------------------------------------------------------------ launchers
// The counts of up to 32 slices a group (as many choices a token as there can be: the size does not depend on top_k), and the loss terms.
size_t k_moe_balance_scratch(int T, int seq, int E) {
  if (T == 0) return 0;
  const Shape s = shape_of(T, seq, E, 64);
  const size_t groups = (size_t)(T / seq);
  return up256(groups * s.slices * E * 4) + up256(groups * s.slices * 4) + up256(groups * s.chunks * 8);
}

// Launches over all groups, `each` blocks a group: a launch has fewer than 2^32 threads, 2^21 blocks of 1024 at most here.
template <typename K>
static hipError_t launch_groups(K kern, int each, int threads, hipStream_t st, BalanceArgs p) {
  const int most = (1 << 21) / each;
  for (long first = 0; first < p.groups; first += most) {
    p.first = (int)first;
    const int n = p.groups - (int)first < most ? p.groups - (int)first : most;
    RP_LAUNCH(kern, dim3(n * each), dim3(threads), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int L, int C, int VEC, bool FULL>
static hipError_t launch_rows_as(hipStream_t st, const BalanceArgs& p, bool small) {
  if (small) return launch_groups(balance_small_kernel<L, C, VEC, FULL>, 1, 1024, st, p);
  return launch_groups(balance_rows_kernel<L, C, VEC, FULL>, p.chunks, 256, st, p);
}
template <int L, int C, int VEC>
static hipError_t launch_rows(hipStream_t st, const BalanceArgs& p, bool small) {
  if (VEC == 4 && p.E == L * C * VEC) return launch_rows_as<L, C, VEC, VEC == 4>(st, p, small);
  return launch_rows_as<L, C, VEC, false>(st, p, small);
}

hipError_t k_moe_balance(hipStream_t st, BalanceArgs p, int T, void* scratch) {
  if (T == 0) {
    const hipError_t e = k_fill_u32(st, p.loss, 3, 0u);
    return e == hipSuccess ? k_fill_u32(st, p.tokens, 1, 0u) : e;
  }
  const Shape s = shape_of(T, p.seq, p.E, p.top_k < 64 ? p.top_k : 64);
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
  // one block is through with a group of 16384 logits (and their choices) in the time of the launch or two that it saves: 256 tokens of 32 experts
  // 12.3 -> 5.7 us
  const bool small = (long)p.seq * p.E <= 16384 && (long)p.seq * p.top_k <= 8192 && (p.groups == 1 || !p.mask || T <= 65536);
  hipError_t e = hipSuccess;      // (RP_LAUNCH forgets what the launch before it left: each is asked for)
  if (!small) {
    e = launch_groups(balance_count_kernel, s.slices, 1024, st, p);
    if (e == hipSuccess && p.total_given) {
      RP_LAUNCH(balance_tokens_kernel, dim3(1), dim3(1024), 0, st, p);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
  }
  const uintptr_t at16 = reinterpret_cast<uintptr_t>(p.logits) | reinterpret_cast<uintptr_t>(p.dlogits) | reinterpret_cast<uintptr_t>(p.dlogits_in);
  if (p.E % 4 == 0 && at16 % 16 == 0) {      // rows on 16-byte boundaries: 16-byte accesses
    if (p.E <= 8) e = launch_rows<2, 1, 4>(st, p, small);
    else if (p.E <= 16) e = launch_rows<4, 1, 4>(st, p, small);
    else if (p.E <= 32) e = launch_rows<4, 2, 4>(st, p, small);
    else if (p.E <= 64) e = launch_rows<8, 2, 4>(st, p, small);
    else if (p.E <= 128) e = launch_rows<16, 2, 4>(st, p, small);
    else if (p.E <= 256) e = launch_rows<32, 2, 4>(st, p, small);
    else if (p.E <= 512) e = launch_rows<64, 2, 4>(st, p, small);
    else e = launch_rows<64, 4, 4>(st, p, small);
  } else {
    if (p.E <= 16) e = launch_rows<16, 1, 1>(st, p, small);
    else if (p.E <= 64) e = launch_rows<64, 1, 1>(st, p, small);
    else if (p.E <= 256) e = launch_rows<64, 4, 1>(st, p, small);
    else e = launch_rows<64, 16, 1>(st, p, small);
  }
  if (e != hipSuccess || (small && p.groups == 1)) return e;
  RP_LAUNCH(balance_total_kernel, dim3(1), dim3(256), 0, st, p, small ? p.groups : p.groups * s.chunks);
  return hipGetLastError();
}
