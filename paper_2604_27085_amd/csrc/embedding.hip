// Embedding: rows of a table by token, and the table's gradient.
//
//   x_t = scale E[id_t];   dE[v] (+)= scale sum over the tokens t with id_t = v of dx_t
//
// A token whose number is outside 0 .. V - 1 (padding) has the row zero and adds nothing.
//
// The gradient sorts the tokens by their number (stably, so equal ones stay in order), cuts the sorted tokens into chunks of equal length and adds up runs of equal
// numbers within them, in ascending order of the tokens: however often a token comes, the work is spread evenly, and no sum depends on timing.  A run that goes on into the next chunk leaves its
// part in scratch; a second kernel adds those up, every eighth part by itself and then the eight.  Sums are fp32.
//
// What bounds it: memory.  16384 tokens of 4096 from 151936 rows: rows 49 us (5.5 TB/s), sort 24, sums 75, join 9, and 388 for the zeros of the rows without tokens (2.4 GB at 6.1 TB/s).
// 4084 tokens of 2880, gradient added to what is there: rows 10, sort 11, sums 17, join 6: three launches that wait for one another.
#include "pack_ops.hpp"

namespace {

constexpr int NT = 256;
constexpr int SMALL = 128;                  // tokens that one block sorts by comparing all pairs (64, 128, 256, 1024 tokens 3.6, 5.9, 10.6, 47 us; by digits 6.0 for 256, 6.4 for 1024)
constexpr int BATCH = 1024;                 // tokens of a radix step
constexpr int MOST_BLOCKS = 64;             // of the radix sort: each reads all blocks' counts
constexpr int MOST_DIGITS = 1024;

// ------------------------------------------------------------------------------------------------ rows
// `lanes` threads take a row's 16-byte pieces; lanes is a power of two.  A token without a row reads what it is about to overwrite, so that loads need no branch of their own (with one, each
// waited for: 16384 rows of 4096 100 us instead of 49, 5.5 TB/s).
constexpr int PIECES = 4;      // of a thread at once
__global__ void __launch_bounds__(NT) embed_rows_kernel(const bf16* table, long ldt, const int* ids, float scale, bf16* x, long ldx, int T, int V, int h8, int lanes) {
  const int lane = threadIdx.x & (lanes - 1);
  const long t = (long)blockIdx.x * (NT / lanes) + threadIdx.x / lanes;
  if (t >= T) return;
  const int id = ids[t];
  const bool in = (unsigned)id < (unsigned)V;
  uint4* const dst = reinterpret_cast<uint4*>(x + t * ldx);
  const uint4* const src = in ? reinterpret_cast<const uint4*>(table + (long)id * ldt) : dst;
  for (int c = lane; c < h8; c += PIECES * lanes) {
    uint4 u[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if (c + i * lanes < h8) u[i] = src[c + i * lanes];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const uint4 y = make_uint4(pack_bf16x2(bf16_lo(u[i].x) * scale, bf16_hi(u[i].x) * scale), pack_bf16x2(bf16_lo(u[i].y) * scale, bf16_hi(u[i].y) * scale),
                                 pack_bf16x2(bf16_lo(u[i].z) * scale, bf16_hi(u[i].z) * scale), pack_bf16x2(bf16_lo(u[i].w) * scale, bf16_hi(u[i].w) * scale));
      if (c + i * lanes < h8) dst[c + i * lanes] = in ? y : make_uint4(0u, 0u, 0u, 0u);
    }
  }
}

// ------------------------------------------------------------------------------------------------ sorting
// Of the lanes that are `in`, those with this lane's digit: four instructions a bit.
RP_DEV unsigned long long same_digit(int digit, int bits, bool in) {
  const unsigned long long used = __ballot(in);
  uint32_t lo = (uint32_t)used, hi = (uint32_t)(used >> 32);
  for (int b = 0; b < bits; ++b) {
    const int mine = __builtin_amdgcn_sbfe(digit, b, 1);      // 0 or -1
    const unsigned long long set = __ballot(mine != 0);
    lo &= ~((uint32_t)set ^ (uint32_t)mine);
    hi &= ~((uint32_t)(set >> 32) ^ (uint32_t)mine);
  }
  return (unsigned long long)hi << 32 | lo;
}
RP_DEV uint32_t key_of(int id, int V) { return (unsigned)id < (unsigned)V ? (uint32_t)id : (uint32_t)V; }

// Up to 128 tokens, one block: a token's place is the number of those before it in the order, found by comparing it with all of them in LDS.  Also clears
// the marks of the rows that have tokens.
__global__ void __launch_bounds__(1024) embed_sort_small_kernel(const int* ids, int T, int V, uint2* sorted, uint32_t* marks) {
  __shared__ __attribute__((aligned(16))) uint32_t keys[SMALL];
  const int i = threadIdx.x;
  const uint32_t mine = i < T ? key_of(ids[i], V) : 0xffffffffu;
  if (i < SMALL) keys[i] = mine;
  if (marks)
    for (int w = i; w < (V + 31) / 32; w += 1024) marks[w] = 0u;
  __syncthreads();
  if (i >= T) return;
  int place = 0;
#pragma unroll 8
  for (int j = 0; j < (T + 3) / 4; ++j) {      // (behind T: the largest number, at higher places)
    const uint4 u = *reinterpret_cast<const uint4*>(keys + 4 * j);
    place += (u.x < mine || (u.x == mine && 4 * j < i)) + (u.y < mine || (u.y == mine && 4 * j + 1 < i)) + (u.z < mine || (u.z == mine && 4 * j + 2 < i)) +
             (u.w < mine || (u.w == mine && 4 * j + 3 < i));
  }
  sorted[place] = make_uint2(mine, (uint32_t)i);
}

// Up to 8192 tokens, one block: radix sort by one or two digits of up to 10 bits, in LDS.  A wave has a 16th of the tokens, 64 at a time; a token's rank among those of its digit
// is that of the wave's earlier ones (counted in LDS) and of the lanes before it (found by ballots).  (4084 tokens: four launches as below 19 us, this one 11.)
constexpr int MID = 8192, MID_EACH = MID / 1024;
struct MidSort {
  uint2 sorted[MID];
  int count[16][MOST_DIGITS];
  int wave[16];
};
__global__ void __launch_bounds__(1024) embed_sort_mid_kernel(const int* ids, int T, int V, int bits, int passes, uint2* out, uint32_t* marks) {
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn_smem[];
  MidSort& m = *reinterpret_cast<MidSort*>(dyn_smem);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, digits = 1 << bits, each = (T + 1023) / 1024;      // each: of a lane
  uint32_t key[MID_EACH], tok[MID_EACH];
#pragma unroll
  for (int j = 0; j < MID_EACH; ++j) {
    const int i = 64 * (each * w + j) + lane;
    tok[j] = (uint32_t)i;
    key[j] = j < each && i < T ? key_of(ids[i], V) : 0u;
  }
  if (marks)
    for (int x = tid; x < (V + 31) / 32; x += 1024) marks[x] = 0u;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    for (int d = lane; d < digits; d += 64) m.count[w][d] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    int rank[MID_EACH];
#pragma unroll
    for (int j = 0; j < MID_EACH; ++j) {
      if (j >= each) break;      // uniform
      const bool in = 64 * (each * w + j) + lane < T;
      const int digit = (int)(key[j] >> shift) & (digits - 1);
      const unsigned long long same = same_digit(digit, bits, in);
      const int ahead = __popcll(same & ((1ull << lane) - 1ull));
      rank[j] = m.count[w][digit] + ahead;      // (all lanes read before the first one of each digit adds, as below)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (in && ahead == 0) m.count[w][digit] += __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // a thread takes a digit: its waves' counts, then where it begins
    int total = 0;
    if (tid < digits)
#pragma unroll
      for (int u = 0; u < 16; ++u) total += m.count[u][tid];
    int sum = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int n = __shfl_up(sum, o, 64);
      if (lane >= o) sum += n;
    }
    if (lane == 63) m.wave[w] = sum;
    __syncthreads();
    int at = sum - total;
    if (tid < digits) {
#pragma unroll
      for (int u = 0; u < 16; ++u) at += u < w ? m.wave[u] : 0;
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const int n = m.count[u][tid];
        m.count[u][tid] = at;
        at += n;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MID_EACH; ++j) {
      const int i = 64 * (each * w + j) + lane;
      if (j < each && i < T) m.sorted[m.count[w][(int)(key[j] >> shift) & (digits - 1)] + rank[j]] = make_uint2(key[j], tok[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MID_EACH; ++j) {
      const int i = 64 * (each * w + j) + lane;
      if (j < each && i < T) {
        const uint2 e = m.sorted[i];
        key[j] = e.x;
        tok[j] = e.y;
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < MID_EACH; ++j) {
    const int i = 64 * (each * w + j) + lane;
    if (j < each && i < T) out[i] = make_uint2(key[j], tok[j]);
  }
}

// More: radix sort by two digits (one where one is enough), each counted and then scattered.  Every block has a run of `run` tokens.  (Counted by atomics while the first
// digit is scattered, the second one's counts of the frequent tokens meet on a few addresses: 62 us for 16384 tokens instead of 8 and a launch.)
struct SortArgs {
  const int* ids;
  uint2 *from, *to;                // {key, token}; the first pass reads ids
  int* counts;                     // [blocks][digits]
  uint32_t* marks;                 // [ceil(V / 32)], cleared here, or NULL
  int T, V, run, blocks, shift, bits, pass;
};

__global__ void __launch_bounds__(NT) embed_count_kernel(const SortArgs p) {
  __shared__ int hist[MOST_DIGITS];
  const int digits = 1 << p.bits, tid = threadIdx.x;
  for (int d = tid; d < digits; d += NT) hist[d] = 0;
  __syncthreads();
  const long first = (long)blockIdx.x * p.run, last = min(first + p.run, (long)p.T);
  for (long i = first + tid; i < last; i += NT) atomicAdd(hist + (int)((p.pass == 0 ? key_of(p.ids[i], p.V) : p.from[i].x) >> p.shift & (digits - 1)), 1);
  __syncthreads();
  int* const mine = p.counts + (long)blockIdx.x * digits;
  for (int d = tid; d < digits; d += NT) mine[d] = hist[d];
  if (p.marks && p.pass == 0)
    for (int w = blockIdx.x * NT + tid; w < (p.V + 31) / 32; w += p.blocks * NT) p.marks[w] = 0u;
}

__global__ void __launch_bounds__(NT) embed_scatter_kernel(const SortArgs p) {
  __shared__ int base[MOST_DIGITS];            // where the block's next token of a digit goes
  __shared__ int count[NT / 64][MOST_DIGITS];  // a wave's, then where its first goes
  __shared__ int wave_total[NT / 64];
  const int digits = 1 << p.bits, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  // places before a digit: all smaller digits, and this one in the blocks before
  int before_chunk = 0;
  for (int d0 = 0; d0 < digits; d0 += NT) {
    const int d = d0 + tid;
    int total = 0, before = 0;
    if (d < digits) {
#pragma unroll 8
      for (int b = 0; b < p.blocks; ++b) {
        const int n = p.counts[(long)b * digits + d];
        before += b < (int)blockIdx.x ? n : 0;
        total += n;
      }
    }
    int sum = total;      // inclusive over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int n = __shfl_up(sum, o, 64);
      if (lane >= o) sum += n;
    }
    if (lane == 63) wave_total[w] = sum;
    __syncthreads();
    int smaller = before_chunk;
    for (int u = 0; u < NT / 64; ++u) {
      if (u < w) smaller += wave_total[u];
      before_chunk += wave_total[u];
    }
    if (d < digits) base[d] = smaller + sum - total + before;
    __syncthreads();
  }
  const long first = (long)blockIdx.x * p.run, last = min(first + p.run, (long)p.T);
  for (long i0 = first; i0 < last; i0 += BATCH) {
    for (int d = tid; d < digits; d += NT)
#pragma unroll
      for (int u = 0; u < NT / 64; ++u) count[u][d] = 0;
    __syncthreads();
    uint32_t key[4], tok[4];
    int digit[4], rank[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long i = i0 + 256 * w + 64 * j + lane;
      const bool in = i < last;
      key[j] = tok[j] = 0u;
      if (in) {
        if (p.pass == 0) {
          key[j] = key_of(p.ids[i], p.V);
          tok[j] = (uint32_t)i;
        } else {
          const uint2 e = p.from[i];
          key[j] = e.x;
          tok[j] = e.y;
        }
      }
      digit[j] = (int)(key[j] >> p.shift) & (digits - 1);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool in = i0 + 256 * w + 64 * j + lane < last;
      const unsigned long long same = same_digit(digit[j], p.bits, in);
      const int ahead = __popcll(same & ((1ull << lane) - 1ull));
      // all lanes read before the first one of each digit adds (LDS works in order for a wave, so the fences are for the compiler)
      rank[j] = count[w][digit[j]] + ahead;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (in && ahead == 0) count[w][digit[j]] += __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (int d = tid; d < digits; d += NT) {
      int at = base[d];
#pragma unroll
      for (int u = 0; u < NT / 64; ++u) {
        const int n = count[u][d];
        count[u][d] = at;
        at += n;
      }
      base[d] = at;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + 256 * w + 64 * j + lane < last) {
        const int at = count[w][digit[j]] + rank[j];
        p.to[at] = make_uint2(key[j], tok[j]);
      }
    }
    __syncthreads();
  }
}

// Zeros for the rows without tokens: `lanes` threads take a row, 16 bytes a thread and step.  lanes is a power of two.  (Blocks that go through the table in steps of the grid, all of
// their threads on one row: 151936 rows of 4096 462 us instead of 432, of 64 35 instead of 15.5.)
__global__ void __launch_bounds__(NT) embed_clear_kernel(const EmbedGrad p, const uint32_t* marks, int lanes) {
  const int h4 = p.h / 4, lane = threadIdx.x & (lanes - 1);
  const long v = (long)blockIdx.x * (NT / lanes) + threadIdx.x / lanes;
  if (v >= p.V || (marks[v >> 5] >> (v & 31) & 1u)) return;
  float4* const row = reinterpret_cast<float4*>(p.dtable + v * p.ldt);
  for (int c = lane; c < h4; c += lanes) row[c] = make_float4(0.f, 0.f, 0.f, 0.f);
}

// ------------------------------------------------------------------------------------------------ sums
struct SumArgs {
  EmbedGrad g;
  const uint2* sorted;
  float* part;      // [2][chunks][h]: a chunk's run that began before it, and its run that goes on behind it
  uint32_t* marks;  // a bit for every row that has tokens, or NULL
  int chunk, chunks, slices, width, lanes;      // width: 8-element pieces of a slice
};

struct Sum8 {
  float v[8];
  RP_DEV void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
  }
  RP_DEV void add(const uint4& u) {
    v[0] += bf16_lo(u.x); v[1] += bf16_hi(u.x); v[2] += bf16_lo(u.y); v[3] += bf16_hi(u.y);
    v[4] += bf16_lo(u.z); v[5] += bf16_hi(u.z); v[6] += bf16_lo(u.w); v[7] += bf16_hi(u.w);
  }
  RP_DEV void add(const float* src) {
    const float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 4);
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
  }
  RP_DEV void store(float* dst) const {
    *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(dst + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
  // to the table
  RP_DEV void finish(const EmbedGrad& p, uint32_t key, int col) const {
    float* const row = p.dtable + (long)key * p.ldt + col;
    Sum8 r;
    r.clear();
    if (p.accumulate) r.add(row);
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] += p.scale * v[e];
    r.store(row);
  }
};

// `lanes` threads take a chunk of the sorted tokens and a slice of the columns.  The rows of eight tokens are on their way at a time: their addresses first, then the
// rows, with no branch in between (a load under a condition waited for the one before: 16384 tokens of 4096 84 us instead of 75, 4084 of 2880 19 instead of 17).
__global__ void __launch_bounds__(NT) embed_sum_kernel(const SumArgs p) {
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & (p.lanes - 1);
  const long unit = (long)blockIdx.x * (NT / p.lanes) + threadIdx.x / p.lanes;
  const int chunk = (int)(unit / p.slices), slice = (int)(unit - (long)chunk * p.slices);
  const int piece = slice * p.width + lane, col = 8 * piece;
  if (chunk >= p.chunks || lane >= p.width || col >= p.g.h) return;
  const int first = chunk * p.chunk, last = min(first + p.chunk, p.g.T);
  const uint32_t none = (uint32_t)p.g.V;
  const uint32_t prev = first > 0 ? p.sorted[first - 1].x : 0xffffffffu, next = last < p.g.T ? p.sorted[last].x : 0xffffffffu;
  Sum8 sum;
  sum.clear();
  uint32_t now = p.sorted[first].x;
  bool began = now != prev;      // the present run began in this chunk
  const bool marks = p.marks && slice == 0 && lane == 0;
  if (marks && began && now != none) atomicOr(p.marks + (now >> 5), 1u << (now & 31));
  for (int i0 = first; i0 < last; i0 += AHEAD) {
    uint4 row[AHEAD];
    uint2 at[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) at[j] = p.sorted[min(i0 + j, last - 1)];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) row[j] = *reinterpret_cast<const uint4*>(p.g.dx + (long)at[j].y * p.g.lddx + col);      // (a token without a row has a dx, which is added to nothing)
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (i0 + j >= last) break;
      if (at[j].x != now) {
        if (now != none) {
          if (began) sum.finish(p.g, now, col);
          else sum.store(p.part + (long)chunk * p.g.h + col);
        }
        sum.clear();
        now = at[j].x;
        began = true;
        if (marks && now != none) atomicOr(p.marks + (now >> 5), 1u << (now & 31));
      }
      sum.add(row[j]);
    }
  }
  if (now == none) return;
  if (!began) sum.store(p.part + (long)chunk * p.g.h + col);                              // also a run through the whole chunk
  else if (now == next) sum.store(p.part + ((long)p.chunks + chunk) * p.g.h + col);
  else sum.finish(p.g, now, col);
}

// The runs over several chunks, at the chunk that they begin in: its last part and the first ones of the chunks behind it.  32 threads take 256 columns,
// eight such groups every eighth part.
__global__ void __launch_bounds__(NT) embed_join_kernel(const SumArgs p) {
  __shared__ float red[8][256];
  __shared__ int parts;
  const int slices = (p.g.h + 255) / 256;
  const int chunk = (int)(blockIdx.x / slices), slice = (int)(blockIdx.x - (unsigned)chunk * slices);
  const int first = chunk * p.chunk, last = first + p.chunk;      // (the last chunk of all has no block)
  const uint32_t v = p.sorted[last - 1].x;
  if (v != p.sorted[last].x || v == (uint32_t)p.g.V) return;                                          // no run goes on
  if (first > 0 && p.sorted[first - 1].x == v && p.sorted[first].x == v) return;                      // it began earlier
  const int tid = threadIdx.x;
  if (tid < 64) {      // chunks behind that begin with it
    int n = 0;
    for (;;) {
      const long at = last + (long)(n + tid) * p.chunk;
      const bool more = at < p.g.T && p.sorted[at].x == v;
      const unsigned long long m = __ballot(more);
      if (~m) {
        n += __builtin_ctzll(~m);
        break;
      }
      n += 64;
    }
    if (tid == 0) parts = n;
  }
  __syncthreads();
  const int grp = tid >> 5, lane = tid & 31, col = slice * 256 + 8 * lane;
  const bool in = col < p.g.h;
  Sum8 sum;
  sum.clear();
  if (in) {
    if (grp == 0) sum.add(p.part + ((long)p.chunks + chunk) * p.g.h + col);
#pragma unroll 4
    for (int i = grp; i < parts; i += 8) sum.add(p.part + (long)(chunk + 1 + i) * p.g.h + col);
  }
  sum.store(&red[grp][8 * lane]);
  __syncthreads();
  if (grp || !in) return;
#pragma unroll
  for (int u = 1; u < 8; ++u) sum.add(&red[u][8 * lane]);
  sum.finish(p.g, v, col);
}

int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }
size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }

// Digits: the numbers 0 .. V in one pass of up to 10 bits, or in two.
struct SortPlan {
  int bits, passes, blocks, run;
  SortPlan(int T, int V) {
    int all = 1;
    while ((1l << all) <= V) ++all;
    passes = all > 10 ? 2 : 1;
    bits = (all + passes - 1) / passes;
    blocks = ceil_div(T, BATCH);
    if (blocks > MOST_BLOCKS) blocks = MOST_BLOCKS;
    if (blocks < 1) blocks = 1;
    run = ceil_div(ceil_div(T, blocks), BATCH) * BATCH;
    blocks = T ? ceil_div(T, run) : 1;
  }
};
// Sorted tokens that a group of threads adds up.
// Shorter chunks keep more of the chip busy, longer ones leave fewer parts to join: both kernels, 4084 tokens of
// 2880 in chunks of 4 | 8 | 16 27.6 | 23.7 | 24.8 us, 16384 of 4096 in 16 | 32 91 | 83.
int chunk_length(int T) { return T >= 8192 ? 32 : T >= 2048 ? 8 : 4; }

struct Places {      // of the scratch memory
  size_t sorted, other, counts, marks, part, end;
  Places(int T, int V, int h) {
    const SortPlan s(T, V);
    sorted = 0;
    other = round16((size_t)T * 8);
    counts = other + (T > MID && s.passes > 1 ? round16((size_t)T * 8) : 0);
    marks = counts + (T > MID ? round16((size_t)s.blocks * (4 << s.bits)) : 0);
    part = marks + round16((size_t)((V + 31) / 32) * 4);
    end = part + (size_t)2 * ceil_div(T, chunk_length(T)) * h * 4;
  }
};

}  // namespace

hipError_t k_embed_fwd(hipStream_t st, const bf16* table, long ldt, const int* ids, float scale, bf16* x, long ldx, int T, int V, int h) {
  if (T == 0 || h == 0) return hipSuccess;
  int lanes = 1;
  while (lanes < NT && lanes < h / 8) lanes <<= 1;
  RP_LAUNCH(embed_rows_kernel, dim3(ceil_div(T, NT / lanes)), dim3(NT), 0, st, table, ldt, ids, scale, x, ldx, T, V, h / 8, lanes);
  return hipGetLastError();
}

size_t k_embed_scratch(int T, int V, int h) { return Places(T, V, h).end; }

hipError_t k_embed_bwd(hipStream_t st, const EmbedGrad& g, void* scratch) {
  if (g.h == 0 || g.V == 0 || (g.T == 0 && g.accumulate)) return hipSuccess;
  hipError_t e = hipSuccess;
  char* const mem = static_cast<char*>(scratch);
  const Places at(g.T, g.V, g.h);
  const SortPlan s(g.T, g.V);
  uint32_t* const marks = g.accumulate ? nullptr : reinterpret_cast<uint32_t*>(mem + at.marks);
  uint2* const sorted = reinterpret_cast<uint2*>(mem + at.sorted);
  if (g.T <= SMALL) {
    RP_LAUNCH(embed_sort_small_kernel, dim3(1), dim3(1024), 0, st, g.ids, g.T, g.V, sorted, marks);
    e = hipGetLastError();
  } else if (g.T <= MID) {
    // (a host-side table entry, not a stream operation: allowed while a graph is captured)
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(embed_sort_mid_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(MidSort));
    if (e != hipSuccess) return e;
    RP_LAUNCH(embed_sort_mid_kernel, dim3(1), dim3(1024), sizeof(MidSort), st, g.ids, g.T, g.V, s.bits, s.passes, sorted, marks);
    e = hipGetLastError();
  } else {
    uint2* const other = reinterpret_cast<uint2*>(mem + at.other);
    SortArgs a{g.ids, nullptr, s.passes > 1 ? other : sorted, reinterpret_cast<int*>(mem + at.counts), marks, g.T, g.V, s.run, s.blocks, 0, s.bits, 0};
    for (int pass = 0; pass < s.passes && e == hipSuccess; ++pass) {
      a.pass = pass;
      a.shift = pass * s.bits;
      if (pass == 1) { a.from = other; a.to = sorted; }
      RP_LAUNCH(embed_count_kernel, dim3(s.blocks), dim3(NT), 0, st, a);
      e = hipGetLastError();
      if (e != hipSuccess) break;
      RP_LAUNCH(embed_scatter_kernel, dim3(s.blocks), dim3(NT), 0, st, a);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  SumArgs a{};
  a.g = g;
  a.sorted = sorted;
  a.part = reinterpret_cast<float*>(mem + at.part);
  a.chunk = chunk_length(g.T);
  a.chunks = ceil_div(g.T, a.chunk);
  a.slices = ceil_div(g.h / 8, NT);
  a.width = ceil_div(g.h / 8, a.slices);
  a.lanes = 1;
  while (a.lanes < a.width) a.lanes <<= 1;
  a.marks = marks;
  if (a.chunks > 0) {
    RP_LAUNCH(embed_sum_kernel, dim3(ceil_div((long)a.chunks * a.slices, NT / a.lanes)), dim3(NT), 0, st, a);
    e = hipGetLastError();
  }
  if (a.chunks > 1 && e == hipSuccess) {
    RP_LAUNCH(embed_join_kernel, dim3((unsigned)(a.chunks - 1) * ((g.h + 255) / 256)), dim3(NT), 0, st, a);
    e = hipGetLastError();
  }
  if (!marks || e != hipSuccess) return e;
  int lanes = 1;
  while (lanes < NT && lanes < g.h / 4) lanes <<= 1;
  RP_LAUNCH(embed_clear_kernel, dim3(ceil_div(g.V, NT / lanes)), dim3(NT), 0, st, g, marks, lanes);
  return hipGetLastError();
}
