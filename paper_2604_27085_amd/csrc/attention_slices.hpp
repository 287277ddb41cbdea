// What the attentions whose loop may be cut into slices share: the slices, their launches and the way they are joined.
#pragma once
#include "attention_device.hpp"

namespace {

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

// The larger of two, for the sizes of LDS.
constexpr int max_i(int a, int b) { return a > b ? a : b; }
template <typename K, typename Args, typename... More>
hipError_t launch(K kern, int grid, int threads, int smem, hipStream_t st, const Args& p, More... more) {
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
// Threads that share a row of n slices.
int join_groups(int n) { return n < 6 ? 1 : n < 24 ? 4 : 16; }

}  // namespace
