// Attention over a prefix that sequences share: the plain kernel.
//
// K and V of the prefix are there once per (layer, KV head), and the newest queries of all sequences that share it are
// the rows of one product with them.  What is left of it for each query head is o = sum 2^(y_n - m) v_n with y_n the logit in log2
// units, the largest of them m and the sum l = sum 2^(y_n - m), all in 32 bits.  Long prefixes are cut over
// workgroups, each piece with an (o, m, l) of its own, and the decode kernels join the pieces with what they have of the
// sequence's own cache (PrefixPieces), so the result is one softmax over all.
#include "gkv_internal.h"

namespace {

constexpr int NWG = 4;

// Dynamic LDS, per wavefront: float qs[d]; float prob[64]
template <typename T>
__global__ __launch_bounds__(NWG * 64) void prefix_generic_kernel(GkvDims dm, PrefixArgs a) {
  extern __shared__ float smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int d = dm.d, g = dm.g;
  const int unit = blockIdx.x, j = unit % dm.Hkv, i = unit / dm.Hkv % a.count, layer = unit / dm.Hkv / a.count;
  float* qs = smem + wave * (d + 64);
  float* prob = qs + d;
  const size_t head0 = ((size_t)layer * dm.B + a.first + i) * dm.Hq + j * g;
  const size_t at = ((size_t)layer * dm.Hkv + j) * a.capacity * d;
  const T* K = (const T*)a.K + at;
  const T* V = (const T*)a.V + at;
  const int n0 = (int)blockIdx.y * a.split_rows, n1 = min(a.rows, n0 + a.split_rows);
  for (int hi = wave; hi < g; hi += NWG) {
    const T* qh = (const T*)a.q + (head0 + hi) * d;
    for (int c = lane; c < d; c += 64) qs[c] = Elem<T>::ld(qh + c);
    constexpr int MOST = 8;                                // d <= 512
    float acc[MOST];
#pragma unroll
    for (int x = 0; x < MOST; ++x) acc[x] = 0.f;
    float m = GKV_NO_MAX, sum = 0.f;
    for (int n = n0; n < n1; n += 64) {
      const bool there = n + lane < n1;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const T* row = K + (size_t)(there ? n + lane : n) * d;
      float z = 0.f;
      for (int c = 0; c < d; ++c) z = fmaf(qs[c], Elem<T>::ld(row + c), z);
      const float mn = fmaxf(m, wave_max(there ? rounded_product(z, dm.scale_l2_hi) : GKV_NO_MAX));
      const float p = there ? exp2f(log2_weight(z, dm.scale_l2_hi, dm.scale_l2_lo, mn)) : 0.f;
      prob[lane] = p;
      const float f = exp2f(m - mn);
      sum = sum * f + wave_sum(p);
      m = mn;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
      for (int x = 0; x < MOST; ++x)
        if (lane + 64 * x < d) {
          float o = acc[x] * f;
          for (int y = 0; y < min(64, n1 - n); ++y) o = fmaf(prob[y], Elem<T>::ld(V + (size_t)(n + y) * d + lane + 64 * x), o);
          acc[x] = o;
        }
    }
    const size_t to = (size_t)blockIdx.y * a.heads + head0 + hi;
#pragma unroll
    for (int x = 0; x < MOST; ++x)
      if (lane + 64 * x < d) a.o[to * d + lane + 64 * x] = acc[x];
    if (lane == 0) {
      a.ms[to] = make_float2(prefix_max(m, sum, n1 > n0), sum);
      if (blockIdx.y == 0) a.n[to] = a.splits;
    }
  }
}

}  // namespace

hipError_t gkv_launch_prefix_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PrefixArgs& a) {
  const dim3 grid(dm.L * a.count * dm.Hkv, a.splits);
  const size_t shmem = sizeof(float) * NWG * (dm.d + 64);
  if (dtype == GKV_F32) return gkv_launch(ln, prefix_generic_kernel<float>, grid, dim3(NWG * 64), shmem, dm, a);
  return gkv_launch(ln, prefix_generic_kernel<uint16_t>, grid, dim3(NWG * 64), shmem, dm, a);
}
