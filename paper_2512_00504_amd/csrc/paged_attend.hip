// Decode attention over pages: the plain vector-ALU kernel, for every type, head_dim, group and page size.
//
// A workgroup of 4 wavefronts per (unit, piece), a wavefront per query head of the group in turn.  A piece is a run of slices of
// 16 rows; its running maximum, sum and weighted values are joined with the other pieces' by the wavefront that comes last.
// A lane takes one of 64 keys for the logits and every 64th channel for the values.
#include "gkv_internal.h"

namespace {

constexpr int NWG = 4, KEYS = 64, MOST = 8;                // channels of a lane: d <= 512

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Dynamic LDS, per wavefront: float qs[d]; float prob[64]; int64 row[64]
template <typename T>
__global__ __launch_bounds__(NWG * 64) void paged_attend_generic_kernel(GkvDims dm, PagedAttendArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem_bytes[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d = dm.d, g = dm.g, pr = a.pages.page_rows;
  const int units = dm.L * dm.B * dm.Hkv, sp = blockIdx.x / units, unit = blockIdx.x % units;
  const int lb = unit / dm.Hkv, j = unit - lb * dm.Hkv, layer = lb / dm.B, i = lb - layer * dm.B;
  const int64_t room = (int64_t)a.pages.width * pr;
  const int len = (int)min((int64_t)max(a.len[i], 0), room);
  const int n_iter = (len + 15) >> 4;
  const int ns = max(1, min(a.splits, max(min((n_iter + a.split_iters - 1) / a.split_iters, a.soft), (n_iter + a.long_iters - 1) / a.long_iters)));
  if (sp >= ns) return;
  const int per = (n_iter + ns - 1) / ns;
  const int n0 = min(len, sp * per * 16), n1 = min(len, (sp + 1) * per * 16);
  float* qs = (float*)(smem_bytes + wave * ((size_t)4 * (d + KEYS) + 8 * KEYS));
  float* prob = qs + d;
  int64_t* row = (int64_t*)(prob + KEYS);
  const size_t layer_rows = (size_t)a.pages.n_pages * dm.Hkv * pr;
  const T* K = (const T*)a.K + layer * layer_rows * d;
  const T* V = (const T*)a.V + layer * layer_rows * d;
  const int32_t* table = a.pages.table + (int64_t)i * a.pages.width;
  for (int hi = wave; hi < g; hi += NWG) {
    const size_t head = (size_t)lb * dm.Hq + j * g + hi;
    const T* qh = (const T*)a.q + head * d;
    wave_sync();
    for (int c = lane; c < d; c += 64) qs[c] = Elem<T>::ld(qh + c);
    float acc[MOST];
#pragma unroll
    for (int x = 0; x < MOST; ++x) acc[x] = 0.f;
    float m = GKV_NO_MAX, sum = 0.f;
    bool any = false;
    for (int n = n0; n < n1; n += KEYS) {
      const int key = min(n + lane, n1 - 1), page = quotient(key, a.pages.by_rows);
      const int32_t id = table[page];
      const bool there = n + lane < n1 && id >= 0 && id < a.pages.n_pages;
      const int64_t at = there ? ((int64_t)id * dm.Hkv + j) * pr + (key - page * pr) : -1;
      wave_sync();
      float z = 0.f;
      if (there)
        for (int c = 0; c < d; ++c) z = fmaf(qs[c], Elem<T>::ld(K + at * d + c), z);
      const float mn = fmaxf(m, wave_max(there ? rounded_product(z, dm.scale_l2_hi) : GKV_NO_MAX));
      const float p = there ? exp2f(log2_weight(z, dm.scale_l2_hi, dm.scale_l2_lo, mn)) : 0.f;
      prob[lane] = p;
      row[lane] = at;
      any |= __any(there);
      const float f = exp2f(m - mn);
      sum = sum * f + wave_sum(p);
      m = mn;
      wave_sync();
#pragma unroll
      for (int x = 0; x < MOST; ++x) acc[x] *= f;
      for (int y = 0; y < min(KEYS, n1 - n); ++y) {
        if (row[y] < 0) continue;                            // uniform
        const T* v = V + row[y] * d;
#pragma unroll
        for (int x = 0; x < MOST; ++x)
          if (lane + 64 * x < d) acc[x] = fmaf(prob[y], Elem<T>::ld(v + lane + 64 * x), acc[x]);
      }
    }
    m = sum == 0.f && any ? -INFINITY : m;                   // keys, none of them with weight
    T* out = (T*)a.out + head * d;
    if (ns == 1) {
      const float inv = inverse_total(sum, m == -INFINITY);
#pragma unroll
      for (int x = 0; x < MOST; ++x)
        if (lane + 64 * x < d) Elem<T>::st(out + lane + 64 * x, acc[x] * inv);
      continue;
    }
    float* to = a.partials + (((size_t)unit * a.most + sp) * g + hi) * (d + 2);
#pragma unroll
    for (int x = 0; x < MOST; ++x)
      if (lane + 64 * x < d) __hip_atomic_store(to + lane + 64 * x, acc[x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (lane == 0) {
      __hip_atomic_store(to + d, m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(to + d + 1, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (ns == 1 || wave >= g) return;
  // A wavefront's heads need the same wavefront's of the other pieces: it waits for its own stores, takes a ticket, and the last one joins.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  uint32_t arrived = 0;
  if (lane == 0)
    arrived = __builtin_amdgcn_atomic_inc32((uint32_t*)a.ticket + ((size_t)unit * GKV_TICKETS + wave) * GKV_PAGED_TICKET, (uint32_t)ns - 1u, __ATOMIC_RELAXED, "agent");
  if ((int)__builtin_amdgcn_readfirstlane(arrived) != ns - 1) return;
  asm volatile("" ::: "memory");
  for (int hi = wave; hi < g; hi += NWG) {
    const float* from = a.partials + ((size_t)unit * a.most * g + hi) * (d + 2);
    const size_t step = (size_t)g * (d + 2);
    auto get = [&](int s, int c) { return __hip_atomic_load(from + s * step + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    float m = GKV_NO_MAX, sum = 0.f;
    bool any = false;
    for (int s = 0; s < ns; ++s) {
      const float ms = get(s, d);
      any |= ms == -INFINITY || get(s, d + 1) != 0.f;
      m = fmaxf(m, ms);
    }
    float acc[MOST];
#pragma unroll
    for (int x = 0; x < MOST; ++x) acc[x] = 0.f;
    for (int s = 0; s < ns; ++s) {                           // (a piece without weight has sums of zero, or NaN from infinite values)
      const float f = exp2f(get(s, d) - m);
      sum = fmaf(get(s, d + 1), f, sum);
#pragma unroll
      for (int x = 0; x < MOST; ++x)
        if (lane + 64 * x < d) acc[x] = fmaf(get(s, lane + 64 * x), f, acc[x]);
    }
    const float inv = inverse_total(sum, any);
    T* out = (T*)a.out + ((size_t)lb * dm.Hq + j * g + hi) * d;
#pragma unroll
    for (int x = 0; x < MOST; ++x)
      if (lane + 64 * x < d) Elem<T>::st(out + lane + 64 * x, acc[x] * inv);
  }
}

}  // namespace

hipError_t gkv_launch_paged_attend_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PagedAttendArgs& a) {
  const dim3 grid(dm.L * dm.B * dm.Hkv * a.splits);
  const size_t shmem = (size_t)NWG * (4 * (dm.d + KEYS) + 8 * KEYS);
  if (dtype == GKV_F32) return gkv_launch(ln, paged_attend_generic_kernel<float>, grid, dim3(NWG * 64), shmem, dm, a);
  return gkv_launch(ln, paged_attend_generic_kernel<uint16_t>, grid, dim3(NWG * 64), shmem, dm, a);
}
