// Decode attention over pages: the plain vector-ALU kernel, for every type, head_dim, group and page size.
//
// A workgroup of 4 wavefronts per (unit, piece).  A piece is a run of slices of 16 rows, of which the wavefronts take 64 at a time in turn, for
// GB of the group's heads at once (a further round over the piece for each GB heads more).  For the logits a lane has a key and reads its row in
// 16-byte pieces, each used for all GB heads; for the values it has CH neighbouring channels of every key.  Wavefronts are joined through LDS,
// pieces of a unit by the workgroup that finishes last, in their order.
// Bound: instructions, 2 d GB of the vector ALU a key and lane and as many reads of LDS.  us, one element at a time and one head a wavefront -> so:
// 8 sequences of 4096 rows, 8 KV heads of 4 heads, fp32, d = 96 531 -> 97 (201 MB, part of them in the memory-side cache; cold 124, 1.6 TB/s); 32 KV heads
// of one, bf16, d = 80 728 -> 220 (1.5 TB/s).
#include "gkv_internal.h"

namespace {

constexpr int NWG = 4, KEYS = 64, GB = 4;

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// N elements side by side as floats; ALIGNED: their address is a multiple of their size.
template <typename T, int N, bool ALIGNED>
__device__ __forceinline__ void load_row(const T* p, float (&x)[N]) {
  if constexpr (ALIGNED) {
    struct __attribute__((aligned(N * sizeof(T)))) { T e[N]; } v;
    v = *(const decltype(v)*)p;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = Elem<T>::ld(v.e + i);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = Elem<T>::ld(p + i);
  }
}

__device__ __forceinline__ void put(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Dynamic LDS: float qs[GB][d]; then per wavefront float prob[GB][64], int64 row[64], float ms[GB][2]; then float sums[NWG][GB][d].
template <typename T, int CH, bool ALIGNED>
__global__ __launch_bounds__(NWG * 64) void paged_attend_generic_kernel(GkvDims dm, PagedAttendArgs a) {
  constexpr int EPC = Elem<T>::EPC;
  extern __shared__ __attribute__((aligned(16))) char smem_bytes[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d = dm.d, g = dm.g, pr = a.pages.page_rows;
  const int units = dm.L * dm.B * dm.Hkv, sp = blockIdx.x / units, unit = blockIdx.x % units;
  const int lb = unit / dm.Hkv, j = unit - lb * dm.Hkv, layer = lb / dm.B, i = lb - layer * dm.B;
  const int64_t room = (int64_t)a.pages.width * pr;
  const int len = (int)min((int64_t)max(a.len[i], 0), room);
  const int n_iter = (len + 15) >> 4;
  const int ns = max(1, min(a.splits, a.cut.pieces(n_iter)));
  if (sp >= ns) return;
  const int per = (n_iter + ns - 1) / ns;
  const int n0 = min(len, sp * per * 16), n1 = min(len, (sp + 1) * per * 16);
  float* qs = (float*)smem_bytes;
  char* own = smem_bytes + (size_t)4 * GB * d;
  constexpr size_t OWN = 4 * GB * KEYS + 8 * KEYS + 8 * GB;
  float* prob = (float*)(own + wave * OWN);                  // [64][GB]
  int64_t* row = (int64_t*)(prob + GB * KEYS);
  float* ms = (float*)(row + KEYS);
  float* sums = (float*)(own + NWG * OWN);
  const size_t layer_rows = (size_t)a.pages.n_pages * dm.Hkv * pr;
  const T* K = (const T*)a.K + layer * layer_rows * d;
  const T* V = (const T*)a.V + layer * layer_rows * d;
  const int32_t* table = a.pages.table + (int64_t)i * a.pages.width;
  const size_t head0 = (size_t)lb * dm.Hq + j * g;
  const int ch = lane * CH;                                   // this lane's first channel
  const bool has = ch < d;                                    // (d is a multiple of CH)
  float* part = a.partials + (size_t)unit * a.most * g * (d + 2);   // [piece][g][d + 2]

  for (int h0 = 0; h0 < g; h0 += GB) {
    __syncthreads();
    for (int x = tid; x < GB * d; x += NWG * 64) {            // (beyond the group: its last head again)
      const int h = x / d;
      qs[x] = Elem<T>::ld((const T*)a.q + (head0 + min(h0 + h, g - 1)) * d + (x - h * d));
    }
    __syncthreads();
    float acc[GB][CH], m[GB], sum[GB];
#pragma unroll
    for (int h = 0; h < GB; ++h) {
      m[h] = GKV_NO_MAX;
      sum[h] = 0.f;
#pragma unroll
      for (int x = 0; x < CH; ++x) acc[h][x] = 0.f;
    }
    bool any = false;
    for (int n = n0 + wave * KEYS; n < n1; n += NWG * KEYS) {
      const int key = min(n + lane, n1 - 1), page = quotient(key, a.pages.by_rows);
      const int32_t id = table[page];
      const bool there = n + lane < n1 && id >= 0 && id < a.pages.n_pages;
      const int64_t at = there ? ((int64_t)id * dm.Hkv + j) * pr + (key - page * pr) : -1;
      float z[GB];
#pragma unroll
      for (int h = 0; h < GB; ++h) z[h] = 0.f;
      if (there)
        for (int c = 0; c < d; c += EPC) {
          float k[EPC];
          load_row<T, EPC, ALIGNED>(K + at * d + c, k);
#pragma unroll
          for (int h = 0; h < GB; ++h)
#pragma unroll
            for (int x = 0; x < EPC; ++x) z[h] = fmaf(qs[h * d + c + x], k[x], z[h]);
        }
      any |= __any(there);
      wave_sync();
#pragma unroll
      for (int h = 0; h < GB; ++h) {
        const float mn = fmaxf(m[h], wave_max(there ? rounded_product(z[h], dm.scale_l2_hi) : GKV_NO_MAX));
        const float p = there ? exp2f(log2_weight(z[h], dm.scale_l2_hi, dm.scale_l2_lo, mn)) : 0.f;
        prob[lane * GB + h] = p;
        const float f = exp2f(m[h] - mn);
        sum[h] = sum[h] * f + wave_sum(p);
        m[h] = mn;
#pragma unroll
        for (int x = 0; x < CH; ++x) acc[h][x] *= f;
      }
      row[lane] = at;
      wave_sync();
      const int most = min(KEYS, n1 - n);
#pragma unroll 4
      for (int y = 0; y < most; ++y) {
        const int64_t r = row[y];
        if (r < 0) continue;                                  // uniform
        float v[CH];
#pragma unroll
        for (int x = 0; x < CH; ++x) v[x] = 0.f;
        if (has) load_row<T, CH, ALIGNED>(V + r * d + ch, v);
#pragma unroll
        for (int h = 0; h < GB; ++h)
#pragma unroll
          for (int x = 0; x < CH; ++x) acc[h][x] = fmaf(prob[y * GB + h], v[x], acc[h][x]);
      }
    }
#pragma unroll
    for (int h = 0; h < GB; ++h) {
      if (has)
#pragma unroll
        for (int x = 0; x < CH; ++x) sums[(wave * GB + h) * d + ch + x] = acc[h][x];
      if (lane == 0) {
        ms[2 * h] = sum[h] == 0.f && any ? -INFINITY : m[h];  // keys, none of them with weight
        ms[2 * h + 1] = sum[h];
      }
    }
    __syncthreads();
    // a wavefront a head
    for (int h = wave; h < min(GB, g - h0); h += NWG) {
      float M = GKV_NO_MAX, total = 0.f, f[NWG];
      bool some = false;
#pragma unroll
      for (int w = 0; w < NWG; ++w) {
        const float* o = (const float*)(own + w * OWN) + GB * KEYS + 2 * KEYS + 2 * h;
        some |= o[0] == -INFINITY || o[1] != 0.f;
        M = fmaxf(M, o[0]);
      }
#pragma unroll
      for (int w = 0; w < NWG; ++w) {
        const float* o = (const float*)(own + w * OWN) + GB * KEYS + 2 * KEYS + 2 * h;
        f[w] = exp2f(o[0] - M);
        total = fmaf(o[1], f[w], total);
      }
      const float inv = ns == 1 ? inverse_total(total, some) : 1.f;
      float* to = part + ((size_t)sp * g + h0 + h) * (d + 2);
      for (int c = lane; c < d; c += 64) {
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < NWG; ++w) o = fmaf(sums[(w * GB + h) * d + c], f[w], o);
        if (ns == 1) Elem<T>::st((T*)a.out + (head0 + h0 + h) * d + c, o * inv);
        else put(to + c, o);
      }
      if (ns > 1 && lane == 0) {
        put(to + d, total == 0.f && some ? -INFINITY : M);
        put(to + d + 1, total);
      }
    }
  }
  if (ns == 1) return;
  // Every wavefront waits for its own stores, the workgroup takes a ticket, and the last one joins.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0)
    *(uint32_t*)smem_bytes = __builtin_amdgcn_atomic_inc32((uint32_t*)a.ticket + (size_t)unit * gkv_paged_parts(g) * GKV_TICKETS * GKV_PAGED_TICKET,
                                                           (uint32_t)ns - 1u, __ATOMIC_RELAXED, "agent");
  __syncthreads();
  if (*(volatile int*)smem_bytes != ns - 1) return;
  for (int h = wave; h < g; h += NWG) {
    const float* from = part + (size_t)h * (d + 2);
    const size_t step = (size_t)g * (d + 2);
    float M = GKV_NO_MAX, total = 0.f;
    bool some = false;
    for (int s = 0; s < ns; ++s) {
      const float x = get(from + s * step + d);
      some |= x == -INFINITY || get(from + s * step + d + 1) != 0.f;
      M = fmaxf(M, x);
    }
    for (int s = 0; s < ns; ++s) total = fmaf(get(from + s * step + d + 1), exp2f(get(from + s * step + d) - M), total);
    const float inv = inverse_total(total, some);
    for (int c = lane; c < d; c += 64) {                      // (a piece without weight has sums of zero, or NaN from infinite values)
      float o = 0.f;
      for (int s = 0; s < ns; ++s) o = fmaf(get(from + s * step + c), exp2f(get(from + s * step + d) - M), o);
      Elem<T>::st((T*)a.out + (head0 + h) * d + c, o * inv);
    }
  }
}

template <typename T, int CH>
hipError_t launch(const GkvLaunch& ln, const GkvDims& dm, const PagedAttendArgs& a, bool aligned) {
  const dim3 grid(dm.L * dm.B * dm.Hkv * a.splits);
  const size_t shmem = (size_t)4 * GB * dm.d + NWG * (4 * GB * KEYS + 8 * KEYS + 8 * GB) + (size_t)4 * NWG * GB * dm.d;
  return gkv_launch(ln, aligned ? paged_attend_generic_kernel<T, CH, true> : paged_attend_generic_kernel<T, CH, false>, grid, dim3(NWG * 64),
                    shmem, dm, a);
}

}  // namespace

hipError_t gkv_launch_paged_attend_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PagedAttendArgs& a, bool aligned) {
  if (dtype == GKV_F32) return dm.d <= 64 ? launch<float, 1>(ln, dm, a, aligned) : dm.d <= 128 ? launch<float, 2>(ln, dm, a, aligned) : launch<float, 4>(ln, dm, a, aligned);
  return dm.d <= 128 ? launch<uint16_t, 2>(ln, dm, a, aligned) : dm.d <= 256 ? launch<uint16_t, 4>(ln, dm, a, aligned) : launch<uint16_t, 8>(ln, dm, a, aligned);
}
