// Rotary positions: queries and keys turned by their tokens' positions, on their own or on the way into a paged cache.
//
// Pair p of a head's first `dim` channels, (x1, x2) = channels (p, p + dim/2) or (2p, 2p + 1), becomes
//   m (x1 cos a - x2 sin a, x1 sin a + x2 cos a),  a = position * freq[p]   (transposed: -a, which is the gradient's way back).
// A position of a million at one radian each needs 20 bits before the point, so the angle is formed and reduced to a quarter turn in
// 64 bits; what is left, within +-pi/4, takes a Taylor polynomial in 32 (remainders 2^-29 and 2^-33).  Products and sums are in 32 bits,
// rounded once to the type.
//
// Bound: memory, each element read and written once.  A workgroup has the cosines and sines of its tokens in LDS, made once for all
// heads (an angle is some 40 instructions, a turned pair 6), while its first loads are on their way.  Neighbouring lanes have neighbouring 16
// bytes in every load and store, and stores are non-temporal: 32749 tokens of 40 and 8 heads, three quarters of 128 channels interleaved, 805 MB, 162 us
// with two neighbouring pieces a lane, 142 so, 131 with those stores; appends of 66 MB 14.5 -> 11.8, of 625 MB 113 -> 107 (non-temporal loads as well:
// 10% slower).  Two items a thread at a time where those had four: the smallest calls 3.06 -> 2.82, 805 MB 138 (5.8 TB/s; a copy of 1 GiB makes 5.1), 625 MB 105.
#include "gkv_internal.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int THREADS = 256, AT_ONCE = 2, MOST_TOKENS = 32;   // of a workgroup; items a thread has on their way; tokens of a workgroup

// cos and sin of position * freq, times m.
__device__ __forceinline__ float2 turn(double freq, int position, float m, int transposed) {
  const double a = (double)position * freq;
  double n = rint(a * 0.63661977236758134308);             // quarter turns
  const double r = fma(-n, 6.123233995736766036e-17, fma(-n, 1.57079632679489661923, a));
  n *= 0.25;
  const int quarter = (int)((n - floor(n)) * 4.0);           // exact
  const float x = (float)r, z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
  if (quarter == 1 || quarter == 2) cs = -cs;
  if ((quarter >= 2) != (transposed != 0)) sn = -sn;
  return make_float2(cs * m, sn * m);
}

// E elements side by side as they are in memory, 16 bytes or less, and as floats.
template <int WORDS> struct Words { typedef uint32_t type __attribute__((ext_vector_type(WORDS))); };
template <> struct Words<1> { typedef uint32_t type; };
template <typename T, int E>
struct Piece {
  typedef typename Words<E * (int)sizeof(T) / 4>::type W;
  uint32_t w[E * sizeof(T) / 4];
  __device__ __forceinline__ void load(const T* p) {
    const W x = *(const W*)p;
    __builtin_memcpy(w, &x, sizeof(x));
  }
  __device__ __forceinline__ void store(T* p) const {
    W x;
    __builtin_memcpy(&x, w, sizeof(x));
    __builtin_nontemporal_store(x, (W*)p);
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
  __device__ __forceinline__ void set2(int i, float a, float b) {
    if constexpr (sizeof(T) == 4) { w[i] = __float_as_uint(a); w[i + 1] = __float_as_uint(b); }
    else w[i >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
  }
};
template <typename T> struct Piece<T, 1> {
  T x;
  __device__ __forceinline__ void load(const T* p) { x = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = x; }
  __device__ __forceinline__ float get(int) const { return Elem<T>::ld(&x); }
  __device__ __forceinline__ void set1(float a) { Elem<T>::st(&x, a); }
};

struct Args {
  RotateArgs in;
  const int32_t *start, *len;
  GkvPages pages; void *K, *V;
  int32_t groups, per_group;       // workgroups of a layer, tokens of each
  int32_t look_first;
  GkvDivisor by_groups, by_per_head, by_heads, by_half;
};

// Which sequence token t is of, and its row there; row < 0: of none.  `before`: entries of `start` at or below t.
struct Place { int seq; int64_t row; };
__device__ __forceinline__ Place place_after(int t, int before, const int32_t* start, const int32_t* len, int B) {
  if (before == 0 || before > B) return Place{0, -1};
  return Place{before - 1, (int64_t)len[before - 1] - ((int64_t)start[before] - t)};
}

// An item is two pieces of a row: of its turned channels the two halves of some pairs (half layout), of the others, and in the interleaved layout,
// one of the first half and one of the second, so that lanes have neighbours.
//   Pieces have E elements, 16 bytes where dim/2 (half layout) or dim (interleaved) is a whole number of them, else fewer.
// Dynamic LDS: float2 angles[per_group][dim/2].
template <typename T, int E, bool HALF, bool APPEND>
__global__ __launch_bounds__(THREADS) void rotate_kernel(GkvDims dm, Args a) {
  constexpr bool VECTOR = E > 1;
  using P = Piece<T, E>;
  extern __shared__ float2 angles[];
  __shared__ int64_t row_of[MOST_TOKENS];                     // in the pages of K and V, in rows of d elements; -1: the row is dropped
  __shared__ int present[MOST_TOKENS], position_of[MOST_TOKENS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int layer = quotient(blockIdx.x, a.by_groups), group = (int)blockIdx.x - layer * a.groups;
  const int t0 = group * a.per_group, n = min(a.per_group, a.in.tokens - t0);
  const int d = dm.d, dim = a.in.rotary.dim, half = dim >> 1, in_half = half / E, pieces = d / E;
  const int hq = a.in.q ? dm.Hq : 0, hk = a.in.k ? dm.Hkv : 0, heads = hq + hk * (APPEND ? 2 : 1);
  const int per_head = (pieces + 1) >> 1, items = n * heads * per_head;

  struct Item { int token, slot, i, p0, p1; bool turned0, turned1; };
  auto item = [&](int x) {
    Item it;
    const int row = quotient(x, a.by_per_head);
    it.i = x - row * per_head;
    it.token = quotient(row, a.by_heads);
    it.slot = row - it.token * heads;
    const bool turns = it.slot < hq + hk;                     // (a row of v does not)
    if constexpr (HALF) {
      it.turned0 = it.turned1 = turns && it.i < in_half;
      const int first = turns ? in_half : 0;                 // the others: pieces from 2 first on, those of the first half of them and of the second
      it.p0 = it.turned0 ? it.i : first + it.i;
      it.p1 = it.turned0 ? it.i + in_half : per_head + it.i;
    } else {
      it.p0 = VECTOR ? it.i : 2 * it.i;
      it.p1 = VECTOR ? it.i + per_head : 2 * it.i + 1;
      it.turned0 = turns && it.p0 * E < dim;
      it.turned1 = turns && it.p1 * E < dim;
    }
    return it;
  };
  auto load = [&](const Item& it, P& x0, P& x1) {
    const int64_t at = (int64_t)layer * a.in.tokens + t0 + it.token;
    const T* from;
    if (it.slot < hq) from = (const T*)a.in.q + at * a.in.q_stride + it.slot * d;
    else if (it.slot < hq + hk) from = (const T*)a.in.k + at * a.in.k_stride + (it.slot - hq) * d;
    else from = (const T*)a.in.v + at * a.in.v_stride + (it.slot - hq - hk) * d;
    x0.load(from + it.p0 * E);
    x1.load(from + min(it.p1, pieces - 1) * E);
  };
  auto store = [&](const Item& it, P& x0, P& x1) {
    if (!present[it.token]) return;
    const float2* w = angles + it.token * half;
    if constexpr (HALF || !VECTOR) {
      if (it.turned0) {
        w += it.i * E;
        if constexpr (VECTOR) {
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const float u0 = x0.get(e), u1 = x0.get(e + 1), v0 = x1.get(e), v1 = x1.get(e + 1);
            x0.set2(e, u0 * w[e].x - v0 * w[e].y, u1 * w[e + 1].x - v1 * w[e + 1].y);
            x1.set2(e, u0 * w[e].y + v0 * w[e].x, u1 * w[e + 1].y + v1 * w[e + 1].x);
          }
        } else {
          const float u = x0.get(0), v = x1.get(0);
          x0.set1(u * w->x - v * w->y);
          x1.set1(u * w->y + v * w->x);
        }
      }
    } else {
      auto pairs = [&](P& x, int p) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 cs = w[(p * E + e) >> 1];
          const float u = x.get(e), v = x.get(e + 1);
          x.set2(e, u * cs.x - v * cs.y, u * cs.y + v * cs.x);
        }
      };
      if (it.turned0) pairs(x0, it.p0);
      if (it.turned1) pairs(x1, it.p1);
    }
    T* to;
    const int64_t at = (int64_t)layer * a.in.tokens + t0 + it.token;
    if (it.slot < hq) to = (T*)a.in.q_out + (at * dm.Hq + it.slot) * d;
    else if constexpr (APPEND) {
      if (row_of[it.token] < 0) return;
      const int h = it.slot - hq;
      to = (T*)(h < hk ? a.K : a.V) + (row_of[it.token] + (int64_t)(h < hk ? h : h - hk) * a.pages.page_rows) * d;
    } else to = (T*)a.in.k_out + (at * dm.Hkv + it.slot - hq) * d;
    x0.store(to + it.p0 * E);
    if (it.p1 < pieces) x1.store(to + it.p1 * E);
  };

  // the first items' pieces are on their way while the angles are made
  Item it[AT_ONCE];
  P x0[AT_ONCE], x1[AT_ONCE];
  auto load_all = [&](int first) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      it[u] = item(min(first + u * THREADS, items - 1));
      load(it[u], x0[u], x1[u]);
    }
  };
  // (of many tokens some workgroups may have nothing but padding, which costs less than a trip to memory ahead of the loads)
  if (APPEND && a.look_first && t0 >= a.start[dm.B]) return;
  load_all(tid);
  auto note = [&](int k, const Place& place) {
    const int t = t0 + k;
    int64_t at = -1;
    if (place.row >= 0 && place.row < (int64_t)a.pages.width * a.pages.page_rows) {
      const int page = quotient((int)place.row, a.pages.by_rows);
      const int32_t id = a.pages.table[(int64_t)place.seq * a.pages.width + page];
      if (id >= 0 && id < a.pages.n_pages)
        at = ((int64_t)layer * a.pages.n_pages + id) * dm.Hkv * a.pages.page_rows + ((int)place.row - page * a.pages.page_rows);
    }
    row_of[k] = at;
    present[k] = place.row >= 0;
    position_of[k] = a.in.positions ? a.in.positions[t] : (int)place.row;
  };
  if constexpr (!APPEND) {
    if (tid < n) {
      present[tid] = 1;
      position_of[tid] = a.in.positions ? a.in.positions[t0 + tid] : resolve_step(dm, a.in.step);
    }
  } else if (!a.start) {
    if (tid < n) note(tid, Place{t0 + tid, (int64_t)a.len[t0 + tid] - 1});
  } else if (a.per_group <= THREADS / 64) {
    // a wavefront a token, which looks through `start` 64 entries at a time
    if (wave < n) {
      const int t = t0 + wave;
      int before = 0;
      for (int i = lane; i - lane <= dm.B; i += 64) before += __popcll(__ballot(i <= dm.B && a.start[min(i, dm.B)] <= t));
      const Place place = place_after(t, before, a.start, a.len, dm.B);
      if (lane == 0) note(wave, place);
    }
  } else if (tid < n) {
    // a lane a token, by halves
    const int t = t0 + tid;
    int before = 0;                                          // entries below it are at or below t, from `end` on above
    for (int end = dm.B + 1; before < end;) {
      const int mid = (before + end) >> 1;
      if (a.start[mid] <= t) before = mid + 1;
      else end = mid;
    }
    note(tid, place_after(t, before, a.start, a.len, dm.B));
  }
  __syncthreads();
  for (int x = tid; x < n * half; x += THREADS) {
    const int k = quotient(x, a.by_half), p = x - k * half;
    angles[x] = turn(a.in.rotary.freq[p], position_of[k], a.in.rotary.amplitude, a.in.rotary.transposed);
  }
  __syncthreads();
  for (int x = tid;;) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
      if (x + u * THREADS < items) store(it[u], x0[u], x1[u]);
    x += AT_ONCE * THREADS;
    if (x >= items) break;
    load_all(x);
  }
}

__global__ void advance_kernel(int32_t* len, const int32_t* start, int B) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= B) return;
  const int now = len[i];
  const int more = start ? start[i + 1] - start[i] : now >= 0 ? 1 : 0;
  if (more > 0) len[i] = max(now, 0) + more;
}

template <typename T, bool APPEND>
hipError_t launch(const GkvLaunch& ln, const GkvDims& dm, Args a) {
  if (a.in.tokens == 0) return hipSuccess;
  const GkvRotary& r = a.in.rotary;
  const bool is_half = r.layout == GKV_ROTARY_HALF;
  // Bytes of a piece: whole numbers of them in everything
  const uintptr_t bits = (uintptr_t)a.in.q | (uintptr_t)a.in.k | (uintptr_t)a.in.v | (uintptr_t)a.in.q_out | (uintptr_t)a.in.k_out |
                         (uintptr_t)a.K | (uintptr_t)a.V | 16 |
                         (uintptr_t)((a.in.q_stride | a.in.k_stride | a.in.v_stride | dm.d | (is_half ? r.dim / 2 : r.dim)) * (int64_t)sizeof(T));
  const int E = (int)((bits & (~bits + 1)) / sizeof(T));
  const int pieces = dm.d / E, per_head = (pieces + 1) / 2;
  const int heads = (a.in.q ? dm.Hq : 0) + (a.in.k ? dm.Hkv : 0) * (APPEND ? 2 : 1);
  const int64_t rows = (int64_t)dm.L * a.in.tokens;
  // Tokens of a workgroup: 512 items, two for each thread, where that leaves a workgroup for every CU.  us, by tokens (items of one): 32749 tokens of 40
  // and 8 heads (384) 1 / 2 / 4 131 / 139 / 146; 2048 appended of 28, 4 and 4 (288) 7.7 / 6.6 / 7.4; 64 in 36 layers of 40, 8 and 8 (448) 11.8 / 11.2 / 12.1;
  // fp32, 8168 in 4 layers of 2 and 2, d = 64 (32) 4 / 8 / 16 / 32 18.8 / 14.0 / 13.0 / 13.1; 8 in 28 layers of 28 and 4 (256) 1 / 2 / 4 3.7 / 4.0 / 4.7.
  const int64_t of_one = (int64_t)heads * per_head, wanted = (512 + of_one / 2) / of_one, most = rows / 256;
  a.per_group = (int)(wanted > most ? most : wanted);
  if (a.per_group < 1) a.per_group = 1;
  if (a.per_group > MOST_TOKENS) a.per_group = MOST_TOKENS;
  a.groups = (a.in.tokens + a.per_group - 1) / a.per_group;
  a.by_groups = gkv_divisor(a.groups);
  a.by_per_head = gkv_divisor(per_head);
  a.by_heads = gkv_divisor(heads);
  a.by_half = gkv_divisor(r.dim > 0 ? r.dim / 2 : 1);
  const size_t shmem = sizeof(float2) * a.per_group * (r.dim / 2);
  a.look_first = a.start && a.in.tokens > 256;
  void (*kern)(GkvDims, Args);
  if constexpr (sizeof(T) == 2) {
    if (E == 8) kern = is_half ? rotate_kernel<T, 8, true, APPEND> : rotate_kernel<T, 8, false, APPEND>;
  }
  if (E == 4) kern = is_half ? rotate_kernel<T, 4, true, APPEND> : rotate_kernel<T, 4, false, APPEND>;
  else if (E == 2) kern = is_half ? rotate_kernel<T, 2, true, APPEND> : rotate_kernel<T, 2, false, APPEND>;
  else if (E < 2) kern = is_half ? rotate_kernel<T, 1, true, APPEND> : rotate_kernel<T, 1, false, APPEND>;
  return gkv_launch(ln, kern, dim3(dm.L * a.groups), dim3(THREADS), shmem, dm, a);
}

}  // namespace

hipError_t gkv_launch_rotate(const GkvLaunch& ln, const GkvDims& dm, int dtype, const RotateArgs& in) {
  Args a{};
  a.in = in;
  return dtype == GKV_F32 ? launch<float, false>(ln, dm, a) : launch<uint16_t, false>(ln, dm, a);
}

hipError_t gkv_launch_paged_append(const GkvLaunch& ln, const GkvDims& dm, int dtype, const AppendArgs& in) {
  Args a{};
  a.in = in.in;
  a.start = in.start; a.len = in.len; a.pages = in.pages; a.K = in.K; a.V = in.V;
  return dtype == GKV_F32 ? launch<float, true>(ln, dm, a) : launch<uint16_t, true>(ln, dm, a);
}

hipError_t gkv_launch_paged_advance(const GkvLaunch& ln, const GkvDims& dm, int32_t* len, const int32_t* start) {
  return gkv_launch(ln, advance_kernel, dim3((dm.B + 255) / 256), dim3(256), 0, len, start, (int)dm.B);
}
