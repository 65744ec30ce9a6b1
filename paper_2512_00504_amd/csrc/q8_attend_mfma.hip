// Decode attention over a cache in 8 bits on the matrix cores: head_dim 64 or 128, group size g <= 16, queries in bf16 or fp32.
//
// One workgroup of NW wavefronts per (unit, piece).  A wavefront owns slices of 32 keys and keeps running maxima, sums and accumulators
// of all g query heads, so every code is read once per KV head.
//   A row is its codes c_n times 2^e_n, so  q . k_n = 2^ek_n (q . c_n)  and  sum p_n v_n = sum (p_n 2^ev_n) c_n:  the scales
//   meet the logits and the probabilities, one multiplication per (head, key) each, and never the elements.  A code has 4
//   significant bits and is exact as a bf16 number, so the products are those of the bf16 matrix cores, 16x16x32.
// Per slice and wavefront (16-key tiles; r = lane % 16, kb = lane / 16):
//   K: a lane's 16-byte load holds 16 channels of key r, two operands' worth after the conversion.  S^T[key, head] = K Q^T; the
//      result lane (head r, block kb) holds keys 4 kb + e of its head per tile, whose scales are 16 bytes of `scales`.
//   V: a lane loads D/16 channels of keys 4 kb + e (a quarter-wave reads a row).  O^T[channel, head] += V^T P^T wants two
//      keys' codes of one channel side by side: one byte permutation for two channels, then the conversion.
//   fp32 queries and their probabilities enter as the sum of three bf16 numbers, which hold all of their 24 bits.  bf16's
//   probabilities are rounded to bf16 under the running maximum: 4e-4 of the result beside the 1.7e-3 of its own rounding (as two
//   numbers: 16 steps and the score of 896 units 469 -> 457 us without the second).
// Bound: HBM in launches of some hundred units and more (18432 units of 1056 rows 850 us, 6.05 TB/s); a slice is about 170 vector
// instructions and 16 matrix instructions (16 cycles each), a fifth of the time its bytes take at the memory's rate.  Below, the chain of
// trips to memory and instructions: us in a graph, this / the kernel of bf16 or fp32 caches, 4 units of 577 rows 6.4 / 5.6, 128 of 577 7.5 / 8.6, 128
// of 1100 10.2 / 13.8, 512 of 577 16.0 / 25.1; fp32, D = 64 2 of 72 4.7 / 4.2.  One slice in flight, K of the next asked for as soon as the
// products with this one are under way (behind them: 861 / 854 us for 18432 units; two slices: 891, 4 of 577 7.0); 4 wavefronts (6: 935, 8: 915);
// slices of 64 keys at D = 64: 2 of 72 6.25, 128 of 528 8.05 -> 6.3, 3584 of 600 56.6 -> 49.5.
// The newest token's row is quantised by every wavefront for itself while its first slice is on the way (a step's call is
// one launch), and replaces what the cache holds in its place in the unit's last slice; the workgroup of the first piece stores it.
#include "e4m3.h"

#include <type_traits>

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u32x4 ld16(const void* p) { return *(const u32x4*)p; }
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
// Two codes of a word's lower or upper half as bf16 numbers, times a power of two.
__device__ __forceinline__ uint32_t lower(uint32_t w, float times = 1.0f) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, times, false));
}
__device__ __forceinline__ uint32_t upper(uint32_t w, float times = 1.0f) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, times, true));
}
__device__ __forceinline__ u32x4 eight_of_k(uint32_t a, uint32_t b) {
  return u32x4{lower(a, Q8_K_SHRUNK), upper(a, Q8_K_SHRUNK), lower(b, Q8_K_SHRUNK), upper(b, Q8_K_SHRUNK)};
}

// x as bf16 (P = 1), or as the sum of P bf16 numbers: three hold all of its bits.
template <int P>
__device__ __forceinline__ void parts_of(const f32x8& x, u32x4 (&p)[P]) {
  f32x8 rest = x;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const bf16x8 h = __builtin_convertvector(rest, bf16x8);
    p[i] = __builtin_bit_cast(u32x4, h);
    if (i < P - 1) rest -= __builtin_convertvector(h, f32x8);
  }
}

template <typename T, int D>
struct Geo {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int KEYS = 32, KT = 2;                    // of a slice, tiles of 16
  static constexpr int NL = D / 64;                          // K loads per tile
  static constexpr int NC = D / 16;                          // channels per lane, accumulators
  static constexpr int VW = D / 64;                          // words of V per lane and key
  static constexpr int QP = F32 ? 3 : 1;                     // bf16 parts of a query
  static constexpr int PP = F32 ? 3 : 1;                     // of a probability
  static constexpr int ROW_BYTES = D * (int)sizeof(T);       // of q, out and the new rows
  static constexpr int OSTR = D + 4, PSTR = D + 2;           // LDS rows of partial outputs; pieces in memory: o[D], m, l
};

template <int VW> struct VCodes { uint32_t w[VW]; };
template <typename T, int D>
struct Slice {
  u32x4 k[Geo<T, D>::KT][Geo<T, D>::NL];
  VCodes<Geo<T, D>::VW> v[4 * Geo<T, D>::KT];
  u32x4 scale[Geo<T, D>::KT];                                // words of keys 4 kb .. 4 kb + 3
};

// Where a wavefront's loads go: the unit's rows (uniform) and this lane's offsets.
template <typename T, int D>
struct Rows {
  const uint8_t *K, *V;
  const uint32_t* scales;
  int n_tiled;
  uint32_t k_tiled, k_rows, v, s;
};

template <typename T, int D>
__device__ __forceinline__ void request_k(Slice<T, D>& x, const Rows<T, D>& at, int it) {
  using G = Geo<T, D>;
#pragma unroll
  for (int tt = 0; tt < G::KT; ++tt) {
    const int t = it * G::KT + tt;                           // (the capacity is whole slices)
    const bool tiled = 16 * t < at.n_tiled;                  // uniform
    const uint8_t* p = at.K + (uint32_t)(t * 16 * D) + (tiled ? at.k_tiled : at.k_rows);
    const uint32_t step = tiled ? 1024 : 64;
#pragma unroll
    for (int c = 0; c < G::NL; ++c) x.k[tt][c] = ld16(p + c * step);
  }
}
template <typename T, int D, bool ONCE>
__device__ __forceinline__ void request_v(Slice<T, D>& x, const Rows<T, D>& at, int it) {
  using G = Geo<T, D>;
#pragma unroll
  for (int tt = 0; tt < G::KT; ++tt) {
    const int t = it * G::KT + tt;
    x.scale[tt] = ld16((const char*)at.scales + (uint32_t)(t * 64) + at.s);
    const uint8_t* p = at.V + (uint32_t)(t * 16 * D) + at.v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (G::VW == 2) {
        const u32x2 a = ONCE ? __builtin_nontemporal_load((const u32x2*)(p + e * D)) : *(const u32x2*)(p + e * D);
        x.v[4 * tt + e].w[0] = a[0]; x.v[4 * tt + e].w[1] = a[1];
      } else {
        x.v[4 * tt + e].w[0] = ONCE ? __builtin_nontemporal_load((const uint32_t*)(p + e * D)) : *(const uint32_t*)(p + e * D);
      }
    }
  }
}

template <typename T, int D, bool ONCE>
__device__ __forceinline__ void request(Slice<T, D>& x, const Rows<T, D>& at, int it) {
  request_k<T, D>(x, at, it);
  request_v<T, D, ONCE>(x, at, it);
}
struct Nothing { __device__ void operator()() const {} };

template <int NC>
struct Running {
  float m, l;                                                // maximum (log2 units) shared by a head's 4 lanes, own part of the sum
  f32x4 o[NC];                                               // o[m][e]: channel m of lane 4 kb + e
};

// Over the four lanes of a head.
__device__ __forceinline__ float over_head(float x, bool max) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t u = __float_as_uint(x);
    const u32x2 y = i == 0 ? __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false))
                           : __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(u, u, false, false));
    const float a = __uint_as_float(y[0]), b = __uint_as_float(y[1]);
    x = max ? fmaxf(a, b) : a + b;
  }
  return x;
}

// The newest token's row as this wavefront holds it: codes in LDS, its scales, and its index (-1: none).
struct NewRow { const uint8_t *k, *v; uint32_t word; int row; };

// edge: the slice holds the unit's end: rows behind it are zeros of scale zero, masked, and the new row is taken from its place in
// LDS.  EXACT: right for every logit (see log2_weight); without it a logit of -inf may give NaN and a huge maximum any
// weight, which shows at the end.
// between: what to do once the products with K are under way, whose registers are free then.
template <typename T, int D, bool EXACT, typename Between>
__device__ __forceinline__ void process(Slice<T, D>& x, Running<D / 16>& st, const u32x4 (&q)[Geo<T, D>::NL][2][Geo<T, D>::QP], int it,
                                        bool edge, float hi, float lo, int r, int kb, int n_tot, const NewRow& fresh, Between between) {
  using G = Geo<T, D>;
  constexpr int NS = 4 * G::KT;
  const int key0 = it * G::KEYS;
  if (edge) {
#pragma unroll
    for (int tt = 0; tt < G::KT; ++tt) {
      const int key = key0 + 16 * tt + r;
#pragma unroll
      for (int c = 0; c < G::NL; ++c) {
        if (key == fresh.row) x.k[tt][c] = ld16(fresh.k + (4 * c + kb) * 16);
        if (key >= n_tot) x.k[tt][c] = u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int vkey = key0 + 16 * tt + 4 * kb + e;
        VCodes<G::VW>& v = x.v[4 * tt + e];
        if (vkey == fresh.row) {
          x.scale[tt][e] = fresh.word;
#pragma unroll
          for (int i = 0; i < G::VW; ++i) v.w[i] = *(const uint32_t*)(fresh.v + r * G::NC + 4 * i);
        }
        if (vkey >= n_tot) {
          x.scale[tt][e] = 0u;
#pragma unroll
          for (int i = 0; i < G::VW; ++i) v.w[i] = 0u;
        }
      }
    }
  }
  float z[NS];
  f32x4 acc[G::KT];
#pragma unroll
  for (int tt = 0; tt < G::KT; ++tt) {
    acc[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < G::NL; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8 a = as_bf16x8(eight_of_k(x.k[tt][c][2 * h], x.k[tt][c][2 * h + 1]));
#pragma unroll
        for (int p = 0; p < G::QP; ++p) acc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, as_bf16x8(q[c][h][p]), acc[tt], 0, 0, 0);
      }
  }
  if constexpr (!std::is_same_v<Between, Nothing>) {
    __builtin_amdgcn_sched_barrier(0);
    between();
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int tt = 0; tt < G::KT; ++tt) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[4 * tt + e] = acc[tt][e] * q8_k_scale(x.scale[tt][e]);
      if (edge && key0 + 16 * tt + 4 * kb + e >= n_tot) z[4 * tt + e] = EXACT ? -INFINITY : -1e30f;
    }
  }
  float mx = z[0];
#pragma unroll
  for (int i = 1; i < NS; ++i) mx = fmaxf(mx, z[i]);
  mx = over_head(mx, true);
  // (Letting m lag behind by up to 8, so that accumulators are seldom rescaled: 443 us where this takes 447, 16 steps of 896 units, but
  // a weight that dominates is 1 here and exact in bf16, there it is not: error 2.0e-3 against 1.7e-3.)
  const float m_new = fmaxf(st.m, rounded_product(mx, hi));
  if (__any(m_new > st.m)) {
    const float f = __builtin_amdgcn_exp2f(st.m - m_new);
    st.l *= f;
#pragma unroll
    for (int m = 0; m < G::NC; ++m) st.o[m] *= f;
    st.m = m_new;
  }
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    z[i] = __builtin_amdgcn_exp2f(EXACT ? log2_weight(z[i], hi, lo, st.m) : fmaf(z[i], lo, fmaf(z[i], hi, -st.m)));
    sum += z[i];
  }
  st.l += sum;
#pragma unroll
  for (int x2 = 0; x2 < G::KT / 2; ++x2) {                   // 32 keys: tiles 2 x2 and 2 x2 + 1
    f32x8 pv;
#pragma unroll
    for (int i = 0; i < 8; ++i) pv[i] = z[8 * x2 + i] * q8_v_scale(x.scale[2 * x2 + (i >> 2)][i & 3]);
    u32x4 p[G::PP];
    parts_of(pv, p);
#pragma unroll
    for (int w = 0; w < G::VW; ++w) {
      // a word holds 4 channels of a key; channels 2 c2 and 2 c2 + 1 of two keys make a word of pairs
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
        u32x4 a, b;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const uint32_t pair = __builtin_amdgcn_perm(x.v[8 * x2 + 2 * y + 1].w[w], x.v[8 * x2 + 2 * y].w[w], c2 ? 0x07030602u : 0x05010400u);
          a[y] = lower(pair);
          b[y] = upper(pair);
        }
        const int m = 4 * w + 2 * c2;
#pragma unroll
        for (int i = 0; i < G::PP; ++i) {
          st.o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(p[i]), st.o[m], 0, 0, 0);
          st.o[m + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(b), as_bf16x8(p[i]), st.o[m + 1], 0, 0, 0);
        }
      }
    }
  }
}

__device__ __forceinline__ void store_row4(float* p, const f32x4& o) { *(f32x4*)p = o; }
__device__ __forceinline__ void store_row4(uint16_t* p, const f32x4& o) {
  u32x2 packed;
  packed[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[0], o[1]}), bf16x2));
  packed[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[2], o[3]}), bf16x2));
  *(u32x2*)p = packed;
}
// Two neighbouring floats to and from memory that workgroups on other XCDs share.
__device__ __forceinline__ void store_agent(float* p, float x, float y) {
  const uint64_t v = ((uint64_t)__float_as_uint(y) << 32) | __float_as_uint(x);
  __hip_atomic_store((uint64_t*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_agent(const float* p) {
  const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

struct KernelArgs {
  const int32_t* d_state; const int32_t* step_base;        // step_base: d_state where there is none, and not used
  const char *q, *k_new, *v_new;
  uint8_t *K, *V; uint32_t* scales; int32_t* pos; char *qwin, *out;
  float2* stats; float* partials; int32_t* ticket;
  GkvDivisor by_splits, by_hkv, by_iters, by_w;
  int32_t splits, split_iters, Hq, Hkv, g, cap, LB, w, step;
  int32_t has_base, copy_q, write_stats;
  float scale_hi, scale_lo;                                // (with Q8_K_GROWN)
  PrefixPart prefix;
};

// Four elements of the newest token's row.
template <typename T>
__device__ __forceinline__ void load4(const char* p, float (&x)[4]) {
  if constexpr (sizeof(T) == 4) {
    const u32x4 a = ld16(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(a[i]);
  } else {
    const u32x2 a = *(const u32x2*)p;
#pragma unroll
    for (int i = 0; i < 2; ++i) { x[2 * i] = __uint_as_float(a[i] << 16); x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
  }
}

// Dynamic LDS: float so[NW][g][OSTR], sm[16][NW], sl[16][NW]; the new row's codes, K then V, per wavefront.
template <typename T, int D, int NW, int OCC, bool ONCE>
__global__ __launch_bounds__(NW * 64, OCC) void q8_attend_mfma_kernel(KernelArgs a) {
  using G = Geo<T, D>;
  constexpr int ROW_BYTES = G::ROW_BYTES, OSTR = G::OSTR, PSTR = G::PSTR;
  extern __shared__ __attribute__((aligned(16))) float smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, kb = lane >> 4;
  const int splits = a.splits, g = a.g, cap = a.cap;
  const int unit = quotient(blockIdx.x, a.by_splits), sp = (int)blockIdx.x - unit * splits;
  const int lb = quotient(unit, a.by_hkv), j = unit - lb * a.Hkv;
  const size_t head0 = (size_t)lb * a.Hq + j * g;
  const char* q_g = a.q + head0 * ROW_BYTES;
  const bool may_grow = a.k_new != nullptr;

  // requested at once: the record, the step counter, the group's queries, the new row
  int4 rec = *(const int4*)(a.d_state + 4 * (size_t)lb);
  const int32_t base = *a.step_base;
  const int32_t prefix_n = *(a.prefix.o ? a.prefix.n + head0 : a.d_state);   // pieces of the prefix, the same for all heads of a sequence
  u32x4 qraw[G::NL][2][G::F32 ? 2 : 1];
#pragma unroll
  for (int c = 0; c < G::NL; ++c)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < (G::F32 ? 2 : 1); ++i)             // channels 16 (4 c + kb) + 8 h .. + 7 (lanes beyond the group repeat its last head)
        qraw[c][h][i] = ld16(q_g + min(r, g - 1) * ROW_BYTES + (16 * (4 * c + kb) + 8 * h) * sizeof(T) + 16 * i);
  float fresh4[4];
  const int nr = lane & 31, which = lane >> 5;               // lanes 0 .. 31: K, the others V; four channels each
  load4<T>((may_grow ? (which ? a.v_new : a.k_new) + (size_t)unit * ROW_BYTES : q_g) + min(nr, D / 4 - 1) * 4 * sizeof(T), fresh4);
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" : "+s"(rec.x), "+s"(rec.y), "+s"(rec.w));
  const int n_pre = a.prefix.o ? prefix_n : 0;

  const SeqState seq = state_record(rec);
  const int step = a.step + (a.has_base ? base : 0);
  const int len0 = length_before_step(seq, step, cap);
  const bool has_new = may_grow && len0 < cap;
  const int n_tot = len0 + (has_new ? 1 : 0);
  const int n_iter = (int)((uint32_t)(n_tot + G::KEYS - 1) / G::KEYS);
  int ns = splits;
  if (splits > 1 && a.split_iters > 0) {
    ns = max(1, min(splits, quotient(n_iter + a.split_iters - 1, a.by_iters)));
    if (sp >= ns) return;
  }
  const int stride = ns * NW, it0 = sp * NW + wave;
  Rows<T, D> at;
  at.K = a.K + (size_t)unit * cap * D; at.V = a.V + (size_t)unit * cap * D; at.scales = a.scales + (size_t)unit * cap;
  at.n_tiled = seq.n_tiled;
  at.k_tiled = lane * 16; at.k_rows = r * D + kb * 16; at.v = kb * 4 * D + r * G::NC; at.s = kb * 16;

  Slice<T, D> s;
  request<T, D, ONCE>(s, at, min(it0, max(n_iter - 1, 0)));  // (wavefronts beyond the end ask for its last slice and do not use it)

  // while that is on its way: the queries' parts, and the new row's codes
  u32x4 q[G::NL][2][G::QP];
#pragma unroll
  for (int c = 0; c < G::NL; ++c)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (G::F32) {
        f32x8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(qraw[c][h][i >> 2][i & 3]);
        parts_of(y, q[c][h]);
      } else {
        q[c][h][0] = qraw[c][h][0];
      }
    }
  uint8_t* codes = (uint8_t*)(smem + NW * g * OSTR + 2 * NW * 16) + wave * 2 * D;
  NewRow fresh{codes, codes + D, 0u, has_new ? len0 : -1};
  uint32_t my_codes = 0u;
  if (may_grow) {                                            // uniform
    float top = fmaxf(fmaxf(q8_finite_magnitude(fresh4[0]), q8_finite_magnitude(fresh4[1])),
                      fmaxf(q8_finite_magnitude(fresh4[2]), q8_finite_magnitude(fresh4[3])));
    top = q8_group_max<5>(top);                              // (lanes beyond the row repeat its end)
    const uint32_t field = q8_scale_field(top);
    my_codes = q8_codes(fresh4[0], fresh4[1], fresh4[2], fresh4[3], q8_inverse(field));
    if (nr < D / 4) *(uint32_t*)(codes + which * D + nr * 4) = my_codes;
    fresh.word = q8_scale_word(__builtin_amdgcn_readlane(field, 0), __builtin_amdgcn_readlane(field, 32));
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }

  Running<G::NC> st;
  auto reset = [&]() {
    st.m = GKV_NO_MAX;
    st.l = 0.f;
#pragma unroll
    for (int m = 0; m < G::NC; ++m) st.o[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  reset();
  auto work = [&](Slice<T, D>& x, int it, auto exact) {
    process<T, D, decltype(exact)::value>(x, st, q, it, it == n_iter - 1, a.scale_hi, a.scale_lo, r, kb, n_tot, fresh, Nothing{});
  };
  if (it0 < n_iter) {
    int it = it0;
    for (; it + stride < n_iter; it += stride) {
      process<T, D, false>(s, st, q, it, false, a.scale_hi, a.scale_lo, r, kb, n_tot, fresh, [&] { request_k<T, D>(s, at, it + stride); });
      request_v<T, D, ONCE>(s, at, it + stride);
    }
    work(s, it, std::false_type{});
    // seldom: a maximum that the short form of the weights is not right for, or a NaN that may be its doing
    if (__any(fabsf(st.m) >= GKV_HUGE_LOG2 || st.l != st.l)) {
      reset();
      for (int it = it0; it < n_iter; it += stride) {
        request<T, D, ONCE>(s, at, it);
        work(s, it, std::true_type{});
      }
    }
  }

  // ---- the wavefronts of this workgroup ---------------------------------------------------------
  float* so = smem;
  float* sm = so + NW * g * OSTR;
  float* sl = sm + NW * 16;
  const float l_tot = over_head(st.l, false);
  if (r < g) {
    float* row = so + (wave * g + r) * OSTR;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int q4 = 0; q4 < G::NC / 4; ++q4)
        *(f32x4*)(row + G::NC * (4 * kb + e) + 4 * q4) = f32x4{st.o[4 * q4][e], st.o[4 * q4 + 1][e], st.o[4 * q4 + 2][e], st.o[4 * q4 + 3][e]};
    if (kb == 0) { sm[r * NW + wave] = st.m; sl[r * NW + wave] = l_tot; }
  }

  constexpr int TPH = D / 4;                                 // threads per head
  T* out = (T*)a.out + head0 * D;
  float* part = a.partials + (size_t)(unit * splits) * g * PSTR;
  const int slot = step - quotient(step, a.by_w) * a.w;
  float2* stats = a.stats + (size_t)slot * a.LB * a.Hq + head0;
  PrefixPieces<GKV_PREFIX_AT_ONCE> pre;
  // the unit's result; ready: the first pieces of the prefix are in `pre`
  auto finish = [&](int x, int h, int c4, float M, float L, f32x4 o, bool ready) {
    if (c4 == 0 && a.write_stats) stats[h] = make_float2(M, L);
    const float inv = prefix_join(a.prefix, head0, h, D, c4, n_pre, ready, pre, M, L, o, n_tot > 0);
    store_row4(out + (uint32_t)(x * 4), o * inv);
  };
  __syncthreads();
  for (int x = tid; x < g * TPH; x += NW * 64) {
    const int h = x / TPH, c4 = (x % TPH) * 4;
    float mw[NW], M = GKV_NO_MAX;
#pragma unroll
    for (int i = 0; i < NW; ++i) { mw[i] = sm[h * NW + i]; M = fmaxf(M, mw[i]); }
    float L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float f = __builtin_amdgcn_exp2f(mw[i] - M);
      L += sl[h * NW + i] * f;
      o += *(const f32x4*)(so + (i * g + h) * OSTR + c4) * f;
    }
    if (ns == 1) {
      finish(x, h, c4, M, L, o, false);
    } else {
      float* ph = part + (uint32_t)((sp * g + h) * PSTR);
      store_agent(ph + c4, o[0], o[1]);
      store_agent(ph + c4 + 2, o[2], o[3]);
      if (c4 == 0) store_agent(ph + D, M, L);
    }
  }

  // ---- pieces: whoever finishes last joins them.  A wavefront's outputs need the same heads of the other pieces only, so
  //      each has a ticket of its own; what it stored is waited for first, and passes the XCDs' L2s by.
  const bool joins = ns > 1 && wave * 64 < g * TPH;          // uniform
  uint32_t arrived = 0;
  if (joins) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (lane == 0) arrived = __builtin_amdgcn_atomic_inc32((uint32_t*)a.ticket + (size_t)unit * GKV_TICKETS + wave, (uint32_t)ns - 1u, __ATOMIC_RELAXED, "agent");
  }

  // (the prefix's first pieces, on their way while the ticket is)
  if (joins && n_pre > 0 && tid < g * TPH) pre.request(a.prefix, head0, tid / TPH, D, (tid % TPH) * 4, 0, n_pre);

  // ---- the new row, its scales and position, and q into the ring -----------------------------------
  if (sp == 0) {
    if (has_new && wave == 0) {
      const size_t row = (size_t)unit * cap + len0;
      if (nr < D / 4) *(uint32_t*)((which ? a.V : a.K) + row * D + nr * 4) = my_codes;
      if (lane == 0) { a.scales[row] = fresh.word; a.pos[row] = step; }
    }
    if (a.copy_q) {
      char* ring = a.qwin + ((size_t)slot * a.LB * a.Hq + head0) * ROW_BYTES;
      for (int x = tid; x < ROW_BYTES / 16 * g; x += NW * 64) *(u32x4*)(ring + (uint32_t)(x * 16)) = ld16(q_g + (uint32_t)(x * 16));
    }
  }

  if (joins && (int)__builtin_amdgcn_readfirstlane(arrived) == ns - 1) {
    asm volatile("" ::: "memory");
    for (int x = tid; x < g * TPH; x += NW * 64) {
      const int h = x / TPH, c4 = (x % TPH) * 4;
      float M = GKV_NO_MAX, L = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      constexpr int AT_ONCE = 8;
      for (int s0 = 0; s0 < ns; s0 += AT_ONCE) {
        float2 got[AT_ONCE][3];
        const float* ph = part + (uint32_t)((s0 * g + h) * PSTR);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
          if (s0 + i < ns) {                                 // uniform, here and below
            got[i][0] = load_agent(ph + D); got[i][1] = load_agent(ph + c4); got[i][2] = load_agent(ph + c4 + 2);
            ph += (uint32_t)(g * PSTR);
          }
        float Mn = M;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
          if (s0 + i < ns) Mn = fmaxf(Mn, got[i][0].x);
        const float f0 = __builtin_amdgcn_exp2f(M - Mn);
        M = Mn;
        L *= f0;
        o *= f0;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
          if (s0 + i < ns) {
            const float f = __builtin_amdgcn_exp2f(got[i][0].x - Mn);
            L += got[i][0].y * f;
            o += f32x4{got[i][1].x, got[i][1].y, got[i][2].x, got[i][2].y} * f;
          }
      }
      finish(x, h, c4, M, L, o, x == tid);
    }
  }
}

template <typename T, int D, int NW, int OCC, bool ONCE = false>
hipError_t launch(const GkvLaunch& ln, const GkvDims& dm, const Q8AttendArgs& a) {
  KernelArgs k;
  k.d_state = a.d_state; k.step_base = dm.step_base ? dm.step_base : a.d_state;
  k.q = (const char*)a.q; k.k_new = (const char*)a.k_new; k.v_new = (const char*)a.v_new;
  k.K = a.K8; k.V = a.V8; k.scales = a.scales; k.pos = a.pos; k.qwin = (char*)a.qwin; k.out = (char*)a.out;
  k.stats = a.ws.stats; k.partials = a.ws.partials; k.ticket = a.ws.split_ticket;
  k.by_splits = gkv_divisor(a.splits); k.by_hkv = dm.by_hkv; k.by_w = gkv_divisor(dm.w);
  k.by_iters = gkv_divisor(a.split_iters > 0 ? a.split_iters : 1);
  k.splits = a.splits; k.split_iters = a.split_iters;
  k.Hq = dm.Hq; k.Hkv = dm.Hkv; k.g = dm.g; k.cap = dm.cap; k.LB = dm.L * dm.B; k.w = dm.w; k.step = a.step;
  k.has_base = dm.step_base != nullptr; k.copy_q = a.copy_q; k.write_stats = a.write_stats;
  k.scale_hi = dm.scale_l2_hi * Q8_K_GROWN; k.scale_lo = dm.scale_l2_lo * Q8_K_GROWN; k.prefix = a.prefix;
  return gkv_launch(ln, q8_attend_mfma_kernel<T, D, NW, OCC, ONCE>, dim3(dm.L * dm.B * dm.Hkv * a.splits), dim3(NW * 64),
                    gkv_q8_attend_mfma_lds(D, dm.g, NW), k);
}

template <typename T, int D>
hipError_t launch_waves(const GkvLaunch& ln, const GkvDims& dm, const Q8AttendArgs& a) {
  if (a.waves == 8) return launch<T, D, 8, 2>(ln, dm, a);
  // V of caches beyond the 256 MiB memory-side cache is read with non-temporal loads beside K's ordinary ones (18432 units of 1056 rows: both
  // ordinary 939 us, this 861; 896 of 640, which that cache holds: both ordinary 462 for 16 steps and the score, this 473)
  constexpr int OCC = sizeof(T) == 4 ? 2 : 3;                // wavefronts per SIMD that the registers leave room for
  const bool once = (int64_t)dm.L * dm.B * dm.Hkv * (dm.b + dm.s / 2) * 2 * D > (int64_t)256 << 20;
  return once ? launch<T, D, 4, OCC, true>(ln, dm, a) : launch<T, D, 4, OCC>(ln, dm, a);
}

}  // namespace

size_t gkv_q8_attend_mfma_lds(int d, int g, int waves) {
  return sizeof(float) * ((size_t)waves * g * (d + 4) + 2 * 16 * (size_t)waves) + (size_t)waves * 2 * d;
}

hipError_t gkv_launch_q8_attend_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8AttendArgs& a) {
  if (dtype == GKV_F32) return dm.d == 64 ? launch_waves<float, 64>(ln, dm, a) : launch_waves<float, 128>(ln, dm, a);
  return dm.d == 64 ? launch_waves<uint16_t, 64>(ln, dm, a) : launch_waves<uint16_t, 128>(ln, dm, a);
}
