// What the matrix-core decode kernels on caches of bf16 and fp32 rows share: a wavefront's slice of 16 (or 32) keys, its
// loads' shape, the online softmax and the two products.  attend_mfma.hip has the layouts and what they cost.
#pragma once

#include "gkv_internal.h"

#include <type_traits>

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ u32x4 ld16(const void* p) { return *(const u32x4*)p; }
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Row geometry of one (element type, head_dim).
template <typename T, int D>
struct Geo {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int ROW_BYTES = D * (int)sizeof(T);
  static constexpr int TILE_BYTES = 16 * ROW_BYTES;
  static constexpr int NL = ROW_BYTES / 64;      // K loads (16 bytes a lane) per tile
  static constexpr int RP = ROW_BYTES / 16;      // 16-byte pieces per row
  static constexpr int NC = D / 16;              // channels per lane, accumulators per lane
  static constexpr int VW = ROW_BYTES / 64;      // 32-bit words of V per lane and key
  static constexpr int V_BYTES = VW == 8 ? 16 : 4 * VW;   // of a row's bytes from a lane's first on, with VW == 8 twice
  static constexpr int OSTR = D + 4;             // padded LDS row of the per-wave partial outputs
  static constexpr int PSTR = D + 2;             // split partial: o[D], m, l
};

// V words of one key for lane r: channels [r*NC, +NC), except rows of 512 bytes, whose lanes take 16
// bytes from each half of the row so that both loads are contiguous over the lanes.
template <int VW> struct VWords { uint32_t w[VW]; };
template <typename T, int D>
__device__ __forceinline__ void ld_v(VWords<Geo<T, D>::VW>& o, const char* p) {
  if constexpr (Geo<T, D>::VW == 2) {
    const u32x2 a = __builtin_nontemporal_load((const u32x2*)p);
    o.w[0] = a[0]; o.w[1] = a[1];
  } else if constexpr (Geo<T, D>::VW == 3) {
#pragma unroll
    for (int i = 0; i < 3; ++i) o.w[i] = __builtin_nontemporal_load((const uint32_t*)p + i);
  } else {
    const u32x4 a = __builtin_nontemporal_load((const u32x4*)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o.w[i] = a[i];
    if constexpr (Geo<T, D>::VW == 8) {
      const u32x4 b = __builtin_nontemporal_load((const u32x4*)(p + 256));
#pragma unroll
      for (int i = 0; i < 4; ++i) o.w[4 + i] = b[i];
    }
  }
}
// One wavefront iteration's loads: KT K tiles (A operands) and 4*KT V rows per lane.
template <typename T, int D, int KT>
struct Slice {
  u32x4 kA[KT][Geo<T, D>::NL];
  VWords<Geo<T, D>::VW> vR[4 * KT];
};

// Two bf16 numbers, zero in place of infinities and NaN.
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  if ((w & 0x00007f80u) == 0x00007f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0x0000ffffu;
  return w;
}

struct Nothing { __device__ void operator()() const {} };

// Flash-decoding state of one wavefront: lane (head = lane%16, blk = lane/16) holds the running
// max (in log2 units, shared by the 4 lanes of a head), its partial running sum, and in
// oacc[m][e] O[head][channel m of lane 4 blk + e].
template <int NC>
struct Running {
  float m_run, l_run;
  f32x4 oacc[NC];
};

// Maximum and sum over the four lanes of a head (lane % 16), in each of them: the halves and then the quarters of
// the wavefront change places in registers, where an exchange through LDS takes 60 ns.
// The compiler keeps the wait states that results of matrix and vector instructions need, across branches too, but does not look into
// inline assembly.  The maximum here is safe by its place: its operands are results of an exchange, never of an MFMA, and the next
// exchange needs a copy of its result, with the wait states of a copy.  (fmaxf would quiet both operands first, an instruction each.)
__device__ __forceinline__ float over_head(float x, bool max) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t u = __float_as_uint(x);
    const u32x2 y = i == 0 ? __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false))
                           : __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(u, u, false, false));
    const float a = __uint_as_float(y[0]), b = __uint_as_float(y[1]);
    if (max) asm("v_max_f32 %0, %1, %2" : "=v"(x) : "v"(a), "v"(b));
    else x = a + b;
  }
  return x;
}

// edge: the slice may contain rows that are not there (gone(row): those past the end), which are masked.  first: the wavefront's first slice, whose
// accumulators are zero.  between: what to do once the products with K are under way, whose registers are free then.
// EXACT: right for every logit and value, infinities and finite ones of any size among them.  Without
// it, which is what a wavefront tries first, a logit of -inf may give NaN (the scale's low part times -inf), a
// huge maximum any weight (see log2_weight), and an infinite value NaN where P enters in parts (bf16, D = 64, and WHOLE); all of
// them show at the end.
// WHOLE (bf16, D = 128): P as the sum of two bf16 numbers.  A P rounded to one has no error where it is 1, at the largest
// logit of those that share a running maximum, and 2^-9 elsewhere, so the error grows as a unit's slices are dealt to fewer
// wavefronts: 128 units of 470 to 3900 rows, 16 running maxima a unit 3.6e-4 of the result beside the 1.657e-3 of its own rounding, 4
// to 8 of them 4.9e-4 (2-norm, against 64 bits).  Launches that are cut, or would be if their units were longer, deal out by what is fastest, and
// with both parts their error is 2e-6.  It costs 26 instructions a slice: 128 steps of 4 units 741 -> 755 us, 128 ragged units 27.7 -> 28.5.
template <typename T, int D, int KT, bool EXACT, bool WHOLE, typename Gone, typename Between>
__device__ __forceinline__ void process_slice(Slice<T, D, KT>& s, Running<D / 16>& st,
                                              const u32x4 (&qB)[Geo<T, D>::NL], int it, bool first, bool edge,
                                              float scale_log2, float scale_log2_lo, int r, int kb, Gone gone,
                                              Between between) {
  using G = Geo<T, D>;
  constexpr int NS = 4 * KT;
  const int key0 = it * 16 * KT;
  // Rows past the end have zeros for K and V (what is stored there must not reach the matrix cores) and start from the
  // logit -1e30, or -inf: all of it before the products, so that the common path has no branch between them and the maximum.
  f32x4 sc[KT];
#pragma unroll
  for (int tt = 0; tt < KT; ++tt) sc[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (edge) {
#pragma unroll
    for (int tt = 0; tt < KT; ++tt)
      if (gone(key0 + 16 * tt + r)) {
#pragma unroll
        for (int c = 0; c < G::NL; ++c) s.kA[tt][c] = u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
    for (int jj = 0; jj < NS; ++jj) {
      const int key = key0 + (jj & 3) + 4 * kb + (jj >> 2) * 16;
      if (gone(key)) {
        if constexpr (!EXACT) sc[jj >> 2][jj & 3] = -1e30f;
#pragma unroll
        for (int i = 0; i < G::VW; ++i) s.vR[jj].w[i] = 0u;
      }
    }
  }

  // scores: sc[tt][e] = q[head r] . k[key0 + 16 tt + 4 kb + e]
#pragma unroll
  for (int tt = 0; tt < KT; ++tt) {
#pragma unroll
    for (int c = 0; c < G::NL; ++c) {
      if constexpr (G::F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sc[tt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(s.kA[tt][c][i]), __uint_as_float(qB[c][i]),
                                                        sc[tt], 0, 0, 0);
      } else {
        sc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(s.kA[tt][c]), as_bf16x8(qB[c]), sc[tt], 0, 0, 0);
      }
    }
  }
  if constexpr (!std::is_same_v<Between, Nothing>) {
    __builtin_amdgcn_sched_barrier(0);
    between();
    __builtin_amdgcn_sched_barrier(0);
  }
  float sv[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    sv[i] = sc[i >> 2][i & 3];
    if constexpr (EXACT) {                                 // (zero times an infinite query is no number)
      const int key = key0 + (i >> 2) * 16 + 4 * kb + (i & 3);
      if (gone(key)) sv[i] = -INFINITY;
    }
  }
  float mx = sv[0];
#pragma unroll
  for (int i = 1; i < NS; ++i) mx = fmaxf(mx, sv[i]);
  mx = over_head(mx, true);
  const float m_new = fmaxf(st.m_run, mx * scale_log2);       // scale > 0: max commutes with it
  if (__any(m_new > st.m_run)) {
    const float corr = __builtin_amdgcn_exp2f(st.m_run - m_new);
    st.l_run *= corr;
    if (!first) {
#pragma unroll
      for (int m = 0; m < G::NC; ++m) st.oacc[m] *= corr;
    }
    st.m_run = m_new;
  }
  float pf[NS];
  float psum = 0.f;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    // exponent of 2 = z * (hi + lo) - m: the window-score kernel forms its own from the same
    // logits, so the sums recorded below are the normalisers of its probabilities
    float y;
    if constexpr (EXACT) y = log2_weight(sv[i], scale_log2, scale_log2_lo, st.m_run);
    else y = fmaf(sv[i], scale_log2_lo, fmaf(sv[i], scale_log2, -st.m_run));
    pf[i] = __builtin_amdgcn_exp2f(y);
    psum += pf[i];
  }
  st.l_run += psum;

  // O^T[channel, head] += V^T . P^T
  if constexpr (G::F32) {
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int m = 0; m < G::NC; ++m)
        st.oacc[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(s.vR[i].w[m]), pf[i], st.oacc[m], 0, 0, 0);
  } else if constexpr (EXACT && D == 64) {       // P whole, V converted word by word
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int m = 0; m < G::NC; ++m) {
        const uint32_t w = s.vR[i].w[m >> 1];
        st.oacc[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((m & 1) ? w & 0xffff0000u : w << 16), pf[i],
                                                          st.oacc[m], 0, 0, 0);
      }
  } else if constexpr (KT == 2) {
    f32x8 p8;
#pragma unroll
    for (int i = 0; i < 8; ++i) p8[i] = pf[i];
    const bf16x8 pB = __builtin_convertvector(p8, bf16x8);
    bf16x8 pM, pL;                               // D = 64: P = pB + pM + pL, all of its 24 bits
    if constexpr (D == 64) {
      const f32x8 r1 = p8 - __builtin_convertvector(pB, f32x8);
      pM = __builtin_convertvector(r1, bf16x8);
      pL = __builtin_convertvector(r1 - __builtin_convertvector(pM, f32x8), bf16x8);
    }
    u32x4 t[G::NC];
#pragma unroll
    for (int m = 0; m < G::NC; ++m) {
#pragma unroll
      for (int y = 0; y < 4; ++y)
        t[m][y] = __builtin_amdgcn_perm(s.vR[2 * y + 1].w[m >> 1], s.vR[2 * y].w[m >> 1],
                                        (m & 1) ? 0x07060302u : 0x05040100u);
      st.oacc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(t[m]), pB, st.oacc[m], 0, 0, 0);
    }
    if constexpr (D == 64) {                     // term by term: an accumulator's products don't wait for each other
#pragma unroll
      for (int m = 0; m < G::NC; ++m) st.oacc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(t[m]), pM, st.oacc[m], 0, 0, 0);
#pragma unroll
      for (int m = 0; m < G::NC; ++m) st.oacc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(t[m]), pL, st.oacc[m], 0, 0, 0);
    }
  } else if constexpr (WHOLE) {
    // P = hi + lo: hi its upper half and lo the rest, each key twice in a product over 32.  lo may be zero where P is not: hi alone
    // makes an infinite value infinite then (EXACT).
    u32x4 pw;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a = __float_as_uint(pf[2 * i]), b = __float_as_uint(pf[2 * i + 1]);
      pw[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      const f32x2 lo = {pf[2 * i] - __uint_as_float(a & 0xffff0000u), pf[2 * i + 1] - __uint_as_float(b & 0xffff0000u)};
      pw[2 + i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2));
    }
#pragma unroll
    for (int m = 0; m < G::NC; ++m) {
      u32x4 t;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        t[y] = __builtin_amdgcn_perm(s.vR[2 * y + 1].w[m >> 1], s.vR[2 * y].w[m >> 1],
                                     (m & 1) ? 0x07060302u : 0x05040100u);
        t[2 + y] = EXACT ? finite_pair(t[y]) : t[y];
      }
      st.oacc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(t), as_bf16x8(pw), st.oacc[m], 0, 0, 0);
    }
  } else {
    f32x4 p4;
#pragma unroll
    for (int i = 0; i < 4; ++i) p4[i] = pf[i];
    u32x2 pw;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      pw[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p4[2 * i], p4[2 * i + 1]}), bf16x2));
    const s16x4 pB = __builtin_bit_cast(s16x4, pw);
#pragma unroll
    for (int m = 0; m < G::NC; ++m) {
      u32x2 t;
#pragma unroll
      for (int y = 0; y < 2; ++y)
        t[y] = __builtin_amdgcn_perm(s.vR[2 * y + 1].w[m >> 1], s.vR[2 * y].w[m >> 1],
                                     (m & 1) ? 0x07060302u : 0x05040100u);
      st.oacc[m] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, t), pB, st.oacc[m], 0, 0, 0);
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
// 1/l in full precision; `fast`: v_rcp_f32 (2^-23), for uncut bf16 units at D = 128, whose P has 8 or 16
// bits.  Nothing attended to: 0; keys whose logits are all -inf: NaN, as softmax gives.
__device__ __forceinline__ float inv_sum(float l, bool any_key, bool fast) {
  if (!(l > 0.f)) return any_key && l == 0.f ? __builtin_nanf("") : 0.f;
  return fast ? __builtin_amdgcn_rcpf(l) : 1.f / l;
}

}  // namespace
