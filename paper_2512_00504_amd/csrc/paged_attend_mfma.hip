// Decode attention over pages on the matrix cores: bf16 or fp32, head_dim 64 or 128, group size g <= 16, pages of any size.
//
// One workgroup of NW wavefronts per (unit, piece).  A wavefront owns slices of 16 rows of its sequence (slice it, it + pieces*NW, ...) and
// keeps running maxima, sums and accumulators of all g query heads, so K and V are read once per KV head.  Products and softmax are
// those of attend_slice.h; bf16 probabilities enter as the sum of two bf16 numbers, which leaves 2^-16 of them.
//   WHOLE_SLICES: pages of a multiple of 16 rows, so a slice lies in one: its number comes by a scalar load, asked for a slice
//   ahead, and addresses are a scalar base, a lane's constant offset and an immediate.
//   Else a lane asks for the page of row r of a slice (one row of K), and for its four rows of V gets theirs from the lanes that have them.
// Rows behind the length are masked in a sequence's last slice.  Rows in pages outside the cache are noticed, and masked when the wavefront goes
// through its slices once more.
// The wavefronts of a workgroup are joined through LDS, pieces of a unit by whichever wavefront comes last, in a fixed order.
#include "attend_slice.h"

namespace {

struct PagedArgs {
  const int32_t *len, *table;
  const char *q, *K, *V;
  char* out;
  float* partials; int32_t* ticket;
  GkvDivisor by_splits, by_hkv, by_batch, by_iters, by_page;   // by_page: rows of a page, or slices
  int64_t layer_bytes;                                         // K of a layer
  int32_t splits, most, split_iters, Hq, Hkv, g, B, width, page_rows, n_pages;
  float scale_hi, scale_lo;
};

template <typename T, int D, int NW, int OCC, bool WHOLE_SLICES>
__global__ __launch_bounds__(NW * 64, OCC) void paged_attend_mfma_kernel(PagedArgs a) {
  using G = Geo<T, D>;
  constexpr bool WHOLE = !G::F32;
  constexpr int ROW_BYTES = G::ROW_BYTES, OSTR = G::OSTR, PSTR = G::PSTR;
  extern __shared__ __attribute__((aligned(16))) float smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, kb = lane >> 4;
  const int g = a.g, page_rows = a.page_rows, n_pages = a.n_pages;
  const int unit = quotient(blockIdx.x, a.by_splits), sp = (int)blockIdx.x - unit * a.splits;
  const int lb = quotient(unit, a.by_hkv), j = unit - lb * a.Hkv;
  const int layer = quotient(lb, a.by_batch), seq = lb - layer * a.B;
  const size_t head0 = (size_t)lb * a.Hq + j * g;
  const char* q_g = a.q + head0 * ROW_BYTES;
  const int32_t* table = a.table + (int64_t)seq * a.width;
  const char* K = a.K + layer * a.layer_bytes;
  const char* V = a.V + layer * a.layer_bytes;

  const int held = a.len[seq];
  u32x4 qB[G::NL];
  {
    const uint32_t at = min(r, g - 1) * ROW_BYTES + kb * 16;   // (lanes beyond the group repeat its last head and are ignored)
#pragma unroll
    for (int c = 0; c < G::NL; ++c) qB[c] = ld16(q_g + at + c * 64);
  }
  const int n_tot = max(0, min(held, a.width * page_rows));
  const int n_iter = (n_tot + 15) >> 4;
  const int ns = max(1, min(a.splits, quotient(n_iter + a.split_iters - 1, a.by_iters)));
  if (sp >= ns) return;
  const int it0 = sp * NW + wave, stride = ns * NW;

  // The page (or pages, a lane each) of a slice, on their way a slice ahead.
  auto ask = [&](int it) -> int {
    if constexpr (WHOLE_SLICES) return table[quotient(min(it, max(n_iter - 1, 0)), a.by_page)];
    else return table[quotient(min(16 * it + r, max(n_tot - 1, 0)), a.by_page)];
  };
  Slice<T, D, 1> s;
  uint32_t missing = 0;                                        // rows of the slice whose pages are not there, a bit each (their loads go to page 0)
  uint32_t k_off = r * ROW_BYTES + kb * 16, v_off = kb * 4 * ROW_BYTES + r * (G::VW == 2 ? 8 : 16);
  asm volatile("" : "+v"(k_off), "+v"(v_off));                 // (offsets stay offsets)
  auto request = [&](int it, int page) {
    if constexpr (WHOLE_SLICES) {
      page = __builtin_amdgcn_readfirstlane(page);
      const bool there = (uint32_t)page < (uint32_t)n_pages;
      missing = there ? 0u : 0xffffu;
      const int in_page = it * 16 - quotient(it, a.by_page) * page_rows;
      int64_t at = (((int64_t)(there ? page : 0) * a.Hkv + j) * page_rows + in_page) * ROW_BYTES;
      asm volatile("" : "+s"(at));                             // (and bases scalar)
      const char *Kt = K + at, *Vt = V + at;
#pragma unroll
      for (int c = 0; c < G::NL; ++c) s.kA[0][c] = ld16(Kt + k_off + c * 64);
#pragma unroll
      for (int e = 0; e < 4; ++e) ld_v<T, D>(s.vR[e], Vt + v_off + e * ROW_BYTES);
    } else {
      const int n = min(16 * it + r, n_tot - 1);
      const bool there = (uint32_t)page < (uint32_t)n_pages;
      missing = (uint32_t)__ballot(!there) & 0xffffu;
      const uint32_t row = there ? ((uint32_t)page * (uint32_t)a.Hkv + (uint32_t)j) * (uint32_t)page_rows + (uint32_t)(n - quotient(n, a.by_page) * page_rows) : 0u;
      const char* Kt = K + (uint64_t)row * ROW_BYTES + kb * 16;
#pragma unroll
      for (int c = 0; c < G::NL; ++c) s.kA[0][c] = ld16(Kt + c * 64);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t v_row = (uint32_t)__shfl((int)row, 4 * kb + e);
        ld_v<T, D>(s.vR[e], V + (uint64_t)v_row * ROW_BYTES + r * (G::VW == 2 ? 8 : 16));
      }
    }
  };
  Running<G::NC> st;
  auto reset = [&]() {
    st.m_run = GKV_NO_MAX;
    st.l_run = 0.f;
#pragma unroll
    for (int m = 0; m < G::NC; ++m) st.oacc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  reset();
  auto process = [&](int it, bool last) {
    process_slice<T, D, 1, false, WHOLE>(s, st, qB, it, false, last, a.scale_hi, a.scale_lo, r, kb, [&](int row) { return row >= n_tot; }, Nothing{});
  };
  if (it0 < n_iter) {
    int page = ask(it0);
    request(it0, page);
    page = ask(it0 + stride);
    uint32_t any_missing = missing;
    int it = it0;
    for (; it + stride < n_iter; it += stride) {
      process(it, false);
      __builtin_amdgcn_sched_barrier(0);                       // (requests that move up between the products need registers of their own)
      request(it + stride, page);
      any_missing |= missing;
      page = ask(it + 2 * stride);
      asm volatile("; next slice");                            // (the same requests ahead of the loop stay apart from these)
    }
    process(it, it == n_iter - 1);
    // Seldom: a page that is not there, a maximum that the short form of the weights is not right for, or a NaN that may be its doing or that
    // of an infinite value and a part of P that is zero.  The slices are gone through again.
    bool again = any_missing != 0 || fabsf(st.m_run) >= GKV_HUGE_LOG2 || st.l_run != st.l_run;
    if constexpr (WHOLE) {
      float x = st.l_run;
#pragma unroll
      for (int m = 0; m < G::NC; ++m)
#pragma unroll
        for (int e = 0; e < 4; e += 2)
          x = __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, st.oacc[m][e]), st.oacc[m][e + 1]);
      again |= x != x;
    }
    if (__any(again)) {
      reset();
      for (int it = it0; it < n_iter; it += stride) {
        request(it, ask(it));
        process_slice<T, D, 1, true, WHOLE>(s, st, qB, it, false, true, a.scale_hi, a.scale_lo, r, kb,
                                            [&](int row) { return row >= n_tot || (missing >> (row & 15)) & 1; }, Nothing{});
      }
    }
  }

  // ---- merge the wavefronts of this workgroup -------------------------------------------------
  float* so = smem;                         // [NW][g][OSTR]
  float* sm = so + NW * g * OSTR;           // [16][NW]
  float* sl = sm + NW * 16;                 // [16][NW]
  const float l_tot = over_head(st.l_run, false);      // the 4 lanes of a head hold partial sums
  if (r < g) {
    float* row = so + (wave * g + r) * OSTR;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int q4 = 0; q4 < G::NC / 4; ++q4) {
        const int ch = (G::F32 && D == 128) ? 64 * q4 + 4 * (4 * kb + e) : G::NC * (4 * kb + e) + 4 * q4;
        *(f32x4*)(row + ch) = f32x4{st.oacc[4 * q4][e], st.oacc[4 * q4 + 1][e], st.oacc[4 * q4 + 2][e], st.oacc[4 * q4 + 3][e]};
      }
    }
    if (kb == 0) { sm[r * NW + wave] = st.m_run; sl[r * NW + wave] = l_tot; }
  }
  constexpr int TPH = D / 4;                // threads per head
  __syncthreads();

  T* out = (T*)a.out + head0 * D;
  float* part = a.partials + (size_t)unit * a.most * g * PSTR;        // [ns][g][PSTR]
  auto finish = [&](int x, float L, f32x4 o) {
    bool any = false;
    if (L == 0.f)                                              // seldom: no row, or none with weight
      for (int p = 0; p * page_rows < n_tot; ++p) any |= (uint32_t)table[p] < (uint32_t)n_pages;
    store_row4(out + (uint32_t)(x * 4), o * inv_sum(L, any, false));
  };
  for (int x = tid; x < g * TPH; x += NW * 64) {
    const int h = x / TPH, c4 = (x % TPH) * 4;
    float mw[NW], lw[NW];
#pragma unroll
    for (int i = 0; i < NW / 4; ++i) {
      const f32x4 m4 = *(const f32x4*)(sm + h * NW + 4 * i), l4 = *(const f32x4*)(sl + h * NW + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) { mw[4 * i + e] = m4[e]; lw[4 * i + e] = l4[e]; }
    }
    float M = GKV_NO_MAX;
#pragma unroll
    for (int wv = 0; wv < NW; ++wv) M = fmaxf(M, mw[wv]);
    float Lsum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int wv = 0; wv < NW; ++wv) {
      const float f = __builtin_amdgcn_exp2f(mw[wv] - M);
      Lsum += lw[wv] * f;
      o += *(const f32x4*)(so + (wv * g + h) * OSTR + c4) * f;
    }
    if (ns == 1) {
      finish(x, Lsum, o);
    } else {
      float* ph = part + (uint32_t)((sp * g + h) * PSTR);
      store_agent(ph + c4, o[0], o[1]);
      store_agent(ph + c4 + 2, o[2], o[3]);
      if (c4 == 0) store_agent(ph + D, M, Lsum);
    }
  }
  if (ns == 1 || wave * 64 >= g * TPH) return;

  // ---- pieces: whoever finishes last joins them -------------------------------------------------
  // A wavefront's outputs are whole heads and need the same heads of the other pieces only: a ticket for each wavefront and no barrier.
  // Partial results go through memory with agent-scope accesses, each wavefront waits for its own stores, and its ticket follows.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  uint32_t arrived = 0;
  if (lane == 0) arrived = __builtin_amdgcn_atomic_inc32((uint32_t*)a.ticket + (size_t)unit * GKV_TICKETS + wave, (uint32_t)ns - 1u, __ATOMIC_RELAXED, "agent");
  if ((int)__builtin_amdgcn_readfirstlane(arrived) != ns - 1) return;
  asm volatile("" ::: "memory");
  for (int x = tid; x < g * TPH; x += NW * 64) {
    const int h = x / TPH, c4 = (x % TPH) * 4;
    float M = GKV_NO_MAX, Lsum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    constexpr int AT_ONCE = 8;
    for (int s0 = 0; s0 < ns; s0 += AT_ONCE) {
      float2 got[AT_ONCE][3];
      const float* ph = part + (size_t)(s0 * g + h) * PSTR;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (s0 + i < ns) {                                   // uniform, here and below
          got[i][0] = load_agent(ph + D); got[i][1] = load_agent(ph + c4); got[i][2] = load_agent(ph + c4 + 2);
          ph += (uint32_t)(g * PSTR);
        }
      float Mn = M;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (s0 + i < ns) Mn = fmaxf(Mn, got[i][0].x);
      const float f0 = __builtin_amdgcn_exp2f(M - Mn);
      M = Mn;
      Lsum *= f0;
      o *= f0;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (s0 + i < ns) {
          const float f = __builtin_amdgcn_exp2f(got[i][0].x - Mn);
          Lsum += got[i][0].y * f;
          o += f32x4{got[i][1].x, got[i][1].y, got[i][2].x, got[i][2].y} * f;
        }
    }
    finish(x, Lsum, o);
  }
}

size_t lds_bytes(const GkvDims& dm, int waves) { return sizeof(float) * waves * ((size_t)dm.g * (dm.d + 4) + 2 * 16); }

template <typename T, int D, int NW, int OCC>
hipError_t launch(const GkvLaunch& ln, const GkvDims& dm, const PagedAttendArgs& a) {
  const bool whole = a.pages.page_rows % 16 == 0;
  PagedArgs k;
  k.len = a.len; k.table = a.pages.table;
  k.q = (const char*)a.q; k.K = (const char*)a.K; k.V = (const char*)a.V; k.out = (char*)a.out;
  k.partials = a.partials; k.ticket = a.ticket;
  k.by_splits = gkv_divisor(a.splits); k.by_hkv = dm.by_hkv; k.by_batch = gkv_divisor(dm.B); k.by_iters = gkv_divisor(a.split_iters);
  k.by_page = gkv_divisor(whole ? a.pages.page_rows / 16 : a.pages.page_rows);
  k.layer_bytes = (int64_t)a.pages.n_pages * dm.Hkv * a.pages.page_rows * Geo<T, D>::ROW_BYTES;
  k.splits = a.splits; k.most = a.most; k.split_iters = a.split_iters;
  k.Hq = dm.Hq; k.Hkv = dm.Hkv; k.g = dm.g; k.B = dm.B;
  k.width = a.pages.width; k.page_rows = a.pages.page_rows; k.n_pages = a.pages.n_pages;
  k.scale_hi = dm.scale_l2_hi; k.scale_lo = dm.scale_l2_lo;
  auto kern = whole ? paged_attend_mfma_kernel<T, D, NW, OCC, true> : paged_attend_mfma_kernel<T, D, NW, OCC, false>;
  return gkv_launch(ln, kern, dim3(dm.L * dm.B * dm.Hkv * a.splits), dim3(NW * 64), lds_bytes(dm, NW), k);
}

}  // namespace

hipError_t gkv_launch_paged_attend_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PagedAttendArgs& a) {
  if (lds_bytes(dm, 8) > GKV_LDS_LIMIT) {                    // d = 128, g = 16
    if (dtype == GKV_F32) return launch<float, 128, 4, 2>(ln, dm, a);
    return launch<uint16_t, 128, 4, 4>(ln, dm, a);
  }
  if (dtype == GKV_F32) return dm.d == 64 ? launch<float, 64, 8, 4>(ln, dm, a) : launch<float, 128, 8, 2>(ln, dm, a);
  return dm.d == 64 ? launch<uint16_t, 64, 8, 4>(ln, dm, a) : launch<uint16_t, 128, 8, 4>(ln, dm, a);
}
