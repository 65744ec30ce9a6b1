// Decode attention over pages on the matrix cores: bf16, head_dim 64, 96, 128 or 256, or fp32, 64 or 128, groups of any size (16 heads at a time), pages of any size.
//
// One workgroup of NW wavefronts per (unit, piece).  A wavefront owns slices of 16 rows of its sequence (slice it, it + pieces*NW, ...) and
// keeps running maxima, sums and accumulators of up to 16 query heads, so K and V are read once per KV head where g is no more.  Products and softmax are
// those of attend_slice.h; bf16 probabilities enter as the sum of two bf16 numbers, within 2^-15 of them (the upper half of their
// bits, and the rest rounded), at d = 64 of three, which have all bits.
//   WHOLE_SLICES: pages of a multiple of 16 rows, so a slice lies in one: its number comes by a scalar load, asked for a slice
//   ahead, and addresses are a scalar base, a lane's constant offset and an immediate.
//   Else a lane asks for the page of row r of a slice (one row of K), and for its four rows of V gets theirs from the lanes that have them.
// Rows behind the length are masked in a sequence's last slice.  Rows in pages outside the cache are noticed, and masked when the wavefront goes
// through its slices once more.
// The wavefronts of a workgroup are joined through LDS, pieces of a unit by whichever wavefront comes last, in a fixed order.
#include "attend_slice.h"

namespace {

__device__ __forceinline__ void store_row2(float* p, const f32x2& o) { *(f32x2*)p = o; }
__device__ __forceinline__ void store_row2(uint16_t* p, const f32x2& o) { *(uint32_t*)p = __builtin_bit_cast(uint32_t, __builtin_convertvector(o, bf16x2)); }

// Maximum or sum over N = 32 or 64 neighbouring lanes, in each of them, without a trip through LDS (12 of those in a row took 0.6 us).
template <int N, bool MAX>
__device__ __forceinline__ float over_lanes(float x) {
  auto with = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
  auto moved = [](float a, auto how) {
    const int u = __float_as_int(a);
    return __int_as_float(__builtin_amdgcn_update_dpp(u, u, decltype(how)::value, 0xf, 0xf, false));
  };
  x = with(x, moved(x, std::integral_constant<int, 0xb1>{}));        // lane ^ 1
  x = with(x, moved(x, std::integral_constant<int, 0x4e>{}));        // lane ^ 2
  x = with(x, moved(x, std::integral_constant<int, 0x141>{}));       // the other four of eight
  x = with(x, moved(x, std::integral_constant<int, 0x140>{}));       // the other eight of sixteen
  const uint32_t u = __float_as_uint(x);
  const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(u, u, false, false));
  x = with(__uint_as_float(y[0]), __uint_as_float(y[1]));
  if (N == 64) {
    const uint32_t v = __float_as_uint(x);
    const u32x2 z = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v, v, false, false));
    x = with(__uint_as_float(z[0]), __uint_as_float(z[1]));
  }
  return x;
}

constexpr int pass(int D) { return D <= 64 ? 16 : D <= 128 ? 8 : 4; }   // heads whose sums go through LDS at a time

struct PagedArgs {
  const int32_t *len, *table;
  const char *q, *K, *V;
  char* out;
  float* partials; int32_t* ticket;
  GkvDivisor by_blocks, by_parts, by_hkv, by_batch, by_iters, by_long, by_page;   // by_page: rows of a page, or slices
  int64_t layer_bytes;                                         // K of a layer
  GkvPagedCut cut;
  int32_t blocks, parts, splits, most, Hq, Hkv, g, B, width, page_rows, n_pages;
  float scale_hi, scale_lo;
};

template <typename T, int D, int NW, int KT, int OCC, bool WHOLE_SLICES>
__global__ __launch_bounds__(NW * 64, OCC) void paged_attend_mfma_kernel(PagedArgs a) {
  using G = Geo<T, D>;
  constexpr bool WHOLE = !G::F32 && KT == 1;
  constexpr int KEYS = 16 * KT;                                // rows of a slice
  constexpr int PASS = pass(D);
  constexpr int ROW_BYTES = G::ROW_BYTES, OSTR = G::OSTR, PSTR = G::PSTR;
  extern __shared__ __attribute__((aligned(16))) float smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, kb = lane >> 4;
  const int page_rows = a.page_rows, n_pages = a.n_pages;
  // (units first: workgroups go to the XCDs in turn, and the last pieces are those of the longest sequences only)
  const int sp = quotient(blockIdx.x, a.by_blocks), block = (int)blockIdx.x - sp * a.blocks;   // of up to 16 heads of a unit
  const int unit = quotient(block, a.by_parts), part0 = (block - unit * a.parts) * 16, g = min(16, a.g - part0);
  const int lb = quotient(unit, a.by_hkv), j = unit - lb * a.Hkv;
  const int layer = quotient(lb, a.by_batch), seq = lb - layer * a.B;
  const size_t head0 = (size_t)lb * a.Hq + j * a.g + part0;
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
  // Pages of a slice, of each 16 rows or a lane each, on their way a slice ahead, the first ones' together with the length: where that ends is
  // not known then, where the table does is.
  const int it_first = sp * NW + wave;                         // (of any number of pieces)
  struct Pages { int of[KT]; };
  auto ask = [&](int it) {
    Pages p;
#pragma unroll
    for (int t = 0; t < KT; ++t) p.of[t] = table[min(quotient(WHOLE_SLICES ? it * KT + t : it * KEYS + 16 * t + r, a.by_page), a.width - 1)];
    return p;
  };
  const Pages pages0 = ask(it_first);
  const int n_tot = max(0, min(held, a.width * page_rows));
  const int n_tiles = (n_tot + 15) >> 4, n_iter = (int)((uint32_t)(n_tot + KEYS - 1) / KEYS);
  // (GkvPagedCut::pieces)
  const int more = (n_tiles >= a.cut.twice) + (n_tiles >= a.cut.four_times);
  const int by_iters = (quotient(n_tiles + a.cut.iters - 1, a.by_iters) + (1 << more) - 1) >> more;
  const int ns = max(1, min(a.splits, max(min(by_iters, a.cut.soft), quotient(n_tiles + a.cut.long_iters - 1, a.by_long))));
  if (sp >= ns) return;
  const int it0 = it_first, stride = ns * NW;

  // Where a slice's rows are, from its page or pages.  missing: rows whose pages are not there, a bit each (their loads go to page 0).
  struct Place { int64_t at[KT]; uint32_t k_row[KT], v_row[KT][4], missing; };
  auto locate = [&](int it, const Pages& p) {
    Place w;
    w.missing = 0;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      if constexpr (WHOLE_SLICES) {
        const int tile = KT == 1 ? it : min(it * KT + t, n_tiles - 1), page = __builtin_amdgcn_readfirstlane(p.of[t]);
        const bool there = (uint32_t)page < (uint32_t)n_pages;
        if (!there && (KT == 1 || it * KT + t < n_tiles)) w.missing |= 0xffffu << (16 * t);
        const int in_page = tile * 16 - quotient(tile, a.by_page) * page_rows;
        w.at[t] = (((int64_t)(there ? page : 0) * a.Hkv + j) * page_rows + in_page) * ROW_BYTES;
      } else {
        const int at = it * KEYS + 16 * t + r, n = min(at, n_tot - 1);
        const bool there = (uint32_t)p.of[t] < (uint32_t)n_pages && at < n_tot;
        w.missing |= ((uint32_t)__ballot(!there && at < n_tot) & 0xffffu) << (16 * t);
        w.k_row[t] = there ? ((uint32_t)p.of[t] * (uint32_t)a.Hkv + (uint32_t)j) * (uint32_t)page_rows + (uint32_t)(n - quotient(n, a.by_page) * page_rows) : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) w.v_row[t][e] = (uint32_t)__shfl((int)w.k_row[t], 4 * kb + e);
      }
    }
    return w;
  };
  uint32_t k_off = r * ROW_BYTES + kb * 16, v_off = kb * 4 * ROW_BYTES + r * G::V_BYTES;
  asm volatile("" : "+v"(k_off), "+v"(v_off));                 // (offsets stay offsets)
  auto request = [&](Slice<T, D, KT>& s, Place w) {
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      if constexpr (WHOLE_SLICES) {
        asm volatile("" : "+s"(w.at[t]));                      // (and bases scalar)
        const char* Kt = K + w.at[t];
#pragma unroll
        for (int c = 0; c < G::NL; ++c) s.kA[t][c] = ld16(Kt + k_off + c * 64);
      } else {
        const char* Kt = K + (uint64_t)w.k_row[t] * ROW_BYTES + kb * 16;
#pragma unroll
        for (int c = 0; c < G::NL; ++c) s.kA[t][c] = ld16(Kt + c * 64);
      }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (WHOLE_SLICES) ld_v<T, D>(s.vR[4 * t + e], V + w.at[t] + v_off + e * ROW_BYTES);
        else ld_v<T, D>(s.vR[4 * t + e], V + (uint64_t)w.v_row[t][e] * ROW_BYTES + r * G::V_BYTES);
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
  auto process = [&](Slice<T, D, KT>& s, int it, bool last) {
    process_slice<T, D, KT, false, WHOLE>(s, st, qB, it, false, last, a.scale_hi, a.scale_lo, r, kb, [&](int row) { return row >= n_tot; }, Nothing{});
  };
  if (it0 < n_iter) {
    Slice<T, D, KT> s0;
    Pages next = ask(it0 + stride);
    Place w = locate(it0, pages0);
    request(s0, w);
    uint32_t any_missing = w.missing;
    int it = it0;
    for (; it + stride < n_iter; it += stride) {
      // the next slice's place is known before this one is there, and the one's after that is asked for
      w = locate(it + stride, next);
      next = ask(it + 2 * stride);
      any_missing |= w.missing;
      process(s0, it, false);
      __builtin_amdgcn_sched_barrier(0);                       // (requests that move up between the products need registers of their own)
      request(s0, w);
      asm volatile("; next slice");                            // (the same requests ahead of the loop stay apart from these)
    }
    process(s0, it, it == n_iter - 1);
    // Seldom: a page that is not there, a maximum that the short form of the weights is not right for, or a NaN that may be its doing or that
    // of an infinite value and a part of P that is zero.  The slices are gone through again.
    bool again = any_missing != 0 || fabsf(st.m_run) >= GKV_HUGE_LOG2 || st.l_run != st.l_run;
    if constexpr (!G::F32) {
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
        w = locate(it, ask(it));
        request(s0, w);
        process_slice<T, D, KT, true, WHOLE>(s0, st, qB, it, false, true, a.scale_hi, a.scale_lo, r, kb,
                                            [&](int row) { return row >= n_tot || (w.missing >> (row & (KEYS - 1))) & 1; }, Nothing{});
      }
    }
  }

  // ---- merge the wavefronts of this workgroup, PASS heads at a time ------------------------------
  const int in_pass = min(g, PASS);
  float* so = smem;                         // [NW][in_pass][OSTR]
  float* sm = so + NW * in_pass * OSTR;     // [16][NW]
  float* sl = sm + NW * 16;                 // [16][NW]
  const float l_tot = over_head(st.l_run, false);      // the 4 lanes of a head hold partial sums
  if (r < g && kb == 0) { sm[r * NW + wave] = st.m_run; sl[r * NW + wave] = l_tot; }
  // threads per head, of CPT channels each (D = 96: some have none)
  constexpr int TPH = D <= 64 ? 32 : 64, CPT = D <= 128 ? 2 : 4;
  typedef float Channels __attribute__((ext_vector_type(CPT)));
  T* out = (T*)a.out + head0 * D;
  // of a unit: outputs [most][its g][D], then maximum and sum [its g][most]
  float* part = a.partials + (size_t)unit * a.most * a.g * PSTR + part0 * D;
  float* part_ms = a.partials + (size_t)unit * a.most * a.g * PSTR + (size_t)a.most * a.g * D + (size_t)part0 * a.most * 2;
  auto finish = [&](int h, int c, float L, Channels o) {
    bool any = false;
    if (L == 0.f)                                              // seldom: no row, or none with weight
      for (int p = 0; p * page_rows < n_tot; ++p) any |= (uint32_t)table[p] < (uint32_t)n_pages;
    o *= inv_sum(L, any, false);
    if constexpr (CPT == 2) store_row2(out + (uint32_t)(h * D + c), o);
    else store_row4(out + (uint32_t)(h * D + c), o);
  };
  for (int first = 0; first < g; first += PASS) {
    if (first > 0) __syncthreads();
    if (r >= first && r < min(g, first + PASS)) {
      float* row = so + (wave * in_pass + r - first) * OSTR;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // neighbouring channels: a lane's are NC from NC (4 kb + e) on, of rows of 512 bytes half as many in either half
        constexpr int W = G::NC % 4 == 0 ? 4 : 2, SIDE = G::VW == 8 ? G::NC / 2 : G::NC;
        typedef float Some __attribute__((ext_vector_type(W)));
#pragma unroll
        for (int m = 0; m < G::NC; m += W) {
          Some x;
#pragma unroll
          for (int i = 0; i < W; ++i) x[i] = st.oacc[m + i][e];
          *(Some*)(row + m / SIDE * (D / 2) + SIDE * (4 * kb + e) + m % SIDE) = x;
        }
      }
    }
    __syncthreads();
    for (int x = first * TPH + tid; x < min(g, first + PASS) * TPH; x += NW * 64) {
      const int h = x / TPH, c = (x % TPH) * CPT;
      if (c >= D) continue;
      float M = GKV_NO_MAX, mw[NW];
#pragma unroll
      for (int wv = 0; wv < NW; ++wv) M = fmaxf(M, mw[wv] = sm[h * NW + wv]);
      float Lsum = 0.f;
      Channels o = 0.f;
#pragma unroll
      for (int wv = 0; wv < NW; ++wv) {
        const float f = __builtin_amdgcn_exp2f(mw[wv] - M);
        Lsum += sl[h * NW + wv] * f;
        o += *(const Channels*)(so + (wv * in_pass + h - first) * OSTR + c) * f;
      }
      if (ns == 1) {
        finish(h, c, Lsum, o);
      } else {
#pragma unroll
        for (int i = 0; i < CPT; i += 2) store_agent(part + (uint32_t)((sp * a.g + h) * D + c + i), o[i], o[i + 1]);
        if (c == 0) store_agent(part_ms + (uint32_t)((h * a.most + sp) * 2), M, Lsum);
      }
    }
  }
  if (ns == 1 || wave * 64 >= in_pass * TPH) return;           // (uniform)

  // ---- pieces: whoever finishes last joins them -------------------------------------------------
  // A wavefront's outputs are whole heads and need the same heads of the other pieces only: a ticket for each wavefront and no barrier.
  // Partial results go through memory with agent-scope accesses, each wavefront waits for its own stores, and its ticket follows.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  uint32_t arrived = 0;
  if (lane == 0)
    arrived = __builtin_amdgcn_atomic_inc32((uint32_t*)a.ticket + ((size_t)block * GKV_TICKETS + wave) * GKV_PAGED_TICKET, (uint32_t)ns - 1u, __ATOMIC_RELAXED, "agent");
  if ((int)__builtin_amdgcn_readfirstlane(arrived) != ns - 1) return;
  asm volatile("" ::: "memory");
  // A lane has maximum and sum of one piece and makes its factor, so all outputs can be asked for at once.  A wavefront has one head (D > 64) or two.
  constexpr int AT_A_TIME = TPH, AT_ONCE = 32 / CPT;
  for (int first = 0; first < g; first += PASS)
    for (int x = first * TPH + tid; x < min(g, first + PASS) * TPH; x += NW * 64) {   // (the outputs whose parts this wavefront stored)
      const int h = x / TPH, c = min((x % TPH) * CPT, D - CPT), in_head = lane % TPH, lane0 = lane - in_head;   // (lanes without channels go along)
      float M = GKV_NO_MAX, Lsum = 0.f;
      Channels o = 0.f;
      float2 got[AT_ONCE][CPT / 2];
      auto ask_for = [&](int s1) {
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
          for (int k = 0; k < CPT / 2; ++k) got[i][k] = load_agent(part + (uint32_t)((min(s1 + i, ns - 1) * a.g + h) * D + c + 2 * k));
      };
      for (int s0 = 0; s0 < ns; s0 += AT_A_TIME) {
        float2 ms = load_agent(part_ms + (uint32_t)((h * a.most + min(s0 + in_head, ns - 1)) * 2));
        ask_for(s0);
        if (s0 + in_head >= ns) ms = make_float2(GKV_NO_MAX, 0.f);
        const float Mn = fmaxf(M, over_lanes<TPH, true>(ms.x));
        const float f = __builtin_amdgcn_exp2f(ms.x - Mn), f0 = __builtin_amdgcn_exp2f(M - Mn);
        M = Mn;
        Lsum = Lsum * f0 + over_lanes<TPH, false>(ms.y * f);
        o *= f0;
        for (int s1 = s0; s1 < min(ns, s0 + AT_A_TIME); s1 += AT_ONCE) {
          if (s1 > s0) ask_for(s1);
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) {
            const int from = (s1 + i - s0) & (TPH - 1);
            const float fi = TPH == 64 ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), from)) : __shfl(f, lane0 + from);
            if (s1 + i < ns) {
#pragma unroll
              for (int k = 0; k < CPT / 2; ++k) {
                o[2 * k] = fmaf(got[i][k].x, fi, o[2 * k]);
                o[2 * k + 1] = fmaf(got[i][k].y, fi, o[2 * k + 1]);
              }
            }
          }
        }
      }
      if ((x % TPH) * CPT < D) finish(h, c, Lsum, o);
    }
}

template <typename T, int D, int NW, int KT, int OCC>
hipError_t launch(const GkvLaunch& ln, const GkvDims& dm, const PagedAttendArgs& a) {
  constexpr int PASS = pass(D);
  static_assert(sizeof(float) * NW * (PASS * (D + 4) + 2 * 16) <= GKV_LDS_LIMIT);
  const bool whole = a.pages.page_rows % 16 == 0;
  PagedArgs k;
  k.len = a.len; k.table = a.pages.table;
  k.q = (const char*)a.q; k.K = (const char*)a.K; k.V = (const char*)a.V; k.out = (char*)a.out;
  k.partials = a.partials; k.ticket = a.ticket;
  k.parts = gkv_paged_parts(dm.g); k.blocks = dm.L * dm.B * dm.Hkv * k.parts;
  k.by_blocks = gkv_divisor(k.blocks); k.by_parts = gkv_divisor(k.parts); k.by_hkv = dm.by_hkv; k.by_batch = gkv_divisor(dm.B); k.by_iters = gkv_divisor(a.cut.iters); k.by_long = gkv_divisor(a.cut.long_iters);
  k.by_page = gkv_divisor(whole ? a.pages.page_rows / 16 : a.pages.page_rows);
  k.layer_bytes = (int64_t)a.pages.n_pages * dm.Hkv * a.pages.page_rows * Geo<T, D>::ROW_BYTES;
  k.splits = a.splits; k.most = a.most; k.cut = a.cut;
  k.Hq = dm.Hq; k.Hkv = dm.Hkv; k.g = dm.g; k.B = dm.B;
  k.width = a.pages.width; k.page_rows = a.pages.page_rows; k.n_pages = a.pages.n_pages;
  k.scale_hi = dm.scale_l2_hi; k.scale_lo = dm.scale_l2_lo;
  auto kern = whole ? paged_attend_mfma_kernel<T, D, NW, KT, OCC, true> : paged_attend_mfma_kernel<T, D, NW, KT, OCC, false>;
  return gkv_launch(ln, kern, dim3(k.blocks * a.splits), dim3(NW * 64), sizeof(float) * NW * ((size_t)(dm.g < PASS ? dm.g : PASS) * (D + 4) + 2 * 16), k);
}

// Wavefronts of a workgroup: 8, or fewer where the longest sequence has fewer slices.  A slice is a wavefront's then, and those without one add
// zeros: the same bits (29344 units of up to 7 rows, d = 64, 125 -> 29 us).  4 also where many units' tables end at 512 rows: a workgroup of 8
// has hardly begun then when it ends (us, 8 / 4: 14336 units of up to 100 rows 93 / 63, 300 209 / 201, 577 362 / 362; 3584 of up to 2100 330 / 345).
template <typename T, int D, int KT, int OCC>
hipError_t by_length(const GkvLaunch& ln, const GkvDims& dm, const PagedAttendArgs& a) {
  const int64_t units = (int64_t)dm.L * dm.B * dm.Hkv, room = (int64_t)a.pages.width * a.pages.page_rows;
  if (a.len_max <= 16 * KT) return launch<T, D, 1, KT, OCC>(ln, dm, a);
  if (a.len_max <= 4 * 16 * KT || (units >= 1024 && room <= 512)) return launch<T, D, 4, KT, OCC>(ln, dm, a);
  return launch<T, D, 8, KT, OCC>(ln, dm, a);
}

}  // namespace

hipError_t gkv_launch_paged_attend_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PagedAttendArgs& a) {
  if (dtype == GKV_F32) return dm.d == 64 ? by_length<float, 64, 1, 4>(ln, dm, a) : by_length<float, 128, 1, 2>(ln, dm, a);
  switch (dm.d) {
    case 64: return by_length<uint16_t, 64, 2, 4>(ln, dm, a);
    case 96: return by_length<uint16_t, 96, 1, 4>(ln, dm, a);
    case 128: return by_length<uint16_t, 128, 1, 4>(ln, dm, a);
    default: return by_length<uint16_t, 256, 1, 2>(ln, dm, a);
  }
}
