// The cache in 8 bits: prompt rows on their way in, rows on their way out, and the plain decode and window-score kernels for
// the shapes the matrix-core kernels do not cover.
#include "e4m3.h"

namespace {

__device__ __forceinline__ q8_u32x4 ld16(const void* p) { return *(const q8_u32x4*)p; }
template <bool ONCE = false>
__device__ __forceinline__ void st16(void* p, q8_u32x4 v) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, (q8_u32x4*)p);
  else *(q8_u32x4*)p = v;
}

// Sixteen elements of a row, as floats.
template <typename T>
__device__ __forceinline__ void load16(const T* p, float (&x)[16]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const q8_u32x4 a = ld16(p + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = __uint_as_float(a[e]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const q8_u32x4 a = ld16(p + 8 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[8 * i + 2 * e] = __uint_as_float(a[e] << 16);
        x[8 * i + 2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
      }
    }
  }
}
// A row's scale, from the pieces of the 2^LANES_LOG lanes that share it.
template <int LANES_LOG>
__device__ __forceinline__ uint32_t row_scale(const float (&x)[16]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, q8_finite_magnitude(x[i]));
  return q8_scale_field(q8_group_max<LANES_LOG>(m));
}
__device__ __forceinline__ q8_u32x4 codes16(const float (&x)[16], uint32_t field) {
  const float inv = q8_inverse(field);
  q8_u32x4 c;
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = q8_codes(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3], inv);
  return c;
}

// ---- prompt rows -----------------------------------------------------------------------------
// A workgroup takes `rows` tokens of one unit; 2^LANES_LOG lanes a row of K and the same row of V, 16 elements each, and a lane
// has ROWS rows on their way.  The source's rows of a unit lie L * B * h_kv rows apart: neighbouring workgroups take neighbouring
// units.  Bound: HBM.
template <typename T, int LANES_LOG>
__global__ __launch_bounds__(256) void q8_store_kernel(GkvDims dm, Q8StoreArgs a) {
  constexpr int LANES = 1 << LANES_LOG, STRIDE = 256 >> LANES_LOG, ROWS = sizeof(T) == 4 ? 1 : 2;
  const int unit = blockIdx.x, lb = quotient(unit, dm.by_hkv), tid = threadIdx.x;
  const int pieces = dm.d >> 4;
  const int64_t units = (int64_t)dm.L * dm.B * dm.Hkv;
  // sequence i's prompt is the positions [t0 - P, t0), its rows 0 .. P - 1
  const int64_t start = (int64_t)a.t0 - a.prompt_len[lb % dm.B];
  const int piece = tid & (LANES - 1);
  const bool idle = piece >= pieces;
  const int64_t skip = start - a.t_first;                            // tokens of this call before the prompt's first
  const int end = (int)max((int64_t)0, min((int64_t)min(a.n, ((int)blockIdx.y + 1) * a.rows), min((int64_t)a.t0 - a.t_first, skip + dm.cap)));
  int first = (int)blockIdx.y * a.rows;
  if (skip > first) first = (int)min(skip, (int64_t)end);
  for (int r0 = first + (tid >> LANES_LOG); r0 < end; r0 += ROWS * STRIDE) {   // the same for all lanes of a row
    float k[ROWS][16], v[ROWS][16];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const size_t src = ((size_t)min(r0 + i * STRIDE, end - 1) * units + unit) * dm.d + (idle ? 0 : piece * 16);
      load16((const T*)a.k + src, k[i]);
      load16((const T*)a.v + src, v[i]);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int r = r0 + i * STRIDE;
      const uint32_t ks = row_scale<LANES_LOG>(k[i]), vs = row_scale<LANES_LOG>(v[i]);
      if (r >= end) break;
      const size_t row = (size_t)unit * dm.cap + (size_t)(r - skip);
      if (!idle) {
        st16<true>(a.K8 + row * dm.d + piece * 16, codes16(k[i], ks));
        st16<true>(a.V8 + row * dm.d + piece * 16, codes16(v[i], vs));
      }
      if (piece == 0) {
        a.scales[row] = q8_scale_word(ks, vs);
        a.pos[row] = (int32_t)((int64_t)a.t_first + r);
      }
    }
  }
}

// ---- rows read back --------------------------------------------------------------------------
__device__ __forceinline__ void store16(float* p, size_t stride, const float (&x)[16]) {   // stride: elements from 16-byte piece to piece
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    q8_u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(x[4 * i + e]);
    st16(p + i * stride, o);
  }
}
__device__ __forceinline__ void store16(uint16_t* p, size_t stride, const float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    q8_u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o[e] = (uint32_t)float_to_bf16_bits(x[8 * i + 2 * e]) | (uint32_t)float_to_bf16_bits(x[8 * i + 2 * e + 1]) << 16;
    st16(p + i * stride, o);
  }
}

// A workgroup takes 16-row tiles of one unit's K or V (blockIdx.z, where both are asked for), a 16-byte piece of codes a thread; what it
// writes has the format of the cache that d_state describes.
// ONCE: the codes are read with non-temporal loads (32 x 4 units of 1090 rows 26.4 -> 23.9 us; 1792 of 1151 325 -> 328, so up to 256 MiB of output).
template <typename T, bool ONCE>
__global__ __launch_bounds__(256) void q8_read_kernel(GkvDims dm, Q8ReadArgs a) {
  constexpr int EPC = Elem<T>::EPC;
  const int step = resolve_step(dm, a.step);
  const int unit = blockIdx.x, lb = quotient(unit, dm.by_hkv), tid = threadIdx.x;
  const bool isK = a.which == 0 || (a.which == 2 && blockIdx.z == 0);
  const SeqState st = load_state(a.d_state, lb);
  const int len = length_before_step(st, step, dm.cap), d = dm.d, pieces = d >> 4;
  const uint8_t* src = (isK ? a.K8 : a.V8) + (size_t)unit * dm.cap * d;
  T* dst = (T*)(isK ? a.K : a.V) + (size_t)unit * dm.cap * d;
  const uint32_t* scales = a.scales + (size_t)unit * dm.cap;
  const int first = (int)blockIdx.y * a.rows, end = min(len, first + a.rows);
  for (int x = tid; x < ((end - first + 15) & ~15) * pieces; x += 256) {
    const int tile = x / (16 * pieces), in = x - tile * 16 * pieces;
    const bool tiled = isK && first + 16 * tile < st.n_tiled;
    const int row = first + 16 * tile + (tiled ? in & 15 : in / pieces), piece = tiled ? in >> 4 : in % pieces;
    if (row >= end) continue;
    const q8_u32x4* from = (const q8_u32x4*)(src + (isK ? q8_k_offset(row, piece, d, st.n_tiled) : (size_t)row * d + piece * 16));
    const q8_u32x4 c = ONCE ? __builtin_nontemporal_load(from) : *from;
    const uint32_t word = scales[row];
    const float scale = isK ? q8_k_scale(word) : q8_v_scale(word);
    float y[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float z[4];
      q8_values(c[i], z);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[4 * i + e] = z[e] * scale;
    }
    if (tiled) store16(dst + (size_t)(row >> 4) * 16 * d + (piece * (16 / EPC)) * 16 * EPC + (row & 15) * EPC, 16 * EPC, y);
    else store16(dst + (size_t)row * d + piece * 16, EPC, y);
  }
}

// ---- decode attention, plain ------------------------------------------------------------------
constexpr int NWG = 4;     // wavefronts per workgroup

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// q . codes of a row of K, for queries that are shrunk (Q8_K_SHRUNK) in their place; `row` and `piece` as q8_k_offset takes them.
__device__ __forceinline__ float dot_codes(const float* qs, const uint8_t* Kh, int row, int d, int n_tiled) {
  float acc = 0.f;
  for (int p = 0; p < d >> 4; ++p) {
    const q8_u32x4 c = ld16(Kh + q8_k_offset(row, p, d, n_tiled));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float z[4];
      q8_values(c[i], z);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = fmaf(qs[16 * p + 4 * i + e], z[e], acc);
    }
  }
  return acc;
}

// One workgroup per unit.  It quantises the new row and writes it first, and attends over what is in the cache then.
// A wavefront takes a whole head: logits a lane per key, outputs a lane per channel.  fp32 throughout.
// Dynamic LDS, per wavefront: float prob[cap + 1]; float qs[d]
template <typename T>
__global__ __launch_bounds__(NWG * 64) void q8_attend_generic_kernel(GkvDims dm, Q8AttendArgs a) {
  const int step = resolve_step(dm, a.step);
  extern __shared__ float smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int unit = blockIdx.x, j = unit % dm.Hkv, lb = unit / dm.Hkv;
  const int d = dm.d, cap = dm.cap, g = dm.g;
  float* prob = smem + (size_t)wave * (cap + 1 + d);
  float* qs = prob + cap + 1;

  const SeqState st = load_state(a.d_state, lb);
  const int len0 = length_before_step(st, step, cap);
  const bool has_new = a.k_new != nullptr && len0 < cap;
  const int n_tot = len0 + (has_new ? 1 : 0);
  uint8_t* Kh = a.K8 + (size_t)unit * cap * d;
  uint8_t* Vh = a.V8 + (size_t)unit * cap * d;
  uint32_t* scales = a.scales + (size_t)unit * cap;

  if (has_new && wave == 0) {
    uint32_t field[2];
    for (int which = 0; which < 2; ++which) {
      const T* src = (const T*)(which ? a.v_new : a.k_new) + (size_t)unit * d;
      uint8_t* dst = (which ? Vh : Kh) + (size_t)len0 * d;                  // (rows are appended row by row)
      float m = 0.f;
      for (int c = lane; c < d; c += 64) m = fmaxf(m, q8_finite_magnitude(Elem<T>::ld(src + c)));
      field[which] = q8_scale_field(wave_max(m));
      const float inv = q8_inverse(field[which]);
      for (int c = lane; c < d; c += 64) dst[c] = (uint8_t)q8_codes(Elem<T>::ld(src + c), 0.f, 0.f, 0.f, inv);
    }
    if (lane == 0) {
      scales[len0] = q8_scale_word(field[0], field[1]);
      a.pos[(size_t)unit * cap + len0] = step;
    }
  }
  __threadfence_block();
  __syncthreads();

  for (int hi = wave; hi < g; hi += NWG) {
    const int head = j * g + hi;
    const size_t row = (size_t)lb * dm.Hq + head;
    const T* qh = (const T*)a.q + row * d;
    for (int c = lane; c < d; c += 64) qs[c] = Elem<T>::ld(qh + c) * Q8_K_SHRUNK;
    wave_sync();
    float mx = GKV_NO_MAX;
    for (int n = lane; n < n_tot; n += 64) {
      const float z = dot_codes(qs, Kh, n, d, st.n_tiled) * q8_k_scale(scales[n]) * Q8_K_GROWN;
      prob[n] = z;
      mx = fmaxf(mx, rounded_product(z, dm.scale_l2_hi));
    }
    mx = wave_max(mx);
    float sm = 0.f;
    for (int n = lane; n < n_tot; n += 64) {
      const float e = exp2f(log2_weight(prob[n], dm.scale_l2_hi, dm.scale_l2_lo, mx));
      prob[n] = e * q8_v_scale(scales[n]);
      sm += e;
    }
    sm = wave_sum(sm);
    wave_sync();
    const PrefixTotal all = prefix_total(a.prefix, row, mx, sm, n_tot > 0);
    const float own = __builtin_amdgcn_exp2f(mx - all.max) * all.inverse;
    T* oh = (T*)a.out + row * d;
    for (int c = lane; c < d; c += 64) {
      float acc = 0.f;
      for (int n = 0; n < n_tot; ++n) acc = fmaf(prob[n], __builtin_amdgcn_cvt_f32_fp8(Vh[(size_t)n * d + c], 0), acc);
      acc = fmaf(prefix_channel(a.prefix, row, d, c, all.max), all.inverse, acc * own);
      Elem<T>::st(oh + c, acc);
    }
    wave_sync();                                           // prob / qs are reused by this wavefront's next head
  }
  if (a.copy_q) {
    __syncthreads();
    const int slot = step % dm.w;
    const size_t nlb = (size_t)dm.L * dm.B;
    for (int x = tid; x < g * d; x += blockDim.x) {
      const size_t at = ((size_t)lb * dm.Hq + j * g) * d + x;
      ((T*)a.qwin)[(size_t)slot * nlb * dm.Hq * d + at] = ((const T*)a.q)[at];
    }
  }
}

// ---- window score, plain ----------------------------------------------------------------------
// As the plain kernel of the other caches: a wavefront per window row, head by head, the rows' largest probabilities
// added up in wavefront order.
// Dynamic LDS, per wavefront: float z[cap]; float rowmax[cap]; float sacc[cap]; float qs[d]
template <typename T>
__global__ void q8_score_generic_kernel(GkvDims dm, ScoreArgs a) {
  const int step = resolve_step(dm, a.step);
  extern __shared__ float smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nw = blockDim.x >> 6;
  const int unit = blockIdx.x, j = unit % dm.Hkv, lb = unit / dm.Hkv;
  const int d = dm.d, cap = dm.cap, g = dm.g, w = dm.w;
  const size_t per_wave = 3 * (size_t)cap + d;
  float* z = smem + wave * per_wave;
  float* rowmax = z + cap;
  float* sacc = rowmax + cap;
  float* qs = sacc + cap;
  const SeqState st = load_state(a.d_state, lb);
  const int l = compression_length(st, step, dm.b, w, cap);
  if (l == 0) return;
  const int c = l - w;
  const uint8_t* Kh = (const uint8_t*)a.K + (size_t)unit * cap * d;
  const uint32_t* scales = a.scales + (size_t)unit * cap;
  for (int n = lane; n < c; n += 64) sacc[n] = 0.f;
  for (int k = wave; k < w; k += nw) {
    const int t_row = step - w + 1 + k, slot = ((t_row % w) + w) % w;
    const int n_vis = c + k + 1;                          // rows [0, c + k] were visible to it
    for (int n = lane; n < c; n += 64) rowmax[n] = 0.f;
    for (int hi = 0; hi < g; ++hi) {
      const T* qh = (const T*)a.qwin + (((size_t)slot * dm.L * dm.B + lb) * dm.Hq + j * g + hi) * d;
      wave_sync();
      for (int ch = lane; ch < d; ch += 64) qs[ch] = Elem<T>::ld(qh + ch) * Q8_K_SHRUNK;
      wave_sync();
      float mx = GKV_NO_MAX;
      for (int n = lane; n < n_vis; n += 64) {
        z[n] = dot_codes(qs, Kh, n, d, st.n_tiled) * q8_k_scale(scales[n]) * Q8_K_GROWN;
        mx = fmaxf(mx, rounded_product(z[n], dm.scale_l2_hi));
      }
      mx = wave_max(mx);
      float sm = 0.f;
      for (int n = lane; n < n_vis; n += 64) {
        z[n] = exp2f(log2_weight(z[n], dm.scale_l2_hi, dm.scale_l2_lo, mx));
        sm += z[n];
      }
      sm = wave_sum(sm);
      for (int n = lane; n < c; n += 64) rowmax[n] = fmaxf(rowmax[n], z[n] / sm);
    }
    for (int n = lane; n < c; n += 64) sacc[n] += rowmax[n];
  }
  __syncthreads();
  float* So = a.S + (size_t)unit * cap;
  for (int n = tid; n < c; n += blockDim.x) {
    float tot = 0.f;
    for (int wv = 0; wv < nw; ++wv) tot += smem[wv * per_wave + 2 * (size_t)cap + n];
    So[n] = tot / (float)w;
  }
}

}  // namespace

template <typename T, int LANES_LOG>
static hipError_t launch_store(const GkvLaunch& ln, const GkvDims& dm, Q8StoreArgs a) {
  // one round of a workgroup: 896 units, prompts of up to 509 rows, bf16, d = 128, cold: 49 us, four of them 54 (non-temporal stores: 49.5
  // where ordinary ones take 53.7; non-temporal loads 63)
  a.rows = (256 >> LANES_LOG) * (sizeof(T) == 4 ? 1 : 2);
  while ((a.n + a.rows - 1) / a.rows > 65535) a.rows *= 2;
  return gkv_launch(ln, q8_store_kernel<T, LANES_LOG>, dim3(dm.L * dm.B * dm.Hkv, (a.n + a.rows - 1) / a.rows), dim3(256), 0, dm, a);
}
template <typename T>
static hipError_t launch_store(const GkvLaunch& ln, const GkvDims& dm, const Q8StoreArgs& a) {
  const int pieces = dm.d / 16;                                      // at most 32, a row being at most 1024 bytes
  return pieces <= 1 ? launch_store<T, 0>(ln, dm, a) : pieces <= 2 ? launch_store<T, 1>(ln, dm, a) : pieces <= 4 ? launch_store<T, 2>(ln, dm, a)
       : pieces <= 8 ? launch_store<T, 3>(ln, dm, a) : pieces <= 16 ? launch_store<T, 4>(ln, dm, a) : launch_store<T, 5>(ln, dm, a);
}
hipError_t gkv_launch_q8_store(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8StoreArgs& a) {
  return dtype == GKV_F32 ? launch_store<float>(ln, dm, a) : launch_store<uint16_t>(ln, dm, a);
}

template <typename T>
static hipError_t launch_read(const GkvLaunch& ln, const GkvDims& dm, Q8ReadArgs a) {
  const int units = dm.L * dm.B * dm.Hkv, caches = a.which == 2 ? 2 : 1;
  a.rows = 128;
  const bool once = (size_t)units * dm.cap * dm.d * sizeof(T) * caches <= (size_t)256 << 20;
  return gkv_launch(ln, once ? q8_read_kernel<T, true> : q8_read_kernel<T, false>, dim3(units, (dm.cap + a.rows - 1) / a.rows, caches),
                    dim3(256), 0, dm, a);
}
hipError_t gkv_launch_q8_read(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8ReadArgs& a) {
  return dtype == GKV_F32 ? launch_read<float>(ln, dm, a) : launch_read<uint16_t>(ln, dm, a);
}

hipError_t gkv_launch_q8_attend_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8AttendArgs& a) {
  const int units = dm.L * dm.B * dm.Hkv;
  const size_t shmem = sizeof(float) * NWG * (size_t)(dm.cap + 1 + dm.d);
  if (dtype == GKV_F32) return gkv_launch(ln, q8_attend_generic_kernel<float>, dim3(units), dim3(NWG * 64), shmem, dm, a);
  return gkv_launch(ln, q8_attend_generic_kernel<uint16_t>, dim3(units), dim3(NWG * 64), shmem, dm, a);
}

hipError_t gkv_launch_q8_score_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const ScoreArgs& a) {
  const int units = dm.L * dm.B * dm.Hkv;
  const size_t per_wave = sizeof(float) * (3 * (size_t)dm.cap + dm.d);
  int nw = (int)(GKV_LDS_LIMIT / per_wave);
  nw = nw < 1 ? 1 : (nw > 4 ? 4 : nw);
  if (dtype == GKV_F32) return gkv_launch(ln, q8_score_generic_kernel<float>, dim3(units), dim3(nw * 64), per_wave * nw, dm, a);
  return gkv_launch(ln, q8_score_generic_kernel<uint16_t>, dim3(units), dim3(nw * 64), per_wave * nw, dm, a);
}
