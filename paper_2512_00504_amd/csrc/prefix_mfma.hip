// Attention over a shared prefix on the matrix cores: bf16 or fp32, head_dim 64 or 128, any number of query rows.
//
// The rows of one (layer, KV head) are its query heads of all sequences that share the prefix: count * g of them, row
// i * g + h.  A workgroup takes up to 4 blocks of 32 rows, a wavefront each, and a piece of the prefix, which passes through LDS in
// tiles of TK keys, brought there once for all of its wavefronts without going through registers, two tiles in turn.
//   S^T[key, row] = K Q^T with products over 32 keys and 32 rows: lane (row = lane % 32, h = lane / 32) gets the keys
//   8 i + 4 h + e of its row, so the softmax stays in the lane but for one exchange with the other half, and they are what the
//   product  O^T[channel, row] += V^T P^T  wants of P in that lane, if V's keys are taken in the same order:
//     bf16: 16x16-transposing reads of LDS give a lane four keys of one channel;  fp32: a lane reads one channel of one key.
//   bf16 rounds P to bf16 (to the nearest, at most 2^-8 of a weight), and l is the sum of the rounded ones: a weight's rounding then moves the result
//   by a part of how far that value is from the mean, and not at all where one key dominates or the values are equal.  Error of the result, whose own
//   rounding makes 1.7e-3: 1.7e-3 to 2.0e-3 with peaked weights (sum of the unrounded ones: 1.9e-3 to 2.4e-3), 2.4e-3 with flat ones.  With the maximum
//   followed at once, not at a distance of up to 8, peaked 1.7e-3 to 1.8e-3, but 5 to 8% more time (28 layers, 64 sequences x 4000 rows 158 -> 169 us).
//   Weights as two bf16 numbers: 1.7e-3 with all of them, but half as many products again (there 158 -> 191, 16 x 8000 92 -> 111, 4 x 8000 71.0 -> 72.3).
// LDS holds a tile's rows as they are, their 16-byte pieces exchanged within the row so that neither kind of read finds two
// rows in the same banks.
// Bound: HBM with few rows (28 layers, 4 KV heads, 32000 rows of d = 128, g = 7: 289 us, 6.3 TB/s).  With several hundred the products
// and the vector unit in turn: 32 keys of 32 rows are 16 products (512 cycles) and 16 x (maximum, fma, exponential, sum, half a
// conversion), about as many; what a wavefront does of one does not overlap with the other, and three of them on a SIMD overlap little
// (64 sequences x 16384 rows, g = 5, 4 layers, 8 KV heads 119 us, 0.72 PFLOP/s; counters: products 48% of the time, vector instructions
// 51%).  Two tiles' logits in turn within a wavefront, which takes the registers of the third: 117 -> 138 us.
#include "gkv_internal.h"

#include <type_traits>

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u32x4 ld16(const void* p) { return *(const u32x4*)p; }

// Maximum or sum over the two halves of a wavefront.
__device__ __forceinline__ float over_halves(float x, bool max) {
  const uint32_t u = __float_as_uint(x);
  const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  const float a = __uint_as_float(y[0]), b = __uint_as_float(y[1]);
  return max ? fmaxf(a, b) : a + b;
}

template <typename T, int D>
struct Geo {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int TK = 32;                   // keys of a tile
  static constexpr int ROW = D * (int)sizeof(T);             // bytes
  static constexpr int CHUNKS = ROW / 16;
  static constexpr int TILE = TK * ROW;                      // bytes of K, and of V
  static constexpr int PIECES = TILE / 1024;                 // of K, and of V
  static constexpr int ROWS_PIECE = 1024 / ROW;
  // what the 16-byte chunks of a row are exchanged by
  __device__ static __forceinline__ int k_swap(int row) { return row & (CHUNKS < 16 ? CHUNKS - 1 : 15); }
  __device__ static __forceinline__ int v_swap(int row) {
    if (F32) return 0;
    return CHUNKS == 8 ? 2 * (row & 1) + 4 * ((row >> 1) & 1) : 4 * (row & 3) + 2 * ((row >> 1) & 1);
  }
};

// A 1 KiB piece from memory to LDS, 16 bytes a lane; `lds` is uniform.  (Written out, because the compiler makes every later read of LDS
// wait for every such request; the wait is the one before the barrier below.  Nothing else in this file uses m0.)
// ONCE: non-temporal.
template <bool ONCE>
__device__ __forceinline__ void to_lds(const char* base, uint32_t offset, uint32_t lds) {
  const uint32_t at = __builtin_amdgcn_readfirstlane(lds);
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(at), "v"(offset), "s"(base) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(at), "v"(offset), "s"(base) : "memory");
}

// What lies at an address of LDS.
template <typename V>
__device__ __forceinline__ V in_lds(uint32_t at) { return *(const __attribute__((address_space(3))) V*)(uintptr_t)at; }

struct KernelArgs {
  PrefixArgs p;
  int32_t L, B, Hq, Hkv, g, tiles, blocks, groups;          // row tiles; blocks of 32 rows per tile at most; (layer, KV head, piece)s
  GkvDivisor by_tiles, by_splits, by_hkv, by_g, by_blocks;
  float scale_hi, scale_lo;
};

// Tiles in turn.  Groups of one wavefront wait for nobody: where LDS has no room for two tiles each (fp32, D = 128: with two groups and a barrier
// 260 us, 14 layers, 2 KV heads, 24000 rows; this 166), or the products are as long as the wait (D = 64: 159 / 146), one has them overlap with the others' loads.
template <typename T, int D, int NK> struct Buffers { static constexpr int N = NK == 4 && Geo<T, D>::F32 ? 1 : 2; };

// NK: groups of a.blocks wavefronts that share the rows and take the tiles in turn (joined through LDS at the end): with one or two
// blocks of rows they make a workgroup of four wavefronts, and the prefix is cut into fewer pieces for the decode kernel to join.
template <typename T, int D, int NK, bool ONCE>
__global__ __launch_bounds__(256, sizeof(T) * D >= 512 && NK > 1 ? 1 : NK > 1 || sizeof(T) == 4 ? 2 : 3) void prefix_mfma_kernel(KernelArgs a) {
  using G = Geo<T, D>;
  constexpr bool ALONE = NK == 4;                            // a group is one wavefront: no barrier (28 layers, 4 sequences x 8000 78.5 -> 73.7 us)
  constexpr int BUFS = Buffers<T, D, NK>::N;
  constexpr int SUB = G::TK / 32, CB = D / 32;
  constexpr uint32_t BUF = NK * 2 * G::TILE;
  extern __shared__ __attribute__((aligned(1024))) char smem[];     // [2][NK][K, V][TILE]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ki = NK == 1 ? 0 : quotient(wave, a.by_blocks), mi = wave - ki * a.blocks;      // group, block of rows
  const int lr = lane & 31, h = lane >> 5;

  // Workgroups go to the XCDs in turn: the row tiles of one piece of the prefix go to the same one, and find it in its L2.
  const int eighth = blockIdx.x >> 3;
  const int round = quotient(eighth, a.by_tiles), tile = eighth - round * a.tiles;
  const int group = round * 8 + (blockIdx.x & 7);
  if (group >= a.groups) return;
  const int unit = quotient(group, a.by_splits), split = group - unit * a.p.splits;
  const int layer = quotient(unit, a.by_hkv), j = unit - layer * a.Hkv;
  const int n0 = split * a.p.split_rows, n1 = min(a.p.rows, n0 + a.p.split_rows);
  const int n_tiles = (n1 - n0 + G::TK - 1) / G::TK, n_rounds = (n_tiles + NK - 1) / NK;
  const char* Kp = (const char*)a.p.K + (((size_t)layer * a.Hkv + j) * a.p.capacity + n0) * G::ROW;
  const char* Vp = (const char*)a.p.V + (((size_t)layer * a.Hkv + j) * a.p.capacity + n0) * G::ROW;

  const int n_rows = a.p.count * a.g;
  const int row = (tile * a.blocks + mi) * 32 + lr, safe = min(row, n_rows - 1);
  const int seq = quotient(safe, a.by_g);
  const size_t head = ((size_t)layer * a.B + a.p.first + seq) * a.Hq + j * a.g + (safe - seq * a.g);
  u32x4 q[D * sizeof(T) / 32];                               // chunks 2 c + h
#pragma unroll
  for (int c = 0; c < D * (int)sizeof(T) / 32; ++c) q[c] = ld16((const char*)a.p.q + head * G::ROW + (2 * c + h) * 16);

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + ki * 2 * G::TILE;
  auto bring = [&](int r) {                                  // the group's tile of round r
    const int first = (r * NK + ki) * G::TK, last = n1 - n0 - 1 - first;
    if (NK > 1 && last < 0) return;
    const char* kt = Kp + (size_t)first * G::ROW;
    const char* vt = Vp + (size_t)first * G::ROW;
    const uint32_t to = lds0 + (BUFS == 2 ? r & 1 : 0) * BUF;
    for (int x = mi; x < G::PIECES; x += a.blocks) {
      const int at = x * G::ROWS_PIECE + lane / G::CHUNKS, chunk = lane % G::CHUNKS;
      const int src = min(at, last);                         // rows behind the end repeat its last one
      to_lds<false>(kt, src * G::ROW + (chunk ^ G::k_swap(at)) * 16, to + x * 1024);
      to_lds<ONCE>(vt, src * G::ROW + (chunk ^ G::v_swap(at)) * 16, to + G::TILE + x * 1024);
    }
  };

  float m = GKV_NO_MAX, l = 0.f;
  f32x16 o[CB];
#pragma unroll
  for (int i = 0; i < CB; ++i) o[i] = f32x16{};
  // This lane's places in a tile: a chunk of K (two of them with h) and a block of channels of V each; the rest of an address is an
  // immediate.
  uint32_t k_at[G::ROW / 32], v_at[CB];
#pragma unroll
  for (int c = 0; c < G::ROW / 32; ++c) k_at[c] = lds0 + lr * G::ROW + ((2 * c + h) ^ G::k_swap(lr)) * 16;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    if constexpr (G::F32) {
      v_at[cb] = lds0 + G::TILE + 4 * h * G::ROW + lr * 4 + cb * 128;
    } else {
      // row 4 h + (lane % 16) / 4 of eight, piece lane % 4 of the 16 channels that its 16 lanes share
      const int at = 4 * h + ((lane & 15) >> 2), chunk = 4 * cb + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      v_at[cb] = lds0 + G::TILE + at * G::ROW + (chunk ^ G::v_swap(at)) * 16 + (lane & 1) * 8;
    }
  }
  // One tile of `there` keys, in the buffer that begins at `buf`; last: it may have fewer than TK.
  auto work = [&](uint32_t buf, int there, auto last) {
    constexpr bool LAST = decltype(last)::value;
    f32x16 s[SUB];
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
      s[i] = f32x16{};
#pragma unroll
      for (int c = 0; c < G::ROW / 32; ++c) {
        const u32x4 k = in_lds<u32x4>(k_at[c] + buf + 32 * i * G::ROW);
        if constexpr (G::F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[e]), __uint_as_float(q[c][e]), s[i], 0, 0, 0);
        } else {
          s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[c]), s[i], 0, 0, 0);
        }
      }
    }
    if constexpr (LAST) {
#pragma unroll
      for (int i = 0; i < SUB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * i + 8 * (e >> 2) + 4 * h + (e & 3) >= there) s[i][e] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int i = 0; i < SUB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[i][e]);
    mx = rounded_product(over_halves(mx, true), a.scale_hi);
    // m follows the largest logit at a distance of up to 8 (weights up to 256): moving it takes a product for every accumulator
    if (__any(mx > m + 8.f)) {
      const float mn = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - mn);
      l *= f;
#pragma unroll
      for (int i = 0; i < CB; ++i) o[i] *= f;
      m = mn;
    }
    // bf16: the scale's lower part is 2^-25 of the exponent, below what its products are rounded by
    if (__any(fabsf(m) >= GKV_HUGE_LOG2 && m != GKV_NO_MAX)) {
#pragma unroll
      for (int i = 0; i < SUB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[i][e] = log2_weight(s[i][e], a.scale_hi, a.scale_lo, m);
    } else {
#pragma unroll
      for (int i = 0; i < SUB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[i][e] = G::F32 ? fmaf(fmaxf(s[i][e], -3.402823466e38f), a.scale_lo, fmaf(s[i][e], a.scale_hi, -m))
                           : fmaf(s[i][e], a.scale_hi, -m);
    }
    float sum = 0.f;
    u32x4 p[G::F32 ? 1 : SUB][2];                            // bf16: the weights of 16 keys each, 8 (2 k) + 4 h + e and 8 (2 k + 1) + 4 h + e
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[i][e] = __builtin_amdgcn_exp2f(s[i][e]);
      if constexpr (G::F32) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += s[i][e];
      } else {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const bf16x2 pair = __builtin_convertvector((f32x2{s[i][2 * x], s[i][2 * x + 1]}), bf16x2);
          p[i][x >> 2][x & 3] = __builtin_bit_cast(uint32_t, pair);
          sum = __builtin_amdgcn_fdot2_f32_bf16(pair, __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
        }
      }
    }
    l += sum;
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
      if constexpr (G::F32) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            float v = in_lds<float>(v_at[cb] + buf + (32 * i + 8 * (e >> 2) + (e & 3)) * G::ROW);
            if (LAST && 32 * i + 8 * (e >> 2) + 4 * h + (e & 3) >= there) v = 0.f;
            o[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[i][e], o[cb], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            s16x4 v[2];
#pragma unroll
            for (int y = 0; y < 2; ++y)
              v[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)(v_at[cb] + buf + (32 * i + 16 * k + 8 * y) * G::ROW));
            u32x2 v0 = __builtin_bit_cast(u32x2, v[0]), v1 = __builtin_bit_cast(u32x2, v[1]);
            if constexpr (LAST) {                            // V behind the end is zero
              const int left = there - (32 * i + 16 * k + 4 * h);
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                v0[y] &= (left > 2 * y ? 0x0000ffffu : 0u) | (left > 2 * y + 1 ? 0xffff0000u : 0u);
                v1[y] &= (left > 8 + 2 * y ? 0x0000ffffu : 0u) | (left > 8 + 2 * y + 1 ? 0xffff0000u : 0u);
              }
            }
            o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, (u32x4{v0[0], v0[1], v1[0], v1[1]})),
                                                            __builtin_bit_cast(bf16x8, p[i][k]), o[cb], 0, 0, 0);
          }
        }
      }
    }
  };
  // The next round's buffer is the one that everybody is through with at the barrier.
  auto there_now = [] {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // this wavefront's share of the tile (and it has read the last one)
    if constexpr (!ALONE) __syncthreads();                   // and everybody's
  };
  if (n_rounds > 0) {
    bring(0);
    uint32_t buf = 0;
    if constexpr (BUFS == 1) {
      for (int r = 0;; ++r) {
        there_now();
        if (r == n_rounds - 1) break;
        work(0, G::TK, std::false_type{});
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        bring(r + 1);
      }
    } else {
      for (int r = 0;; r += 2) {
        there_now();
        if (r == n_rounds - 1) break;
        bring(r + 1);
        work(0, G::TK, std::false_type{});
        there_now();
        buf = BUF;
        if (r + 1 == n_rounds - 1) break;
        buf = 0;
        bring(r + 2);
        work(BUF, G::TK, std::false_type{});
      }
    }
    const int t = (n_rounds - 1) * NK + ki;
    if (NK == 1 || t == n_tiles - 1) work(buf, n1 - n0 - t * G::TK, std::true_type{});
    else if (t < n_tiles - 1) work(buf, G::TK, std::false_type{});
  }
  if constexpr (NK > 1) {
    // the groups' results, lane by lane: 4 x CB pieces of 16 bytes, and (m, l)
    __syncthreads();
    constexpr int PER = 64 * (16 * CB + 2);                  // floats of a wavefront
    float* mine = (float*)smem + (size_t)(wave - a.blocks) * PER;   // (the first group keeps its own)
    if (ki > 0) {
#pragma unroll
      for (int i = 0; i < 4 * CB; ++i)
        *(f32x4*)(mine + (i * 64 + lane) * 4) = f32x4{o[i >> 2][4 * (i & 3)], o[i >> 2][4 * (i & 3) + 1], o[i >> 2][4 * (i & 3) + 2], o[i >> 2][4 * (i & 3) + 3]};
      *(f32x2*)(mine + 64 * 16 * CB + lane * 2) = f32x2{m, l};
    }
    __syncthreads();
    if (ki > 0) return;
#pragma unroll 1
    for (int k = 1; k < NK; ++k) {
      const float* other = (float*)smem + (size_t)((k - 1) * a.blocks + mi) * PER;
      const f32x2 ml = *(const f32x2*)(other + 64 * 16 * CB + lane * 2);
      const float mn = fmaxf(m, ml[0]), f = __builtin_amdgcn_exp2f(m - mn), g = __builtin_amdgcn_exp2f(ml[0] - mn);
      l = l * f + ml[1] * g;
      m = mn;
#pragma unroll
      for (int i = 0; i < 4 * CB; ++i) {
        const f32x4 x = *(const f32x4*)(other + (i * 64 + lane) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i >> 2][4 * (i & 3) + e] = o[i >> 2][4 * (i & 3) + e] * f + x[e] * g;
      }
    }
  }
  if (row >= n_rows) return;
  l = over_halves(l, false);
  const size_t piece = (size_t)split * a.p.heads + head;
  float* to = a.p.o + piece * D;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(f32x4*)(to + 32 * cb + 8 * i + 4 * h) = f32x4{o[cb][4 * i], o[cb][4 * i + 1], o[cb][4 * i + 2], o[cb][4 * i + 3]};
  if (h == 0) {
    a.p.ms[piece] = make_float2(prefix_max(m, l, n1 > n0), l);
    if (split == 0) a.p.n[head] = a.p.splits;
  }
}

template <typename T, int D, int NK, bool ONCE = false>
hipError_t launch(const GkvLaunch& ln, const GkvDims& dm, const PrefixArgs& p, const PrefixPlan& plan) {
  KernelArgs a{p, dm.L, dm.B, dm.Hq, dm.Hkv, dm.g, plan.tiles, plan.blocks, dm.L * dm.Hkv * p.splits,
               gkv_divisor(plan.tiles), gkv_divisor(p.splits), dm.by_hkv, gkv_divisor(dm.g), gkv_divisor(plan.blocks),
               dm.scale_l2_hi, dm.scale_l2_lo};
  const int64_t grid = (int64_t)(a.groups + 7) / 8 * 8 * plan.tiles;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  constexpr size_t shmem = NK * 2 * Buffers<T, D, NK>::N * Geo<T, D>::TILE;
  // the results of all groups but the first: (NK - 1) * blocks wavefronts, four in all at most
  static_assert(shmem <= 131072 && (NK == 1 || shmem >= (NK == 4 ? 3 : 2) * 64 * (D / 2 + 2) * sizeof(float)), "tiles, or the groups' results");
  if (plan.blocks * NK > 4) return hipErrorInvalidConfiguration;
  auto kern = prefix_mfma_kernel<T, D, NK, ONCE>;
  if (shmem > GKV_LDS_LIMIT) {                               // beyond the default per-workgroup limit: opt in (a CU holds 160 KiB)
    const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)shmem);
    if (e != hipSuccess) return e;
  }
  return gkv_launch(ln, kern, dim3((unsigned)grid), dim3(plan.blocks * NK * 64), shmem, a);
}

template <typename T, int D>
hipError_t launch_groups(const GkvLaunch& ln, const GkvDims& dm, const PrefixArgs& p, const PrefixPlan& plan) {
  // V of prefixes that are read once and beyond the 256 MiB memory-side cache is read with non-temporal loads beside K's ordinary ones (bf16, d =
  // 128, 28 layers, 4 KV heads, 8000 rows: 4 sequences 94 us, this 78, K too 86; 16 sequences 107 / 98; 1 layer of 32000 18.8 / 21.0)
  const bool once = plan.tiles == 1 && (int64_t)dm.L * dm.Hkv * p.rows * 2 * Geo<T, D>::ROW > (int64_t)256 << 20;
  if (plan.key_groups == 4) return once ? launch<T, D, 4, true>(ln, dm, p, plan) : launch<T, D, 4>(ln, dm, p, plan);
  if (plan.key_groups == 2) return once ? launch<T, D, 2, true>(ln, dm, p, plan) : launch<T, D, 2>(ln, dm, p, plan);
  return once ? launch<T, D, 1, true>(ln, dm, p, plan) : launch<T, D, 1>(ln, dm, p, plan);
}

}  // namespace

hipError_t gkv_launch_prefix_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PrefixArgs& a, const PrefixPlan& plan) {
  if (dtype == GKV_F32) return dm.d == 64 ? launch_groups<float, 64>(ln, dm, a, plan) : launch_groups<float, 128>(ln, dm, a, plan);
  return dm.d == 64 ? launch_groups<uint16_t, 64>(ln, dm, a, plan) : launch_groups<uint16_t, 128>(ln, dm, a, plan);
}
