// Internal declarations shared by the C-ABI layer and the kernel files.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gkv.h"
#include "gkv_bench.h"

// x / d = (2 x mul) >> (32 + shift) for 0 <= x < 2^31, with mul = 2^(31 + shift) / d rounded up and
// 2^shift >= d the smallest (mul d exceeds 2^(31 + shift) by less than d <= 2^shift).
struct GkvDivisor { uint32_t mul; uint32_t shift; };
static inline GkvDivisor gkv_divisor(int32_t d) {
  uint32_t shift = 0;
  while ((int64_t)1 << shift < d) ++shift;
  return GkvDivisor{(uint32_t)((((uint64_t)1 << (31 + shift)) + d - 1) / d), shift};
}

// Dimensions every kernel needs, passed by value.
struct GkvDims {
  int32_t L, B, Hq, Hkv, d, g;
  int32_t b, w, s, cap;
  int32_t combine;
  float alpha;
  float scale;   // softmax scale of Eq. 1
  // scale * log2(e) as an unevaluated sum hi + lo: the matrix-core kernels form the exponent of
  // 2 as fma(z, lo, fma(z, hi, -m)), two roundings of a small number and no systematic error
  // from a rounded scale, and the decode and window-score kernels form it the same way
  float scale_l2_hi, scale_l2_lo;
  // Device-side step counter (null: none).  When set, the `step` argument of a call is relative
  // and the kernels use *step_base + step, so recorded launches (HIP graphs) can be replayed.
  const int32_t* step_base;
  GkvDivisor by_hkv;
};

struct GkvProfile;   // event pools, defined in gkv_api.hip

// Decode calls that the library cuts by its own choice use one of this many sets of tickets and partial
// results in the workspace, by the stream they are enqueued on: calls on one stream follow each other,
// calls on different ones may overlap.  A recorded call runs later than what is enqueued on its stream
// now, so each capture counts as a stream of its own.
constexpr int GKV_SPLIT_SETS = 8;
constexpr int GKV_TICKETS = 8;   // tickets per unit and set: one for each wavefront that has outputs (g * d / 256, at most 8)
constexpr int GKV_PREFIX_PIECES = 64;   // that a shared prefix is cut into at most
struct GkvStreamKey { const void* stream; unsigned long long capture; };

struct gkv_ctx {
  gkv_config cfg;
  GkvDims dims;
  int32_t esz;            // bytes per element
  int32_t attend_splits;  // 0 = automatic
  int32_t ws_splits;      // "attend_splits" the workspace was sized for by gkv_workspace_bytes (1 = no partials)
  int32_t ws_auto_splits; // the same for the library's own choice
  const void* split_ws;   // workspace whose tickets gkv_workspace_init of this context zeroed
  int32_t n_split_keys;   // streams that have a set so far; they keep it for the context's life, recorded calls being replayed at any time
  GkvStreamKey split_key[GKV_SPLIT_SETS];
  int32_t attend_tile;    // keys per wavefront iteration of the matrix-core attend kernel: 16 or 32
  int32_t force_generic;
  int32_t attend_waves;   // 0 = automatic
  int32_t fuse_global;    // gkv_evict: as fuse_select (the global score is not a launch of its own)
  int32_t fuse_select;    // gkv_evict: global score at the head of the top-k kernel (default)
  int32_t compact_ppt;    // 16-byte pieces per thread and chunk round of the compaction kernel: 4, 8 or 16
  int32_t reuse_stats;    // window score may reuse the softmax statistics the decode kernel recorded
  bool mfma_shape;        // d == 64 or 128, g <= 16: the matrix-core decode and window-score kernels cover it
  int32_t prefix_rows;    // prefix rows that gkv_prefix_bytes has been asked for
  bool mfma_redundancy;   // bf16, d == 128, g <= 16: the matrix-core redundancy kernel does
  GkvProfile* prof;
  // Host record of which ring slots hold softmax statistics written by the matrix-core decode
  // kernel: stats_step[slot] = decode step whose statistics the slot holds (-1 = none), valid for
  // exactly these buffers.
  int32_t* stats_step;    // [w]
  const void* stats_ws; const void* stats_K; const void* stats_qwin;
  GkvStreamKey stats_key;   // stream of the last decode call
  bool stats_mixed;         // the context has decoded another K cache on another stream
};

// Workspace layout (bytes from the base):
//   [0, 4*GKV_TICKETS*units*sets)   split tickets (int32, self-resetting); sets = GKV_SPLIT_SETS and one for
//                                   "attend_splits", or the latter alone where the library never cuts
//   [.., + 4*L*B)                   compaction tickets
//   [.., + 8*w*L*B*h_q)             softmax statistics ring: per (slot, layer, sequence, query head)
//                                   the running max (log2 units) and the sum of the decode step
//                                   whose q sits in that slot of the window ring
//   [.., + 4*units*splits*g*(d+2) per set)  split-K partials (float)
struct GkvWorkspace {
  int32_t* split_ticket;  // of the call's set, as partials
  int32_t* state_ticket;  // [L*B]: compaction workgroups of a (layer, sequence) that have finished; zero between launches
  float2* stats;
  float* partials;
};

static inline size_t gkv_align256(size_t x) { return (x + 255) & ~size_t(255); }

constexpr size_t GKV_LDS_LIMIT = 65536;
size_t gkv_max_lds_bytes(const gkv_config* cfg);
GkvWorkspace gkv_carve_workspace(const gkv_ctx* ctx, void* base, int split_set = 0);

// Launch record for profiling: the wrappers launch through gkv_launch() below.
struct GkvLaunch {
  gkv_ctx* ctx;
  int kernel_id;
  hipStream_t stream;
  bool continued = false;   // a further launch of the same call: its time counts, the call does not count again
};

// The results over a shared prefix: n[head] pieces for each (layer, sequence, query head), `heads` of them in all, and of each
// piece [piece][head] the unnormalised outputs and the maximum (log2 units) and sum.  o == nullptr: no prefix.
struct PrefixPart { const float* o; const float2* ms; const int32_t* n; int64_t heads; };

// ---- launch wrappers implemented in the kernel files -------------------------------------
struct AttendArgs {
  const void* q; const void* k_new; const void* v_new;
  void* K; void* V; int32_t* pos; int32_t step; void* qwin; const int32_t* d_state; void* out;
  GkvWorkspace ws; int32_t splits; int32_t tile_keys;
  int32_t copy_q;   // 0 when q already is the ring slot of this step
  int32_t write_stats;   // record (max, sum) of every query head's softmax in ws.stats
  int32_t waves;         // wavefronts per workgroup of the matrix-core kernel: 4, 8 or 16
  int32_t split_iters;   // slices per piece (a unit of n slices is cut into ceil(n / split_iters)); 0 = all splits
  PrefixPart prefix;     // joined to the result
};
hipError_t gkv_launch_attend_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const AttendArgs& a);
hipError_t gkv_launch_attend_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const AttendArgs& a);
// LDS of a workgroup of that kernel (bytes)
size_t gkv_attend_mfma_lds(int esz, int d, int g, int waves);

struct ScoreArgs {
  const void* qwin; const void* K; const int32_t* d_state; int32_t step; float* S;
  const float2* stats;   // softmax statistics of the window's decode steps, or null: compute them
  const uint32_t* scales = nullptr;   // of the rows of a K in 8 bits
};
hipError_t gkv_launch_score_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const ScoreArgs& a);
hipError_t gkv_launch_score_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const ScoreArgs& a, int len_max);

hipError_t gkv_launch_global_update(const GkvLaunch& ln, const GkvDims& dm, const float* S,
                                    const float* F_hist, const int32_t* d_state, int32_t step, float* F_out);
hipError_t gkv_launch_select_topk(const GkvLaunch& ln, const GkvDims& dm, const float* F,
                                  const int32_t* d_state, int32_t step, int32_t* keep_idx);
hipError_t gkv_launch_update_and_select(const GkvLaunch& ln, const GkvDims& dm, const float* S, const float* F_hist,
                                        const int32_t* d_state, int32_t step, float* F_out, int32_t* keep_idx);
hipError_t gkv_launch_compact(const GkvLaunch& ln, const GkvDims& dm, int esz, const int32_t* keep_idx,
                              const float* F, void* K, void* V, float* F_hist, int32_t* pos,
                              int32_t* d_state, int32_t step, int32_t* state_ticket);
hipError_t gkv_launch_redundancy(const GkvLaunch& ln, const GkvDims& dm, int dtype, bool mfma, bool f64_mfma, const void* K,
                                 const int32_t* d_state, int32_t step, const float* F, float lambda, float tau,
                                 float eps, int32_t n_recent, float* R_norm, float* F_sel);
hipError_t gkv_launch_pool_scores(const GkvLaunch& ln, const GkvDims& dm, const float* F, const int32_t* d_state,
                                  int32_t step, int32_t kernel, float* F_out);
hipError_t gkv_launch_evicted_positions(const GkvLaunch& ln, const GkvDims& dm, const int32_t* keep_idx,
                                        const int32_t* pos, const int32_t* d_state, int32_t step, int32_t* evicted);

// ---- cache in 8 bits (see e4m3.h) ----------------------------------------------------------
struct Q8StoreArgs {
  const void* k; const void* v; int32_t n, t_first, t0; const int32_t* prompt_len;
  uint8_t* K8; uint8_t* V8; uint32_t* scales; int32_t* pos;
  int32_t rows;                 // of a workgroup (set by the launch)
};
struct Q8ReadArgs {
  const uint8_t* K8; const uint8_t* V8; const uint32_t* scales; const int32_t* d_state; int32_t step;
  void* K; void* V; int32_t which;   // 0: K, 1: V, 2: both
  int32_t rows;                 // of a workgroup (set by the launch)
};
struct Q8AttendArgs {
  const void* q; const void* k_new; const void* v_new;
  uint8_t* K8; uint8_t* V8; uint32_t* scales; int32_t* pos; int32_t step; void* qwin; const int32_t* d_state; void* out;
  PrefixPart prefix;
  GkvWorkspace ws; int32_t splits, split_iters, waves, copy_q, write_stats;   // as in AttendArgs
};
hipError_t gkv_launch_q8_store(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8StoreArgs& a);
hipError_t gkv_launch_q8_read(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8ReadArgs& a);
hipError_t gkv_launch_q8_attend_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8AttendArgs& a);
size_t gkv_q8_attend_mfma_lds(int d, int g, int waves);   // LDS of a workgroup of that kernel (bytes)
hipError_t gkv_launch_q8_attend_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const Q8AttendArgs& a);
hipError_t gkv_launch_q8_score_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const ScoreArgs& a);
hipError_t gkv_launch_q8_compact(const GkvLaunch& ln, const GkvDims& dm, const int32_t* keep_idx, const float* F, void* K8,
                                 void* V8, uint32_t* scales, float* F_hist, int32_t* pos, int32_t* d_state, int32_t step,
                                 int32_t* state_ticket);

// ---- shared prefix ---------------------------------------------------------------------------
struct PrefixArgs {
  const void* q; const void* K; const void* V;
  int32_t rows, capacity, first, count;
  int32_t splits, split_rows;   // pieces, rows of each
  float* o; float2* ms; int32_t* n; int64_t heads;   // as PrefixPart has them
};
// How the matrix-core kernel's rows are dealt out: `tiles` workgroups of up to `blocks` wavefronts of 32 rows per piece.
// key_groups: groups of so many wavefronts in a workgroup, which take its keys in turn.
struct PrefixPlan { int32_t splits, tiles, blocks, key_groups; };
hipError_t gkv_launch_prefix_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PrefixArgs& a, const PrefixPlan& plan);
hipError_t gkv_launch_prefix_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PrefixArgs& a);
// ---- rotary positions, paged caches ----------------------------------------------------------
// freq: radians a position of each pair (64 bits); null: nothing is turned.
struct GkvRotary { const double* freq; int32_t dim, layout; float amplitude; int32_t transposed; };
struct RotateArgs {
  const void* q; const void* k; const void* v;           // null: none of them
  int64_t q_stride, k_stride, v_stride;                  // elements between tokens
  int32_t tokens; const int32_t* positions; int32_t step;   // positions == nullptr: `step` for all (rotate), the row (append)
  GkvRotary rotary;
  void* q_out; void* k_out;                              // [L, tokens, heads, d]
};
struct GkvPages {                                        // K, V [L, n_pages, h_kv, page_rows, d]
  const int32_t* table; int32_t width, page_rows, n_pages;
  GkvDivisor by_rows;
};
struct AppendArgs {
  RotateArgs in;                                         // k_out not used
  const int32_t* start; const int32_t* len;
  GkvPages pages; void* K; void* V;
};
hipError_t gkv_launch_rotate(const GkvLaunch& ln, const GkvDims& dm, int dtype, const RotateArgs& a);
hipError_t gkv_launch_paged_append(const GkvLaunch& ln, const GkvDims& dm, int dtype, const AppendArgs& a);
hipError_t gkv_launch_paged_advance(const GkvLaunch& ln, const GkvDims& dm, int32_t* len, const int32_t* start);

// A unit's ticket has a 128-byte line of its own: its pieces' additions to it come one after the other, and would wait for other units' too.
constexpr int GKV_PAGED_TICKET = 32;
// The matrix-core kernel takes a group's heads 16 at a time.
constexpr int gkv_paged_parts(int g) { return (g + 15) / 16; }
// How a unit is cut, by its own n slices of 16 rows alone: `iters` slices a piece, twice and four times as many from `twice` and `four_times` slices on, not
// more than `soft` pieces; of long_iters slices where those are more.
struct GkvPagedCut {
  int32_t iters, twice, four_times, soft, long_iters;
  constexpr int pieces(int n) const {
    const int by = iters << ((n >= twice) + (n >= four_times));
    const int a = (n + by - 1) / by, b = (n + long_iters - 1) / long_iters;
    return (a < soft ? a : soft) > b ? (a < soft ? a : soft) : b;
  }
  // of any unit of up to n slices
  constexpr int most(int n) const {
    int x = pieces(n);
    if (n >= twice && pieces(twice - 1) > x) x = pieces(twice - 1);
    if (n >= four_times && pieces(four_times - 1) > x) x = pieces(four_times - 1);
    return x;
  }
};
struct PagedAttendArgs {
  const void* q; const void* K; const void* V; GkvPages pages; const int32_t* len; void* out;
  int32_t* ticket; float* partials;                      // [units][parts][GKV_TICKETS][GKV_PAGED_TICKET]; [units][most][g][d + 2]
  int32_t most;                                          // pieces of a unit that there is room for
  int32_t splits;                                        // pieces that the launch has
  GkvPagedCut cut;
  int32_t len_max;
};
hipError_t gkv_launch_paged_attend_generic(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PagedAttendArgs& a, bool aligned);
hipError_t gkv_launch_paged_attend_mfma(const GkvLaunch& ln, const GkvDims& dm, int dtype, const PagedAttendArgs& a);

hipError_t gkv_launch_fill_zero(hipStream_t stream, int32_t* p, size_t n);
hipError_t gkv_launch_add_int(hipStream_t stream, int32_t* p, int32_t delta);

// Event bracketing for profiling (gkv_api.hip).  Returns the events to pass to
// hipExtLaunchKernelGGL, or nulls when profiling is off.
void gkv_profile_events(const GkvLaunch& ln, hipEvent_t* start, hipEvent_t* stop);

// ---- device helpers ------------------------------------------------------------------------
#ifdef __HIPCC__
#include <hip/hip_ext.h>

template <typename... Args, typename F = void (*)(Args...)>
static inline hipError_t gkv_launch(const GkvLaunch& ln, F kernel, dim3 grid, dim3 block,
                                    size_t shmem, Args... args) {
  hipEvent_t e0 = nullptr, e1 = nullptr;
  gkv_profile_events(ln, &e0, &e1);
  if (e0) {
    hipExtLaunchKernelGGL(kernel, grid, block, shmem, ln.stream, e0, e1, 0, args...);
  } else {
    hipLaunchKernelGGL(kernel, grid, block, shmem, ln.stream, args...);
  }
  return hipGetLastError();
}

// x / d for 0 <= x < 2^31.  An integer division is some twenty instructions, at the start of kernels whose first
// requests wait for it.
__device__ __forceinline__ int quotient(int x, GkvDivisor d) { return (int)(__umulhi(2u * (uint32_t)x, d.mul) >> d.shift); }

// The per-(layer, sequence) record of d_state, read with one 16-byte load.
struct SeqState {
  int32_t len, len_step, n_hist, n_tiled;
};
__device__ __forceinline__ SeqState state_record(const int4& v) {
  // the tiled prefix is whole tiles and never reaches past the stored length
  int nt = v.w & ~15;
  const int lim = (v.x > 0 ? v.x : 0) & ~15;
  nt = nt < 0 ? 0 : (nt > lim ? lim : nt);
  return SeqState{v.x, v.y, v.z, nt};
}
__device__ __forceinline__ SeqState load_state(const int32_t* d_state, int lb) {
  return state_record(*(const int4*)(d_state + 4 * (size_t)lb));
}
// Length before decode step `t` (every step since len_step appended one row), kept inside [0, cap].
__device__ __forceinline__ int length_before_step(const SeqState& s, int t, int cap) {
  const int l = s.len + (t - s.len_step);
  return l < 0 ? 0 : (l > cap ? cap : l);
}

// The decode step a kernel works on: its argument, plus the device-side step base if there is one.
__device__ __forceinline__ int resolve_step(const GkvDims& dm, int step) {
  return dm.step_base ? step + *dm.step_base : step;
}

// Whether the compression after decode step `step` applies to this (layer, sequence): its cache
// must exceed the budget, and the observation window must consist of generated tokens, i.e. at
// least w steps were decoded since the cache was loaded or last compacted (a prompt brings keys
// and values but no window queries).  Returns the length l the compression sees, or 0 for "skip".
__device__ __forceinline__ int compression_length(const SeqState& s, int step, int b, int w, int cap) {
  const int l = length_before_step(s, step + 1, cap);
  return (l > b && step + 1 - s.len_step >= w) ? l : 0;
}

// Element offset of (row n, channel c) in one KV head's K block whose first n_tiled rows are in
// tiled format; EPC = elements per 16 bytes.
template <int EPC>
__device__ __forceinline__ int k_elem_offset(int n, int c, int d, int n_tiled) {
  if (n >= n_tiled) return n * d + c;
  return (n >> 4) * 16 * d + (c / EPC) * (16 * EPC) + (n & 15) * EPC + (c % EPC);
}

__device__ __forceinline__ float bf16_bits_to_float(uint16_t b) {
  return __uint_as_float(((uint32_t)b) << 16);
}
__device__ __forceinline__ uint16_t float_to_bf16_bits(float f) {   // round to nearest even
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);   // NaN stays NaN
  u += 0x7fffu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}

template <typename T> struct Elem;
template <> struct Elem<float> {
  static constexpr int EPC = 4;
  __device__ static __forceinline__ float ld(const float* p) { return *p; }
  __device__ static __forceinline__ void st(float* p, float v) { *p = v; }
};
template <> struct Elem<uint16_t> {     // bf16 bit patterns
  static constexpr int EPC = 8;
  __device__ static __forceinline__ float ld(const uint16_t* p) { return bf16_bits_to_float(*p); }
  __device__ static __forceinline__ void st(uint16_t* p, float v) { *p = float_to_bf16_bits(v); }
};

// Running maximum (log2 units) before the first key.
constexpr float GKV_NO_MAX = -3.402823466e38f;
// From this magnitude of a running maximum on, products with the scale are rounded one by one.
constexpr float GKV_HUGE_LOG2 = 0x1p22f;
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
// z * (hi + lo) - m, the exponent of 2 of a logit's weight under the running maximum m = round(max z * hi),
// with two roundings of a small number.  For the largest logit that is what rounding m left over, up to
// |m| * 2^-24, which must not reach the exponential once m is in the millions: there the product is rounded
// as m was (as the plain kernels round theirs), which gives the largest logit exactly 0.  A logit of -inf
// gives -inf (weight 0) whatever the sign of lo, one of +inf or NaN gives NaN, as exp(z - max) does.
__device__ __forceinline__ float log2_weight(float z, float hi, float lo, float m) {
  if (fabsf(m) >= GKV_HUGE_LOG2) return rounded_product(z, hi) - m;
  return fmaf(fmaxf(z, -3.402823466e38f), lo, fmaf(z, hi, -m));
}

// The maximum as a piece of a prefix holds it: -inf where there were keys, all of weight zero.
__device__ __forceinline__ float prefix_max(float m, float sum, bool any_key) {
  return sum == 0.f ? (any_key ? -INFINITY : GKV_NO_MAX) : m;
}
// 1 / total of a softmax's weights.  Nothing attended to: 0; keys whose logits are all -inf: NaN, as softmax gives.
__device__ __forceinline__ float inverse_total(float total, bool any_key) {
  return total == 0.f ? (any_key ? __builtin_nanf("") : 0.f) : 1.f / total;
}
// Pieces of a prefix on their way: of head head0 + h (head0 uniform), channels c .. c + 3, AT_ONCE of them from piece s0 on.
typedef float gkv_f32x4 __attribute__((ext_vector_type(4)));
template <int AT_ONCE>
struct PrefixPieces {
  float2 ms[AT_ONCE];
  gkv_f32x4 o[AT_ONCE];
  __device__ __forceinline__ void request(const PrefixPart& p, size_t head0, int h, int d, int c, int s0, int n) {
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {                      // (without a branch: beyond the last piece that one again)
      const size_t at = (size_t)min(s0 + i, n - 1) * p.heads + head0;
      ms[i] = *(const float2*)((const char*)(p.ms + at) + (uint32_t)(h * 8));
      o[i] = *(const gkv_f32x4*)((const char*)(p.o + at * d) + (uint32_t)((h * d + c) * 4));
    }
  }
  // with a sum o of weighted values, its maximum m (GKV_NO_MAX or more) and sum l.  A piece without weight has an o of 0 and a maximum
  // that is at most GKV_NO_MAX: its factor multiplies zeros.
  __device__ __forceinline__ void join(int s0, int n, float& m, float& l, gkv_f32x4& sum) const {
    float mn = m;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) mn = fmaxf(mn, ms[i].x);
    const float f0 = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= f0;
    sum *= f0;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
      if (s0 + i < n) {                                      // uniform
        const float f = __builtin_amdgcn_exp2f(ms[i].x - mn);
        l += ms[i].y * f;
        sum += o[i] * f;
      }
  }
};
constexpr int GKV_PREFIX_AT_ONCE = 4;
// All n pieces joined with m, l, sum, `first` the first of them if `ready`, the next on their way while some are added up.
// Returns 1 / total.  any_key: the sequence has rows of its own.
__device__ __forceinline__ float prefix_join(const PrefixPart& p, size_t head0, int h, int d, int c, int n, bool ready,
                                             PrefixPieces<GKV_PREFIX_AT_ONCE>& first, float m, float l, gkv_f32x4& sum, bool any_key) {
  constexpr int N = GKV_PREFIX_AT_ONCE;
  if (n > 0) {
    PrefixPieces<N> second;
    if (!ready) first.request(p, head0, h, d, c, 0, n);
    for (int s = 0;; s += 2 * N) {
      if (s + N < n) second.request(p, head0, h, d, c, s + N, n);
      first.join(s, n, m, l, sum);
      if (s + N >= n) break;
      if (s + 2 * N < n) first.request(p, head0, h, d, c, s + 2 * N, n);
      second.join(s + N, n, m, l, sum);
      if (s + 2 * N >= n) break;
    }
    if (l == 0.f && !any_key)                                // seldom
      for (int s = 0; s < n; ++s) any_key |= p.ms[(size_t)s * p.heads + head0 + h].x == -INFINITY;
  }
  return inverse_total(l, any_key);
}
// The same for the plain kernels, one channel a lane: maximum and inverse of the joint total, and the pieces' share of a channel.
struct PrefixTotal { float max, inverse; };
__device__ __forceinline__ PrefixTotal prefix_total(const PrefixPart& p, size_t head, float m, float l, bool any_key) {
  const int n = p.o ? p.n[head] : 0;
  float mx = m, total = 0.f;
  for (int s = 0; s < n; ++s) {
    const float2 ms = p.ms[s * p.heads + head];
    any_key |= ms.x == -INFINITY;
    if (ms.y != 0.f) mx = fmaxf(mx, ms.x);
  }
  total = l * __builtin_amdgcn_exp2f(m - mx);
  for (int s = 0; s < n; ++s) {
    const float2 ms = p.ms[s * p.heads + head];
    if (ms.y != 0.f) total += ms.y * __builtin_amdgcn_exp2f(ms.x - mx);
  }
  return PrefixTotal{mx, inverse_total(total, any_key)};
}
__device__ __forceinline__ float prefix_channel(const PrefixPart& p, size_t head, int d, int c, float mx) {
  const int n = p.o ? p.n[head] : 0;
  float x = 0.f;
  for (int s = 0; s < n; ++s) {
    const size_t at = s * p.heads + head;
    const float2 ms = p.ms[at];
    if (ms.y != 0.f) x = fmaf(p.o[at * d + c], __builtin_amdgcn_exp2f(ms.x - mx), x);
  }
  return x;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
#endif  // __HIPCC__
