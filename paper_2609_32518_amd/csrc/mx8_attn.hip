// Attention of a chunk's quantised queries over the retained rows of a quantised cache (mx8.hpp's format):
// out = sum_m w_m v_m / sum_m w_m, w_m = 2^(q k_m), q holding the softmax scale times log2 e.
//
// QK is v_mfma_scale_f32_32x32x64_f8f6f4 on the bytes as they are, at twice the bf16 rate: keys on the
// M side, the wave's 32 queries on N.  Of the 64 dimensions of one such product, two blocks of 32, lane l
// holds bytes 16 (l / 32) .. + 15 of each block of its row, and the scale of block l / 32.  The
// instruction adds the 16 products of such a group after cutting each below 2^-13 of the largest
// (measured), so a score is off by about 2^-14 of its largest product: for normalised queries and
// keys (products below 16, mostly below 1) less than the probabilities' rounding.  PV is
// v_mfma_f32_32x32x16_bf16: the probabilities, at most 1 at the row's maximum and rounded to bf16 (half a step, a
// relative 2^-8 each, averaged over the keys), times the values, which a tile's load turns into bf16
// exactly.  Sums, maxima and accumulators are fp32.
//
// What bounds it: the matrix cores at a power-limited clock, and beside them LDS and the vector unit.  4680
// queries x 18720 keys x 12 heads take 344-352 us (1.53 PFLOP/s; the matrix instructions alone 239-244, over the bf16
// cache 433-454): per CU the matrix cores are busy 62% of the time, LDS 48%, the vector units 54%.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "attn_schedule.hpp"
#include "kernels.hpp"
#include "mx8.hpp"
#include "seg_table.hpp"

namespace unstep {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kBlockK = kAttnBlockK;
constexpr int kBlockQ = kAttnBlockQ;
constexpr int kRow8 = kHeadDim;               // bytes of a quantised row
constexpr int kRow16 = kHeadDim * 2;          // bytes of a bf16 row
constexpr int kXcds = 8;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
typedef __attribute__((address_space(3))) uint32_t lds_u32_t;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;
typedef __attribute__((address_space(3))) void lds_void_t;

// LDS slots of 16 bytes are XOR-swizzled by the row: 256-byte V rows so that the transposing reads (4 rows x
// 4 slots per half-wave), 128-byte K rows so that the fragment reads (16 rows at one slot), meet no bank twice.
__device__ __forceinline__ int swz16(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }
__device__ __forceinline__ int swz8(int row) { return (row >> 1) & 7; }

// Transposing LDS read: within each 16-lane group, lane i receives element (i & 3) of the 4 x b16 rows
// addressed by lanes 4e + (i >> 2), e = 0..3.
__device__ __forceinline__ u32x2_t lds_read_tr(uint32_t addr) {
  const i16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(uintptr_t)(addr));
  return __builtin_bit_cast(u32x2_t, v);
}

// 16 e4m3 values times one power of two, in bf16
__device__ __forceinline__ void to_bf16(u32x4_t x, float s, u32x4_t (&o)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, false);
    const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, true);
    o[i >> 1][2 * (i & 1)] = __builtin_bit_cast(uint32_t, lo);
    o[i >> 1][2 * (i & 1) + 1] = __builtin_bit_cast(uint32_t, hi);
  }
}

__device__ __forceinline__ i32x8_t join(u32x4_t a, u32x4_t b) {
  return i32x8_t{int(a.x), int(a.y), int(a.z), int(a.w), int(b.x), int(b.y), int(b.z), int(b.w)};
}

// ---- the walk of a 256-query tile over a key range -------------------------------------------------
//
// Work-group: 8 waves of 32 queries.  Waves w and w + 4 share a SIMD and run half a tile apart (groups A
// and B): in each phase one of them multiplies while the other computes the softmax of its tile.  Per
// 64-key tile t:
//   M phase: O^T += V^T(t-1) P^T(t-1) (16 bf16 products) and S^T(t) = K(t) Q^T - m (4 scaled 8-bit ones)
//   V phase: this thread's 16 bytes of K(t+2) and of V(t+1), loaded a tile ago, go to LDS, V as bf16;
//            those of K(t+3) and V(t+2) are loaded; P(t) = exp2(S(t)) in bf16, row sums
// K tiles in LDS: ring of three, K(u) written in V phase u - 2, which for group B is the phase before group
// A's M phase u, and overwriting K(u-3), last read one phase before group A's write.  V tiles: ring of
// three, V(u) written in V phase u - 1 and read in M phase u + 1.  One barrier per phase.
//
// The row sums of a call without a log-sum are four 16x16x32 products a tile, of P^T as it lies in the registers: its
// lanes are 16 columns of 32 rows there, keys 0..7 and 8..15 of queries 0..15 in lanes 0..15 and 32..47, those of
// queries 16..31 in the others, so a row of ones for the first and one for the second pick both sums.  They are the
// sums of the rounded weights, whose rounding then cancels where few keys hold a row (error against float64 of a step
// with scores of tens 0.0022 instead of 0.0024-0.0025), and cost less than 32 additions (359 us instead of 362 for
// 4680 queries x 18720 keys x 12 heads).  A log-sum needs the weights before their rounding, and both take 2.5% longer.
// A product spreads a NaN or infinity of one query to the one 16 on: such a sum sends the work-group through its range
// again, with additions.
//
// The exponent offset m is the row's maximum over the range's first tile and enters the product as its
// accumulator, so a score costs one exp2, one add and half a conversion; a row whose sum passes 2^64
// makes the work-group redo its range with the exact maximum.
constexpr int kRing = 3;
constexpr int kTile8 = kBlockK * kRow8, kTile16 = kBlockK * kRow16, kTileS = kBlockK * kMxBlocks;
constexpr int kLdsV = kRing * kTile8, kLdsS = kLdsV + kRing * kTile16,
              kLdsDump = kLdsS + kRing * kTileS, kLdsBytes = kLdsDump + kRing * kTileS;
// output staging of a finished query tile in the rings: 272-byte rows
constexpr int kOutPitch = kRow16 + 16;
static_assert(kBlockQ * kOutPitch <= kLdsBytes, "the output tile must fit the rings");
// ... and of its partials, half a tile at a time: 528-byte rows, kRowsAtOnce of them by all threads
constexpr int kHalfQ = kBlockQ / 2, kPartRow = kHeadDim * 4, kPartPitch = kPartRow + 16, kRowsAtOnce = kThreads / 32;
static_assert(kHalfQ * kPartPitch <= kLdsBytes && kHalfQ * 2 == kBlockQ, "half the partials must fit the rings");
constexpr int kFetchAhead = 4;               // fragments read ahead of the product that uses them

struct Walk {
  const uint8_t *k8, *v8;                    // this (batch, head)'s rows
  SegTable seg;
  int32_t k_begin, k_end, n;                 // logical key range, its tiles
  int half;
  int lrow;                                  // loader: tile row of this thread
  uint32_t lpiece;                           // ... byte in the row
  uint32_t lshift;                           // ... shift of its block's byte in the row's scale word
  bool lkey;                                 // ... whether it loads the row's K scale word (else V's)
  const uint8_t* lbase;                      // ... and those words
  RowCursor kc, vc;                          // ... cursors of ranges of several runs
  uint32_t wk, wv[2], ws;                    // LDS addresses of what it writes, in slot 0
  uint32_t koff[4], soff;                    // LDS: K fragment halves of d-steps 0, 1; scale words
  uint32_t voff[2][4];                       // LDS: V^T fragment (upper 8 keys, d block)
};

// What a thread has loaded of a K tile and of a V tile, and a scale word: the first of the 8 threads of a row
// holds its K row's, the others their V row's.
struct Stage {
  u32x4_t k, v;
  uint32_t sc;
};

struct Acc {
  f32x16_t o[4];               // O^T: head dims 32 d .. 32 d + 31 x the wave's 32 queries
  f32x16_t s[2];               // S^T of the current tile: keys 32 kb .. 32 kb + 31
  bf16x8_t p[2][2];            // P^T of the previous tile: (key block, 16-key step)
  f32x16_t negm;               // - exponent offset, in every element
  float l;                     // row sum (this lane's half of the keys, or half the sum)
  f32x4_t sum;                 // sums by products: element 0 query lane, 1 query 16 + lane, in lanes 0..15
  bf16x8_t pick;               // ... and the rows that pick them
  float mx;                    // running row max (max-only walk)
};

__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <bool kOneRun>
__device__ __forceinline__ int32_t stage_row(const Walk& w, RowCursor& c, int32_t kt0) {
  int32_t row[1];
  tile_rows<kOneRun, kBlockK, 1, 1>(w.seg, w.k_end, c, kt0, w.lrow, row);
  return row[0];
}

// The loads of K tile tk and V tile tv.
template <bool kOneRun>
__device__ __forceinline__ void load_stage(Stage& st, Walk& w, int32_t tk, int32_t tv) {
  const uint32_t rk = uint32_t(stage_row<kOneRun>(w, w.kc, w.k_begin + tk * kBlockK));
  const uint32_t rv = uint32_t(stage_row<kOneRun>(w, w.vc, w.k_begin + tv * kBlockK));
  st.k = *reinterpret_cast<const u32x4_t*>(w.k8 + (rk * uint32_t(kRow8) + w.lpiece));
  st.v = *reinterpret_cast<const u32x4_t*>(w.v8 + (rv * uint32_t(kRow8) + w.lpiece));
  st.sc = *reinterpret_cast<const uint32_t*>(w.lbase + (w.lkey ? rk : rv) * uint32_t(kMxBlocks));
}
__device__ __forceinline__ void store_k(const Stage& st, const Walk& w, int slot) {
  *reinterpret_cast<lds_u32x4_t*>(uintptr_t(w.wk + slot * kTile8)) = st.k;
  *reinterpret_cast<lds_u32_t*>(uintptr_t(w.ws + slot * kTileS)) = st.sc;
}
__device__ __forceinline__ void store_v(const Stage& st, const Walk& w, int slot) {
  // the first thread of a row takes the V word of the second
  const uint32_t sc = uint32_t(__builtin_amdgcn_update_dpp(0, int(st.sc), 0xe5, 0xf, 0xf, false));   // quad_perm 1,1,2,3
  u32x4_t b[2];
  to_bf16(st.v, mx8_scale((sc >> w.lshift) & 0xffu), b);
#pragma unroll
  for (int i = 0; i < 2; ++i) *reinterpret_cast<lds_u32x4_t*>(uintptr_t(w.wv[i] + slot * kTile16)) = b[i];
}

struct Queries {
  i32x8_t f[2];                // d-steps of 64
  int scale;
};

// Jobs of an M phase: 0..15 the PV product (key block j / 8, 16-key step (j / 4) % 2, d block j % 4),
// 16..19 the QK product (key block (j - 16) / 2, d-step (j - 16) % 2).  Issue order: a QK job after every
// four PV jobs, so that the two steps into one accumulator are apart.
__device__ __forceinline__ constexpr int job_id(int i) { return i % 5 == 4 ? 16 + i / 5 : i - i / 5; }

union Frag {
  u32x4_t r[2];
};

__device__ __forceinline__ Frag fetch(int j, int kslot, int vslot, const Walk& w) {
  Frag f;
  if (j < 16) {
    const uint32_t rel = vslot * kTile16 + (32 * (j >> 3) + 16 * ((j >> 2) & 1)) * kRow16;
    const u32x2_t lo = lds_read_tr(w.voff[0][j & 3] + rel), hi = lds_read_tr(w.voff[1][j & 3] + rel);
    f.r[0] = u32x4_t{lo.x, lo.y, hi.x, hi.y};
  } else {
    const uint32_t rel = kslot * kTile8 + 32 * ((j - 16) >> 1) * kRow8;
    const int st = j & 1;
    f.r[0] = *reinterpret_cast<const lds_u32x4_t*>(uintptr_t(w.koff[2 * st] + rel));
    f.r[1] = *reinterpret_cast<const lds_u32x4_t*>(uintptr_t(w.koff[2 * st + 1] + rel));
  }
  return f;
}

template <bool kZero, bool kSum>
__device__ __forceinline__ void run(Acc& a, int j, const Frag& f, const uint32_t (&ks)[2], const Queries& q) {
  if (j < 16) {
    a.o[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f.r[0]), a.p[j >> 3][(j >> 2) & 1],
                                                         a.o[j & 3], 0, 0, 0);
    if (kSum && (j & 3) == 0)
      a.sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.pick, a.p[j >> 3][(j >> 2) & 1], a.sum, 0, 0, 0);
  } else {
    const int kb = (j - 16) >> 1;
    const f32x16_t zero = {};
    if (j & 1)
      a.s[kb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(f.r[0], f.r[1]), q.f[1], a.s[kb], 0, 0, 2, int(ks[kb]), 2, q.scale);
    else
      a.s[kb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(f.r[0], f.r[1]), q.f[0], kZero ? zero : a.negm, 0, 0, 0,
                                                                int(ks[kb]), 0, q.scale);
  }
}

// kPart 0: all 20 jobs; 1: the QK jobs alone (a walk's first tile); 2: the PV jobs alone (after its last).
template <int kPart>
__device__ __forceinline__ constexpr int jobs() { return kPart == 0 ? 20 : kPart == 1 ? 4 : 16; }
template <int kPart>
__device__ __forceinline__ constexpr int job_at(int i) { return kPart == 0 ? job_id(i) : kPart == 1 ? 16 + i : i; }

template <int kPart, bool kZero, bool kSum, int J>
struct MJob {
  static __device__ __forceinline__ void go(Acc& a, Frag (&f)[jobs<kPart>()], int kslot, int vslot, const uint32_t (&ks)[2],
                                            const Queries& q, const Walk& w) {
    constexpr int kNext = J + kFetchAhead;
    if constexpr (kNext < jobs<kPart>()) f[kNext] = fetch(job_at<kPart>(kNext), kslot, vslot, w);
    run<kZero, kSum>(a, job_at<kPart>(J), f[J], ks, q);
    __builtin_amdgcn_sched_group_barrier(0x008, kSum && job_at<kPart>(J) < 16 && (job_at<kPart>(J) & 3) == 0 ? 2 : 1, 0);
    if constexpr (kNext < jobs<kPart>()) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    if constexpr (J + 1 < jobs<kPart>()) MJob<kPart, kZero, kSum, J + 1>::go(a, f, kslot, vslot, ks, q, w);
  }
};

template <int kPart, bool kZero, bool kSum>
__device__ __forceinline__ void m_phase(Acc& a, int kslot, int vslot, const Queries& q, const Walk& w) {
  Frag f[jobs<kPart>()];
  uint32_t ks[2] = {0, 0};
  if (kPart != 2) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
      ks[kb] = *reinterpret_cast<const lds_u32_t*>(uintptr_t(w.soff + kslot * kTileS + 32 * kb * kMxBlocks)) >> (8 * w.half);
  }
#pragma unroll
  for (int i = 0; i < kFetchAhead; ++i) f[i] = fetch(job_at<kPart>(i), kslot, vslot, w);
  __builtin_amdgcn_sched_group_barrier(0x100, 2 * kFetchAhead + (kPart != 2 ? 2 : 0), 0);
  MJob<kPart, kZero, kSum, 0>::go(a, f, kslot, vslot, ks, q, w);
  // the products stay in this phase: their results are first used after the barrier, past which the compiler
  // would otherwise move them, into the other wave's multiplying phase
  if (kPart != 2) asm volatile("" : "+v"(a.s[0]), "+v"(a.s[1]));
  if (kPart != 1) asm volatile("" : "+v"(a.o[0]), "+v"(a.o[1]), "+v"(a.o[2]), "+v"(a.o[3]));
  if (kPart != 1 && kSum) asm volatile("" : "+v"(a.sum));
}

// V phase of tile t (kSlot = t % 3).  kMode 0: offsets from the first tile; 1: offsets given; 2: row max only.
// The loader's part, in order: what was loaded a tile ago goes to LDS (K(t + 2) into the slot of K(t - 1),
// V(t + 1) into that of V(t - 2)), K(t + 3) and V(t + 2) start; past the range's end it repeats the last
// tile, whose copies nothing reads.  It runs between quarters of the softmax, so that the four waves of a phase do
// not queue at the memory pipelines at once.
template <int kMode, int kSlot, bool kSum, bool kOneRun, bool kIdle, bool kFirst>
__device__ __forceinline__ void v_phase(Acc& a, Stage& st, Walk& w, int32_t t) {
  if (kIdle) {
    store_k(st, w, (kSlot + 2) % kRing);
    store_v(st, w, (kSlot + 1) % kRing);
    load_stage<kOneRun>(st, w, min(t + 3, w.n - 1), min(t + 2, w.n - 1));
    return;
  }
  const int32_t kt0 = w.k_begin + t * kBlockK;
  if (kt0 + kBlockK > w.k_end) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kt0 + 32 * kb + 8 * (i >> 2) + 4 * w.half + (i & 3) >= w.k_end) a.s[kb][i] = -INFINITY;
  }
  if (kMode == 2) {
#pragma unroll
    for (int i = 0; i < 16; ++i) a.mx = fmaxf(a.mx, fmaxf(a.s[0][i], a.s[1][i]));
  }
  if (kMode == 0 && kFirst) {
    float m = a.s[0][0];
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(fmaxf(m, a.s[0][i]), a.s[1][i]);
    m = fmaxf(fmaxf(m, __shfl_xor(m, 32)), -FLT_MAX);   // finite: scores of -infinity weigh nothing
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      a.negm[i] = -m;
      a.s[0][i] -= m;
      a.s[1][i] -= m;
    }
  }
  float acc0 = 0.f, acc1 = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q == 0) store_k(st, w, (kSlot + 2) % kRing);
    if (q == 1) store_v(st, w, (kSlot + 1) % kRing);
    if (q == 2) load_stage<kOneRun>(st, w, min(t + 3, w.n - 1), min(t + 2, w.n - 1));
    if (kMode != 2) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const int kb = q >> 1, i = 8 * (q & 1) + e;
        const float e0 = __builtin_amdgcn_exp2f(a.s[kb][i]);
        const float e1 = __builtin_amdgcn_exp2f(a.s[kb][i + 1]);
        if (!kSum) {
          acc0 += e0;
          acc1 += e1;
        }
        a.p[kb][i >> 3][i & 7] = (__bf16)e0;
        a.p[kb][i >> 3][(i & 7) + 1] = (__bf16)e1;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (!kSum) a.l += acc0 + acc1;
}

template <int kMode, int kSlot, bool kSum, bool kOneRun, bool kIdle, bool kFirst = false>
__device__ __forceinline__ void step(Acc& a, Stage& st, Walk& w, const Queries& q, int32_t t) {
  if (t >= w.n) return;
  if (!kIdle) m_phase<kFirst ? 1 : 0, (kFirst && kMode == 0) || kMode == 2, kSum>(a, kSlot, (kSlot + 2) % kRing, q, w);
  barrier();
  v_phase<kMode, kSlot, kSum, kOneRun, kIdle, kFirst>(a, st, w, t);
  barrier();
}

// A walk's first loads, all at once: K 0 and V 0, K 1, and K 2 and V 1, which stay in st.
struct Start {
  Stage first, second;
};
template <bool kOneRun>
__device__ __forceinline__ void walk_load(Start& b, Stage& st, Walk& w) {
  if (!kOneRun) {
    cursor_at(w.seg, w.k_end, w.k_begin, w.kc);
    w.vc = w.kc;
  }
  load_stage<kOneRun>(b.first, w, 0, 0);
  load_stage<kOneRun>(b.second, w, min(1, w.n - 1), 0);
  load_stage<kOneRun>(st, w, min(2, w.n - 1), min(1, w.n - 1));
}
// Fills the rings' first slots, which every wave has left.
__device__ __forceinline__ void walk_fill(const Start& b, const Walk& w) {
  barrier();
  store_k(b.first, w, 0);
  store_v(b.first, w, 0);
  store_k(b.second, w, 1);
}

// kSum: the row sums by products with rows of ones and zeros, of the rounded weights (mode 0).
template <int kMode, bool kSum, bool kOneRun, bool kIdle>
__device__ __forceinline__ void walk(Acc& a, Stage& st, Walk& w, const Queries& q, int group) {
  const f32x16_t zero = {};
#pragma unroll
  for (int d = 0; d < 4; ++d) a.o[d] = zero;
  a.l = 0.f;
  a.mx = -INFINITY;
  if (kSum) {
    const int row = threadIdx.x & 15;
    const uint32_t one = row < 2 && ((threadIdx.x >> 4) & 1) == row ? 0x3f803f80u : 0u;
    a.pick = __builtin_bit_cast(bf16x8_t, u32x4_t{one, one, one, one});
    a.sum = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  barrier();                                   // the first slots are complete: global phase 0
  if (group == 1) barrier();                   // group B idles in phase 0
  step<kMode, 0, kSum, kOneRun, kIdle, true>(a, st, w, q, 0);
  for (int32_t t0 = 1; t0 < w.n; t0 += kRing) {
    step<kMode, 1, kSum, kOneRun, kIdle>(a, st, w, q, t0);
    step<kMode, 2, kSum, kOneRun, kIdle>(a, st, w, q, t0 + 1);
    step<kMode, 0, kSum, kOneRun, kIdle>(a, st, w, q, t0 + 2);
  }
  if (!kIdle && kMode != 2) m_phase<2, false, kSum>(a, 0, (w.n - 1) % kRing, q, w);
  if (!kIdle && kSum) {
    const int col = threadIdx.x & 31;
    const float low = __shfl(a.sum[0], col & 15), high = __shfl(a.sum[1], col & 15);
    a.l = 0.5f * (col < 16 ? low : high);
  }
  barrier();
  if (group == 0) barrier();                   // group A idles in the last phase
}

// A whole range: offsets from its first tile, and again with the exact maxima where a sum left its range
// (rare, so it has one path, with the loader of any number of runs).
template <bool kIdle>
__device__ __forceinline__ void walk_again(Acc& a, Stage& st, Walk& w, const Queries& q, int group) {
  Start b;
  walk_load<false>(b, st, w);
  walk_fill(b, w);
  walk<2, false, false, kIdle>(a, st, w, q, group);
  const float m = fmaxf(fmaxf(a.mx, __shfl_xor(a.mx, 32)), -FLT_MAX);
#pragma unroll
  for (int i = 0; i < 16; ++i) a.negm[i] = -m;
  walk_load<false>(b, st, w);
  walk_fill(b, w);
  walk<1, false, false, kIdle>(a, st, w, q, group);
}

// kParts: a whole number of work-groups per query tile (a.parts), one segment each.  kSum: as in walk().
template <bool kParts, bool kSum>
__global__ __launch_bounds__(kThreads) void mx8_attn_kernel(Mx8AttnArgs m) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes];
  const AttnArgs& a = m.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = wave >> 2, half = lane >> 5, col = lane & 31;
  const int32_t N = a.N, H = a.H, G = gridDim.x;
  // hardware work-group i runs on XCD i % 8: each XCD gets a contiguous range of logical work-groups
  const int32_t xcd = blockIdx.x % kXcds;
  const int32_t g = xcd * (G / kXcds) + min(xcd, G % kXcds) + blockIdx.x / kXcds;
  int32_t qtiles;
  const Schedule sc = make_schedule(a, &qtiles);

  Walk w;
  w.seg = SegTable{a.seg_l0[1], a.seg_l0[2], a.seg_l0[3], a.seg_row0[0], a.seg_row0[1], a.seg_row0[2], a.seg_row0[3]};
  w.half = half;
  const uint32_t lds0 = uint32_t(uintptr_t((lds_void_t*)lds));
  w.lrow = tid >> 3;
  {
    const int ts = tid & 7;
    w.lpiece = 16 * ts;
    w.lshift = 8 * (ts >> 1);
    w.lkey = ts == 0;
    w.wk = lds0 + w.lrow * kRow8 + (ts ^ swz8(w.lrow)) * 16;
    w.ws = lds0 + (ts == 0 ? kLdsS + w.lrow * kMxBlocks : kLdsDump + 4 * (tid & 63));
#pragma unroll
    for (int i = 0; i < 2; ++i) w.wv[i] = lds0 + kLdsV + w.lrow * kRow16 + ((2 * ts + i) ^ swz16(w.lrow)) * 16;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w.koff[i] = lds0 + col * kRow8 + ((2 * i + half) ^ swz8(col)) * 16;
  w.soff = lds0 + kLdsS + col * kMxBlocks;
  {
    const int e = (lane & 15) >> 2, q = lane & 3, g16 = lane >> 4;
#pragma unroll
    for (int up = 0; up < 2; ++up)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int row = 8 * up + 4 * half + e;
        const int piece = 4 * d + 2 * (g16 & 1) + (q >> 1);
        w.voff[up][d] = lds0 + kLdsV + row * kRow16 + (piece ^ swz16(row)) * 16 + (q & 1) * 8;
      }
  }

  const int64_t u_begin = kParts ? 0 : sc.start(g);
  int64_t u_hi = kParts ? 0 : sc.start(int64_t(g) + 1);
  do {
    const Segment sg = kParts ? part_segment(sc.Tk, a.parts, g) : take_segment(sc, u_begin, u_hi);
    const int32_t t = int32_t(sg.t), qt = t % qtiles, bh = t / qtiles, h = bh % H, b = bh / H;
    const int64_t row0 = int64_t(bh) * a.slots;
    w.k8 = m.k8 + row0 * kRow8;
    w.v8 = m.v8 + row0 * kRow8;
    w.lbase = (w.lkey ? m.k_scale : m.v_scale) + row0 * kMxBlocks;
    w.k_begin = sg.k0 * kBlockK;
    w.k_end = min(a.n_keys, sg.k1 * kBlockK);
    w.n = (w.k_end - w.k_begin + kBlockK - 1) / kBlockK;
    const bool one_run = w.k_end <= w.seg.l1;
    // the first tiles' loads and the queries' are on their way together: a first touch of memory takes about
    // 2 us, which a launch of few tiles would otherwise pay two or three times
    Stage st;
    Start start;
    if (one_run)
      walk_load<true>(start, st, w);
    else
      walk_load<false>(start, st, w);

    const int32_t r = wave * 32 + col, qi = qt * kBlockQ + r;
    Queries q;
    {
      const int64_t qrow = (int64_t(b) * N + min(qi, N - 1)) * H + h;
      const u32x4_t* qp = reinterpret_cast<const u32x4_t*>(m.q8 + qrow * kRow8 + 16 * half);
      q.f[0] = join(qp[0], qp[2]);
      q.f[1] = join(qp[4], qp[6]);
      q.scale = int(*reinterpret_cast<const uint32_t*>(m.q_scale + qrow * kMxBlocks) >> (8 * half));
    }
    walk_fill(start, w);
    Acc acc;
    // a wave whose 32 queries all lie past the chunk's end runs the loads and barriers only
    const bool idle = qt * kBlockQ + wave * 32 >= N;
    if (one_run)
      idle ? walk<0, kSum, true, true>(acc, st, w, q, group) : walk<0, kSum, true, false>(acc, st, w, q, group);
    else
      idle ? walk<0, kSum, false, true>(acc, st, w, q, group) : walk<0, kSum, false, false>(acc, st, w, q, group);
    if (__syncthreads_or(!idle && !(acc.l <= 0x1p64f)))
      idle ? walk_again<true>(acc, st, w, q, group) : walk_again<false>(acc, st, w, q, group);

    const float l_tot = acc.l + __shfl_xor(acc.l, 32), off = -acc.negm[0];
    if (sg.full) {
      // the tile's rows go out through the rings as whole 256-byte rows; rows past the end are staged, not stored
      barrier();
      const float inv = 1.f / l_tot;
      const uint32_t orow = lds0 + uint32_t(r * kOutPitch + 8 * half);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int gg = 0; gg < 4; ++gg) {
          bf16x4_t rr;
#pragma unroll
          for (int e = 0; e < 4; ++e) rr[e] = (__bf16)(acc.o[d][4 * gg + e] * inv);
          *reinterpret_cast<lds_bf16x4_t*>(uintptr_t(orow + (d * 32 + 8 * gg) * 2)) = rr;
        }
      barrier();
      const int pc = tid & 15;
#pragma unroll
      for (int i = 0; i < kBlockQ / (kThreads / 16); ++i) {
        const int rs = (tid >> 4) + (kThreads / 16) * i;
        const int32_t qs = qt * kBlockQ + rs;
        const u32x4_t v = *reinterpret_cast<const lds_u32x4_t*>(uintptr_t(lds0 + uint32_t(rs * kOutPitch + pc * 16)));
        if (qs < N) *reinterpret_cast<u32x4_t*>(a.out + ((int64_t(b) * N + qs) * H + h) * kHeadDim + 8 * pc) = v;
      }
      if (qi < N && a.lse && half == 0) a.lse[(int64_t(b) * H + h) * N + qi] = off * a.scale + logf(l_tot);
    } else {
      const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
      const int64_t prow0 = (int64_t(g) * 2 + sg.slot) * kBlockQ;
      if (qi < N && half == 0) {
        a.part_ml[(prow0 + r) * 2] = l_tot > 0.f ? off : -INFINITY;
        a.part_ml[(prow0 + r) * 2 + 1] = l_tot;
      }
      // partials of a tile with queries of both groups leave through the rings as whole rows, A's and then B's; those
      // of few queries, or of a contiguous split's two ends, from where they are, 32 bytes of 32 rows at a time
      // (us, through the rings and not: 10 heads of [782 queries, 4692 keys] 30.3 and 31.9, 24 of [390, 3120] 27.5 and
      // 28.8, 6 of [1568, 29792] 106.6 and 108.5; 130 of [20, 1600] in a contiguous split 39.3 and 23.6)
      if (!kParts || qt * kBlockQ + kHalfQ >= N) {
        if (qi < N) {
          float* op = a.part_o + (prow0 + r) * kHeadDim + 4 * half;
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int gg = 0; gg < 4; ++gg)
              *reinterpret_cast<float4*>(op + d * 32 + 8 * gg) =
                  make_float4(acc.o[d][4 * gg] * inv, acc.o[d][4 * gg + 1] * inv, acc.o[d][4 * gg + 2] * inv,
                              acc.o[d][4 * gg + 3] * inv);
        }
      } else {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          barrier();
          if (group == part) {
            const uint32_t orow = lds0 + uint32_t((r % kHalfQ) * kPartPitch + 16 * half);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
              for (int gg = 0; gg < 4; ++gg)
                *reinterpret_cast<lds_f32x4_t*>(uintptr_t(orow + (d * 32 + 8 * gg) * 4)) =
                    f32x4_t{acc.o[d][4 * gg] * inv, acc.o[d][4 * gg + 1] * inv, acc.o[d][4 * gg + 2] * inv, acc.o[d][4 * gg + 3] * inv};
          }
          barrier();
          const int pc = tid & 31;
#pragma unroll
          for (int i = 0; i < kHalfQ / kRowsAtOnce; ++i) {
            // every work-group from another row on: the partials lie 256 KB apart, and 256 work-groups that write the
            // same rows at once meet in the same memory channels (35.2 us instead of 33.5 for 8 heads of [1024, 4096])
            const int rs = (tid >> 5) + kRowsAtOnce * ((i + g) % (kHalfQ / kRowsAtOnce)), rt = kHalfQ * part + rs;
            const f32x4_t v = *reinterpret_cast<const lds_f32x4_t*>(uintptr_t(lds0 + uint32_t(rs * kPartPitch + pc * 16)));
            if (qt * kBlockQ + rt < N) *reinterpret_cast<f32x4_t*>(a.part_o + (prow0 + rt) * kHeadDim + 4 * pc) = v;
          }
        }
      }
    }
  } while (!kParts && u_hi > u_begin);
}

}  // namespace

hipError_t launch_mx8_attn(const Mx8AttnArgs& m, hipStream_t stream) {
  if (mx8_few(m.a.B, m.a.H, m.a.N, m.a.n_keys)) {
    const hipError_t e = launch_mx8_attn_few(m, stream);
    if (e != hipSuccess || m.a.N > kMx8FewQueries) return e == hipSuccess ? launch_attn_combine(m.a, stream) : e;
    // few rows leave the chip to the slices: as many as leave each one batch of partials, loaded together
    const int32_t p = m.a.parts;
    return launch_attn_combine(m.a, stream, p > 16 ? 8 : p > 8 ? 4 : p > 4 ? 2 : 1);
  }
  const auto kernel = m.a.parts ? (m.a.lse ? mx8_attn_kernel<true, false> : mx8_attn_kernel<true, true>)
                                : (m.a.lse ? mx8_attn_kernel<false, false> : mx8_attn_kernel<false, true>);
  hipLaunchKernelGGL(kernel, dim3(unsigned(m.a.groups)), dim3(kThreads), 0, stream, m);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? launch_attn_combine(m.a, stream) : e;
}

}  // namespace unstep
