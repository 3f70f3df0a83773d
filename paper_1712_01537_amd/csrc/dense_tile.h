// The tile kernel of the dense layers' products on the matrix cores:
//   out[p][q] = sum over r of A(p, r) B(r, q)
// with either operand stored along the reduction ("row" operands: [P][R], [Q][R])
// or across it ("column" operands: [R][P], [R][Q]), so that one kernel serves the
// forward (x, w), the input gradient (dz, w along its columns) and the weight
// gradient (x and dz across their rows) without transposing anything in memory.
//
// A workgroup owns a BM x BN tile, its waves TM x 64 pieces of it, and walks the
// reduction BK at a time through two or more LDS buffers: while one is multiplied the
// next ones land in the others, one barrier a step.  The product is formed transposed
// (the MFMA's first operand is B), so that a lane ends up with four consecutive columns
// of one row.  The epilogue passes the sums through LDS, so that a lane has eight columns
// of a row and reads and writes whole vectors.
//
// bf16 operands whose rows are whole 16-byte vectors (of which what is behind a
// row's end holds zeros) go from memory to LDS directly (buffer_load ... lds; what is
// out of range reads as zero); others, and fp32 ones, pass through registers, where
// fp32 values are split in three bf16 parts (split3.h), so that each is split once
// per tile.  fp32: six MFMAs a product.
//
// LDS layouts, in 16-byte vectors: a row operand keeps its rows (BK values) with
// the vectors of a row rotated by XOR, a column operand keeps [BK][BM or BN] the
// same way and is read by the transposing load (ds_read_b64_tr_b16: lane i of a
// 16-lane group receives element i % 4 of the 8-byte rows read by lanes 4 r + i /
// 4, r = 0..3).  The XORs put the vectors that one pass of a read serves on
// distinct banks.
#pragma once

#include "dense.h"
#include "split3.h"

namespace oc {

struct TileArgs {
  const void *a, *b;
  int64_t P, R;
  int32_t Q;                // columns of the product (2 n with glu)
  int64_t lda, ldb;         // elements from row to row of A and B in memory
  int32_t half;             // first column of the other half in B with glu
  int32_t ntm, ntn;         // tiles
  // The first `whole` tiles have a workgroup each.  The rest are shared, in
  // `members` runs of `run` tiles (member g has tiles whole + g + members j, those
  // there are): the steps of a run, `steps` a tile, are dealt out to `classes`
  // workgroups, `share` each (at most a tile's, so of at most two tiles).  So the
  // members' workgroups of one class walk the same range of the reduction, next to
  // each other in the order of the tiles, and share what they read in L2.  Sums of
  // a workgroup (class c, member g) that are not all of its tile j's go to
  // part[(c + j) members + g][BM][BN].
  int32_t whole, members, run, classes;
  int64_t steps, share;
  float* part;
  Epi epi;
};

// Tile shapes, by type; see gemm() for which is taken.
enum TileShape { TILE_LARGE, TILE_TWO, TILE_MEDIUM, TILE_SMALL, TILE_SHAPES };
struct TileInfo {
  int bm, bn, threads, bk;
  int nb;  // LDS buffers of BK terms (direct operands; others take two)
};
template <typename T>
constexpr TileInfo tile_info(int shape) {
  constexpr bool f32 = sizeof(T) == 4;
  return shape == TILE_LARGE    ? (f32 ? TileInfo{256, 128, 512, 32, 2} : TileInfo{256, 256, 512, 64, 2})
         : shape == TILE_TWO    ? (f32 ? TileInfo{128, 64, 256, 32, 2} : TileInfo{256, 128, 256, 32, 2})
         : shape == TILE_MEDIUM ? (f32 ? TileInfo{128, 128, 512, 32, 2} : TileInfo{128, 128, 256, 64, 2})
                                : (f32 ? TileInfo{64, 64, 256, 32, 2} : TileInfo{64, 64, 256, 64, 2});
}

// Enqueue the tile kernel for fp32 or bf16 operands (dense_f32.hip, dense_bf16.hip).
void tile_f32(int shape, bool a_rs, bool b_rs, bool main, const TileArgs& t, hipStream_t s);
void tile_bf16(int shape, bool a_rs, bool b_rs, bool direct, bool main, const TileArgs& t,
               hipStream_t s);
void tiles2_f32(int shape, const TileArgs& dx, const TileArgs& dw, bool swapped, hipStream_t s);
void tiles2_bf16(int shape, bool direct, const TileArgs& dx, const TileArgs& dw, bool swapped,
                 hipStream_t s);

// --- device side ---------------------------------------------------------

typedef __attribute__((address_space(3))) void* dt_lptr;
typedef short dt_v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) dt_v4s dt_lds_v4s;
typedef int32_t dt_sv4 __attribute__((ext_vector_type(4)));

// The rotation of row `row`'s vectors in a row operand (CK vectors a row).
template <int CK>
__device__ __forceinline__ int row_xor(int row) {
  return CK == 8 ? (row >> 1) & 7 : (4 - (row >> 2)) & 3;
}
// The rotation of line k's vectors in a column operand (CR vectors a line).
template <int CR>
__device__ __forceinline__ int col_xor(int k) {
  return CR >= 16 ? 2 * ((k & 3) | ((k >> 3) & 1) << 2)
                  : 2 * (((k >> 1) & 1) | ((k >> 3) & 1) << 1);
}

// Workgroup barrier that orders LDS accesses only.
__device__ __forceinline__ void dt_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// At most N of this wave's vector memory operations are outstanding (they complete
// in order; the compiler adds none of its own to the loop that counts them, which
// must not spill).
template <int N>
__device__ __forceinline__ void dt_wait_vm() {
  static_assert(N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// s3_split8 with the differences as subtractions: the dot products that it forms
// them with are one instruction where these are two, but issue at a quarter of the
// rate (a step of the large tile alone on its CU: 2.0 us with them, 1.7 without).
__device__ __forceinline__ Split8 dt_split8(const s3_v4f& x, const s3_v4f& y) {
  Split8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = (i < 2 ? x : y)[2 * (i & 1)] * kSplitUp;
    float b = (i < 2 ? x : y)[2 * (i & 1) + 1] * kSplitUp;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint32_t h = s3_round2(a, b);
      r.p[k][i] = h;
      a -= __builtin_bit_cast(float, h << 16);
      b -= __builtin_bit_cast(float, h & 0xffff0000u);
    }
  }
  return r;
}

// Memory to LDS: lane i's 16 bytes at byte `off` of the resource land at lds +
// 16 i; an offset past the resource's end stores zeros.
__device__ __forceinline__ void dt_lds_load16(dt_sv4 rsrc, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds),
               "v"(off), "s"(rsrc)
               : "memory", "m0");
}
constexpr uint32_t kPastEnd = 0x80000000u;  // of any resource
__device__ __forceinline__ dt_sv4 dt_rsrc(const char* p, int64_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  const int64_t most = 0x7ffffff0;  // below kPastEnd; an end before p leaves nothing in range
  return dt_sv4{(int32_t)(uint32_t)a, (int32_t)((a >> 32) & 0xffffu),
                (int32_t)(bytes < 0 ? 0 : bytes < most ? bytes : most), 0x00020000};
}

// Terms r .. r + 3 of row or column `at` of an fp32 operand (RS: stored across the
// reduction); those from `end` on read as zero.
template <bool RS>
__device__ __forceinline__ s3_v4f dt_terms(const float* m, int64_t ld, int64_t at, int64_t r,
                                           int64_t end) {
  if (!RS && r + 4 <= end) return *(const d_v4f_any*)(m + at * ld + r);
  s3_v4f v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = r + e < end ? m[RS ? (r + e) * ld + at : at * ld + r + e] : 0.f;
  return v;
}

// Row and column of tile i: groups of eight rows of tiles, so that the tiles an XCD
// works on at a time share operands in its L2.
struct TilePos {
  int m, n;
};
__host__ __device__ __forceinline__ TilePos tile_pos(int ntm, int ntn, uint32_t i) {
  const uint32_t group = i / (8 * ntn), j = i - group * 8 * ntn;
  const uint32_t left = ntm - group * 8, rows = left < 8 ? left : 8;
  const uint32_t n = j / rows;
  return TilePos{(int)(group * 8 + (j - n * rows)), (int)n};
}

// LDS of a workgroup, in 16-byte vectors: the operands' buffers, or the epilogue's
// pieces, ROWS rows of 64 sums per wave at a time.
template <typename T, int BM, int BN, int WGM, int BK, int BUFS, bool DIRECT>
constexpr int tile_lds() {
  constexpr int TM = BM / WGM, STAGE = (sizeof(T) == 4 ? 3 : 1) * (BM + BN) * (BK / 8);
  constexpr int ROWS = TM < 64 ? TM : 64, EPI = WGM * (BN / 64) * ROWS * 16;
  constexpr int OPS = (DIRECT ? BUFS : 2) * STAGE;
  return OPS > EPI ? OPS : EPI;
}

// The work of workgroup `block` of the `blocks` of a product.
template <typename T, int BM, int BN, int WGM, int BK, int BUFS, bool ARS, bool BRS, bool GLU,
          bool DIRECT, bool DZ>
__device__ __forceinline__ void tile_run(const TileArgs& t, uint32_t block, uint32_t blocks,
                                         s3_v4u* lds) {
  constexpr bool F32 = sizeof(T) == 4;
  static_assert(!(F32 && DIRECT), "fp32 operands are split in registers");
  constexpr int PARTS = F32 ? 3 : 1;
  constexpr int WGN = BN / 64, NTHR = 64 * WGM * WGN;
  constexpr int TM = BM / WGM, TN = 64, MI = TM / 16, NI = 4;
  constexpr int CK = BK / 8, CA = BM * CK, CB = BN * CK;
  constexpr int ITA = CA / NTHR, ITB = CB / NTHR, IT = ITA + ITB;
  static_assert(CA % NTHR == 0 && CB % NTHR == 0 && TM % 16 == 0, "whole vectors per thread");
  static_assert(!(GLU || DZ) || (!ARS && BRS), "the forward's layout");
  constexpr int STAGE = PARTS * (CA + CB), NB = DIRECT ? BUFS : 2;
  constexpr int ROWS = TM < 64 ? TM : 64;  // of the epilogue's pieces

  const int n = t.epi.n;

  // this workgroup's tile, or its shares of two
  const bool shared = block >= (uint32_t)t.whole;
  const uint32_t w = shared ? xcd_order(block - t.whole, blocks - t.whole)
                            : xcd_order(block, t.whole);
  const uint32_t cls = shared ? w / t.members : 0, member = w - cls * t.members;
  int64_t unit = cls * t.share;
  const int64_t all = shared ? t.steps * t.run : t.steps;
  const int64_t unit_end = !shared || unit + t.share > all ? all : unit + t.share;
#pragma unroll 1
  while (unit < unit_end) {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // nothing of a tile is worked out ahead of the loop
  const int lane = tid & 63, li = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const uint32_t nth = (uint32_t)(unit / t.steps);  // of the run
  const int64_t s0 = unit - nth * t.steps;
  const int64_t s1 = s0 + (unit_end - unit) < t.steps ? s0 + (unit_end - unit) : t.steps;
  unit += s1 - s0;
  const bool partial = s1 - s0 < t.steps;
  const uint32_t tile = shared ? t.whole + member + nth * t.members : w;
  if (tile >= (uint32_t)(t.ntm * t.ntn)) break;  // this member's run is shorter
  const TilePos pos = tile_pos(t.ntm, t.ntn, tile);
  const int64_t p0 = (int64_t)pos.m * BM;
  const int q0 = pos.n * (GLU ? BN / 2 : BN);  // first output column
  const int64_t r0 = s0 * BK;
  const int64_t r1 = s1 * BK < t.R ? s1 * BK : t.R;
  const int nk = (int)(s1 - s0);

  // This thread's vectors: element offset from the operand's tile corner, how
  // many of the eight values exist (rows past the end repeat the last one, whose
  // results are dropped), and the vector's place along the reduction.
  uint32_t off[IT];
  int cnt[IT], kof[IT];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const bool isa = i < ITA;
    const int c = (isa ? i : i - ITA) * NTHR + tid;
    if (isa ? !ARS : !BRS) {
      const int row = c / CK;
      kof[i] = ((c % CK) ^ row_xor<CK>(row)) * 8;
      const int64_t lim = isa ? t.P - p0 : (int64_t)t.Q - q0;
      const int rr = row < lim ? row : (int)lim - 1;
      off[i] = (uint32_t)rr * (uint32_t)(isa ? t.lda : t.ldb) + kof[i];
      cnt[i] = 8;
    } else {
      constexpr int CRA = BM / 8, CRB = BN / 8;
      const int cr = isa ? CRA : CRB;
      kof[i] = c / cr;
      const int x = isa ? col_xor<CRA>(kof[i]) : col_xor<CRB>(kof[i]);
      const int col = ((c % cr) ^ x) * 8;
      int lim, e, add = 0;  // of the columns' range, the column, what is added to it
      if (isa) {
        lim = (int)(t.P - p0 < BM ? t.P - p0 : BM), e = col;
      } else if (GLU) {
        lim = n - q0;
        e = col / TN * (TN / 2) + col % (TN / 2);
        add = col % TN >= TN / 2 ? t.half : 0;
      } else {
        lim = t.Q - q0, e = col;
      }
      cnt[i] = lim - e < 0 ? 0 : lim - e < 8 ? lim - e : 8;
      const uint32_t ld = (uint32_t)(isa ? t.lda : t.ldb);
      off[i] = (uint32_t)kof[i] * ld + (cnt[i] > 0 ? e + add : 0);
    }
  }
  const char* const abase = (const char*)t.a + (ARS ? r0 * t.lda + p0 : p0 * t.lda + r0) * sizeof(T);
  const char* const bbase =
      (const char*)t.b + (BRS ? r0 * t.ldb + q0 : q0 * t.ldb + r0) * sizeof(T);
  const int64_t astep = (ARS ? BK * t.lda : BK) * sizeof(T);
  const int64_t bstep = (BRS ? BK * t.ldb : BK) * sizeof(T);
  const int64_t asize = (ARS ? t.R : t.P) * t.lda, bsize = (BRS ? t.R : (int64_t)t.Q) * t.ldb;

  // Direct: start the loads of vectors from .. to of step ks into the buffer at vector
  // `buf`.  (Of steps past the last: nothing is read, zeros are stored; so a wave's
  // count of loads is known.)
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(dt_lptr)lds);
  auto issue = [&](int ks, int buf, int from, int to) __attribute__((always_inline)) {
    const char* pa = abase + ks * astep;
    const char* pb = bbase + ks * bstep;
    const dt_sv4 ra = dt_rsrc(pa, (const char*)t.a + asize * (int64_t)sizeof(T) - pa);
    const dt_sv4 rb = dt_rsrc(pb, (const char*)t.b + bsize * (int64_t)sizeof(T) - pb);
    const int64_t left = r1 - r0 - (int64_t)ks * BK;
#pragma unroll
    for (int i = from; i < to; ++i) {
      const bool isa = i < ITA;
      const uint32_t o = cnt[i] > 0 && kof[i] < left ? off[i] * 2 : kPastEnd;
      const uint32_t at = (isa ? i : i - ITA) * NTHR + wave * 64 + (isa ? 0 : CA);
      dt_lds_load16(isa ? ra : rb, o, lds0 + (buf + at) * 16);
    }
  };

  // Through registers: load vectors from .. to of step ks, then split and store them
  // to the buffer at vector `buf`.  The first `plain` steps read whole vectors: what
  // such a vector holds of a column past the end goes to sums that are dropped, and lies
  // inside the operand as long as its last lines are not read or the tile has no such
  // column.
  s3_v4u reg[IT][F32 ? 2 : 1];
  int plain = 0;
  if constexpr (!DIRECT) {
    bool whole = true;
#pragma unroll
    for (int i = 0; i < IT; ++i) whole = whole && (cnt[i] == 8 || cnt[i] == 0);
    whole = __syncthreads_and(whole);
    const int64_t la = ARS ? (t.lda + 7) / t.lda : 0, lb = BRS ? (t.ldb + 7) / t.ldb : 0;
    const int64_t end = t.R - (la > lb ? la : lb);  // lines that a vector leaves room behind
    plain = (int)(((whole || r1 < end ? r1 : end) - r0) / BK);
  }
  auto fetch_plain = [&](int ks, int from, int to) __attribute__((always_inline)) {
    const char* pa = abase + ks * astep;
    const char* pb = bbase + ks * bstep;
#pragma unroll
    for (int i = from; i < to; ++i) {
      const char* p = (i < ITA ? pa : pb) + (uint32_t)(off[i] * sizeof(T));
      if (F32) {
        reg[i][0] = __builtin_bit_cast(s3_v4u, *(const d_v4f_any*)p);
        reg[i][F32] = __builtin_bit_cast(s3_v4u, *(const d_v4f_any*)(p + 16));
      } else {
        reg[i][0] = *(const d_v4u_any*)p;
      }
    }
  };
  // The other steps: what lies behind a vector's end is set to zero, and vectors at
  // the operand's end are read as its last eight elements and moved down.
  auto fetch_tail = [&](int ks) __attribute__((always_inline)) {
    const char* pa = abase + ks * astep;
    const char* pb = bbase + ks * bstep;
    const int64_t left = r1 - r0 - (int64_t)ks * BK;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const bool isa = i < ITA;
      const int64_t size = isa ? asize : bsize;
      const int64_t at = ((isa ? pa - (const char*)t.a : pb - (const char*)t.b) / (int)sizeof(T)) +
                         off[i];
      const int64_t l = left - kof[i];
      int m = l <= 0 ? 0 : cnt[i];
      if ((isa ? !ARS : !BRS) && l < m) m = l < 0 ? 0 : (int)l;
      const void* base = isa ? t.a : t.b;
      float v[8];
      if (size >= 8) {
        const int64_t from = at + 8 <= size ? at : size - 8;
        const int by = m > 0 ? (int)(at - from) : 0;
        load8(base, !F32, from, v);
        if (__any(by > 0)) {
#pragma unroll
          for (int h = 4; h > 0; h >>= 1)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = by & h ? v[k + h < 8 ? k + h : k] : v[k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < m ? load1(base, !F32, at + k) : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < m ? v[k] : 0.f;
      if (F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          reg[i][0][k] = __builtin_bit_cast(uint32_t, v[k]);
          reg[i][F32][k] = __builtin_bit_cast(uint32_t, v[4 + k]);
        }
      } else {
        reg[i][0] = s3_v4u{bf_pair(v[0], v[1]), bf_pair(v[2], v[3]), bf_pair(v[4], v[5]),
                           bf_pair(v[6], v[7])};
      }
    }
  };
  auto fetch = [&](int ks) __attribute__((always_inline)) {
    if (ks < plain) fetch_plain(ks, 0, IT);
    else fetch_tail(ks);
  };
  auto stash = [&](int buf, int from, int to) __attribute__((always_inline)) {
#pragma unroll
    for (int i = from; i < to; ++i) {
      const bool isa = i < ITA;
      const int c = buf + (isa ? i : i - ITA) * NTHR + tid + (isa ? 0 : PARTS * CA);
      if constexpr (F32) {
        const Split8 p = dt_split8(__builtin_bit_cast(s3_v4f, reg[i][0]),
                                   __builtin_bit_cast(s3_v4f, reg[i][F32]));
#pragma unroll
        for (int k = 0; k < 3; ++k) lds[c + k * (isa ? CA : CB)] = p.p[k];
      } else {
        lds[c] = reg[i][0];
      }
    }
  };

  s3_v4f acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = s3_v4f{0.f, 0.f, 0.f, 0.f};

  // Operands of one MFMA: eight consecutive terms of the reduction for row (A) or
  // column (B) li of the fragment, terms 8 q .. of the 32 of sub-step kk.
  auto tr = [&](const char* p, int line) __attribute__((always_inline)) {
    const auto* a = (const __attribute__((address_space(3))) char*)p;
    const s3_v2u lo = __builtin_bit_cast(s3_v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((dt_lds_v4s*)a));
    const s3_v2u hi = __builtin_bit_cast(
        s3_v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((dt_lds_v4s*)(a + 4 * line)));
    return s3_v4u{lo[0], lo[1], hi[0], hi[1]};
  };
  auto frag_a = [&](int buf, int part, int kk, int mi) __attribute__((always_inline)) {
    const s3_v4u* base = lds + buf + part * CA;
    if constexpr (!ARS) {
      const int row = wm * TM + mi * 16 + li;
      return base[row * CK + ((kk * 4 + q) ^ row_xor<CK>(li))];
    } else {
      constexpr int CR = BM / 8;
      const int k = kk * 32 + q * 8 + (li >> 2);
      const int c = wm * (TM / 8) + mi * 2 + ((li & 3) >> 1);
      return tr((const char*)(base + k * CR + (c ^ col_xor<CR>(k))) + (li & 1) * 8,
                CR * 16);
    }
  };
  auto frag_b = [&](int buf, int part, int kk, int ni) __attribute__((always_inline)) {
    const s3_v4u* base = lds + buf + PARTS * CA + part * CB;
    if constexpr (!BRS) {
      const int row = wn * TN + ni * 16 + li;
      return base[row * CK + ((kk * 4 + q) ^ row_xor<CK>(li))];
    } else {
      constexpr int CR = BN / 8;
      const int k = kk * 32 + q * 8 + (li >> 2);
      const int c = wn * (TN / 8) + ni * 2 + ((li & 3) >> 1);
      return tr((const char*)(base + k * CR + (c ^ col_xor<CR>(k))) + (li & 1) * 8, CR * 16);
    }
  };

  // A step is NU units: MI row fragments for each of the BK / 32 sub-steps.  A
  // unit's row fragment is read AD units ahead and a sub-step's column fragments
  // ahead of its first unit.  Ahead of the last AD units all of this step's
  // fragments are in registers: there the workgroup meets, and what follows reads
  // the next step's buffer and refills this one's, while the matrix cores still
  // have AD units to do.
  constexpr int KK = BK / 32, NU = KK * MI, AD = DIRECT && MI >= 4 ? 3 : 1;
  static_assert(AD <= MI, "a sub-step's columns are read within the one before it");
  s3_v4u a[AD + 1][PARTS], b[2][NI][PARTS];
  auto read_a = [&](s3_v4u(&f)[PARTS], int s, int u) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < PARTS; ++k) f[k] = frag_a(s, k, u / MI, u % MI);
  };
  auto read_b = [&](s3_v4u(&f)[NI][PARTS], int s, int kk) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int k = 0; k < PARTS; ++k) f[j][k] = frag_b(s, k, kk, j);
  };

  // The large fp32 tile's step: four units of two row and two column fragments, 24
  // MFMAs and six LDS reads each, every read into registers that the unit before has
  // done with.  (Row by row, a step's twelve column reads of every wave came at once
  // after the barrier, and took 960 cycles of the LDS: 2.33 us a step.)
  constexpr bool QUAD = F32 && MI == 4;

  if constexpr (QUAD) {
    s3_v4u fa[4][PARTS], fb[4][PARTS];
    auto read2a = [&](int s, int i) __attribute__((always_inline)) {
      read_a(fa[i], s, i);
      read_a(fa[i + 1], s, i + 1);
    };
    auto read2b = [&](int s, int j) __attribute__((always_inline)) {
#pragma unroll
      for (int x = j; x < j + 2; ++x)
#pragma unroll
        for (int k = 0; k < PARTS; ++k) fb[x][k] = frag_b(s, k, 0, x);
    };
    auto multiply = [&](int i, int j) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 6; ++x)
#pragma unroll
        for (int m = 0; m < 4; ++m)
          acc[i + m / 2][j + m % 2] =
              s3_product(x, fb[j + m % 2], fa[i + m / 2], acc[i + m / 2][j + m % 2]);
#pragma unroll
      for (int x = 0; x < 24; ++x) {  // splits and LDS accesses in the shadow of the MFMAs
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    static_assert(IT == 3, "a vector for each of the units ahead of the barrier");
    // Step ks.  ahead(i): load vector i of step ks + 2, right behind its place's use.
    auto step = [&](int s, int nx, auto&& ahead) __attribute__((always_inline)) {
      read2b(s, 2);
      stash(nx, 0, 1);
      ahead(0);
      multiply(0, 0);
      read2a(s, 2);
      stash(nx, 1, 2);
      ahead(1);
      multiply(0, 2);
      stash(nx, 2, 3);
      ahead(2);
      multiply(2, 0);
      dt_barrier();  // step ks + 1 is in LDS, and step ks in registers
      read2a(nx, 0);  // (of the last step: what lies there, never used)
      read2b(nx, 0);
      multiply(2, 2);
    };
    fetch(0);
    stash(0, 0, IT);
    dt_barrier();
    if (nk > 1) fetch(1);
    read2a(0, 0);
    read2b(0, 0);
    int ks = 0;
    // no branch between the loads, so that each is waited for by itself
    for (; ks + 2 < plain; ++ks)
      step((ks & 1) * STAGE, (~ks & 1) * STAGE, [&](int i) __attribute__((always_inline)) { fetch_plain(ks + 2, i, i + 1); });
#pragma unroll 1
    for (; ks < nk; ++ks) {
      step((ks & 1) * STAGE, (~ks & 1) * STAGE, [](int) {});
      if (ks + 2 < nk) fetch(ks + 2);
    }
  } else {
  // Loads are started LP a unit from the barrier on, so that no wave stands still
  // while a whole step's worth of them finds its way into the memory pipeline (input
  // gradient, 256x256 tiles: 1493 TFLOP/s, all at once 1430).  The small tile's few
  // steps wait for their arrival instead (alone on a CU 0.48 us a step, two a unit 0.6).
  constexpr int LP = TM >= 128 ? 2 : MI >= 4 ? 4 : IT;
  constexpr int AHEAD = LP * AD < IT ? LP * AD : IT;  // ahead of the next step's first unit
  if constexpr (DIRECT) {
#pragma unroll
    for (int k = 0; k < NB; ++k) issue(k, k * STAGE, 0, k < NB - 1 ? IT : AHEAD);
    dt_wait_vm<(NB - 2) * IT + AHEAD>();
    dt_barrier();
  } else {
    fetch(0);
    stash(0, 0, IT);
    dt_barrier();
    if (nk > 1) fetch(1);
  }
  read_b(b[0], 0, 0);
#pragma unroll
  for (int u = 0; u < AD; ++u) read_a(a[u], 0, u);
  int buf = 0, last = (NB - 1) * STAGE;  // buffers of steps ks and ks - 1
  for (int ks = 0; ks < nk; ++ks) {
    const int nx = buf == (NB - 1) * STAGE ? 0 : buf + STAGE;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      constexpr int FREE = NU - AD;  // units ahead of the barrier
      if (!DIRECT && FREE == 0 && u == 0) stash(nx, 0, IT);
      if (u == FREE) {
        // this wave's part of step ks + 1 is in LDS, and it reads step ks no more
        if (DIRECT) dt_wait_vm<(NB - 2) * IT>();
        dt_barrier();
        if constexpr (!DIRECT)
          if (ks + 2 < nk) fetch(ks + 2);
      }
      if constexpr (DIRECT) {
        const int from = LP * (u < FREE ? u + AD : u - FREE);
        if (from < IT)
          issue(u < FREE ? ks - 1 + NB : ks + NB, u < FREE ? last : buf, from,
                from + LP < IT ? from + LP : IT);
      }
      // (of the last step: what lies in the other buffer, never used)
      read_a(a[AD], u + AD < NU ? buf : nx, (u + AD) % NU);
      if (u % MI == MI - AD) read_b(b[1], u / MI + 1 < KK ? buf : nx, (u / MI + 1) % KK);
      if (!DIRECT && u < FREE)
        stash(nx, IT * u / (FREE ? FREE : 1), IT * (u + 1) / (FREE ? FREE : 1));
      if constexpr (F32) {
#pragma unroll
        for (int x = 0; x < 6; ++x)
#pragma unroll
          for (int j = 0; j < NI; ++j)
            acc[u % MI][j] = s3_product(x, b[0][j], a[0], acc[u % MI][j]);
      } else {
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[u % MI][j] = s3_mfma(b[0][j][0], a[0][0], acc[u % MI][j]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < AD; ++i)
#pragma unroll
        for (int k = 0; k < PARTS; ++k) a[i][k] = a[i + 1][k];
      if (u % MI == MI - 1)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int k = 0; k < PARTS; ++k) b[0][j][k] = b[1][j][k];
    }
    last = buf;
    buf = nx;
  }
  if (DIRECT) dt_wait_vm<0>();  // nothing lands in LDS any more
  }

  // Epilogue: the wave's piece to LDS, ROWS rows at a time (16 vectors a row, XORed
  // by the row), and back with eight columns of a row per lane (with glu, eight of
  // either half).
  constexpr int COLS = GLU ? 32 : 64, LR = COLS / 8;  // output columns, lanes a row
  constexpr int MOST = TM > ROWS ? 2 : 4;  // sums still in registers leave room for fewer
  constexpr int RI = 64 / LR, U = ROWS / RI < MOST ? ROWS / RI : MOST;
  static_assert(ROWS % (RI * U) == 0, "whole groups of rows");
  s3_v4u* const mine = lds + wave * ROWS * 16;
  const int c = q0 + wn * COLS + lane % LR * 8, cols = n - c;
  float b0[8] = {}, b1[8] = {};
  if (t.epi.bias && !partial && cols > 0) {
    load8n(t.epi.bias, false, c, cols, t.Q, b0);
    if (GLU) load8n(t.epi.bias, false, n + c, cols, t.Q, b1);
  }
  float c0[8] = {}, c1[8] = {};  // DZ: column sums of this lane's rows
  dt_barrier();  // no wave reads operands from LDS any more
#pragma unroll
  for (int pass = 0; pass < TM / ROWS; ++pass) {
#pragma unroll
    for (int i = 0; i < ROWS / 16; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
        mine[(i * 16 + li) * 16 + ((j * 4 + q) ^ li)] = __builtin_bit_cast(
            s3_v4u, F32 ? acc[pass * (ROWS / 16) + i][j] * kSplitDown : acc[pass * (ROWS / 16) + i][j]);
    if constexpr (F32) {
      // What the three parts cannot represent is formed again in plain fp32 (operands
      // of 2^103 and more, sums of 2^80 and more, infinities, NaN): sixteen rows that hold
      // such a sum by 64 columns at a time, with fp32 MFMAs, and of those results the ones
      // that are not finite replaced.  (35472 x 512 -> 1024 with one NaN weight, which
      // every row tile meets: forward 399 us, 224 without; a lane a result took 4340.)
      bool bad = false;
#pragma unroll
      for (int i = 0; i < ROWS / 16; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) bad |= s3_bad(acc[pass * (ROWS / 16) + i][j]);
      if (__any(bad)) {
        const int64_t p = p0 + wm * TM + pass * ROWS + li;
        int cols16[NI];  // this lane's first column of an MFMA's sixteen, and in B column li
        int64_t bcol[NI];
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const int first = GLU ? q0 + wn * 32 + (j & 1) * 16 : q0 + wn * 64 + j * 16;
          cols16[j] = first + 4 * q;
          bcol[j] = (first + li < n ? first + li : n - 1) + (GLU && j > 1 ? t.half : 0);
        }
#pragma unroll 1
        for (int i = 0; i < ROWS / 16; ++i) {
          const auto at = [&](int j) __attribute__((always_inline)) {
            return (i * 16 + li) * 16 + ((j * 4 + q) ^ li);
          };
          bool again = false;
#pragma unroll
          for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              again |= p + i * 16 < t.P && cols16[j] + k < n &&
                       !(fabsf(__builtin_bit_cast(s3_v4f, mine[at(j)])[k]) < INFINITY);
          if (!__any(again)) continue;
          const int64_t row = p + i * 16 < t.P ? p + i * 16 : t.P - 1;
          s3_v4f sum[NI], fa, fb[NI], na, nb[NI];
          const auto load = [&](int64_t r, s3_v4f& x, s3_v4f(&y)[NI]) __attribute__((always_inline)) {
            x = dt_terms<ARS>((const float*)t.a, t.lda, row, r + 4 * q, r1);
#pragma unroll
            for (int j = 0; j < NI; ++j)
              y[j] = dt_terms<BRS>((const float*)t.b, t.ldb, bcol[j], r + 4 * q, r1);
          };
#pragma unroll
          for (int j = 0; j < NI; ++j) sum[j] = s3_v4f{0.f, 0.f, 0.f, 0.f};
          load(r0, fa, fb);
#pragma unroll 1
          for (int64_t r = r0; r < r1; r += 16) {  // term 4 q + e of the sixteen in MFMA e
            load(r + 16, na, nb);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int j = 0; j < NI; ++j)
                sum[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[j][e], fa[e], sum[j], 0, 0, 0);
            fa = na;
#pragma unroll
            for (int j = 0; j < NI; ++j) fb[j] = nb[j];
          }
#pragma unroll
          for (int j = 0; j < NI; ++j) {
            s3_v4f v = __builtin_bit_cast(s3_v4f, mine[at(j)]);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = fabsf(v[k]) < INFINITY ? v[k] : sum[j][k];
            mine[at(j)] = __builtin_bit_cast(s3_v4u, v);
          }
        }
      }
    }
#pragma unroll 1
    for (int g = 0; g < ROWS / (RI * U); ++g) {
      float v[U][8], u[U][8];
      int64_t p[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int row = (g * U + i) * RI + lane / LR;
        p[i] = p0 + wm * TM + pass * ROWS + row;
        auto get = [&](int col, float* w) __attribute__((always_inline)) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const s3_v4f x = __builtin_bit_cast(
                s3_v4f, mine[row * 16 + ((col / 4 + h) ^ (row & 15))]);
#pragma unroll
            for (int k = 0; k < 4; ++k) w[h * 4 + k] = x[k];
          }
        };
        get(lane % LR * 8, v[i]);
        if (GLU) get(32 + lane % LR * 8, u[i]);
      }
      if (cols <= 0) continue;
      if (partial) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int row = (int)(p[i] - p0);
          const int64_t slot = (int64_t)(cls + nth) * t.members + member;
          float* o = t.part + (slot * BM + row) * BN + wn * TN + lane % LR * 8;
          store8(o, false, 0, v[i]);
          if (GLU) store8(o, false, 32, u[i]);
        }
      } else if constexpr (DZ) {
        epilogue_dz<U, GLU>(t.epi, p, t.P, c, b0, b1, v, u, c0, c1);
      } else {
        epilogue<U, GLU>(t.epi, p, t.P, c, b0, b1, v, u);
      }
    }
  }
  if constexpr (DZ) {
    // the tile's column sums: a wave's lanes, then its row of waves, in a fixed order
    if (t.epi.colsum) {
      float* const cs = (float*)lds;
#pragma unroll
      for (int m = LR; m < 64; m <<= 1)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          c0[k] += __shfl_xor(c0[k], m);
          if (GLU) c1[k] += __shfl_xor(c1[k], m);
        }
      dt_barrier();
      if (lane < LR)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          cs[wave * 64 + lane * 8 + k] = c0[k];
          if (GLU) cs[wave * 64 + 32 + lane * 8 + k] = c1[k];
        }
      dt_barrier();
      if (tid < BN) {
        const int col = tid & 63, g = tid >> 6;
        const int cc = q0 + (GLU ? g * 32 + (col & 31) : tid);
        float a = 0.f;
        for (int m = 0; m < WGM; ++m) a += cs[(m * WGN + g) * 64 + col];
        if (cc < n) t.epi.colsum[(int64_t)pos.m * t.Q + (GLU && col >= 32 ? n + cc : cc)] = a;
      }
    }
  }
  if (DIRECT) dt_wait_vm<0>();  // stores are not counted among the next tile's loads
  dt_barrier();                 // whose operands go where the sums were
  }
}

template <typename T, int BM, int BN, int WGM, int BK, int BUFS, bool ARS, bool BRS, bool GLU,
          bool DIRECT, bool DZ>
__global__ __launch_bounds__(64 * WGM * (BN / 64), 2) void k_dense_tile(TileArgs t) {
  __shared__ __attribute__((aligned(16))) s3_v4u lds[tile_lds<T, BM, BN, WGM, BK, BUFS, DIRECT>()];
  tile_run<T, BM, BN, WGM, BK, BUFS, ARS, BRS, GLU, DIRECT, DZ>(t, blockIdx.x, gridDim.x, lds);
}

// Both products of a backward in one launch: the first `split` workgroups are the
// weight gradient's (swapped: the input gradient's), the others the other one's.
template <typename T, int BM, int BN, int WGM, int BK, int BUFS, bool DIRECT>
__global__ __launch_bounds__(64 * WGM * (BN / 64), 2) void k_dense_tiles2(TileArgs dx, TileArgs dw,
                                                                          uint32_t split,
                                                                          bool swapped) {
  __shared__ __attribute__((aligned(16))) s3_v4u lds[tile_lds<T, BM, BN, WGM, BK, BUFS, DIRECT>()];
  const bool head = blockIdx.x < split;
  const uint32_t block = head ? blockIdx.x : blockIdx.x - split;
  const uint32_t blocks = head ? split : gridDim.x - split;
  if (head != swapped)
    tile_run<T, BM, BN, WGM, BK, BUFS, true, true, false, DIRECT, false>(dw, block, blocks, lds);
  else
    tile_run<T, BM, BN, WGM, BK, BUFS, false, false, false, DIRECT, false>(dx, block, blocks, lds);
}

}  // namespace oc
