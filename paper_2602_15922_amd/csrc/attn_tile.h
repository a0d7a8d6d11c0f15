// Building blocks of the bf16 flash attentions (attn.hip, attn_ragged.hip): a 64-key tile of K and
// V in swizzled LDS, its scores, the online softmax and the value product for 32 queries of one
// wavefront.
#pragma once
#include "common.h"

namespace wam {

constexpr int BM = 128;  // query rows per workgroup
constexpr int BN = 64;   // keys per tile
constexpr int NT = 256;  // threads per workgroup
constexpr float RESCALE_LOG2 = 8.0f;  // allowed growth of exp2 arguments before a rescale

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

// The value held by lane l ^ 32 (the lane with the same query and the other half of the
// keys): one v_permlane32_swap, which exchanges the upper half of its first operand with
// the lower half of its second, instead of a round trip through LDS (ds_bpermute).
WAM_DEV float other_half(float v) {
  const unsigned u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// LDS swizzles (XOR of the 16-byte chunk index).  gfx950 LDS serves 256 bytes (64
// banks) per cycle: 16 lanes of a 16-byte read, 32 lanes of an 8-byte read.
//  K: the fragment read has 16 lanes on 16 consecutive rows at one logical chunk;
//     with 256-byte rows (Dh=128) XOR by row&15, with 128-byte rows by (row>>1)&7.
//  V: a transposing read covers 4 consecutive rows x 64 bytes per 32 lanes, so the
//     4 rows' 64-byte groups must fall in different quarters of the 256-byte line:
//     XOR by 4*(row&3) (Dh=128) or 4*((row>>1)&1) (Dh=64, two rows per line).
template <int DH>
WAM_DEV int kswz(int row, int ch) { return DH == 128 ? (ch ^ (row & 15)) : (ch ^ ((row >> 1) & 7)); }
template <int DH>
WAM_DEV int vswz(int row, int ch) { return DH == 128 ? (ch ^ (4 * (row & 3))) : (ch ^ (4 * ((row >> 1) & 1))); }

// V^T fragments through inline asm.  The compiler cannot prove that these LDS reads miss
// the direct-to-LDS prefetch of the next tile still in flight, so before its own form of
// the transposing read it waits for all outstanding vector memory, i.e. for the next
// tile's loads, every tile.  Issued as asm, the reads wait only on the LDS counter, which
// the code below sets itself: the reads of P.V MFMA i+2 are issued before MFMA i, which
// then waits until at most the 4 younger reads are outstanding (LDS reads complete in
// order).  The asm results are tied through the wait so nothing reads them earlier.
template <int OFF>
WAM_DEV s16x4 tr16(unsigned addr) {
  s16x4 r;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "i"(OFF));
  return r;
}
WAM_DEV unsigned lds_addr(const void* p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)(p);
}
template <int N>
WAM_DEV void wait_lgkm(s16x4& a, s16x4& b) {
  asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "i"(N));
}

// the two reads of P.V MFMA i = (mt, nt, hf): keys 32 nt + 16 hf + (0..7, 8..15) of dims
// 32 mt + (lane's 4), from the lane's base address of output tile mt
template <int DH, int I>
WAM_DEV void vread(const unsigned* va, s16x4* lo, s16x4* hi) {
  constexpr int ROWB = DH * 2, mt = I >> 2, nt = (I >> 1) & 1, hf = I & 1, off = (32 * nt + 16 * hf) * ROWB;
  lo[I % 3] = tr16<off>(va[mt]);
  hi[I % 3] = tr16<off + 8 * ROWB>(va[mt]);
}

template <int DH, int I>
WAM_DEV void pv_steps(const unsigned* va, s16x4* lo, s16x4* hi, const bf16x8 (*pb)[2], f32x16* acc) {
  constexpr int NMF = DH / 8, mt = I >> 2, nt = (I >> 1) & 1, hf = I & 1;  // NMF = 4 MT MFMAs
  if constexpr (I + 2 < NMF) {
    vread<DH, I + 2>(va, lo, hi);
    wait_lgkm<4>(lo[I % 3], hi[I % 3]);
  } else if constexpr (I + 1 < NMF) {
    wait_lgkm<2>(lo[I % 3], hi[I % 3]);
  } else {
    wait_lgkm<0>(lo[I % 3], hi[I % 3]);
  }
  const s16x4 v8[2] = {lo[I % 3], hi[I % 3]};
  acc[mt] = mfma32(*reinterpret_cast<const bf16x8*>(v8), pb[nt][hf], acc[mt]);
  if constexpr (I + 1 < NMF) pv_steps<DH, I + 1>(va, lo, hi, pb, acc);
}

// K fragments of the score MFMAs, likewise as asm: the compiler's schedule issued each
// read one MFMA ahead of its use, exposing the LDS latency once the tile's other stall was
// gone; here the read of score MFMA i+3 is issued before MFMA i (measured best of 2, 3, 5
// and 7 ahead).  Score MFMA i = (ks = i/2, nt = i%2) alternates the two accumulators.
constexpr int KAHEAD = 3;
template <int OFF>
WAM_DEV bf16x8 kread(unsigned addr) {
  bf16x8 r;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "i"(OFF));
  return r;
}
template <int N>
WAM_DEV void wait_k(bf16x8& a) {
  asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(a) : "i"(N));
}
template <int DH, int I>
WAM_DEV void kload(const unsigned* ka, bf16x8* kf) {
  constexpr int ks = I >> 1, nt = I & 1;
  kf[I % (KAHEAD + 1)] = kread<nt * 32 * DH * 2>(ka[ks]);
}
template <int DH, int I>
WAM_DEV void score_steps(const unsigned* ka, bf16x8* kf, const bf16x8* qf, f32x16* s) {
  constexpr int NS = DH / 8, ks = I >> 1, nt = I & 1;  // NS = 2 KS score MFMAs
  if constexpr (I + KAHEAD < NS) {
    kload<DH, I + KAHEAD>(ka, kf);
    wait_k<KAHEAD>(kf[I % (KAHEAD + 1)]);
  } else {
    wait_k<NS - 1 - I>(kf[I % (KAHEAD + 1)]);
  }
  s[nt] = mfma32(kf[I % (KAHEAD + 1)], qf[ks], s[nt]);
  if constexpr (I + 1 < NS) score_steps<DH, I + 1>(ka, kf, qf, s);
}
template <int DH, int I>
WAM_DEV void kloads(const unsigned* ka, bf16x8* kf) {
  kload<DH, I>(ka, kf);
  if constexpr (I + 1 < KAHEAD) kloads<DH, I + 1>(ka, kf);
}
// S^T = K Q^T for one tile (keys 0..31 into s[0], 32..63 into s[1])
template <int DH>
WAM_DEV void scores_tile(const char* Ks, const int* kofs, const bf16x8* qf, f32x16* s) {
  constexpr int KS = DH / 16;
  unsigned ka[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) ka[ks] = lds_addr(Ks + kofs[ks]);
  bf16x8 kf[KAHEAD + 1];
  kloads<DH, 0>(ka, kf);
  score_steps<DH, 0>(ka, kf, qf, s);
}

// O^T += V^T P^T for one tile: 4 MT MFMAs, each with its two transposing V reads
template <int DH>
WAM_DEV void pv_tile(const char* Vs, const int* vofs, const bf16x8 (*pb)[2], f32x16* acc) {
  constexpr int MT = DH / 32;
  unsigned va[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) va[mt] = lds_addr(Vs + vofs[mt]);
  s16x4 lo[3], hi[3];
  vread<DH, 0>(va, lo, hi);
  vread<DH, 1>(va, lo, hi);
  pv_steps<DH, 0>(va, lo, hi, pb, acc);
}

// The online softmax of a tile's (masked) scores s with a lazily raised reference, and O^T +=
// V^T P^T.  vofs[mt]: the lane's byte offset of its transposing V read for output tile mt.
template <int DH>
WAM_DEV void softmax_pv(const f32x16* s, const char* Vs, f32x16* acc, float& m_ref, float& l_part, const int* vofs,
                        float c, float thr) {
  constexpr int MT = DH / 32;
  float mx = s[0][0];
#pragma unroll
  for (int nt = 0; nt < 2; ++nt)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[nt][r]);
  mx = fmaxf(mx, other_half(mx));
  const bool raise = mx > m_ref + thr || (m_ref == -INFINITY && mx != -INFINITY);
  if (__any(raise)) {
    const float m_new = raise ? mx : m_ref;
    const float alpha = m_ref == -INFINITY ? 0.f : exp2_fast((m_ref - m_new) * c);
    m_ref = m_new;
    l_part *= alpha;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] *= alpha;
  }
  const float ms = m_ref == -INFINITY ? 0.f : m_ref * c;
  bf16x8 pb[2][2];
#pragma unroll
  for (int nt = 0; nt < 2; ++nt)
#pragma unroll
    for (int r = 0; r < 16; ++r) pb[nt][r >> 3][r & 7] = (bf16)exp2_fast(__builtin_fmaf(s[nt][r], c, -ms));
  // row sum of exactly the bf16 probabilities the PV product uses, two per dot2
  const bf16x2 ones = {(bf16)1.0f, (bf16)1.0f};
#pragma unroll
  for (int nt = 0; nt < 2; ++nt)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x2 pr = {pb[nt][hf][2 * e], pb[nt][hf][2 * e + 1]};
        l_part = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_part, false);
      }
  pv_tile<DH>(Vs, vofs, pb, acc);
}

// Wait for this wave's direct loads of the next tile, then sync the workgroup.
WAM_DEV void tile_sync() {
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
}

}  // namespace wam
