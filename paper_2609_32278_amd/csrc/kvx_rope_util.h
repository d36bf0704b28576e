// Device code of the stores that rotate: RMS norm and rotation of head rows by the lanes of a
// workgroup, and the angles of a page.  Included by store kernels, inside no namespace.
//
// A head row of D bf16 values is D/8 16-byte chunks held by D/8 consecutive
// lanes; the RMS sum is reduced across those lanes, and in the half layout a
// chunk of the first half meets its plane partners in the chunk rotary_dim/16
// lanes further on (one lane shuffle per value).
#pragma once

#include "kvx_store_util.h"

namespace kvx {
namespace {

constexpr int kStoreThreads = 256;
constexpr int kRopeBatch = 4;  // chunks per thread in flight

template <int D, bool INTERLEAVED>
struct RopeLane {
  static constexpr int CPR = D / 8;
  int cc;           // chunk of the row this lane handles (fixed for the thread)
  int partner;      // lane holding the plane partners (half layout)
  int jb;           // first plane of the chunk
  bool rot;         // the chunk lies inside rotary_dim
  float sgn;        // half layout: -1 for the plane's first dims, +1 for its second

  __device__ RopeLane(int rotary_dim) {
    cc = threadIdx.x % CPR;
    const int lane = threadIdx.x & 63;
    if constexpr (INTERLEAVED) {
      rot = cc < (rotary_dim >> 3);
      jb = 4 * cc;
      partner = lane;
      sgn = 0.0f;
    } else {
      const int r16 = rotary_dim >> 4;
      const bool first = cc < r16;
      rot = cc < 2 * r16;
      jb = first ? 8 * cc : 8 * (cc - r16);
      partner = lane + (first ? r16 : (rot ? -r16 : 0));
      sgn = first ? -1.0f : 1.0f;
    }
  }
};

// x: the 8 values of this lane's chunk of one row at `slot`; in place -> rotated.
// Every lane of the row must execute this (shuffles).
template <int D, bool INTERLEAVED>
__device__ __forceinline__ void rope_chunk(float (&x)[8], const RopeLane<D, INTERLEAVED>& rl,
                                           const float2* cs_slot) {
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float2 t = rl.rot ? cs_slot[rl.jb + i] : make_float2(1.0f, 0.0f);
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * t.x - b * t.y;
      x[2 * i + 1] = a * t.y + b * t.x;
    }
  } else {
    float pe[8];
#pragma unroll
    for (int e = 0; e < 8; e++) pe[e] = __shfl(x[e], rl.partner, 64);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float2 t = rl.rot ? cs_slot[rl.jb + e] : make_float2(1.0f, 0.0f);
      // first dims: a cos - b sin (b = partner); second dims: b cos + a sin (a = partner)
      x[e] = x[e] * t.x + rl.sgn * (pe[e] * t.y);
    }
  }
}

// Normalise and rotate `nh` heads from h0 on (nh <= 1 << lg) of the unit's ntok tokens
// (src: the first token's row, [token][heads][D] bf16) and hand each chunk's results
// to out(token, head, chunk, y).  The first loads are issued before angles() -- which
// fills cs and ends in a barrier -- so that they are in flight meanwhile.
template <int D, bool INTERLEAVED, class Angles, class Out>
__device__ __forceinline__ void rope_rows(const uint16_t* __restrict__ src, int ntok, int heads, int h0, int nh, int lg,
                                          int slot_begin, const float2 (*cs)[kRopeMaxPlanes],
                                          const uint16_t* norm_w, float eps, int rotary_dim, Angles&& angles,
                                          Out&& out) {
  constexpr int CPR = D / 8;
  const RopeLane<D, INTERLEAVED> rl(rotary_dim);
  // row index rr = token << lg | head of the group; rows past the group's heads idle
  const int n = ntok << lg;
  constexpr int ROWS = kStoreThreads / CPR;  // rows per step
  const int r0 = threadIdx.x / CPR;
  auto load = [&](int rr) {
    const int tok = rr >> lg, hh = rr & ((1 << lg) - 1);
    return rr < n && hh < nh ? *(const uint4*)(src + ((size_t)tok * heads + h0 + hh) * D + rl.cc * 8)
                             : make_uint4(0, 0, 0, 0);
  };
  uint4 raw[kRopeBatch];
#pragma unroll
  for (int b = 0; b < kRopeBatch; b++) raw[b] = load(r0 + b * ROWS);
  float w[8];
  if (norm_w) {
    const uint4 wr = *(const uint4*)(norm_w + rl.cc * 8);
    const uint16_t* wh = (const uint16_t*)&wr;
#pragma unroll
    for (int e = 0; e < 8; e++) w[e] = bf16_to_f32(wh[e]);
  }
  angles();
  for (int c0 = r0; c0 - r0 < n; c0 += kRopeBatch * ROWS) {
    uint4 next[kRopeBatch];
#pragma unroll
    for (int b = 0; b < kRopeBatch; b++) next[b] = load(c0 + (kRopeBatch + b) * ROWS);
#pragma unroll
    for (int b = 0; b < kRopeBatch; b++) {
      const int rr = c0 + b * ROWS;
      if (rr - r0 >= n) break;  // uniform
      const int tok = rr >> lg, hh = rr & ((1 << lg) - 1);
      const uint16_t* h16 = (const uint16_t*)&raw[b];
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] = bf16_to_f32(h16[e]);
      if (norm_w) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e++) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int m = 1; m < CPR; m <<= 1) ss += __shfl_xor(ss, m, 64);
        const float inv = 1.0f / sqrtf(ss * (1.0f / D) + eps);
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = (x[e] * inv) * w[e];
      }
      rope_chunk<D, INTERLEAVED>(x, rl, cs[slot_begin + (rr < n ? tok : 0)]);
      if (rr < n && hh < nh) out(tok, h0 + hh, rl.cc, x);
    }
#pragma unroll
    for (int b = 0; b < kRopeBatch; b++) raw[b] = next[b];
  }
}

// (cos, sin) of every live slot of the unit's page and every plane, by all threads of the
// workgroup: each angle is reduced to [-1/2, 1/2] turn in float64, exactly.  The caller's
// barrier follows.
__device__ __forceinline__ void fill_angles(float2 (*cs)[kRopeMaxPlanes], const RopeUnit& u, int rotary_dim,
                                            const double* rev_freq) {
  const int planes = rotary_dim / 2, ntok = u.slot_end - u.slot_begin;
  for (int e = threadIdx.x; e < ntok * planes; e += kStoreThreads) {
    const int s = u.slot_begin + e / planes, j = e % planes;
    double rev = (double)(u.pos_slot0 + s) * rev_freq[j];  // exact position times the rate
    rev -= rint(rev);
    float sn, cn;
    sincospif(2.0f * (float)rev, &sn, &cn);
    cs[s][j] = make_float2(cn, sn);
  }
}

}  // namespace
}  // namespace kvx
