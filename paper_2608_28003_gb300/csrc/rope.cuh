// Rotation of a head by units of 16 dims: what the kernels that rotate heads share (the mathematics is in rope.cu).
#pragma once

#include "paged.cuh"

namespace w8a8 {

constexpr int kAhead = 4;  // heads whose loads are in flight

struct RopeArgs {
  const uint64_t* turns;
  float scale;
  int rot, inter;
};

// Where a unit's two 16-byte parts lie in a head: rotated units hold 8 pairs, the others 16 plain dims.
__device__ __forceinline__ void unit_place(const RopeArgs& r, int unit, bool& rotated, int& at0, int& at1) {
  rotated = unit < r.rot / 16;
  if (rotated && !r.inter) {
    at0 = 8 * unit;
    at1 = r.rot / 2 + 8 * unit;
  } else {
    at0 = 16 * unit;
    at1 = at0 + 8;
  }
}

__device__ __forceinline__ void unit_angles(const RopeArgs& r, int unit, int pos, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint64_t turn = (uint64_t)(int64_t)pos * r.turns[8 * unit + e];
    const float half_turns = (float)(int64_t)turn * 0x1p-63f;
    sincospif(half_turns, &s[e], &c[e]);
    s[e] *= r.scale;
    c[e] *= r.scale;
  }
}

struct Unit {
  uint4 a, b;
};
__device__ __forceinline__ Unit unit_load(const uint16_t* p, int at0, int at1) {
  return Unit{*reinterpret_cast<const uint4*>(p + at0), *reinterpret_cast<const uint4*>(p + at1)};
}
template <bool kBf16>
__device__ __forceinline__ void unit_values(const Unit& u, float (&x)[16]) {
  const uint32_t w[8] = {u.a.x, u.a.y, u.a.z, u.a.w, u.b.x, u.b.y, u.b.z, u.b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 f = unpack2<kBf16>(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
template <bool kBf16>
__device__ __forceinline__ void unit_store(uint16_t* p, int at0, int at1, const float (&x)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = pack2<kBf16>(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<uint4*>(p + at0) = make_uint4(w[0], w[1], w[2], w[3]);
  *reinterpret_cast<uint4*>(p + at1) = make_uint4(w[4], w[5], w[6], w[7]);
}
// half layout: pair e is (x[e], x[8 + e]); interleaved: (x[2e], x[2e + 1])
__device__ __forceinline__ void unit_rotate(bool inter, const float (&c)[8], const float (&s)[8], float (&x)[16]) {
  if (inter) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = x[2 * e], b = x[2 * e + 1];
      x[2 * e] = a * c[e] - b * s[e];
      x[2 * e + 1] = b * c[e] + a * s[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = x[e], b = x[8 + e];
      x[e] = a * c[e] - b * s[e];
      x[8 + e] = b * c[e] + a * s[e];
    }
  }
}

// The threads a row's heads are spread over: as many as fill the SMs once (their registers hold 512 of a thread's 16 values, angles
// and loads ahead), so that few rows spread over the heads, and many compute their angles once for all heads.  2400 rows of
// 24 heads of 128: 11.5 us with one such wave, 16.4 with four (a thread a head, its angles for that head alone); 8192 rows of
// which a part rotates: 23.9 and 27.4.
inline int head_step(int64_t rows, int units, int heads, int sms) {
  const int64_t want = (int64_t)sms * 512;
  const int64_t step = want / (rows * units);
  return (int)(step < 1 ? 1 : step > heads ? heads : step);
}

}  // namespace w8a8
