// Position rotation of 16-byte chunks of a head, shared by the append to the paged cache and the rotation alone:
// unpacking and packing eight bf16, the angles of a token's pairs, and the turn. Internal; included by the
// kernel sources only.
#pragma once

#include "fa_device.h"
#include "fa_internal.h"

namespace fa {
namespace {

// Eight bf16 as fp32 and back (RNE).
struct F8 {
  float x[8];
};
__device__ __forceinline__ F8 unpack8(const u32x4& w) {
  F8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.x[2 * i] = __uint_as_float(w[i] << 16);
    r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ u32x4 pack8(const F8& f) {
  return u32x4{pack_bf16x2(f.x[0], f.x[1]), pack_bf16x2(f.x[2], f.x[3]), pack_bf16x2(f.x[4], f.x[5]),
               pack_bf16x2(f.x[6], f.x[7])};
}

// A product that is rounded by itself: left to the compiler, which of two products that are added is rounded, and which
// joins the sum exactly, differs from place to place.
__device__ __forceinline__ float product(float a, float b) {
  float x = a * b;
  asm("" : "+v"(x));
  return x;
}

// A pair (x, y) becomes (x cos - y sin, y cos + x sin), the products with the sine rounded first. Halves: the pairs are the
// elements of two chunks; else neighbouring elements of one, by the first four angles.
__device__ __forceinline__ void turn_halves(F8& x, F8& y, const F8& cs, const F8& sn) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float a = x.x[e], c = y.x[e];
    x.x[e] = fmaf(a, cs.x[e], -product(c, sn.x[e]));
    y.x[e] = fmaf(c, cs.x[e], product(a, sn.x[e]));
  }
}
__device__ __forceinline__ void turn_neighbours(F8& x, const F8& cs, const F8& sn) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float a = x.x[2 * e], c = x.x[2 * e + 1];
    x.x[2 * e] = fmaf(a, cs.x[e], -product(c, sn.x[e]));
    x.x[2 * e + 1] = fmaf(c, cs.x[e], product(a, sn.x[e]));
  }
}

// Cosines and sines of pairs 4 i .. 4 i + 3 into places 4 at .. of cs and sn; a table row holds the cosines of the row's
// rot / 2 angles, then the sines.
__device__ __forceinline__ void angles_of_row(F8& cs, F8& sn, int at, const float* row, int rot, int i) {
  const f32x4 c4 = *reinterpret_cast<const f32x4*>(row + 4 * i), s4 = *reinterpret_cast<const f32x4*>(row + rot / 2 + 4 * i);
#pragma unroll
  for (int e = 0; e < 4; ++e) cs.x[4 * at + e] = c4[e], sn.x[4 * at + e] = s4[e];
}
// The same by the positions of a token (its first axis at `pos`, the others axis_stride apart): one axis, or each pair by
// that which pair_axes names. Four pairs of one axis are read at once. What the arrays hold is clamped to the table.
__device__ __forceinline__ void angles_at(F8& cs, F8& sn, int at, const Positions& ps, const int* pos, const float* table,
                                          int rot, int i) {
  auto row_of = [&](uint32_t axis) {
    const int p = pos[(int64_t)min(axis, (uint32_t)ps.n_axes - 1u) * ps.axis];
    return table + (int64_t)min(max(p, 0), ps.n_pos - 1) * rot;
  };
  const uint32_t four = ps.pair_axes != nullptr ? *reinterpret_cast<const uint32_t*>(ps.pair_axes + 4 * i) : 0u;
  if (four == (four & 0xffu) * 0x01010101u) {
    angles_of_row(cs, sn, at, row_of(four & 0xffu), rot, i);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* row = row_of((four >> (8 * e)) & 0xffu) + 4 * i + e;
      cs.x[4 * at + e] = row[0];
      sn.x[4 * at + e] = row[rot / 2];
    }
  }
}

// What a thread holds of a head: the first `turned` tasks are the chunks that turn (each with its partner `half` chunks
// on, where dim c turns with dim c + rot / 2), the others are copied.
struct TurnTasks {
  int half, first, turned, tasks;
  __device__ __forceinline__ TurnTasks(int d, int rot, int begin, int inter)
      : half(inter ? 0 : rot / 16), first(begin / 8), turned(inter ? rot / 8 : half), tasks(d / 8 - half) {}
  __device__ __forceinline__ int chunk(int j) const {
    if (j < turned) return first + j;
    const int o = j - turned;  // o-th of the chunks outside [first, first + turned + half)
    return o < first ? o : o + turned + half;
  }
};

}  // namespace
}  // namespace fa
