// Rows of one head (128 channels of 16 bits) by eight lanes: loads, stores and the position rotation, for kivi_norm_rotate and
// kivi_paged_append.
//
// Lane j of the eight holds two pieces of eight channels such that the pairs of the rotation never leave a lane: pieces j and
// j + rotary/16 where pairs are half a rotary dimension apart (of the channels that do not rotate, two neighbouring pieces), pieces 2 j and 2 j + 1
// where they are interleaved.  Either way lane j needs the cosines and sines 8 j .. 8 j + 7, and rotates if j < rotary/16.
#pragma once

#include "kivi_internal.h"

namespace kivi {
namespace head_rows {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfloat8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// kivi_rotation_t as the kernels take it; half = rotary_dim / 2, 0: no rotation
struct RotationParams {
    const float* table;
    const int32_t* positions;
    int32_t n_positions, half, interleaved;
};

struct TensorParams {
    __half* data;
    int64_t stride_b, stride_h, stride_t;
};

__device__ __forceinline__ void to_floats(uint4v raw, bool bf16, float (&x)[8]) {
    if (bf16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(raw[i] << 16);
            x[2 * i + 1] = __uint_as_float(raw[i] & 0xFFFF0000u);
        }
    } else {
        const half8 h = __builtin_bit_cast(half8, raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)h[i];
    }
}
// rounded to nearest even
__device__ __forceinline__ uint4v from_floats(const float (&x)[8], bool bf16) {
    if (bf16) {
        bfloat8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (__bf16)x[i];
        return __builtin_bit_cast(uint4v, r);
    }
    half8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (_Float16)x[i];
    return __builtin_bit_cast(uint4v, r);
}

// the two pieces of lane j, in pieces of eight channels
struct Pieces { int a, b; };
__device__ __forceinline__ Pieces pieces_of(int j, int half, int interleaved) {
    const int turning = half / 8;                      // lanes that rotate
    if (interleaved || turning == 0) return Pieces{2 * j, 2 * j + 1};
    return j < turning ? Pieces{j, j + turning} : Pieces{2 * j, 2 * j + 1};
}

__device__ __forceinline__ int clamped_position(const RotationParams& r, int at) { return min(max(at, 0), r.n_positions - 1); }

struct Turn { float cos[8], sin[8]; };
__device__ __forceinline__ void load_turn(const RotationParams& r, int position, int j, Turn& t) {
    const float* row = r.table + (int64_t)position * (2 * r.half) + 8 * j;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4v c = *reinterpret_cast<const float4v*>(row + 4 * i), s = *reinterpret_cast<const float4v*>(row + r.half + 4 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) { t.cos[4 * i + k] = c[k]; t.sin[4 * i + k] = s[k]; }
    }
}
// one pair: each product and the difference rounded on its own
__device__ __forceinline__ void turn_pair(float& x, float& y, float c, float s) {
#pragma clang fp contract(off)
    const float xc = x * c, ys = y * s, yc = y * c, xs = x * s;
    x = xc - ys;
    y = yc + xs;
}
__device__ __forceinline__ void turn_pieces(float (&a)[8], float (&b)[8], const Turn& t, int interleaved) {
    if (interleaved) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            turn_pair(a[2 * m], a[2 * m + 1], t.cos[m], t.sin[m]);
            turn_pair(b[2 * m], b[2 * m + 1], t.cos[4 + m], t.sin[4 + m]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn_pair(a[e], b[e], t.cos[e], t.sin[e]);
    }
}

}  // namespace head_rows

struct NormRotateParams {
    struct Job {
        head_rows::TensorParams src, dst;
        const __half* weight;          // null: no norm
        float weight_offset;
        int32_t src_bf16, dst_bf16;
    } job[2];
    int32_t heads0, heads;             // of the first tensor, of both
    int32_t n_rows;
    float eps;
    head_rows::RotationParams rotation;
};
hipError_t launch_norm_rotate(const NormRotateParams& p, hipStream_t stream);

}  // namespace kivi
