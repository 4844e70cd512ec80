// Norms of query and key heads and the position rotation in one pass (kivi_norm_rotate).
//
//   y = x / sqrt(mean(x^2) + eps) * (w + offset), then pairs (x, y) -> (x cos - y sin, y cos + x sin); fp32, rounded once.
//
// Eight lanes hold a head's 128 channels (kivi_head_rows.h), so the mean takes three exchanges inside eight lanes and the rotation none.
// A wavefront takes two times eight heads of one row: the row's cosines and sines are read once for them, and four loads per lane are
// in flight.  Bound: memory; every byte is read and written once.  65 536 rows x 64 heads, bf16: 397 us, 5.4 TB/s (one time eight heads 428, four
// times 422; a plain copy of as many bytes 440); one row of 40 heads 2.7 us, which is a launch.
#include "kivi_head_rows.h"

namespace kivi {
namespace {

using namespace head_rows;

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sum_of_eight(float x) {
    x += dpp<0xB1>(x);                 // lanes 1 apart
    x += dpp<0x4E>(x);                 // 2 apart
    return x + dpp<0x141>(x);          // mirrored within eight
}

struct Args : NormRotateParams {
    FastDiv by_pieces;
    int32_t pieces;                    // wavefronts per row
    int32_t n_waves;
};

constexpr int U = 2;                   // times eight heads of a wavefront

__global__ __launch_bounds__(256) void norm_rotate_kernel(Args p) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int at = (int)blockIdx.x * 4 + wave;
    if (at >= p.n_waves) return;
    const int row = p.by_pieces.of(at), head0 = (at - row * p.pieces) * 8 * U + (lane >> 3), j = lane & 7;
    const RotationParams& r = p.rotation;
    const Pieces pc = pieces_of(j, r.half, r.interleaved);
    const bool turns = j < r.half / 8;
    uint4v ra[U], rb[U];
    auto job_of = [&](int head) -> const NormRotateParams::Job& { return p.job[head < p.heads0 ? 0 : 1]; };
    auto row_of = [&](const TensorParams& t, int head) { return t.data + row * t.stride_t + (int64_t)(head < p.heads0 ? head : head - p.heads0) * t.stride_h; };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int head = head0 + 8 * u;
        if (head < p.heads) {
            const __half* src = row_of(job_of(head).src, head);
            ra[u] = *reinterpret_cast<const uint4v*>(src + pc.a * 8);
            rb[u] = *reinterpret_cast<const uint4v*>(src + pc.b * 8);
        }
    }
    Turn t{};
    if (turns) load_turn(r, clamped_position(r, r.positions[row]), j, t);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int head = head0 + 8 * u;
        if (head < p.heads) {
            const NormRotateParams::Job& job = job_of(head);
            float a[8], b[8];
            to_floats(ra[u], job.src_bf16, a);
            to_floats(rb[u], job.src_bf16, b);
            if (job.weight) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(a[e], a[e], fmaf(b[e], b[e], sum));
                const float f = 1.f / sqrtf(sum_of_eight(sum) * (1.f / kHeadDim) + p.eps);
                float wa[8], wb[8];
                to_floats(*reinterpret_cast<const uint4v*>(job.weight + pc.a * 8), job.src_bf16, wa);
                to_floats(*reinterpret_cast<const uint4v*>(job.weight + pc.b * 8), job.src_bf16, wb);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    a[e] = a[e] * f * (wa[e] + job.weight_offset);
                    b[e] = b[e] * f * (wb[e] + job.weight_offset);
                }
            }
            if (turns) turn_pieces(a, b, t, r.interleaved);
            __half* dst = row_of(job.dst, head);
            *reinterpret_cast<uint4v*>(dst + pc.a * 8) = from_floats(a, job.dst_bf16);
            *reinterpret_cast<uint4v*>(dst + pc.b * 8) = from_floats(b, job.dst_bf16);
        }
    }
}

}  // namespace

hipError_t launch_norm_rotate(const NormRotateParams& params, hipStream_t stream) {
    Args p{};
    static_cast<NormRotateParams&>(p) = params;
    p.pieces = (p.heads + 8 * U - 1) / (8 * U);
    p.by_pieces = FastDiv::by(p.pieces);
    const int64_t waves = (int64_t)p.n_rows * p.pieces;
    if (waves > 0x7ffffff0) return hipErrorInvalidValue;
    p.n_waves = (int32_t)waves;
    norm_rotate_kernel<<<(unsigned)((waves + 3) / 4), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace kivi
