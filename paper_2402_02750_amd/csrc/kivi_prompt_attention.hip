// Attention of prompts over 16-bit keys and values (kivi_prompt_attention): one pass over the keys with the running maximum and sum
// of a softmax, causal, with an optional window and first keys that stay visible.
//
// A workgroup has 128 queries of one head, 32 per wavefront, and walks over tiles of 64 keys that all four wavefronts read
// from LDS.  All products are 32x32x16 matrix instructions, and everything is kept transposed so that a query is a lane:
//   S^T = K Q^T    operand rows are keys (out of LDS), columns are queries (in registers): lane (q = lane % 32, h = lane / 32) gets
//                  the logits of keys 8 (i / 4) + 4 h + i % 4, i = 0..15: half of its query's; the other half is 32 lanes away
//   O^T = V^T P^T  the probabilities of a lane are, in the order the lane has them, its share of the second operand of an instruction over
//                  16 keys, so they change neither lane nor order; the value rows are taken in that order too, transposed by the LDS read
//                  (4 keys of one channel per lane and read).
// Masked elements are set to -inf in tiles that the mask cuts; tiles that it leaves empty are not visited.  The running maximum
// starts at a finite number, so that rows which have seen nothing yet stay 0.  It moves only where a logit passes it by more
// than 2^8 (the probabilities are at most 2^8 then, which both types hold); sums and outputs are fp32.
// Probabilities are rounded to the tensors' type, to nearest: an error of 2^-12 (bf16: 2^-9) of each term at most.
#include "kivi_prompt.h"

#include <type_traits>

namespace kivi {
namespace {

using namespace head_rows;
typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kWaveQueries = 32, kQueries = kWaves * kWaveQueries, kKeys = 64;
constexpr int kTileBytes = kKeys * kHeadDim * 2;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;                  // log2 headroom of the running maximum
constexpr float kNothing = -1e30f;             // running maximum of a row that has seen nothing

struct Args : PromptParams {
    int32_t q_tiles;                   // of the longest sequence
    int32_t by_die;                    // > 0: (sequence, kv-head) pairs per die, each pair's workgroups on one of the eight
};

// Asynchronous copy of 16 bytes per lane to LDS offset lds + 16 lane.  (Wait states between a vector instruction that writes the scalar operand and
// this one: the compiler does not look into the block.  m0 is a reserved register, so the compiler warns that it keeps no value there: nor shall it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t lane_offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy_to_lds(const void* lane_ptr, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(lane_ptr) : "memory", "m0");
}
#pragma clang diagnostic pop
// Workgroup barrier that orders LDS traffic only (a __syncthreads() would also wait for the copies in flight)
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <bool BF16>
__device__ __forceinline__ float16v product(uint4v a, uint4v b, float16v c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bfloat8, a), __builtin_bit_cast(bfloat8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float max_halves(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    return fmaxf(__int_as_float(a[0]), __int_as_float(a[1]));
}
__device__ __forceinline__ float add_halves(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    return __int_as_float(a[0]) + __int_as_float(a[1]);
}

// Where 16-byte piece `piece` of row `row` of a tile is: pieces change place so that the lanes of a read meet different banks.  Key
// reads take one piece of 16 rows at a time, value reads 64 bytes of four rows.
__device__ __forceinline__ int key_offset(int row, int piece) { return row * 256 + ((piece ^ (row & 15)) << 4); }
__device__ __forceinline__ int value_offset(int row, int piece) { return row * 256 + ((piece ^ ((row & 3) << 2)) << 4); }

typedef __attribute__((address_space(3))) short4v* LdsShort4;

template <bool BF16>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_attention_kernel(Args p) {
    __shared__ __align__(16) unsigned char sm[2][2][kTileBytes];          // [buffer][keys, values]
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rep = p.n_q_heads / p.n_kv_heads;
    int at = blockIdx.x, b, head, q_tile;                                    // the longest rows first
    if (p.by_die > 0) {
        const int die = at & 7, in_die = at >> 3, r = in_die % rep, pair = in_die / rep % p.by_die * 8 + die;
        b = pair / p.n_kv_heads;
        head = (pair - b * p.n_kv_heads) * rep + r;
        q_tile = p.q_tiles - 1 - in_die / rep / p.by_die;
    } else {
        head = at % p.n_q_heads;
        at /= p.n_q_heads;
        b = at % p.batch;
        q_tile = p.q_tiles - 1 - at / p.batch;
    }
    // the sequence
    int n_q = p.max_q, n_k = p.max_k;
    int64_t q_row = 0, k_row = 0;
    if (p.q_starts) {
        const int first = p.q_starts[b], end = p.q_starts[b + 1];
        n_q = first >= 0 && end <= p.q_rows && end >= first && (int64_t)end - first <= p.max_q ? end - first : 0;
        q_row = first;
    }
    if (p.k_starts) {
        const int first = p.k_starts[b], end = p.k_starts[b + 1];
        if (!(first >= 0 && end <= p.k_rows && end >= first && (int64_t)end - first <= p.max_k)) return;
        n_k = end - first;
        k_row = first;
    }
    const int q0 = q_tile * kQueries;
    if (q0 >= n_q) return;
    const int kv_head = head / rep;
    const int shift = n_k - n_q;                                   // query i stands at key i + shift
    const int first_at = q0 + shift, last_at = min(q0 + kQueries, n_q) - 1 + shift;
    const int my_q = q0 + wave * kWaveQueries + col, my_at = my_q + shift;

    // queries: columns of the first product
    const float c = fmaxf(fabsf(p.softmax_scale) * kLog2e, 1e-30f);        // (not 0: masked logits stay -inf)
    uint4v qf[8];
    {
        const __half* src = p.q.data + (p.q_starts ? 0 : b * p.q.stride_b) + head * p.q.stride_h + (q_row + min(my_q, n_q - 1)) * p.q.stride_t + half * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            qf[i] = *reinterpret_cast<const uint4v*>(src + i * 16);
            if (p.softmax_scale < 0.f) qf[i] ^= 0x80008000u;
        }
    }
    float16v o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m = kNothing, l = 0.f;

    // key tiles: those of the first keys, then those that the window reaches
    const int lowest = p.window > 0 ? max(first_at - p.window + 1, 0) : 0;
    const int sink_tiles = p.window > 0 ? (min(p.sinks, lowest) + kKeys - 1) / kKeys : 0;
    const int first_tile = max(lowest / kKeys, sink_tiles), end_tile = last_at < 0 ? 0 : last_at / kKeys + 1;
    const int n_tiles = last_at < 0 ? 0 : min(sink_tiles, end_tile) + max(end_tile - first_tile, 0);
    const __half* k_base = p.k.data + (p.k_starts ? 0 : b * p.k.stride_b) + kv_head * p.k.stride_h + k_row * p.k.stride_t;
    const __half* v_base = p.v.data + (p.k_starts ? 0 : b * p.v.stride_b) + kv_head * p.v.stride_h + k_row * p.v.stride_t;

    // ---- copies: a wavefront has 16 rows of keys and of values, four per instruction ----
    const uint32_t sm_lds = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)&sm[0][0][0]);
    const int copy_row = lane >> 4, copy_slot = lane & 15;
    uint32_t k_lane[4], v_lane[4];                                    // byte offsets of this lane's piece from the instruction's first row
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k_lane[i] = copy_row * (uint32_t)p.k.stride_t * 2 + ((copy_slot ^ (i * 4 + copy_row)) << 4);
        v_lane[i] = copy_row * (uint32_t)p.v.stride_t * 2 + ((copy_slot ^ (copy_row << 2)) << 4);
    }
    auto tile_key = [&](int it) { return (it < sink_tiles ? it : it - sink_tiles + first_tile) * kKeys; };
    auto copy_rows = [&](const __half* base, int64_t stride, const uint32_t (&lane_offset)[4], int it, uint32_t lds) {
        const int row0 = tile_key(it) + wave * 16;
        if (row0 + 16 <= n_k) {
#pragma unroll
            for (int i = 0; i < 4; ++i) copy_to_lds(base + (row0 + i * 4) * stride, lane_offset[i], lds + i * 1024);
        } else {                                                   // rows past the end re-read the last one
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = min(row0 + i * 4 + copy_row, n_k - 1);
                copy_to_lds(base + key * stride + (int)(lane_offset[i] - copy_row * (uint32_t)stride * 2) / 2, lds + i * 1024);
            }
        }
    };
    auto copy_keys = [&](int it, int buffer) { copy_rows(k_base, p.k.stride_t, k_lane, it, sm_lds + buffer * 2 * kTileBytes + wave * 16 * 256); };
    auto copy_values = [&](int it, int buffer) { copy_rows(v_base, p.v.stride_t, v_lane, it, sm_lds + (buffer * 2 + 1) * kTileBytes + wave * 16 * 256); };
    float16v s[2];
    // logits of a tile out of its keys in LDS
    auto logits = [&](const unsigned char* sm_k, float16v (&to)[2]) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int e = 0; e < 16; ++e) to[kb][e] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                to[kb] = product<BF16>(*reinterpret_cast<const uint4v*>(sm_k + key_offset(kb * 32 + col, 2 * i + half)), qf[i], to[kb]);
        }
    };
    if (n_tiles > 0) {
        copy_keys(0, 0);
        copy_values(0, 0);
        if (n_tiles > 1) copy_keys(1, 1);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        logits(sm[0][0], s);
    }
    for (int it = 0; it < n_tiles; ++it) {
        const int key0 = tile_key(it);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // this wavefront's rows of the tiles are there,
        lds_barrier();                                             // everybody's, and nobody reads the other buffers any more
        if (it + 2 < n_tiles) copy_keys(it + 2, it & 1);
        if (it + 1 < n_tiles) copy_values(it + 1, (it + 1) & 1);
        const unsigned char *sm_v = sm[it & 1][1];
        // tiles that the mask cuts for some query of the workgroup
        if (key0 + kKeys - 1 > first_at) {
            const int behind = my_at - key0 - 4 * half;            // the last visible key of the lane's, counted from its first
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[kb][e] = kb * 32 + (e & 3) + 8 * (e >> 2) <= behind ? s[kb][e] : -INFINITY;
        }
        if (p.window > 0 && key0 <= last_at - p.window) {
            const int lowest_key = my_at - p.window + 1 - key0 - 4 * half, end_sinks = p.sinks - key0 - 4 * half;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = kb * 32 + (e & 3) + 8 * (e >> 2);
                    s[kb][e] = (key >= lowest_key) | (key < end_sinks) ? s[kb][e] : -INFINITY;
                }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
        mx = max_halves(mx) * c;
        if (__any(mx > m + kSlack || (m == kNothing && mx > kNothing))) {
            const float mn = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] *= f;
        }
        uint4v pf[4];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            float pr[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) pr[e] = __builtin_amdgcn_exp2f(fmaf(s[kk >> 1][(kk & 1) * 8 + e], c, -m));
            pf[kk] = from_floats(pr, BF16);
#pragma unroll
            for (int e = 0; e < 8; ++e) l += pr[e];
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) {
                const int g = lane >> 4, i = lane & 15, channel = cb * 32 + 16 * (g & 1) + 4 * (i & 3);
                union { short4v s4[2]; uint4v v; } vf;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = kk * 16 + 8 * r + 4 * (g >> 1) + (i >> 2);
                    vf.s4[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4)(sm_v + value_offset(row, channel >> 3) + (channel & 7) * 2));
                }
                o[cb] = product<BF16>(vf.v, pf[kk], o[cb]);
            }
        if (it + 1 < n_tiles) logits(sm[(it + 1) & 1][0], s);
    }
    l = add_halves(l);
    if (my_q < n_q) {
        const float f = l > 0.f ? 1.f / l : 0.f;
        __half* dst = p.out.data + (p.q_starts ? 0 : b * p.out.stride_b) + head * p.out.stride_h + (q_row + my_q) * p.out.stride_t;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float r[8] = {o[cb][4 * i] * f, o[cb][4 * i + 1] * f, o[cb][4 * i + 2] * f, o[cb][4 * i + 3] * f, 0.f, 0.f, 0.f, 0.f};
                const uint4v w = from_floats(r, BF16);
                *reinterpret_cast<uint2*>(dst + cb * 32 + 8 * i + 4 * half) = make_uint2(w[0], w[1]);
            }
    }
}

}  // namespace

size_t prompt_workspace_bytes(const PromptParams& p) { return 0; }

hipError_t launch_prompt_attention(const PromptParams& params, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    Args p{};
    static_cast<PromptParams&>(p) = params;
    p.q_tiles = (p.max_q + kQueries - 1) / kQueries;
    // (the copies' lane offsets are 32 bits over four rows)
    if (p.k.stride_t >= 1 << 28 || p.v.stride_t >= 1 << 28) return hipErrorNotSupported;
    const int64_t pairs = (int64_t)p.batch * p.n_kv_heads;
    p.by_die = pairs % 8 == 0 ? (int32_t)(pairs / 8) : 0;
    const int64_t blocks = (int64_t)p.batch * p.n_q_heads * p.q_tiles;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    if (p.bf16) prompt_attention_kernel<true><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(p);
    else prompt_attention_kernel<false><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace kivi
