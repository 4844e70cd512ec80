// Attention of prompts over 16-bit keys and values (kivi_prompt_attention): one pass over the keys with the running maximum and sum
// of a softmax, causal, with an optional window and first keys that stay visible.
//
// A row is a query of one head; rows of the heads that share a kv-head stand side by side (row = query * heads + head), so that a tile of rows
// spans few queries: less of a tile is cut off by the mask, and keys and values are read once for all of them.  A wavefront has 32 rows.
// All products are 32x32x16 matrix instructions, and everything is kept transposed so that a row is a lane:
//   S^T = K Q^T    operand rows are keys (out of LDS), columns are rows (in registers): lane (col = lane % 32, half = lane / 32) gets
//                  the logits of keys 8 (i / 4) + 4 half + i % 4, i = 0..15: half of its row's; the other half is 32 lanes away
//   O^T = V^T P^T  the probabilities of a lane are, in the order the lane has them, its share of the second operand of an instruction over
//                  16 keys, so they change neither lane nor order; the value rows are taken in that order too, transposed by the LDS read
//                  (4 keys of one channel per lane and read).
// Masked elements are set to -inf in tiles that the mask cuts; tiles that it leaves empty are not visited.  The running maximum
// starts at a finite number, so that rows which have seen nothing yet stay 0.  It moves only where a logit passes it by more
// than 2^8 (the probabilities are at most 2^8 then, which both types hold); sums and outputs are fp32.
// Probabilities are rounded to the tensors' type, to nearest: an error of 2^-12 (bf16: 2^-9) of each term at most.
//
// Two kernels.  prompt_tiles_kernel: a workgroup has 128 rows and walks over tiles of 64 keys that its four wavefronts share.
// prompt_rows_kernel, where those workgroups would not fill the device or would have 32 rows at most: 32 rows, and one to four wavefronts that take the tiles
// (of 32 keys) in turn, each with buffers of its own and without barriers, and join in LDS; with a workspace, several workgroups share the keys of the same rows, and a second launch joins them.
//
// Tiles arrive by asynchronous copies into two buffers of keys and two of values, one tile ahead; the logits of the next tile are asked for before the
// exponentials of this one, and its maximum before the barrier.  In LDS the 16-byte pieces of a row change place so that no read has bank conflicts.
// Bound: the card's power.  4 x 4096 tokens, 32 / 8 heads, bf16 546 us, 1.01 PFLOP/s (a library product of 8192^3 1.19); on zeros instead of normal numbers it
// runs in 414 us (the product: 1.76 PFLOP/s).  The clock is at 1.8 of 2.4 GHz, matrix instructions take half of the cycles, vector ones 40 %.  What did not help:
// interleaving the two by hand (598-619 us), wavefront priorities (583-594), sums of probabilities by dot products (550), eight wavefronts per workgroup (559),
// the workgroups of one pair after another (555).  8001 tokens, window 2048 and 4 first keys, fp16 263 us (0.89 PFLOP/s); 1001 tokens, 4 heads 13.6.
#include "kivi_prompt.h"

#include <algorithm>
#include <type_traits>

namespace kivi {
namespace {

using namespace head_rows;
typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kWaveRows = 32, kRowBytes = kHeadDim * 2;
constexpr int kComputeUnits = 256;
// Tiles per wavefront from which the keys of a tile of rows are split, and how many are left then, at least.  (One query, 8000 keys before it, 32 / 8 heads, and
// five queries, 7000 keys, 4 heads: not split 84 and 73 us; left 2: 19.4, 17.5; 4: 18.5, 17.0; 8: 22.4, 22.3.  One query, 32 / 8 heads after 1000, 1500, 2000
// keys, not split 14.7, 18.7, 23.0, split 16.5, 16.7, 16.8, which is the second launch and the binding's workspace.)
constexpr int kSplitTiles = 4, kSplitFrom = 10;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;                  // log2 headroom of the running maximum
constexpr float kNothing = -1e30f;             // running maximum of a row that has seen nothing

struct Args : PromptParams {
    FastDiv by_rep;
    int32_t pairs, row_tiles;          // (sequence, kv-head) pairs; tiles of rows of the longest sequence
    int32_t by_die;                    // > 0: pairs per die, each pair's workgroups on one of the eight
    int32_t splits;
    float *part_o, *part_ml;           // workspace: [pair][tile][row][split] outputs; maximum and sum
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

// What a workgroup of 32 or 128 rows has to do
struct Work {
    int b, kv_head, n_q, n_k;
    int64_t q_row, k_row;              // first rows of the sequence in the tensors
    int row0, rows;                    // first row, rows of the sequence and kv-head
    int shift, first_at, last_at;      // query i stands at key i + shift; the first and last of the workgroup's
    bool valid;
};
__device__ __forceinline__ Work work_of(const Args& p, int pair, int tile, int tile_rows) {
    Work w;
    const int rep = p.n_q_heads / p.n_kv_heads;
    w.b = pair / p.n_kv_heads;
    w.kv_head = pair - w.b * p.n_kv_heads;
    w.n_q = p.max_q;
    w.n_k = p.max_k;
    w.q_row = w.k_row = 0;
    w.valid = true;
    if (p.q_starts) {
        const int first = p.q_starts[w.b], end = p.q_starts[w.b + 1];
        w.valid = first >= 0 && end <= p.q_rows && end >= first && (int64_t)end - first <= p.max_q;
        w.n_q = end - first;
        w.q_row = first;
    }
    if (p.k_starts) {
        const int first = p.k_starts[w.b], end = p.k_starts[w.b + 1];
        w.valid = w.valid && first >= 0 && end <= p.k_rows && end >= first && (int64_t)end - first <= p.max_k;
        w.n_k = end - first;
        w.k_row = first;
    }
    w.rows = w.valid ? w.n_q * rep : 0;
    w.row0 = tile * tile_rows;
    w.valid = w.valid && w.row0 < w.rows;
    w.shift = w.n_k - w.n_q;
    w.first_at = p.by_rep.of(w.row0) + w.shift;
    w.last_at = p.by_rep.of(min(w.row0 + tile_rows, max(w.rows, 1)) - 1) + w.shift;
    return w;
}
// The tiles of KEYS keys that some row of the workgroup sees: those of the first keys, then those that the window reaches
template <int KEYS>
struct Tiles {
    int sinks, first, count;           // tiles of the first keys; the first one of the window; all
    __device__ __forceinline__ Tiles(const Args& p, const Work& w) {
        const int lowest = p.window > 0 ? max(w.first_at - p.window + 1, 0) : 0, end = w.last_at < 0 ? 0 : w.last_at / KEYS + 1;
        sinks = p.window > 0 ? min((min(p.sinks, lowest) + KEYS - 1) / KEYS, end) : 0;
        first = max(lowest / KEYS, sinks);
        count = sinks + max(end - first, 0);
    }
    __device__ __forceinline__ int key(int i) const { return (i < sinks ? i : i - sinks + first) * KEYS; }
};
__device__ __forceinline__ const __half* base_of(const TensorParams& t, const int32_t* starts, const Work& w) {
    return t.data + (starts ? 0 : w.b * t.stride_b) + w.kv_head * t.stride_h + w.k_row * t.stride_t;
}

// Copies of 16 rows of a tensor (four per instruction) into LDS.  swap(row): by how much the pieces of a row change place.  Rows are taken in
// order, `step` rows further each time; only skip() moves elsewhere.  (Scalar instructions count: with the rows' addresses made anew for every
// tile a wavefront spent 148 of them per tile, a fifth of its time.)
template <class Swap>
struct Copier {
    uint32_t lane_offset[4];
    const char* next;                  // the next rows
    int64_t stride, advance;           // bytes from row to row, from step to step
    int row;
    __device__ __forceinline__ Copier(const __half* base, int64_t stride_t, int first, int step, int lane, Swap swap)
        : next(reinterpret_cast<const char*>(base) + first * stride_t * 2), stride(stride_t * 2), advance(step * stride_t * 2), row(first) {
#pragma unroll
        for (int i = 0; i < 4; ++i) lane_offset[i] = (uint32_t)(i * 4 + (lane >> 4)) * (uint32_t)stride + (((lane & 15) ^ swap(i * 4 + (lane >> 4))) << 4);
    }
    __device__ __forceinline__ void skip(int rows) {
        next += rows * stride;
        row += rows;
    }
    __device__ __forceinline__ void copy(int n_rows, int step, int lane, uint32_t lds) {
        if (row + 16 <= n_rows) {
#pragma unroll
            for (int i = 0; i < 4; ++i) copy_to_lds(next, lane_offset[i], lds + i * 1024);
        } else {                                                   // rows past the end re-read the last one
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 4 + (lane >> 4), there = min(r, n_rows - 1 - row);
                copy_to_lds(next + there * stride + (int)(lane_offset[i] - (uint32_t)r * (uint32_t)stride), lds + i * 1024);
            }
        }
        next += advance;
        row += step;
    }
};
struct KeySwap { __device__ __forceinline__ int operator()(int row) const { return row & 15; } };
struct ValueSwap { __device__ __forceinline__ int operator()(int row) const { return (row & 3) << 2; } };

// 32 rows of a wavefront; KB: halves of 32 keys in a tile
template <bool BF16, int KB>
struct Rows {
    uint4v qf[8];                      // columns of the first product
    float16v o[4];                     // o[cb][i]: channel 32 cb + 8 (i / 4) + 4 half + i % 4
    float c, m, l;
    int at;                            // where this lane's query stands

    __device__ __forceinline__ void start(const Args& p, const Work& w, int row, int half) {
        const int query = p.by_rep.of(min(row, w.rows - 1)), r = min(row, w.rows - 1) - query * (p.n_q_heads / p.n_kv_heads);
        at = query + w.shift;
        const __half* src = p.q.data + (p.q_starts ? 0 : w.b * p.q.stride_b) + (w.kv_head * (p.n_q_heads / p.n_kv_heads) + r) * p.q.stride_h +
                            (w.q_row + query) * p.q.stride_t + half * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            qf[i] = *reinterpret_cast<const uint4v*>(src + i * 16);
            if (p.softmax_scale < 0.f) qf[i] ^= 0x80008000u;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
        c = fmaxf(fabsf(p.softmax_scale) * kLog2e, 1e-30f);        // (not 0: masked logits stay -inf)
        m = kNothing;
        l = 0.f;
    }
    __device__ __forceinline__ void logits(const unsigned char* sm_k, int lane, float16v (&s)[KB]) const {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[kb] = product<BF16>(*reinterpret_cast<const uint4v*>(sm_k + key_offset(kb * 32 + (lane & 31), 2 * i + (lane >> 5))), qf[i], s[kb]);
        }
    }
    // what the mask hides of a tile that begins with key0
    __device__ __forceinline__ void mask(const Args& p, const Work& w, int key0, int half, float16v (&s)[KB]) const {
        if (key0 + KB * 32 - 1 > w.first_at) {
            const int behind = at - key0 - 4 * half;               // the last visible key, counted from the lane's first
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[kb][e] = kb * 32 + (e & 3) + 8 * (e >> 2) <= behind ? s[kb][e] : -INFINITY;
        }
        if (p.window > 0 && key0 <= w.last_at - p.window) {
            const int lowest = at - p.window + 1 - key0 - 4 * half, end_sinks = p.sinks - key0 - 4 * half;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = kb * 32 + (e & 3) + 8 * (e >> 2);
                    s[kb][e] = ((key >= lowest) | (key < end_sinks)) ? s[kb][e] : -INFINITY;
                }
        }
    }
    // the largest logit of this lane's row in a tile
    __device__ __forceinline__ float largest(const float16v (&s)[KB]) const {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
        return max_halves(mx) * c;
    }
    __device__ __forceinline__ void raise(float mx) {
        if (__any(mx > m + kSlack || (m == kNothing && mx > kNothing))) {
            const float mn = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] *= f;
        }
    }
    __device__ __forceinline__ void add(const unsigned char* sm_v, int lane, const float16v (&s)[KB]) {
        uint4v pf[2 * KB];
#pragma unroll
        for (int kk = 0; kk < 2 * KB; ++kk) {
            float pr[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) pr[e] = __builtin_amdgcn_exp2f(fmaf(s[kk >> 1][(kk & 1) * 8 + e], c, -m));
            pf[kk] = from_floats(pr, BF16);
#pragma unroll
            for (int e = 0; e < 8; ++e) l += pr[e];
        }
#pragma unroll
        for (int kk = 0; kk < 2 * KB; ++kk)
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
    }
};
// four channels of a row
template <bool BF16>
__device__ __forceinline__ void store_four(__half* dst, float a, float b, float c, float d) {
    const float r[8] = {a, b, c, d, 0.f, 0.f, 0.f, 0.f};
    const uint4v w = from_floats(r, BF16);
    *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
}
__device__ __forceinline__ __half* out_row(const Args& p, const Work& w, int row) {
    const int rep = p.n_q_heads / p.n_kv_heads, query = p.by_rep.of(row), r = row - query * rep;
    return p.out.data + (p.q_starts ? 0 : w.b * p.out.stride_b) + (w.kv_head * rep + r) * p.out.stride_h + (w.q_row + query) * p.out.stride_t;
}
__device__ __forceinline__ uint32_t lds_address(unsigned char* p) {
    return (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)p);
}
// (pair, tile) of a workgroup: the tiles with the most keys first; by_die: all workgroups of a pair on one die, whose L2 then has its keys
__device__ __forceinline__ void place_of(const Args& p, int at, int& pair, int& tile) {
    if (p.by_die > 0) {
        pair = (at >> 3) % p.by_die * 8 + (at & 7);
        tile = p.row_tiles - 1 - (at >> 3) / p.by_die;
    } else {
        pair = at % p.pairs;
        tile = p.row_tiles - 1 - at / p.pairs;
    }
}

template <bool BF16>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_tiles_kernel(Args p) {
    constexpr int kKeys = 64, kTileBytes = kKeys * kRowBytes;
    __shared__ __align__(16) unsigned char sm[2][2][kTileBytes];          // [buffer][keys, values]
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int pair, tile;
    place_of(p, blockIdx.x, pair, tile);
    const Work w = work_of(p, pair, tile, kWaves * kWaveRows);
    if (!w.valid) return;
    const int row = w.row0 + wave * kWaveRows + (lane & 31);
    Rows<BF16, 2> r;
    r.start(p, w, row, half);
    const Tiles<kKeys> tiles(p, w);
    const int key_first = tiles.key(0) + wave * 16;
    Copier<KeySwap> keys(base_of(p.k, p.k_starts, w), p.k.stride_t, key_first, kKeys, lane, KeySwap{});
    Copier<ValueSwap> values(base_of(p.v, p.k_starts, w), p.v.stride_t, key_first, kKeys, lane, ValueSwap{});
    const uint32_t lds = lds_address(&sm[0][0][0]) + wave * 16 * kRowBytes;
    const int jump = (tiles.first - tiles.sinks) * kKeys;          // rows between the tiles of the first keys and the window's
    auto copy_keys = [&](int i, int buffer) {
        if (i == tiles.sinks && jump > 0 && i > 0) keys.skip(jump);
        keys.copy(w.n_k, kKeys, lane, lds + buffer * 2 * kTileBytes);
    };
    auto copy_values = [&](int i, int buffer) {
        if (i == tiles.sinks && jump > 0 && i > 0) values.skip(jump);
        values.copy(w.n_k, kKeys, lane, lds + (buffer * 2 + 1) * kTileBytes);
    };
    const int count = tiles.count;
    float16v s[2], next[2];
    if (count > 0) {
        copy_keys(0, 0);
        copy_values(0, 0);
        if (count > 1) copy_keys(1, 1);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        r.logits(sm[0][0], lane, s);
    }
    float mx = 0.f;
    if (count > 0) {
        r.mask(p, w, tiles.key(0), half, s);
        mx = r.largest(s);
    }
    // tile i, whose logits are there, and the next one's logits
    auto step = [&](int i, auto parity, const float16v (&now)[2], float16v (&then)[2]) {
        constexpr int B = decltype(parity)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // this wavefront's rows of the tiles are there,
        lds_barrier();                                             // everybody's, and nobody reads the other buffers any more
        if (i + 2 < count) copy_keys(i + 2, B);
        if (i + 1 < count) copy_values(i + 1, B ^ 1);
        r.raise(mx);
        r.logits(sm[B ^ 1][0], lane, then);                        // (after the last tile: of what the buffer holds, not used)
        r.add(sm[B][1], lane, now);
        r.mask(p, w, tiles.key(i + 1), half, then);
        mx = r.largest(then);
    };
    for (int i = 0; i < count; i += 2) {
        step(i, std::integral_constant<int, 0>{}, s, next);
        if (i + 1 == count) break;
        step(i + 1, std::integral_constant<int, 1>{}, next, s);
    }
    const float l = add_halves(r.l);
    if (row < w.rows) {
        const float f = l > 0.f ? 1.f / l : 0.f;
        __half* dst = out_row(p, w, row) + 4 * half;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int i = 0; i < 4; ++i) store_four<BF16>(dst + cb * 32 + 8 * i, r.o[cb][4 * i] * f, r.o[cb][4 * i + 1] * f, r.o[cb][4 * i + 2] * f, r.o[cb][4 * i + 3] * f);
    }
}

template <bool BF16, int W>
__global__ __launch_bounds__(64 * W, 1) void prompt_rows_kernel(Args p) {
    constexpr int kKeys = 32, kTileBytes = kKeys * kRowBytes;
    __shared__ __align__(16) unsigned char sm[W][2][2][kTileBytes];  // [wavefront][buffer][keys, values]; then outputs [wavefront][channel][row]
    __shared__ float sm_ml[W][2][kWaveRows];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int pair, tile;
    const int at = (int)blockIdx.x / p.splits, split = (int)blockIdx.x - at * p.splits;
    place_of(p, at, pair, tile);
    const Work w = work_of(p, pair, tile, kWaveRows);
    if (!w.valid) return;
    Rows<BF16, 1> r;
    r.start(p, w, w.row0 + col, half);
    const Tiles<kKeys> tiles(p, w);
    // this workgroup's tiles: [from, to), of which the wavefronts take turns
    const int from = (int)((int64_t)tiles.count * split / p.splits), to = (int)((int64_t)tiles.count * (split + 1) / p.splits);
    Copier<KeySwap> keys(base_of(p.k, p.k_starts, w), p.k.stride_t, 0, 16, lane, KeySwap{});
    Copier<ValueSwap> values(base_of(p.v, p.k_starts, w), p.v.stride_t, 0, 16, lane, ValueSwap{});
    const uint32_t lds = lds_address(&sm[wave][0][0][0]);
    auto copy_tile = [&](int i, int buffer) {                      // 16 instructions
        keys.skip(tiles.key(i) - keys.row);
        values.skip(tiles.key(i) - values.row);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            keys.copy(w.n_k, 16, lane, lds + buffer * 2 * kTileBytes + x * 16 * kRowBytes);
            values.copy(w.n_k, 16, lane, lds + (buffer * 2 + 1) * kTileBytes + x * 16 * kRowBytes);
        }
    };
    int buffer = 0;
    if (from + wave < to) copy_tile(from + wave, 0);
    for (int i = from + wave; i < to; i += W) {
        if (i + W < to) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the other buffer's last reads are done
            copy_tile(i + W, buffer ^ 1);
            asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        float16v s[1];
        r.logits(sm[wave][buffer][0], lane, s);
        r.mask(p, w, tiles.key(i), half, s);
        r.raise(r.largest(s));
        r.add(sm[wave][buffer][1], lane, s);
        buffer ^= 1;
    }
    // ---- join the wavefronts ----
    const float lw = add_halves(r.l);
    float* mine = reinterpret_cast<float*>(&sm[wave][0][0][0]);    // [channel][row]
    static_assert(kHeadDim * kWaveRows * sizeof(float) <= sizeof(sm[0]), "outputs of a wavefront");
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int e = 0; e < 16; ++e) mine[(cb * 32 + 8 * (e >> 2) + 4 * half + (e & 3)) * kWaveRows + col] = r.o[cb][e];
    if (half == 0) {
        sm_ml[wave][0][col] = r.m;
        sm_ml[wave][1][col] = lw;
    }
    __syncthreads();
    // 32 channels after the other, this wavefront's first (half: the upper sixteen), of all rows
    float m = kNothing, l = 0.f, f[W];
#pragma unroll
    for (int x = 0; x < W; ++x) m = fmaxf(m, sm_ml[x][0][col]);
#pragma unroll
    for (int x = 0; x < W; ++x) {
        f[x] = __builtin_amdgcn_exp2f(sm_ml[x][0][col] - m);
        l = fmaf(sm_ml[x][1][col], f[x], l);
    }
    const int row = w.row0 + col;
    if (row >= w.rows) return;
#pragma unroll
    for (int cb = wave; cb < 4; cb += W) {
        const int c0 = cb * 32 + half * 16;
        float o[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            o[e] = 0.f;
#pragma unroll
            for (int x = 0; x < W; ++x) o[e] = fmaf(reinterpret_cast<const float*>(&sm[x][0][0][0])[(c0 + e) * kWaveRows + col], f[x], o[e]);
        }
        if (p.splits == 1) {
            const float g = l > 0.f ? 1.f / l : 0.f;
            __half* dst = out_row(p, w, row) + c0;
#pragma unroll
            for (int e = 0; e < 16; e += 4) store_four<BF16>(dst + e, o[e] * g, o[e + 1] * g, o[e + 2] * g, o[e + 3] * g);
        } else {
            const int64_t part = (((int64_t)pair * p.row_tiles + tile) * kWaveRows + col) * p.splits + split;
            float4v* dst = reinterpret_cast<float4v*>(p.part_o + part * kHeadDim + c0);
#pragma unroll
            for (int e = 0; e < 16; e += 4) dst[e / 4] = float4v{o[e], o[e + 1], o[e + 2], o[e + 3]};
            if (c0 == 0) *reinterpret_cast<float2*>(p.part_ml + part * 2) = make_float2(m, l);
        }
    }
}

// Joins the parts of prompt_rows_kernel: 32 lanes per row, four channels each
template <bool BF16>
__global__ __launch_bounds__(256) void prompt_join_kernel(Args p) {
    const int at = (int)blockIdx.x * 8 + (int)(threadIdx.x >> 5), c = (threadIdx.x & 31) * 4;
    const int tile_at = at / kWaveRows, pair = tile_at / p.row_tiles, tile = tile_at - pair * p.row_tiles;
    if (pair >= p.pairs) return;
    const Work w = work_of(p, pair, tile, kWaveRows);
    const int row = w.row0 + at % kWaveRows;
    if (!w.valid || row >= w.rows) return;
    const int64_t part = (((int64_t)pair * p.row_tiles + tile) * kWaveRows + at % kWaveRows) * p.splits;
    float m = kNothing, l = 0.f;
    for (int s = 0; s < p.splits; ++s) m = fmaxf(m, p.part_ml[(part + s) * 2]);
    float4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + (part + s) * 2);
        const float f = __builtin_amdgcn_exp2f(ml.x - m);
        l = fmaf(ml.y, f, l);
        o += *reinterpret_cast<const float4v*>(p.part_o + (part + s) * kHeadDim + c) * f;
    }
    const float f = l > 0.f ? 1.f / l : 0.f;
    store_four<BF16>(out_row(p, w, row) + c, o[0] * f, o[1] * f, o[2] * f, o[3] * f);
}

// What a call runs: tiles of 128 rows, or of 32 by `waves` wavefronts with `splits` workgroups each
struct Plan { bool small; int waves, splits; };
Plan plan_of(const PromptParams& p) {
    const int64_t rows = (int64_t)p.max_q * (p.n_q_heads / p.n_kv_heads), pairs = (int64_t)p.batch * p.n_kv_heads;
    const int64_t groups = pairs * ((rows + kWaveRows - 1) / kWaveRows);
    Plan plan{false, kWaves, 1};
    if (rows == 0) return plan;
    // (124 workgroups of 128 rows, 4 heads x 3900 tokens: 79.8 us, in rows of 32 50.6; 64 of them, 2000 tokens: 44.4, 25.9; 160, 2 x 600, 16 / 8 heads: 18.0,
    // 21.9; 220, 7000 tokens, window 500: 24.0, 44.3)
    plan.small = rows <= kWaveRows || pairs * ((rows + 127) / 128) <= kComputeUnits / 2;
    // One tile of rows per pair leaves three wavefronts of a 128-row workgroup idle.  Four wavefronts take a compute unit's LDS, so more workgroups than
    // compute units have two each, or one.  (128 rows, 4, 2, 1 wavefronts: 288 pairs, 5 tokens after 315 16.0, 18.4, 13.8, 16.8 us; 512, 20 after 500 28.1, 29.4,
    // 26.0, 26.3; 1600, 32 / 8 heads, 1 after 100 28.6, 36.4, 27.8, 22.8; 1888, 13 tokens 23.3, 37.6, 20.0, 12.5)
    if (rows <= kWaveRows) plan.waves = groups <= kComputeUnits ? 4 : groups <= 2 * kComputeUnits ? 2 : 1;
    if (plan.small) {
        // keys that a tile of rows sees at most, in tiles
        int64_t keys = p.max_k;
        if (p.window > 0) keys = std::min<int64_t>(keys, (int64_t)p.window + kWaveRows + std::min(p.sinks, p.max_k));
        const int64_t tiles = (keys + 31) / 32;
        if (tiles >= kWaves * kSplitFrom) plan.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kComputeUnits / groups, tiles / (kWaves * kSplitTiles)));
    }
    return plan;
}

}  // namespace

size_t prompt_workspace_bytes(const PromptParams& p) {
    const Plan plan = plan_of(p);
    if (plan.splits == 1) return 0;
    const size_t rows = (size_t)p.max_q * (p.n_q_heads / p.n_kv_heads), tiles = (rows + kWaveRows - 1) / kWaveRows;
    return (size_t)p.batch * p.n_kv_heads * tiles * kWaveRows * plan.splits * (kHeadDim + 2) * sizeof(float);
}

hipError_t launch_prompt_attention(const PromptParams& params, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    Args p{};
    static_cast<PromptParams&>(p) = params;
    // (the copies' lane offsets are 32 bits over 16 rows)
    const int rep = p.n_q_heads / p.n_kv_heads;
    const int64_t rows = (int64_t)p.max_q * rep, pairs = (int64_t)p.batch * p.n_kv_heads;
    if (p.k.stride_t >= 1 << 26 || p.v.stride_t >= 1 << 26) return hipErrorNotSupported;
    Plan plan = plan_of(p);
    if (!workspace || workspace_bytes < prompt_workspace_bytes(p)) plan.splits = 1;
    const int tile_rows = plan.small ? kWaveRows : kWaves * kWaveRows;
    p.by_rep = FastDiv::by(rep);
    p.pairs = (int32_t)pairs;
    p.row_tiles = (int32_t)((rows + tile_rows - 1) / tile_rows);
    p.splits = plan.splits;
    p.by_die = pairs % 8 == 0 ? (int32_t)(pairs / 8) : 0;
    const int64_t blocks = pairs * p.row_tiles * plan.splits;
    if (blocks > 0x7fffffff) return hipErrorNotSupported;
    if (!plan.small) {
        if (p.bf16) prompt_tiles_kernel<true><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(p);
        else prompt_tiles_kernel<false><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(p);
        return hipGetLastError();
    }
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o + (size_t)pairs * p.row_tiles * kWaveRows * plan.splits * kHeadDim;
#define KIVI_ROWS(W) p.bf16 ? prompt_rows_kernel<true, W><<<(unsigned)blocks, 64 * W, 0, stream>>>(p) : prompt_rows_kernel<false, W><<<(unsigned)blocks, 64 * W, 0, stream>>>(p)
    if (plan.waves == 4) KIVI_ROWS(4);
    else if (plan.waves == 2) KIVI_ROWS(2);
    else KIVI_ROWS(1);
#undef KIVI_ROWS
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || plan.splits == 1) return e;
    const int64_t join_blocks = pairs * p.row_tiles * kWaveRows / 8;
    if (p.bf16) prompt_join_kernel<true><<<(unsigned)join_blocks, 256, 0, stream>>>(p);
    else prompt_join_kernel<false><<<(unsigned)join_blocks, 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace kivi
