// Append to the paged cache (kivi_paged_append): rotation on the way, quantisation of the groups that leave the window, and the fp16
// rows that stay.
//
// A sequence's state follows from its length, so every wavefront works out from lengths[b] and the number of new rows
// what there is for it to do.  Two roles:
//   groups  one wavefront per (sequence, group that leaves the window in this call, kv-head, keys or values): loads its 32 tokens out of
//           the fp16 rows or the new ones, rotates the new keys and quantises in registers (kivi_quantize_tile.h)
//   rows    one wavefront per (sequence, new token, eight heads of q, k and v): rotates, and stores queries, and keys and
//           values of tokens that stay in the window
// The roles do not wait for each other.  Rows are stored at slot t % cap_r, groups read slots of tokens before the call: the first read
// is at most n + R + 30 tokens before the last one written, so one launch is right while that is less than cap_r; otherwise
// the rows are a launch after the groups.  (One wavefront for the groups that read slots and the rows that replace them, all in one launch: its
// registers slowed the groups down, 16 x 4096 tokens, 32 heads 305 us against 266.)
//
// Bound: memory for prompts (16 x 4096 tokens, 32 heads 264 us, 4.9 TB/s, as a copy; 16 of them are the rows' launch, which has 83 MB to move), the launch for
// single tokens (32 heads 3.0 us, 64 sequences, 32 / 8 heads with queries 7).  Four tokens per wavefront of the rows: 267; rows of sequences that had
// nothing before in the groups' launch: 272.
//
// The packed codes are a bit contract, so the rotation is one too: fp32 products and one difference, each rounded on its own
// (this file is compiled without contraction), then one rounding to fp16.
#include "kivi_paged.h"
#include "kivi_quantize_tile.h"

#include <algorithm>

namespace kivi {
namespace {

using namespace head_rows;
using tile::half2v;

struct Args : PagedAppendParams {
    FastDiv by_kv_heads, by_groups, by_tokens, by_pieces;
    int32_t groups, tokens, pieces;    // per sequence: groups, tokens looked at; per token: runs of eight heads
    int32_t row_heads;                 // q, k and v
    int32_t group_blocks, group_waves, row_waves;
};

struct Sequence {
    int before, after, first_row, slot;            // tokens before and after the call; the row of its first new token
    bool valid;
};
__device__ __forceinline__ Sequence sequence_of(const Args& p, int b) {
    Sequence s;
    s.after = p.lengths[b];
    const int64_t row0 = p.starts ? p.starts[b] : (int64_t)b * p.max_new;
    const int64_t n = p.starts ? (int64_t)p.starts[b + 1] - row0 : p.max_new;
    s.slot = p.slots ? p.slots[b] : b;
    s.valid = n >= 0 && n <= p.max_new && n <= s.after && row0 >= 0 && row0 + n <= p.n_rows && s.slot >= 0 && s.slot < p.max_sequences;
    s.before = s.after - (int)n;
    s.first_row = (int)row0;
    return s;
}

// Channels 2 lane, 2 lane + 1 of a row of `bits16` after the rotation, from the row's raw pairs; `partner`: the pair of the lane
// that holds the other channels
__device__ __forceinline__ half2v turned_pair(const RotationParams& r, uint32_t raw, bool bf16, bool rotates, int position, int lane) {
    auto pair_of = [&](uint32_t w, float& x, float& y) {
        if (bf16) {
            x = __uint_as_float(w << 16);
            y = __uint_as_float(w & 0xFFFF0000u);
        } else {
            x = (float)tile::as_half2(w).x;
            y = (float)tile::as_half2(w).y;
        }
    };
    float x, y;
    pair_of(raw, x, y);
    if (rotates) {
        const float* row = r.table + (int64_t)position * (2 * r.half);
        const int c = 2 * lane;
        if (r.interleaved) {
            if (c < 2 * r.half) turn_pair(x, y, row[lane], row[r.half + lane]);
        } else {
            const bool low = c < r.half, turns = c < 2 * r.half;
            const int other = turns ? (low ? lane + r.half / 2 : lane - r.half / 2) : lane;
            float px, py;
            pair_of((uint32_t)__shfl((int)raw, other), px, py);
            if (turns) {
                const int i = low ? c : c - r.half;
                const float2 cs = *reinterpret_cast<const float2*>(row + i), sn = *reinterpret_cast<const float2*>(row + r.half + i);
                // (x cos - y sin, y cos + x sin): this lane has the first or the second of the pair
                const float x0 = low ? x : px, x1 = low ? y : py;
                float y0 = low ? px : x, y1 = low ? py : y, a0 = x0, a1 = x1;
                turn_pair(a0, y0, cs.x, sn.x);
                turn_pair(a1, y1, cs.y, sn.y);
                x = low ? a0 : y0;
                y = low ? a1 : y1;
            }
        }
    }
    half2v h;
    h.x = (_Float16)x;
    h.y = (_Float16)y;
    return h;
}

template <int BITS>
__device__ __forceinline__ void pack_group(const Args& p, const Sequence& s, int b, int h, int kv, int record, int lane) {
    const int entry = record >> p.page_shift;
    if (entry >= p.max_pages) return;
    const int page = p.page_table[b * p.page_table_stride + entry];
    if (page < 0 || page >= p.n_pages) return;
    char* rec = p.pages + (((((int64_t)page * p.n_kv_heads + h) << p.page_shift) + (record & ((1 << p.page_shift) - 1))) * record_bytes(BITS));
    constexpr int kWords = kTileTokens * kHeadDim * BITS / 32;
    uint32_t* words = reinterpret_cast<uint32_t*>(rec);
    const int t0 = record * kTileTokens;
    const __half* ring = (kv ? p.v_resid : p.k_resid) + ((int64_t)s.slot * p.n_kv_heads + h) * p.cap_r * kHeadDim;
    const TensorParams& fresh = kv ? p.v : p.k;
    const __half* rows = fresh.data + (int64_t)h * fresh.stride_h + (int64_t)s.first_row * fresh.stride_t;
    int slot0 = t0 % p.cap_r;
    auto row_at = [&](int i) -> const __half* {                // of token t0 + i
        const int t = t0 + i, slot = slot0 + i - (slot0 + i >= p.cap_r ? p.cap_r : 0);
        return t < s.before ? ring + slot * kHeadDim : rows + (int64_t)(t - s.before) * fresh.stride_t;
    };
    if (!kv) {
        uint32_t raw[kTileTokens];
        half2v x[kTileTokens];
#pragma unroll
        for (int i = 0; i < kTileTokens; ++i) raw[i] = *reinterpret_cast<const uint32_t*>(row_at(i) + 2 * lane);
#pragma unroll
        for (int i = 0; i < kTileTokens; ++i) {
            const bool is_new = t0 + i >= s.before;
            x[i] = tile::as_half2(raw[i]);
            if (is_new && (p.bf16 || p.rotates)) {
                int position = t0 + i;
                if (p.rotates) position = clamped_position(p.rotation, p.rotation.positions ? p.rotation.positions[s.first_row + t0 + i - s.before] : position);
                x[i] = turned_pair(p.rotation, raw[i], p.bf16, p.rotates, position, lane);
            }
        }
        half2v* scales = reinterpret_cast<half2v*>(words + kWords);
        tile::quantize_key_tile<BITS>(x, lane,
            [&](half2v s2, half2v z2) {
                scales[lane] = s2;
                scales[64 + lane] = z2;
            },
            [&](int i, uint32_t w) { words[i] = w; });
    } else {
        tile::ValueRow x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i].v4 = *reinterpret_cast<const tile::uint4v*>(row_at((lane >> 4) * 8 + i) + (lane & 15) * 8);
        if (p.bf16) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (t0 + (lane >> 4) * 8 + i >= s.before) {
                    float f[8];
                    to_floats(x[i].v4, true, f);
                    x[i].v4 = from_floats(f, false);
                }
        }
        _Float16* scales = reinterpret_cast<_Float16*>(words + kWords + 128);
        tile::quantize_value_tile<BITS>(x, lane,
            [&](int i, _Float16 sc, _Float16 z) {
                scales[i] = sc;
                scales[128 + i] = z;
            },
            [&](int i, uint32_t w) { words[kWords + 256 + i] = w; });
    }
}

// One row by eight lanes: of a query (which 0), key (1) or value (2) head h of new row `row`, token t of its sequence
__device__ __forceinline__ void store_row(const Args& p, const Sequence& s, int which, int h, int64_t row, int t, int lane) {
    const int j = lane & 7;
    const TensorParams& from = which == 0 ? p.q : which == 1 ? p.k : p.v;
    const __half* src = from.data + row * from.stride_t + h * from.stride_h;
    __half* dst;
    if (which == 0) dst = p.q_out.data + row * p.q_out.stride_t + h * p.q_out.stride_h;
    else dst = (which == 1 ? p.k_resid : p.v_resid) + (((int64_t)s.slot * p.n_kv_heads + h) * p.cap_r + t % p.cap_r) * kHeadDim;
    const Pieces pc = pieces_of(j, p.rotates ? p.rotation.half : 0, p.rotation.interleaved);
    uint4v a4 = *reinterpret_cast<const uint4v*>(src + pc.a * 8), b4 = *reinterpret_cast<const uint4v*>(src + pc.b * 8);
    const bool turns = p.rotates && which != 2 && j < p.rotation.half / 8;
    if (turns || p.bf16) {
        float x[8], y[8];
        to_floats(a4, p.bf16, x);
        to_floats(b4, p.bf16, y);
        if (turns) {
            Turn turn;
            load_turn(p.rotation, clamped_position(p.rotation, p.rotation.positions ? p.rotation.positions[row] : t), j, turn);
            turn_pieces(x, y, turn, p.rotation.interleaved);
        }
        a4 = from_floats(x, false);
        b4 = from_floats(y, false);
    }
    *reinterpret_cast<uint4v*>(dst + pc.a * 8) = a4;
    *reinterpret_cast<uint4v*>(dst + pc.b * 8) = b4;
}

template <int BITS>
__device__ __forceinline__ void group_role(const Args& p, int at, int lane) {
    const int kv = at & 1;
    at >>= 1;
    const int by_heads = p.by_kv_heads.of(at), h = at - by_heads * p.n_kv_heads, b = p.by_groups.of(by_heads), g = by_heads - b * p.groups;
    const Sequence s = sequence_of(p, b);
    const int record = packed_records(s.before, p.residual) + g;
    if (s.valid && record < packed_records(s.after, p.residual)) pack_group<BITS>(p, s, b, h, kv, record, lane);
}

__device__ __forceinline__ void row_role(const Args& p, int at, int lane) {
    const int by_pieces = p.by_pieces.of(at), piece = at - by_pieces * p.pieces, b = p.by_tokens.of(by_pieces), from_end = by_pieces - b * p.tokens;
    const Sequence s = sequence_of(p, b);
    const int t = s.after - 1 - from_end, head = piece * 8 + (lane >> 3);
    if (!s.valid || t < s.before || head >= p.row_heads) return;
    const bool stays = t >= packed_records(s.after, p.residual) * kTileTokens;
    const int n_q = p.q_out.data ? p.n_q_heads : 0, which = head < n_q ? 0 : head < n_q + p.n_kv_heads ? 1 : 2;
    if (which > 0 && !stays) return;
    store_row(p, s, which, which == 0 ? head : which == 1 ? head - n_q : head - n_q - p.n_kv_heads, (int64_t)s.first_row + t - s.before, t, lane);
}

template <int BITS, bool GROUPS, bool ROWS>
__global__ __launch_bounds__(256) void paged_append_kernel(Args p) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (GROUPS && (!ROWS || (int)blockIdx.x < p.group_blocks)) {
        const int at = (int)blockIdx.x * 4 + wave;
        if (at < p.group_waves) group_role<BITS>(p, at, lane);
    } else if (ROWS) {
        const int at = ((int)blockIdx.x - (GROUPS ? p.group_blocks : 0)) * 4 + wave;
        if (at < p.row_waves) row_role(p, at, lane);
    }
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendParams& params, hipStream_t stream) {
    Args p{};
    static_cast<PagedAppendParams&>(p) = params;
    const bool queries = p.q_out.data != nullptr;
    p.groups = (p.max_new - 1) / kTileTokens + 1;
    p.tokens = queries ? p.max_new : std::min(p.max_new, p.residual + kTileTokens - 1);      // (rows that stay, at most)
    p.row_heads = (queries ? p.n_q_heads : 0) + 2 * p.n_kv_heads;
    p.pieces = (p.row_heads + 7) / 8;
    // (batch times heads fits 31 bits)
    const int64_t groups = (int64_t)p.batch * p.n_kv_heads * p.groups * 2, rows_each = (int64_t)p.batch * p.pieces;
    if (rows_each > 0x7fffffff || groups + rows_each * p.tokens > 0x7ffffff0) return hipErrorNotSupported;
    const int64_t rows = rows_each * p.tokens;
    p.group_waves = (int32_t)groups;
    p.row_waves = (int32_t)rows;
    p.group_blocks = (int32_t)((groups + 3) / 4);
    p.by_kv_heads = FastDiv::by(p.n_kv_heads);
    p.by_groups = FastDiv::by(p.groups);
    p.by_tokens = FastDiv::by(p.tokens);
    p.by_pieces = FastDiv::by(p.pieces);
    const unsigned group_blocks = (unsigned)p.group_blocks, row_blocks = (unsigned)((rows + 3) / 4);
    if ((int64_t)p.max_new + p.residual + 30 < p.cap_r) {
        if (p.bits == 2) paged_append_kernel<2, true, true><<<group_blocks + row_blocks, 256, 0, stream>>>(p);
        else paged_append_kernel<4, true, true><<<group_blocks + row_blocks, 256, 0, stream>>>(p);
        return hipGetLastError();
    }
    if (p.bits == 2) paged_append_kernel<2, true, false><<<group_blocks, 256, 0, stream>>>(p);
    else paged_append_kernel<4, true, false><<<group_blocks, 256, 0, stream>>>(p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    paged_append_kernel<2, false, true><<<row_blocks, 256, 0, stream>>>(p);        // (the bits are the groups')
    return hipGetLastError();
}

}  // namespace kivi
