// Attention of one token per sequence over the paged cache (kivi_paged_attention).
//
// Work: a unit is (sequence, kv-head, run of up to eight query heads).  What a unit has to visit -- its visible records and tiles of 32
// fp16 rows -- follows from the sequence's length, and is put on one axis for all units, in steps of one record or tile per
// wavefront.  Every workgroup adds up the lengths by itself (sums across lanes without LDS) and takes one interval of the axis, so the
// device is divided evenly whatever the lengths, and nothing but the batch's size is known to the host: a captured call follows lengths and
// pages.  Where no piece gets longer (few units, short ones), each unit is cut evenly on its own instead, and no workgroup
// enters two: 8 sequences of 500 tokens, 32 / 8 heads 20.6 -> 12.6 us.  A unit that lies in one interval is written out by it; of one that several
// share each leaves a part (maximum, sum, outputs) in the workspace, and the last to come joins them.  A workgroup shares its first and its
// last unit at most, so the workspace has two parts per workgroup whatever the batch; a unit is counted where its first workgroup is.  Entering and leaving
// a unit has its place on the axis too, in front of the unit's steps; an interval that begins in it begins with the steps.
//
// Products: 16x16x32 matrix instructions; operand rows are tokens (keys) and channels (values), columns are query heads.  Lane
// (n = lane % 16, kb = lane / 16) makes the eight contraction elements 8 kb .. 8 kb + 7 of column n: head n % HP; n < 8: rounded products, n >= 8: what
// the rounding left, so that a pair of columns together has 21 bits.  (Rounded products alone: 2e-4 of the output by estimate, as much as its own rounding.)  Codes
// are operands as they are, as subnormal fp16 numbers (their place in the 16 bits is a power of two that goes into the other factor); scales go into the
// other operand:
//   logit_t = sum_c code_tc (s_c q_c) + sum_c z_c q_c,     o_c = sum_t code_tc (p_t s_tg) + sum_t p_t z_tg
// Queries enter times a power of two that puts the largest element into [2^8, 2^9), probabilities times 2^8 (4 bits: 2^11); tiles with
// scales that could leave fp16's range with that (keys 2^6, values 2^3; 4 bits 2^0) take the scales 2^-9, or from then on the probabilities 2^-4.
// The running maximum moves where a logit passes it by more than 2^4.  One query head per kv-head (HP = 1) makes the same products in another
// way, below at record_one: 32 x 16 001 tokens, window 4096 99 -> 82 us, 16 x 4096 53 -> 46, 4 bits 8 x 8191, 40 heads 79 -> 78.
//
// A record is one contiguous piece of memory, so it takes three (4 bits: five) asynchronous copies of 1 KB into the wavefront's own ring in LDS,
// NB records ahead, across unit borders, without barriers; the page number comes through the scalar cache.  fp16 rows are loaded straight into
// registers: keys are operands as they are, value rows are turned by byte permutes.
//
// Bound: issue of vector instructions and memory, which overlap in part: of 64 sequences of 500-8000 tokens (32 / 8 heads, 2 bits, 257 MB) the copies
// alone take 49 us, the arithmetic alone 46, both 59 (4.4 TB/s); 12 us of each are what a launch pays once (lengths, first page, first record: 5; leaving units,
// counting, joining: 7).  16 x 32 767 tokens, 64 / 8 heads, 4 bits 121 us (5.6 TB/s); 32 x 16 001 tokens, 32 heads, window 4096 82 (5.6 TB/s);
// one sequence of 3001 tokens, 32 heads 13.5.  Four wavefronts per SIMD (128 registers) spill: 64 -> 104 us; a ring of four records at 2 bits, units counted
// at the end of an interval, the first fp16 rows asked for with the query (spills), priorities that also fall with a workgroup's age: no gain.  Operands
// through LDS as at record_one for two and four heads as well: a sixth fewer vector instructions, as fast at 2 bits, 75 -> 83 us at 4.
#include "kivi_paged.h"

#include <algorithm>

namespace kivi {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

union Frag {                           // one lane's share of an operand: eight halves
    half8 h;
    half2v p[4];
    uint32_t r[4];
    uint4v v;
};

constexpr int kWaves = 4;
constexpr int kWorkgroups = 768;       // three per compute unit; a multiple of the eight dies
// What entering and leaving a unit costs in steps of records, before its first step on the axis.  (A step of fp16 rows is as many as one of records.
// 0, 2, 3, 4 with rows 1; 0, 2, 3 with rows 2: 64 x 500-8000 tokens, 32 / 8 heads -, 60, 58.6, 61; 66, 61, 63 us; 200 x 500-2000 -, 63, 61, 64; 67, 66, 64;
// 64 x 500-8000, 64 / 8 -, 71, 66, 67; 73, 70, 71.)
constexpr int kUnitCost = 3;
constexpr int kJoined = 8;             // parts that are loaded at a time where they are joined
// Steps of an interval, at least; 1 where units have kJoined steps or fewer.  (1, 2, 3: 8 sequences of 500 tokens, 32 / 8 heads 12.5, 14.2, 15.9 us; 4 heads x 1023
// tokens 10.9, 9.6, 11.1; 8000 tokens, 32 / 8 heads 20.9, 18.4, 19.3; one sequence of 3001 tokens, 32 / 8 heads 15.6, 14.9, 16.8.)
constexpr int kMinCost = 2;
constexpr int kScanned = 4;            // times 64 sequences whose costs stay in registers
constexpr int kMaxHeads = 8;           // query heads of a unit
constexpr int kPartFloats = kHeadDim;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kKeyUnscale = 4194304.0f, kValueUnscale = 262144.0f;   // codes enter times 2^-22, 2^-18
constexpr int kSlack = 4;
constexpr int kQueryExp = 8;
constexpr uint32_t kKeyScaleLimit = 0x5400u;                           // 64
constexpr int kKeyScaleShift = 9;
template <int BITS> constexpr int kProbExp = BITS == 2 ? 8 : 11;
template <int BITS> constexpr uint32_t kValueScaleLimit = BITS == 2 ? 0x4800u : 0x3C00u;      // 8, 1
constexpr float kNothing = -1e30f;     // running maximum of a row that has seen nothing

template <int CTRL>
__device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true)); }
constexpr int kRor8 = 0x128;           // the other column of a head
constexpr int kRor4 = 0x124;
template <int BANKS>                   // x of the other column in the lanes of BANKS, own in the others
__device__ __forceinline__ half2v from_partner(half2v own, half2v x) {
    return __builtin_bit_cast(half2v, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, own), __builtin_bit_cast(int, x), kRor8, 0xF, BANKS, false));
}
constexpr int kHiLanes = 0x3, kLoLanes = 0xC;
__device__ __forceinline__ float add_rows(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
    x = __int_as_float(a[0]) + __int_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    return __int_as_float(b[0]) + __int_as_float(b[1]);
}
__device__ __forceinline__ float max_rows(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
    x = fmaxf(__int_as_float(a[0]), __int_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    return fmaxf(__int_as_float(b[0]), __int_as_float(b[1]));
}
// sum of this and the lanes before
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_from(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ int sum_upto(int x) {
    x = add_from<0x111, 0xF>(x);       // 1, 2, 4, 8 lanes before, within 16
    x = add_from<0x112, 0xF>(x);
    x = add_from<0x114, 0xF>(x);
    x = add_from<0x118, 0xF>(x);
    x = add_from<0x142, 0xA>(x);       // the last of 16 to the next 16, the last of 32 to the next 32
    return add_from<0x143, 0xC>(x);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141;
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp<kXor1>(x);
    x += dpp<kXor2>(x);
    x += dpp<kHalfMirror>(x);
    return add_rows(x + dpp<kRor8>(x));
}
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, dpp<kXor1>(x));
    x = fmaxf(x, dpp<kXor2>(x));
    x = fmaxf(x, dpp<kHalfMirror>(x));
    return max_rows(fmaxf(x, dpp<kRor8>(x)));
}
// Products of two fp16 numbers with fp32 ones as x = hi + lo 2^-11.  a, b: the fp32 factors, a_up, b_up: 2^11 times those.
constexpr float kLoMagnify = 2048.f, kLoShrink = 1.f / 2048.f;
__device__ __forceinline__ void split_products(half2v s, float a, float b, float a_up, float b_up, half2v& hi, half2v& lo) {
    // (fused operations with a zero, or with fp16 results: one mixed-precision instruction each)
    hi = half2v{(_Float16)fmaf((float)s[0], a, 0.f), (_Float16)fmaf((float)s[1], b, 0.f)};
    asm("" : "+v"(hi));                // (or its upper half is made twice)
    lo = half2v{(_Float16)fmaf((float)hi[0], -kLoMagnify, fmaf((float)s[0], a_up, 0.f)),
                (_Float16)fmaf((float)hi[1], -kLoMagnify, fmaf((float)s[1], b_up, 0.f))};
}
__device__ __forceinline__ half2v pack_rtz(float a, float b) { return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(a, b)); }
__device__ __forceinline__ float2 load_shared(const float* p) {      // of what another workgroup has stored
    return __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ void store_shared(float* p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, make_float2(x, y)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Code operands: tile coordinate u = 2 pair + odd, see include/kivi.h; codes as high in the subnormals as the ten bits allow
template <int BITS>
__device__ __forceinline__ half8 key_fragment(const uint32_t* w, int pair, int odd) {
    Frag f;
    if constexpr (BITS == 2) {
        const uint32_t x = odd ? w[pair] >> 6 : w[pair] << 2;
        f.r[0] = x & 0x000C000Cu; f.r[1] = x & 0x00300030u;
        f.r[2] = x & 0x00C000C0u; f.r[3] = x & 0x03000300u;
    } else {
        const uint32_t x0 = odd ? w[pair * 2] >> 6 : w[pair * 2] << 2, x1 = odd ? w[pair * 2 + 1] >> 6 : w[pair * 2 + 1] << 2;
        f.r[0] = x0 & 0x003C003Cu; f.r[1] = x0 & 0x03C003C0u;
        f.r[2] = x1 & 0x003C003Cu; f.r[3] = x1 & 0x03C003C0u;
    }
    return f.h;
}
template <int BITS>
__device__ __forceinline__ half8 value_fragment(const uint32_t* w, int pair, int odd) {
    Frag f;
    if constexpr (BITS == 2) {
        const uint32_t x = odd ? w[pair] >> 2 : w[pair] << 6, y = odd ? w[pair] >> 6 : w[pair] << 2;
        f.r[0] = x & 0x00C000C0u; f.r[1] = x & 0x03000300u;
        f.r[2] = y & 0x00C000C0u; f.r[3] = y & 0x03000300u;
    } else {
        const uint32_t w0 = w[pair * 2], w1 = w[pair * 2 + 1];
        f.r[0] = (odd ? w0 >> 2 : w0 << 6) & 0x03C003C0u; f.r[1] = (odd ? w0 >> 6 : w0 << 2) & 0x03C003C0u;
        f.r[2] = (odd ? w1 >> 2 : w1 << 6) & 0x03C003C0u; f.r[3] = (odd ? w1 >> 6 : w1 << 2) & 0x03C003C0u;
    }
    return f.h;
}

__device__ __forceinline__ void wave_lds_sync() {      // LDS instructions of one wavefront execute in order
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}
// Workgroup barrier that orders LDS traffic only (a __syncthreads() would also wait for the copies in flight)
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
// Wave-uniform read of what earlier work left in memory, through the scalar cache
__device__ __forceinline__ int scalar(const int32_t* base, int64_t i) {
    return reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(base))[i];
}
// Asynchronous copy of 16 bytes per lane to LDS offset lds + 16 lane.  (Wait states between a vector instruction that writes the scalar operand and
// this one: the compiler does not look into the block.  m0 is a reserved register, so the compiler warns that it keeps no value there: nor shall it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t lane_offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(lane_offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void wait_copies() {        // at most N vector-memory operations still in flight
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

struct Args : PagedAttentionParams {
    int32_t runs, run;                 // runs of query heads per kv-head, heads of a run
    FastDiv by_runs;
};

// What a sequence shows its newest token
struct View {
    int length, packed;                // tokens; records
    int lowest;                        // first token of the window
    int sinks;                         // visible first tokens before it
    int records, sink_records, skip;   // visible records: i < sink_records: i, else i + skip
    int row0, row_tiles;               // first token of the first tile of fp16 rows, tiles of 32
    int row_steps, steps;
    __device__ __forceinline__ int cost() const { return row_steps + steps; }
};
__device__ __forceinline__ View view_of(const Args& p, int length) {
    View v;
    v.length = length;
    const int all = packed_records(v.length, p.residual);
    v.packed = min(all, p.max_pages << p.page_shift);                  // (records behind the table are masked)
    v.lowest = p.window > 0 ? max(v.length - p.window, 0) : 0;
    v.sinks = min(p.sinks, v.lowest);
    if (p.window == 0) v.sinks = 0;
    const int from = min(v.lowest / kTileTokens, v.packed);
    v.sink_records = min((v.sinks + kTileTokens - 1) / kTileTokens, from);
    v.skip = from - v.sink_records;
    v.records = v.packed - v.skip;
    const int rows0 = all * kTileTokens;
    // (tiles before the window are left out, unless first tokens are among them)
    v.row0 = v.sinks > rows0 || v.lowest <= rows0 ? rows0 : rows0 + (v.lowest - rows0) / kTileTokens * kTileTokens;
    v.row_tiles = (v.length - v.row0 + kTileTokens - 1) / kTileTokens;
    v.row_steps = (v.row_tiles + kWaves - 1) / kWaves;
    v.steps = (v.records + kWaves - 1) / kWaves;
    if (v.row_steps + v.steps == 0) v.steps = 1;                       // (nothing of it is visible: its rows become 0)
    return v;
}
template <int BITS, int HP>
__global__ __launch_bounds__(64 * kWaves, 3) void paged_attention_kernel(Args p) {
    constexpr int kCodeBytes = kTileTokens * kHeadDim * BITS / 8, kPlanes = BITS / 2, kScaleOff = kCodeBytes;
    constexpr int kRecord = record_bytes(BITS), NI = kRecord / 1024;   // copy instructions of a record
    constexpr int NB = BITS == 2 ? 3 : 2;                              // records in flight per wavefront
    constexpr int NS = HP / 2;                                         // value-side operands: columns of a head share the channel groups
    constexpr int HR = BITS == 4 && HP == 8 ? 4 : HP;                  // heads that meet in LDS at once
    __shared__ __align__(16) unsigned char sm_ring[kWaves][NB][kRecord];
    __shared__ __align__(16) float sm_o[kWaves][HR][kHeadDim];
    __shared__ float sm_ml[kWaves][HP][2];
    // HP = 1, operands of a record: key side rounded products (128), 16 halves of skew, remainders; value side 8 columns of 32 tokens
    constexpr int kKeyColumn = 144, kOperandHalves = HP == 1 ? 272 : 8;
    __shared__ __align__(16) _Float16 sm_operand[kWaves][kOperandHalves];
    __shared__ int sm_last;
    static_assert(sizeof(sm_ring) + sizeof(sm_o) + sizeof(sm_ml) + sizeof(sm_operand) + 16 <= 160 * 1024 / 3 / 1280 * 1280, "three workgroups per compute unit");
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kb = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool is_lo = n >= 8;
    const int head = n & (HP - 1);
    const int row_pos = (n & 3) | ((n >> 3) & 1) << 2 | ((n >> 2) & 1) << 3;        // operand row m holds token row_pos of its half
    const int tok0 = (kb & 1) * 8 + (kb >> 1) * 4, tok = tok0 + (is_lo ? 16 : 0);   // this lane's tokens: tok + i
    const int my_group = HP == 1 ? (n & 1) * 2 + ((n >> 1) & 1) : HP == 2 ? (n >> 1) & 3 : HP == 4 ? (n >> 2) & 1 : 0;
    const int rep = p.n_q_heads / p.n_kv_heads, units_per_sequence = p.n_kv_heads * p.runs;

    // ---- this workgroup's interval of the axis ----
    const int wg = ((int)blockIdx.x & 7) * (kWorkgroups / 8) + ((int)blockIdx.x >> 3);      // neighbours on the axis share a die
    // (a sequence without tokens or with a slot outside the cache: 0)
    auto length_of = [&](int b) {
        const int slot = p.slots ? p.slots[b] : b;
        return slot >= 0 && slot < p.max_sequences ? max(p.lengths[b], 0) : 0;
    };
    auto cost_of = [&](int tokens) { return tokens > 0 ? view_of(p, tokens).cost() : 0; };
    auto sum_all = [&](int x) { return __builtin_amdgcn_readlane(sum_upto(x), 63); };
    int tokens[kScanned], costs[kScanned];                             // of the first sequences, 64 at a time
    int total = 0, units = 0;
#pragma unroll
    for (int i = 0; i < kScanned; ++i) {
        tokens[i] = costs[i] = 0;
        if (i * 64 < p.batch) {
            if (i * 64 + lane < p.batch) tokens[i] = length_of(i * 64 + lane);
            costs[i] = cost_of(tokens[i]);
            const int some = __popcll(__ballot(costs[i] > 0));
            total += (sum_all(costs[i]) + some * kUnitCost) * units_per_sequence;
            units += some * units_per_sequence;
        }
    }
    for (int b0 = kScanned * 64; b0 < p.batch; b0 += 64) {
        const int cost = b0 + lane < p.batch ? cost_of(length_of(b0 + lane)) : 0;
        total += sum_all(cost > 0 ? cost + kUnitCost : 0) * units_per_sequence;
    }
    if (total == 0) return;
    // An interval of `length` of the axis for every workgroup, or, where no piece gets longer, every unit cut evenly on its own: `length`
    // is then the longest piece, and no workgroup enters two units.
    int length = max((total + kWorkgroups - 1) / kWorkgroups, kMinCost);
    bool own_pieces = false;
    if (p.batch <= kScanned * 64 && units < kWorkgroups) {
        auto fits = [&](int piece) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < kScanned; ++i)
                if (i * 64 < p.batch) n += sum_all((costs[i] + piece - 1) / piece) * units_per_sequence;
            return n <= kWorkgroups;
        };
        own_pieces = fits(length);
        if (own_pieces) {
            int low = max((total - units * kUnitCost + kWorkgroups - 1) / kWorkgroups, kMinCost), high = length;
            while (low < high) {
                const int mid = (low + high) / 2;
                if (fits(mid)) high = mid;
                else low = mid + 1;
            }
            length = low;
            bool few = length == kMinCost;
#pragma unroll
            for (int i = 0; i < kScanned; ++i) few = few && !__any(costs[i] > kJoined);
            if (few && fits(1)) length = 1;
        }
    }
    // what of the axis is in front of a sequence: workgroups with pieces of their own, cost otherwise
    const int unit_cost = own_pieces ? 0 : kUnitCost;
    auto share_of = [&](int cost) { return (own_pieces ? (cost + length - 1) / length : cost > 0 ? cost + unit_cost : 0) * units_per_sequence; };
    const int x_first = own_pieces ? wg : wg * length;
    int b = -1, before = 0, n_tokens = 0;                              // the sequence of this workgroup's first unit, and where it begins
    {
        int sum = 0;
        auto look = [&](int b0, int length, int cost) {
            const int mine = share_of(cost), upto = sum_upto(mine);
            const uint64_t here = __ballot(sum + upto > x_first);
            if (here) {
                const int at = __builtin_ctzll(here);
                b = b0 + at;
                before = sum + __builtin_amdgcn_readlane(upto - mine, at);
                n_tokens = __builtin_amdgcn_readlane(length, at);
            }
            sum += __builtin_amdgcn_readlane(upto, 63);
        };
#pragma unroll
        for (int i = 0; i < kScanned; ++i)
            if (b < 0 && i * 64 < p.batch) look(i * 64, tokens[i], costs[i]);
        for (int b0 = kScanned * 64; b < 0 && b0 < p.batch; b0 += 64) {
            const int n = b0 + lane < p.batch ? length_of(b0 + lane) : 0;
            look(b0, n, cost_of(n));
        }
    }
    b = __builtin_amdgcn_readfirstlane(b);
    before = __builtin_amdgcn_readfirstlane(before);
    n_tokens = __builtin_amdgcn_readfirstlane(n_tokens);
    if (b < 0) return;                                                 // (more workgroups than pieces, or than intervals)
    // A place on the axis: sequence, unit in it, and where the unit's steps begin
    struct Place { int b, unit, unit0; View view; };
    int x0, x1, pieces = 1, piece = 0;                                 // the interval; own pieces: of the unit
    auto next_unit = [&](Place& u) {                                   // (only where another one follows)
        u.unit0 += u.view.cost() + unit_cost;
        if (++u.unit == units_per_sequence) {
            u.unit = 0;
            int n = 0, slot = -1;
            while (++u.b < p.batch) {
                n = scalar(p.lengths, u.b);
                slot = p.slots ? scalar(p.slots, u.b) : u.b;
                if (n > 0 && slot >= 0 && slot < p.max_sequences) break;
            }
            if (u.b >= p.batch) {                                      // (lengths that change under the call: it ends here)
                u.b = p.batch - 1;
                u.unit0 = x1;
                n = 0;
            }
            u.view = view_of(p, n);
        }
    };
    Place here;
    here.b = b;
    here.view = view_of(p, n_tokens);
    {
        const int cost = here.view.cost();
        if (own_pieces) {
            pieces = (cost + length - 1) / length;
            here.unit = (wg - before) / pieces;
            piece = wg - before - here.unit * pieces;
            here.unit0 = 0;
            x0 = cost * piece / pieces;
            x1 = cost * (piece + 1) / pieces;
        } else {
            here.unit = (x_first - before) / (cost + unit_cost);
            here.unit0 = before + here.unit * (cost + unit_cost) + unit_cost;
            x0 = x_first;
            x1 = min(x0 + length, total);
            if (here.unit0 >= x1) return;                              // (nothing but what comes before the steps)
        }
    }
    // its steps of records in this interval: [first, end)
    auto records_from = [&](const Place& u) { return max(x0 - u.unit0 - u.view.row_steps, 0); };
    auto records_to = [&](const Place& u) { return u.view.records > 0 ? max(min(x1 - u.unit0, u.view.cost()) - u.view.row_steps, 0) : 0; };

    // ---- copies of records into this wavefront's ring, NB ahead ----
    const uint32_t ring_lds = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)&sm_ring[wave][0][0]);
    const uint32_t lane16 = lane * 16;
    Place cursor = here;
    // of the cursor's unit: row of the page table, the kv-head's records of page 0, this wavefront's next record, the last record, steps left
    const int32_t* c_table;
    const char* c_base;
    int c_record, c_last, c_left;
    const int64_t page_bytes = ((int64_t)p.n_kv_heads << p.page_shift) * kRecord;
    auto enter_unit = [&](int first) {
        c_table = p.page_table + cursor.b * p.page_table_stride;
        c_base = p.pages + ((int64_t)p.by_runs.of(cursor.unit) << p.page_shift) * kRecord;
        c_record = first * kWaves + wave;
        c_last = cursor.view.records - 1;
        c_left = records_to(cursor) - first;
    };
    enter_unit(records_from(cursor));
    int c_slot = 0, in_flight = 0;
    uint32_t lost = 0;                                                 // slots whose record has no page
    auto advance_copy = [&]() {
        while (c_left <= 0) {
            if (cursor.unit0 + cursor.view.cost() + unit_cost >= x1) return;
            next_unit(cursor);
            enter_unit(0);
        }
        const int i = min(c_record, c_last);                           // (no record for this wavefront: any)
        const int r = i < cursor.view.sink_records ? i : i + cursor.view.skip;
        int page = scalar(c_table, r >> p.page_shift);
        c_record += kWaves;
        --c_left;
        const uint32_t bit = 1u << c_slot;
        lost &= ~bit;
        if ((uint32_t)page >= (uint32_t)p.n_pages) {
            page = 0;
            lost |= bit;
        }
        const char* rec = c_base + page * page_bytes + (r & ((1 << p.page_shift) - 1)) * kRecord;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // the slot's last readers have their data
#pragma unroll
        for (int j = 0; j < NI; ++j) copy_to_lds(rec + j * 1024, lane16, ring_lds + c_slot * kRecord + j * 1024);
        c_slot = c_slot + 1 == NB ? 0 : c_slot + 1;
        ++in_flight;
    };
    auto wait_oldest = [&]() {
        if (in_flight >= NB) wait_copies<(NB - 1) * NI>();
        else if (NB > 2 && in_flight == 2) wait_copies<NI>();
        else wait_copies<0>();
        --in_flight;
    };

    // ---- state of a wavefront ----
    float4v acc[8];                    // code sums: acc[u][i] = channel 16 u + 4 kb + i, column n
    float4v zsum;                      // zero-point sums: channel group i, column n
    float m, l, prob_exp;              // running maximum (log2 domain), this lane's sum, exponent of the probabilities
    half2v qz[4][4], qk[4][4];         // q 2^a; times 1 / place of the codes
    half2v q_zero[4];                  // HP < 8: q 2^a of channel block n / 4
    float c_code, c_zero;              // logit = code sum * c_code + zero sum * c_zero
    half2v rounded[4] = {};            // keys' products in the lo columns, 0 in the hi columns
    // HP = 1: the token of every record, and the channel groups 2 own_pair, + 1, whose value operand this lane makes; log2 of the factor of that
    // token's codes; this lane's channels 2 lane, + 1 of q 2^a over the codes' places, 2^11 times those, and as they are; sums of this lane's
    // probabilities and zero-points
    const int own_i = (n >> 1) & 3, own_pair = n & 1, own_tok = kb * 4 + own_i + (is_lo ? 16 : 0);
    const float own_exp = BITS == 2 && (own_i & 2) ? 2.f : 0.f;
    float own_q[2], own_q_up[2], l_own = 0.f, z_own[2] = {0.f, 0.f};
    half2v own_qz;
    constexpr uint64_t kLoColumns = 0xFF00FF00FF00FF00ull;

    auto set_query = [&](const half8 (&raw)[4], half2v own) {
        float mx = 0.f;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf((float)raw[cb][e]));
        mx = max_rows(mx);
        const bool on = mx > 0.f;
        const int a = on ? min(kQueryExp + 127 - (int)(__float_as_uint(mx) >> 23), 28) : 0, a1 = a / 2;
        const _Float16 up1 = on ? (_Float16)__uint_as_float((uint32_t)(127 + a1) << 23) : (_Float16)0.f;
        const _Float16 up2 = (_Float16)__uint_as_float((uint32_t)(127 + a - a1) << 23 | (p.softmax_scale < 0.f ? 0x80000000u : 0u));
        c_zero = fmaxf(fabsf(p.softmax_scale) * kLog2e, 1e-30f) * __uint_as_float((uint32_t)(127 - a) << 23);      // (not 0: masked logits stay -inf)
        c_code = c_zero * kKeyUnscale;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
            Frag f;
            f.h = raw[cb];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const _Float16 pf = BITS == 2 ? (_Float16)(1.f / (float)(1 << (2 * r))) : (_Float16)((r & 1) ? 1.f / 16.f : 1.f);
                qz[cb][r] = f.p[r] * half2v{up1, up1} * half2v{up2, up2};
                qk[cb][r] = qz[cb][r] * half2v{pf, pf};
            }
        }
        if constexpr (HP == 1) {
            own_qz = own * half2v{up1, up1} * half2v{up2, up2};
            const float place = __uint_as_float((uint32_t)(127 - (BITS == 2 ? 2 * (lane & 3) : 4 * (lane & 1))) << 23);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                own_q[i] = (float)own_qz[i] * place;
                own_q_up[i] = own_q[i] * kLoMagnify;
            }
        }
        if constexpr (HP > 1 && HP < 8) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const half2v even = is_lo ? qz[2][r] : qz[0][r], odd = is_lo ? qz[3][r] : qz[1][r];
                q_zero[r] = n & 4 ? odd : even;
            }
        }
    };
    auto query_frag = [&](int cb) -> half8 {
        Frag f;
#pragma unroll
        for (int r = 0; r < 4; ++r) f.p[r] = qz[cb][r];
        return f.h;
    };
    // Probabilities 2^(prob_exp + logit - m) of this lane's four tokens, logit = x cx + zk; raises the maximum, and rescales the state by
    // rescale(factor), when a logit passes it by the slack
    auto softmax = [&](const float (&x)[4], float cx, float zk, float (&pv)[4], auto&& rescale) {
        auto logits = [&](float off) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pv[i] = fmaf(x[i], cx, off);
            return fmaxf(fmaxf(pv[0], pv[1]), fmaxf(pv[2], pv[3]));
        };
        const float mx = logits(zk - (m - prob_exp));
        if (__any(mx > prob_exp + kSlack)) {
            float t = logits(zk);
            t = max_rows(fmaxf(t, dpp<kRor8>(t)));
            const float mn = fmaxf(m, t), f = __builtin_amdgcn_exp2f(m - mn);
            rescale(f);
            l *= f;
            m = mn;
            logits(zk - (m - prob_exp));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) pv[i] = __builtin_amdgcn_exp2f(pv[i]);
        l += (pv[0] + pv[1]) + (pv[2] + pv[3]);
    };
    auto rescale_acc = [&](float f) {
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[u] *= f;
        zsum *= f;
        if constexpr (HP == 1) {
            z_own[0] *= f;
            z_own[1] *= f;
            l_own *= f;
        }
    };
    // fb: rounded (hi columns) or the remainder (lo columns), fa: the rounded ones in the lo columns, 0 in the others;
    // lane kb gets tokens 8 kb .. 8 kb + 7
    auto split = [&](const float (&pv)[4], Frag& fa, Frag& fb) {
        const half2v none = {(_Float16)0.f, (_Float16)0.f};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const half2v hi = pack_rtz(pv[2 * r], pv[2 * r + 1]);
            float l0, l1;                              // the remainders (exact in fp32) with one mixed-precision instruction each
            asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(l0) : "v"(hi), "v"(pv[2 * r]));
            asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(l1) : "v"(hi), "v"(pv[2 * r + 1]));
            const half2v lo = pack_rtz(l0, l1);
            fb.p[r] = from_partner<kLoLanes>(hi, lo);
            fb.p[r + 2] = from_partner<kHiLanes>(lo, hi);
            fa.p[r] = from_partner<kLoLanes>(none, hi);
            fa.p[r + 2] = is_lo ? hi : none;
        }
        auto exchange = [&](Frag& f) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                auto s = __builtin_amdgcn_permlane32_swap(f.r[r], f.r[r + 2], false, false);
                f.r[r] = s[0];
                f.r[r + 2] = s[1];
            }
        };
        exchange(fa);
        exchange(fb);
    };
    // masks this lane's tokens of a tile that begins with token t0 (their factor is positive)
    auto mask = [&](const View& v, int t0, float (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + tok + i;
            x[i] = ((t < v.length) & ((t >= v.lowest) | (t < v.sinks))) ? x[i] : -INFINITY;
        }
    };
    auto any_above = [&](uint32_t s2, uint32_t limit) -> bool {                      // of 128 scales, two per lane
        typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
        const uint32_t l2 = limit | limit << 16;
        return __any(__builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, s2), __builtin_bit_cast(ushort2v, l2))) != l2);
    };

    // ---- one record out of an LDS slot ----
    // HP = 1: with one head the columns would be copies of each other if every lane made its own.  Instead a lane makes two elements of the key
    // operand (two channels) and of the value operand (one token, two channel groups), which fill the columns through LDS, and its softmax work is one token.
    auto record_one = [&](const unsigned char* sl, const View& v, int r) {
        if constexpr (HP == 1) {
            const unsigned char* scales = sl + kScaleOff;
            const uint32_t k_scale = *reinterpret_cast<const uint32_t*>(scales + lane * 4), k_zero = *reinterpret_cast<const uint32_t*>(scales + 256 + lane * 4);
            const unsigned char* own = scales + 512 + own_tok * 8 + own_pair * 4;
            const uint32_t v_scale = *reinterpret_cast<const uint32_t*>(own), v_zero = *reinterpret_cast<const uint32_t*>(own + 256);
            uint32_t kw[2 * BITS], vw[2 * BITS];
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl) {
                const uint4v a = *reinterpret_cast<const uint4v*>(sl + pl * 1024 + lane16), b = *reinterpret_cast<const uint4v*>(sl + kScaleOff + 1024 + pl * 1024 + lane16);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    kw[4 * pl + k] = a[k];
                    vw[4 * pl + k] = b[k];
                }
            }
            _Float16* operand = sm_operand[wave];
            half2v hi, lo;
            const bool big = any_above(k_scale, kKeyScaleLimit);
            const float f = big ? 1.f / (1 << kKeyScaleShift) : 1.f;
            split_products(__builtin_bit_cast(half2v, k_scale), own_q[0] * f, own_q[1] * f, own_q_up[0] * f, own_q_up[1] * f, hi, lo);
            *reinterpret_cast<half2v*>(operand + 2 * lane) = hi;
            *reinterpret_cast<half2v*>(operand + kKeyColumn + 2 * lane) = lo;
            wave_lds_sync();
            half8 kf[4];
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) kf[cb] = *reinterpret_cast<const half8*>(operand + (is_lo ? kKeyColumn : 0) + cb * 32 + kb * 8);
            const float zk = wave_sum(__builtin_amdgcn_fdot2(own_qz, __builtin_bit_cast(half2v, k_zero), 0.f, false)) * c_zero;
            float4v d0 = {0.f, 0.f, 0.f, 0.f}, d1 = d0;
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) {
                d0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_fragment<BITS>(kw, cb, 0), kf[cb], d0, 0, 0, 0);
                d1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_fragment<BITS>(kw, cb, 1), kf[cb], d1, 0, 0, 0);
            }
            auto own_of = [&](const float4v& x) -> float {
                const float a = own_i & 1 ? x[1] : x[0], b = own_i & 1 ? x[3] : x[2];
                return own_i & 2 ? b : a;
            };
            // the token's sum over the rounded products from one column of the pair, over the remainders from the other
            const float x0 = own_of(d0), x1 = own_of(d1), c = big ? c_code * (float)(1 << kKeyScaleShift) : c_code;
            float x = fmaf(is_lo ? x1 : x0, is_lo ? c * kLoShrink : c, fmaf(dpp<kRor8>(is_lo ? x0 : x1), is_lo ? c : c * kLoShrink, zk));
            if (r * kTileTokens < v.lowest) {
                const int t = r * kTileTokens + own_tok;
                x = ((t >= v.lowest) | (t < v.sinks)) ? x : -INFINITY;
            }
            if (__any(x > m + kSlack)) {
                const float mn = fmaxf(m, wave_max(x)), g = __builtin_amdgcn_exp2f(m - mn);
                rescale_acc(g);
                l *= g;
                m = mn;
            }
            if (prob_exp > 0.f && any_above(v_scale, kValueScaleLimit<BITS>)) {
                const float g = __builtin_amdgcn_exp2f(-(float)kSlack - prob_exp);
                rescale_acc(g);
                l *= g;
                prob_exp = -(float)kSlack;
            }
            const float pv = __builtin_amdgcn_exp2f(x + (prob_exp - own_exp - m)), pv_up = pv * kLoMagnify;
            const half2v vz = __builtin_bit_cast(half2v, v_zero);
            l_own += pv;
            z_own[0] = fmaf(pv, (float)vz[0], z_own[0]);
            z_own[1] = fmaf(pv, (float)vz[1], z_own[1]);
            split_products(__builtin_bit_cast(half2v, v_scale), pv, pv, pv_up, pv_up, hi, lo);
            wave_lds_sync();
            _Float16* column = operand + own_pair * 4 * 32 + own_tok;       // columns (group, rounded / remainder)
            column[0] = hi[0];
            column[32] = lo[0];
            column[64] = hi[1];
            column[96] = lo[1];
            wave_lds_sync();
            const half8 vf = *reinterpret_cast<const half8*>(operand + (my_group * 2 + (is_lo ? 1 : 0)) * 32 + kb * 8);
#pragma unroll
            for (int u = 0; u < 8; ++u) acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value_fragment<BITS>(vw, u >> 1, u & 1), vf, acc[u], 0, 0, 0);
            wave_lds_sync();
        }
    };
    auto record_many = [&](const unsigned char* sl, const View& v, int r) {
        if constexpr (HP > 1) {
            uint32_t w[2 * BITS];
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl) {
                const uint4v q4 = *reinterpret_cast<const uint4v*>(sl + pl * 1024 + (kb * 16 + row_pos) * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[4 * pl + k] = q4[k];
            }
            const bool big = any_above(*reinterpret_cast<const uint32_t*>(sl + kScaleOff + lane * 4), kKeyScaleLimit);
            float4v d0 = {0.f, 0.f, 0.f, 0.f}, d1 = d0, dz = d0;
            Frag s[4];
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) {
                s[cb].v = *reinterpret_cast<const uint4v*>(sl + kScaleOff + cb * 64 + kb * 16);
                if constexpr (HP >= 8) {
                    Frag z;
                    z.v = *reinterpret_cast<const uint4v*>(sl + kScaleOff + 256 + cb * 64 + kb * 16);
                    dz = __builtin_amdgcn_mfma_f32_16x16x32_f16(z.h, query_frag(cb), dz, 0, 0, 0);
                }
            }
            if constexpr (HP < 8) {
                // (eight channels in each of the four columns that share a head and kb)
                Frag z;
                z.v = *reinterpret_cast<const uint4v*>(sl + kScaleOff + 256 + (n >> 2) * 64 + kb * 16);
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) sum = __builtin_amdgcn_fdot2(q_zero[k], z.p[k], sum, false);
                sum += dpp<kRor8>(sum);
                sum += dpp<kRor4>(sum);
                dz[0] = add_rows(sum);
            }
            if (big) {
                const half2v f = {(_Float16)(1.f / (1 << kKeyScaleShift)), (_Float16)(1.f / (1 << kKeyScaleShift))};
#pragma unroll
                for (int cb = 0; cb < 4; ++cb)
#pragma unroll
                    for (int k = 0; k < 4; ++k) s[cb].p[k] *= f;
            }
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) {
                Frag f;
                // in the lo columns alone; the hi columns' zeros stay
                uint64_t active;
                asm("s_and_saveexec_b64 %4, %13\n\tv_pk_mul_f16 %0, %5, %9\n\tv_pk_mul_f16 %1, %6, %10\n\tv_pk_mul_f16 %2, %7, %11\n\tv_pk_mul_f16 %3, %8, %12\n\ts_mov_b64 exec, %4"
                    : "+&v"(rounded[0]), "+&v"(rounded[1]), "+&v"(rounded[2]), "+&v"(rounded[3]), "=&s"(active)
                    : "v"(qk[cb][0]), "v"(qk[cb][1]), "v"(qk[cb][2]), "v"(qk[cb][3]), "v"(s[cb].p[0]), "v"(s[cb].p[1]), "v"(s[cb].p[2]), "v"(s[cb].p[3]), "s"(kLoColumns)
                    : "scc");
#pragma unroll
                for (int k = 0; k < 4; ++k) f.p[k] = __builtin_elementwise_fma(qk[cb][k], s[cb].p[k], -rounded[k]);
                d0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_fragment<BITS>(w, cb, 0), f.h, d0, 0, 0, 0);
                d1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_fragment<BITS>(w, cb, 1), f.h, d1, 0, 0, 0);
            }
            float x[4], pv[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // hi and lo column of a head share its tokens: hi columns take tok0 + k, lo columns 16 + tok0 + k
                x[k] = is_lo ? d1[k] : d0[k];
                x[k] += dpp<kRor8>(is_lo ? d0[k] : d1[k]);
            }
            if (prob_exp > 0.f && any_above(*reinterpret_cast<const uint32_t*>(sl + kScaleOff + 512 + lane * 4), kValueScaleLimit<BITS>)) {
                const float f = __builtin_amdgcn_exp2f(-(float)kSlack - prob_exp);
                rescale_acc(f);
                l *= f;
                prob_exp = -(float)kSlack;
            }
            if (r * kTileTokens < v.lowest) mask(v, r * kTileTokens, x);
            softmax(x, big ? c_code * (float)(1 << kKeyScaleShift) : c_code, dz[0] * c_zero, pv, rescale_acc);
            // outputs: this lane's tokens 8 kb .. 8 kb + 7, as pairs, of a channel group
            Frag fa, fb, z;
            split(pv, fa, fb);
            const unsigned char* vs = sl + kScaleOff + 512 + kb * 64;
            {
                const uint32_t sel = (n & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned char* t = vs + 256 + 16 * k + (n & 2) * 2;
                    const uint32_t t0 = *reinterpret_cast<const uint32_t*>(t), t1 = *reinterpret_cast<const uint32_t*>(t + 8);
                    z.r[k] = __builtin_amdgcn_perm(t1, t0, sel);
                }
            }
            zsum = __builtin_amdgcn_mfma_f32_16x16x32_f16(z.h, fb.h, zsum, 0, 0, 0);       // rows = channel groups
            Frag sv[NS];
            if constexpr (HP == 2) {
                const uint32_t sel = (my_group & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned char* t = vs + 16 * k + (my_group & 2) * 2;
                    const uint32_t t0 = *reinterpret_cast<const uint32_t*>(t), t1 = *reinterpret_cast<const uint32_t*>(t + 8);
                    sv[0].r[k] = __builtin_amdgcn_perm(t1, t0, sel);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4v t = *reinterpret_cast<const uint4v*>(vs + 16 * k);         // tokens 2 k and 2 k + 1, four groups each
                    if constexpr (HP == 4) {
                        const uint32_t sel = my_group ? 0x07060302u : 0x05040100u;
                        sv[0].r[k] = __builtin_amdgcn_perm(t[2], t[0], sel);
                        sv[1].r[k] = __builtin_amdgcn_perm(t[3], t[1], sel);
                    } else {
                        sv[0].r[k] = __builtin_amdgcn_perm(t[2], t[0], 0x05040100u);
                        sv[1].r[k] = __builtin_amdgcn_perm(t[2], t[0], 0x07060302u);
                        sv[2].r[k] = __builtin_amdgcn_perm(t[3], t[1], 0x05040100u);
                        sv[3].r[k] = __builtin_amdgcn_perm(t[3], t[1], 0x07060302u);
                    }
                }
            }
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl) {
                const uint4v q4 = *reinterpret_cast<const uint4v*>(sl + kScaleOff + 1024 + pl * 1024 + lane16);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[4 * pl + k] = q4[k];
            }
            if constexpr (BITS == 2) {
                const half2v pf = {(_Float16)0.25f, (_Float16)0.25f};
                fa.p[1] *= pf; fa.p[3] *= pf;
                fb.p[1] *= pf; fb.p[3] *= pf;
            }
            Frag f[NS];
#pragma unroll
            for (int g = 0; g < NS; ++g)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const half2v t = fa.p[k] * sv[g].p[k];
                    f[g].p[k] = __builtin_elementwise_fma(fb.p[k], sv[g].p[k], __builtin_elementwise_fma(fa.p[k], sv[g].p[k], -t));
                }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value_fragment<BITS>(w, u >> 1, u & 1), f[(u >> 1) * NS / 4].h, acc[u], 0, 0, 0);
        }
    };
    auto record_tile = [&](const unsigned char* sl, const View& v, int r) {
        if constexpr (HP == 1) record_one(sl, v, r);
        else record_many(sl, v, r);
    };

    // ---- 32 fp16 rows: keys are operands as they are; value rows, eight tokens by eight channels per lane, are turned in registers ----
    auto row_tile = [&](const View& v, int64_t ring, int i, float4v (&ro)[8]) {
        const int t0 = v.row0 + i * kTileTokens, last = v.length - 1, base = t0 % p.cap_r;
        auto slot_of = [&](int t) {                                    // (rows past the end re-read the last one)
            const int s = base + min(t, last) - t0;
            return s >= p.cap_r ? s - p.cap_r : s;
        };
        Frag kr[2][4], vr[8];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int cb = 0; cb < 4; ++cb)
                kr[hf][cb].v = *reinterpret_cast<const uint4v*>(p.k_resid + ring + slot_of(t0 + hf * 16 + row_pos) * kHeadDim + cb * 32 + kb * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) vr[e].v = *reinterpret_cast<const uint4v*>(p.v_resid + ring + slot_of(t0 + kb * 8 + e) * kHeadDim + n * 8);
        float4v d[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            d[hf] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) d[hf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kr[hf][cb].h, query_frag(cb), d[hf], 0, 0, 0);
        }
        float x[4], pv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = is_lo ? d[1][k] : d[0][k];
        if (t0 < v.lowest || t0 + kTileTokens > v.length) mask(v, t0, x);
        softmax(x, c_zero, 0.f, pv, [&](float f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) ro[e] *= f;
        });
        Frag fa, fb;
        split(pv, fa, fb);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            Frag a;                                                    // rows: channels 8 n + e
#pragma unroll
            for (int k = 0; k < 4; ++k) a.r[k] = __builtin_amdgcn_perm(vr[2 * k + 1].r[e / 2], vr[2 * k].r[e / 2], e & 1 ? 0x07060302u : 0x05040100u);
            ro[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, fb.h, ro[e], 0, 0, 0);
        }
    };
    // the lane of a head's pair of columns that holds channels 16 u + 4 kb .. of it
    auto holds = [&](int u) { return !is_lo && (HP == 1 ? n < 4 && my_group == (u >> 1) : HP == 8 || (HP == 4 ? my_group == ((u >> 1) & 1) : my_group == (u >> 1))); };

    bool first_unit = true;
    int slot = 0;
    advance_copy();
    // The instruction arbiter favours the oldest wavefront of a SIMD, so the workgroups of a compute unit would finish one after the other,
    // the last one alone: a wavefront's priority falls with the share of its interval that is done.
    const int quarter = (x1 - x0) >> 2;
    int priority = 3, drop_at = x0 + quarter;
    __builtin_amdgcn_s_setprio(3);
    auto progress = [&](int x) {
        if (x < drop_at || priority == 0) return;
        --priority;
        drop_at += quarter;
        if (priority == 2) __builtin_amdgcn_s_setprio(2);
        else if (priority == 1) __builtin_amdgcn_s_setprio(1);
        else __builtin_amdgcn_s_setprio(0);
    };
    while (true) {
        const View& view = here.view;
        const int cost = view.cost(), kvh = p.by_runs.of(here.unit), h0 = (here.unit - kvh * p.runs) * p.run, live = min(p.run, rep - h0);
        const int64_t q_row = (int64_t)here.b * p.n_q_heads + kvh * rep + h0;
        {
            Frag raw[4];
            half8 r8[4];
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) {
                raw[cb].v = *reinterpret_cast<const uint4v*>(p.q + (q_row + min(head, live - 1)) * kHeadDim + cb * 32 + kb * 8);
                r8[cb] = raw[cb].h;
            }
            half2v own = {(_Float16)0.f, (_Float16)0.f};
            if constexpr (HP == 1) own = *reinterpret_cast<const half2v*>(p.q + q_row * kHeadDim + 2 * lane);
            set_query(r8, own);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[u] = float4v{0.f, 0.f, 0.f, 0.f};
        zsum = float4v{0.f, 0.f, 0.f, 0.f};
        m = kNothing;
        l = l_own = z_own[0] = z_own[1] = 0.f;
        prob_exp = (float)kProbExp<BITS>;
#pragma unroll 1
        while (in_flight < NB) {
            const int was = in_flight;
            advance_copy();
            if (in_flight == was) break;
        }
        // its steps of fp16 rows in the interval
        const int row_from = min(max(x0 - here.unit0, 0), view.row_steps), row_end = min(x1 - here.unit0, view.row_steps);
        if (row_from < row_end) {
            const int slot_of_rows = p.slots ? scalar(p.slots, here.b) : here.b;
            const int64_t ring = ((int64_t)slot_of_rows * p.n_kv_heads + kvh) * p.cap_r * kHeadDim;
            float4v ro[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) ro[e] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int j = row_from; j < row_end; ++j)
                if (j * kWaves + wave < view.row_tiles) row_tile(view, ring, j * kWaves + wave, ro);
            // into the records' order
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) ro[e][i] = (ro[e][i] + dpp<kRor8>(ro[e][i])) * (1.f / kValueUnscale);
#pragma unroll 1
            for (int g0 = 0; g0 < HP; g0 += HR) {
                wave_lds_sync();
                if (n >= g0 && n < g0 + HR) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float4v* dst = reinterpret_cast<float4v*>(&sm_o[wave][n - g0][(kb * 4 + i) * 8]);
                        dst[0] = float4v{ro[0][i], ro[1][i], ro[2][i], ro[3][i]};
                        dst[1] = float4v{ro[4][i], ro[5][i], ro[6][i], ro[7][i]};
                    }
                }
                wave_lds_sync();
                if (head >= g0 && head < g0 + HR) {
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (holds(u)) acc[u] = *reinterpret_cast<const float4v*>(&sm_o[wave][head - g0][u * 16 + kb * 4]);
                }
            }
            wave_lds_sync();
        }
        const int j1 = records_to(here);
        for (int j = records_from(here); j < j1; ++j) {
            progress(here.unit0 + view.row_steps + j);
            wait_oldest();
            const int i = j * kWaves + wave;
            if (i < view.records && !((lost >> slot) & 1)) record_tile(&sm_ring[wave][slot][0], view, i < view.sink_records ? i : i + view.skip);
            advance_copy();
            slot = slot + 1 == NB ? 0 : slot + 1;
        }
        // ---- leave the unit ----
        {
            float lw = add_rows(l + dpp<kRor8>(l));
            if constexpr (HP == 1) lw += wave_sum(l_own * (BITS == 2 && (own_i & 2) ? 2.f : 0.5f));      // (every token is two lanes')
            if (lane < HP) {
                sm_ml[wave][lane][0] = m - prob_exp;                   // sums and outputs are relative to 2^this
                sm_ml[wave][lane][1] = lw;
            }
        }
        const int owner0 = own_pieces ? wg - piece : here.unit0 / length;         // the first workgroup of the unit
        const int parts = own_pieces ? pieces : (here.unit0 + cost - 1) / length - owner0 + 1;
        auto write_out = [&](int hh, int c, float ox, float oy, float sum) {
            const float f = sum > 0.f ? 1.f / sum : 0.f;
            const int64_t i = (q_row + hh) * kHeadDim + c;
            if (p.out_bf16) {
                typedef __bf16 bfloat2 __attribute__((ext_vector_type(2)));
                *reinterpret_cast<bfloat2*>(static_cast<__bf16*>(p.out) + i) = bfloat2{(__bf16)(ox * f), (__bf16)(oy * f)};
            } else {
                *reinterpret_cast<half2v*>(static_cast<_Float16*>(p.out) + i) = half2v{(_Float16)(ox * f), (_Float16)(oy * f)};
            }
        };
        const int c2 = (tid & 63) * 2, my_part = wg * 2 + (first_unit ? 0 : 1);
        float zz[4];                                                   // zero-points' share of this lane's head, by channel group
        if constexpr (HP == 1) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float t = z_own[k] * (BITS == 2 && (own_i & 2) ? 4.f : 1.f);
                t += dpp<kXor2>(t);
                t += dpp<kRor4>(t);
                zz[k] = zz[k + 2] = add_rows(t + dpp<kRor8>(t));
            }
        } else {
#pragma unroll
            for (int g = 0; g < 4; ++g) zz[g] = zsum[g] + dpp<kRor8>(zsum[g]);
        }
#pragma unroll 1
        for (int g0 = 0; g0 < HP; g0 += HR) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                float4v o;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float remainders = dpp<kRor8>(acc[u][i]);
                    o[i] = fmaf(HP == 1 ? fmaf(remainders, kLoShrink, acc[u][i]) : acc[u][i] + remainders, kValueUnscale, zz[u >> 1]);
                }
                if (holds(u) && head >= g0 && head < g0 + HR) *reinterpret_cast<float4v*>(&sm_o[wave][head - g0][u * 16 + kb * 4]) = o;
            }
            lds_barrier();
            for (int hh = g0 + wave; hh < min(g0 + HR, live); hh += kWaves) {
                float mm = kNothing, sum = 0.f, ox = 0.f, oy = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, sm_ml[w][hh][0]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = __builtin_amdgcn_exp2f(sm_ml[w][hh][0] - mm);
                    const float2 o2 = *reinterpret_cast<const float2*>(&sm_o[w][hh - g0][c2]);
                    sum = fmaf(sm_ml[w][hh][1], f, sum);
                    ox = fmaf(o2.x, f, ox);
                    oy = fmaf(o2.y, f, oy);
                }
                if (parts == 1) {
                    write_out(hh, c2, ox, oy, sum);
                } else {
                    store_shared(p.part_o + ((int64_t)my_part * kMaxHeads + hh) * kPartFloats + c2, ox, oy);
                    if (lane == 0) store_shared(p.part_ml + ((int64_t)my_part * kMaxHeads + hh) * 2, mm, sum);
                }
            }
            lds_barrier();                                             // (LDS is written again)
        }
        if (parts > 1) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // the part is where the others can see it
            lds_barrier();
            if (tid == 0) sm_last = __hip_atomic_fetch_add(p.counters + owner0, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
            lds_barrier();
            if (sm_last) {
                // the unit is the first one of every workgroup but, maybe, the first of them
                const int second = !own_pieces && owner0 * length < here.unit0 - unit_cost ? 1 : 0;
                for (int hh = wave; hh < live; hh += kWaves) {
                    float mm = kNothing, sum = 0.f, ox = 0.f, oy = 0.f;
#pragma unroll 1
                    for (int g0 = 0; g0 < parts; g0 += kJoined) {
                        float2 st[kJoined], o2[kJoined];
#pragma unroll
                        for (int g = 0; g < kJoined; ++g) {
                            const int at = min(g0 + g, parts - 1), part = (owner0 + at) * 2 + (at == 0 ? second : 0);
                            st[g] = load_shared(p.part_ml + ((int64_t)part * kMaxHeads + hh) * 2);
                            o2[g] = load_shared(p.part_o + ((int64_t)part * kMaxHeads + hh) * kPartFloats + c2);
                        }
                        float mn = mm;
#pragma unroll
                        for (int g = 0; g < kJoined; ++g) mn = fmaxf(mn, st[g].x);
                        const float f0 = __builtin_amdgcn_exp2f(mm - mn);
                        mm = mn;
                        sum *= f0;
                        ox *= f0;
                        oy *= f0;
#pragma unroll
                        for (int g = 0; g < kJoined; ++g) {
                            const float f = g0 + g < parts ? __builtin_amdgcn_exp2f(st[g].x - mn) : 0.f;
                            sum = fmaf(st[g].y, f, sum);
                            ox = fmaf(o2[g].x, f, ox);
                            oy = fmaf(o2[g].y, f, oy);
                        }
                    }
                    write_out(hh, c2, ox, oy, sum);
                }
                if (tid == 0) __hip_atomic_store(p.counters + owner0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            lds_barrier();
        }
        if (here.unit0 + cost + unit_cost >= x1) break;
        first_unit = false;
        next_unit(here);
    }
    wait_copies<0>();                                                  // no copy may land in LDS that has been given back
}

}  // namespace

size_t paged_workspace_bytes() {
    return kWorkgroups * sizeof(int32_t) + (size_t)kWorkgroups * 2 * kMaxHeads * (kPartFloats + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedAttentionParams& params, hipStream_t stream) {
    Args p{};
    static_cast<PagedAttentionParams&>(p) = params;
    const int rep = p.n_q_heads / p.n_kv_heads;
    p.runs = (rep + kMaxHeads - 1) / kMaxHeads;
    p.run = (rep + p.runs - 1) / p.runs;
    p.by_runs = FastDiv::by(p.runs);
    // (the axis has to fit 31 bits)
    const int64_t records = (int64_t)p.max_pages << p.page_shift, rows = (p.residual + 2 * kTileTokens) / kTileTokens;
    const int64_t cost = (records + kWaves - 1) / kWaves + (rows + kWaves - 1) / kWaves + kUnitCost;
    if (cost > 0x200000 || cost * p.batch * p.n_kv_heads * p.runs > 0x40000000) return hipErrorNotSupported;
    char* ws = reinterpret_cast<char*>(p.counters);
    p.part_o = reinterpret_cast<float*>(ws + kWorkgroups * sizeof(int32_t));
    p.part_ml = p.part_o + (size_t)kWorkgroups * 2 * kMaxHeads * kPartFloats;
#define KIVI_PAGED(B, H) paged_attention_kernel<B, H><<<kWorkgroups, 64 * kWaves, 0, stream>>>(p)
    if (p.bits == 2) {
        if (p.run == 1) KIVI_PAGED(2, 1);
        else if (p.run == 2) KIVI_PAGED(2, 2);
        else if (p.run <= 4) KIVI_PAGED(2, 4);
        else KIVI_PAGED(2, 8);
    } else {
        if (p.run == 1) KIVI_PAGED(4, 1);
        else if (p.run == 2) KIVI_PAGED(4, 2);
        else if (p.run <= 4) KIVI_PAGED(4, 4);
        else KIVI_PAGED(4, 8);
    }
#undef KIVI_PAGED
    return hipGetLastError();
}

}  // namespace kivi
