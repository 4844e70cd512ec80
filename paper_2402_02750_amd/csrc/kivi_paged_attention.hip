// Attention of one token per sequence over the paged cache (kivi_paged_attention).
//
// Work: a unit is (sequence, kv-head, run of up to eight query heads).  What a unit has to visit -- its visible records and tiles of 32
// fp16 rows -- follows from the sequence's length, and is put on one axis for all units, in steps of one record or tile per
// wavefront.  Every workgroup adds up the lengths by itself and takes one interval of the axis, so the device is divided
// evenly whatever the lengths, and nothing but the batch's size is known to the host.  A unit that lies in one interval is written
// out by it; of one that several share each leaves a part (maximum, sum, outputs) in the workspace, and the last to come joins them.
//
// Products: 16x16x32 matrix instructions; operand rows are tokens (keys) and channels (values), columns are query heads.  Lane
// (n = lane % 16, kb = lane / 16) makes the eight contraction elements 8 kb .. 8 kb + 7 of column n: head n % HP; n < 8: rounded products, n >= 8: what
// the rounding left, so that a pair of columns together has 21 bits.  Codes are operands as they are, as subnormal fp16 numbers
// (their place in the 16 bits is a power of two that goes into the other factor); scales go into the other operand:
//   logit_t = sum_c code_tc (s_c q_c) + sum_c z_c q_c,     o_c = sum_t code_tc (p_t s_tg) + sum_t p_t z_tg
// Queries enter times a power of two that puts the largest element into [2^8, 2^9), probabilities times 2^8 (4 bits: 2^11); tiles with
// scales that could leave fp16's range with that (keys 2^6, values 2^3; 4 bits 2^0) take the scales 2^-9, or from then on the probabilities 2^-4.
// The running maximum moves where a logit passes it by more than 2^4.
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
constexpr int kMinCost = 4;            // of an interval
constexpr int kRowCost = 3;            // of a step of fp16 rows, in steps of records
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

struct Args : PagedAttentionParams {
    int32_t runs, run;                 // runs of query heads per kv-head, heads of a run
};

// What a sequence shows its newest token
struct View {
    int length, packed;                // tokens; records
    int lowest;                        // first token of the window
    int sinks;                         // visible first tokens before it
    int records, sink_records, skip;   // visible records: i < sink_records: i, else i + skip
    int row0, row_tiles;               // first token of the first tile of fp16 rows, tiles of 32
    int row_steps, steps;
    __device__ __forceinline__ int cost() const { return row_steps * kRowCost + steps; }
};
__device__ __forceinline__ View view_of(const Args& p, int length, int slot) {
    View v;
    v.length = slot >= 0 && slot < p.max_sequences ? max(length, 0) : 0;
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
    return v;
}
__device__ __forceinline__ View view_of(const Args& p, int b) { return view_of(p, p.lengths[b], p.slots ? p.slots[b] : b); }

template <int BITS, int HP>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_kernel(Args p) {
    constexpr int kCodeBytes = kTileTokens * kHeadDim * BITS / 8, kPlanes = BITS / 2, kScaleOff = kCodeBytes;
    constexpr int kRecord = record_bytes(BITS);
    constexpr int NS = HP / 2;                                         // value-side operands: columns of a head share the channel groups
    __shared__ __align__(16) unsigned char sm_record[kWaves][kRecord];
    __shared__ __align__(16) float sm_o[kWaves][HP][kHeadDim];
    __shared__ float sm_ml[kWaves][HP][2];
    __shared__ int sm_last;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kb = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool is_lo = n >= 8;
    const int head = n & (HP - 1);
    const int row_pos = (n & 3) | ((n >> 3) & 1) << 2 | ((n >> 2) & 1) << 3;        // operand row m holds token row_pos of its half
    const int tok0 = (kb & 1) * 8 + (kb >> 1) * 4, tok = tok0 + (is_lo ? 16 : 0);   // this lane's tokens: tok + i
    const int my_group = HP == 2 ? (n >> 1) & 3 : HP == 4 ? (n >> 2) & 1 : 0;
    const int rep = p.n_q_heads / p.n_kv_heads, units_per_sequence = p.n_kv_heads * p.runs;

    // ---- this workgroup's interval of the axis ----
    const int wg = ((int)blockIdx.x & 7) * (kWorkgroups / 8) + ((int)blockIdx.x >> 3);      // neighbours on the axis share a die
    int total = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
        int c = b0 + lane < p.batch ? view_of(p, b0 + lane).cost() * units_per_sequence : 0;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) c += __shfl_xor(c, d);
        total += c;
    }
    const int length = max((total + kWorkgroups - 1) / kWorkgroups, kMinCost);
    const int x0 = wg * length, x1 = min(x0 + length, total);
    if (x0 >= x1) return;
    int b = 0, before = 0;                                             // the sequence of x0, and where it begins
    {
        int sum = 0;
        for (int b0 = 0; b0 < p.batch; b0 += 64) {
            const int mine = b0 + lane < p.batch ? view_of(p, b0 + lane).cost() * units_per_sequence : 0;
            int upto = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
            const uint64_t here = __ballot(sum + upto > x0);
            if (here) {
                const int at = __builtin_ctzll(here);
                b = b0 + at;
                before = sum + __shfl(upto - mine, at);
                break;
            }
            sum += __shfl(upto, 63);
        }
    }
    b = __builtin_amdgcn_readfirstlane(b);
    before = __builtin_amdgcn_readfirstlane(before);
    View view = view_of(p, b);
    int unit = (x0 - before) / view.cost();                            // of the sequence

    float4v acc[8], zsum, ro[8];
    float m, l, prob_exp;
    half2v qz[4][4], qk[4][4];
    float c_zero, c_code;


    int x = x0;
    bool first_unit = true;
    while (true) {
        const int cost = view.cost(), unit0 = before + unit * cost;    // where the unit begins
        const int kvh = unit / p.runs, h0 = (unit - kvh * p.runs) * p.run, live = min(p.run, rep - h0);
        const int64_t q_row = (int64_t)b * p.n_q_heads + kvh * rep + h0;
        const int slot = p.slots ? p.slots[b] : b;
        const __half* k_ring = p.k_resid + ((int64_t)slot * p.n_kv_heads + kvh) * p.cap_r * kHeadDim;
        const __half* v_ring = p.v_resid + ((int64_t)slot * p.n_kv_heads + kvh) * p.cap_r * kHeadDim;
        // ---- query ----
        {
            Frag raw[4];
            float mx = 0.f;
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) {
                raw[cb].v = *reinterpret_cast<const uint4v*>(p.q + (q_row + min(head, live - 1)) * kHeadDim + cb * 32 + kb * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf((float)raw[cb].h[e]));
            }
            mx = max_rows(mx);
            const bool on = mx > 0.f;
            const int a = on ? min(kQueryExp + 127 - (int)(__float_as_uint(mx) >> 23), 28) : 0, a1 = a / 2;
            const _Float16 up1 = on ? (_Float16)__uint_as_float((uint32_t)(127 + a1) << 23) : (_Float16)0.f;
            const _Float16 up2 = (_Float16)__uint_as_float((uint32_t)(127 + a - a1) << 23);
            c_zero = p.softmax_scale * kLog2e * __uint_as_float((uint32_t)(127 - a) << 23);
            c_code = c_zero * kKeyUnscale;
#pragma unroll
            for (int cb = 0; cb < 4; ++cb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const _Float16 pf = BITS == 2 ? (_Float16)(1.f / (float)(1 << (2 * r))) : (_Float16)((r & 1) ? 1.f / 16.f : 1.f);
                    qz[cb][r] = raw[cb].p[r] * half2v{up1, up1} * half2v{up2, up2};
                    qk[cb][r] = qz[cb][r] * half2v{pf, pf};
                }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acc[i] = float4v{0.f, 0.f, 0.f, 0.f};
            ro[i] = float4v{0.f, 0.f, 0.f, 0.f};
        }
        zsum = float4v{0.f, 0.f, 0.f, 0.f};
        m = kNothing;
        l = 0.f;
        prob_exp = (float)kProbExp<BITS>;

        auto rescale = [&](float f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) { acc[i] *= f; ro[i] *= f; }
            zsum *= f;
            l *= f;
        };
        // probabilities 2^(prob_exp + logit - m) of this lane's four tokens out of x[i] (log2 domain; -inf: masked)
        auto softmax = [&](float (&x4)[4]) {
            float mx = fmaxf(fmaxf(x4[0], x4[1]), fmaxf(x4[2], x4[3]));
            if (__any(mx > m + kSlack || (m == kNothing && mx > kNothing))) {
                mx = max_rows(fmaxf(mx, dpp<kRor8>(mx)));
                const float mn = fmaxf(m, mx);
                rescale(__builtin_amdgcn_exp2f(m - mn));
                m = mn;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x4[i] = __builtin_amdgcn_exp2f(x4[i] - m + prob_exp);
            l += (x4[0] + x4[1]) + (x4[2] + x4[3]);
        };
        // fb: rounded (hi columns) or the remainder (lo columns), fa: the rounded ones in the lo columns, 0 in the others;
        // lane kb gets tokens 8 kb .. 8 kb + 7
        auto split = [&](const float (&pv)[4], Frag& fa, Frag& fb) {
            const half2v none = {(_Float16)0.f, (_Float16)0.f};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const half2v hi = pack_rtz(pv[2 * r], pv[2 * r + 1]);
                const half2v lo = pack_rtz(pv[2 * r] - (float)hi[0], pv[2 * r + 1] - (float)hi[1]);
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
        // mask of this lane's tokens of a tile that begins with token t0
        auto mask = [&](int t0, float (&x4)[4]) {
            if (t0 < view.lowest || t0 + kTileTokens > view.length) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = t0 + tok + i;
                    if (t >= view.length || (t < view.lowest && t >= view.sinks)) x4[i] = -INFINITY;
                }
            }
        };

        auto record_tile = [&](int i) {
            const int r = i < view.sink_records ? i : i + view.skip;
            const int page = p.page_table[b * p.page_table_stride + (r >> p.page_shift)];
            if (page < 0 || page >= p.n_pages) return;
            const char* rec = p.pages + (((((int64_t)page * p.n_kv_heads + kvh) << p.page_shift) + (r & ((1 << p.page_shift) - 1))) * kRecord);
            unsigned char* sl = &sm_record[wave][0];
            uint4v in[kRecord / 1024];
#pragma unroll
            for (int j = 0; j < kRecord / 1024; ++j) in[j] = *reinterpret_cast<const uint4v*>(rec + j * 1024 + lane * 16);
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int j = 0; j < kRecord / 1024; ++j) *reinterpret_cast<uint4v*>(sl + j * 1024 + lane * 16) = in[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            uint32_t w[2 * BITS];
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl) {
                const uint4v v = *reinterpret_cast<const uint4v*>(sl + pl * 1024 + (kb * 16 + row_pos) * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[4 * pl + k] = v[k];
            }
            // logits
            const uint32_t ks2 = *reinterpret_cast<const uint32_t*>(sl + kScaleOff + lane * 4);
            const bool big = __any(ks2 >> 16 >= kKeyScaleLimit || (ks2 & 0xFFFFu) >= kKeyScaleLimit);
            float4v d0 = {0.f, 0.f, 0.f, 0.f}, d1 = d0, dz = d0;
#pragma unroll
            for (int cb = 0; cb < 4; ++cb) {
                Frag s, z, f, qf;
                s.v = *reinterpret_cast<const uint4v*>(sl + kScaleOff + cb * 64 + kb * 16);
                z.v = *reinterpret_cast<const uint4v*>(sl + kScaleOff + 256 + cb * 64 + kb * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (big) s.p[k] *= half2v{(_Float16)(1.f / (1 << kKeyScaleShift)), (_Float16)(1.f / (1 << kKeyScaleShift))};
                    const half2v t = qk[cb][k] * s.p[k], none = {(_Float16)0.f, (_Float16)0.f};
                    f.p[k] = __builtin_elementwise_fma(qk[cb][k], s.p[k], is_lo ? -t : none);
                    qf.p[k] = qz[cb][k];
                }
                dz = __builtin_amdgcn_mfma_f32_16x16x32_f16(z.h, qf.h, dz, 0, 0, 0);
                d0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_fragment<BITS>(w, cb, 0), f.h, d0, 0, 0, 0);
                d1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_fragment<BITS>(w, cb, 1), f.h, d1, 0, 0, 0);
            }
            float x4[4];
            const float cx = big ? c_code * (float)(1 << kKeyScaleShift) : c_code, zk = dz[0] * c_zero;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // hi and lo column of a head share its tokens: hi columns take tok0 + k, lo columns 16 + tok0 + k
                x4[k] = is_lo ? d1[k] : d0[k];
                x4[k] += dpp<kRor8>(is_lo ? d0[k] : d1[k]);
                x4[k] = fmaf(x4[k], cx, zk);
            }
            mask(r * kTileTokens, x4);
            // outputs
            const uint32_t vs2 = *reinterpret_cast<const uint32_t*>(sl + kScaleOff + 512 + lane * 4);
            if (prob_exp > 0.f && __any(vs2 >> 16 >= kValueScaleLimit<BITS> || (vs2 & 0xFFFFu) >= kValueScaleLimit<BITS>)) {
                rescale(__builtin_amdgcn_exp2f(-(float)kSlack - prob_exp));
                prob_exp = -(float)kSlack;
            }
            softmax(x4);
            Frag fa, fb, z;
            split(x4, fa, fb);
            auto pairs = [&](int off, int group, Frag& to) {           // of this lane's tokens, one channel group
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t a = *reinterpret_cast<const uint16_t*>(sl + off + (kb * 8 + 2 * k) * 8 + group * 2);
                    const uint32_t c = *reinterpret_cast<const uint16_t*>(sl + off + (kb * 8 + 2 * k + 1) * 8 + group * 2);
                    to.r[k] = a | c << 16;
                }
            };
            pairs(kScaleOff + 768, n & 3, z);
            zsum = __builtin_amdgcn_mfma_f32_16x16x32_f16(z.h, fb.h, zsum, 0, 0, 0);       // rows = channel groups
            if constexpr (BITS == 2) {
                const half2v pf = {(_Float16)0.25f, (_Float16)0.25f};
                fa.p[1] *= pf; fa.p[3] *= pf;
                fb.p[1] *= pf; fb.p[3] *= pf;
            }
            Frag f[NS];
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                Frag sv;
                pairs(kScaleOff + 512, HP == 2 ? my_group : HP == 4 ? 2 * s + my_group : s, sv);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const half2v t = fa.p[k] * sv.p[k];
                    f[s].p[k] = __builtin_elementwise_fma(fb.p[k], sv.p[k], __builtin_elementwise_fma(fa.p[k], sv.p[k], -t));
                }
            }
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl) {
                const uint4v v = *reinterpret_cast<const uint4v*>(sl + kScaleOff + 1024 + pl * 1024 + lane * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[4 * pl + k] = v[k];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value_fragment<BITS>(w, u >> 1, u & 1), f[(u >> 1) * NS / 4].h, acc[u], 0, 0, 0);
            __builtin_amdgcn_wave_barrier();
        };
        // 32 fp16 rows: keys are operands as they are; value rows, eight tokens by eight channels per lane, are turned in registers
        auto row_tile = [&](int i) {
            const int t0 = view.row0 + i * kTileTokens, last = view.length - 1;
            const int base = t0 % p.cap_r;
            auto slot_of = [&](int t) {                                // (rows past the end re-read the last one)
                const int s = base + min(t, last) - t0;
                return s >= p.cap_r ? s - p.cap_r : s;
            };
            Frag kr[2][4], vr[8];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int cb = 0; cb < 4; ++cb)
                    kr[hf][cb].v = *reinterpret_cast<const uint4v*>(k_ring + slot_of(t0 + hf * 16 + row_pos) * kHeadDim + cb * 32 + kb * 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) vr[e].v = *reinterpret_cast<const uint4v*>(v_ring + slot_of(t0 + kb * 8 + e) * kHeadDim + n * 8);
            float4v d[2];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                d[hf] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int cb = 0; cb < 4; ++cb) {
                    Frag qf;
#pragma unroll
                    for (int k = 0; k < 4; ++k) qf.p[k] = qz[cb][k];
                    d[hf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kr[hf][cb].h, qf.h, d[hf], 0, 0, 0);
                }
            }
            float x4[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x4[k] = (is_lo ? d[1][k] : d[0][k]) * c_zero;
            mask(t0, x4);
            softmax(x4);
            Frag fa, fb;
            split(x4, fa, fb);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                Frag a;                                                // rows: channels 8 n + e
#pragma unroll
                for (int k = 0; k < 4; ++k) a.r[k] = __builtin_amdgcn_perm(vr[2 * k + 1].r[e / 2], vr[2 * k].r[e / 2], e & 1 ? 0x07060302u : 0x05040100u);
                ro[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, fb.h, ro[e], 0, 0, 0);
            }
        };

        // ---- the interval's steps of this unit ----
        const int end = min(x1, unit0 + cost);
        {
            const int a = x - unit0, z = end - unit0;                  // steps that begin in [a, z)
            const int rows_cost = view.row_steps * kRowCost;
            for (int j = (min(a, rows_cost) + kRowCost - 1) / kRowCost; j * kRowCost < min(z, rows_cost); ++j)
                if (j * kWaves + wave < view.row_tiles) row_tile(j * kWaves + wave);
            for (int j = max(a - rows_cost, 0); j < z - rows_cost; ++j)
                if (j * kWaves + wave < view.records) record_tile(j * kWaves + wave);
        }
        // ---- leave the unit ----
        {
            const float lw = add_rows(l + dpp<kRor8>(l));
            if (lane < HP) {
                sm_ml[wave][lane][0] = m - prob_exp;                   // sums and outputs are relative to 2^this
                sm_ml[wave][lane][1] = lw;
            }
            // outputs of the records: head `head`, channels 16 u + 4 kb + i; of the rows: channels 8 (4 kb + i) + e
            float zz[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) zz[g] = zsum[g] + dpp<kRor8>(zsum[g]);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int g = u >> 1;
                float4v o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = fmaf(acc[u][i] + dpp<kRor8>(acc[u][i]), kValueUnscale, zz[g]);
                const bool valid = !is_lo && (HP == 8 || (HP == 4 ? my_group == (g & 1) : my_group == g));
                if (valid) *reinterpret_cast<float4v*>(&sm_o[wave][head][u * 16 + kb * 4]) = o;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) ro[e][i] += dpp<kRor8>(ro[e][i]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (n < HP) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float4v* dst = reinterpret_cast<float4v*>(&sm_o[wave][n][(kb * 4 + i) * 8]);
                    dst[0] += float4v{ro[0][i], ro[1][i], ro[2][i], ro[3][i]};
                    dst[1] += float4v{ro[4][i], ro[5][i], ro[6][i], ro[7][i]};
                }
            }
        }
        __syncthreads();
        const int owner0 = unit0 / length, parts = (unit0 + cost - 1) / length - owner0 + 1;
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
        const int c2 = (tid & 63) * 2;
        const int my_part = wg * 2 + (first_unit ? 0 : 1);
        for (int hh = wave; hh < live; hh += kWaves) {
            float mm = kNothing, sum = 0.f, ox = 0.f, oy = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, sm_ml[w][hh][0]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(sm_ml[w][hh][0] - mm);
                sum = fmaf(sm_ml[w][hh][1], f, sum);
                ox = fmaf(sm_o[w][hh][c2], f, ox);
                oy = fmaf(sm_o[w][hh][c2 + 1], f, oy);
            }
            if (parts == 1) {
                write_out(hh, c2, ox, oy, sum);
            } else {
                store_shared(p.part_o + ((int64_t)my_part * kMaxHeads + hh) * kPartFloats + c2, ox, oy);
                if (lane == 0) store_shared(p.part_ml + ((int64_t)my_part * kMaxHeads + hh) * 2, mm, sum);
            }
        }
        if (parts > 1) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) sm_last = __hip_atomic_fetch_add(p.counters + owner0, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
            __syncthreads();
            if (sm_last) {
                for (int hh = wave; hh < live; hh += kWaves) {
                    float mm = kNothing, sum = 0.f, ox = 0.f, oy = 0.f;
                    for (int g = 0; g < parts; ++g) {
                        // the unit is the first one of every workgroup but, maybe, the first of them
                        const int part = (owner0 + g) * 2 + (g == 0 && owner0 * length < unit0 ? 1 : 0);
                        const float2 st = load_shared(p.part_ml + ((int64_t)part * kMaxHeads + hh) * 2);
                        const float2 o2 = load_shared(p.part_o + ((int64_t)part * kMaxHeads + hh) * kPartFloats + c2);
                        const float mn = fmaxf(mm, st.x), f0 = __builtin_amdgcn_exp2f(mm - mn), f1 = __builtin_amdgcn_exp2f(st.x - mn);
                        mm = mn;
                        sum = fmaf(st.y, f1, sum * f0);
                        ox = fmaf(o2.x, f1, ox * f0);
                        oy = fmaf(o2.y, f1, oy * f0);
                    }
                    write_out(hh, c2, ox, oy, sum);
                }
                if (tid == 0) __hip_atomic_store(p.counters + owner0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        if (end >= x1) break;
        __syncthreads();
        x = end;
        first_unit = false;
        if (++unit == units_per_sequence) {
            before += units_per_sequence * cost;
            unit = 0;
            do {
                view = view_of(p, ++b);
            } while (view.cost() == 0);                                // (x < total: there is another sequence with tokens)
        }
    }
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
    // (the axis has to fit 31 bits)
    const int64_t records = (int64_t)p.max_pages << p.page_shift, rows = (p.residual + 2 * kTileTokens) / kTileTokens;
    const int64_t cost = (records + kWaves - 1) / kWaves + ((rows + kWaves - 1) / kWaves) * kRowCost;
    if (cost * p.batch * p.n_kv_heads * p.runs > 0x40000000) return hipErrorNotSupported;
    char* ws = reinterpret_cast<char*>(p.counters);
    p.part_o = reinterpret_cast<float*>(ws + kWorkgroups * sizeof(int32_t));
    p.part_ml = p.part_o + (size_t)kWorkgroups * 2 * kMaxHeads * kPartFloats;
#define KIVI_PAGED(B, H) paged_attention_kernel<B, H><<<kWorkgroups, 64 * kWaves, 0, stream>>>(p)
    if (p.bits == 2) {
        if (p.run <= 2) KIVI_PAGED(2, 2);
        else if (p.run <= 4) KIVI_PAGED(2, 4);
        else KIVI_PAGED(2, 8);
    } else {
        if (p.run <= 2) KIVI_PAGED(4, 2);
        else if (p.run <= 4) KIVI_PAGED(4, 4);
        else KIVI_PAGED(4, 8);
    }
#undef KIVI_PAGED
    return hipGetLastError();
}

}  // namespace kivi
