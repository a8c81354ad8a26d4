// Attention over the paged, quantized key/value cache (see flatquant.h for the layout): causal, with a sliding window and first tokens
// that stay visible, or for a tree of drafted tokens.
//
// The rows of a (sequence, key/value head) are its new tokens' query heads that share the head: row r is token r / G, query head r % G of
// the group.  A wave takes 16 NT of them and 32 tokens of the cache a step, on v_mfma_f32_16x16x32_f16:
//   S^T[token, row] = K Q^T      A: lane (i, g) has token i's channels 32 g .. 32 g + 31, a quarter of its codes in one load; Q lies in
//                                registers in the order in which those codes become fp16
//   O^T[channel, row] += V^T P^T A: lane (i, g) has channels 8 i .. 8 i + 7 of eight tokens, 4 g .. 4 g + 3 of each half of the 32:
//                                those whose weights the lane of S^T already holds, so the weights need no exchange
// Codes become fp16 without a conversion.  Few rows: a code in its place, masked, is a subnormal fp16 number (2^(s - 24) code), which the
// matrix instructions take as it is; the powers of two are taken out of the queries and of the results, and the zero points out of the sums
// (sum_d q_d (c_d - z) = sum_d q_d c_d - z sum_d q_d).  Many rows share the work of taking the zero point off each code, in LDS.  The keys'
// steps scale the scores, the values' steps the weights.
//
// Softmax in one pass: weights are 2^(score - M), M a reference per row that is raised only where a weight times its step would pass
// 2^15 (fp16's range) or the weights 2^40: most steps neither reduce a maximum nor touch the accumulators.  When it is raised it is put
// so that the largest product is 2^7: those below 2^-21 of it, fp16's subnormals, lose no more than 2^-32 of it.  (Capped scores of many rows over 2^14 tokens at most: 2^2, 2^-16
// and 2^-27; see largest_of.)
//
// The 4, 8 or 16 waves of a workgroup take its steps in turn and meet in LDS at the end; where the rows are few the axis is split further over
// workgroups, whose partial results (M, sum, channels, in fp32) a second kernel joins.
//
// Measured (copy of 1 GB 4.73 TB/s): one row each of 64 sequences of 4096 tokens, 8 heads of 4 queries, 4 bits 46 us = 88 % of the copy rate; 16 of 6000,
// 32 heads, 4 and 2 bits 54 us = 90 %; 1 of 131072 41 us, 30 of it memory and 7 the join; 1 of 1000 10 us, latencies one after the other.  A first
// version without the ring, the subnormal operands and the launches of few rows took 66, 94, 113 and 11 us.
#pragma once
#include "fq_internal.h"
#include "fq_device.h"
#include "fq_cache_device.h"

namespace fq {

constexpr int ATT_D = 128;
constexpr int ATT_WAVES = 4;
constexpr int ATT_NT = 64 * ATT_WAVES;
constexpr int ATT_STEP = 32;               // tokens per step of a wave
constexpr int ATT_PITCH = ATT_D + 4;       // floats per row of partial channels in LDS
constexpr int kMaxSplits = 128;
constexpr float ATT_NONE = -0x1p125f;        // reference of a row that has seen nothing: below every finite score

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Lists that no kernel writes, read at uniform addresses: by scalar loads, which do not stand in the queue of the codes' loads.
typedef const __attribute__((address_space(4))) int32_t* list_t;

struct AttnDev {
    CacheDev c;
    const _Float16* q;
    _Float16* out;
    const uint64_t* visible;
    float* part;              // partial channels, 128 a row, and pairs of M and sum: [T * Hq, splits] rows, or two tiles a workgroup (balanced)
    float* stats;
    int64_t q_stride, out_stride;
    float scale2;             // scale * log2(e)
    int Hq, G, window, sinks, chunk, splits, min_units;
};

// With scores that are capped, lowered by a distance, or seen through a prefix (flatquant_cache_scored_attention), in the exponent's base 2.
struct ScoredDev : AttnDev {
    int bend;                 // 0: no cap, 1: scale2 takes scores to exponents of tanh, whose results are in units of 2 cap, 2: a large cap
    float cap, per_cap;       // of a large one, and its reciprocal
    float unit;               // what scores are in
    const float* slopes;      // of a query head; null: none
    const int32_t* prefix;    // of a sequence; null: none
};
template <typename DEV>
constexpr bool kScored = std::is_same_v<DEV, ScoredDev>;
// x, or none if it is infinite.  (tanh would make a number of a score whose key's step is none.)
__device__ __forceinline__ float if_finite(float x) { return __builtin_fmaf(x, 0.0f, x); }
// A sum over values.  An infinite one has a step that is none, or its negative, among them: no number.
template <typename DEV>
__device__ __forceinline__ float outcome(float x) {
    if constexpr (kScored<DEV>) return if_finite(x);
    return x;
}
// Whether a span's steps are gone through from the last one on: with slopes, whose scores are highest there, so that references need not be raised at every step
// (2048 rows at 8192 tokens 1077 -> 586 us, 64 sequences of 4096 51.5 -> 47.0).  A step behind the last one in this order has tokens below zero.
template <typename DEV>
__device__ __forceinline__ bool backwards(const DEV& p) {
    if constexpr (kScored<DEV>) return p.slopes != nullptr;
    return false;
}
template <typename DEV>
__device__ __forceinline__ int in_order(const DEV& p, int steps, int x) { return backwards(p) ? steps - 1 - x : x; }
// Tokens of sequence b that all of its rows see, wherever they are.
template <typename DEV>
__device__ __forceinline__ int prefix_of(const DEV& p, int b) {
    int n = 0;
    if constexpr (kScored<DEV>) n = p.prefix ? p.prefix[b] : 0;
    return n > 0 ? n : 0;
}

// The last token that a row at `position` sees but for its window, or the last of the prefix.
__device__ __forceinline__ int last_of(int position, int prefix) { return prefix > 0 && prefix - 1 > position ? prefix - 1 : position; }

template <int N, int K = 0, typename F>
__device__ __forceinline__ void each(F&& f) {                                  // f(0) .. f(N - 1), constants
    if constexpr (K < N) {
        f(std::integral_constant<int, K>{});
        each<N, K + 1>(f);
    }
}

// ---- codes to fp16

// Two codes in bits [S, S + QB) of the halves of x, S + QB <= 10: as fp16 bits that is 2^(S - 24) code, a subnormal number, which the matrix
// instructions take at its value.  They align the products to the largest of them, though, by its exponent as if it were normalised, and drop what
// lies 24 bits below (measured: one code unit beside others is off by up to 2^-13.4 of itself at S = 0, by nothing at 2 and above for weights within
// a factor of 20): S is 2 at least.
// RAISED: with 1024 in the exponent, 1024 + 2^S code.
constexpr uint32_t kRaise = 0x64006400u;
template <int QB, int S>
constexpr uint32_t field_mask() {
    static_assert(S >= 2 && S + QB <= 10, "mantissa bits");
    return (((1u << QB) - 1u) << S) * 0x00010001u;
}
// The masks of raised fields, by S, in scalar registers that are written here: the compiler would keep them across a loop, out of registers, and fetch them back
// with more instructions.
template <int QB>
struct Masks {
    uint32_t m[9];
    __device__ __forceinline__ Masks() {
        asm volatile("s_mov_b32 %0, %1" : "=s"(m[0]) : "i"(0x000F000Fu));      // of zero points
        fill<2>();
    }
    template <int S>
    __device__ __forceinline__ void fill() {
        constexpr bool used = QB == 4 ? S == 2 || S == 6 : QB == 3 ? S >= 4 && S <= 7 : S == 4 || S == 6 || S == 8;
        if constexpr (used) asm volatile("s_mov_b32 %0, %1" : "=s"(m[S]) : "i"(field_mask<QB, S>()));
        if constexpr (S < 8) fill<S + 1>();
    }
};
struct NoMasks {};
template <int QB, int S, typename M>
__device__ __forceinline__ uint32_t field(uint32_t x, const M& masks) {
    if constexpr (std::is_same_v<M, NoMasks>) {
        return x & field_mask<QB, S>();
    } else {
        uint32_t r;                                                            // (one instruction: of two constants the compiler makes two)
        asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "s"(masks.m[S]), "v"(kRaise));
        return r;
    }
}
__device__ __forceinline__ constexpr uint32_t raise_of(const NoMasks&) { return 0u; }
template <int QB>
__device__ __forceinline__ constexpr uint32_t raise_of(const Masks<QB>&) { return kRaise; }
// code - zero point of a raised field; `z`: 1024 + the zero points, in fp16.  One packed fma takes 1024 and the zero point off, exactly.
template <int S>
__device__ __forceinline__ half2v code_value(uint32_t f, half2v z) {
    const half2v raised = as_half2(f);
    constexpr _Float16 down = (_Float16)(1.0f / (float)(1 << S)), off = (_Float16)(1024.0f - 1024.0f / (float)(1 << S));
    return __builtin_elementwise_fma(raised, half2v{down, down}, half2v{off, off} - z);
}
template <int QB>
__device__ __forceinline__ half2v raised_zeros(const Masks<QB>& masks, uint32_t low, uint32_t high) {  // of two tokens' parameters
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(__builtin_amdgcn_perm(high, low, 0x07060302u)), "s"(masks.m[0]), "v"(kRaise));
    return as_half2(r);
}

// The 32 codes of a lane's quarter of a key, as 16 pairs of fields; pair p is (first(p), second(p)) of the 32, at bit shift(p).
template <int QB>
struct KeyCodes;
template <>
struct KeyCodes<4> {
    typedef u32x4 words;
    static constexpr int first(int p) { return 8 * (p >> 2) + (p & 3); }
    static constexpr int second(int p) { return first(p) + 4; }
    static constexpr int shift(int p) { return p & 1 ? 6 : 2; }
    template <typename M>
    static __device__ __forceinline__ void fields(const words& w, uint32_t (&o)[16], const M& masks) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            o[4 * k] = field<4, 2>(w[k] << 2, masks);
            o[4 * k + 1] = field<4, 6>(w[k] << 2, masks);
            o[4 * k + 2] = field<4, 2>(w[k] >> 6, masks);
            o[4 * k + 3] = field<4, 6>(w[k] >> 6, masks);
        }
    }
};
__device__ __forceinline__ constexpr int shift2(int c) { return c < 3 ? 4 + 2 * c : c < 5 ? 2 * c : 2 * c - 6; }      // of the 2-bit codes of a half
template <>
struct KeyCodes<2> {
    typedef uint32_t words __attribute__((ext_vector_type(2)));
    static constexpr int first(int p) { return 16 * (p >> 3) + (p & 7); }
    static constexpr int second(int p) { return first(p) + 8; }
    static constexpr int shift(int p) { return shift2(p & 7); }
    template <typename M>
    static __device__ __forceinline__ void fields(const words& w, uint32_t (&o)[16], const M& masks) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            o[8 * k] = field<2, 4>(w[k] << 4, masks);
            o[8 * k + 1] = field<2, 6>(w[k] << 4, masks);
            o[8 * k + 2] = field<2, 8>(w[k] << 4, masks);
            o[8 * k + 3] = field<2, 6>(w[k], masks);
            o[8 * k + 4] = field<2, 8>(w[k], masks);
            o[8 * k + 5] = field<2, 4>(w[k] >> 6, masks);
            o[8 * k + 6] = field<2, 6>(w[k] >> 6, masks);
            o[8 * k + 7] = field<2, 8>(w[k] >> 6, masks);
        }
    }
};
template <>
struct KeyCodes<3> {
    typedef uint32_t words __attribute__((ext_vector_type(3)));
    static constexpr int first(int p) { return p; }
    static constexpr int second(int p) { return p + 16; }
    // sixteen codes are 48 bits, three halves x0, x1, x2: codes 5 and 10 straddle two of them
    static constexpr int shift(int p) {
        constexpr int at[16] = {4, 7, 6, 4, 7, 6, 5, 5, 4, 7, 6, 5, 4, 7, 4, 7};
        return at[p];
    }
    template <typename M>
    static __device__ __forceinline__ void fields(const words& w, uint32_t (&o)[16], const M& masks) {
        // bits 0 .. 47 in the low halves, 48 .. 95 in the high ones
        const uint32_t x0 = __builtin_amdgcn_perm(w[1], w[0], 0x07060100u), x1 = __builtin_amdgcn_perm(w[2], w[0], 0x05040302u),
                       x2 = __builtin_amdgcn_perm(w[2], w[1], 0x07060100u);
        o[0] = field<3, 4>(x0 << 4, masks);
        o[1] = field<3, 7>(x0 << 4, masks);
        o[2] = field<3, 6>(x0, masks);
        o[3] = field<3, 4>(x0 >> 5, masks);
        o[4] = field<3, 7>(x0 >> 5, masks);
        o[5] = (x0 >> 9 & 0x00400040u) | (x1 << 7 & 0x01800180u) | raise_of(masks);
        o[6] = field<3, 5>(x1 << 3, masks);
        o[7] = field<3, 5>(x1, masks);
        o[8] = field<3, 4>(x1 >> 4, masks);
        o[9] = field<3, 7>(x1 >> 4, masks);
        o[10] = (x1 >> 8 & 0x00C000C0u) | (x2 << 8 & 0x01000100u) | raise_of(masks);
        o[11] = field<3, 5>(x2 << 4, masks);
        o[12] = field<3, 4>(x2, masks);
        o[13] = field<3, 7>(x2, masks);
        o[14] = field<3, 4>(x2 >> 6, masks);
        o[15] = field<3, 7>(x2 >> 6, masks);
    }
};

// Four of a lane's eight channels (HALF 0: 0 .. 3, 1: 4 .. 7) of two tokens (low half, high half), channel c of the eight at bit shift(c).
template <int QB>
struct ValueCodes {
    static constexpr int shift(int c) {
        constexpr int at[8] = {4, 7, 6, 4, 7, 6, 5, 5};
        return QB == 4 ? (c & 1 ? 6 : 2) : QB == 2 ? shift2(c) : at[c];
    }
    template <int HALF, typename M>
    static __device__ __forceinline__ void fields(uint32_t a, uint32_t b, uint32_t (&o)[4], const M& masks) {
        const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05040100u);
        if constexpr (QB == 4) {
            const uint32_t y = HALF ? __builtin_amdgcn_perm(b, a, 0x07060302u) : x;
            o[0] = field<4, 2>(y << 2, masks);
            o[1] = field<4, 6>(y << 2, masks);
            o[2] = field<4, 2>(y >> 6, masks);
            o[3] = field<4, 6>(y >> 6, masks);
        } else if constexpr (QB == 2 && HALF == 0) {
            o[0] = field<2, 4>(x << 4, masks);
            o[1] = field<2, 6>(x << 4, masks);
            o[2] = field<2, 8>(x << 4, masks);
            o[3] = field<2, 6>(x, masks);
        } else if constexpr (QB == 2) {
            o[0] = field<2, 8>(x, masks);
            o[1] = field<2, 4>(x >> 6, masks);
            o[2] = field<2, 6>(x >> 6, masks);
            o[3] = field<2, 8>(x >> 6, masks);
        } else if constexpr (HALF == 0) {
            o[0] = field<3, 4>(x << 4, masks);
            o[1] = field<3, 7>(x << 4, masks);
            o[2] = field<3, 6>(x, masks);
            o[3] = field<3, 4>(x >> 5, masks);
        } else {
            const uint32_t y = __builtin_amdgcn_perm(b, a, 0x07060302u);
            o[0] = field<3, 7>(x >> 5, masks);
            o[1] = (x >> 9 & 0x00400040u) | (y << 7 & 0x01800180u) | raise_of(masks);
            o[2] = field<3, 5>(y << 3, masks);
            o[3] = field<3, 5>(y, masks);
        }
    }
};

// ---- a wave's ring of steps in LDS (few rows)
//
// A slot holds 32 tokens: two pieces of 16 keys' codes, two of values', and the 64 parameters.  Global-to-LDS loads fill it, one 16-byte
// chunk a lane and one instruction a piece (4 bits; fewer lanes for fewer bits), so that a step costs five loads and no registers while
// it is on its way.  At 4 bits the lanes fetch the chunks in the order that makes the reads free of bank conflicts: keys by quarters of all
// 16 tokens, values by tokens 4 g + r of all four g.
template <int KB, int VB>
struct Ring {
    static constexpr int K_PIECE = 256 * KB, V_PIECE = 256 * VB;
    static constexpr int V_AT = 2 * K_PIECE, P_AT = V_AT + 2 * V_PIECE, SLOT = P_AT + 256;
    static constexpr int LOADS = 5;
};
typedef const __attribute__((address_space(1))) void* att_gptr;
typedef __attribute__((address_space(3))) void* att_lptr;
template <int BITS, bool VALUES>
__device__ __forceinline__ void load_piece(const uint8_t* src, unsigned char* dst, int l) {
    // byte of the piece that lane l fetches
    const int from = BITS != 4 ? 16 * l : VALUES ? 64 * (4 * (l >> 2 & 3) + (l >> 4)) + 16 * (l & 3) : 64 * (l & 15) + 16 * (l >> 4);
    if (BITS == 4 || l < 16 * BITS) __builtin_amdgcn_global_load_lds((att_gptr)(src + from), (att_lptr)dst, 16, 0, 0);
}
// Tokens k0 .. k0 + 15 and k0 + 16 .. k0 + 31 in pages pg[0] and pg[1] (the caller has checked the numbers): whole pages are memory that may be
// read, whatever of them has been written.
template <int KB, int VB>
__device__ __forceinline__ void load_step(const CacheDev& c, int head, int k0, const int (&pg)[2], int l, unsigned char* slot) {
    typedef Ring<KB, VB> R;
    int64_t at[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        at[t] = (((int64_t)pg[t] * c.H + head) << c.page_shift) + ((k0 + 16 * t) & ((1 << c.page_shift) - 1));
        load_piece<KB, false>(c.codes[0] + at[t] * (16 * KB), slot + t * R::K_PIECE, l);
        load_piece<VB, true>(c.codes[1] + at[t] * (16 * VB), slot + R::V_AT + t * R::V_PIECE, l);
    }
    // (chosen as numbers: of a choice between two pointers the compiler made a look-up in an array that it kept in memory for 2-bit keys with 4-bit values,
    // and that load's wait stood behind the codes on their way: 64 x 4096 tokens 43.8 -> 39.5 us, 1 x 131072 37.5 -> 35.0)
    const uintptr_t keys = reinterpret_cast<uintptr_t>(c.params[0]), values = reinterpret_cast<uintptr_t>(c.params[1]);
    const uint32_t* params = reinterpret_cast<const uint32_t*>(l < 32 ? keys : values) + (l & 16 ? at[1] : at[0]) + (l & 15);
    __builtin_amdgcn_global_load_lds((att_gptr)params, (att_lptr)(slot + R::P_AT), 4, 0, 0);
}
// The lane's quarter of token i's key in piece t; its four values' codes (tokens 4 g + r, r = 0 .. 3, channels 8 i .. 8 i + 7) in piece t.
template <int KB>
__device__ __forceinline__ typename KeyCodes<KB>::words ring_key(const unsigned char* piece, int i, int g) {
    typename KeyCodes<KB>::words w;
    if constexpr (KB == 4) w = *reinterpret_cast<const u32x4*>(piece + 16 * (16 * g + i));
    else
#pragma unroll
        for (int k = 0; k < KB; ++k) w[k] = reinterpret_cast<const uint32_t*>(piece)[4 * KB * i + KB * g + k];
    return w;
}
template <int VB>
__device__ __forceinline__ uint32_t ring_value(const unsigned char* piece, int i, int g, int r) {
    if constexpr (VB == 4) return reinterpret_cast<const uint32_t*>(piece)[64 * r + 16 * g + i];
    if constexpr (VB == 2) return reinterpret_cast<const uint16_t*>(piece)[16 * (4 * g + r) + i];
    const uint32_t* w = reinterpret_cast<const uint32_t*>(piece) + 12 * (4 * g + r) + (3 * i >> 2);      // (the last lane's second word is never used)
    return __builtin_amdgcn_alignbit(w[(3 * i & 3) > 1 ? 1 : 0], w[0], 8 * (3 * i & 3));
}

// The zero point as it stands in a token's parameters: 2^-24 of it, a subnormal fp16 number, as is what the mixed-precision fma reads in place.
__device__ __forceinline__ _Float16 zero_bits(uint32_t params) { return as_half2(params)[1]; }
__device__ __forceinline__ _Float16 step_bits(uint32_t params) { return as_half2(params)[0]; }
__device__ __forceinline__ float step_of(uint32_t params) { return (float)__builtin_bit_cast(_Float16, (uint16_t)params); }

template <typename T>
__device__ __forceinline__ T across_groups(T x, T (*op)(T, T)) {               // over the four lanes of a row of S^T's transpose
    x = op(x, __shfl_xor(x, 16));
    return op(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float fmax_op(float a, float b) { return __builtin_fmaxf(a, b); }
__device__ __forceinline__ float fadd_op(float a, float b) { return a + b; }

// What the scores of a row are in, by the time that they are weighed.
template <typename DEV>
__device__ __forceinline__ float unit_of(const DEV& p, float factor) {
    if constexpr (kScored<DEV>) return p.unit;
    else return factor;
}

// What a key's step makes of a score, or no number if it is none.
template <typename DEV>
__device__ __forceinline__ float key_factor(const DEV& p, float step) {
    if constexpr (kScored<DEV>) return if_finite(step) * p.scale2;
    return step * p.scale2;
}

// The tokens that a tile of rows goes through: whole steps over the first tokens [0, 32 first_steps), then from `begin` (a multiple of 32) to `end`.
struct Span {
    int first_steps, begin, end, steps;
    __device__ __forceinline__ int token(int x) const { return x < first_steps ? ATT_STEP * x : begin + ATT_STEP * (x - first_steps); }
};
__device__ __forceinline__ Span span_of(const AttnDev& p, int length, int pos_lo, int pos_hi, int prefix) {
    Span s;
    const int64_t held = (int64_t)p.c.table_width << p.c.page_shift;           // (2^31 - 2^16 at most: steps behind the end are still ints)
    s.end = held < length ? (int)held : length;
    s.begin = s.first_steps = 0;
    if (!p.visible) {
        const int last = last_of(pos_hi, prefix);
        s.end = last < s.end ? last + 1 : s.end;
        if (p.window > 0) {
            const int64_t from = (int64_t)pos_lo - p.window + 1;
            s.begin = from > 0 ? (int)from & ~(ATT_STEP - 1) : 0;
            int firsts = prefix > 0 && prefix > p.sinks ? prefix : p.sinks;
            firsts = firsts < s.begin ? firsts : s.begin;
            firsts = firsts < s.end ? firsts : s.end;
            s.first_steps = firsts > 0 ? (firsts + ATT_STEP - 1) / ATT_STEP : 0;
        }
    }
    s.steps = s.first_steps + (s.end > s.begin ? (s.end - s.begin + ATT_STEP - 1) / ATT_STEP : 0);
    return s;
}
// The power of 2 of a row's largest product behind a raised reference (many rows).  With a cap scores spread over its range and cost more to weigh again: 2 instead of 7, so that
// references are raised less often (2048 rows at 8192 tokens capped 744 -> 715 us, 64 at 1500 of 32 sequences 100 -> 93, trees of 13 49.6 -> 46.8; few rows, bound by memory, gain
// nothing).  Products in fp16's subnormals then lose 2^-27 of the row's largest each, 2^-32 before: up to 2^14 tokens, that is 2^-13 in all, a quarter of what one product in fp16 is
// rounded by.
constexpr int kLowReferenceSteps = (1 << 14) / ATT_STEP;
template <typename DEV>
__device__ __forceinline__ float largest_of(const DEV& p, const Span& span) {
    if constexpr (kScored<DEV>) return p.bend && span.steps <= kLowReferenceSteps ? 2.0f : 7.0f;
    return 7.0f;
}
// Steps of a split: the plan's, or with other scores as many as all splits need to go through a span that is longer than the plan knows (a prefix beside a window: the host
// plans for splits of 256 tokens).
template <typename DEV>
__device__ __forceinline__ int steps_of_split(const DEV& p, int steps) {
    const int per = p.chunk / ATT_STEP;
    if constexpr (kScored<DEV>) {
        const int even = ((steps + p.splits - 1) / p.splits + 3) & ~3;
        return even > per ? even : per;
    }
    return per;
}
template <typename DEV>
__device__ __forceinline__ int splits_used(const DEV& p, int steps) {
    const int per = steps_of_split(p, steps), used = (steps + per - 1) / per;
    return used < 1 ? 1 : used < p.splits ? used : p.splits;
}
// Rows of a sequence, cut to the row tensors.
struct Sequence {
    int first, rows, length;
};
__device__ __forceinline__ Sequence sequence_of(const CacheDev& c, int b) {
    const list_t starts = (list_t)c.row_starts;
    const int first = starts[b], last = starts[b + 1], T = (int)c.T;
    Sequence s;
    s.length = ((list_t)c.lengths)[b];
    s.first = first > 0 ? first : 0;
    s.rows = (last < T ? last : T) - s.first;
    return s;
}

// Whether a row sees token k: its bounds are [lo, hi], below `firsts`, or (in a tree) the bits of `seen` from token `before` on.
struct Sight {
    int lo, hi, firsts;
    uint64_t seen;
};
__device__ __forceinline__ Sight sight_of(const AttnDev& p, int before, int token, int row, int prefix) {
    Sight s;
    s.hi = p.visible ? before - 1 : before + token;
    const int64_t lo = (int64_t)s.hi - p.window + 1;
    s.lo = !p.visible && p.window > 0 && lo > 0 ? (int)lo : 0;
    s.firsts = !p.visible && p.window > 0 ? (p.sinks < s.hi + 1 ? p.sinks : s.hi + 1) : 0;
    if (prefix > 0 && prefix > s.firsts) s.firsts = prefix;
    s.seen = p.visible ? p.visible[row] : 0;
    return s;
}
__device__ __forceinline__ bool sees(const Sight& s, int k) { return ((k >= s.lo) & (k <= s.hi)) | (k < s.firsts); }
__device__ __forceinline__ bool sees_drafted(const Sight& s, int before, int k) {
    const unsigned bit = (unsigned)k - (unsigned)before;
    return (bit < 64u) & (int)((bit & 32 ? (uint32_t)(s.seen >> 32) : (uint32_t)s.seen) >> (bit & 31) & 1u);
}
// Parameters of a value that not every row sees: a step that is a number and a zero point of four bits, so that a weight of zero makes a product of zero
// whatever the page holds.
__device__ __forceinline__ uint32_t usable_parameters(uint32_t w) { return (w & 0x7C00u) == 0x7C00u ? 0u : w & 0x000FFFFFu; }
__device__ __forceinline__ float times_step(uint32_t params, float x) {
    float r;
    asm("v_fma_mix_f32 %0, %1, %2, 0 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(params), "v"(x));
    return r;
}
// x, or NaN where a token's step is no number.
__device__ __forceinline__ float if_number(uint32_t params, float x) {
    asm("v_fma_mix_f32 %0, %1, 0, %0 op_sel_hi:[1,0,0]" : "+v"(x) : "v"(params));
    return x;
}
// sum + product (a half of `pair`) times the zero point in a token's parameters, both read where they are.
template <int HI>
__device__ __forceinline__ float zero_sum(uint32_t pair, uint32_t params, float sum) {
    if constexpr (HI) asm("v_fma_mix_f32 %0, %1, %2, %0 op_sel:[1,1,0] op_sel_hi:[1,1,0]" : "+v"(sum) : "v"(pair), "v"(params));
    else asm("v_fma_mix_f32 %0, %1, %2, %0 op_sel:[0,1,0] op_sel_hi:[1,1,0]" : "+v"(sum) : "v"(pair), "v"(params));
    return sum;
}
// Scores of N tokens (all factors taken in; none infinite), capped and lowered; `distance(k)` is the token's position less the row's.  What is no number stays none.
//   cap tanh(x / cap) = cap - 2 cap / (1 + e^(2 x / cap)): the exponent of 2 is what comes in, the cap alone is a constant of the row, which weights do not depend on, and the
//   rest goes on in units of 2 cap: an exponential, an addition and a reciprocal.  It is off by 2^-21 of the cap, whatever the score.
//   Caps beyond kLargeCap take the series of tanh below a quarter instead, so that the error is 2^-19 of the score there (2048 rows at 8192 tokens 715 us, so 919); up to
//   there it is below 2^-13, a quarter of what the weights are rounded by.
constexpr float kLargeCap = 256.0f;        // base 2
template <int N, typename Distance>
__device__ __forceinline__ void rescore(const ScoredDev& p, float (&score)[N], float slope, Distance distance) {
    if (p.bend == 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) score[k] = __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(score[k]));
    } else if (p.bend == 2) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float x = score[k], y = x * p.per_cap, y2 = y * y;
            const float far = __builtin_fmaf(-2.0f * p.cap, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y * 2.8853900817779268f)), p.cap);
            const float near = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(-17.0f / 315, y2, 2.0f / 15), y2, -1.0f / 3) * y2, x, x);
            score[k] = y2 < 0.0625f ? near : far;
        }
    }
    if (p.slopes)
#pragma unroll
        for (int k = 0; k < N; ++k) score[k] = __builtin_fmaf(-slope, __builtin_fabsf(distance(k)), score[k]);
}
// Slope of a query head, in the units of the scores.  (Beyond 2^60, where a token further on has no weight either, it is held there: sums stay finite.)
__device__ __forceinline__ float slope_of(const ScoredDev& p, int hq) {
    return p.slopes ? __builtin_fminf(__builtin_fmaxf(p.slopes[hq] * 1.44269504088896340736f, -0x1p60f), 0x1p60f) / p.unit : 0.0f;
}

// Weights 2^(factor score - ref), their products with the values' steps and the weights' sum; true if a lane of the wave needs a higher reference.
// CAPPED, with a raised reference: of scores beyond 2^24 that reference is off by more than their exponents bear, and the products are held at 2^14.
template <int N, bool CAPPED, typename Scores, typename Factor, typename Step>
__device__ __forceinline__ bool weigh(const Scores& score, Factor factor, Step step, float ref, float (&prod)[N], float& sum) {
    float big = 0.0f;
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float e = __builtin_amdgcn_exp2f(__builtin_fmaf(score[k], factor(k), -ref));
        if constexpr (CAPPED) {
            const float cap = 0x1p14f * __builtin_amdgcn_rcpf(__builtin_fmaxf(step(k), 0x1p-25f));
            e = e > cap ? cap : e;                                             // (a NaN stays one)
        }
        sum += e;
        prod[k] = e * step(k);
        big = __builtin_fmaxf(big, prod[k]);
    }
    return __any(big > 32768.0f || sum > 0x1p40f);
}
// Raises the reference so that the row's largest product here is at most 2^7 (a step below 2^-25 counts as that), or 2^4 more for scores near 2^24: so much lower that
// the largest weight of all scores, however large, is not lost to the reference's rounding.  Returns the factor for what has been summed.
// `largest`: 7, or of many rows 2 where largest_of says so.
template <int N, typename Scores, typename Factor, typename Step, typename Row>
__device__ __forceinline__ float raise_reference(const Scores& score, Factor factor, Step step, float& ref, float largest, Row row_max) {
    float top = ATT_NONE;
#pragma unroll
    for (int k = 0; k < N; ++k) top = __builtin_fmaxf(top, score[k] * factor(k) + __builtin_fmaxf(__builtin_amdgcn_logf(step(k)), -25.0f));
    top = __builtin_fminf(row_max(top), 0x1p120f);
    const float to = __builtin_fmaxf(ref, top - largest - __builtin_fabsf(top) * 0x1p-22f), f = __builtin_amdgcn_exp2f(ref - to);
    ref = to;
    return f;
}

// ---- few rows: a wave has 16 NT of them and every NW-th step of a stretch of the sequence
template <int KB, int VB, int NT, int NW>
struct FewRows {
    static constexpr int DEPTH = 2;                                            // slots of a wave's ring (the waits in the loop are for two)
    static constexpr int RING = NW * DEPTH * Ring<KB, VB>::SLOT, SUMS = NW * 16 * ATT_PITCH * 4;
    static constexpr int STATS = RING > SUMS ? RING : SUMS;                    // references and sums of the rows, behind what the ring and the join share
    static constexpr int LDS = STATS + 2 * NW * 16 * NT * 4;
};
// Rows row0 .. row_end - 1 (16 NT at most) of head `head` of sequence b over steps [x_begin, x_end) of their span.  The result is the output, or (partial) what
// the join needs, rows from partial_at on.
// V = 2 (scores that cost more than the products: ScoredDev): there are 8 rows at most, each is in two of the 16 columns, and each of these takes the scores of
// half of the tokens, with a reference and sums of its own and weights of zero for the others: the work of a score is done by all lanes instead of those that
// have a row.  The columns meet behind the last step.
template <int KB, int VB, int NT, int NW, int V, typename DEV>
__device__ __forceinline__ void few_rows(const DEV& p, unsigned char* smem, int b, int head, const Sequence& seq, int row0, int row_end, const Span& span,
                                         int x_begin, int x_end, bool partial, int64_t partial_at) {
    typedef Ring<KB, VB> R;
    typedef FewRows<KB, VB, NT, NW> F;
    constexpr int DEPTH = F::DEPTH;
    const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned char* ring = smem + w * DEPTH * R::SLOT;
    float (*sums)[16][ATT_PITCH] = reinterpret_cast<float (*)[16][ATT_PITCH]>(smem);
    float (*refs)[16 * NT] = reinterpret_cast<float (*)[16 * NT]>(smem + F::STATS);
    float (*totals)[16 * NT] = refs + NW;
    const list_t table = (list_t)p.c.page_table + b * p.c.table_stride;
    const int before = seq.length - seq.rows;                                  // position of row 0's token
    const int pos_lo = before + row0 / p.G, pos_hi = before + (row_end - 1) / p.G;
    const int prefix = prefix_of(p, b);

    // (a step behind the last one: no harm, what its table entries say is checked before it is followed)
    auto pages_of = [&](int x, int (&pg)[2]) {
        const int k0 = span.token(in_order(p, span.steps, x));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const unsigned j = (unsigned)(k0 + 16 * t) >> p.c.page_shift;
            pg[t] = table[j < (unsigned)p.c.table_width ? j : p.c.table_width - 1];        // (behind the width is behind the end)
        }
    };
    auto load = [&](int x, const int (&pg)[2], int slot) {
        const int ok[2] = {(unsigned)pg[0] < (unsigned)p.c.pages ? pg[0] : 0, (unsigned)pg[1] < (unsigned)p.c.pages ? pg[1] : 0};
        load_step<KB, VB>(p.c, head, span.token(in_order(p, span.steps, x)), ok, l, ring + slot * R::SLOT);
    };
    int x = x_begin + w;
    int pg[DEPTH + 1][2];
    const bool any = x < x_end;
    if (any)
#pragma unroll
        for (int k = 0; k <= DEPTH; ++k) pages_of(x + NW * k, pg[k]);

    // Rows: queries in the order of the codes, brought up to 2^9 and down by the codes' shifts (a power of two each, and back in `factor`; the sign of the
    // scale is in the queries), their sums, positions.  A channel that becomes a subnormal fp16 number is rounded by 2^-25 of the row's norm at most, less than
    // the fp32 sums of its 128 products lose.  Asked for before the first steps: loads return in order.
    half8 raw[NT][4];
    Sight sight[NT];
    float slope[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        int r = row0 + 16 * n + (V > 1 ? i % (16 / V) : i);
        r = r < row_end ? r : row_end - 1;
        const int token = r / p.G, sub = r - token * p.G;
        const _Float16* src = p.q + (seq.first + token) * p.q_stride + (head * p.G + sub) * ATT_D + 32 * g;
#pragma unroll
        for (int m = 0; m < 4; ++m) raw[n][m] = *reinterpret_cast<const half8*>(src + 8 * m);
        sight[n] = sight_of(p, before, token, seq.first + token, prefix);
        if constexpr (kScored<DEV>) slope[n] = slope_of(p, head * p.G + sub);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (any)
#pragma unroll
        for (int k = 0; k < DEPTH; ++k)
            if (x + NW * k < x_end) load(x + NW * k, pg[k], k);
    __builtin_amdgcn_sched_barrier(0);
    half8 q[NT][4];
    float q_sum[NT], factor[NT];                                               // q_sum: minus the sum, as the instruction adds it up
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float squares = 0.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const u32x4 r = __builtin_bit_cast(u32x4, raw[n][m]);
#pragma unroll
            for (int k = 0; k < 4; ++k) squares = __builtin_amdgcn_fdot2(as_half2(r[k]), as_half2(r[k]), squares, false);
        }
        int up = 9 - ((__builtin_amdgcn_frexp_expf(across_groups(squares, fadd_op)) + 1) >> 1);
        up = up < 17 ? up : 17;                                                // (what is that small is exact all the same: multiples of 2^-24)
        // never zero: what is not visible scores -infinity before this factor
        factor[n] = __builtin_amdgcn_fmed3f(__builtin_ldexpf(__builtin_fabsf(p.scale2), 24 - up), 0x1p-120f, 0x1p100f);
        const float sign = p.scale2 < 0.0f ? -1.0f : 1.0f;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        each<4>([&](auto mm) {
            constexpr int m = decltype(mm)::value;
            u32x4 o, back;
            each<4>([&](auto ee) {
                constexpr int e = decltype(ee)::value, pair = 4 * m + e, a = KeyCodes<KB>::first(pair), z = KeyCodes<KB>::second(pair), S = KeyCodes<KB>::shift(pair);
                const _Float16 by = (_Float16)__builtin_ldexpf(sign, up - S), off = (_Float16)(-(float)(1 << S));
                o[e] = as_u32(half2v{raw[n][a >> 3][a & 7], raw[n][z >> 3][z & 7]} * half2v{by, by});
                back[e] = as_u32(half2v{off, off});
            });
            q[n][m] = __builtin_bit_cast(half8, o);
            sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, back), q[n][m], sum, 0, 0, 0);
        });
        q_sum[n] = sum[0];
    }

    f32x4 acc[NT][8];
    float ref[NT], total[NT], zeros[NT];                                   // zeros: sum of the products times their tokens' zero points
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        ref[n] = ATT_NONE;
        total[n] = zeros[n] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[n][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    auto work = [&](int x, const int (&pg)[2], const unsigned char* slot) {
        const int k0 = span.token(in_order(p, span.steps, x));
        f32x4 sc[NT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            __builtin_amdgcn_sched_barrier(0);
            uint32_t kk[16];
            KeyCodes<KB>::fields(ring_key<KB>(slot + t * R::K_PIECE, i, g), kk, NoMasks{});
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[n][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const u32x4 a = {kk[4 * m], kk[4 * m + 1], kk[4 * m + 2], kk[4 * m + 3]};
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    sc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), q[n][m], sc[n][t], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        half8 pw[NT];
        // whether all rows see all of the step (called behind the sums: what it takes is not kept over them)
        auto whole = [&] {
            const bool pages_ok = (unsigned)pg[0] < (unsigned)p.c.pages && (unsigned)pg[1] < (unsigned)p.c.pages;
            const int all_see = p.visible ? before - 1 : last_of(pos_lo, prefix);      // every row sees the tokens up to here, but for the window
            return pages_ok && k0 + ATT_STEP - 1 <= all_see && k0 + ATT_STEP <= span.end && (p.window <= 0 || p.visible || k0 > pos_hi - p.window);
        };
        if constexpr (V > 1) {
            static_assert(V == 2 && NT == 1, "columns 8 further on have the second 16 tokens");
            constexpr int N = 4;                                               // tokens of a lane, one behind the other
            const int tile = i / 8, first = 16 * tile + 4 * g;
            const u32x4 kp = *reinterpret_cast<const u32x4*>(slot + R::P_AT + 4 * first), v = *reinterpret_cast<const u32x4*>(slot + R::P_AT + 128 + 4 * first);
            float s[N], prod[N], sum;
            uint32_t vp[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float x = tile ? sc[0][1][k] : sc[0][0][k];
                s[k] = if_finite(times_step(kp[k], __builtin_fmaf((float)zero_bits(kp[k]), q_sum[0], x)) * factor[0]);
                vp[k] = v[k];
            }
            const float from = (float)(k0 + first - sight[0].hi);              // (no slopes in trees: hi is the row's position)
            rescore(p, s, slope[0], [&](int k) { return from + (float)k; });
            if (!whole()) {
                const bool page_ok = (unsigned)(tile ? pg[1] : pg[0]) < (unsigned)p.c.pages;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int at = k0 + first + k;
                    bool ok = sees(sight[0], at);
                    if (p.visible) ok |= sees_drafted(sight[0], before, at);
                    s[k] = (ok & page_ok & (at < span.end)) ? if_number(vp[k], s[k]) : -__builtin_inff();
                    vp[k] = usable_parameters(vp[k]);
                }
            }
            auto by = [&](int) { return unit_of(p, factor[0]); };
            auto step = [&](int k) { return (float)step_bits(vp[k]); };
            if (weigh<N, false>(s, by, step, ref[0], prod, sum)) {
                const float f = raise_reference<N>(s, by, step, ref[0], 7.0f, [](float top) { return across_groups(top, fmax_op); });
                total[0] *= f;
                zeros[0] *= f;
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[0][j] *= f;
                weigh<N, true>(s, by, step, ref[0], prod, sum);
            }
            total[0] += sum;
            u32x4 pp;
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
                const uint32_t two = as_u32(half2v{(_Float16)prod[2 * k], (_Float16)prod[2 * k + 1]});
                zeros[0] = zero_sum<0>(two, vp[2 * k], zeros[0]);
                zeros[0] = zero_sum<1>(two, vp[2 * k + 1], zeros[0]);
                pp[k] = tile ? 0u : two;
                pp[2 + k] = tile ? two : 0u;
            }
            pw[0] = __builtin_bit_cast(half8, pp);
        } else {
            // sum_d q_d (c_d - z) = (sum_d q_d c_d) - z sum_d q_d
            uint32_t vp[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const u32x4 kp = *reinterpret_cast<const u32x4*>(slot + R::P_AT + 64 * t + 16 * g), v4 = *reinterpret_cast<const u32x4*>(slot + R::P_AT + 128 + 64 * t + 16 * g);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        sc[n][t][r] = times_step(kp[r], __builtin_fmaf((float)zero_bits(kp[r]), q_sum[n], sc[n][t][r]));
                    vp[4 * t + r] = v4[r];
                }
            }
            if constexpr (kScored<DEV>)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float from = (float)(k0 + 4 * g - sight[n].hi);          // (no slopes in trees: hi is the row's position)
                    float s8[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) s8[k] = if_finite(sc[n][k >> 2][k & 3] * factor[n]);
                    rescore(p, s8, slope[n], [&](int k) { return from + (float)(16 * (k >> 2) + (k & 3)); });
#pragma unroll
                    for (int k = 0; k < 8; ++k) sc[n][k >> 2][k & 3] = s8[k];
                }
            if (!whole()) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bool page_ok = (unsigned)pg[t] < (unsigned)p.c.pages;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int k = k0 + 16 * t + 4 * g + r;
                        const bool held = page_ok & (k < span.end);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            bool ok = sees(sight[n], k);
                            if (p.visible) ok |= sees_drafted(sight[n], before, k);
                            sc[n][t][r] = (ok & held) ? if_number(vp[4 * t + r], sc[n][t][r]) : -__builtin_inff();
                        }
                        vp[4 * t + r] = usable_parameters(vp[4 * t + r]);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float s8[8], prod[8], sum;
                auto by = [&](int) { return unit_of(p, factor[n]); };
                auto step = [&](int k) { return (float)step_bits(vp[k]); };
#pragma unroll
                for (int k = 0; k < 8; ++k) s8[k] = sc[n][k >> 2][k & 3];
                if (weigh<8, false>(s8, by, step, ref[n], prod, sum)) {
                    const float f = raise_reference<8>(s8, by, step, ref[n], 7.0f, [](float top) { return across_groups(top, fmax_op); });
                    total[n] *= f;
                    zeros[n] *= f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[n][j] *= f;
                    weigh<8, true>(s8, by, step, ref[n], prod, sum);
                }
                total[n] += sum;
                u32x4 pp;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    pp[k] = as_u32(half2v{(_Float16)prod[2 * k], (_Float16)prod[2 * k + 1]});
                    zeros[n] = zero_sum<0>(pp[k], vp[2 * k], zeros[n]);
                    zeros[n] = zero_sum<1>(pp[k], vp[2 * k + 1], zeros[n]);
                }
                pw[n] = __builtin_bit_cast(half8, pp);
            }
        }
        uint32_t vc[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) vc[k] = ring_value<VB>(slot + R::V_AT + (k >> 2) * R::V_PIECE, i, g, k & 3);
        auto values = [&](auto part) {
            constexpr int HALF = decltype(part)::value;
            uint32_t vv[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) ValueCodes<VB>::template fields<HALF>(vc[2 * k], vc[2 * k + 1], vv[k], NoMasks{});
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u32x4 a = {vv[0][j], vv[1][j], vv[2][j], vv[3][j]};
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    acc[n][4 * HALF + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), pw[n], acc[n][4 * HALF + j], 0, 0, 0);
            }
        };
        values(std::integral_constant<int, 0>{});
        __builtin_amdgcn_sched_barrier(0);                                 // (four channels' fragments at a time: registers)
        values(std::integral_constant<int, 1>{});
    };
    if (any) {
        int slot = 0;
        for (; x < x_end; x += NW) {
            if (x + NW < x_end) wait_vm_pending<R::LOADS>();                   // the next step alone may still be on its way
            else wait_vm_pending<0>();
            int next[2];
            pages_of(x + NW * (DEPTH + 1), next);
            work(x, pg[0], ring + slot * R::SLOT);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                 // the slot has been read: it may take another step
            if (x + NW * DEPTH < x_end) load(x + NW * DEPTH, pg[DEPTH], slot);
#pragma unroll
            for (int k = 0; k < DEPTH; ++k) {
                pg[k][0] = pg[k + 1][0];
                pg[k][1] = pg[k + 1][1];
            }
            pg[DEPTH][0] = next[0];
            pg[DEPTH][1] = next[1];
            slot = slot + 1 == DEPTH ? 0 : slot + 1;
        }
    }

    if constexpr (V > 1) {                                                     // the columns of a row meet
        const float top = __builtin_fmaxf(ref[0], dpp_move<0x128>(ref[0]));    // row_ror:8
        const float f = __builtin_amdgcn_exp2f(ref[0] - top);
        ref[0] = top;
        auto meet = [&](float x) {
            x *= f;
            return x + dpp_move<0x128>(x);
        };
        total[0] = meet(total[0]);
        zeros[0] = meet(zeros[0]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[0][j][r] = meet(acc[0][j][r]);
    }
    // ---- the waves meet
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        total[n] = across_groups(total[n], fadd_op);
        zeros[n] = across_groups(zeros[n], fadd_op) * 0x1p24f;
        if (g == 0) {
            refs[w][16 * n + i] = ref[n];
            totals[w][16 * n + i] = total[n];
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float top = refs[0][16 * n + i];
#pragma unroll
        for (int k = 1; k < NW; ++k) top = __builtin_fmaxf(top, refs[k][16 * n + i]);
        const float f = __builtin_amdgcn_exp2f(ref[n] - top);
        if (n > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o[j] = __builtin_fmaf(acc[n][4 * half + j][r], f * (float)(1 << (24 - ValueCodes<VB>::shift(4 * half + j))), -zeros[n] * f);
                *reinterpret_cast<f32x4*>(&sums[w][i][8 * (4 * g + r) + 4 * half]) = o;
            }
        __syncthreads();
        // 16 rows of 128 channels: 2048 / (64 NW) channels a thread
        constexpr int CH = 32 / NW;
        const int rr = threadIdx.x / (ATT_D / CH), d = CH * (threadIdx.x % (ATT_D / CH));
        const int r = row0 + 16 * n + rr;
        if (r < row_end) {
            float ref_all = refs[0][16 * n + rr], sum = 0.0f, o[CH] = {};
#pragma unroll
            for (int k = 1; k < NW; ++k) ref_all = __builtin_fmaxf(ref_all, refs[k][16 * n + rr]);
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                sum += totals[k][16 * n + rr] * __builtin_amdgcn_exp2f(refs[k][16 * n + rr] - ref_all);
#pragma unroll
                for (int e = 0; e < CH; ++e) o[e] += sums[k][rr][d + e];
            }
            const int64_t token = seq.first + r / p.G;
            const int hq = head * p.G + r % p.G;
            if (!partial) {
                const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
                typedef _Float16 halves __attribute__((ext_vector_type(CH)));
                halves y;
#pragma unroll
                for (int e = 0; e < CH; ++e) y[e] = (_Float16)(outcome<DEV>(o[e]) * inv);
                *reinterpret_cast<halves*>(p.out + token * p.out_stride + hq * ATT_D + d) = y;
            } else {
                typedef float floats __attribute__((ext_vector_type(CH)));
                const int64_t at = partial_at + 16 * n + rr;
                floats y;
#pragma unroll
                for (int e = 0; e < CH; ++e) y[e] = o[e];
                *reinterpret_cast<floats*>(p.part + at * ATT_D + d) = y;
                if (d == 0) reinterpret_cast<float2*>(p.stats)[at] = float2{ref_all, sum};
            }
        }
    }
    __syncthreads();                                                           // what follows fills the ring again
}

// A tile of rows, and the steps of the rows' span, of a sequence of few rows.
struct Tile {
    int row0, row_end;
    Span span;
};
template <int ROWS>
__device__ __forceinline__ Tile tile_of(const AttnDev& p, const Sequence& seq, int tile, int prefix) {
    Tile t;
    const int all = seq.rows * p.G, before = seq.length - seq.rows;
    t.row0 = tile * ROWS;
    t.row_end = t.row0 + ROWS < all ? t.row0 + ROWS : all;
    t.span = span_of(p, seq.length, before + t.row0 / p.G, before + (t.row_end - 1) / p.G, prefix);
    return t;
}

// blockIdx: (sequence and head, tile of rows).
template <int KB, int VB, int NT, int NW, typename DEV, int V = 1>
__global__ __launch_bounds__(64 * NW, NW > 4 ? 4 : NT == 1 ? 3 : 2) void whole_attention_kernel(DEV p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int b = blockIdx.x / p.c.H, head = blockIdx.x - b * p.c.H;
    const Sequence seq = sequence_of(p.c, b);
    constexpr int ROWS = 16 * NT / V;
    const int tiles = (seq.rows * p.G + ROWS - 1) / ROWS;
    for (int tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
        const Tile t = tile_of<ROWS>(p, seq, tiles - 1 - tile, prefix_of(p, b));       // the last rows, which see most, first
        few_rows<KB, VB, NT, NW, V>(p, smem, b, head, seq, t.row0, t.row_end, t.span, 0, t.span.steps, false, 0);
    }
}

// The balanced launch: the steps of all sequences and heads behind each other, in units of 4 (128 tokens), are cut into gridDim.x equal stretches, whatever
// the lengths.  A workgroup goes through the (sequence, head) pairs of its stretch; the first and the last may be shared with its neighbours, and leave
// partial results in the workgroup's two places.
// A sequence that has none of the units is gone through whole, a head a workgroup.
constexpr int kBalancedSequences = 256;
// Units of one head of a sequence (one for rows that see nothing: they still have an output); 0: not among the units, because it has no rows, more of them
// than a tile, or so many tokens that the units of all sequences would pass 32 bits.
template <int ROWS>
__device__ __forceinline__ int share_of(const AttnDev& p, const Sequence& seq, int prefix) {
    if (seq.rows <= 0 || seq.rows * p.G > ROWS) return 0;
    const int n = (tile_of<ROWS>(p, seq, 0, prefix).span.steps + 3) >> 2;
    return n > 0x7f000000 / kBalancedSequences / p.c.H ? 0 : n > 1 ? n : 1;
}
struct Cut {                  // in LDS
    int first[kBalancedSequences], rows[kBalancedSequences], length[kBalancedSequences];
    int share[kBalancedSequences], begin[kBalancedSequences];                 // units of a head, first unit
    int all, per;             // units of all, of a workgroup
};
// The first wave works the cut out, a lane four sequences, for the workgroup.
template <int ROWS, typename DEV>
__device__ __forceinline__ void make_cut(const DEV& p, int workgroups, Cut& cut) {
    if (threadIdx.x < 64) {
        const int l = threadIdx.x;
        int share[4], mine = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int b = l + 64 * k;
            Sequence seq{0, 0, 0};
            if (b < p.c.B) {
                const int first = p.c.row_starts[b], last = p.c.row_starts[b + 1], T = (int)p.c.T;
                seq.length = p.c.lengths[b];
                seq.first = first > 0 ? first : 0;
                seq.rows = (last < T ? last : T) - seq.first;
            }
            cut.first[b] = seq.first;
            cut.rows[b] = seq.rows;
            cut.length[b] = seq.length;
            cut.share[b] = share[k] = share_of<ROWS>(p, seq, b < p.c.B ? prefix_of(p, b) : 0);
        }
        // the order of the units is that of (k, lane): sequences in their order
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            int sum = share[k] * p.c.H;
            if (64 * k < p.c.B) {
#pragma unroll
                for (int m = 1; m < 64; m *= 2) {
                    const int other = __shfl_up(sum, m);
                    sum += l >= m ? other : 0;
                }
            }
            cut.begin[l + 64 * k] = mine + sum - share[k] * p.c.H;
            mine += __builtin_amdgcn_readlane(sum, 63);
        }
        if (l == 0) {
            cut.all = mine;
            const int per = (mine + workgroups - 1) / workgroups;
            cut.per = per > p.min_units ? per : p.min_units;
        }
    }
    __syncthreads();
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Sequence sequence_of(const Cut& c, int b) { return Sequence{uniform(c.first[b]), uniform(c.rows[b]), uniform(c.length[b])}; }
// The sequence that has unit u: the last that begins at u or before (those without units begin where the next one does).
__device__ __forceinline__ int sequence_at(const Cut& c, int B, int u) {
    const int l = threadIdx.x & 63;
    int n = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) n += __builtin_popcountll(__ballot(l + 64 * k < B && c.begin[l + 64 * k] <= u));
    return n - 1;
}

template <int KB, int VB, int NT, int NW, typename DEV, int V = 1>
__global__ __launch_bounds__(64 * NW, NT == 1 ? 3 : 2) void balanced_attention_kernel(DEV p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    constexpr int ROWS = 16 * NT / V;
    Cut& cut = *reinterpret_cast<Cut*>(smem + FewRows<KB, VB, NT, NW>::LDS);
    make_cut<ROWS>(p, gridDim.x, cut);
    const int wg = blockIdx.x, per = uniform(cut.per), begin = wg * per, end = min(begin + per, uniform(cut.all));
    int u = begin, bh = wg, tile = 0;                                          // then, pair by pair and tile by tile, what is not among the units
    for (;;) {
        const bool units = u < end;
        int b, head, from = 0, to = 0x7fffffff / 4;
        bool partial = false;
        int64_t at = 0;
        if (units) {
            b = sequence_at(cut, p.c.B, u);
            const int n = uniform(cut.share[b]), in = u - uniform(cut.begin[b]);
            head = in / n;
            from = in - head * n;
            to = min(n, from + end - u);
            partial = from > 0 || to < n;
            at = ((int64_t)2 * wg + (u == begin ? 0 : 1)) * ROWS;
            u += to - from;
        } else {
            if (bh >= p.c.B * p.c.H) break;
            b = bh / p.c.H;
            head = bh - b * p.c.H;
            if (uniform(cut.share[b]) || tile * ROWS >= uniform(cut.rows[b]) * p.G) {
                bh += gridDim.x;
                tile = 0;
                continue;
            }
        }
        const Sequence seq = sequence_of(cut, b);
        const Tile t = tile_of<ROWS>(p, seq, tile, prefix_of(p, b));
        tile += !units;
        few_rows<KB, VB, NT, NW, V>(p, smem, b, head, seq, t.row0, t.row_end, t.span, 4 * from, min(t.span.steps, 4 * to), partial, at);
    }
}

// Joins the partial results of the (sequence, head) pairs that more than one workgroup had: blockIdx (pair, part of its rows).  Up to 16 workgroups: a wave a row;
// more: a row at a time, its workgroups dealt out to the waves.
template <int NT, typename DEV, int V = 1>
__global__ __launch_bounds__(ATT_NT) void balanced_join_kernel(DEV p, int workgroups) {
    __shared__ float tops[ATT_WAVES], totals[ATT_WAVES], sums[ATT_WAVES][ATT_D];
    constexpr int ROWS = 16 * NT / V;
    const int l = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / p.c.H, head = blockIdx.x - b * p.c.H;
    __shared__ Cut cut;
    make_cut<ROWS>(p, workgroups, cut);
    const Sequence seq = sequence_of(cut, b);
    const int n = uniform(cut.share[b]), per = uniform(cut.per), u = uniform(cut.begin[b]) + head * n;
    const int first = u / per, last = (u + n - 1) / per;
    if (n == 0 || first == last) return;
    constexpr int AT_ONCE = 16;
    const bool together = last - first >= AT_ONCE;
    for (int r = together ? blockIdx.y : ATT_WAVES * blockIdx.y + w; r < seq.rows * p.G; r += together ? gridDim.y : ATT_WAVES * gridDim.y) {
        auto place = [&](int wg) { return ((int64_t)2 * wg + (wg > first || u == first * per ? 0 : 1)) * ROWS + r; };
        const int from = together ? first + w : first, by = together ? ATT_WAVES : 1;
        float top = ATT_NONE, sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
        for (int k = from; k <= last; k += AT_ONCE * by) {
            float2 s[AT_ONCE], v[AT_ONCE];
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) {
                const int64_t at = place(min(k + by * e, last));
                s[e] = reinterpret_cast<const float2*>(p.stats)[at];
                v[e] = reinterpret_cast<const float2*>(p.part + at * ATT_D)[l];
            }
            float to = top;
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) to = __builtin_fmaxf(to, s[e].x);
            const float f = __builtin_amdgcn_exp2f(top - to);
            top = to;
            sum *= f;
            o0 *= f;
            o1 *= f;
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) {
                const float g = k + by * e <= last ? __builtin_amdgcn_exp2f(s[e].x - to) : 0.0f;
                sum += s[e].y * g;
                o0 += v[e].x * g;
                o1 += v[e].y * g;
            }
        }
        if (together) {
            if (l == 0) {
                tops[w] = top;
                totals[w] = sum;
            }
            reinterpret_cast<float2*>(sums[w])[l] = float2{o0, o1};
            __syncthreads();
            float all = tops[0];
#pragma unroll
            for (int k = 1; k < ATT_WAVES; ++k) all = __builtin_fmaxf(all, tops[k]);
            sum = o0 = o1 = 0.0f;
#pragma unroll
            for (int k = 0; k < ATT_WAVES; ++k) {
                const float f = __builtin_amdgcn_exp2f(tops[k] - all);
                const float2 v = reinterpret_cast<const float2*>(sums[k])[l];
                sum += totals[k] * f;
                o0 += v.x * f;
                o1 += v.y * f;
            }
            __syncthreads();
        }
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        const int64_t token = seq.first + r / p.G;
        if (!together || w == 0)
            reinterpret_cast<half2v*>(p.out + token * p.out_stride + (head * p.G + r % p.G) * ATT_D)[l] = half2v{(_Float16)(outcome<DEV>(o0) * inv), (_Float16)(outcome<DEV>(o1) * inv)};
    }
}

// ---- many rows: the tokens' codes become fp16 once per workgroup
//
// Waves of 32 rows each on v_mfma_f32_32x32x16_f16.  Four of them turn 64 tokens into fp16 in the LDS buffer of the next step (waves 0 and 1 the
// keys of one half of them, waves 2 and 3 the values) while all attend to those of this one; eight waves take 128 tokens a step, and so convert half as
// much a row.  Keys lie row by row in the order of their codes, values channel by channel with the eight tokens of a fragment (those whose weights a
// lane holds) in 16 bytes.  16 bytes of padding a row spread the reads of a fragment over all banks, and leave one address a lane and constants (chunks
// exchanged by row took 45 registers of addresses, and spilled).
//
// Bound by issue: 2048 rows of 64 heads at 8192 tokens take 505 us (0.95 PFLOP/s) launch after launch, once the clock has settled, which takes about 70 of them
// (610 in the first ones after a pause).  The matrix cores are busy for 38 % of it and the vector units for 45 % (a wave's 16 weights of a tile cost 90 instructions and 16 exponentials, twice what its 16 matrix instructions take): two waves a SIMD, all
// that the registers allow, overlap the two only in part.  Raised wave priority around the matrix instructions was slower (640 / 615, both after a pause), and so
// was the conversion at the start of a step for half of the waves (635 / 615).

constexpr int SH_ROWS = 32;                // rows per wave
constexpr int SH_K_PITCH = 2 * ATT_D + 16, SH_V_PITCH = 2 * 64 + 16;
constexpr int SH_K_BYTES = 64 * SH_K_PITCH, SH_V_BYTES = ATT_D * SH_V_PITCH, SH_STEP_BYTES = 2 * 64 * 4;
constexpr int SH_BUFFER = SH_K_BYTES + SH_V_BYTES + SH_STEP_BYTES;

// x, as far as the compiler can tell another one every time: what follows from it is worked out where it is used and not kept in registers over the loop, of
// which a wave has all (a spilled one waits for every load on its way).
__device__ __forceinline__ int again(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A thread's share of 64 tokens: two quarters of a key, or eight channels of eight values, and which of the four pages of 16 tokens are pages.
// (Vectors that both kinds of waves assign as a whole, behind their branch: of arrays that each branch stores into, two words stay in memory, and every step then
// waits for its loads at once.)
struct ShareCodes {
    u32x4 words[2], parameters[2];
    __device__ __forceinline__ uint32_t w(int k) const { return words[k >> 2][k & 3]; }
    __device__ __forceinline__ uint32_t params(int k) const { return parameters[k >> 2][k & 3]; }
    int pages;                             // (uniform) bit k: tokens 16 k .. of the 64
};

template <int KB, int VB, int NW, typename DEV>
__global__ __launch_bounds__(64 * NW, 2) void shared_attention_kernel(DEV p) {
    constexpr int PARTS = NW / 4;                                              // of 64 tokens, a step
    extern __shared__ __attribute__((aligned(16))) unsigned char sh_smem[];
    const int l = threadIdx.x & 63, c = l & 31, h = l >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / p.c.H, head = blockIdx.x - b * p.c.H;
    const Sequence seq = sequence_of(p.c, b);
    const int all_rows = seq.rows * p.G;
    constexpr int TILE = SH_ROWS * NW;
    const int prefix = prefix_of(p, b);
    const int part = w / 4, role = w % 4;
    const int tiles = (all_rows + TILE - 1) / TILE;
    for (int tile_no = blockIdx.y; tile_no < tiles; tile_no += gridDim.y) {
        const int row0 = (tiles - 1 - tile_no) * TILE;
        const int row_end = row0 + TILE < all_rows ? row0 + TILE : all_rows;
        const int before = seq.length - seq.rows;
        const Span span = span_of(p, seq.length, before + row0 / p.G, before + (row_end - 1) / p.G, prefix);
        const int used = splits_used(p, span.steps);
        if ((int)blockIdx.z >= used) continue;
        const int per = steps_of_split(p, span.steps);
        const int x_begin = (int)blockIdx.z * per;
        const int x_end = (int)blockIdx.z == p.splits - 1 ? span.steps : min(span.steps, x_begin + per);

        // this wave's rows; of 64 or fewer, waves 2 and 3 have those of waves 0 and 1, and each the tokens of its half of a step
        const bool halved = NW == 4 && row_end - row0 <= 2 * SH_ROWS;
        const int my_half = w >> 1;
        const int wrow0 = row0 + SH_ROWS * (halved ? w & 1 : w), wrow_end = wrow0 + SH_ROWS < row_end ? wrow0 + SH_ROWS : row_end;
        const bool busy = wrow0 < wrow_end;
        const int pos_lo = before + wrow0 / p.G, pos_hi = before + (wrow_end - 1) / p.G;
        int r = wrow0 + c;
        r = r < row_end ? r : row_end - 1;
        const int token = r / p.G, sub = r - token * p.G;
        half8 q[8];                                                            // fragment k: chunk 2 k + h of the key rows
        {
            const _Float16* src = p.q + (seq.first + token) * p.q_stride + (head * p.G + sub) * ATT_D;
#pragma unroll
            for (int quarter = 0; quarter < 4; ++quarter) {
                half8 raw[4];
#pragma unroll
                for (int m = 0; m < 4; ++m) raw[m] = *reinterpret_cast<const half8*>(src + 32 * quarter + 8 * m);
                auto pick = [&](int at) { return raw[at >> 3][at & 7]; };
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int lo = 8 * k + e, hi = lo + 4;                 // pairs of chunk 2 k and of chunk 2 k + 1
                        q[2 * quarter + k][2 * e] = h ? pick(KeyCodes<KB>::first(hi)) : pick(KeyCodes<KB>::first(lo));
                        q[2 * quarter + k][2 * e + 1] = h ? pick(KeyCodes<KB>::second(hi)) : pick(KeyCodes<KB>::second(lo));
                    }
            }
            // A row with such a channel: none of them, so that every score is none (infinite ones tanh would make numbers of).  Nothing in the loop.
            if constexpr (kScored<DEV>) {
                uint32_t none = 0;                                             // bits 15 and 31: of a channel that is an infinity or no number
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) none |= (__builtin_bit_cast(u32x4, q[k])[e] & 0x7C007C00u) + 0x04000400u;
                none |= __shfl_xor(none, 32);
                if (__any(none & 0x80008000u)) {
                    const uint32_t fill = none & 0x80008000u ? 0x7E007E00u : 0u;
#pragma unroll
                    for (int k = 0; k < 8; ++k) q[k] = __builtin_bit_cast(half8, __builtin_bit_cast(u32x4, q[k]) | fill);
                }
            }
        }
        f32x16 acc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[t][k] = 0.0f;
        float ref = ATT_NONE, total = 0.0f, slope = 0.0f;
        if constexpr (kScored<DEV>) slope = slope_of(p, head * p.G + sub);

        const int lower = backwards(p) ? 1 : 0;                                // which of two steps has the lower tokens
        // codes of steps x and x + 1 of the span, 32 tokens each, which need not follow each other
        // The page of tokens 16 n .. of the step from x on, by every lane n of NW: looked up in all lanes at once (a scalar look-up each took more time than the
        // conversion), a step before the loads that follow it, in whose queue it stands.
        auto page_of = [&](int x) {
            const int n = again(l) % NW, y = in_order(p, span.steps, x + (n >> 1));
            const unsigned token = (unsigned)((y < span.first_steps ? ATT_STEP * y : span.begin + ATT_STEP * (y - span.first_steps)) + 16 * (n & 1));
            const unsigned j = token >> p.c.page_shift, last = (unsigned)p.c.table_width - 1u;
            return p.c.page_table[b * p.c.table_stride + (j < last ? j : last)];           // (behind the width: behind the end)
        };
        auto load = [&](int x, int page, ShareCodes& s) {
            const bool ok = (unsigned)page < (unsigned)p.c.pages;
            s.pages = (int)__ballot(ok) & ((1 << NW) - 1);
            const int held = ok ? page : 0, mine = 2 * (2 * part + w % 2);
            const int pg[2] = {__builtin_amdgcn_readlane(held, mine), __builtin_amdgcn_readlane(held, mine + 1)};      // of this wave's 32 tokens
            const int k0 = span.token(in_order(p, span.steps, x + 2 * part + w % 2));
            const int mask = (1 << p.c.page_shift) - 1;
            const int lane = again(l);
            u32x4 words[2] = {}, parameters[2] = {};
            if (role < 2) {                                                    // token c of the half, quarters 2 h and 2 h + 1
                const int c = lane & 31, h = lane >> 5;
                const int64_t at = (((int64_t)(c < 16 ? pg[0] : pg[1]) * p.c.H + head) << p.c.page_shift) + ((k0 + c) & mask);
                typedef uint32_t words2 __attribute__((ext_vector_type(2)));
                const words2* from = reinterpret_cast<const words2*>(p.c.codes[0] + at * (16 * KB) + h * (8 * KB));
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    const words2 two = from[k];
                    words[k >> 1][2 * (k & 1)] = two[0];
                    words[k >> 1][2 * (k & 1) + 1] = two[1];
                }
                parameters[0][0] = p.c.params[0][at];
            } else {                                                           // channels 8 i .. 8 i + 7 of tokens 16 (g >> 1) + 4 (g & 1) + {0 .. 3, 8 .. 11}
                const int i = lane & 15, g = lane >> 4;
                const int64_t at = (((int64_t)(g < 2 ? pg[0] : pg[1]) * p.c.H + head) << p.c.page_shift) +
                                   ((k0 + 16 * (g >> 1) + 4 * (g & 1)) & mask);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint8_t* row = p.c.codes[1] + (at + (k & 3) + 8 * (k >> 2)) * (16 * VB);
                    if constexpr (VB == 4) words[k >> 2][k & 3] = reinterpret_cast<const uint32_t*>(row)[i];
                    else if constexpr (VB == 2) words[k >> 2][k & 3] = reinterpret_cast<const uint16_t*>(row)[i];
                    else {
                        typedef uint32_t loose __attribute__((aligned(1)));
                        words[k >> 2][k & 3] = *reinterpret_cast<const loose*>(row + (i < 15 ? 3 * i : 44));
                    }
                }
                parameters[0] = *reinterpret_cast<const u32x4*>(p.c.params[1] + at);
                parameters[1] = *reinterpret_cast<const u32x4*>(p.c.params[1] + at + 8);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                s.words[k] = words[k];
                s.parameters[k] = parameters[k];
            }
        };
        auto convert = [&](const ShareCodes& s, int buf) {
            unsigned char* base = sh_smem + (PARTS * buf + part) * SH_BUFFER;
            float* steps = reinterpret_cast<float*>(base + SH_K_BYTES + SH_V_BYTES);
            if (role < 2) {
                const Masks<KB> masks;
                const half2v z = raised_zeros(masks, s.params(0), s.params(0));
                const int tok = 32 * role + c;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    typename KeyCodes<KB>::words cw;
#pragma unroll
                    for (int k = 0; k < KB; ++k) cw[k] = s.w(KB * half + k);
                    uint32_t kk[16];
                    KeyCodes<KB>::fields(cw, kk, masks);
                    each<4>([&](auto mm) {
                        constexpr int m = decltype(mm)::value;
                        const int chunk = 4 * (2 * h + half) + m;
                        u32x4 o;
                        each<4>([&](auto ee) {
                            constexpr int e = decltype(ee)::value;
                            o[e] = as_u32(code_value<KeyCodes<KB>::shift(4 * m + e)>(kk[4 * m + e], z));
                        });
                        *reinterpret_cast<u32x4*>(base + tok * SH_K_PITCH + 16 * chunk) = o;
                    });
                }
                if (h == 0) steps[tok] = key_factor(p, step_of(s.params(0)));
            } else {
                const int i = l & 15, g = l >> 4, chunk = 4 * (role - 2) + g;
                const Masks<VB> masks;
                auto values = [&](auto part) {
                    constexpr int HALF = decltype(part)::value;
                    uint32_t vv[4][4];
                    half2v z[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        z[k] = raised_zeros(masks, s.params(2 * k), s.params(2 * k + 1));
                        const int down = VB == 3 && i == 15 ? 8 : 0;
                        ValueCodes<VB>::template fields<HALF>(s.w(2 * k) >> down, s.w(2 * k + 1) >> down, vv[k], masks);
                    }
                    each<4>([&](auto jj) {
                        constexpr int j = decltype(jj)::value;
                        const int row = 16 * (4 * HALF + j) + i;               // of channel 8 i + 4 HALF + j: the lanes' rows lie next to each other
                        u32x4 o;
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[k] = as_u32(code_value<ValueCodes<VB>::shift(4 * HALF + j)>(vv[k][j], z[k]));
                        *reinterpret_cast<u32x4*>(base + SH_K_BYTES + row * SH_V_PITCH + 16 * chunk) = o;
                    });
                };
                values(std::integral_constant<int, 0>{});
                values(std::integral_constant<int, 1>{});
                if (i == 0) {
                    f32x4* at = reinterpret_cast<f32x4*>(steps + 64 + 32 * (role - 2) + 16 * (g >> 1) + 4 * (g & 1));
                    at[0] = f32x4{step_of(s.params(0)), step_of(s.params(1)), step_of(s.params(2)), step_of(s.params(3))};
                    at[2] = f32x4{step_of(s.params(4)), step_of(s.params(5)), step_of(s.params(6)), step_of(s.params(7))};
                }
            }
        };
        // Two tiles of 32 tokens a step.  The matrix instructions of one stage stand between the vector instructions of another:
        // QK of tile 0 with the conversion of the next step, QK of tile 1 with the weights of tile 0, PV of tile 0 with the weights of tile 1.
        auto scores = [&](const unsigned char* base, int t, f32x16& sc) {
#pragma unroll
            for (int k = 0; k < 16; ++k) sc[k] = 0.0f;
            half8 a[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) a[k] = *reinterpret_cast<const half8*>(base + (32 * t + c) * SH_K_PITCH + 16 * h + 32 * k);
#pragma unroll
            for (int k = 0; k < 8; ++k) sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[k], q[k], sc, 0, 0, 0);
        };
        auto factors = [&](const unsigned char* base, int at, float (&f)[16]) {
            const float* from = reinterpret_cast<const float*>(base + SH_K_BYTES + SH_V_BYTES) + at + 4 * h;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(from + 8 * k);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[4 * k + e] = v[e];
            }
        };
        auto factor_of = [&](const float (&fk)[16], int k) {
            if constexpr (kScored<DEV>) return p.unit;                         // (the keys' steps are in the scores by then)
            else return fk[k];
        };
        // scores of tokens that a row does not see: -infinity (the factors are one then), and steps of zero: a weight of zero times what the page holds, an
        // infinity of either sign or a NaN, need not be zero
        auto mask = [&](int x, int t, int pages, f32x16& sc, float (&fk)[16], float (&vs)[16]) {
            const int k0 = span.token(in_order(p, span.steps, x + t));
            const int pages_ok = pages >> (2 * t) & 3, all_see = p.visible ? before - 1 : last_of(pos_lo, prefix);
            if (pages_ok == 3 && k0 + 31 <= all_see && k0 + 32 <= span.end && x + t < x_end && (p.window <= 0 || p.visible || k0 > pos_hi - p.window)) return;
            const int end = x + t < x_end ? span.end : kScored<DEV> ? -0x7fffffff : 0;        // (in the other order tokens behind the last step are below zero)
            const int row = again(token);
            const Sight sight = sight_of(p, before, row, seq.first + row, prefix);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int kk = k0 + 8 * (k >> 2) + 4 * h + (k & 3);
                bool ok = sees(sight, kk);
                if (p.visible) ok |= sees_drafted(sight, before, kk);
                ok = ok & (kk < end) & (pages_ok >> (k >> 3) & 1);
                if constexpr (kScored<DEV>) {
                    sc[k] = ok ? sc[k] : -__builtin_inff();
                } else {
                    sc[k] = ok ? sc[k] * fk[k] : -__builtin_inff();
                    fk[k] = 1.0f;
                }
                vs[k] = ok ? vs[k] : 0.0f;
            }
        };
        auto raise = [&](const f32x16& sc, const float (&fk)[16], const float (&vs)[16], float (&prod)[16], float& sum) {
            auto by = [&](int k) { return factor_of(fk, k); };
            auto step = [&](int k) { return vs[k]; };
            const float f = raise_reference<16>(sc, by, step, ref, largest_of(p, span), [](float top) { return __builtin_fmaxf(top, __shfl_xor(top, 32)); });
            total *= f;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[dt][k] *= f;
            weigh<16, true>(sc, by, step, ref, prod, sum);
        };
        auto values = [&](const unsigned char* base, int t, const half8 (&pw)[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    const half8 a = *reinterpret_cast<const half8*>(base + SH_K_BYTES + (32 * dt + c) * SH_V_PITCH + 16 * h + 64 * t + 32 * s);
                    acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, pw[s], acc[dt], 0, 0, 0);
                }
        };
        auto halves = [&](const float (&prod)[16], half8 (&pw)[2]) {
#pragma unroll
            for (int k = 0; k < 16; ++k) pw[k >> 3][k & 7] = (_Float16)prod[k];
        };

        if (x_begin < x_end) {
            ShareCodes s;
            constexpr int STEPS = 2 * PARTS;
            int next = page_of(x_begin + STEPS);
            load(x_begin, page_of(x_begin), s);
            convert(s, 0);
            int pages = s.pages;
            load(x_begin + STEPS, next, s);
            next = page_of(x_begin + 2 * STEPS);
            __syncthreads();
            int buf = 0;
            for (int x = x_begin; x < x_end; x += STEPS) {
#pragma unroll
                for (int y = 0; y < PARTS; ++y) {
                    const unsigned char* base = sh_smem + (PARTS * buf + y) * SH_BUFFER;
                    // (the first tokens lie before everything else)
                    if (!busy || x + 2 * y >= x_end || !(p.visible || span.token(in_order(p, span.steps, x + 2 * y + lower)) <= last_of(pos_hi, prefix))) continue;
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (halved && t != my_half) continue;
                        f32x16 sc;
                        float fk[16], vs[16], prod[16], sum;
                        half8 pw[2];
                        auto by = [&](int k) { return factor_of(fk, k); };
                        auto step = [&](int k) { return vs[k]; };
                        scores(base, t, sc);
                        factors(base, 32 * t, fk);
                        factors(base, 64 + 32 * t, vs);
                        if constexpr (kScored<DEV>) {
                            const float from = (float)(span.token(in_order(p, span.steps, x + 2 * y + t)) + 4 * h - before - again(token));
                            float s16[16];
#pragma unroll
                            for (int k = 0; k < 16; ++k) s16[k] = sc[k] * fk[k];
                            rescore(p, s16, slope, [&](int k) { return from + (float)(8 * (k >> 2) + (k & 3)); });
#pragma unroll
                            for (int k = 0; k < 16; ++k) sc[k] = s16[k];
                        }
                        mask(x + 2 * y, t, pages >> (4 * y), sc, fk, vs);
                        if (weigh<16, false>(sc, by, step, ref, prod, sum)) raise(sc, fk, vs, prod, sum);
                        total += sum;
                        halves(prod, pw);
                        values(base, t, pw);
                    }
                }
                convert(s, buf ^ 1);
                const int next_pages = s.pages;
                load(x + 2 * STEPS, next, s);
                next = page_of(x + 3 * STEPS);
                pages = next_pages;
                __syncthreads();
                buf ^= 1;
            }
        }
        total += __shfl_xor(total, 32);
        if (halved) {                                                          // waves 2 and 3 hand theirs over, through what the loop is done with
            f32x4* sums = reinterpret_cast<f32x4*>(sh_smem) + (w & 1) * (16 * 64);
            float2* stats = reinterpret_cast<float2*>(sh_smem + 2 * 16 * 64 * 16) + (w & 1) * 64;
            if (my_half == 1) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const f32x16& from = acc[k >> 2];
                    sums[64 * k + l] = f32x4{from[4 * (k & 3)], from[4 * (k & 3) + 1], from[4 * (k & 3) + 2], from[4 * (k & 3) + 3]};
                }
                stats[l] = float2{ref, total};
            }
            __syncthreads();
            if (my_half == 0) {
                const float2 other = stats[l];
                const float top = __builtin_fmaxf(ref, other.x), f = __builtin_amdgcn_exp2f(ref - top), g = __builtin_amdgcn_exp2f(other.x - top);
                ref = top;
                total = total * f + other.y * g;
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const f32x4 o = sums[64 * k + l];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[k >> 2][4 * (k & 3) + e] = acc[k >> 2][4 * (k & 3) + e] * f + o[e] * g;
                }
            }
        }
        if (wrow0 + c < wrow_end && !(halved && my_half == 1)) {
            const int64_t row_token = seq.first + token;
            const int hq = head * p.G + sub;
            if (used == 1) {
                const float inv = total > 0.0f ? 1.0f / total : 0.0f;
                _Float16* dst = p.out + row_token * p.out_stride + hq * ATT_D;
                // rows 16 j + i of the product: a lane has all eight j of i = 4 h + {0 .. 3, 8 .. 11}, channels 8 i .. 8 i + 7
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    half8 y;
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = (_Float16)(outcome<DEV>(acc[j >> 1][k + 8 * (j & 1)]) * inv);
                    *reinterpret_cast<half8*>(dst + 8 * (8 * (k >> 2) + 4 * h + (k & 3))) = y;
                }
            } else {
                const int64_t at = (row_token * p.Hq + hq) * p.splits + blockIdx.z;
                float* dst = p.part + at * ATT_D;
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int j = 0; j < 8; j += 4)
                        *reinterpret_cast<f32x4*>(dst + 8 * (8 * (k >> 2) + 4 * h + (k & 3)) + j) =
                            f32x4{acc[j >> 1][k], acc[j >> 1][k + 8], acc[(j >> 1) + 1][k], acc[(j >> 1) + 1][k + 8]};
                if (h == 0) {
                    reinterpret_cast<float2*>(p.stats)[at] = float2{ref, total};
                }
            }
        }
        __syncthreads();                                                       // the next tile writes buffer 0
    }
}

// Joins the splits of every (row, query head) that has more than one: one wave each, two channels a lane.  ROWS: of the tiles that were split.
template <int ROWS, typename DEV>
__global__ __launch_bounds__(ATT_NT) void attention_join_kernel(DEV p) {
    const int l = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / p.c.H, head = blockIdx.x - b * p.c.H;
    const Sequence seq = sequence_of(p.c, b);
    const int all_rows = seq.rows * p.G;
    for (int r = (int)blockIdx.y * ATT_WAVES + w; r < all_rows; r += (int)gridDim.y * ATT_WAVES) {
        const int row0 = r / ROWS * ROWS, row_end = row0 + ROWS < all_rows ? row0 + ROWS : all_rows;
        const int before = seq.length - seq.rows;
        const Span span = span_of(p, seq.length, before + row0 / p.G, before + (row_end - 1) / p.G, prefix_of(p, b));
        const int used = splits_used(p, span.steps);
        if (used == 1) continue;
        const int64_t token = seq.first + r / p.G;
        const int hq = head * p.G + r % p.G;
        const int64_t at = (token * p.Hq + hq) * p.splits;
        const float2* pair = reinterpret_cast<const float2*>(p.stats) + at;
        const float2* part = reinterpret_cast<const float2*>(p.part + at * ATT_D) + l;
        // the splits' references and sums, a split a lane (kMaxSplits of them at most), and their factors
        float2 mine[kMaxSplits / 64];
        float top = ATT_NONE, sum = 0.0f, f[kMaxSplits / 64];
#pragma unroll
        for (int k = 0; k < kMaxSplits / 64; ++k) {
            mine[k] = 64 * k + l < used ? pair[64 * k + l] : float2{ATT_NONE, 0.0f};
            top = __builtin_fmaxf(top, mine[k].x);
        }
        top = wave_max(top);
#pragma unroll
        for (int k = 0; k < kMaxSplits / 64; ++k) {
            f[k] = __builtin_amdgcn_exp2f(mine[k].x - top);
            sum += mine[k].y * f[k];
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
        float o0 = 0.0f, o1 = 0.0f;
#pragma unroll
        for (int k = 0; k < kMaxSplits / 64; ++k)
            for (int m = 0; 64 * k + m < used && m < 64; m += 8) {
                float2 v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int x = 64 * k + m + e;
                    v[e] = part[(int64_t)(x < used ? x : used - 1) * (ATT_D / 2)];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // (a lane behind the last split holds a factor of 2^(none - top): zero, or one of an empty row's zeros)
                    const float g = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f[k]), m + e));
                    o0 += 64 * k + m + e < used ? v[e].x * g : 0.0f;
                    o1 += 64 * k + m + e < used ? v[e].y * g : 0.0f;
                }
            }
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        reinterpret_cast<half2v*>(p.out + token * p.out_stride + hq * ATT_D)[l] = half2v{(_Float16)(outcome<DEV>(o0) * inv), (_Float16)(outcome<DEV>(o1) * inv)};
    }
}

// Compute units of the card: the plan (and with it the workspace) follows from the host's figures alone.
constexpr int64_t kPlanCus = 256;

// A kernel whose dynamic LDS may be more than the default.
template <typename Kernel, typename DEV>
static hipError_t large_launch(Kernel kernel, dim3 grid, int threads, int lds, OccCache& cache, hipStream_t stream, const DEV& d) {
    int occ = 0;
    const hipError_t e = kernel_occupancy(reinterpret_cast<const void*>(kernel), threads, lds, cache, occ);
    return e == hipSuccess ? launch(kernel, grid, dim3((unsigned)threads), lds, stream, d) : e;
}
// Tiles of 16 NT rows (of 16 / V).
template <int KB, int VB, int NT, int V, typename DEV>
static hipError_t few_rows_launch(const DEV& d, const AttnPlan& plan, int64_t max_rows, hipStream_t stream) {
    static OccCache caches[4];
    constexpr int ROWS = 16 * NT / V;
    const int64_t rows = max_rows * d.G, tiles = (rows + ROWS - 1) / ROWS;
    const dim3 pairs((unsigned)(d.c.B * d.c.H), (unsigned)(tiles < 1 ? 1 : tiles > 65535 ? 65535 : tiles));
    if (plan.workgroups > 0) {
        const hipError_t e = large_launch(balanced_attention_kernel<KB, VB, NT, 4, DEV, V>, dim3((unsigned)plan.workgroups), 256,
                                          FewRows<KB, VB, NT, 4>::LDS + (int)sizeof(Cut), caches[0], stream, d);
        if (e != hipSuccess) return e;
        // a workgroup a row where there are few pairs and so many partial results of each, else one for four rows
        const int64_t parts = pairs.x < kPlanCus ? rows : (rows + ATT_WAVES - 1) / ATT_WAVES;
        const dim3 join(pairs.x, (unsigned)(parts < 1 ? 1 : parts < 16 * NT ? parts : 16 * NT));
        return launch(balanced_join_kernel<NT, DEV, V>, join, dim3(ATT_NT), 0, stream, d, plan.workgroups);
    }
    if constexpr (NT == 1) {
        if (plan.waves == 16) return large_launch(whole_attention_kernel<KB, VB, NT, 16, DEV, V>, pairs, 1024, FewRows<KB, VB, NT, 16>::LDS, caches[1], stream, d);
        if (plan.waves == 8) return large_launch(whole_attention_kernel<KB, VB, NT, 8, DEV, V>, pairs, 512, FewRows<KB, VB, NT, 8>::LDS, caches[2], stream, d);
    }
    return large_launch(whole_attention_kernel<KB, VB, NT, 4, DEV, V>, pairs, 256, FewRows<KB, VB, NT, 4>::LDS, caches[3], stream, d);
}
template <int KB, int VB, typename DEV>
static hipError_t attention_launch_bits(const DEV& d, const AttnPlan& plan, int64_t max_rows, hipStream_t stream) {
    if (plan.tile_rows == 16) {
        if constexpr (kScored<DEV>) {
            const int64_t rows = max_rows * d.G;
            // us, one column a row / two: 64 sequences of 4096, 8 heads of 1, 4 and 8 queries, capped 54.1 / 49.5, 52.5 / 48.5, 52.7 / 49.3, with slopes 51.4 / 47.5, 51.9 / 47.7,
            // 52.5 / 48.5; 1 of 1000 11.8 / 11.0 and 10.8 / 10.1.  (Four columns for four rows: as two.)
            if (rows <= 8) return few_rows_launch<KB, VB, 1, 2>(d, plan, max_rows, stream);
        }
        return few_rows_launch<KB, VB, 1, 1>(d, plan, max_rows, stream);
    }
    if (plan.tile_rows == 32) return few_rows_launch<KB, VB, 2, 1>(d, plan, max_rows, stream);
    static OccCache caches[2];
    const int64_t tiles = (max_rows * d.G + plan.tile_rows - 1) / plan.tile_rows;
    const dim3 pairs((unsigned)(d.c.B * d.c.H), (unsigned)(tiles < 1 ? 1 : tiles > 65535 ? 65535 : tiles), (unsigned)d.splits);
    if (plan.waves == 8) return large_launch(shared_attention_kernel<KB, VB, 8, DEV>, pairs, 512, 4 * SH_BUFFER, caches[0], stream, d);
    const hipError_t e = large_launch(shared_attention_kernel<KB, VB, 4, DEV>, pairs, ATT_NT, 2 * SH_BUFFER, caches[1], stream, d);
    if (e != hipSuccess || d.splits == 1) return e;
    const int64_t rows = (max_rows * d.G + ATT_WAVES - 1) / ATT_WAVES;
    return launch(attention_join_kernel<SH_ROWS * ATT_WAVES, DEV>, dim3(pairs.x, (unsigned)(rows < 1 ? 1 : rows > 65535 ? 65535 : rows)), dim3(ATT_NT), 0, stream, d);
}

// What every launch has of the arguments and the plan.
inline void fill_attention(AttnDev& d, const CacheDev& c, const AttnArgs& a, const AttnPlan& plan) {
    d.c = c;
    d.q = a.q; d.out = a.out; d.visible = a.visible; d.part = a.workspace; d.stats = a.workspace + plan.stats_at;
    d.q_stride = a.q_stride; d.out_stride = a.out_stride;
    // Scores and, times a key's step, factors stay finite: two scores of finite rows that differ do so by 2^-48 of the scale or more, so that from 2^64 on the
    // larger one has all the weight, whatever the scale.
    d.scale2 = __builtin_fminf(__builtin_fmaxf(a.scale * 1.44269504088896340736f, -0x1p64f), 0x1p64f);
    d.Hq = a.Hq; d.G = a.Hq / c.H; d.window = a.window; d.sinks = a.sinks;
    d.chunk = plan.chunk; d.splits = plan.splits; d.min_units = tuned(Knob::ATT_CHUNK, 512) / 128;
    d.min_units = d.min_units < 1 ? 1 : d.min_units < 1 << 20 ? d.min_units : 1 << 20;
}
template <typename DEV>
static hipError_t attention_launch_any(const DEV& d, const AttnPlan& plan, int64_t max_rows, hipStream_t stream) {
    switch (d.c.bits[0] * 8 + d.c.bits[1]) {
        case 2 * 8 + 2: return attention_launch_bits<2, 2>(d, plan, max_rows, stream);
        case 2 * 8 + 3: return attention_launch_bits<2, 3>(d, plan, max_rows, stream);
        case 2 * 8 + 4: return attention_launch_bits<2, 4>(d, plan, max_rows, stream);
        case 3 * 8 + 2: return attention_launch_bits<3, 2>(d, plan, max_rows, stream);
        case 3 * 8 + 3: return attention_launch_bits<3, 3>(d, plan, max_rows, stream);
        case 3 * 8 + 4: return attention_launch_bits<3, 4>(d, plan, max_rows, stream);
        case 4 * 8 + 2: return attention_launch_bits<4, 2>(d, plan, max_rows, stream);
        case 4 * 8 + 3: return attention_launch_bits<4, 3>(d, plan, max_rows, stream);
        case 4 * 8 + 4: return attention_launch_bits<4, 4>(d, plan, max_rows, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace fq
