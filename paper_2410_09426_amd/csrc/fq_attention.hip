// Attention over the paged, quantized key/value cache (see flatquant.h for the layout): causal, with a sliding window and first tokens
// that stay visible, or for a tree of drafted tokens.
//
// The rows of a (sequence, key/value head) are its new tokens' query heads that share the head: row r is token r / G, query head r % G of
// the group.  A wave takes 16 NT of them and 32 tokens of the cache a step, on v_mfma_f32_16x16x32_f16:
//   S^T[token, row] = K Q^T      A: lane (i, g) has token i's channels 32 g .. 32 g + 31, a quarter of its codes in one load; Q lies in
//                                registers in the order in which those codes become fp16
//   O^T[channel, row] += V^T P^T A: lane (i, g) has channels 8 i .. 8 i + 7 of eight tokens, 4 g .. 4 g + 3 of each half of the 32:
//                                those whose weights the lane of S^T already holds, so the weights need no exchange
// Codes become fp16 without a conversion: a code's bits in the mantissa of 1024 (or of 1024 at bit s: 1024 + 2^s code), then one packed
// fma takes 1024 and the zero point off, exactly.  The keys' steps scale the scores, the values' steps the weights.
//
// Softmax in one pass: weights are 2^(score - M), M a reference per row that is raised only where a weight times its step would pass
// 2^15 (fp16's range) or a weight 2^40: most steps neither reduce a maximum nor touch the accumulators.  When it is raised it is put
// 2^7 above the largest product, so that products below 2^-14 of it, in fp16's subnormals, lose no more than 2^-32 of that product.
//
// The waves of a workgroup take every fourth step and meet in LDS at the end; where the rows are few the axis is split further over
// workgroups, whose partial results (M, sum, channels, in fp32) a second kernel joins.
#include "fq_internal.h"
#include "fq_device.h"

namespace fq {

constexpr int ATT_D = 128;
constexpr int ATT_WAVES = 4;
constexpr int ATT_NT = 64 * ATT_WAVES;
constexpr int ATT_STEP = 32;               // tokens per step of a wave
constexpr int ATT_PITCH = ATT_D + 4;       // floats per row of partial channels in LDS
constexpr float ATT_NONE = -1e30f;         // reference of a row that has seen nothing: below every finite score

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct AttnDev {
    CacheDev c;
    const _Float16* q;
    _Float16* out;
    const uint64_t* visible;
    float* part;              // [T * Hq, splits, 128] channels, then [T * Hq, splits] pairs of M and sum
    int64_t q_stride, out_stride;
    float scale2;             // scale * log2(e)
    int Hq, G, window, sinks, chunk, splits;
};

// ---- codes to fp16

__device__ __forceinline__ half2v as_half2(uint32_t x) { return __builtin_bit_cast(half2v, x); }
__device__ __forceinline__ uint32_t as_u32(half2v x) { return __builtin_bit_cast(uint32_t, x); }

// Two codes in bits [S, S + QB) of the halves of x, minus the zero points in `z` (packed fp16 whole numbers).
template <int QB, int S>
__device__ __forceinline__ half2v code_pair(uint32_t x, half2v z) {
    constexpr uint32_t mask = (((1u << QB) - 1u) << S) * 0x00010001u;
    const half2v raised = as_half2((x & mask) | 0x64006400u);                  // 1024 + 2^S code
    if constexpr (S == 0) return raised - (z + (half2v)(_Float16)1024.0f);
    constexpr _Float16 down = (_Float16)(1.0f / (float)(1 << S)), off = (_Float16)(-1024.0f / (float)(1 << S));
    return __builtin_elementwise_fma(raised, half2v{down, down}, half2v{off, off} - z);
}

// The 32 codes of a lane's quarter of a key, as 16 pairs; pair p is (first(p), second(p)) of the 32.
template <int QB>
struct KeyCodes;
template <>
struct KeyCodes<4> {
    typedef u32x4 words;
    static constexpr int first(int p) { return 8 * (p >> 2) + (p & 3); }
    static constexpr int second(int p) { return first(p) + 4; }
    static __device__ __forceinline__ void expand(const words& w, half2v z, half2v (&o)[16]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t hi = w[k] >> 8;
            o[4 * k] = code_pair<4, 0>(w[k], z);
            o[4 * k + 1] = code_pair<4, 4>(w[k], z);
            o[4 * k + 2] = code_pair<4, 0>(hi, z);
            o[4 * k + 3] = code_pair<4, 4>(hi, z);
        }
    }
};
template <>
struct KeyCodes<2> {
    typedef uint32_t words __attribute__((ext_vector_type(2)));
    static constexpr int first(int p) { return 16 * (p >> 3) + (p & 7); }
    static constexpr int second(int p) { return first(p) + 8; }
    static __device__ __forceinline__ void expand(const words& w, half2v z, half2v (&o)[16]) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t hi = w[k] >> 10;
            o[8 * k] = code_pair<2, 0>(w[k], z);
            o[8 * k + 1] = code_pair<2, 2>(w[k], z);
            o[8 * k + 2] = code_pair<2, 4>(w[k], z);
            o[8 * k + 3] = code_pair<2, 6>(w[k], z);
            o[8 * k + 4] = code_pair<2, 8>(w[k], z);
            o[8 * k + 5] = code_pair<2, 0>(hi, z);
            o[8 * k + 6] = code_pair<2, 2>(hi, z);
            o[8 * k + 7] = code_pair<2, 4>(hi, z);
        }
    }
};
// Sixteen codes are 48 bits, three halves X0, X1, X2: codes 5 and 10 straddle two of them.
__device__ __forceinline__ void expand48(uint32_t x0, uint32_t x1, uint32_t x2, half2v z, half2v (&o)[16]) {
    const uint32_t y0 = x0 >> 9, y1 = x1 >> 8, y2 = x2 >> 10;
    o[0] = code_pair<3, 0>(x0, z);
    o[1] = code_pair<3, 3>(x0, z);
    o[2] = code_pair<3, 6>(x0, z);
    o[3] = code_pair<3, 0>(y0, z);
    o[4] = code_pair<3, 3>(y0, z);
    o[5] = code_pair<3, 6>((y0 & 0x00400040u) | (x1 << 7 & 0x01800180u), z);
    o[6] = code_pair<3, 2>(x1, z);
    o[7] = code_pair<3, 5>(x1, z);
    o[8] = code_pair<3, 0>(y1, z);
    o[9] = code_pair<3, 3>(y1, z);
    o[10] = code_pair<3, 6>((y1 & 0x00C000C0u) | (x2 << 8 & 0x01000100u), z);
    o[11] = code_pair<3, 1>(x2, z);
    o[12] = code_pair<3, 4>(x2, z);
    o[13] = code_pair<3, 7>(x2, z);
    o[14] = code_pair<3, 0>(y2, z);
    o[15] = code_pair<3, 3>(y2, z);
}
template <>
struct KeyCodes<3> {
    typedef uint32_t words __attribute__((ext_vector_type(3)));
    static constexpr int first(int p) { return p; }
    static constexpr int second(int p) { return p + 16; }
    static __device__ __forceinline__ void expand(const words& w, half2v z, half2v (&o)[16]) {
        // bits 0 .. 47 in the low halves, 48 .. 95 in the high ones
        expand48(__builtin_amdgcn_perm(w[1], w[0], 0x07060100u), __builtin_amdgcn_perm(w[2], w[0], 0x05040302u),
                 __builtin_amdgcn_perm(w[2], w[1], 0x07060100u), z, o);
    }
};

// A lane's eight channels of two tokens (low half, high half): o[channel].
template <int QB>
__device__ __forceinline__ void value_pairs(uint32_t a, uint32_t b, half2v z, half2v (&o)[8]) {
    const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05040100u);
    if constexpr (QB == 4) {
        const uint32_t y = __builtin_amdgcn_perm(b, a, 0x07060302u), xh = x >> 8, yh = y >> 8;
        o[0] = code_pair<4, 0>(x, z);
        o[1] = code_pair<4, 4>(x, z);
        o[2] = code_pair<4, 0>(xh, z);
        o[3] = code_pair<4, 4>(xh, z);
        o[4] = code_pair<4, 0>(y, z);
        o[5] = code_pair<4, 4>(y, z);
        o[6] = code_pair<4, 0>(yh, z);
        o[7] = code_pair<4, 4>(yh, z);
    } else if constexpr (QB == 2) {
        const uint32_t xh = x >> 10;
        o[0] = code_pair<2, 0>(x, z);
        o[1] = code_pair<2, 2>(x, z);
        o[2] = code_pair<2, 4>(x, z);
        o[3] = code_pair<2, 6>(x, z);
        o[4] = code_pair<2, 8>(x, z);
        o[5] = code_pair<2, 0>(xh, z);
        o[6] = code_pair<2, 2>(xh, z);
        o[7] = code_pair<2, 4>(xh, z);
    } else {
        const uint32_t y = __builtin_amdgcn_perm(b, a, 0x07060302u), xh = x >> 9;
        o[0] = code_pair<3, 0>(x, z);
        o[1] = code_pair<3, 3>(x, z);
        o[2] = code_pair<3, 6>(x, z);
        o[3] = code_pair<3, 0>(xh, z);
        o[4] = code_pair<3, 3>(xh, z);
        o[5] = code_pair<3, 6>((xh & 0x00400040u) | (y << 7 & 0x01800180u), z);
        o[6] = code_pair<3, 2>(y, z);
        o[7] = code_pair<3, 5>(y, z);
    }
}

// ---- one step's tokens

template <int KB, int VB>
struct StepCodes {
    typename KeyCodes<KB>::words k[2];
    uint32_t kz[2];                        // parameters of the token that is the lane's row of A
    u32x4 ks[2];                           // parameters of the four tokens that are the lane's rows of S^T
    uint32_t v[8];
    u32x4 vs[2];
};
// Codes and parameters of tokens k0 .. k0 + 15 and k0 + 16 .. k0 + 31, in pages p[0] and p[1] (the caller has checked the numbers): whole
// pages are memory that may be read, whatever of them has been written.
template <int KB, int VB>
__device__ __forceinline__ void load_step(const CacheDev& c, int head, int k0, const int (&p)[2], int i, int g, StepCodes<KB, VB>& s) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t at = (((int64_t)p[t] * c.H + head) << c.page_shift) + ((k0 + 16 * t) & ((1 << c.page_shift) - 1));
        const uint8_t* kc = c.codes[0] + at * (16 * KB);
        const uint8_t* vc = c.codes[1] + at * (16 * VB);
        const uint32_t* kp = c.params[0] + at;
        const uint32_t* vp = c.params[1] + at;
        __builtin_memcpy(&s.k[t], __builtin_assume_aligned(kc + i * (16 * KB) + g * (4 * KB), 4), 4 * KB);
        s.kz[t] = kp[i];
        s.ks[t] = *reinterpret_cast<const u32x4*>(kp + 4 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint8_t* row = vc + (4 * g + r) * (16 * VB);
            if constexpr (VB == 4) {
                s.v[4 * t + r] = reinterpret_cast<const uint32_t*>(row)[i];
            } else if constexpr (VB == 2) {
                s.v[4 * t + r] = reinterpret_cast<const uint16_t*>(row)[i];
            } else {                       // three bytes at 3 i, as four that do not leave the row (shifted where they are used)
                uint32_t w;
                __builtin_memcpy(&w, row + (i < 15 ? 3 * i : 44), 4);
                s.v[4 * t + r] = w;
            }
        }
        s.vs[t] = *reinterpret_cast<const u32x4*>(vp + 4 * g);
    }
}

__device__ __forceinline__ float step_of(uint32_t params) { return (float)__builtin_bit_cast(_Float16, (uint16_t)params); }

template <typename T>
__device__ __forceinline__ T across_groups(T x, T (*op)(T, T)) {               // over the four lanes of a row of S^T's transpose
    x = op(x, __shfl_xor(x, 16));
    return op(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float fmax_op(float a, float b) { return __builtin_fmaxf(a, b); }
__device__ __forceinline__ float fadd_op(float a, float b) { return a + b; }

// The tokens that a tile of rows goes through: whole steps over the first tokens [0, 32 first_steps), then from `begin` (a multiple of 32) to `end`.
struct Span {
    int first_steps, begin, end, steps;
    __device__ __forceinline__ int token(int x) const { return x < first_steps ? ATT_STEP * x : begin + ATT_STEP * (x - first_steps); }
};
__device__ __forceinline__ Span span_of(const AttnDev& p, int length, int pos_lo, int pos_hi) {
    Span s;
    const int64_t held = (int64_t)p.c.table_width << p.c.page_shift;
    s.end = held < length ? (int)held : length;
    s.end = s.end < 0x7FFFFF00 ? s.end : 0x7FFFFF00;                           // a step behind it is still an int
    s.begin = s.first_steps = 0;
    if (!p.visible) {
        s.end = pos_hi < s.end ? pos_hi + 1 : s.end;
        if (p.window > 0) {
            const int64_t from = (int64_t)pos_lo - p.window + 1;
            s.begin = from > 0 ? (int)from & ~(ATT_STEP - 1) : 0;
            int firsts = p.sinks < s.begin ? p.sinks : s.begin;
            firsts = firsts < s.end ? firsts : s.end;
            s.first_steps = firsts > 0 ? (firsts + ATT_STEP - 1) / ATT_STEP : 0;
        }
    }
    s.steps = s.first_steps + (s.end > s.begin ? (s.end - s.begin + ATT_STEP - 1) / ATT_STEP : 0);
    return s;
}
__device__ __forceinline__ int splits_used(const AttnDev& p, int steps) {
    const int per = p.chunk / ATT_STEP, used = (steps + per - 1) / per;
    return used < 1 ? 1 : used < p.splits ? used : p.splits;
}
// Rows of a sequence, cut to the row tensors.
struct Sequence {
    int first, rows, length;
};
__device__ __forceinline__ Sequence sequence_of(const CacheDev& c, int b) {
    const int last = c.row_starts[b + 1], T = (int)c.T;
    Sequence s;
    s.first = c.row_starts[b] > 0 ? c.row_starts[b] : 0;
    s.rows = (last < T ? last : T) - s.first;
    s.length = c.lengths[b];
    return s;
}

// blockIdx: (sequence and head, tile of rows, split).
template <int KB, int VB, int NT>
__global__ __launch_bounds__(ATT_NT) void attention_kernel(AttnDev p) {
    __shared__ __attribute__((aligned(16))) float sums[ATT_WAVES][16][ATT_PITCH];
    __shared__ float refs[ATT_WAVES][16 * NT], totals[ATT_WAVES][16 * NT];
    const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / p.c.H, head = blockIdx.x - b * p.c.H;
    const Sequence seq = sequence_of(p.c, b);
    const int64_t all_rows = (int64_t)seq.rows * p.G;
    const int tiles = (int)((all_rows + 16 * NT - 1) / (16 * NT));
    const int32_t* table = p.c.page_table + b * p.c.table_stride;
    for (int tile_no = blockIdx.y; tile_no < tiles; tile_no += gridDim.y) {
        const int64_t row0 = (int64_t)(tiles - 1 - tile_no) * (16 * NT);      // the last rows, which see most, first
        const int64_t row_end = row0 + 16 * NT < all_rows ? row0 + 16 * NT : all_rows;
        const int before = seq.length - seq.rows;                              // position of row 0's token
        const int pos_lo = before + (int)(row0 / p.G), pos_hi = before + (int)((row_end - 1) / p.G);
        const Span span = span_of(p, seq.length, pos_lo, pos_hi);
        const int used = splits_used(p, span.steps);
        if ((int)blockIdx.z >= used) continue;
        const int per = p.chunk / ATT_STEP;
        const int x_end = (int)blockIdx.z == p.splits - 1 ? span.steps : min(span.steps, ((int)blockIdx.z + 1) * per);

        // rows: queries in the order of the codes, positions
        half8 q[NT][4];
        int pos[NT];
        uint64_t seen[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            int64_t r = row0 + 16 * n + i;
            r = r < row_end ? r : row_end - 1;
            const int token = (int)(r / p.G), sub = (int)(r - (int64_t)token * p.G);
            const _Float16* src = p.q + (seq.first + token) * p.q_stride + (head * p.G + sub) * ATT_D + 32 * g;
            half8 raw[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) raw[m] = *reinterpret_cast<const half8*>(src + 8 * m);
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int a = KeyCodes<KB>::first(4 * m + e), z = KeyCodes<KB>::second(4 * m + e);
                    q[n][m][2 * e] = raw[a >> 3][a & 7];
                    q[n][m][2 * e + 1] = raw[z >> 3][z & 7];
                }
            pos[n] = p.visible ? before - 1 : before + token;
            seen[n] = p.visible ? p.visible[seq.first + token] : 0;
        }

        f32x4 acc[NT][8];
        float ref[NT], total[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            ref[n] = ATT_NONE;
            total[n] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[n][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        auto pages_of = [&](int x, int (&pg)[2]) {
            x = x < span.steps ? x : span.steps - 1;
            const int k0 = span.token(x);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                int j = (k0 + 16 * t) >> p.c.page_shift;
                j = j < p.c.table_width ? j : p.c.table_width - 1;             // only tokens behind the end: masked
                pg[t] = table[j];
            }
        };
        auto load = [&](int x, const int (&pg)[2], StepCodes<KB, VB>& s) {
            x = x < span.steps ? x : span.steps - 1;
            const int ok[2] = {(unsigned)pg[0] < (unsigned)p.c.pages ? pg[0] : 0, (unsigned)pg[1] < (unsigned)p.c.pages ? pg[1] : 0};
            load_step<KB, VB>(p.c, head, span.token(x), ok, i, g, s);
        };
        auto work = [&](int x, const int (&pg)[2], const StepCodes<KB, VB>& s) {
            const int k0 = span.token(x);
            f32x4 sc[NT][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const half2v z = as_half2((s.kz[t] >> 16 & 15u) * 0x00010001u | 0x64006400u) - (half2v)(_Float16)1024.0f;
                half2v kk[16];
                KeyCodes<KB>::expand(s.k[t], z, kk);
#pragma unroll
                for (int n = 0; n < NT; ++n) sc[n][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const u32x4 a = {as_u32(kk[4 * m]), as_u32(kk[4 * m + 1]), as_u32(kk[4 * m + 2]), as_u32(kk[4 * m + 3])};
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        sc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), q[n][m], sc[n][t], 0, 0, 0);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[n][t][r] *= step_of(s.ks[t][r]) * p.scale2;
            const bool pages_ok = (unsigned)pg[0] < (unsigned)p.c.pages && (unsigned)pg[1] < (unsigned)p.c.pages;
            const int all_see = p.visible ? before - 1 : pos_lo;               // every row sees the tokens up to here, but for the window
            if (!(pages_ok && k0 + ATT_STEP - 1 <= all_see && k0 + ATT_STEP <= span.end && (p.window <= 0 || p.visible || k0 > pos_hi - p.window))) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bool page_ok = (unsigned)pg[t] < (unsigned)p.c.pages;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int k = k0 + 16 * t + 4 * g + r;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            bool ok = k <= pos[n];
                            if (p.visible) {
                                const int bit = k - before;
                                ok = ok || (bit >= 0 && bit < 64 && (seen[n] >> (bit & 63) & 1));
                            } else if (p.window > 0) {
                                ok = ok && ((int64_t)k > (int64_t)pos[n] - p.window || k < p.sinks);
                            }
                            sc[n][t][r] = ok && page_ok && k < span.end ? sc[n][t][r] : -__builtin_inff();
                        }
                    }
                }
            }
            float vs[8];
            half2v vz[4];
#pragma unroll
            for (int k = 0; k < 8; ++k) vs[k] = step_of(s.vs[k >> 2][k & 3]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                vz[k] = as_half2((__builtin_amdgcn_perm(s.vs[k >> 1][2 * (k & 1) + 1], s.vs[k >> 1][2 * (k & 1)], 0x07060302u) & 0x000F000Fu) | 0x64006400u) -
                        (half2v)(_Float16)1024.0f;
            half8 pw[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float e[8], prod[8];
                auto weigh = [&]() {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float x = sc[n][k >> 2][k & 3];
                        e[k] = __builtin_amdgcn_exp2f(x - ref[n]);
                        prod[k] = x == -__builtin_inff() ? 0.0f : e[k] * vs[k];   // what is not visible may have any step
                    }
                };
                weigh();
                float big = 0.0f, bigp = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    big = __builtin_fmaxf(big, e[k]);
                    bigp = __builtin_fmaxf(bigp, prod[k]);
                }
                if (__any(bigp > 32768.0f || big > 0x1p40f)) {
                    float top = ATT_NONE;
#pragma unroll
                    for (int k = 0; k < 8; ++k) top = __builtin_fmaxf(top, sc[n][k >> 2][k & 3] + __builtin_fmaxf(__builtin_amdgcn_logf(vs[k]), -25.0f));
                    top = across_groups(top, fmax_op) - 7.0f;
                    const float to = __builtin_fmaxf(ref[n], top), f = __builtin_amdgcn_exp2f(ref[n] - to);
                    ref[n] = to;
                    total[n] *= f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[n][j] *= f;
                    weigh();
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    total[n] += e[k];
                    pw[n][k] = (_Float16)prod[k];
                }
            }
            half2v vv[4][8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t a = s.v[2 * k], z = s.v[2 * k + 1];
                if constexpr (VB == 3) {
                    const int sh = i < 15 ? 0 : 8;
                    a >>= sh;
                    z >>= sh;
                }
                value_pairs<VB>(a, z, vz[k], vv[k]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const u32x4 a = {as_u32(vv[0][j]), as_u32(vv[1][j]), as_u32(vv[2][j]), as_u32(vv[3][j])};
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), pw[n], acc[n][j], 0, 0, 0);
            }
        };

        int x = (int)blockIdx.z * per + w;
        if (x < x_end) {
            StepCodes<KB, VB> cur, nxt;
            int pc[2], pn[2], pf[2];
            pages_of(x, pc);
            pages_of(x + ATT_WAVES, pn);
            load(x, pc, cur);
            while (x < x_end) {
                pages_of(x + 2 * ATT_WAVES, pf);
                load(x + ATT_WAVES, pn, nxt);
                work(x, pc, cur);
                cur = nxt;
                pc[0] = pn[0]; pc[1] = pn[1];
                pn[0] = pf[0]; pn[1] = pf[1];
                x += ATT_WAVES;
            }
        }

        // ---- the waves meet
        __syncthreads();                                                       // of an earlier tile's reads
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            total[n] = across_groups(total[n], fadd_op);
            if (g == 0) {
                refs[w][16 * n + i] = ref[n];
                totals[w][16 * n + i] = total[n];
            }
        }
        __syncthreads();
        for (int n = 0; n < NT; ++n) {
            float top = refs[0][16 * n + i];
#pragma unroll
            for (int k = 1; k < ATT_WAVES; ++k) top = __builtin_fmaxf(top, refs[k][16 * n + i]);
            const float f = __builtin_amdgcn_exp2f(ref[n] - top);
            if (n > 0) __syncthreads();
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    f32x4 o;
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = acc[n][4 * half + j][r] * f;
                    *reinterpret_cast<f32x4*>(&sums[w][i][8 * (4 * g + r) + 4 * half]) = o;
                }
            __syncthreads();
            const int rr = threadIdx.x >> 4, d = 8 * (threadIdx.x & 15);
            float ref_all = refs[0][16 * n + rr], sum = 0.0f, o[8] = {};
#pragma unroll
            for (int k = 1; k < ATT_WAVES; ++k) ref_all = __builtin_fmaxf(ref_all, refs[k][16 * n + rr]);
#pragma unroll
            for (int k = 0; k < ATT_WAVES; ++k) {
                sum += totals[k][16 * n + rr] * __builtin_amdgcn_exp2f(refs[k][16 * n + rr] - ref_all);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += sums[k][rr][d + e];
            }
            const int64_t r = row0 + 16 * n + rr;
            if (r < row_end) {
                const int64_t token = seq.first + r / p.G;
                const int hq = head * p.G + (int)(r % p.G);
                if (used == 1) {
                    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
                    half8 y;
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = (_Float16)(o[e] * inv);
                    *reinterpret_cast<half8*>(p.out + token * p.out_stride + hq * ATT_D + d) = y;
                } else {
                    const int64_t at = (token * p.Hq + hq) * p.splits + blockIdx.z;
                    float* dst = p.part + at * ATT_D + d;
                    *reinterpret_cast<f32x4*>(dst) = f32x4{o[0], o[1], o[2], o[3]};
                    *reinterpret_cast<f32x4*>(dst + 4) = f32x4{o[4], o[5], o[6], o[7]};
                    if (d == 0) {
                        float* pair = p.part + p.c.T * p.Hq * p.splits * ATT_D + 2 * at;
                        pair[0] = ref_all;
                        pair[1] = sum;
                    }
                }
            }
        }
    }
}

// Joins the splits of every (row, query head) that has more than one: one wave each, two channels a lane.
template <int ROWS>
__global__ __launch_bounds__(ATT_NT) void attention_join_kernel(AttnDev p) {
    const int l = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / p.c.H, head = blockIdx.x - b * p.c.H;
    const Sequence seq = sequence_of(p.c, b);
    const int64_t all_rows = (int64_t)seq.rows * p.G;
    const int tiles = (int)((all_rows + ROWS - 1) / ROWS);
    for (int tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
        const int64_t row0 = (int64_t)tile * ROWS, row_end = row0 + ROWS < all_rows ? row0 + ROWS : all_rows;
        const int before = seq.length - seq.rows;
        const Span span = span_of(p, seq.length, before + (int)(row0 / p.G), before + (int)((row_end - 1) / p.G));
        const int used = splits_used(p, span.steps);
        if (used == 1) continue;
        for (int64_t r = row0 + w + (int64_t)ATT_WAVES * blockIdx.z; r < row_end; r += ATT_WAVES * gridDim.z) {
            const int64_t token = seq.first + r / p.G;
            const int hq = head * p.G + (int)(r % p.G);
            const int64_t at = (token * p.Hq + hq) * p.splits;
            const float2* pair = reinterpret_cast<const float2*>(p.part + p.c.T * p.Hq * p.splits * ATT_D) + at;
            float top = ATT_NONE;
            for (int k = 0; k < used; ++k) top = __builtin_fmaxf(top, pair[k].x);
            float sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
            for (int k = 0; k < used; ++k) {
                const float2 e = pair[k], v = reinterpret_cast<const float2*>(p.part + (at + k) * ATT_D)[l];
                const float f = __builtin_amdgcn_exp2f(e.x - top);
                sum += e.y * f;
                o0 += v.x * f;
                o1 += v.y * f;
            }
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            reinterpret_cast<half2v*>(p.out + token * p.out_stride + hq * ATT_D)[l] = half2v{(_Float16)(o0 * inv), (_Float16)(o1 * inv)};
        }
    }
}

// Compute units of the card: the plan (and with it the workspace) follows from the host's figures alone.
constexpr int64_t kPlanCus = 256;

AttnPlan attention_plan(int64_t B, int64_t T, int H, int Hq, int64_t max_rows, int64_t max_length) {
    AttnPlan plan;
    max_rows = max_rows < T ? max_rows : T;                                    // positions and rows are 32-bit numbers
    max_length = max_length < 0x7fffffff ? max_length : 0x7fffffff;
    const int64_t rows = max_rows * (Hq / H);
    plan.col_tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const int64_t tiles = (rows + 16 * plan.col_tiles - 1) / (16 * plan.col_tiles), groups = B * H * (tiles > 0 ? tiles : 1);
    // workgroups for three per CU, of no less than 256 tokens each
    int64_t splits = (3 * kPlanCus + groups - 1) / groups;
    const int64_t most = (max_length + 255) / 256;
    splits = splits < most ? splits : most;
    splits = splits < 1 ? 1 : splits > 128 ? 128 : splits;
    const int64_t per = ((max_length + splits - 1) / splits + 127) / 128 * 128;
    plan.chunk = per < 128 ? 128 : per > (1 << 30) ? 1 << 30 : (int)per;
    splits = splits > 1 ? (max_length + plan.chunk - 1) / plan.chunk : 1;
    plan.splits = (int)(splits < 1 ? 1 : splits);
    plan.workspace = plan.splits > 1 ? T * Hq * plan.splits * (ATT_D + 2) * 4 : 0;
    return plan;
}

template <int KB, int VB, int NT>
static hipError_t attention_launch_as(const AttnDev& d, int64_t max_rows, hipStream_t stream) {
    const int64_t tiles = (max_rows * d.G + 16 * NT - 1) / (16 * NT);
    const dim3 grid((unsigned)(d.c.B * d.c.H), (unsigned)(tiles < 1 ? 1 : tiles > 65535 ? 65535 : tiles), (unsigned)d.splits);
    hipError_t e = launch(attention_kernel<KB, VB, NT>, grid, dim3(ATT_NT), 0, stream, d);
    if (e != hipSuccess || d.splits == 1) return e;
    return launch(attention_join_kernel<16 * NT>, dim3(grid.x, grid.y, NT), dim3(ATT_NT), 0, stream, d);
}

template <int KB, int VB>
static hipError_t attention_launch_bits(const AttnDev& d, const AttnPlan& plan, int64_t max_rows, hipStream_t stream) {
    switch (plan.col_tiles) {
        case 1: return attention_launch_as<KB, VB, 1>(d, max_rows, stream);
        case 2: return attention_launch_as<KB, VB, 2>(d, max_rows, stream);
        default: return attention_launch_as<KB, VB, 4>(d, max_rows, stream);
    }
}

hipError_t attention_launch(const CacheDev& c, const AttnArgs& a, const AttnPlan& plan, hipStream_t stream) {
    AttnDev d;
    d.c = c;
    d.q = a.q; d.out = a.out; d.visible = a.visible; d.part = a.workspace;
    d.q_stride = a.q_stride; d.out_stride = a.out_stride;
    d.scale2 = a.scale * 1.44269504088896340736f;
    d.Hq = a.Hq; d.G = a.Hq / c.H; d.window = a.window; d.sinks = a.sinks;
    d.chunk = plan.chunk; d.splits = plan.splits;
    switch (c.bits[0] * 8 + c.bits[1]) {
        case 2 * 8 + 2: return attention_launch_bits<2, 2>(d, plan, a.max_rows, stream);
        case 2 * 8 + 3: return attention_launch_bits<2, 3>(d, plan, a.max_rows, stream);
        case 2 * 8 + 4: return attention_launch_bits<2, 4>(d, plan, a.max_rows, stream);
        case 3 * 8 + 2: return attention_launch_bits<3, 2>(d, plan, a.max_rows, stream);
        case 3 * 8 + 3: return attention_launch_bits<3, 3>(d, plan, a.max_rows, stream);
        case 3 * 8 + 4: return attention_launch_bits<3, 4>(d, plan, a.max_rows, stream);
        case 4 * 8 + 2: return attention_launch_bits<4, 2>(d, plan, a.max_rows, stream);
        case 4 * 8 + 3: return attention_launch_bits<4, 3>(d, plan, a.max_rows, stream);
        case 4 * 8 + 4: return attention_launch_bits<4, 4>(d, plan, a.max_rows, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace fq
