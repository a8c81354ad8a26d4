// The paged key/value cache: rows quantized into their sequences' pages, and read back (see flatquant.h for the layout).
//
// Both are one pass over the data: 16 lanes hold a (row, head) group of 128 channels, 8 each (16 bytes of fp16; 4, 3 or 2 bytes of
// codes).  A wave takes 4 N consecutive rows of one head, so that the rows of a head that follow each other in a page are written
// by the same wave into one piece; its lanes find the places of a row each, once, and hand them on.  Neighbouring waves and workgroups
// take the other heads of the same rows.
//
// Bound by memory: 16384 rows of 32 heads (268 MB of fp16, 62 MB of codes) are written in 78 us and read back in 73 to 78, 4.2 to 4.5 TB/s (a copy
// of 1 GB 4.73), several sets of rows and pages in turn; writing issues 75 vector instructions for the eight values of a lane, which is most of what it lacks (150 took 107 us).  Rows of
// few tokens (a decode step) are a launch and four loads one after the other: 3.6 us.
#include "fq_internal.h"
#include "fq_device.h"
#include "fq_cache_device.h"

// every rounding below is meant: products and sums are not to be contracted
#pragma clang fp contract(off)

namespace fq {

constexpr int CACHE_D = 128;
constexpr int CACHE_WAVES = 4;

// Largest of the 16 lanes' values, by halves.
__device__ __forceinline__ half2v row16_max(half2v x) {
    auto other = [&](auto ctrl) { return as_half2((uint32_t)__builtin_amdgcn_mov_dpp((int)as_u32(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    x = __builtin_elementwise_max(x, other(std::integral_constant<int, 0xB1>{}));     // quad_perm [1,0,3,2]
    x = __builtin_elementwise_max(x, other(std::integral_constant<int, 0x4E>{}));     // quad_perm [2,3,0,1]
    x = __builtin_elementwise_max(x, other(std::integral_constant<int, 0x141>{}));    // row_half_mirror
    return __builtin_elementwise_max(x, other(std::integral_constant<int, 0x140>{})); // row_mirror
}

// a / b rounded once, for b whose reciprocal `inv` is correctly rounded and a quotient in the normal range
__device__ __forceinline__ float quotient(float a, float b, float inv) {
    const float q = a * inv;
    return __builtin_fmaf(__builtin_fmaf(-b, q, a), inv, q);
}

// The 8 codes of a lane, at bits [QB k, QB k + QB), and the group's step and zero point as one word.
template <int QB>
__device__ __forceinline__ uint32_t quantize8(const half8& y, float clip, uint32_t& params) {
    constexpr float LV = (float)((1 << QB) - 1);
    // the range, (largest, largest of the negated), in fp16: comparisons round nothing
    half2v up = half2v{0, 0}, down = half2v{0, 0};
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const half2v v = half2v{y[k], y[k + 1]};
        up = __builtin_elementwise_max(up, v);
        down = __builtin_elementwise_max(down, -v);
    }
    const half2v range = row16_max(__builtin_elementwise_max(half2v{up[0], down[0]}, half2v{up[1], down[1]}));
    const float mx = (float)range[0] * clip, below = (float)range[1] * clip;
    // rounded to fp32 and then to fp16, as two conversions: the compiler would make one v_fma_mixlo_f16 of the last fma and the conversion, which
    // rounds once and puts one group in 2000 of the 3-bit grid on the other side of an fp16 midpoint
    const float width = mx + below;
    float wide = width <= 3.4028234e38f ? quotient(width, LV, 1.0f / LV) : width;      // (of an infinity the remainder is no number)
    asm("" : "+v"(wide));
    const _Float16 step = (_Float16)wide;
    const bool usable = (float)step > 0.0f && (float)step <= 65504.0f;   // a step that overflows has zero codes, like one of zero
    const float s = usable ? (float)step : 1.0f;
    // the reciprocal of an 11-bit number is never within 2^-35 of a tie, so one step from v_rcp_f32's last bit rounds it correctly
    const float r = __builtin_amdgcn_rcpf(s);
    const float inv = usable ? __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r) : 0.0f;
    const float z = __builtin_amdgcn_fmed3f(__builtin_rintf(quotient(below, s, inv)), 0.0f, LV);
    // round_half_even(y / s), clamped to -z .. LV - z.  y / s is a tie exactly or, both being 11-bit numbers, at least 2^-12 away from one.  One fma against
    // 1.5 * 2^10 rounds y inv, within 2^-19 of y / s where the clamp leaves it, to a multiple of 2^-13: onto the tie in the first case, and not over it in the second.
    // The clamp's ends are multiples too.  1.5 * 2^23 in its place rounds that to the integer, two's complement in the low bits; shift-adds chain eight of
    // them, and one addition takes the constants off and puts the zero points on, modulo 2^32 (as each is 0 .. LV then, the fields hold the codes).
    constexpr float FINE = 1536.0f, WHOLE = 12582912.0f;
    constexpr uint32_t FIELDS = 1u + (1u << QB) + (1u << 2 * QB) + (1u << 3 * QB) + (1u << 4 * QB) + (1u << 5 * QB) + (1u << 6 * QB) + (1u << 7 * QB);
    const float lo = FINE - z, hi = FINE + (LV - z);
    uint32_t codes = 0;
#pragma unroll
    for (int k = 7; k >= 0; --k) {
        const float q = __builtin_amdgcn_fmed3f(__builtin_fmaf((float)y[k], inv, FINE), lo, hi) + (WHOLE - FINE);
        codes = (codes << QB) + __builtin_bit_cast(uint32_t, q);
    }
    codes += (uint32_t)z * FIELDS - 0x4B400000u * FIELDS;
    params = (uint32_t)__builtin_bit_cast(uint16_t, step) | (uint32_t)z << 16;
    return codes;
}

// The 8 values of a lane.  step (code - zero point) has 16 bits at most: one rounding to fp16, which the packed product is.
template <int QB>
__device__ __forceinline__ half8 values8(uint32_t codes, uint32_t params) {
    constexpr uint32_t MASK = (1u << QB) - 1u;
    const half2v step = as_half2(params << 16 | (params & 0xFFFFu)), zero = as_half2((params >> 16) * 0x00010001u + 0x64006400u);   // 1024 + z
    half8 y;
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const int up = 16 - QB * (k + 1);                                      // of the second code, to bits 16 ..
        const uint32_t low = (codes >> (QB * k) & MASK) | 0x64006400u, both = ((up >= 0 ? codes << (up & 31) : codes >> (-up & 31)) & MASK << 16) | low;
        const half2v v = (as_half2(both) - zero) * step;
        y[k] = v[0];
        y[k + 1] = v[1];
    }
    return y;
}

__device__ __forceinline__ uint32_t from_next_lane(uint32_t x) {   // of the quad; the last lane keeps its own
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xF9, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t from_previous_lane(uint32_t x) {   // of the quad; the first lane keeps its own
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x90, 0xF, 0xF, true);
}

// Codes of lane i of 16 to or from the 16 QB bytes of a row.  3 bits: four lanes' 24 bits are three dwords.
template <int QB>
__device__ __forceinline__ void store_codes(uint8_t* row, int i, uint32_t codes) {
    if constexpr (QB == 4) {
        reinterpret_cast<uint32_t*>(row)[i] = codes;
    } else if constexpr (QB == 2) {
        reinterpret_cast<uint16_t*>(row)[i] = (uint16_t)codes;
    } else {
        const int k = i & 3;
        const uint32_t word = codes >> (8 * k) | from_next_lane(codes) << (24 - 8 * k);
        if (k < 3) reinterpret_cast<uint32_t*>(row)[3 * (i >> 2) + k] = word;
    }
}
template <int QB>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* row, int i) {
    if constexpr (QB == 4) return reinterpret_cast<const uint32_t*>(row)[i];
    if constexpr (QB == 2) return reinterpret_cast<const uint16_t*>(row)[i];
    const int k = i & 3;
    return reinterpret_cast<const uint32_t*>(row)[3 * (i >> 2) + (k < 3 ? k : 2)];
}
template <int QB>
__device__ __forceinline__ uint32_t loaded_codes(uint32_t word, int i) {
    if constexpr (QB != 3) return word;
    const int k = i & 3;
    return __builtin_amdgcn_alignbit(word, from_previous_lane(word), (32 - 8 * k) & 31);
}

// Rows t0 .. t0 + 4 N - 1 of the keys (X = 0) or values (1) of one head, by one wave, four loads of each lane ahead of their use.
template <int QB, int N, bool WRITE>
__device__ __forceinline__ void move_rows(const CacheDev& c, _Float16* rows, int64_t stride, float clip, uint8_t* codes, uint32_t* params,
                                          int64_t t0, int head) {
    constexpr int AHEAD = N < 4 ? N : 4;
    const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
    rows += head * CACHE_D + 8 * i;
    half8 y[AHEAD];
    auto load = [&](int k0) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int64_t t = t0 + 4 * (k0 + k) + g;
            y[k] = *reinterpret_cast<const half8*>(rows + (t < c.T ? t : c.T - 1) * stride);
        }
    };
    if constexpr (WRITE) load(0);
    const int64_t mine = l < 4 * N ? token_place(c, t0 + l, head) : NO_ROW;
    for (int k0 = 0; k0 < N && t0 + 4 * k0 < c.T; k0 += AHEAD) {
        int64_t at[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) at[k] = __shfl((long long)mine, 4 * (k0 + k) + g);
        if constexpr (WRITE) {
            if (k0 > 0) load(k0);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                uint32_t word;
                const uint32_t q = quantize8<QB>(y[k], clip, word);
                if (at[k] >= 0) {
                    store_codes<QB>(codes + at[k] * (16 * QB), i, q);
                    if (i == 0) params[at[k]] = word;
                }
            }
        } else {
            uint32_t word[AHEAD], par[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                word[k] = par[k] = 0;
                if (at[k] >= 0) {
                    word[k] = load_codes<QB>(codes + at[k] * (16 * QB), i);
                    par[k] = params[at[k]];
                }
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const half8 v = values8<QB>(loaded_codes<QB>(word[k], i), par[k]);
                if (at[k] != NO_ROW) *reinterpret_cast<half8*>(rows + (t0 + 4 * (k0 + k) + g) * stride) = v;
            }
        }
    }
}

// blockIdx.x: 2^head_shift heads of the keys, then of the values (of what the call has of them), so that what runs at the same time covers whole rows; the
// waves beyond those take more rows.
template <int N, bool WRITE>
__global__ __launch_bounds__(64 * CACHE_WAVES) void cache_rows_kernel(CacheDev c, CacheRows r, int head_shift) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int groups = (c.H + (1 << head_shift) - 1) >> head_shift, second = (int)blockIdx.x >= groups;
    const int x = r.rows[0] ? second : 1, head = (((int)blockIdx.x - (second ? groups : 0)) << head_shift) + (w & ((1 << head_shift) - 1));
    if (head >= c.H) return;
    _Float16* rows = static_cast<_Float16*>(r.rows[x]);
    const int64_t step = (int64_t)(4 * N) * (CACHE_WAVES >> head_shift);
    for (int64_t t0 = blockIdx.y * step + 4 * N * (w >> head_shift); t0 < c.T; t0 += gridDim.y * step) {
        switch (c.bits[x]) {
            case 2: move_rows<2, N, WRITE>(c, rows, r.stride[x], r.clip[x], c.codes[x], c.params[x], t0, head); break;
            case 3: move_rows<3, N, WRITE>(c, rows, r.stride[x], r.clip[x], c.codes[x], c.params[x], t0, head); break;
            default: move_rows<4, N, WRITE>(c, rows, r.stride[x], r.clip[x], c.codes[x], c.params[x], t0, head); break;
        }
    }
}

template <int N, bool WRITE>
static hipError_t rows_launch(const CacheDev& c, const CacheRows& r, hipStream_t stream) {
    const int head_shift = c.H >= 4 ? 2 : c.H >= 2 ? 1 : 0;
    const int64_t step = (int64_t)(4 * N) * (CACHE_WAVES >> head_shift), blocks = (c.T + step - 1) / step;
    const unsigned halves = (r.rows[0] ? 1u : 0u) + (r.rows[1] ? 1u : 0u);
    const dim3 grid(halves * (unsigned)((c.H + (1 << head_shift) - 1) >> head_shift), (unsigned)(blocks < 65535 ? blocks : 65535));
    return launch(cache_rows_kernel<N, WRITE>, grid, dim3(64 * CACHE_WAVES), 0, stream, c, r, head_shift);
}
template <bool WRITE>
static hipError_t rows_launch(const CacheDev& c, const CacheRows& r, hipStream_t stream) {
    // 4 or 16 rows a wave?  4096 groups (rows x heads) of keys and values written in 3.5 / 4.5 us and read back in 3.6 / 3.9, 8192 in 4.4 / 4.6 and 4.2 / 4.2, 16384 in
    // 5.6 / 5.3 and 5.7 / 4.9.  16 or 64?  Keys and values of 2048 x 8 rows and heads written in 6.6 / 10.3 us, of 4096 x 32 in 24.3 / 24.7, of 32768 x 8 in 43.6 / 37.5, of 32768 x 32
    // in 145 / 142; read back in 5.3 / 8.2, 16.7 / 20.6, 28.2 / 31.3, 147 / 152.
    if (c.T * c.H <= 4096) return rows_launch<1, WRITE>(c, r, stream);
    if constexpr (WRITE) {
        if (c.T * c.H > 1 << 17) return rows_launch<16, WRITE>(c, r, stream);
    }
    return rows_launch<4, WRITE>(c, r, stream);
}

hipError_t cache_write_launch(const CacheDev& c, const CacheRows& r, hipStream_t stream) {
    CacheRows plain = r;
    for (int x = 0; x < 2; ++x) {
        if (!r.rows[x] || !r.P[x]) continue;
        const hipError_t e = kv_paged_launch(c, r, x, stream);
        if (e != hipSuccess) return e;
        plain.rows[x] = nullptr;
    }
    if (!plain.rows[0] && !plain.rows[1]) return hipSuccess;
    return rows_launch<true>(c, plain, stream);
}
hipError_t cache_read_launch(const CacheDev& c, const CacheRows& r, hipStream_t stream) { return rows_launch<false>(c, r, stream); }

}  // namespace fq
