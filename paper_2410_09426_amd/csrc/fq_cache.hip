// The paged key/value cache: rows quantized into their sequences' pages, and read back (see flatquant.h for the layout).
//
// Both are one pass over the data: 16 lanes hold a (row, head) group of 128 channels, 8 each (16 bytes of fp16; 4, 3 or 2 bytes of
// codes).  A wave takes 4 * N consecutive rows of one head, so that the rows of a head that follow each other in a page are written
// by the same wave into one piece.  The sequence of a row is found on the device (row_starts), its page in the table.
#include "fq_internal.h"
#include "fq_device.h"

// every rounding below is meant: products and sums are not to be contracted
#pragma clang fp contract(off)

namespace fq {

constexpr int CACHE_D = 128;
constexpr int CACHE_WAVES = 4;

// Page of row t's token and its slot there; NO_TOKEN if it has no place in the pages, NO_ROW if t is no row of the batch.
// The first guess is where the row would lie if all sequences had the same number of rows (a decode step: it is right); then bisection.
constexpr int64_t NO_TOKEN = -1, NO_ROW = -2;
__device__ __forceinline__ int64_t token_place(const CacheDev& c, int64_t t, int& slot) {
    slot = 0;
    if (t >= c.T) return NO_ROW;
    int lo = 0, hi = c.B - 1;                                   // the sequence is the last one that starts at t or before and has rows
    const int guess = (int)(t * c.B / c.T);
    if (c.row_starts[guess] <= t && t < c.row_starts[guess + 1]) {
        lo = guess;
    } else {
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (c.row_starts[mid] <= t) lo = mid;
            else hi = mid - 1;
        }
    }
    const int64_t first = c.row_starts[lo], last = c.row_starts[lo + 1];
    if (t < first || t >= last) return NO_ROW;                  // padding behind the last sequence
    const int64_t pos = c.lengths[lo] - (last < c.T ? last : c.T) + t;
    if (pos < 0) return NO_TOKEN;
    const int64_t j = pos >> c.page_shift;
    if (j >= c.table_width) return NO_TOKEN;
    const int page = c.page_table[lo * c.table_stride + j];
    if (page < 0 || page >= c.pages) return NO_TOKEN;
    slot = (int)(pos & ((1 << c.page_shift) - 1));
    return page;
}

template <typename Op>
__device__ __forceinline__ float row16_reduce(float x, Op op) {
    x = op(x, dpp_move<0xB1>(x));    // quad_perm [1,0,3,2]
    x = op(x, dpp_move<0x4E>(x));    // quad_perm [2,3,0,1]
    x = op(x, dpp_move<0x141>(x));   // row_half_mirror
    return op(x, dpp_move<0x140>(x));   // row_mirror
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
    float mx = 0.0f, mn = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        mx = __builtin_fmaxf(mx, (float)y[k]);
        mn = __builtin_fminf(mn, (float)y[k]);
    }
    mx = row16_reduce(mx, [](float a, float b) { return __builtin_fmaxf(a, b); });
    mn = row16_reduce(mn, [](float a, float b) { return __builtin_fminf(a, b); });
    mx *= clip;
    mn *= clip;
    // rounded to fp32 and then to fp16, as two conversions: the compiler would make one v_fma_mixlo_f16 of the last fma and the conversion, which
    // rounds once and puts one group in 2000 of the 3-bit grid on the other side of an fp16 midpoint
    float wide = quotient(mx - mn, LV, 1.0f / LV);
    asm("" : "+v"(wide));
    const _Float16 step = (_Float16)wide;
    const bool usable = (float)step > 0.0f && (float)step <= 65504.0f;   // a step that overflows has zero codes, like one of zero
    const float s = usable ? (float)step : 1.0f;
    // the reciprocal of an 11-bit number is never within 2^-35 of a tie, so one step from v_rcp_f32's last bit rounds it correctly
    const float r = __builtin_amdgcn_rcpf(s);
    const float inv = usable ? __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r) : 0.0f;
    const float z = __builtin_amdgcn_fmed3f(__builtin_rintf(quotient(-mn, s, inv)), 0.0f, LV);
    uint32_t codes = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        // y / s is a tie exactly or at least 2^-12 away from one: the rounded quotient falls on the same side
        const float q = __builtin_amdgcn_fmed3f(__builtin_rintf(quotient((float)y[k], s, inv)) + z, 0.0f, LV);
        codes |= (uint32_t)q << (QB * k);
    }
    params = (uint32_t)__builtin_bit_cast(uint16_t, step) | (uint32_t)z << 16;
    return codes;
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

// One wave: 4 N consecutive rows of one head of the keys (X = 0) or values (1).
template <int QB, int N>
__device__ __forceinline__ void write_rows(const CacheDev& c, const _Float16* rows, int64_t stride, float clip, uint8_t* codes, uint32_t* params,
                                           int64_t t0, int head) {
    const int l = threadIdx.x & 63, i = l & 15;
    half8 y[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        int64_t t = t0 + 4 * k + (l >> 4);
        t = t < c.T ? t : c.T - 1;
        y[k] = *reinterpret_cast<const half8*>(rows + t * stride + head * CACHE_D + 8 * i);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        int slot;
        const int64_t page = token_place(c, t0 + 4 * k + (l >> 4), slot);
        uint32_t word;
        const uint32_t q = quantize8<QB>(y[k], clip, word);
        const int64_t at = ((page * c.H + head) << c.page_shift) + slot;
        if (page >= 0) {
            store_codes<QB>(codes + at * (16 * QB), i, q);
            if (i == 0) params[at] = word;
        }
    }
}

template <int QB, int N>
__device__ __forceinline__ void read_rows(const CacheDev& c, _Float16* rows, int64_t stride, const uint8_t* codes, const uint32_t* params,
                                          int64_t t0, int head) {
    const int l = threadIdx.x & 63, i = l & 15;
    constexpr uint32_t MASK = (1u << QB) - 1u;
    uint32_t word[N], par[N];
    bool row[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        int slot;
        const int64_t page = token_place(c, t0 + 4 * k + (l >> 4), slot);
        row[k] = page != NO_ROW;
        const int64_t at = ((page * c.H + head) << c.page_shift) + slot;
        word[k] = par[k] = 0;
        if (page >= 0) {
            word[k] = load_codes<QB>(codes + at * (16 * QB), i);
            par[k] = params[at];
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t q = loaded_codes<QB>(word[k], i);
        const float s = (float)__builtin_bit_cast(_Float16, (uint16_t)par[k]);
        const int z = (int)(par[k] >> 16);
        half8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (_Float16)(s * (float)((int)(q >> (QB * e) & MASK) - z));
        if (row[k]) *reinterpret_cast<half8*>(rows + (t0 + 4 * k + (l >> 4)) * stride + head * CACHE_D + 8 * i) = y;
    }
}

// blockIdx.y: head; blockIdx.z: keys or values.
template <int N, bool WRITE>
__global__ __launch_bounds__(64 * CACHE_WAVES) void cache_rows_kernel(CacheDev c, CacheRows r) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t0 = ((int64_t)blockIdx.x * CACHE_WAVES + w) * (4 * N);
    const int x = blockIdx.z, head = blockIdx.y;
    _Float16* rows = static_cast<_Float16*>(r.rows[x]);
    if (!rows || t0 >= c.T) return;
    auto go = [&](auto bits) {
        constexpr int QB = decltype(bits)::value;
        if constexpr (WRITE) write_rows<QB, N>(c, rows, r.stride[x], r.clip[x], c.codes[x], c.params[x], t0, head);
        else read_rows<QB, N>(c, rows, r.stride[x], c.codes[x], c.params[x], t0, head);
    };
    switch (c.bits[x]) {
        case 2: go(std::integral_constant<int, 2>{}); break;
        case 3: go(std::integral_constant<int, 3>{}); break;
        default: go(std::integral_constant<int, 4>{}); break;
    }
}

template <bool WRITE>
static hipError_t rows_launch(const CacheDev& c, const CacheRows& r, hipStream_t stream) {
    auto grid = [&](int n) { return dim3((unsigned)((c.T + 4 * n * CACHE_WAVES - 1) / (4 * n * CACHE_WAVES)), (unsigned)c.H, 2); };
    if (c.T * c.H <= 4096) return launch(cache_rows_kernel<1, WRITE>, grid(1), dim3(64 * CACHE_WAVES), 0, stream, c, r);
    return launch(cache_rows_kernel<4, WRITE>, grid(4), dim3(64 * CACHE_WAVES), 0, stream, c, r);
}

hipError_t cache_write_launch(const CacheDev& c, const CacheRows& r, hipStream_t stream) { return rows_launch<true>(c, r, stream); }
hipError_t cache_read_launch(const CacheDev& c, const CacheRows& r, hipStream_t stream) { return rows_launch<false>(c, r, stream); }

}  // namespace fq
