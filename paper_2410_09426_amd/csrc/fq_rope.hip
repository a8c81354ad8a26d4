// Queries and keys between their product and the cache, head by head: norm over the 128 channels, rotation by the row's position, and for a
// transformed key cache the matrix of the head (see flatquant.h).
//
//     y = x w / sqrt(mean x^2 + eps),   (a, b) -> (a cos - b sin, b cos + a sin) of every rotated pair,   out = fp16(y) or fp16(fp16(y) P).
//
// The angle of pair i at position p is p f_i, f_i in units of 2^-64 of a turn: the product modulo 2^64 is exact at every position, and what is left of it in
// 32 bits, a whole number of quarter turns taken off, is below an eighth of a turn, where few terms of the series give both functions to 2^-24.
//
// Without a matrix: 16 lanes a (row, head) group, eight channels each; a wave takes four rows and some of the heads, so that the angles are worked out
// once for all of them, four pairs a lane (the lane that holds the pairs' other numbers has the other four), and the weights go into the cosines and sines.  Bound by memory:
// 16384 rows of 40 heads (336 MB) in 60 us; 64 rows in 3.4, a launch and two loads one after the other.  Stores past the caches: 4096 rows of 40 heads 22.5 -> 16.9 us.
// With one: 32 groups a wave as the columns of v_mfma_f32_32x32x16_f16, as they come from memory: a lane holds 8 channels of every 16 of its group, both of
// every pair, so that it turns them in its registers before they are the right operand.  8192 rows of 32 + 8 heads (168 MB, 8.6 GFLOP) through one matrix in 39 us, 33 of
// them memory at a copy's rate; through one each 77, as every group's angles are worked out for it alone, 32 a lane, which takes more than the products.
#include "fq_internal.h"
#include "fq_device.h"
#include "fq_cache_device.h"

namespace fq {

constexpr int RP_D = 128;
constexpr int RP_WAVES = 4;
constexpr int RP_NT = 64 * RP_WAVES;

// Bits 32 .. 63 of position * turns: the angle in units of 2^-32 of a turn.
__device__ __forceinline__ uint32_t angle_of(uint32_t position, uint64_t turns) {
    return __umulhi(position, (uint32_t)turns) + position * (uint32_t)(turns >> 32);
}
__device__ __forceinline__ void cos_sin(uint32_t angle, float& c, float& s) {
    const uint32_t quarter = angle + 0x20000000u;                              // its top two bits: quarter turns, to the nearest
    const float x = (float)(int32_t)(angle - (quarter & 0xC0000000u)) * 0x1.921fb6p-30f;       // pi / 2^31: within pi / 4 of zero
    const float x2 = x * x;
    // the next terms are below 2^-29 and 2^-25
    const float sine = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(1.0f / 362880, x2, -1.0f / 5040), x2, 1.0f / 120), x2, -1.0f / 6) * x2, x, x);
    const float cosine = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(1.0f / 40320, x2, -1.0f / 720), x2, 1.0f / 24), x2, -0.5f), x2, 1.0f);
    const bool odd = quarter & 0x40000000u;
    const uint32_t cb = __builtin_bit_cast(uint32_t, odd ? sine : cosine), sb = __builtin_bit_cast(uint32_t, odd ? cosine : sine);
    c = __builtin_bit_cast(float, cb ^ ((quarter ^ quarter << 1) & 0x80000000u));              // negative in the second and third quarter
    s = __builtin_bit_cast(float, sb ^ (quarter & 0x80000000u));
}
__device__ __forceinline__ float dot8(const half8& x, float sum) {
    const u32x4 v = __builtin_bit_cast(u32x4, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) sum = __builtin_amdgcn_fdot2(as_half2(v[k]), as_half2(v[k]), sum, false);
    return sum;
}
__device__ __forceinline__ float row16_sum(float x) {
    x += dpp_move<0xB1>(x);
    x += dpp_move<0x4E>(x);
    x += dpp_move<0x141>(x);
    return x + dpp_move<0x140>(x);
}

// ---- without a matrix

// Rows 4 block .. + 3 of heads `first` .. + per - 1, queries first, by one wave.
template <int AHEAD>
__device__ __forceinline__ void turn_rows(const RopeDev& d, int64_t block, int first, int per) {
    const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
    const int64_t row = 4 * block + g, t = row < d.T ? row : d.T - 1;
    const int all = d.heads[0] + d.heads[1], last = min(first + per, all);
    if (first >= last) return;
    const int position = d.positions[t];
    const bool live = row < d.T && position >= 0;

    auto load = [&](int x, half8 (&y)[AHEAD]) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int at = min(x + k, last - 1), role = at >= d.heads[0];
            y[k] = *reinterpret_cast<const half8*>(d.rows[role] + t * d.stride[role] + (at - (role ? d.heads[0] : 0)) * RP_D + 8 * i);
        }
    };
    half8 next[AHEAD];
    load(first, next);
    __builtin_amdgcn_sched_barrier(0);

    // cosines, and sines with the sign that the pair's other number has in this one
    const int half = d.rotary >> 1, ch = 8 * i;
    const bool turned = ch < d.rotary, second = ch >= half;
    // the lane that has the other numbers (of those that are not turned: itself)
    const int other = 4 * (!d.interleaved && turned ? l + (second ? -(half >> 3) : half >> 3) : l);
    const bool across = !d.interleaved && d.rotary == 2 * 64;
    auto exchange = [&](uint32_t x) {
        return (uint32_t)(across ? __builtin_amdgcn_mov_dpp((int)x, 0x128, 0xF, 0xF, true) : __builtin_amdgcn_ds_bpermute(other, (int)x));     // row_ror:8
    };
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        cs[e] = 1.0f;
        sn[e] = 0.0f;
    }
    if (d.rotary > 0) {
        // four pairs a lane: all that its neighbours have, or half of those that it shares with the other lane
        const uint32_t p = position < 0 ? 0u : (uint32_t)position;
        const int pair = !turned ? 0 : d.interleaved ? 4 * i : second ? ch - half + 4 : ch;
        float c[4], s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) cos_sin(angle_of(p, d.turns[pair + e]), c[e], s[e]);
        if (d.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                cs[2 * e] = cs[2 * e + 1] = turned ? c[e] : 1.0f;
                sn[2 * e] = turned ? -s[e] : 0.0f;
                sn[2 * e + 1] = turned ? s[e] : 0.0f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float co = __builtin_bit_cast(float, exchange(__builtin_bit_cast(uint32_t, c[e]))), so = __builtin_bit_cast(float, exchange(__builtin_bit_cast(uint32_t, s[e])));
                cs[e] = !turned ? 1.0f : second ? co : c[e];
                cs[4 + e] = !turned ? 1.0f : second ? c[e] : co;
                sn[e] = !turned ? 0.0f : second ? so : -s[e];
                sn[4 + e] = !turned ? 0.0f : second ? s[e] : -so;
            }
        }
    }

    int role = -1;
    float cw[8], sw[8];
    for (int x = first; x < last; x += AHEAD) {
        half8 y[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) y[k] = next[k];
        if (x + AHEAD < last) load(x + AHEAD, next);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int at = x + k;
            if (at >= last) break;
            const int is = at >= d.heads[0];
            if (is != role) {                                                  // the weights of queries or keys
                role = is;
                const _Float16* weights = d.w[role];
                half8 mine, others;
#pragma unroll
                for (int e = 0; e < 8; ++e) mine[e] = others[e] = (_Float16)1.0f;
                if (weights) {
                    mine = *reinterpret_cast<const half8*>(weights + ch);
                    others = *reinterpret_cast<const half8*>(weights + (!d.interleaved && turned ? (second ? ch - half : ch + half) : ch));
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    cw[e] = cs[e] * (float)mine[e];
                    sw[e] = sn[e] * (float)(d.interleaved ? others[e ^ 1] : others[e]);
                }
            }
            const u32x4 v = __builtin_bit_cast(u32x4, y[k]);
            u32x4 o;
            if (d.interleaved) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __builtin_amdgcn_alignbit(v[e], v[e], 16);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = exchange(v[e]);
            }
            if (d.rotary < RP_D)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = turned ? o[e] : 0u;         // (a sine of zero times an infinity is no number)
            const half8 z = __builtin_bit_cast(half8, o);
            half8 r;
            if (d.w[role]) {
                const float by = __builtin_amdgcn_rsqf(__builtin_fmaf(row16_sum(dot8(y[k], 0.0f)), 1.0f / RP_D, d.eps));
#pragma unroll
                for (int e = 0; e < 8; ++e) r[e] = (_Float16)(__builtin_fmaf((float)y[k][e], cw[e], (float)z[e] * sw[e]) * by);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) r[e] = (_Float16)__builtin_fmaf((float)y[k][e], cw[e], (float)z[e] * sw[e]);
            }
            if (live) __builtin_nontemporal_store(r, reinterpret_cast<half8*>(d.out[role] + row * d.out_stride[role] + (at - (role ? d.heads[0] : 0)) * RP_D + ch));
        }
    }
}

// blockIdx: (four rows, heads); a wave has `per` heads.
template <int AHEAD>
__global__ __launch_bounds__(RP_NT) void rope_kernel(RopeDev d, int per) {
    const int first = ((int)blockIdx.y * RP_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * per;
    for (int64_t block = blockIdx.x; 4 * block < d.T; block += gridDim.x) turn_rows<AHEAD>(d, block, first, per);
}

// ---- with a matrix

constexpr int RM_GROUPS = 32;              // (row, head) groups of a wave
constexpr int RM_MT = RP_D / 32, RM_KB = RP_D / 16;
constexpr int RM_FRAG_BYTES = RM_MT * RM_KB * 64 * 16;
constexpr int RM_FLAT_BYTES = RP_D * (RP_D + 8) * 2;
constexpr int RM_OUT_PITCH = 2 * RP_D + 16;
constexpr int RM_STAGE_BYTES = RP_WAVES * RM_GROUPS * RM_OUT_PITCH;
constexpr int RM_LOOP_AT = RM_FRAG_BYTES, RM_TABLE_AT = RM_LOOP_AT + (RM_FLAT_BYTES > RM_STAGE_BYTES ? RM_FLAT_BYTES : RM_STAGE_BYTES);
constexpr int RM_ANGLES_AT = RM_TABLE_AT + 64 * 8 + RP_D * 4;

// Weights, and what the lanes need of the angles, in LDS: either the turns, and a lane works its 32 angles out, or cosines and sines of all the rows that the
// groups have, which are few where the heads follow each other: 32 groups of 32 heads have one row, and its 64 angles take a lane one where they would
// take it 32.
constexpr int RM_ANGLES = 64 + 2;          // pairs of a row in the table, two of padding
constexpr int RM_ROWS = 4;                 // rows of a wave's table
constexpr int RM_LDS_DIRECT = RM_ANGLES_AT, RM_LDS_TABLE = RM_ANGLES_AT + RP_WAVES * RM_ROWS * RM_ANGLES * 8;
struct RopeTable {
    const uint64_t* turns;
    const float* weights;
    float2* angles;
};
__device__ __forceinline__ void fill_table(const RopeDev& d, int role, uint64_t* turns, float* weights) {
    if ((int)threadIdx.x < d.rotary / 2) turns[threadIdx.x] = d.turns[threadIdx.x];
    if (threadIdx.x < RP_D) weights[threadIdx.x] = d.w[role] ? (float)d.w[role][threadIdx.x] : 1.0f;
}

// Channels 16 kb + 8 h .. + 7 of a group in rows[kb]: norm and rotation, each number rounded to fp16, which the matrix instructions take.  R: rotary / 32.
// `angles`: of the group's row, or null, and the position says.
template <int R, bool PAIRS, bool DIRECT>
__device__ __forceinline__ void turn_group(u32x4 (&rows)[RM_KB], const RopeTable& table, bool norm, float eps, uint32_t position, const float2* angles, int h) {
    float by = 1.0f;
    if (norm) {
        float sum = 0.0f;
#pragma unroll
        for (int kb = 0; kb < RM_KB; ++kb) sum = dot8(__builtin_bit_cast(half8, rows[kb]), sum);
        sum += __shfl_xor(sum, 32);
        by = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.0f / RP_D, eps));
    }
    auto scaled = [&](const half8& x, int kb, float (&y)[8]) {
        const float* w = table.weights + 16 * kb + 8 * h;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = norm ? (float)x[e] * w[e] * by : (float)x[e];
    };
    auto turn = [&](int pair, float& c, float& s) {
        if constexpr (DIRECT) {
            cos_sin(angle_of(position, table.turns[pair]), c, s);
        } else {
            const float2 a = angles[pair];
            c = a.x;
            s = a.y;
        }
    };
    auto put = [&](int kb, const float (&y)[8]) {
        half8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (_Float16)y[e];
        rows[kb] = __builtin_bit_cast(u32x4, o);
    };
    if constexpr (PAIRS) {
#pragma unroll
        for (int kb = 0; kb < 2 * R; ++kb) {
            float y[8], z[8];
            scaled(__builtin_bit_cast(half8, rows[kb]), kb, y);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float c, s;
                turn(8 * kb + 4 * h + e, c, s);
                z[2 * e] = __builtin_fmaf(y[2 * e], c, -y[2 * e + 1] * s);
                z[2 * e + 1] = __builtin_fmaf(y[2 * e + 1], c, y[2 * e] * s);
            }
            put(kb, z);
        }
    } else {
#pragma unroll
        for (int kb = 0; kb < R; ++kb) {
            float a[8], b[8];
            scaled(__builtin_bit_cast(half8, rows[kb]), kb, a);
            scaled(__builtin_bit_cast(half8, rows[kb + R]), kb + R, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float c, s;
                turn(16 * kb + 8 * h + e, c, s);
                const float x = a[e], y = b[e];
                a[e] = __builtin_fmaf(x, c, -y * s);
                b[e] = __builtin_fmaf(y, c, x * s);
            }
            put(kb, a);
            put(kb + R, b);
        }
    }
    if (norm)
#pragma unroll
        for (int kb = 2 * R; kb < RM_KB; ++kb) {
            float y[8];
            scaled(__builtin_bit_cast(half8, rows[kb]), kb, y);
            put(kb, y);
        }
}

// The groups that a matrix has: all of a role's, or those of one head.
struct RopeGroups {
    const RopeDev& d;
    int role, head, per_row;
    int64_t count;
    __device__ __forceinline__ RopeGroups(const RopeDev& dev, int matrix) : d(dev) {
        if (d.per_head) {
            role = matrix >= d.heads[0];
            head = matrix - (role ? d.heads[0] : 0);
            per_row = 1;
        } else {
            role = matrix > 0 || !d.rows[0];
            head = 0;
            per_row = d.heads[role];
        }
        count = d.T * per_row;
    }
    __device__ __forceinline__ const _Float16* matrix() const { return d.P[role] + (int64_t)head * RP_D * RP_D; }
    __device__ __forceinline__ void at(int64_t n, int64_t& row, int& of) const {               // counts stay below 2^31
        row = per_row == 1 ? (uint32_t)n : (uint32_t)n / (uint32_t)per_row;
        of = head + (int)(n - row * per_row);
    }
};

template <int R, bool PAIRS, bool DIRECT>
__global__ __launch_bounds__(RP_NT) __attribute__((amdgpu_waves_per_eu(2))) void rope_matrix_kernel(RopeDev d, RopeDev plain) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    u32x4* Pf = reinterpret_cast<u32x4*>(smem);                                // fragment table
    _Float16* Pflat = reinterpret_cast<_Float16*>(smem + RM_LOOP_AT);          // prologue only
    const int tid = threadIdx.x;
    const int l = tid & 63, c = l & 31, h = l >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RopeGroups groups(d, blockIdx.y);
    const int64_t blocks = (groups.count + RM_GROUPS - 1) / RM_GROUPS, step = (int64_t)gridDim.x * RP_WAVES;
    // The side without a matrix goes along, eight heads of four rows at a time by a wave, the last workgroups first, some of which may have nothing else to do: at the start in one
    // half of the workgroups, at the end in the other, so that what is bound by memory runs beside what has products to do (8192 rows of 32 + 8 heads 38.8 us; in two launches 41.3).
    const int plain_heads = plain.heads[0] + plain.heads[1], chunks = (plain_heads + 7) / 8;
    auto turn_plain = [&] {
        const int64_t all = plain_heads > 0 ? (plain.T + 3) / 4 * chunks : 0;
        const int64_t waves = (int64_t)gridDim.x * gridDim.y * RP_WAVES;
        for (int64_t k = waves - 1 - (((int64_t)blockIdx.x * gridDim.y + blockIdx.y) * RP_WAVES + w); k < all; k += waves)
            turn_rows<4>(plain, k / chunks, (int)(k % chunks) * 8, 8);
    };
    const bool plain_first = 2 * blockIdx.x < gridDim.x;
    if (plain_first) turn_plain();
    if ((int64_t)blockIdx.x * RP_WAVES >= blocks) {
        if (!plain_first) turn_plain();
        return;
    }

    // A group's row, or the last one's behind the end, and where its output starts (below zero: nowhere)
    struct Block {
        u32x4 rows[RM_KB];
        int position, from_first;          // rows behind the first group's
        int64_t to;
    };
    auto issue = [&](int64_t block, Block& b) {
        const int64_t mine = block * RM_GROUPS + c, n = mine < groups.count ? mine : groups.count - 1;
        int64_t row;
        int of;
        groups.at(n, row, of);
        const u32x4* from = reinterpret_cast<const u32x4*>(d.rows[groups.role] + row * d.stride[groups.role] + of * RP_D);
#pragma unroll
        for (int kb = 0; kb < RM_KB; ++kb) b.rows[kb] = from[2 * kb + h];
        b.position = d.positions[row];
        if constexpr (!DIRECT) b.from_first = (int)(row - __shfl((long long)row, 0));
        b.to = mine < groups.count ? row * d.out_stride[groups.role] + of * RP_D : -1;
    };

    // P: coalesced loads, all of them before the first rows (which come from further away and would stand before those of a workgroup that starts a little
    // later), to LDS, and as fragments: lane (c, h) of fragment (mt, kb) holds P[16 kb + 8 h + s][32 mt + c'], s = 0 .. 7, c' = c with its 4-column chunks
    // 1 and 2 (of each 16) exchanged, so that a lane's results are runs of 8 channels.
    const _Float16* P = groups.matrix();
    constexpr int CHUNKS = RP_D * RP_D / 8;
    u32x4 v[CHUNKS / RP_NT];
#pragma unroll
    for (int k = 0; k < CHUNKS / RP_NT; ++k) v[k] = reinterpret_cast<const u32x4*>(P)[tid + k * RP_NT];
    uint64_t* turns = reinterpret_cast<uint64_t*>(smem + RM_TABLE_AT);
    float* weights = reinterpret_cast<float*>(smem + RM_TABLE_AT + 64 * 8);
    const RopeTable table{turns, weights, reinterpret_cast<float2*>(smem + RM_ANGLES_AT) + w * RM_ROWS * RM_ANGLES};
    fill_table(d, groups.role, turns, weights);
#pragma unroll
    for (int k = 0; k < CHUNKS / RP_NT; ++k) {
        const int q = tid + k * RP_NT;
        *reinterpret_cast<u32x4*>(Pflat + (q >> 4) * (RP_D + 8) + (q & 15) * 8) = v[k];
    }
    int64_t block = (int64_t)blockIdx.x * RP_WAVES + w;
    Block cur, nxt;
    __builtin_amdgcn_sched_barrier(0);
    issue(block, cur);
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    for (int e = tid; e < RM_MT * RM_KB * 64; e += RP_NT) {
        const int ln = e & 63, kb = (e >> 6) % RM_KB, mt = (e >> 6) / RM_KB;
        *reinterpret_cast<half8*>(&Pf[e]) = lds_column8<true>(Pflat, RP_D + 8, 16 * kb + 8 * (ln >> 5), 4, 32 * mt + (ln & 16), ln & 15);
        (void)mt;
    }
    __syncthreads();                                                           // the flat copy's place becomes the waves' stages

    unsigned char* stage = smem + RM_LOOP_AT + w * RM_GROUPS * RM_OUT_PITCH;
    _Float16* out = d.out[groups.role];
    auto work = [&](int64_t at, Block& b, Block& far) {
        issue(at + step < blocks ? at + step : blocks - 1, far);
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t position = b.position < 0 ? 0u : (uint32_t)b.position;
        if constexpr (!DIRECT && R > 0) {                                      // a pair a lane, row by row
            const int rows = __builtin_amdgcn_readlane(b.from_first, RM_GROUPS - 1) + 1;
            for (int k = 0; k < rows; ++k) {
                const uint64_t has = __ballot(b.from_first == k && h == 0);    // (rows follow each other: every k has a lane)
                const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)position, has ? __builtin_ctzll(has) : 0);
                float2 a;
                cos_sin(angle_of(p, turns[l < 16 * R ? l : 0]), a.x, a.y);
                if (l < 16 * R && k < RM_ROWS) table.angles[k * RM_ANGLES + l] = a;
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
        turn_group<R, PAIRS, DIRECT>(b.rows, table, d.w[groups.role] != nullptr, d.eps, position, table.angles + (DIRECT ? 0 : b.from_first) * RM_ANGLES, h);
        f32x16 acc[RM_MT];
#pragma unroll
        for (int mt = 0; mt < RM_MT; ++mt)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[mt][r] = 0.0f;
#pragma unroll
        for (int kb = 0; kb < RM_KB; ++kb)
#pragma unroll
            for (int mt = 0; mt < RM_MT; ++mt)
                acc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8*>(&Pf[(mt * RM_KB + kb) * 64 + l]),
                                                                 __builtin_bit_cast(half8, b.rows[kb]), acc[mt], 0, 0, 0);
        // whole rows leave with 16-byte stores, by way of the wave's stage
        unsigned char* mine = stage + c * RM_OUT_PITCH;
#pragma unroll
        for (int mt = 0; mt < RM_MT; ++mt)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                half8 y;
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = (_Float16)acc[mt][8 * u + k];
                *reinterpret_cast<half8*>(mine + 2 * (32 * mt + 16 * u + 8 * h)) = y;
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const int64_t to = b.position >= 0 ? b.to : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int r = (l >> 4) + 4 * k;
            const u32x4 y = *reinterpret_cast<const u32x4*>(stage + r * RM_OUT_PITCH + 16 * (l & 15));
            const int64_t dst = __shfl((long long)to, r);
            if (dst >= 0) __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(out + dst + 8 * (l & 15)));
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();                                       // read before the next block overwrites it
    };
    while (block < blocks) {
        work(block, cur, nxt);
        block += step;
        if (block >= blocks) break;
        work(block, nxt, cur);
        block += step;
    }
    if (!plain_first) turn_plain();
}

// Few groups: a workgroup takes 32 of them, each of its waves 32 of the 128 outputs; its quarter of P goes through a part of LDS of its own, the angles of the
// groups' rows are worked out by all.  Same arithmetic in the same order as above: the same bits.  The workgroups behind those (blockIdx.y = matrices) have the
// side without a matrix, a head a wave: one launch for both.
template <int R, bool PAIRS>
__global__ __launch_bounds__(RP_NT) void rope_matrix_few_kernel(RopeDev d, RopeDev plain, int matrices) {
    constexpr int PITCH = 32 + 8;
    __shared__ __attribute__((aligned(16))) _Float16 Pw_all[RP_WAVES * RP_D * PITCH];
    __shared__ __attribute__((aligned(16))) float weights[RP_D];
    __shared__ __attribute__((aligned(16))) float2 angles[RM_GROUPS * RM_ANGLES];
    const int l = threadIdx.x & 63, c = l & 31, h = l >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.y == matrices) {
        const int heads = plain.heads[0] + plain.heads[1], waves = (heads + RP_WAVES - 1) / RP_WAVES;
        for (int64_t k = blockIdx.x; k < (plain.T + 3) / 4 * waves; k += gridDim.x) turn_rows<1>(plain, k / waves, (int)(k % waves) * RP_WAVES + w, 1);
        return;
    }
    const RopeGroups groups(d, blockIdx.y);
    if ((int64_t)blockIdx.x * RM_GROUPS >= groups.count) return;
    const _Float16* P = groups.matrix() + 32 * w;
    _Float16* Pw = Pw_all + w * RP_D * PITCH;
    const int64_t mine = (int64_t)blockIdx.x * RM_GROUPS + c, n = mine < groups.count ? mine : groups.count - 1;
    int64_t row;
    int of;
    groups.at(n, row, of);
    // what the angles take first: loads return in order.  Positions of the groups' rows, one a lane; a wave takes every fourth of them, a lane a pair
    const int64_t first = __shfl((long long)row, 0), last = __shfl((long long)row, RM_GROUPS - 1);
    const uint64_t turn = R > 0 ? d.turns[l < 16 * R ? l : 0] : 0;
    const int positions = d.positions[first + c <= last ? first + c : last];
    const float weight = d.w[groups.role] ? (float)d.w[groups.role][threadIdx.x & (RP_D - 1)] : 1.0f;
    __builtin_amdgcn_sched_barrier(0);
    u32x4 v[8], rows[RM_KB];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const u32x4*>(P + (16 * k + (l >> 2)) * RP_D + 8 * (l & 3));
    const u32x4* from = reinterpret_cast<const u32x4*>(d.rows[groups.role] + row * d.stride[groups.role] + of * RP_D);
#pragma unroll
    for (int kb = 0; kb < RM_KB; ++kb) rows[kb] = from[2 * kb + h];
    __builtin_amdgcn_sched_barrier(0);
    if ((int)threadIdx.x < RP_D) weights[threadIdx.x] = weight;
    if constexpr (R > 0)
        for (int k = w; first + k <= last; k += RP_WAVES) {
            const int p = __builtin_amdgcn_readlane(positions, k);
            float2 a;
            cos_sin(angle_of(p < 0 ? 0u : (uint32_t)p, turn), a.x, a.y);
            if (l < 16 * R) angles[k * RM_ANGLES + l] = a;
        }
#pragma unroll
    for (int k = 0; k < 8; ++k) *reinterpret_cast<u32x4*>(Pw + (16 * k + (l >> 2)) * PITCH + 8 * (l & 3)) = v[k];
    __syncthreads();
    turn_group<R, PAIRS, false>(rows, RopeTable{nullptr, weights, angles}, d.w[groups.role] != nullptr, d.eps, 0u, angles + (int)(row - first) * RM_ANGLES, h);
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
#pragma unroll
    for (int kb = 0; kb < RM_KB; ++kb)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_column8<true>(Pw, PITCH, 16 * kb + 8 * h, 4, c & 16, l & 15), __builtin_bit_cast(half8, rows[kb]), acc, 0, 0, 0);
    const int position = __shfl(positions, (int)(row - first));
    if (mine >= groups.count || position < 0) return;
    _Float16* out = d.out[groups.role] + row * d.out_stride[groups.role] + of * RP_D + 32 * w + 8 * h;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        half8 o;
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = (_Float16)acc[8 * u + k];
        *reinterpret_cast<half8*>(out + 16 * u) = o;
    }
}

// Rows of 32 groups at most.
static int rows_of_groups(const RopeDev& d) {
    if (d.per_head) return RM_GROUPS;
    int heads = 1 << 30;
    for (int x = 0; x < 2; ++x)
        if (d.rows[x] && d.heads[x] < heads) heads = d.heads[x];
    return RM_GROUPS % heads == 0 ? RM_GROUPS / heads : (RM_GROUPS - 1) / heads + 2;
}
template <int R, bool PAIRS>
static hipError_t rope_matrix_launch(const RopeDev& d, const RopeDev& plain, hipStream_t stream) {
    const unsigned matrices = d.per_head ? (unsigned)(d.heads[0] + d.heads[1]) : (unsigned)((d.rows[0] != nullptr) + (d.rows[1] != nullptr));
    const int64_t most = d.per_head ? d.T : d.T * (d.heads[0] > d.heads[1] ? d.heads[0] : d.heads[1]);
    const int64_t blocks = (most + RM_GROUPS - 1) / RM_GROUPS;
    // Up to one workgroup a CU the kernel for few.  us, few / many: 32 + 8 heads, the queries through one matrix, 150 rows 6.6 / 8.7, 256 6.9 / 8.8, 400 8.6 / 9.0, 500 10.0 / 9.4;
    // 32 + 32 heads, 256 rows 7.1 / 8.9, 300 9.4 / 9.0, 400 12.1 / 9.7; through one each, 32 + 8 heads, 150 rows 7.8 / 10.3, 200 10.4 / 10.5, 300 10.7 / 11.2.
    if (blocks * matrices <= cu_count()) {
        const bool both = plain.heads[0] + plain.heads[1] > 0;
        return launch(rope_matrix_few_kernel<R, PAIRS>, dim3((unsigned)blocks, matrices + both), dim3(RP_NT), 0, stream, d, plain, (int)matrices);
    }
    auto many = [&](auto kernel, int lds, OccCache& cache) {
        int occ = 0;
        const hipError_t e = kernel_occupancy(reinterpret_cast<const void*>(kernel), RP_NT, lds, cache, occ);
        if (e != hipSuccess) return e;
        const int64_t need = (blocks + RP_WAVES - 1) / RP_WAVES;
        int64_t gx = ((int64_t)cu_count() * occ + matrices - 1) / matrices;
        const int64_t rounds = (need + gx - 1) / gx;
        const int64_t most = gx, tasks = (plain.T + 3) / 4 * ((plain.heads[0] + plain.heads[1] + 7) / 8), others = (tasks + RP_WAVES * matrices - 1) / (RP_WAVES * matrices);
        gx = (need + rounds - 1) / rounds;
        if (rounds == 1) gx = gx + others < most ? gx + others : most;         // workgroups for the side without a matrix, where there is room
        return launch(kernel, dim3((unsigned)gx, matrices), dim3(RP_NT), lds, stream, d, plain);
    };
    static OccCache caches[2];
    // (8192 rows of 32 + 8 heads, the queries through one matrix: 38.5 us with the table, 45.5 without)
    if (rows_of_groups(d) <= RM_ROWS) return many(rope_matrix_kernel<R, PAIRS, false>, RM_LDS_TABLE, caches[0]);
    return many(rope_matrix_kernel<R, PAIRS, true>, RM_LDS_DIRECT, caches[1]);
}

constexpr int64_t kMostBlocks = 1 << 20;   // (a grid has less than 2^32 threads)
hipError_t rope_launch(const RopeDev& all, hipStream_t stream) {
    RopeDev plain = all, through = all;
    for (int x = 0; x < 2; ++x) {
        RopeDev& not_here = all.P[x] ? plain : through;
        not_here.rows[x] = nullptr;
        not_here.heads[x] = 0;
        if (!all.rows[x]) plain.heads[x] = through.heads[x] = 0;
    }
    if (through.rows[0] || through.rows[1]) {
        const int r = all.rotary / 32;
        const bool pairs = all.interleaved && r > 0;
        hipError_t e = hipErrorInvalidValue;
        switch (2 * r + pairs) {
            case 0: e = rope_matrix_launch<0, false>(through, plain, stream); break;
            case 2: e = rope_matrix_launch<1, false>(through, plain, stream); break;
            case 3: e = rope_matrix_launch<1, true>(through, plain, stream); break;
            case 4: e = rope_matrix_launch<2, false>(through, plain, stream); break;
            case 5: e = rope_matrix_launch<2, true>(through, plain, stream); break;
            case 6: e = rope_matrix_launch<3, false>(through, plain, stream); break;
            case 7: e = rope_matrix_launch<3, true>(through, plain, stream); break;
            case 8: e = rope_matrix_launch<4, false>(through, plain, stream); break;
            case 9: e = rope_matrix_launch<4, true>(through, plain, stream); break;
        }
        return e;
    }
    const int heads = plain.heads[0] + plain.heads[1];
    if (heads == 0) return hipSuccess;
    const int64_t blocks = (plain.T + 3) / 4;
    // Heads of a wave, which works the angles of its four rows out for all of them: as many as leave 2048 waves, two a SIMD, and 8 at most.  us with 1024 / 2048 / 4096 waves left:
    // 777 rows of 40 heads 7.6 / 6.8 / 7.3, 1500 14.1 / 10.9 / 10.3, 512 of 64 8.6 / 7.5 / 7.4; with 4 / 8 / 16 heads at most: 16384 of 40 64.7 / 59.7 / 66.9, 4096 18.3 / 16.9 / 16.6.
    int per = 1;
    while (per < 8 && blocks * ((heads + 2 * per - 1) / (2 * per)) >= 2048) per *= 2;
    const dim3 grid((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks), (unsigned)((heads + RP_WAVES * per - 1) / (RP_WAVES * per)));
    if (per == 1) return launch(rope_kernel<1>, grid, dim3(RP_NT), 0, stream, plain, per);
    if (per == 2) return launch(rope_kernel<2>, grid, dim3(RP_NT), 0, stream, plain, per);
    return launch(rope_kernel<4>, grid, dim3(RP_NT), 0, stream, plain, per);
}

}  // namespace fq
