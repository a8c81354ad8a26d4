// The tables of a step on the paged key/value cache: row starts, lengths, pages taken from and given back to the ring of free ones, and the rows'
// positions and places (see flatquant.h).
//
// With n_b rows of sequence b and P = ceil(tokens / page), cut to the table's width: starts are the running sum of n, the pages that sequence b takes are
// max(0, P(keep + n) - P(held)) and lie in the ring behind those of the sequences before it, and what it gives back, max(0, P(held) - P(keep + n)) entries
// but those that are no page, is put behind the ring's last in the same order.  All of it follows from running sums over the sequences, so one
// workgroup works it out, 1024 sequences at a time: the order of the pages is that of the sequences, whatever runs first, and nothing has to be cleared or
// counted in memory.  Entries that change are dealt out to its waves evenly, as one sequence may have most of them: a wave looks for the sequences of its first and its
// last entry, and those between by bisection in LDS.
//
// Bound by latency, and on its one CU by the instructions of an entry: 64 decoding sequences 4.7 us (replayed; a launch, the sequences' loads, three running sums, rows), 512 in mixed states
// (1150 pages taken, 15800 given back) 11 and 4 for their 18500 rows, 16 prompts of 65536 tokens (42900 pages, 686000 rows) 12 and 6.  Rows of more than a few
// thousand tokens are worked out by a second kernel on all CUs.
#include "fq_internal.h"
#include "fq_cache_device.h"

namespace fq {

constexpr int ADV_NT = 1024;               // sequences of a chunk, threads
constexpr int ADV_WAVES = ADV_NT / 64;
constexpr int kSaturated = 1 << 30;        // of row counts: above every T

// (as numbers without a sign: two that are saturated add up to 2^31)
constexpr __host__ __device__ __forceinline__ int saturated_add(int a, int b) {
    const uint32_t sum = (uint32_t)a + (uint32_t)b;
    return sum < (uint32_t)kSaturated ? (int)sum : kSaturated;
}
static_assert(saturated_add(kSaturated, kSaturated) == kSaturated && saturated_add(kSaturated - 1, 1) == kSaturated && saturated_add(kSaturated, 0) == kSaturated &&
                  saturated_add(3, 4) == 7, "sums of row counts");
// Value of the lane N places before in its row of 16 (SHIFT), or of the last lane of the row or half before; zero where there is none.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t lane_before(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false); }
// Running sums over the lanes of a wave, the lane's own among them.
template <typename Add>
__device__ __forceinline__ uint32_t wave_sums(uint32_t x, Add add) {
    x = add(x, lane_before<0x111>(x));                                         // row_shr:1, 2, 4, 8
    x = add(x, lane_before<0x112>(x));
    x = add(x, lane_before<0x114>(x));
    x = add(x, lane_before<0x118>(x));
    x = add(x, lane_before<0x142, 0xA>(x));                                    // row_bcast:15 to rows 1 and 3
    return add(x, lane_before<0x143, 0xC>(x));                                 // row_bcast:31 to rows 2 and 3
}
__device__ __forceinline__ uint32_t add_plain(uint32_t a, uint32_t b) { return a + b; }
__device__ __forceinline__ uint32_t add_rows(uint32_t a, uint32_t b) { return (uint32_t)saturated_add((int)a, (int)b); }
// A barrier for what lies in LDS: stores to memory may still be on their way.
__device__ __forceinline__ void local_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// Sums over the threads before this one, and of all (`all`).  `parts`: one of two arrays, taken in turn, so that one sync is enough.
template <typename Add>
__device__ __forceinline__ uint32_t running_sum(uint32_t mine, uint32_t (&parts)[2][ADV_WAVES], int& turn, uint32_t& all, Add add) {
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t s = wave_sums(mine, add);
    uint32_t (&part)[ADV_WAVES] = parts[turn];
    turn ^= 1;
    if (l == 63) part[w] = s;
    local_barrier();
    uint32_t t = l < ADV_WAVES ? part[l] : 0u;
    t = add(t, lane_before<0x111>(t));
    t = add(t, lane_before<0x112>(t));
    t = add(t, lane_before<0x114>(t));
    t = add(t, lane_before<0x118>(t));
    all = (uint32_t)__builtin_amdgcn_readlane((int)t, ADV_WAVES - 1);
    const uint32_t before = w > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)t, w - 1) : 0u;
    const uint32_t up = __shfl_up(s, 1);
    return l > 0 ? add(before, up) : before;
}

__device__ __forceinline__ int pages_of(const AdvanceDev& a, int tokens) {
    return min((int)(((uint32_t)tokens + (1u << a.page_shift) - 1u) >> a.page_shift), a.table_width);
}

// What a chunk's threads know of their sequences.
struct Step {
    int keep, rows, start, have, need;
    int taken, released;                   // entries [have, need), or [need, have)
};
// Of sequence b, with `rows_before` rows in the chunks before.  `chunk_rows`: rows behind this chunk.
__device__ __forceinline__ Step step_of(const AdvanceDev& a, int b, int rows_before, uint32_t (&parts)[2][ADV_WAVES], int& turn, int& chunk_rows) {
    Step s{};
    int held = 0, want = 0;
    if (b < a.B) {
        held = max(a.held[b], 0);
        s.keep = min(max(a.keep[b], 0), held);
        want = min(max(a.rows[b], 0), 0x7fffffff - s.keep);                    // lengths are 32-bit numbers
        want = min(want, (int)a.T);
    }
    uint32_t all;
    const int before = (int)running_sum((uint32_t)want, parts, turn, all, add_rows);
    s.start = min(saturated_add(rows_before, before), (int)a.T);
    s.rows = min(saturated_add(s.start, want), (int)a.T) - s.start;
    chunk_rows = min(saturated_add(rows_before, (int)all), (int)a.T);
    if (b < a.B) {
        s.have = pages_of(a, held);
        s.need = pages_of(a, s.keep + s.rows);
        s.taken = max(s.need - s.have, 0);
        s.released = max(s.have - s.need, 0);
    }
    return s;
}

// The sequence of the chunk that has entry x: the last whose first entry is x or before (those without entries begin where the next one does).
__device__ __forceinline__ int owner_of(const uint32_t (&first)[ADV_NT], uint32_t x) {
    int lo = 0;
#pragma unroll
    for (int m = ADV_NT / 2; m > 0; m /= 2) lo += first[lo + m] <= x ? m : 0;
    return lo;
}

__device__ __forceinline__ int64_t place_of(const AdvanceDev& a, int b, int pos) {
    const int j = pos >> a.page_shift;
    const int page = j < a.table_width ? a.page_table[b * a.table_stride + j] : -1;
    return (uint32_t)page < (uint32_t)a.pages ? ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
}

// The sequence of entry x, the same in all lanes: of every 16th sequence, then of 16.
__device__ __forceinline__ int owner_of_all(const uint32_t (&first)[ADV_NT], uint32_t x) {
    const int l = threadIdx.x & 63;
    const int s = 16 * (__builtin_popcountll(__ballot(first[16 * l] <= x)) - 1);
    return s + __builtin_popcountll(__ballot(first[s + (l & 15)] <= x) & 0xffff) - 1;
}
// Where entries x0 + 64 k + lane of a chunk's (taken or given back), k < PER, lie in the table (at[o] + x for one of sequence o); x0 is the wave's.  What lies behind
// the last, `all` of them, is the last's place.
template <int PER>
__device__ __forceinline__ void entries(const uint32_t (&first)[ADV_NT], const int64_t (&at)[ADV_NT], uint32_t x0, uint32_t all, int64_t (&place)[PER]) {
    const uint32_t last = all - 1, x1 = x0 + (threadIdx.x & 63);
    const int lo = owner_of_all(first, min(x0, last)), hi = owner_of_all(first, min(x0 + 64 * PER - 1, last));
    int o[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) o[k] = lo;
    for (int m = hi > lo ? 1 << (31 - __builtin_clz(hi - lo)) : 0; m > 0; m /= 2)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int next = min(o[k] + m, hi);                                // (all of them, a step at a time: the reads do not wait for each other)
            o[k] = first[next] <= min(x1 + 64 * k, last) ? next : o[k];
        }
#pragma unroll
    for (int k = 0; k < PER; ++k) place[k] = at[o[k]] + min(x1 + 64 * k, last);
}

// ROWS: with the rows' positions and places (of a batch of one chunk).
template <bool ROWS>
__global__ __launch_bounds__(ADV_NT) void advance_kernel(AdvanceDev a) {
    __shared__ uint32_t taken_first[ADV_NT], first[ADV_NT];                    // first entry of a sequence among the chunk's taken and given ones; then its first row
    __shared__ int64_t taken_at[ADV_NT], at_first[ADV_NT];                     // entry x is in place x + this of the table; then a row's position less the row
    __shared__ uint32_t parts[2][ADV_WAVES];
    __shared__ unsigned long long wanted_all;
    int turn = 0;
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    int64_t taken = a.state[0], given = a.state[1];
    asm volatile("" : "+v"(taken), "+v"(given));                               // (have arrived before the first barrier: the next state may take their place behind the last)
    const int64_t capacity = a.capacity;
    int64_t available = (int64_t)((uint64_t)given - (uint64_t)taken);          // (of a state that is none: what the ring can hold at most)
    available = available < 0 ? 0 : available < capacity ? available : capacity;
    const bool one = a.B <= ADV_NT;

    // Entries that the call takes: all of them or none.
    int64_t wanted = 0;
    if (!one) {
        if (tid == 0) wanted_all = 0;
        int rows = 0;
        int64_t mine = 0;
        for (int b0 = 0; b0 < a.B; b0 += ADV_NT) mine += step_of(a, b0 + tid, rows, parts, turn, rows).taken;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) mine += __shfl_xor((long long)mine, m);
        if (l == 0) atomicAdd(&wanted_all, (unsigned long long)mine);  // (integers: any order gives the same)
        __syncthreads();
        wanted = (int64_t)wanted_all;
    }

    int rows_before = 0;
    uint32_t taken_before = 0;
    int64_t released = 0;
    auto in_ring = [&](int64_t at) {
        const int64_t r = at % capacity;
        return (uint32_t)(r < 0 ? r + capacity : r);
    };
    for (int b0 = 0; b0 < a.B; b0 += ADV_NT) {
        const int b = b0 + tid;
        int rows_behind;
        const Step s = step_of(a, b, rows_before, parts, turn, rows_behind);
        // entries taken and given back: 2^30 at most, as tables have 2^20 a row
        uint32_t takes, gone;
        const uint32_t take_at = running_sum((uint32_t)s.taken, parts, turn, takes, add_plain);
        const uint32_t gone_at = running_sum((uint32_t)s.released, parts, turn, gone, add_plain);
        if (one) wanted = takes;
        const bool enough = wanted <= available;
        if (b < a.B) {
            a.lengths[b] = s.keep + s.rows;
            a.row_starts[b] = s.start;
        }
        if (takes > 0 || gone > 0) {
            taken_first[tid] = take_at;
            taken_at[tid] = b * a.table_stride + s.have - take_at;
            first[tid] = gone_at;
            at_first[tid] = b * a.table_stride + s.need - gone_at;
            local_barrier();
        }
        if (takes > 0) {
            const uint32_t head = in_ring(taken);
            auto take = [&](auto per) {
                constexpr int PER = decltype(per)::value;
                for (uint32_t x0 = 64 * PER * w; x0 < takes; x0 += ADV_NT * PER) {
                    int page[PER];
                    int64_t place[PER];
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        const uint32_t x = x0 + 64 * k + l, r = head + taken_before + x;       // (all of them below 2^31, and the sum below twice the capacity)
                        page[k] = enough && x < takes ? a.ring[r >= (uint32_t)capacity ? r - (uint32_t)capacity : r] : -1;
                    }
                    entries<PER>(taken_first, taken_at, x0, takes, place);
#pragma unroll
                    for (int k = 0; k < PER; ++k)
                        if (x0 + 64 * k + l < takes) a.page_table[place[k]] = page[k];
                }
            };
            // 1200 entries 6.7 us one at a time by a thread, 7.9 eight at a time; 2700 7.5 / 8.1, 5700 8.7 / 8.7, 42900 23.4 / 17.7
            if (takes <= 4 * ADV_NT) take(std::integral_constant<int, 1>{});
            else take(std::integral_constant<int, 8>{});
            taken_before += enough ? takes : 0;
        }
        // what is given back, in the order of its entries
        if (gone > 0) {
            uint32_t tail = in_ring((int64_t)((uint64_t)given + (uint64_t)released));
            auto give = [&](auto per) {
                constexpr int PER = decltype(per)::value;
                for (uint32_t x0 = 0; x0 < gone; x0 += ADV_NT * PER) {
                    const uint32_t x1 = x0 + 64 * PER * w + l;
                    int page[PER];
                    int64_t place[PER];
                    entries<PER>(first, at_first, x0 + 64 * PER * w, gone, place);
#pragma unroll
                    for (int k = 0; k < PER; ++k) page[k] = a.page_table[place[k]];
                    uint64_t is[PER];
                    uint32_t mine = 0, all;
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        is[k] = __ballot((uint32_t)page[k] < (uint32_t)a.pages && x1 + 64 * k < gone);
                        mine += __builtin_popcountll(is[k]);
                    }
                    uint32_t at = tail + running_sum(l == 63 ? mine : 0u, parts, turn, all, add_plain);        // of the waves before
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        uint32_t r = __builtin_amdgcn_mbcnt_hi((uint32_t)(is[k] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)is[k], at));
                        if (capacity > ADV_NT * PER) r = r >= (uint32_t)capacity ? r - (uint32_t)capacity : r;
                        else r %= (uint32_t)capacity;
                        if (is[k] >> l & 1) {
                            a.ring[r] = page[k];
                            if (!enough) a.page_table[place[k]] = -1;          // the call is made again with the same figures: it finds no page there
                        }
                        at += __builtin_popcountll(is[k]);
                    }
                    tail = (tail + all) % (uint32_t)capacity;
                    released += all;
                }
            };
            // (of 2000 entries 9.9 us one at a time by a thread, 8.3 four, 11.7 sixteen; of 15800 23.7, 14.9 and 14.6)
            if (gone <= ADV_NT) give(std::integral_constant<int, 1>{});
            else give(std::integral_constant<int, 4>{});
        }
        rows_before = rows_behind;
        if constexpr (ROWS) {
            __syncthreads();                                                   // the table's new entries are there
            first[tid] = b < a.B ? (uint32_t)s.start : 0xffffffffu;
            at_first[tid] = (int64_t)s.keep - s.start;
            local_barrier();
            for (int t = tid; t < (int)a.T; t += ADV_NT) {
                int pos = -1;
                int64_t at = -1;
                if (t < rows_behind) {
                    const int o = owner_of(first, (uint32_t)t);
                    pos = (int)at_first[o] + t;
                    if (a.slots) at = place_of(a, o, pos);
                }
                if (a.positions) a.positions[t] = pos;
                if (a.slots) a.slots[t] = at;
            }
        }
    }
    if (tid == 0) {
        a.row_starts[a.B] = rows_before;
        const bool enough = wanted <= available;
        a.next[0] = enough ? taken + wanted : taken;
        a.next[1] = (int64_t)((uint64_t)given + (uint64_t)released);
        a.next[2] = enough ? 0 : wanted - available;
    }
}

// The last of sequences lo .. hi that starts at row t or before, the same t in all lanes of the wave: 64 of them a look.
__device__ __forceinline__ int sequence_of_row(const AdvanceDev& a, int lo, int hi, int t) {
    const int l = threadIdx.x & 63;
    while (hi > lo) {
        const int stride = (hi - lo + 64) / 64, at = lo + stride * l;          // lane 0 has lo, which does
        const int n = __builtin_popcountll(__ballot(at <= hi && a.row_starts[min(at, hi)] <= t));
        lo += stride * (n - 1);
        hi = min(hi, lo + stride - 1);
    }
    return lo;
}
// Positions and places of the rows of a batch, a row a lane.  A wave looks for the sequences of its first and its last row; those between, 64 or fewer, lie
// in its lanes.
__global__ __launch_bounds__(256) void advance_rows_kernel(AdvanceDev a) {
    const int l = threadIdx.x & 63;
    const int rows = a.row_starts[a.B];
    for (int64_t t0 = (int64_t)blockIdx.x * 256 + 64 * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); t0 < a.T; t0 += (int64_t)gridDim.x * 256) {
        const int t = (int)t0 + l;
        int pos = -1;
        int64_t at = -1;
        if ((int)t0 < rows) {
            int lo = sequence_of_row(a, 0, a.B - 1, (int)t0);
            const int last = sequence_of_row(a, lo, a.B - 1, min((int)t0 + 63, rows - 1));
            if (last > lo) {
                const int count = last - lo;
                if (count < 64) {
                    const int starts = a.row_starts[lo + min(l, count)];
                    int n = 0;
#pragma unroll
                    for (int m = 32; m > 0; m /= 2) {
                        const int start = __shfl(starts, min(n + m, count));   // (all lanes take part)
                        n += n + m <= count && start <= t ? m : 0;
                    }
                    lo += n;
                } else {
                    int hi = last;
                    while (lo < hi) {
                        const int mid = (lo + hi + 1) >> 1;
                        if (a.row_starts[mid] <= t) lo = mid;
                        else hi = mid - 1;
                    }
                }
            }
            if (t < rows) {
                pos = a.lengths[lo] - a.row_starts[lo + 1] + t;
                if (a.slots) at = place_of(a, lo, pos);
            }
        }
        if (t < a.T) {
            if (a.positions) a.positions[t] = pos;
            if (a.slots) a.slots[t] = at;
        }
    }
}

hipError_t advance_launch(const AdvanceDev& a, hipStream_t stream) {
    const bool maps = (a.positions || a.slots) && a.T > 0;
    // The rows in the same kernel, or in one of their own?  us: 64 sequences of a row 4.7 / 6.1, 8 of 300 rows 5.1 / 6.7, of 600 5.9 / 7.2, of 2000 11.1 / 6.6, of 6000 24.5 / 6.9.
    if (maps && a.B <= ADV_NT && a.T <= 4 * ADV_NT) return launch(advance_kernel<true>, dim3(1), dim3(ADV_NT), 0, stream, a);
    const hipError_t e = launch(advance_kernel<false>, dim3(1), dim3(ADV_NT), 0, stream, a);
    if (e != hipSuccess || !maps) return e;
    const int64_t blocks = (a.T + 255) / 256, most = 16LL * cu_count();
    return launch(advance_rows_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream, a);
}

}  // namespace fq
