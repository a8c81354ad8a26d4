// The tables of a step on the paged key/value cache: row starts, lengths, pages taken from and given back to the ring of free ones, and the rows'
// positions and places (see flatquant.h).
//
// With n_b rows of sequence b and P = ceil(tokens / page), cut to the table's width: starts are the running sum of n, the pages that sequence b takes are
// max(0, P(keep + n) - P(held)) and lie in the ring behind those of the sequences before it, and what it gives back, max(0, P(held) - P(keep + n)) entries
// but those that are no page, is put behind the ring's last in the same order.  All of it follows from running sums over the sequences, so one
// workgroup works it out, 1024 sequences at a time: the order of the pages is that of the sequences, whatever runs first, and nothing has to be cleared or
// counted in memory.  Entries that change are dealt out to its threads evenly (a thread finds the sequence of its entry by bisection in LDS), as
// one sequence may have most of them.
//
// Bound by latency: loads of a chunk, one running sum in LDS, ring to table, rows.  Rows of more than a few thousand tokens are worked out by a second
// kernel on all CUs, whose stores bound it.
#include "fq_internal.h"
#include "fq_cache_device.h"

namespace fq {

constexpr int ADV_NT = 1024;               // sequences of a chunk, threads
constexpr int ADV_WAVES = ADV_NT / 64;
constexpr int kSaturated = 1 << 30;        // of row counts: above every T

// Sums over the sequences before this thread's (`before`), and of all of the chunk (`all`).  Two syncs.
struct Sums {
    int rows;            // stays at kSaturated
    uint32_t pages;      // modulo 2^32: used where all of them fit the ring
};
__device__ __forceinline__ int saturated_add(int a, int b) { return min(a + b, kSaturated); }
__device__ __forceinline__ Sums running_sums(Sums mine, Sums (&parts)[ADV_WAVES], Sums& all) {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    Sums s = mine;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int r = __shfl_up(s.rows, m);
        const uint32_t p = __shfl_up(s.pages, m);
        if (l >= m) {
            s.rows = saturated_add(s.rows, r);
            s.pages += p;
        }
    }
    __syncthreads();                                                           // (parts may still be read from the last time)
    if (l == 63) parts[w] = s;
    __syncthreads();
    // of the waves: lanes 0 .. 15 of every wave
    Sums t = l < ADV_WAVES ? parts[l] : Sums{0, 0};
#pragma unroll
    for (int m = 1; m < ADV_WAVES; m *= 2) {
        const int r = __shfl_up(t.rows, m);
        const uint32_t p = __shfl_up(t.pages, m);
        if (l >= m) {
            t.rows = saturated_add(t.rows, r);
            t.pages += p;
        }
    }
    all.rows = __shfl(t.rows, ADV_WAVES - 1);
    all.pages = __shfl(t.pages, ADV_WAVES - 1);
    Sums before{__shfl_up(s.rows, 1), __shfl_up(s.pages, 1)};
    if (l == 0) before = Sums{0, 0};
    if (w > 0) {
        before.rows = saturated_add(before.rows, __shfl(t.rows, w - 1));
        before.pages += __shfl(t.pages, w - 1);
    }
    return before;
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
__device__ __forceinline__ Step step_of(const AdvanceDev& a, int b, int rows_before, Sums (&parts)[ADV_WAVES], int& chunk_rows) {
    Step s{};
    int held = 0, want = 0;
    if (b < a.B) {
        held = max(a.held[b], 0);
        s.keep = min(max(a.keep[b], 0), held);
        want = min(max(a.rows[b], 0), 0x7fffffff - s.keep);                    // lengths are 32-bit numbers
        want = min(want, (int)a.T);
    }
    Sums all;
    const Sums before = running_sums(Sums{want, 0}, parts, all);
    s.start = min(saturated_add(rows_before, before.rows), (int)a.T);
    s.rows = min(saturated_add(s.start, want), (int)a.T) - s.start;
    chunk_rows = min(saturated_add(rows_before, all.rows), (int)a.T);
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

// ROWS: with the rows' positions and places (of a batch of one chunk).
template <bool ROWS>
__global__ __launch_bounds__(ADV_NT) void advance_kernel(AdvanceDev a) {
    __shared__ uint32_t first[ADV_NT];                                         // first entry of a sequence among the chunk's; then its first row
    __shared__ int from[ADV_NT];                                               // its place in the table; then its position
    __shared__ Sums parts[ADV_WAVES];
    __shared__ unsigned long long wanted_all;
    const int tid = threadIdx.x;
    const int64_t taken = a.state[0], given = a.state[1];
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
        for (int b0 = 0; b0 < a.B; b0 += ADV_NT) mine += step_of(a, b0 + tid, rows, parts, rows).taken;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) mine += __shfl_xor((long long)mine, m);
        if ((tid & 63) == 0) atomicAdd(&wanted_all, (unsigned long long)mine);  // (integers: any order gives the same)
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
    const uint32_t head = in_ring(taken);
    uint32_t tail = in_ring(given);
    auto behind = [&](uint32_t at, uint32_t n) {                               // at + n modulo the capacity, n less than it
        const uint32_t r = at + n;                                             // (both below 2^31)
        return r >= (uint32_t)capacity ? r - (uint32_t)capacity : r;
    };
    for (int b0 = 0; b0 < a.B; b0 += ADV_NT) {
        const int b = b0 + tid;
        int rows_behind;
        const Step s = step_of(a, b, rows_before, parts, rows_behind);
        Sums all;                                                              // entries given back (rows) and taken (pages): 2^30 at most, as tables have 2^20 a row
        const Sums t0 = running_sums(Sums{s.released, (uint32_t)s.taken}, parts, all);
        if (one) wanted = all.pages;
        const bool enough = wanted <= available;
        if (b < a.B) {
            a.lengths[b] = s.keep + s.rows;
            a.row_starts[b] = s.start;
        }
        if (all.pages > 0) {
            __syncthreads();
            first[tid] = t0.pages;
            from[tid] = s.have;
            __syncthreads();
            for (uint32_t x = tid; x < all.pages; x += ADV_NT) {
                const int o = owner_of(first, x);
                a.page_table[(b0 + o) * a.table_stride + from[o] + (int)(x - first[o])] = enough ? a.ring[behind(head, taken_before + x)] : -1;
            }
            taken_before += enough ? all.pages : 0;
        }
        // what is given back, in the order of its entries
        if (all.rows > 0) {
            __syncthreads();
            first[tid] = (uint32_t)t0.rows;
            from[tid] = s.need;
            __syncthreads();
            for (int x0 = 0; x0 < all.rows; x0 += ADV_NT) {
                const int x = x0 + tid;
                int page = -1;
                if (x < all.rows) {
                    const int o = owner_of(first, (uint32_t)x);
                    page = a.page_table[(b0 + o) * a.table_stride + from[o] + (x - (int)first[o])];
                }
                const bool is = (uint32_t)page < (uint32_t)a.pages;
                Sums tile;
                const Sums at = running_sums(Sums{0, is ? 1u : 0u}, parts, tile);
                if (is) a.ring[(tail + at.pages) % (uint32_t)capacity] = page;
                tail = (tail + tile.pages) % (uint32_t)capacity;
                released += tile.pages;
            }
        }
        rows_before = rows_behind;
        if constexpr (ROWS) {
            __syncthreads();
            first[tid] = b < a.B ? (uint32_t)s.start : 0xffffffffu;
            from[tid] = s.keep;
            __syncthreads();
            for (int t = tid; t < (int)a.T; t += ADV_NT) {
                int pos = -1;
                int64_t at = -1;
                if (t < rows_behind) {
                    const int o = owner_of(first, (uint32_t)t);
                    pos = from[o] + (t - (int)first[o]);
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
        a.next[1] = given + released;
        a.next[2] = enough ? 0 : wanted - available;
    }
}

// Positions and places of the rows of a batch, a row a thread: the sequence by a guess (equal numbers of rows), then bisection.
__global__ __launch_bounds__(256) void advance_rows_kernel(AdvanceDev a) {
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < a.T; t += (int64_t)gridDim.x * 256) {
        int pos = -1;
        int64_t at = -1;
        if (t < a.row_starts[a.B]) {
            int lo = 0, hi = a.B - 1;                                          // the last that starts at t or before
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.row_starts[mid] <= t) lo = mid;
                else hi = mid - 1;
            }
            pos = a.lengths[lo] - a.row_starts[lo + 1] + (int)t;
            if (a.slots) at = place_of(a, lo, pos);
        }
        if (a.positions) a.positions[t] = pos;
        if (a.slots) a.slots[t] = at;
    }
}

hipError_t advance_launch(const AdvanceDev& a, hipStream_t stream) {
    const bool maps = (a.positions || a.slots) && a.T > 0;
    if (maps && a.B <= ADV_NT && a.T <= 4 * ADV_NT) return launch(advance_kernel<true>, dim3(1), dim3(ADV_NT), 0, stream, a);
    const hipError_t e = launch(advance_kernel<false>, dim3(1), dim3(ADV_NT), 0, stream, a);
    if (e != hipSuccess || !maps) return e;
    const int64_t blocks = (a.T + 255) / 256, most = 16LL * cu_count();
    return launch(advance_rows_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream, a);
}

}  // namespace fq
