// Attention over the paged key/value cache: how a launch is cut, and the kernels (fq_attention_kernels.h) for plain scores.
#include "fq_attention_kernels.h"

namespace fq {

// `length`: of the longest sequence, `seen` of its tokens at most by a row's tile (fewer with a window).  The workspace is that of seen == length: with fewer the
// launch needs as much or less.
AttnPlan attention_plan(int64_t B, int64_t T, int H, int Hq, int64_t max_rows, int64_t length, int64_t seen) {
    AttnPlan plan;
    max_rows = max_rows < T ? max_rows : T;                                    // positions and rows are 32-bit numbers
    length = length < 0x7fffffff ? length : 0x7fffffff;
    seen = seen < length ? seen : length;
    const int64_t rows = max_rows * (Hq / H), pairs = B * H;
    plan.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : SH_ROWS * ATT_WAVES;
    plan.splits = 1;
    plan.chunk = 1 << 30;
    plan.waves = ATT_WAVES;
    plan.workgroups = 0;
    int64_t partials = 0;
    if (plan.tile_rows <= 32) {
        // A workgroup a pair, or balanced?  us, measured at 16 rows, u = units of 128 tokens: a pair of 8 waves takes 6 + 0.58 u, of 16 waves 8 + 0.44 u (up to one a CU),
        // the balanced launch 14 (two kernels and the cut) and what its bytes take, 0.94 u of a pair on every CU, of three quarters of the longest.
        // 1 x 32 pairs of 1000 tokens 10.7 (8 waves) / 14.6, of 4000 22.0 (16) / 14.8; 128 of 4096 22.7 / 24.7, of 16000 66 / 51; 512 of 4096 46.9 (8) / 52.
        // More pairs than two workgroups of 8 waves a CU hold: of 4 waves, three a CU, in short contexts (us, 4 / 8 waves: 520 of 300 tokens 10.6 / 12.0, of 1000 20.0 / 21.2, of
        // 2500 35 / 33, of 4000 61 / 47; 768 of 1000 21.5 / 22.6, of 4000 65 / 68; 1024 of 300 13.7 / 17.3, of 3000 62 / 66, of 4000 85 / 82; 2048 of 1000 46.5 / 54.3, of 4000
        // 155 / 147).
        // Tiles of 32 rows have workgroups of 4 waves: 7 + 1.23 u, the balanced launch 23 and 0.72 u of a pair on every CU.  20 rows, 8 heads: 1 sequence of 1000 tokens
        // 16.7 / 18.9, of 8000 83 / 24; 16 of 2000 27 / 31, of 4000 46 / 36, of 8000 85 / 47; 32 of 4000 47 / 46, of 16000 165 / 111; 48 of 4000 65 / 64, of 8000
        // 118 / 95; 64 of 8000 117 / 119; 32 rows the same within 8 %.
        const double u = (double)(seen + 127) / 128, each = u * (double)pairs / kPlanCus;
        const bool balanced = B <= kBalancedSequences;
        int waves;
        if (plan.tile_rows == 16) {
            const double pair8 = 6 + 0.58 * u, pair16 = 8 + 0.44 * u;
            waves = pairs > 2 * kPlanCus && seen < 3500 ? 4 : pairs > kPlanCus || pair8 < pair16 ? 8 : 16;
            if (balanced && pairs <= kPlanCus && 14 + 0.7 * each < (pair8 < pair16 ? pair8 : pair16)) waves = 0;
        } else {
            waves = balanced && 23 + 0.72 * each < 7 + 1.23 * u ? 0 : 4;
        }
        waves = tuned(Knob::ATT_WAVES, waves);
        if (waves == 0 && !balanced) waves = 4;
        plan.waves = waves > 4 && plan.tile_rows == 16 ? (waves > 8 ? 16 : 8) : 4;
        if (waves == 0) {
            const int per_cu = tuned(Knob::ATT_WG_PER_CU, plan.tile_rows == 16 ? 3 : 2);
            plan.workgroups = (int)kPlanCus * (per_cu < 1 ? 1 : per_cu < 8 ? per_cu : 8);
            partials = (int64_t)plan.workgroups * 2 * plan.tile_rows;
        }
    } else {
        // Eight waves convert a token for twice the rows, where they fill every CU and the tokens are many (us, 4 / 8 waves: 2 x 8192 rows of 64 heads at
        // 8192 tokens 2454 / 2260; 2048 of 64 at 2048 126 / 104; 8 x 256 of 32 at 1500 70 / 63; 8 x 1024 of 32 at 1024 88 / 93; 512 of 64 at 8192, workgroups
        // for half of the CUs, 195 / 269), and the rows are enough for them: the last tile of eight has idle waves behind its last row, the last of four takes 64 rows or
        // fewer in half the time.  (8 heads of 4 queries; 64 sequences of 13 rows at 3000 tokens 98 / 149, of 32 135 / 160; 32 of 80 at 8000 393 / 408, of 128
        // 543 / 482.)  One workgroup for each CU, all at the same time, bears half as many rows, or in a short context a quarter, which four waves would have to split
        // and join: 32 sequences of 48 rows at 3000 117 / 105, of 24 at 1500 56 / 48 and at 8000 178 / 207, of 13 at 1500 43 / 46.
        const int64_t tiles8 = (rows + 2 * plan.tile_rows - 1) / (2 * plan.tile_rows), groups8 = pairs * tiles8;
        const int64_t rest = rows % plan.tile_rows, rows4 = rows - rest + (rest > plan.tile_rows / 2 ? plan.tile_rows : rest > 0 ? plan.tile_rows / 2 : 0);
        const bool filled = tiles8 * 2 * plan.tile_rows * 8 <= rows4 * 9 ||
                            (groups8 == kPlanCus && (rows > plan.tile_rows || (rows > plan.tile_rows / 2 && seen < 3000)));
        if (tuned(Knob::ATT_WAVES, groups8 >= kPlanCus && seen >= 1280 && filled ? 8 : 4) == 8 && pairs < 1 << 23) {   // (a grid has less than 2^32 threads)
            plan.waves = 8;
            plan.tile_rows *= 2;
        }
        const int64_t tiles = (rows + plan.tile_rows - 1) / plan.tile_rows, groups = pairs * (tiles > 0 ? tiles : 1);
        int64_t splits = (2 * kPlanCus + groups - 1) / groups;
        const int64_t most = (seen + 255) / 256;                               // of no less than 256 tokens each
        splits = splits < most ? splits : most;
        splits = splits < 1 || plan.waves == 8 ? 1 : splits > kMaxSplits ? kMaxSplits : splits;
        const int64_t per = ((seen + splits - 1) / splits + 127) / 128 * 128;
        plan.chunk = per < 128 ? 128 : per > (1 << 30) ? 1 << 30 : (int)per;
        const int chunk = plan.waves == 8 ? 0 : tuned(Knob::ATT_CHUNK, 0);
        if (chunk > 0) plan.chunk = ((chunk < 1 << 30 ? chunk : 1 << 30) + 127) / 128 * 128;
        splits = chunk > 0 || splits > 1 ? (seen + plan.chunk - 1) / plan.chunk : 1;
        plan.splits = (int)(splits < 1 ? 1 : splits > kMaxSplits ? kMaxSplits : splits);
        if (plan.splits > 1) partials = T * Hq * plan.splits;
    }
    plan.stats_at = partials * ATT_D;
    plan.workspace = partials * (ATT_D + 2) * 4;
    return plan;
}

// The plan of a call: with a window, of the steps of 32 tokens around a tile's windows and the first tokens, if that needs no more workspace than the whole length, which the
// caller has for it.  With a prefix beside it rows see any number of tokens, which the device alone knows: the plan of the whole length, whose balanced launch cuts what there is,
// and whose splits the kernels lengthen from 256 tokens on.  us, 1024 tokens of window planned alone / as it is now: 1 sequence of 131072 tokens (8 x 4 heads) with a prefix of
// 100000 592 / 37, 64 rows of it 6462 / 271; with one of 5 tokens 10.6 / 18.5 and 24.5 / 25.2; 16 sequences of 8192, prefixes of 6000 47.4 / 38.9, of 5 11.4 / 12.5.
AttnPlan attention_plan_window(int64_t B, int64_t T, int H, int Hq, int64_t max_rows, int64_t length, int window, int sinks, bool prefix) {
    AttnPlan plan = attention_plan(B, T, H, Hq, max_rows, length, length);
    if (window <= 0) return plan;
    if (!prefix) {
        const AttnPlan fewer = attention_plan(B, T, H, Hq, max_rows, length, (int64_t)window + sinks + max_rows + 64);
        return fewer.workspace <= plan.workspace ? fewer : plan;
    }
    if (plan.splits > 1 && plan.chunk > 256 && tuned(Knob::ATT_CHUNK, 0) <= 0) plan.chunk = 256;
    return plan;
}

hipError_t attention_launch(const CacheDev& c, const AttnArgs& a, const AttnPlan& plan, hipStream_t stream) {
    AttnDev d;
    fill_attention(d, c, a, plan);
    return attention_launch_any(d, plan, a.max_rows, stream);
}

}  // namespace fq
