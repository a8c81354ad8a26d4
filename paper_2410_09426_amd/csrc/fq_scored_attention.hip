// Attention over the paged key/value cache with scores that are capped by a tanh, lowered by a distance, or seen through a prefix: the kernels of
// fq_attention_kernels.h with ScoredDev, in the launches that attention_plan chooses for plain scores.
#include "fq_attention_kernels.h"

namespace fq {

hipError_t scored_attention_launch(const CacheDev& c, const AttnArgs& a, const ScoreArgs& s, const AttnPlan& plan, hipStream_t stream) {
    constexpr float LOG2E = 1.44269504088896340736f;
    ScoredDev d;
    fill_attention(d, c, a, plan);
    // a cap below 2^-20 leaves scores that differ by less than the weights are rounded by, one beyond 2^100 is none for scores of 2^64 times a product of rows
    d.cap = s.cap > 0.0f ? __builtin_fminf(__builtin_fmaxf(s.cap * LOG2E, 0x1p-20f), 0x1p100f) : 0.0f;
    d.per_cap = s.cap > 0.0f ? 1.0f / d.cap : 0.0f;
    d.bend = s.cap <= 0.0f ? 0 : d.cap <= kLargeCap ? 1 : 2;
    d.unit = d.bend == 1 ? 2.0f * d.cap : 1.0f;
    // (held at 2^64 as for plain scores: with a cap, what differs by 2^-48 of that has reached it on one side or the other)
    if (d.bend == 1) d.scale2 = __builtin_fminf(__builtin_fmaxf(d.scale2 * (2.0f * LOG2E * d.per_cap), -0x1p64f), 0x1p64f);
    d.slopes = s.slopes;
    d.prefix = s.prefix;
    return attention_launch_any(d, plan, a.max_rows, stream);
}

}  // namespace fq
