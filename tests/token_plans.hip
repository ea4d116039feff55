// Checks of the host side's plans of the operators for token models, on the CPU (no kernel is launched): built and run by test_token_plans_host.py, once for each
// of the two sources.  Prints what is wrong and returns 1, or "ok".
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <random>
#include <set>
#include <vector>
#ifdef PLANS_OF_ATTENTION
#include "../paper_2605_24584_amd/csrc/attention_kernels.hip"
#else
#include "../paper_2605_24584_amd/csrc/logprob_kernels.hip"
#endif

namespace laplex {
void profile_before(const char*, hipStream_t) {}
void profile_after(const char*, hipStream_t) {}
}  // namespace laplex

using namespace laplex;

static std::mt19937_64 rng(1);
static int64_t any(double lo, double hi) { return (int64_t)std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi + 0.9))(rng)); }

#define REQUIRE(what, ...)                                        \
    do {                                                          \
        if (!(what)) { printf(#what ": " __VA_ARGS__); puts(""); return 1; } \
    } while (0)

#ifdef PLANS_OF_ATTENTION

// The workspace that is asked for holds the states of every plan, and serves smaller calls.
static int workspaces()
{
    for (int n = 0; n < 300000; ++n) {
        int64_t tokens = any(1, 33554432), sequences = any(1, 1048576);
        const int heads = (int)any(1, n % 9 ? 64 : 65535), dk = 1 + rng() % 256, dv = 1 + rng() % 256;
        if (n % 3 == 0) tokens = tokens / sequences * sequences;
        if (n % 5 == 0) tokens = std::max<int64_t>(1, tokens / 64) * 64 + (int)(rng() % 3) - 1;
        tokens = std::min<int64_t>(tokens, 33554432);
        const size_t have = attention_workspace(tokens, sequences, heads, dk, dv);
        for (int i = 0; i < 8; ++i) {
            const int walks = i & 1 ? 3 : 1;
            const bool equal = i & 2, bf16 = i & 4;
            if (equal && tokens % sequences) continue;
            const Plan P = plan_of(bf16, tokens, sequences, heads, dk, dv, walks, equal);
            const size_t need = P.cut ? (size_t)(walks > 1 ? 2 : 1) * P.places * heads * P.slices * P.dk * P.cols * sizeof(float) : 0;
            REQUIRE(need <= have, "%ld tokens, %ld sequences, %d heads, %d, %d: %zu of %zu", (long)tokens, (long)sequences, heads, dk, dv, need, have);
            REQUIRE(!P.cut || P.places > 0, "%ld tokens", (long)tokens);
            REQUIRE(P.cut || P.stretch >= (equal ? tokens / sequences : tokens), "%ld tokens", (long)tokens);
        }
        const int64_t fewer_tokens = tokens - any(1, std::max<double>(1, tokens)), fewer = std::max<int64_t>(0, sequences - any(1, sequences));
        REQUIRE(attention_workspace(std::max<int64_t>(0, fewer_tokens), fewer, heads, dk, dv) <= have, "%ld tokens", (long)tokens);
        REQUIRE(attention_workspace(std::max<int64_t>(0, fewer_tokens), sequences, heads, dk, dv) <= have, "%ld tokens", (long)tokens);
    }
    return 0;
}

// The numbering of the places, as the kernels have it: no two stretches share one, none lies outside, also where starts are garbage.
static int places()
{
    for (int n = 0; n < 20000; ++n) {
        const int64_t stretch = 64 * (1 + rng() % 4), sequences = 1 + rng() % 60, tokens = 1 + rng() % 3000;
        std::vector<int64_t> starts(sequences + 1);
        const bool garbage = n % 4 == 0;
        for (auto& v : starts) v = garbage ? (int64_t)(rng() % 6000) - 1500 : (int64_t)(rng() % (tokens + 1));
        if (!garbage) std::sort(starts.begin(), starts.end());
        const auto start = [&](int64_t b) { return std::min(std::max<int64_t>(starts[b], 0), tokens); };
        const auto first = [&](int64_t b) { return start(b) / stretch + std::min(b, start(b) / (stretch + 1)); };
        const int64_t most = tokens / stretch + std::min(sequences, tokens / (stretch + 1));
        std::set<int64_t> taken;
        for (int64_t b = 0; b < sequences; ++b) {
            const int64_t count = std::max<int64_t>(0, start(b + 1) - start(b));
            for (int64_t i = 0; count > stretch && i < (count + stretch - 1) / stretch; ++i) {
                REQUIRE(first(b) + i >= 0 && first(b) + i < most, "sequence %ld", (long)b);
                REQUIRE(taken.insert(first(b) + i).second || garbage, "sequence %ld", (long)b);
            }
        }
        // the search from a place finds the sequence that it belongs to
        for (int64_t b = 0; b < sequences && !garbage; ++b) {
            const int64_t count = start(b + 1) - start(b);
            for (int64_t i = 0; count > stretch && i < (count + stretch - 1) / stretch; ++i) {
                int64_t last = 0;
                for (int64_t c = 0; c < sequences; ++c)
                    if (first(c) <= first(b) + i) last = c;
                REQUIRE(last == b, "sequence %ld", (long)b);
            }
        }
    }
    return 0;
}

int main() { return workspaces() || places() || !puts("ok"); }

#else

// Every row and column is in some workgroup's share, and no workgroup is without any.
static int shapes()
{
    for (int n = 0; n < 1000000; ++n) {
        const int64_t k = any(1, 4294967294.0), batch = any(1, 33554432);
        for (int back = 0; back < 2; ++back) {
            const Shape S = back ? shape_of(k, batch, kBackRows, kBackTarget, false) : shape_of(k, batch, kGroup, kRowsTarget, true);
            const int64_t row_lanes = (back ? kRowThreads : S.threads) >> S.lanes_log2, rows = back ? kBackRows : kGroup;      // (what the gradient is launched with)
            const __int128 turn = (__int128)S.turns * row_lanes * rows;
            REQUIRE(S.blocks * turn >= k && (S.blocks - 1) * turn < k, "%ld x %ld, gradient %d: %ld workgroups", (long)k, (long)batch, back, (long)S.blocks);
            REQUIRE((S.slabs << S.lanes_log2) * S.vec >= batch, "%ld x %ld", (long)k, (long)batch);
            REQUIRE(S.slabs * S.blocks * (int64_t)S.threads < (int64_t(1) << 32) - (int64_t(1) << 30), "%ld x %ld", (long)k, (long)batch);
        }
    }
    return 0;
}

int main() { return shapes() || !puts("ok"); }

#endif
