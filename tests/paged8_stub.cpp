// What the kernels of the paged cache of 8-bit floating point work out from device arrays (paper_2505_18610_amd/csrc/kvq_paged8.h), on the CPU.
// tests/test_paged8_stub.py builds it with sanitizers; argument: the scenario.  Exit code 0 = pass.  No GPU and no HIP library is involved.
#include <algorithm>
#include <barrier>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <random>
#include <set>
#include <string>
#include <thread>
#include <vector>

using std::max;
using std::min;

// ---- A wavefront: 64 threads, and what its lanes tell one another
struct Dim {
    unsigned x;
};
thread_local Dim threadIdx;
std::barrier<> lanes(64);
int told[64];
template <class F>
auto tell(int x, F f) {
    told[threadIdx.x] = x;
    lanes.arrive_and_wait();
    const auto y = f();
    lanes.arrive_and_wait();
    return y;
}
inline int dpp(int old, int x, int ctrl, int rows, int, bool) {
    return tell(x, [&] {
        const int lane = threadIdx.x, row = lane >> 4, shift = ctrl & 15;
        if (!(rows >> row & 1)) return old;
        if (ctrl > 0x110 && ctrl < 0x120) return (lane & 15) >= shift ? told[lane - shift] : old;  // row_shr
        if (ctrl == 0x142) return row ? told[16 * row - 1] : old;                                  // row_bcast:15
        if (ctrl == 0x143) return row >= 2 ? told[31] : old;                                       // row_bcast:31
        abort();
    });
}
inline int readlane(int x, int lane) {
    return tell(x, [&] { return told[lane & 63]; });
}
inline uint64_t ballot(bool x) {
    return tell(x, [&] {
        uint64_t bits = 0;
        for (int i = 0; i < 64; ++i) bits |= (uint64_t)(told[i] != 0) << i;
        return bits;
    });
}
template <class F>
void wavefront(F f) {
    std::vector<std::thread> threads;
    for (unsigned i = 0; i < 64; ++i)
        threads.emplace_back([i, &f] {
            threadIdx.x = i;
            f((int)i);
        });
    for (auto& t : threads) t.join();
}
#define __builtin_amdgcn_update_dpp dpp
#define __builtin_amdgcn_readlane readlane
#define __ballot ballot
#include "../paper_2505_18610_amd/csrc/kvq_paged8.h"

namespace {

int failures = 0;
#define CHECK(cond, ...)                                                                                                        \
    do {                                                                                                                        \
        if (!(cond) && ++failures < 20) { printf("line %d: %s: ", __LINE__, #cond); printf(__VA_ARGS__); printf("\n"); fflush(stdout); } \
    } while (0)

// ---- The join of a unit's pieces, in any order of arrival.  At each level a workgroup writes the word that `word` says and all its wavefronts read it
// behind a barrier; the next barrier is that of the next level that has a neighbour: whether its word is that of the level before says
// whether a slower wavefront's read can meet the write.
int joins_on_a_word_still_read(int pieces, const std::function<int(int)>& word, std::mt19937& rng) {
    using namespace kvq_p8;
    int bad = 0;
    std::vector<int> order(pieces), stored(pieces, 0);
    std::vector<std::set<int>> holds(pieces);
    std::set<int> counters;
    for (int p = 0; p < pieces; ++p) order[p] = p, holds[p] = {p};
    std::shuffle(order.begin(), order.end(), rng);
    int whole = 0;
    for (int piece : order) {
        std::set<int> mine = {piece};
        bool go_on = true;
        int last = -1;
        for (int width = 1, at = piece, level = 0; go_on && width < pieces; width *= 2, ++level) {
            const int other = join_other(at, width), begin = min(at, other), second = max(at, other);
            if (second >= pieces) continue;
            const int w = word(level);
            CHECK(w >= 0 && w < kJoinLevels && level < kJoinLevels, "word %d at level %d of %d pieces", w, level, pieces);
            bad += w == last;
            last = w;
            if (stored[second] == 0) {  // the first of the two: its results stay in its slot
                stored[second] = 1;
                holds[at] = mine;
                go_on = false;
            } else {  // a pair's counter is its second half's: of one level only
                CHECK(stored[second] == 1 && counters.insert(second).second, "the counter of piece %d of %d twice", second, pieces);
                stored[second] = 2;
                for (int p : holds[other]) CHECK(mine.insert(p).second, "piece %d of %d twice", p, pieces);
            }
            at = begin;
        }
        if (go_on) {
            ++whole;
            CHECK((int)mine.size() == pieces, "%d of %d pieces", (int)mine.size(), pieces);
        }
    }
    CHECK(whole == 1, "%d results of %d pieces", whole, pieces);
    return bad;
}
void join() {
    std::mt19937 rng(1);
    std::set<int> alternating;
    for (int pieces = 1; pieces <= 256; ++pieces)
        for (int turn = 0; turn < 20; ++turn) {
            CHECK(joins_on_a_word_still_read(pieces, kvq_p8::join_word, rng) == 0, "%d pieces", pieces);
            if (joins_on_a_word_still_read(pieces, [](int level) { return level & 1; }, rng)) alternating.insert(pieces);
        }
    // (two words in turn would not do: levels are passed without a barrier)
    for (int pieces : {6, 11, 12, 14}) CHECK(alternating.count(pieces), "%d pieces, two words", pieces);
}

// ---- Which sequence a thing belongs to, also where the counts change between two readings
void lookup() {
    std::mt19937 rng(2);
    const auto upto = [&](int n) { return (int)(rng() % n); };
    for (int n : {1, 2, 63, 64, 65, 128, 300, 1000, 4096}) {
        std::vector<int> now(n);
        for (int& x : now) x = upto(3) ? upto(9) : 0;
        now[upto(n)] = 40;
        std::vector<int> starts;
        for (int s = 0, at = 0; s < n; at += now[s++]) starts.push_back(at);
        const int total = starts[n - 1] + now[n - 1];
        const std::vector<int> before = now;
        std::vector<int> things = {0, total - 1};
        for (int i = 0; i < 12; ++i) things.push_back(upto(total));
        std::vector<std::vector<int>> after;
        after.push_back(std::vector<int>(n, 0));  // all gone; some fewer; more
        after.push_back(before);
        for (int& x : after.back()) x = x && upto(2) ? x - 1 : x;
        after.push_back(before);
        for (int& x : after.back()) x += upto(4);
        wavefront([&](int lane) {
            const auto count = [&](int s) { return now.at(s); };
            const kvq_p8::Census<decltype(count)> census(count, n);
            if (lane == 0) CHECK(census.total == total, "%d of %d things", census.total, total);
            for (int p : things) {
                int first;
                const int s = census.find(p, first);
                if (lane == 0) CHECK(s >= 0 && s < n && first == starts[s] && p < first + before[s], "thing %d of %d: sequence %d of %d", p, total, s, n);
                for (int q : {p, min(total - 1, p + 1), total - 1}) {
                    int t = s, at = first;
                    const bool there = kvq_p8::walk(count, n, q, t, at);
                    if (lane == 0) CHECK(there && t < n && at == starts[t] && q < at + before[t], "thing %d from sequence %d", q, s);
                }
            }
            for (const auto& changed : after) {
                lanes.arrive_and_wait();
                if (lane == 0) now = changed;
                lanes.arrive_and_wait();
                for (int p : things) {
                    int first = 0;
                    const int s = census.find(p, first);
                    if (lane == 0) CHECK(s >= -1 && s < n, "sequence %d of %d", s, n);
                    if (s < 0) continue;
                    if (lane == 0) CHECK(first >= 0 && first <= p, "first %d of thing %d", first, p);
                    int t = s, at = first;
                    const bool there = kvq_p8::walk(count, n, total - 1, t, at);  // (counts are read with their bounds checked)
                    if (lane == 0 && there) CHECK(t < n && at <= total - 1 && total - 1 < at + now[t], "thing %d: sequence %d", total - 1, t);
                }
            }
        });
    }
}

// ---- Whether rows are no more than the tensors have, also where row numbers fall, up to the largest that there can be
void rows() {
    std::mt19937 rng(3);
    const auto upto = [&](int64_t n) { return (int32_t)(rng() % n); };
    for (int n : {1, 5, 64, 65, 4096})
        for (int n_rows : {1, 77, 100000, INT32_MAX / 64})
            for (int kind = 0; kind < 4; ++kind) {
                std::vector<int32_t> begin(n + 1), lengths(n, 5), table(n, 0);
                for (int32_t& b : begin) b = upto((int64_t)n_rows + 1);
                if (kind < 2) std::sort(begin.begin(), begin.end());
                if (kind == 1) begin[0] = -7, begin[n] = INT32_MAX;
                if (kind == 3)
                    for (int s = 0; s <= n; ++s) begin[s] = s & 1 ? n_rows : 0;
                KvqP8 P{nullptr, nullptr, table.data(), lengths.data(), begin.data(), 1, 1, 1, 5, 1, n, n_rows, kind == 1 ? max(1, n_rows / 2) : n_rows};
                int64_t all = 0;
                for (int s = 0; s < n; ++s) all += kvq_p8::seq_of(P, s).rows;
                wavefront([&](int lane) {
                    const bool fit = kvq_p8::rows_fit(P);
                    if (lane == 0) CHECK(fit == (all <= n_rows), "%lld of %d rows, %d sequences", (long long)all, n_rows, n);
                });
                CHECK(kind >= 2 || all <= n_rows, "%lld of %d rows", (long long)all, n_rows);
            }
}

}  // namespace

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "join") join();
    else if (what == "lookup") lookup();
    else if (what == "rows") rows();
    else return 2;
    if (failures) printf("%d failures\n", failures);
    else printf("ok\n");
    return failures ? 1 : 0;
}
