// The host's picture of a cache (struct kvq_cache) and what the host translation units share of it: kvq_host.cpp keeps the
// books, kvq_tree.hip and kvq_moves.hip read and change them for their entry points.
#ifndef KVQ_CACHE_H
#define KVQ_CACHE_H

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <vector>

#include "../../include/kvq.h"
#include "kvq_internal.h"
#include "kvq_ring.h"

namespace kvq_host {

constexpr int kMaxOrder = 4;  // allocation blocks of 1, 2, 4, 8, 16 units; a unit is one metadata block
constexpr int kRingSegments = 4;
constexpr uint64_t kRingSegmentBytes = 1u << 20;  // the pinned staging ring: 4 segments of 1 MiB
constexpr uint64_t kNoSum = 0x7ff0dead0000beefull;  // a signalling NaN

// Markers of the staging ring: one HIP event per segment, recorded on the cache's stream.
struct RingEvents {
    hipEvent_t ev[kRingSegments] = {};
    hipStream_t stream = nullptr;
    bool record(int i) { return hipEventRecord(ev[i], stream) == hipSuccess; }
    bool wait(int i) { return hipEventSynchronize(ev[i]) == hipSuccess; }
};

inline int order_of_bits(int bits) { return bits == 16 ? 4 : bits == 8 ? 3 : bits == 4 ? 2 : 1; }
// Kernel time of one 2/4/8/16-bit tile, measured, in units of which a workgroup does 1,000 in 0.9 us.
constexpr int kTileTime[4] = {100, 145, 250, 300};
inline bool valid_bits(int b) { return b == 16 || b == 8 || b == 4 || b == 2; }

// A set of numbers below n that finds its smallest: a bit for each, and a bit per word of the level below on the levels above.
class NumberSet {
public:
    bool init(uint64_t n, bool full) {
        levels_.clear();
        for (uint64_t bits = n;;) {
            const uint64_t words = std::max<uint64_t>(1, (bits + 63) / 64);
            levels_.emplace_back(static_cast<uint64_t*>(std::calloc(words, sizeof(uint64_t))));  // (pages of zeros cost nothing until written)
            if (!levels_.back()) return false;
            if (full) {
                std::memset(levels_.back().get(), 0xff, (size_t)(bits / 64) * sizeof(uint64_t));
                if (bits % 64) levels_.back()[(size_t)(bits / 64)] = (1ull << (bits % 64)) - 1;
            }
            if (words == 1) return true;
            bits = words;
        }
    }
    bool empty() const { return levels_.back()[0] == 0; }
    uint32_t smallest() const {
        uint64_t i = 0;
        for (size_t l = levels_.size(); l-- > 0;) i = i * 64 + (uint64_t)__builtin_ctzll(levels_[l][i]);
        return (uint32_t)i;
    }
    bool has(uint32_t i) const { return levels_[0][i / 64] >> (i % 64) & 1; }
    void add(uint32_t i) {
        for (auto& words : levels_) {
            const uint64_t old = words[i / 64];
            words[i / 64] = old | 1ull << (i % 64);
            if (old) return;
            i /= 64;
        }
    }
    void remove(uint32_t i) {
        for (auto& words : levels_) {
            if (words[i / 64] &= ~(1ull << (i % 64))) return;
            i /= 64;
        }
    }

private:
    struct Free { void operator()(uint64_t* p) const { std::free(p); } };
    std::vector<std::unique_ptr<uint64_t[], Free>> levels_;
};

// Buddy allocator in units.  Code blocks need 2^order units (2-bit: 2, 4-bit: 4, 8-bit: 8, 16-bit: 16),
// metadata blocks one unit, so every size is a power of two and freed space coalesces without compaction.
// (With the free blocks in std::set a prompt of 16,000 tokens that is shrunk twice spent 55 of the host's 137 us here, and more than a
// launch takes on most calls.)
class Buddy {
public:
    bool init(uint32_t n_super) {
        for (int o = 0; o <= kMaxOrder; ++o)
            if (!free_[o].init((uint64_t)n_super << (kMaxOrder - o), o == kMaxOrder)) return false;
        free_units_ = (uint64_t)n_super << kMaxOrder;
        return true;
    }
    bool alloc(int order, uint32_t* off) {
        int o = order;
        while (o <= kMaxOrder && free_[o].empty()) ++o;
        if (o > kMaxOrder) return false;
        uint32_t blk = free_[o].smallest();
        free_[o].remove(blk);
        blk <<= o;
        while (o > order) {
            --o;
            free_[o].add((blk >> o) + 1);
        }
        free_units_ -= 1u << order;
        *off = blk;
        return true;
    }
    void release(uint32_t off, int order) {
        free_units_ += 1u << order;
        uint32_t blk = off >> order;
        while (order < kMaxOrder && free_[order].has(blk ^ 1)) {
            free_[order].remove(blk ^ 1);
            blk >>= 1;
            ++order;
        }
        free_[order].add(blk);
    }
    uint64_t free_units() const { return free_units_; }

private:
    NumberSet free_[kMaxOrder + 1];
    uint64_t free_units_ = 0;
};

struct Page {
    int bits = 16;
    int n = 0;              // tokens stored
    uint32_t code_unit = 0; // allocation offsets in units
    uint32_t meta_unit = 0; // valid when the page has metadata (bits < 16, or the integer 16-bit tier)
};

struct Run {  // neighbouring pages of one width
    int page_end, bits;
};

struct Layer {
    uint64_t budget = 0;
    int fbit = 2;
    int T = 0;
    bool reparam = false;  // keys stored as K / lambda, queries multiplied by lambda (Sec. 3.3)
    bool poisoned = false; // an enqueue failed after the host tables had been updated: unusable until kvq_cache_reset
    std::vector<Page> pages;
    int resumed = -1;      // the page inside which a fork or a cut has ended; see plan_append
    // the pages as runs of one width, of the state runs_version; see runs_of
    mutable std::vector<Run> runs;
    mutable uint64_t runs_version = ~0ull;
    // what the split count was worked out from and the count itself; split plan cache of kvq_decode_attention
    uint64_t count_key[3] = {};
    int count_splits = 1;
    int plan_tiles = -1, plan_splits = 0;
    bool plan_side_by_side = false;
    uint64_t version = 0, plan_version = ~0ull;
    int32_t split_begin[KVQ_MAX_SPLITS + 1];
};

}  // namespace kvq_host

struct kvq_cache {
    kvq_config_t cfg;
    int units = 0, tpp = 0, gqa = 0, max_pages = 0;
    bool dry = false;
    uint8_t* arena = nullptr;
    uint64_t arena_bytes = 0;
    uint64_t unit_bytes = 0;
    uint64_t table_off = 0, jobs_off = 0, part_o_off = 0, part_ml_off = 0, counters_off = 0, flags_off = 0, pages_off = 0;
    uint64_t reparam_off = 0;  // per block: lambda [n_kv_heads][128] fp32, then 1 / lambda
    uint32_t v_epoch = 4;      // see KvqVMark; 0 is what a cleared word holds
    uint32_t v_turn = 1;       // tag of the next launch that appends below 16 bits, above the epoch; see kvq_v_marked
    KvqVMark v_mark() const { return KvqVMark{reinterpret_cast<uint32_t*>(arena + flags_off), v_epoch}; }
    kvq_host::Buddy buddy;
    std::vector<kvq_host::Layer> layers;
    uint8_t* ring = nullptr;
    uint8_t* ring_dev = nullptr;  // the same pinned memory as the device addresses it
    KvqStagingRing<kvq_host::RingEvents, kvq_host::kRingSegments> ring_ctl;
    kvq_host::RingEvents ring_events;
    uint64_t* sums = nullptr;   // behind the ring: 2 sums for each workgroup of the error kernel, kNoSum between calls
    bool sums_at_rest = false;
    bool device_ready = false;
    bool enqueue_failed = false;  // a block was left unusable since the device's counters were last cleared
    int splits_override = 0;
    int fused_merge = 1;
    int deterministic = 0;
    int shift_strategy = KVQ_SHIFT_EQUIVALENT;  // how 2b -> b steps treat codes, S and Z (Sec. 4.3.1)
    int tier16 = KVQ_TIER16_FP16;               // what a 16-bit token is: raw fp16, or 16-bit codes with (S, Z)
    bool int16() const { return tier16 == KVQ_TIER16_INT16; }
    bool has_meta(int bits) const { return bits < 16 || int16(); }
    int tile_cost[4] = {kvq_host::kTileTime[0], kvq_host::kTileTime[1], kvq_host::kTileTime[2], kvq_host::kTileTime[3]};  // KVQ_OPT_TILE_COST_*
    int target_workgroups = 256;

    uint64_t bpth(int bits) const {
        return kvq_bytes_per_token_head(bits, cfg.head_dim, cfg.group, cfg.count_metadata_in_budget, int16() ? 1 : 0);
    }
    uint64_t unit_off_bytes(uint32_t unit) const { return pages_off + (uint64_t)unit * unit_bytes; }
    KvqPageDesc desc(const kvq_host::Page& p) const {
        KvqPageDesc d;
        d.code_off256 = (uint32_t)(unit_off_bytes(p.code_unit) / 256);
        d.meta_off256 = has_meta(p.bits) ? (uint32_t)(unit_off_bytes(p.meta_unit) / 256) : 0u;
        d.bits = (uint32_t)p.bits;
        d.int16 = (p.bits == 16 && int16()) ? 1u : 0u;
        return d;
    }
    float* lambda_dev(int layer) const {  // lambda of the block; its reciprocals follow
        return reinterpret_cast<float*>(arena + reparam_off) + (size_t)layer * 2 * cfg.n_kv_heads * KVQ_D;
    }
    KvqPageDesc* table_dev(int layer) const {
        return reinterpret_cast<KvqPageDesc*>(arena + table_off) + (size_t)layer * max_pages;
    }
};

namespace kvq_host {

// Whether tokens enter at 16 bits by the policy, whatever the block's width.
inline bool appends_at_16(const kvq_cache* c) { return c->cfg.policy == KVQ_POLICY_OLDEST_FIRST || c->cfg.window > 0; }
inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }
// kvq_host.cpp
kvq_status_t upload(kvq_cache* c, void* dst_dev, const void* src, uint64_t bytes, hipStream_t s);
kvq_status_t ensure_device(kvq_cache* c, hipStream_t s);
uint64_t bytes_used(const kvq_cache* c, const Layer& L);
void empty_block(kvq_cache* c, Layer& L);
void start_over_if_empty(kvq_cache* c);

}  // namespace kvq_host

#endif
