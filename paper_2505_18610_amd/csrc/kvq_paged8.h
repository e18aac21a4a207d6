// The paged cache of 8-bit floating point (gfx950): what its kernels and its host code share.
//
// A page holds page_tokens tokens of every KV head; the codes (e4m3) of 32 tokens of one head are a K tile and a V tile of 4 KiB in the
// arrangement of kvq_layout.h for 8 bits, so that a lane's 16-byte loads are operands of the matrix cores once they have been widened.
// Keys and values of a page and head have one scale each, a power of two: a page whose largest value grows has its codes multiplied by a
// power of two, which is exact for all but the smallest of them.  The scale word holds the exponent + KVQ_P8_BIAS in its low byte and
// KVQ_P8_NAN where one of the page's codes of that head and kind may be NaN.
//
// Page tables, lengths and row numbers are device arrays that a kernel holds against the sizes that the host knows, so that one captured
// launch serves while the sequences grow: rows of a sequence beyond max_rows or beyond the tensors, tokens beyond the table and entries of
// the table that name no page do not exist.  A row is the token that the sequence's length says, whether the table has it or not.
#ifndef KVQ_PAGED8_H
#define KVQ_PAGED8_H

#include <hip/hip_runtime.h>
#include "kvq_layout.h"

#define KVQ_P8_TILE_BYTES 8192  // K tile and V tile
#define KVQ_P8_BIAS 64
#define KVQ_P8_LOW (-40)        // the smallest exponent of a scale
#define KVQ_P8_NAN 0x100
#define KVQ_P8_MOST_SEQS 4096

struct KvqP8 {
    uint8_t* codes;
    int32_t* words;
    const int32_t *table, *lengths, *row_begin;
    int64_t table_stride;
    int32_t n_pages, n_kv, page_shift, table_pages, n_seqs, n_rows, max_rows;
};

namespace kvq_p8 {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Seq {
    int32_t row0, rows, end, tokens;  // first row, rows; tokens up to and with those of the rows, and how many of them the table has
};
__device__ inline Seq seq_of(const KvqP8& P, int s) {
    Seq q;
    q.row0 = s;
    int32_t end = s + 1;
    if (P.row_begin) {
        q.row0 = min(max(P.row_begin[s], 0), P.n_rows);
        end = min(P.row_begin[s + 1], P.n_rows);
    }
    q.rows = min(max(end - q.row0, 0), P.max_rows);
    q.end = max(P.lengths[s], 0);
    q.tokens = min(q.end, P.table_pages << P.page_shift);
    return q;
}
// The page that holds page `at` of a sequence, or -1.
__device__ inline int page_of(const KvqP8& P, int s, int at) {
    if (at < 0 || at >= P.table_pages) return -1;
    const int page = P.table[s * P.table_stride + at];
    return (uint32_t)page < (uint32_t)P.n_pages ? page : -1;
}
__device__ inline uint8_t* tile_of(const KvqP8& P, int page, int kv, int tile) {
    const int per_page = 1 << (P.page_shift - 5);
    return P.codes + (((int64_t)page * P.n_kv + kv) * per_page + tile) * KVQ_P8_TILE_BYTES;
}
__device__ inline int exponent_of(int word) { return (word & 0xff) - KVQ_P8_BIAS; }

// Sums over the lanes of a wavefront up to and with each lane's own, by data-parallel moves: within rows of 16, then row by row.
__device__ inline int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
    return x;
}
__device__ inline int wave_max(int x) {  // of values of at least zero, in every lane
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(x, 63);
}

// Things counted by sequence (at most 64 x 64 sequences, the sum below 2^31), by a whole wavefront: how many
// there are, and which sequence the one with a given number belongs to.
template <class Count>
struct Census {
    const Count& count;
    int n, per, lane, mine, upto, total;
    __device__ Census(const Count& c, int n_seqs) : count(c), n(n_seqs), per((n_seqs + 63) >> 6), lane(threadIdx.x & 63), mine(0) {
        for (int k = 0; k < per; ++k) {
            const int s = lane * per + k;
            mine += s < n ? count(s) : 0;
        }
        upto = wave_scan(mine);
        total = __builtin_amdgcn_readlane(upto, 63);
    }
    // The sequence of thing p (0 <= p < total) and, in `first`, the number of the sequence's first one; -1 where counts that are asked again have
    // changed meanwhile.
    __device__ int find(int p, int& first) const {
        const int at = __builtin_ctzll(__ballot(upto > p)), before = __builtin_amdgcn_readlane(upto - mine, at);
        if (per == 1) {
            first = before;
            return at;
        }
        const int s = at * per + lane, x = lane < per && s < n ? count(s) : 0, sum = before + wave_scan(x);
        const uint64_t behind = __ballot(sum > p);
        if (!behind) return -1;
        const int k = __builtin_ctzll(behind);
        first = __builtin_amdgcn_readlane(sum - x, k);
        return at * per + k;
    }
};

// What an fp16 output takes of a value: a rounded code may lie beyond the largest one.  NaN stays.
__device__ inline float half_range(float x) { return fabsf(x) > 65504.f ? copysignf(65504.f, x) : x; }

// Whether the sequences have no more rows together than the tensors (row numbers that fall can have it otherwise).
__device__ inline bool rows_fit(const KvqP8& P) {
    const int lane = threadIdx.x & 63, per = (P.n_seqs + 63) >> 6;
    int mine = 0;  // (64 times n_rows are within 32 bits)
    for (int k = 0; k < per; ++k)
        if (lane * per + k < P.n_seqs) mine += seq_of(P, lane * per + k).rows;
    return !__ballot(mine > P.n_rows) && __builtin_amdgcn_readlane(wave_scan(min(mine, P.n_rows)), 63) <= P.n_rows;
}

// On from sequence s, whose first thing has the number `first` <= p, to the sequence of thing p; false where there is none (any more).
template <class Count>
__device__ inline bool walk(const Count& count, int n, int p, int& s, int& first) {
    for (;;) {
        const int things = count(s);
        if (p - first < things) return true;
        first += things;
        if (++s >= n) return false;
    }
}

// A unit's pieces are joined level by level, width = 1, 2, 4, ...: of two neighbours whoever finds the other's results stored joins them and goes on
// as the first.  A level's answer goes through a word of LDS of its own: a piece without a neighbour at a level passes it without a barrier, so
// that at the next one slower wavefronts may still be reading the word of the level before.
constexpr int kJoinLevels = 8;  // of at most 256 pieces
KVQ_HD int join_other(int at, int width) { return at ^ width; }
KVQ_HD int join_word(int level) { return level; }

}  // namespace kvq_p8

#endif
