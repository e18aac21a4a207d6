// Attention over the paged cache of 8-bit floating point, of single tokens, drafted tokens and chunks of prompts in one ragged call, with
// one softmax map or with the difference of two (kvq_paged8_attention, kvq_paged8_diff_attention).
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/kvq.h"
#include "kvq_flash.h"
#include "kvq_paged8.h"
#include "kvq_paged8_host.h"

namespace {

using namespace kvq_p8;
using kvq_flash::half8;
using kvq_flash::half2v;
using kvq_flash::float4v;
using kvq_flash::mma;
using kvq_flash::State;
using kvq_flash::quarters_sum;
using kvq_flash::reference_of;
using kvq_flash::softmax_group;
using kvq_flash::to_half8;

#define KVQ_P8_GROUPS 512        // pieces of 16 rows that units are cut into where they are few: two workgroups a compute unit (384 and 768 pieces: 4 x
                                 // 32,768 tokens 53.3 and 55.7 us, 512 49.3).  Of 32 rows half as many, whose workgroups have a compute unit each:
                                 // 32 sequences of 8 rows x 32 heads over 2,000 tokens 27.4 us, with 384 39.0, with 512 40.6.
#define KVQ_P8_COUNTER_STRIDE 16 // words: a line for each arrival counter
#define KVQ_P8_LEAST_SHARE 8     // tiles of a piece, at least: one for each wavefront
#define KVQ_P8_WHOLE 16          // tiles of units that are not cut: a second round takes 0.6 us, joining 1.7 (300 tokens 8.3 -> 7.2 us)
#define KVQ_P8_MANY_SHARE 24     // tiles of a piece where units are many, at least (264 units of 22 to 32 tiles 19.4 -> 15.9 us)
#define KVQ_P8_MOST_PIECES 128   // of a unit
#define KVQ_P8_ROOT 0.7f         // tiles of a piece by the root of the longest unit's, at least: more pieces take longer to join than they save
                                 // (0.5, 0.7, 0.9: 18,547 tokens with two maps 23.9, 21.9, 20.8 us, four sequences of up to 81,508 25.9, 25.1, 25.9)
#define KVQ_P8_CHUNK_GROUPS 256  // workgroups of a launch over chunks, at most: one a compute unit
#define KVQ_P8_LEAST_CHUNK 16    // tiles of a workgroup with a chunk, at least
#define KVQ_P8_MAP_BYTES 17408   // partial results of a wavefront with a chunk and one map
// Calls in which chunks are taken like few rows: units of 32 rows and their tiles, at most (200 rows x 16 heads with two maps over 4,000 tokens 68 -> 38 us;
// with more tiles twelve sequences of 32 rows x 32 heads over 4,000 60 -> 80).
#define KVQ_P8_SMALL_UNITS 512
#define KVQ_P8_SMALL_TILES 40000

struct AttnArgs {
    KvqP8 p;
    const _Float16* q;
    void* out;
    float* lse;
    const float *lambda, *weight;  // two maps: a factor for each head; weights of the norm or NULL
    uint32_t* counters;
    float* part;
    int64_t q_rs, q_hs, o_rs, o_hs, lse_hs;
    int32_t gqa, maps, out_fp32;   // gqa: query heads of a KV head
    int32_t few_rows;              // sequences with more flat rows (of one map) are chunks, unless the call is small
    int32_t packed;                // the line of all chunks was measured for n_rows rows in all, not for max_rows of every sequence
    float scale_log2, eps, out_scale;
    uint32_t flip;                 // sign bits to turn over in the queries (a negative scale)
};

// Tokens that row i of a sequence's rows sees: up to and with its own, of those that the table has.
__device__ inline int sees(const Seq& q, int i) { return min(q.tokens, max(0, q.end - q.rows + i + 1)); }

// A value that the compiler takes for a new one: what follows from it is worked out where it is used, not kept in registers through a loop.
__device__ inline int opaque(int x) {
    asm volatile("" : "+v"(x));
    return x;
}
// A lane's eight codes of one operand, widened: exact but for values below 2^-21, which keep the 2^-25 that fp16 has there.
__device__ inline half8 widen(uint32_t lo, uint32_t hi, float scale) {
    const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
    const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
    return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// What a raw score times gives its place in the softmax, in log2 units (kept from zero and infinity, which would make NaN of masked scores).
__device__ inline float score_factor(float scale_log2, int word) {
    return fminf(fmaxf(ldexpf(scale_log2, exponent_of(word)), 0x1p-126f), 0x1p126f);
}
// Values of a page are taken times 2^(6 - behind) times their code, where `behind` is how far the page's exponent lies behind the largest, `top`, that the
// wavefront or workgroup has come to (scale words' low bytes); accumulators stand for 2^(top - KVQ_P8_BIAS - 6) and follow when it grows.  448 2^6 is within
// fp16, and what fp16 rounds away at its small end, 2^-25, is 2^-38 of that page's largest value (with values as they are, halved, those
// below 2^-20 lost bits and 2^-24 all of them).
__device__ inline float value_scale(int behind) { return __builtin_ldexpf(64.f, -behind); }
__device__ inline float value_unit(int top) { return __builtin_ldexpf(1.f, top - KVQ_P8_BIAS - 6); }

// What NaN codes among a lane's eight of one V operand, of tokens token, token + 1, ..., add to a row that sees those below limit; the codes
// become zeros.
__device__ inline float4v nan_codes(uint32_t (&w)[2], int token, int limit) {
    half8 nan, sees;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int at = 8 * (e & 3);
        const bool is = ((w[e >> 2] >> at) & 0x7fu) == 0x7fu;
        sees[e] = token + e < limit ? (_Float16)1.f : (_Float16)0.f;
        nan[e] = is ? (_Float16)1.f : (_Float16)0.f;
        if (is) w[e >> 2] &= ~(0xffu << at);
    }
    const float4v count = mma(nan, sees, float4v{0.f, 0.f, 0.f, 0.f});
    float4v x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = count[i] > 0.f ? __builtin_nanf("") : 0.f;
    return x;
}

// A unit: the rows of one block of one KV head of one sequence.  Rows follow one another token by token, of a token head by head, of a head
// map by map; a block has 16 R of them.  Units of many tiles are cut into pieces of `share` tiles at most, one workgroup each: where the units
// are fewer than the workgroups that the device takes at a time, of the smallest share that leaves no more pieces than those (a workgroup that came
// behind them would have the device for itself; twice or three times as many are slower throughout), else of what an equal share of all tiles is, short units behind long pieces as workgroups end.
// Calls in which sequences of many rows are taken like those of few: what they would be joined by costs more than their larger blocks save.
__device__ inline bool small_call(int units, int tiles) { return units <= KVQ_P8_SMALL_UNITS && tiles <= KVQ_P8_SMALL_TILES; }
// What a sequence adds to either number: no more than is too many, so that the sums of 4,096 sequences stay within 32 bits.
__device__ inline int small_units(int units) { return min(units, KVQ_P8_SMALL_UNITS + 1); }
__device__ inline int small_tiles(int units, int tiles) { return min(small_units(units) * min(tiles, KVQ_P8_SMALL_TILES + 1), KVQ_P8_SMALL_TILES + 1); }
// Whether units are cut into no more pieces than the device takes at a time (200 units of 125 tiles 50 -> 38 us; up to half as many before).
__host__ __device__ inline bool few_units(int64_t units, int64_t at_a_time) { return units <= at_a_time - (at_a_time >> 4); }
struct Piece {
    int seq, unit, tiles, pieces, piece;
    int slot;  // of the unit's first piece among those of all units that are cut
};
struct Cuts {
    struct Shape { int tiles, units, few; };  // few: 1 where the sequence has few rows
    const Shape* all;  // of all sequences, where they are more than lanes
    Shape mine;
    bool small;
    int n, per, lane, share;

    // over this lane's sequences
    template <class F>
    __device__ int sum(F f) const {
        const auto part = [&](Shape x) { return f(Shape{x.tiles, small || x.few ? x.units : 0, 0}); };  // without what is another kernel's
        if (per == 1) return part(mine);
        int x = 0;
        for (int k = 0; k < per; ++k)
            if (lane * per + k < n) x += part(all[lane * per + k]);
        return x;
    }
    template <class F>
    __device__ int total(F f) const { return __builtin_amdgcn_readlane(wave_scan(sum(f)), 63); }
    __device__ int cuts_of(int tiles) const { return tiles <= KVQ_P8_WHOLE ? 1 : (uint32_t)(tiles + share - 1) / (uint32_t)share; }

    __device__ Cuts(const Shape* shapes, int n_seqs, Shape own, int lane_, int wanted) : all(shapes), mine(own), small(true), n(n_seqs), per((n_seqs + 63) >> 6), lane(lane_) {
        int units = total([](Shape x) { return small_units(x.units); }), tiles = total([](Shape x) { return small_tiles(x.units, x.tiles); });
        if (!small_call(units, tiles)) {
            small = false;
            units = total([](Shape x) { return x.units; });
            tiles = total([](Shape x) { return x.units * x.tiles; });
        }
        int longest = 0;
        sum([&](Shape x) { longest = max(longest, x.units ? x.tiles : 0); return 0; });
        longest = wave_max(longest);
        int low = max(max(KVQ_P8_LEAST_SHARE, (tiles + wanted - 1) / wanted),
                      max((longest + KVQ_P8_MOST_PIECES - 1) / KVQ_P8_MOST_PIECES, (int)(KVQ_P8_ROOT * sqrtf((float)longest))));
        const auto all_pieces = [&]() { return total([&](Shape x) { return x.units * cuts_of(x.tiles); }); };
        if (2 * units > wanted) low = max(low, KVQ_P8_MANY_SHARE);
        share = low;
        if (longest <= KVQ_P8_WHOLE || !few_units(units, wanted) || (2 * units > wanted && all_pieces() <= wanted)) return;
        int high = max(low, (tiles + wanted - units - 1) / (wanted - units));  // enough: a unit has at most one piece more than its tiles by the share
        while (high - low > low >> 4) {
            share = (low + high) >> 1;
            if (all_pieces() <= wanted) high = share;
            else low = share + 1;
        }
        share = high;
    }
    // Piece `id`, the same in all lanes.
    __device__ bool find(int id, Piece& p) const {
        const auto pieces = [&](Shape x) { return x.units * cuts_of(x.tiles); };
        const auto cut = [&](Shape x) { const int c = cuts_of(x.tiles); return c > 1 ? x.units * c : 0; };
        int x = sum(pieces), y = sum(cut), upto = wave_scan(x), cut_upto = wave_scan(y);
        uint64_t behind = __ballot(upto > id);
        if (!behind) return false;
        int at = __builtin_ctzll(behind);
        int before = __builtin_amdgcn_readlane(upto - x, at), slots = __builtin_amdgcn_readlane(cut_upto - y, at);
        Shape s = mine;
        p.seq = at;
        if (per > 1) {  // among that lane's sequences, one a lane
            const int i = at * per + lane;
            s = lane < per && i < n ? all[i] : Shape{1, 0, 0};
            if (!small && !s.few) s.units = 0;
            x = pieces(s);
            y = cut(s);
            upto = before + wave_scan(x);
            cut_upto = slots + wave_scan(y);
            at = __builtin_ctzll(__ballot(upto > id));
            before = __builtin_amdgcn_readlane(upto - x, at);
            slots = __builtin_amdgcn_readlane(cut_upto - y, at);
            p.seq = __builtin_amdgcn_readlane(i, at);
        }
        p.tiles = __builtin_amdgcn_readlane(s.tiles, at);
        p.pieces = cuts_of(p.tiles);
        p.unit = (uint32_t)(id - before) / (uint32_t)p.pieces;
        p.piece = id - before - p.unit * p.pieces;
        p.slot = slots + p.unit * p.pieces;
        return true;
    }
};

// A piece a workgroup; the pieces of a unit are joined by the last of them to arrive.  Eight wavefronts take a piece's tiles in turn, every one
// from memory straight into operand registers: nothing but the queries is shared before the end.  S^T = K q^T and O^T += V^T P^T with the rows
// in the N dimension, the reference and sums of kvq_flash.h; a scale is a power of two, K's goes to the scores, V's into the widening.
// Memory bounds it: a unit's codes are read once, 16 wavefronts of a compute unit have 128 KB on their way (R = 1, at most 128 registers, which is why the
// queries lie in LDS: 67.0 -> 54.8 us).  4 x 32,768 tokens x 40 heads 49.4 us = 5.4 TB/s, as much as a copy moves; two maps over eight sequences of up
// to 16,384 tokens 42 us = 5.0; 48 sequences of 41 to 30,000 tokens 49 us = 4.8 (107 with equal shares of all tiles over the units, as short
// units then waited for one another in one workgroup).  A short call is a chain of trips: 1,001 tokens x 8 heads 8.7 us.
// The hand-over: partial results go out with device-scope stores (sc1), a wait and a barrier stand before the arrival counter, the last to arrive reads
// them with device-scope loads and leaves the counter at zero for the next call.
template <int R>
__global__ __launch_bounds__(512, R == 1 ? 4 : 2) void kvq_paged8_ranges_kernel(const AttnArgs A) {
    constexpr int RB = 16 * R, W = 8;
    __shared__ float4v lds_o[W][16][32];     // a wavefront's outputs of 16 rows, chunks of four channels turned by the row
    __shared__ float4v lds_ml[W][16];        // reference, sum, sum of the unrounded, what the outputs stand for
    __shared__ u32x4 lds_q[R][4][64];        // queries as operands: registers are for tiles on their way
    __shared__ int lds_last;
    const KvqP8& P = A.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, n = lane & 15;
    const int rows_per_token = A.gqa * A.maps;

    // ---- which piece
    const auto shape = [&](const Seq& q) {
        const uint32_t blocks = (uint32_t)(q.rows * rows_per_token + RB - 1) / RB;
        return Cuts::Shape{max(1, (q.tokens + 31) >> 5), (int)blocks * P.n_kv, q.rows * A.gqa <= A.few_rows ? 1 : 0};
    };
    Cuts::Shape* const shapes = reinterpret_cast<Cuts::Shape*>(lds_o);
    Seq seq = {0, 0, 0, 0};
    if (P.n_seqs > 64) {
        for (int at = threadIdx.x; at < P.n_seqs; at += 512) shapes[at] = shape(seq_of(P, at));
        __syncthreads();
    } else if (lane < P.n_seqs) {
        seq = seq_of(P, lane);
    }
    Cuts cuts(shapes, P.n_seqs, shape(seq), lane, KVQ_P8_GROUPS / R);
    Piece pc;
    if (!cuts.find(blockIdx.x, pc)) return;
    const int s = pc.seq, tiles = pc.tiles, pieces = pc.pieces, piece = pc.piece;
    if (P.n_seqs > 64) seq = seq_of(P, s);
    else seq = Seq{__builtin_amdgcn_readlane(seq.row0, s), __builtin_amdgcn_readlane(seq.rows, s), __builtin_amdgcn_readlane(seq.end, s), __builtin_amdgcn_readlane(seq.tokens, s)};
    const int blocks = (uint32_t)(seq.rows * rows_per_token + RB - 1) / RB;
    if (pc.unit >= blocks * P.n_kv) return;  // (rows have changed since the units were counted)
    const int kv = (uint32_t)pc.unit / (uint32_t)blocks, block = pc.unit - kv * blocks;
    // (equal ranges: 33 tiles are 17 and 16, not 32 and 1)
    const int each = (uint32_t)tiles / (uint32_t)pieces, left = tiles - each * pieces;
    const int t0 = piece * each + min(piece, left), t1 = t0 + each + (piece < left ? 1 : 0);
    int limit[R], row_i[R];
    int most = 0, least = 0x7fffffff;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        row_i[r] = (uint32_t)(block * RB + 16 * r + n) / (uint32_t)rows_per_token;
        const bool real = row_i[r] < seq.rows;
        limit[r] = real ? sees(seq, row_i[r]) : seq.tokens;
        most = max(most, real ? limit[r] : 0);
        least = min(least, limit[r]);
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
    }
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);
    const int end = min(t1, (most + 31) >> 5);

    // ---- the wavefront's tiles: pages and scale words of 64 of them, one a lane, and one tile's codes on their way.  What lies behind the last, or
    // on no page, is behind its buffer's end: a load under a condition would make the compiler wait for it at once.
    int from = t0 + wave, page = -1;
    u32x2 words = {0, 0};
    u32x4 kc[4], vc[4];
    const auto describe = [&]() {
        const int mine = from + lane * W;
        page = mine < end ? page_of(P, s, mine >> (P.page_shift - 5)) : -1;
        words = u32x2{0, 0};
        if (page >= 0) words = *reinterpret_cast<const u32x2*>(P.words + ((int64_t)page * P.n_kv + kv) * 2);
    };
    const auto tile_at = [&](int k) {
        const int pg = k < 64 ? __builtin_amdgcn_readlane(page, k & 63) : -1;
        return __builtin_amdgcn_make_buffer_rsrc(tile_of(P, max(0, pg), kv, (from + k * W) & ((1 << (P.page_shift - 5)) - 1)), 0,
                                                 pg >= 0 ? KVQ_P8_TILE_BYTES : 0, 0x00020000);
    };
    const auto load_k = [&](__amdgpu_buffer_rsrc_t p) {  // (2: read once)
#pragma unroll
        for (int c = 0; c < 4; ++c) kc[c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(p, lane * 16, c * 1024, 2));
    };
    const auto load_v = [&](__amdgpu_buffer_rsrc_t p) {
#pragma unroll
        for (int c = 0; c < 4; ++c) vc[c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(p, lane * 16, 4096 + c * 1024, 2));
    };
    u32x4 q_mine[R];
    if (wave < 4) {  // four channel groups of the rows, one a wavefront
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int rest = block * RB + 16 * r + n - row_i[r] * rows_per_token;
            const int h = A.maps == 2 ? rest >> 1 : rest, map = A.maps == 2 ? rest & 1 : 0;
            q_mine[r] = u32x4{0, 0, 0, 0};
            if (row_i[r] < seq.rows && (A.maps == 1 || (wave >> 1) == map)) {
                q_mine[r] = *reinterpret_cast<const u32x4*>(A.q + (seq.row0 + row_i[r]) * A.q_rs + (int64_t)(kv * A.gqa + h) * A.q_hs + 32 * wave + 8 * j);
                q_mine[r] ^= A.flip;
            }
        }
    }
    describe();
    load_k(tile_at(0));
    load_v(tile_at(0));
    if (wave < 4)
#pragma unroll
        for (int r = 0; r < R; ++r) lds_q[r][wave][lane] = q_mine[r];
    __syncthreads();

    State<R> st;
    st.clear();
    int top = wave_max((int)(words[1] & 0xffu));
    while (from < end) {
        const int todo = min(64, (int)((uint32_t)(end - from + W - 1) / W));
        for (int k = 0; k < todo; ++k) {
            const __amdgpu_buffer_rsrc_t next = tile_at(k + 1);
            const int kw = __builtin_amdgcn_readlane(words[0], k), vw = __builtin_amdgcn_readlane(words[1], k);
            const bool there = __builtin_amdgcn_readlane(page, k) >= 0;
            const int tok = (from + k * W) * 32;
            float4v sc[R][1][2];
            asm volatile("" ::: "memory");  // (queries would be kept in registers)
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
                for (int r = 0; r < R; ++r) sc[r][0][sub] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int grp = 0; grp < 4; ++grp) {
                    const u32x4 w = kc[2 * sub + (grp >> 1)];
                    const half8 a = widen(w[2 * (grp & 1)], w[2 * (grp & 1) + 1], 1.f);
#pragma unroll
                    for (int r = 0; r < R; ++r) sc[r][0][sub] = mma(a, to_half8(lds_q[r][grp][lane]), sc[r][0][sub]);
                }
            }
            load_k(next);
            if (there) {
                if (least < tok + 32) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int over = limit[r] - tok - 8 * j;
#pragma unroll
                        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (4 * sub + i >= over) sc[r][0][sub][i] = -INFINITY;
                    }
                }
                uint32_t p[R][1][4];
                const float factor = score_factor(A.scale_log2, kw);
#pragma unroll
                for (int r = 0; r < R; ++r) softmax_group<R, 1, false, true>(st, r, sc[r], factor, A.lse != nullptr, p[r]);
                const float vs = value_scale(top - (vw & 0xff));
                const bool nan = (vw & KVQ_P8_NAN) != 0;
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) {
                    uint32_t w[2] = {vc[nt >> 1][2 * (nt & 1)], vc[nt >> 1][2 * (nt & 1) + 1]};
                    if (nan) {
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            uint32_t x[2] = {w[0], w[1]};
                            st.o[r][nt] += nan_codes(x, tok + 8 * j, limit[r]);
                            if (r == R - 1) w[0] = x[0], w[1] = x[1];
                        }
                    }
                    const half8 a = widen(w[0], w[1], vs);
#pragma unroll
                    for (int r = 0; r < R; ++r) st.o[r][nt] = mma(a, to_half8(p[r][0]), st.o[r][nt]);
                }
            }
            load_v(next);
        }
        from += 64 * W;
        if (from < end) {
            describe();
            load_k(tile_at(0));
            load_v(tile_at(0));
            const int top_here = max(top, wave_max((int)(words[1] & 0xffu)));
            const float by = __builtin_ldexpf(1.f, top - top_here);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) st.o[r][nt] *= by;
            top = top_here;
        }
    }

    // ---- the wavefronts' states together, then the pieces of the unit, then the rows of the output
    {
        // (the thread's index afresh: what follows from it would be kept in registers through the loop above)
        const int tid = opaque(threadIdx.x), lane = tid & 63, j = lane >> 4, n = lane & 15;
        const int real_rows = min(RB, seq.rows * rows_per_token - block * RB);
        const auto slot = [&](int k) { return A.part + (int64_t)(pc.slot + k) * (R * (KVQ_PART_BYTES / 4)); };
        const int row = tid >> 5, chunk = tid & 31;
        float4v o[R];
        float m[R], l[R], fine[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            __syncthreads();
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) lds_o[wave][n][(4 * nt + j + n) & 31] = st.o[r][nt];
            const float sum = quarters_sum(st.l[r]), fine_sum = quarters_sum(st.fine[r]);
            if (lane < 16) lds_ml[wave][n] = float4v{st.m[r], sum, fine_sum, value_unit(top)};
            __syncthreads();
            m[r] = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) m[r] = fmaxf(m[r], lds_ml[w][row][0]);
            o[r] = float4v{0.f, 0.f, 0.f, 0.f};
            l[r] = fine[r] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float4v ml = lds_ml[w][row];
                const float weight = __builtin_amdgcn_exp2f(ml[0] - reference_of(m[r]));
                o[r] += lds_o[w][row][(chunk + row) & 31] * (weight * ml[3]);
                l[r] += ml[1] * weight;
                fine[r] += ml[2] * weight;
            }
        }
        bool mine = true;
        if (pieces > 1) {
            float* const to = slot(piece);
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(to, 0, R * KVQ_PART_BYTES, 0x00020000);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (16 * r + row >= real_rows) continue;
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o[r]), buf, r * KVQ_PART_BYTES + tid * 16, 0, 16);
                if (chunk == 0)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, float4v{m[r], l[r], fine[r], 0.f}), buf,
                                                           r * KVQ_PART_BYTES + KVQ_PART_O_FLOATS * 4 + row * 16, 0, 16);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) {
                uint32_t* const counter = A.counters + (int64_t)pc.slot * KVQ_P8_COUNTER_STRIDE;
                const uint32_t got = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                const bool last = got == (uint32_t)pieces - 1u;
                if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                lds_last = last ? 1 : 0;
            }
            __syncthreads();
            mine = lds_last != 0;
            asm volatile("" ::: "memory");
            if (mine) {
                // All pieces of a row by the 32 lanes that have its channels: references and sums a piece a lane, whose weights pass through LDS, then the
                // outputs, eight pieces on their way together.  Pieces beyond the last read as zeros, by the buffer's range, with a weight of zero.
                float(*const weights)[KVQ_P8_MOST_PIECES] = reinterpret_cast<float(*)[KVQ_P8_MOST_PIECES]>(lds_o);
                const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(slot(0), 0, pieces * R * KVQ_PART_BYTES, 0x00020000);
                constexpr int STEP = R * KVQ_PART_BYTES;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (16 * r + row >= real_rows) continue;
                    const auto load = [&](int k) {
                        return __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, k * STEP + r * KVQ_PART_BYTES + tid * 16, 0, 16));
                    };
                    float4v x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = load(k);
                    constexpr int PER = KVQ_P8_MOST_PIECES / 32;
                    float4v ml[PER];
#pragma unroll
                    for (int c = 0; c < PER; ++c)
                        ml[c] = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, (chunk + 32 * c) * STEP + r * KVQ_PART_BYTES + KVQ_PART_O_FLOATS * 4 + row * 16, 0, 16));
                    m[r] = -INFINITY;
#pragma unroll
                    for (int c = 0; c < PER; ++c) m[r] = chunk + 32 * c < pieces ? fmaxf(m[r], ml[c][0]) : m[r];
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) m[r] = fmaxf(m[r], __shfl_xor(m[r], d));
                    const float ref = reference_of(m[r]);
                    l[r] = fine[r] = 0.f;
#pragma unroll
                    for (int c = 0; c < PER; ++c) {
                        const float w = chunk + 32 * c < pieces ? __builtin_amdgcn_exp2f(ml[c][0] - ref) : 0.f;
                        l[r] += ml[c][1] * w;
                        fine[r] += ml[c][2] * w;
                        weights[row][chunk + 32 * c] = w;
                    }
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        l[r] += __shfl_xor(l[r], d);
                        fine[r] += __shfl_xor(fine[r], d);
                    }
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // (a row's weights are written and read by one wavefront)
                    __builtin_amdgcn_wave_barrier();
                    o[r] = float4v{0.f, 0.f, 0.f, 0.f};
                    for (int k0 = 0; k0 < pieces; k0 += 8) {
                        float4v y[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = x[k];
                        if (k0 + 8 < pieces)
#pragma unroll
                            for (int k = 0; k < 8; ++k) x[k] = load(k0 + 8 + k);
#pragma unroll
                        for (int k = 0; k < 8; ++k) o[r] += y[k] * weights[row][k0 + k];
                    }
                }
            }
        }
        if (mine) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int f = block * RB + 16 * r + row, i = f / rows_per_token, rest = f - i * rows_per_token;
                float4v x = o[r] * kvq_flash::inverse_of(l[r]);
                const int h = kv * A.gqa + (A.maps == 2 ? rest >> 1 : rest);
                const bool real = i < seq.rows;
                if (A.maps == 2) {
                    // the second map's row lies 32 lanes on
                    const float lam = real ? A.lambda[h] : 0.f;
                    float square = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = x[e] - lam * __shfl_xor(x[e], 32);
                        square = fmaf(x[e], x[e], square);
                    }
                    if (A.weight) {
#pragma unroll
                        for (int d = 1; d < 32; d <<= 1) square += __shfl_xor(square, d);
                        const float mean = square * (1.f / KVQ_D) + A.eps;
                        x *= mean > 0.f ? 1.f / sqrtf(mean) : mean;  // (nothing but zeros and no eps: zeros; NaN stays)
                        x *= *reinterpret_cast<const float4v*>(A.weight + 4 * chunk);
                    }
                    x *= A.out_scale;
                }
                if (!real || (A.maps == 2 && (rest & 1))) continue;
                const int64_t to = (seq.row0 + i) * A.o_rs + h * A.o_hs;
                void* const dst = A.out_fp32 ? static_cast<void*>(static_cast<float*>(A.out) + to) : static_cast<void*>(static_cast<_Float16*>(A.out) + to);
                if (!A.out_fp32)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = half_range(x[e]);
                kvq_flash::store_out4(dst, A.out_fp32, 4 * chunk, x);
                if (A.lse && chunk == 0)
                    A.lse[h * A.lse_hs + seq.row0 + i] = fine[r] == 0.f ? -INFINITY : (m[r] + __builtin_amdgcn_logf(fine[r])) * 0.69314718055994530942f;
            }
        }
    }
}

// ---- Sequences with many rows: chunks of prompts

// Where the work of the units lies on one line that workgroups take equal shares of.  A block's length on it is its tiles, by the tokens that its last
// row sees, and kLead for what a block costs beside them (33 sequences, chunks of up to 965 rows x 64 heads among them, 246 us with 4, 211 with 8, 213
// with 12; a prompt of 8,192 tokens with two maps 836, 837, 849); blocks of a KV head lie one after the other, KV heads, sequences.
struct Line {
    int rows, blocks;     // flat rows, blocks
    int length;           // of all blocks of one KV head
    double seen, growth;  // tiles that the rows of the first token see; half of those that a block adds to what the next one sees
    static constexpr int kLead = 8;
    // where block b begins (in 64-bit floating point, the same in every workgroup, where whole numbers would take a division that is a loop)
    __device__ static int place(int b, double seen, double growth) { return (int)__builtin_fma((double)b * (b + 1), growth, b * seen) + kLead * b; }
    __device__ int at(int b) const { return __builtin_amdgcn_readfirstlane(place(b, seen, growth)); }
};
template <int RB>
__device__ inline Line line_of(const Seq& q, int per_token, int few_rows) {
    Line x;
    x.rows = q.rows * per_token;
    x.seen = min(max(0, q.end - q.rows), q.tokens) * (1. / 32);
    x.growth = RB / 64. / per_token;
    x.blocks = x.rows > few_rows ? (x.rows + RB - 1) / RB : 0;
    x.length = Line::place(x.blocks, x.seen, x.growth);
    return x;
}

typedef float float16v __attribute__((ext_vector_type(16)));
#ifdef KVQ_NO_ARITHMETIC
__device__ inline float16v mma32(half8, half8, float16v c) { return c; }
#else
__device__ inline float16v mma32(half8 a, half8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
#endif
// over the two halves of a wavefront, in every lane
__device__ inline float halves_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float halves_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// One softmax map of 32 rows of a wavefront, as kvq_flash.h's State but by v_mfma_f32_32x32x16_f16: lane = 32 h + n has row n.
struct Map {
    float16v o[4];  // o[cb][i]: channel 32 cb + 8 (i / 4) + 4 h + i % 4
    float m;        // the reference (log2 units), equal in both halves
    float l, fine;  // this half's shares of the sums
    __device__ void clear() {
        m = -INFINITY;
        l = fine = 0.f;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[cb][i] = 0.f;
    }
    __device__ void scale(float by) {
        l *= by;
        fine *= by;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) o[cb] *= by;
    }
};
// Probabilities of NT tiles from raw scores (masked ones at -inf), the tiles with a factor each; reference and sums as in kvq_flash.h.
// s[x][i]: token 16 (i / 8) + 8 h + i % 8 of tile x, and p in that order.
template <int NT>
__device__ inline void softmax_tiles(Map& st, const float16v (&s)[NT], const float (&factor)[NT], bool fine, uint32_t (&p)[NT][8]) {
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        float most = s[x][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, s[x][i]);
        top = fmaxf(top, most * factor[x]);
    }
    if (__any(top > st.m + (KVQ_BELOW + KVQ_FOLLOW))) {
        const float m_new = fmaxf(st.m, halves_max(top) - KVQ_BELOW);
        st.scale(__builtin_amdgcn_exp2f(st.m - reference_of(m_new)));
        st.m = m_new;
    }
    const float ref = reference_of(st.m);
    const half2v ones = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[x][i], factor[x], -ref));
        if (fine) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st.fine += e[i];
        }
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            p[x][v] = kvq_flash::pack2(e[2 * v], e[2 * v + 1]);
            const uint32_t two = p[x][v];
            st.l = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, two), ones, st.l, false);
        }
    }
}

// A block of 256 rows, 32 a wavefront, MAPS softmax maps of each, against the tiles of a piece of its unit.  Two groups of four wavefronts, one of
// either on a SIMD, take turns: while one has its products (scores of a stage of NT tiles, and the probabilities of the stage before times its values),
// the other has its softmax, widens the codes of a stage two further on into LDS and loads the next.  A barrier stands between the turns.  A stage is
// written in the turns 2 s - 3 and 2 s - 2, its keys are read in 2 s and 2 s + 1, its values in 2 s + 2 and 2 s + 3: four buffers.
// Products and vector instructions bound it, which overlap by half at best (16,000 products of one wavefront a SIMD 298 us, 128,000 multiply-adds of another
// 316, both 439): matrix cores 40 % busy, vector instructions, products among them, 44 %.  So what counts is few instructions: codes are widened once a
// workgroup of 256 rows, products are of 32 x 32 (half the instructions and operand reads of 16 x 16), a lane has one row's statistics, the sum is a dot
// product of the rounded pairs.  Two chunks of 1,024 behind 16,000 tokens x 40 heads 700 us = 929 TFLOP/s where a library product of 8,192^3 has 1,160 (770
// with four wavefronts of 32 rows each and products of 16 x 16, two workgroups a compute unit), a prompt of 8,192 x 28 heads with two maps 837 us =
// 863 TFLOP/s (1,110).
template <int MAPS>
__global__ __launch_bounds__(512, 2) void kvq_paged8_chunk_kernel(const AttnArgs A) {
    constexpr int RB = 256, NT = MAPS == 1 ? 2 : 1, KB = 8 / MAPS, TILE = 2 * KVQ_FLASH_TILE_BYTES, STAGE = NT * TILE, AHEAD = 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * STAGE];
    __shared__ u32x4 lds_q[MAPS == 2 ? 8 : 1][4][64];  // two maps: the second's queries, for which there are no registers
    static_assert(KVQ_P8_CHUNK_GROUPS <= 1 << kJoinLevels, "levels of a join");
    __shared__ int lds_last[kJoinLevels];
    const KvqP8& P = A.p;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_page = P.page_shift - 5;

    {
        const auto units_of = [&](int s) { return small_units((seq_of(P, s).rows * A.gqa * MAPS + 31) / 32 * P.n_kv); };  // as the launch over pieces counts them
        const auto tiles_of = [&](int s) { return small_tiles(units_of(s), max(1, (seq_of(P, s).tokens + 31) >> 5)); };
        const Census<decltype(units_of)> units(units_of, P.n_seqs);
        const Census<decltype(tiles_of)> tiles(tiles_of, P.n_seqs);
        if (small_call(units.total, tiles.total)) return;
    }
    if (A.packed && !rows_fit(P)) return;
    const auto line = [&](const Seq& q) { return line_of<RB>(q, A.gqa, A.few_rows); };
    const auto count = [&](int s) { return line(seq_of(P, s)).length * P.n_kv; };
    const Census<decltype(count)> census(count, P.n_seqs);
    if (census.total == 0) return;
    const int groups = gridDim.x, share = max(KVQ_P8_LEAST_CHUNK, (census.total + groups - 1) / groups);
    // neighbours on the line go to one XCD, whose L2 then holds the keys and values that they have in common
    const int wg = groups % 8 == 0 ? (blockIdx.x & 7) * (groups >> 3) + (blockIdx.x >> 3) : blockIdx.x;
    int pos = wg * share;
    if (pos >= census.total) return;
    const int range_end = min(census.total, pos + share);
    int first;
    int s = __builtin_amdgcn_readfirstlane(census.find(pos, first));
    if (s < 0) return;
    first = __builtin_amdgcn_readfirstlane(first);
    while (pos < range_end) {
        Seq seq;
        Line ln;
        const auto length_of = [&](int s) {
            seq = seq_of(P, s);
            ln = line(seq);
            return __builtin_amdgcn_readfirstlane(ln.length) * P.n_kv;
        };
        if (!walk(length_of, P.n_seqs, pos, s, first)) return;
        int gqa = A.gqa;
        asm volatile("" : "+s"(gqa));  // (as opaque(): its reciprocal would be kept in registers throughout)
        const int flat = seq.rows * gqa;
        const int head_length = __builtin_amdgcn_readfirstlane(ln.length), kv = (pos - first) / head_length, in_head = pos - first - kv * head_length;
        int block = 0;
        for (int step = 1 << 26; step; step >>= 1)
            if (block + step < ln.blocks && ln.at(block + step) <= in_head) block += step;
        const int unit = pos - in_head + ln.at(block), length = ln.at(block + 1) - ln.at(block);  // the unit's place on the line
        const int unit_end = min(range_end, unit + length);

        // the lane's row
        struct Row { int i, head; bool real; };
        const auto row_of = [&](int at) {
            const int f = block * RB + wave * 32 + at, i = f / gqa;
            return Row{i, kv * gqa + f - i * gqa, f < flat};
        };
        int limit;
        half8 q[KB];
        int most, least;
        {
            const int lane = opaque(threadIdx.x) & 63, h = lane >> 5, n = lane & 31;
            const Row row = row_of(n);
            limit = least = row.real ? sees(seq, row.i) : seq.tokens;
            most = row.real ? limit : 0;
            const _Float16* const src = A.q + (seq.row0 + (row.real ? row.i : 0)) * A.q_rs + (int64_t)(row.real ? row.head : kv * gqa) * A.q_hs + 8 * h;
#pragma unroll
            for (int kb = 0; kb < 8; ++kb) {
                u32x4 w = *reinterpret_cast<const u32x4*>(src + 16 * kb);
                w ^= A.flip;
                if (!row.real) w = u32x4{0, 0, 0, 0};
                if (kb < KB) q[kb] = to_half8(w);
                else lds_q[wave][kb & 3][lane] = w;
            }
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            most = max(most, __shfl_xor(most, d));
            least = min(least, __shfl_xor(least, d));
        }
        most = __builtin_amdgcn_readfirstlane(most);
        least = __builtin_amdgcn_readfirstlane(least);
        // the block's tiles: those that its last row sees
        const int last_row = min(flat, (block + 1) * RB) - 1;
        const int tiles = (sees(seq, last_row / gqa) + 31) >> 5;
        const auto tile_at = [&](int x) { return __builtin_amdgcn_readfirstlane((int)((double)(x - unit) * tiles / length)); };
        const int t0 = tile_at(pos), t1 = tile_at(unit_end), stages = (t1 - t0 + NT - 1) / NT;

        Map st[MAPS];
#pragma unroll
        for (int m = 0; m < MAPS; ++m) st[m].clear();

        // Pages and scale words of 64 tiles, one a lane: those that are loaded from, what the softmax needs of those that it has come to, and the 64
        // tiles behind.  A scale's info: exponents of keys and values in the low bytes (values': how far behind the largest of these and
        // earlier tiles, which is kTop's byte), kNan, kThere.
        constexpr int kNan = 1 << 16, kThere = 1 << 17, kTop = 18;
        const auto top_of = [](int info) { return __builtin_amdgcn_readfirstlane(info) >> kTop; };
        const auto ranked = [&](int info, int top) {
            top = max(top, wave_max(info & kThere ? (info >> 8) & 0xff : 0));
            return (info & ~0xff00) + (((top - (info >> 8)) & 0xff) << 8) + (top << kTop);
        };
        const auto page_at = [&](int t) { const int lane = opaque(threadIdx.x) & 63; return t + lane < t1 ? page_of(P, s, (t + lane) >> per_page) : -1; };
        const auto info_of = [&](int pg) {
            if (pg < 0) return 0;
            const u32x2 w = *reinterpret_cast<const u32x2*>(P.words + ((int64_t)pg * P.n_kv + kv) * 2);
            return (int)((w[0] & 0xffu) | (w[1] & 0xffu) << 8 | (w[1] & KVQ_P8_NAN ? kNan : 0) | kThere);
        };
        int load_batch = t0, soft_batch = t0;
        int page = page_at(t0), page_next = page_at(t0 + 64), info = ranked(info_of(page), 0), info_soft = info, info_next = 0;

        struct Raw {
            u32x4 w[NT];
            int info;
        } raw;
        const auto load = [&](int stage, Raw& raw) {  // an eighth of a stage a wavefront: of two tiles a quarter of one, of one tile a quarter of its keys or values
            const int t = t0 + stage * NT + (NT == 2 ? wave >> 2 : 0), lane = opaque(threadIdx.x) & 63;
            if (t0 + stage * NT - load_batch >= 64) {
                page = page_next;
                info = ranked(info_next, top_of(info));
                load_batch += 64;
                page_next = page_at(load_batch + 64);
            }
            if (t0 + stage * NT - load_batch == 32) info_next = info_of(page_next);
            const int page_here = __builtin_amdgcn_readlane(page, t - load_batch);
            raw.info = __builtin_amdgcn_readlane(info, t - load_batch);
            const uint8_t* const at = tile_of(P, max(0, page_here), kv, t & ((1 << per_page) - 1)) + (wave & 3) * 1024 + lane * 16;
            if (NT == 2) {
                raw.w[0] = *reinterpret_cast<const u32x4*>(at);
                raw.w[NT - 1] = *reinterpret_cast<const u32x4*>(at + 4096);
            } else {
                raw.w[0] = *reinterpret_cast<const u32x4*>(at + (wave >> 2) * 4096);
            }
        };
        const auto store = [&](int stage, const Raw& raw) {
            uint8_t* const to = lds + (stage & 3) * STAGE + (NT == 2 ? wave >> 2 : 0) * TILE;
            const int c = wave & 3, lane = opaque(threadIdx.x) & 63;
            const auto keys = [&](u32x4 w) {  // sub-tile c / 2, channel groups 2 (c % 2) and + 1
                const int at = ((lane >> 3) & 1) * 4096 + (lane >> 4) * 256 + ((c >> 1) * 8 + (lane & 7)) * 16 + (c & 1) * 2048;
#pragma unroll
                for (int k = 0; k < 2; ++k) *reinterpret_cast<half8*>(to + at + k * 1024) = widen(w[2 * k], w[2 * k + 1], 1.f);
            };
            const auto values = [&](u32x4 w) {  // channel blocks 2 c and + 1
                if (!(raw.info & kThere)) w = u32x4{0, 0, 0, 0};
                if (raw.info & kNan) {
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int b = 0; b < 32; b += 8)
                            if (((w[d] >> b) & 0x7fu) == 0x7fu) w[d] &= ~(0xffu << b);
                }
                const float vs = value_scale((raw.info >> 8) & 0xff);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    *reinterpret_cast<half8*>(to + KVQ_FLASH_TILE_BYTES + (2 * c + k) * 1024 + lane * 16) = widen(w[2 * k], w[2 * k + 1], vs);
            };
            if (NT == 2) {
                keys(raw.w[0]);
                values(raw.w[NT - 1]);
            } else if (wave < 4) {
                keys(raw.w[0]);
            } else {
                values(raw.w[0]);
            }
        };
        if constexpr (MAPS == 1) {  // the first two stages on their way together (of two maps there are no registers for it)
            Raw early;
            if (stages > 0) load(0, early);
            if (stages > 1) load(1, raw);
            if (stages > 0) store(0, early);
        } else {
            if (stages > 0) load(0, raw), store(0, raw);
            if (stages > 1) load(1, raw);
        }
        if (stages > 1) store(1, raw);
        if (stages > 2) load(2, raw);
        __syncthreads();
        const bool late = wave >= 4;
        if (late) __syncthreads();

        // Where the lane's operands lie.  Of keys, row n of the product is token 16 (n / 16) + 8 (n / 4 % 2) + 4 (n / 8 % 2) + n % 4, so that a half of the
        // wavefront receives runs of eight tokens; the 16 rows of either half tile lie together, 256 bytes for eight channels, which 16 lanes read.
        const auto keys_at = [](int lane) { return ((lane >> 4) & 1) * 4096 + (lane >> 5) * 256 + (lane & 15) * 16; };
        const auto values_at = [](int lane) { return KVQ_FLASH_TILE_BYTES + ((lane >> 4) & 1) * 1024 + (lane >> 5) * 256 + (lane & 15) * 16; };

        // stages that the wavefront's rows see; behind them it only loads (in a loop of its own: under a condition in one loop the accumulators were copied)
        const int seen = max(0, min(stages, ((most + 31) / 32 - t0 + NT - 1) / NT));
        int nan = 0;
        uint32_t p[MAPS][NT][8];
        // Products whose operands are read AHEAD steps in front of them, in this order (left to itself the compiler waits for every one)
        const auto scores = [&](int stage, float16v (&sc)[MAPS][NT]) {
            const int lane = opaque(threadIdx.x) & 63;
            const uint8_t* const kt = lds + (stage & 3) * STAGE + keys_at(lane);
            // step i: of two maps their 16 channels in turn, of one map the tiles
            const auto kb_of = [](int i) { return MAPS == 2 ? (i & 1) * KB + (i >> 1) : i >> 1; };
            const auto key = [&](int i) {
                const int kb = kb_of(i), x = MAPS == 2 ? 0 : i & 1;
                return to_half8(*reinterpret_cast<const u32x4*>(kt + x * TILE + (kb >> 1) * 1024 + (kb & 1) * 512));
            };
            half8 a[AHEAD], b[2];  // (b: the second map's queries, of every other step)
            const auto query = [&](int i) { return to_half8(lds_q[wave][kb_of(i) & 3][lane]); };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) a[i] = key(i);
            if (MAPS == 2) b[0] = query(1), b[1] = query(3);
#pragma unroll
            for (int m = 0; m < MAPS; ++m)
#pragma unroll
                for (int x = 0; x < NT; ++x)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[m][x][i] = 0.f;
#pragma unroll
            for (int i = 0; i < 8 * NT; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                const int m = MAPS == 2 ? i & 1 : 0, x = MAPS == 2 ? 0 : i & 1;
                sc[m][x] = mma32(a[i % AHEAD], m == 1 ? b[(i >> 1) & 1] : q[kb_of(i) % KB], sc[m][x]);
                if (i + AHEAD < 8 * NT) a[i % AHEAD] = key(i + AHEAD);
                if (m == 1 && i + 4 < 8) b[(i >> 1) & 1] = query(i + 4);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        const auto values_times = [&](int stage) {
            const int lane = opaque(threadIdx.x) & 63;
            const uint8_t* const vt = lds + (stage & 3) * STAGE + values_at(lane);
            const auto value = [&](int i) {  // step i: channel block i % 4 of tokens 16 (i / 4 % 2) .. of tile i / 8
                return to_half8(*reinterpret_cast<const u32x4*>(vt + (i >> 3) * TILE + (i & 3) * 2048 + ((i >> 2) & 1) * 512));
            };
            half8 a[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) a[i] = value(i);
#pragma unroll
            for (int i = 0; i < 8 * NT; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                const int x = i >> 3, u = (i >> 2) & 1;
#pragma unroll
                for (int m = 0; m < MAPS; ++m)
                    st[m].o[i & 3] = mma32(a[i % AHEAD], to_half8(u32x4{p[m][x][4 * u], p[m][x][4 * u + 1], p[m][x][4 * u + 2], p[m][x][4 * u + 3]}), st[m].o[i & 3]);
                if (i + AHEAD < 8 * NT) a[i % AHEAD] = value(i + AHEAD);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        const auto softmax = [&](int stage, float16v (&sc)[MAPS][NT]) {
            const int tok = (t0 + stage * NT) * 32, h = (opaque(threadIdx.x) >> 5) & 1;
            if (t0 + stage * NT - soft_batch >= 64) {
                if (top_of(info) != top_of(info_soft)) {
                    const float by = __builtin_ldexpf(1.f, top_of(info_soft) - top_of(info));
#pragma unroll
                    for (int m = 0; m < MAPS; ++m)
#pragma unroll
                        for (int cb = 0; cb < 4; ++cb) st[m].o[cb] *= by;
                }
                info_soft = info;
                soft_batch += 64;
            }
            int flags = kThere, here = 0, of[NT];
            float factor[NT];
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                of[x] = __builtin_amdgcn_readlane(info_soft, t0 + stage * NT + x - soft_batch);
                factor[x] = score_factor(A.scale_log2, of[x]);
                flags &= of[x];
                here |= of[x];
            }
            if (least < tok + NT * 32 || !flags) {
#pragma unroll
                for (int x = 0; x < NT; ++x) {
                    const int over = (of[x] & kThere ? limit - tok - 32 * x : 0) - 8 * h;
#pragma unroll
                    for (int m = 0; m < MAPS; ++m)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            sc[m][x][i] = 16 * (i >> 3) + (i & 7) < over ? sc[m][x][i] : -INFINITY;
                }
            }
#pragma unroll
            for (int m = 0; m < MAPS; ++m) {
                softmax_tiles<NT>(st[m], sc[m], factor, MAPS == 1 && A.lse != nullptr, p[m]);
                if (MAPS == 2) __builtin_amdgcn_sched_barrier(0);  // (side by side they take more registers than there are)
            }
            nan |= here;
        };
        const auto fetch = [&](int stage) {
            if (stage + 2 < stages) store(stage + 2, raw);
            if (stage + 3 < stages) load(stage + 3, raw);
            __syncthreads();
        };
        for (int stage = 0; stage <= stages; ++stage) {
            if (stage > 0 && stage <= seen) values_times(stage - 1);
            float16v sc[MAPS][NT];  // (not beyond the turn: kept from one stage to the next they would be in the way of the outputs)
            if (stage < seen) scores(stage, sc);
            __syncthreads();
            if (stage < seen) {
                // (scores where they are: with the conditions before and behind the barrier taken together, half of them were copied)
#pragma unroll
                for (int m = 0; m < MAPS; ++m)
#pragma unroll
                    for (int x = 0; x < NT; ++x) asm volatile("" : "+v"(sc[m][x]));
                softmax(stage, sc);
            }
            fetch(stage);
        }
        if (!late) __syncthreads();
        // NaN values, where a page has any: to the rows that see them, once more over the tiles (their codes were zeros above)
        if (nan & kNan) {
            const int lane = opaque(threadIdx.x) & 63, h = lane >> 5, n = lane & 31;
            for (int tile = t0; tile < min(t1, t0 + seen * NT); ++tile) {
                const int pg = __builtin_amdgcn_readfirstlane(page_of(P, s, tile >> per_page));
                if (pg < 0 || !(P.words[((int64_t)pg * P.n_kv + kv) * 2 + 1] & KVQ_P8_NAN)) continue;
                const uint8_t* const at = tile_of(P, pg, kv, tile & ((1 << per_page) - 1)) + 4096 + h * 256 + (n & 15) * 16 + (n >> 4) * 8;
#pragma unroll
                for (int cb = 0; cb < 4; ++cb) {
                    float16v found;
#pragma unroll
                    for (int i = 0; i < 16; ++i) found[i] = 0.f;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const u32x2 w = *reinterpret_cast<const u32x2*>(at + cb * 1024 + u * 512);
                        half8 is, sees;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            is[e] = ((w[e >> 2] >> (8 * (e & 3))) & 0x7fu) == 0x7fu ? (_Float16)1.f : (_Float16)0.f;
                            sees[e] = tile * 32 + 16 * u + 8 * h + e < limit ? (_Float16)1.f : (_Float16)0.f;
                        }
                        found = mma32(is, sees, found);
                    }
#pragma unroll
                    for (int m = 0; m < MAPS; ++m)
#pragma unroll
                        for (int i = 0; i < 16; ++i) st[m].o[cb][i] += found[i] > 0.f ? __builtin_nanf("") : 0.f;
                }
            }
        }

        // ---- the pieces of a unit that lies in several workgroups' shares, joined two by two as a tree over their order on the line: of two neighbours
        // whoever finds the other's stored joins it to its own, in registers, and goes on to the next level.  Products are rounded before they are added,
        // so that it does not matter who (all pieces joined by the last of them, one after the other: 232 rows x 4 heads with two maps over 48,010 tokens, in a
        // batch of nine, 267 us; so 137).  A pair's counter is that of the workgroup at which its second half begins, its slot that of its first.
        // (no piece lies behind the line's end, also where lengths have changed since it was measured)
        const int w0 = unit / share, pieces = (min(unit + length, census.total) - 1) / share - w0 + 1;
        bool mine = true;
        float unit_of_o = value_unit(top_of(info_soft));
        for (int width = 1, at = wg - w0, level = 0; mine && width < pieces; width *= 2, ++level) {
            const int other = join_other(at, width), begin = min(at, other), second = max(at, other);
            if (second >= pieces) continue;
            constexpr int MAP = KVQ_P8_MAP_BYTES, SLOT = 8 * MAPS * MAP, FLY = MAPS == 1 ? 16 : 8;
            const bool rows_here = block * RB + wave * 32 < flat;  // whether the wavefront has any
            const auto slot = [&](int k) {
                return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<uint8_t*>(A.part) + (int64_t)(2 * (w0 + k) + (k == 0 ? 1 : 0)) * SLOT, 0, SLOT, 0x00020000);
            };
            const int own_at = wave * MAPS * MAP + (opaque(threadIdx.x) & 63) * 16;
            uint32_t* const counter = A.counters + (int64_t)(w0 + second) * KVQ_P8_COUNTER_STRIDE;
            if (threadIdx.x == 0) lds_last[join_word(level)] = __hip_atomic_load(counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 1u ? 1 : 0;
            __syncthreads();
            mine = lds_last[join_word(level)] != 0;
            if (!mine) {
                const __amdgpu_buffer_rsrc_t to = slot(at);
                if (rows_here)
#pragma unroll
                for (int m = 0; m < MAPS; ++m) {
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const float16v& o = st[m].o[v >> 2];
                        const float4v x = {o[4 * (v & 3)], o[4 * (v & 3) + 1], o[4 * (v & 3) + 2], o[4 * (v & 3) + 3]};
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), to, own_at + m * MAP + v * 1024, 0, 16);
                    }
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, float4v{st[m].m, st[m].l, st[m].fine, unit_of_o}), to, own_at + m * MAP + 16384, 0, 16);
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (threadIdx.x == 0) lds_last[join_word(level)] = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 1u ? 1 : 0;
                __syncthreads();
                mine = lds_last[join_word(level)] != 0;
            }
            if (mine && threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("" ::: "memory");
            if (mine && rows_here) {
                const __amdgpu_buffer_rsrc_t from = slot(other);
                const auto load = [&](int i) {  // the outputs of both maps, one after the other
                    return __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, own_at + (i >> 4) * MAP + (i & 15) * 1024, 0, 16));
                };
                float4v ml[MAPS], x[FLY];
#pragma unroll
                for (int m = 0; m < MAPS; ++m) ml[m] = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, own_at + m * MAP + 16384, 0, 16));
#pragma unroll
                for (int i = 0; i < FLY; ++i) x[i] = load(i);
#pragma unroll
                for (int m = 0; m < MAPS; ++m) {
                    const float m_new = fmaxf(st[m].m, ml[m][0]), ref = reference_of(m_new);
                    float a = __builtin_amdgcn_exp2f(st[m].m - ref), b = __builtin_amdgcn_exp2f(ml[m][0] - ref);
                    st[m].m = m_new;
                    st[m].l = __fadd_rn(__fmul_rn(st[m].l, a), __fmul_rn(ml[m][1], b));
                    st[m].fine = __fadd_rn(__fmul_rn(st[m].fine, a), __fmul_rn(ml[m][2], b));
                    a *= unit_of_o;
                    b *= ml[m][3];
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int i = m * 16 + v;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            st[m].o[v >> 2][4 * (v & 3) + e] = __fadd_rn(__fmul_rn(st[m].o[v >> 2][4 * (v & 3) + e], a), __fmul_rn(x[i % FLY][e], b));
                        if (i + FLY < 16 * MAPS) x[i % FLY] = load(i + FLY);
                    }
                }
                unit_of_o = 1.f;
            }
            at = begin;
        }
        if (mine) {
            const int lane = opaque(threadIdx.x) & 63, h = lane >> 5, n = lane & 31;
            const Row row = row_of(n);
            float inv[MAPS], by;
#pragma unroll
            for (int m = 0; m < MAPS; ++m) inv[m] = unit_of_o * kvq_flash::inverse_of(halves_sum(st[m].l));
            by = inv[0];
            const float fine = MAPS == 1 ? halves_sum(st[0].fine) : 0.f;
            if (MAPS == 2) {
                inv[MAPS - 1] *= row.real ? A.lambda[row.head] : 0.f;
                float square = 0.f;
#pragma unroll
                for (int cb = 0; cb < 4; ++cb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float x = st[0].o[cb][i] * inv[0] - st[MAPS - 1].o[cb][i] * inv[MAPS - 1];
                        st[0].o[cb][i] = x;
                        square = fmaf(x, x, square);
                    }
                by = A.out_scale;
                if (A.weight) {
                    const float mean = halves_sum(square) * (1.f / KVQ_D) + A.eps;
                    by *= mean > 0.f ? 1.f / sqrtf(mean) : mean;
                }
            }
            if (row.real) {
                const int64_t to = (seq.row0 + row.i) * A.o_rs + row.head * A.o_hs;
                // two runs of eight channels at a time: after the exchange a half of the wavefront has one of them whole
#pragma unroll
                for (int v = 0; v < 16; v += 2) {
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float c = st[0].o[v >> 2][4 * (v & 3) + i], d = st[0].o[v >> 2][4 * (v & 3) + 4 + i];
                        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(c), __float_as_uint(d), false, false);
                        y[i] = __uint_as_float(both[0]) * by;
                        y[4 + i] = __uint_as_float(both[1]) * by;
                    }
                    const int channel = 8 * (v + h);
                    float4v lo = {y[0], y[1], y[2], y[3]}, hi = {y[4], y[5], y[6], y[7]};
                    if (MAPS == 2 && A.weight) {
                        lo *= *reinterpret_cast<const float4v*>(A.weight + channel);
                        hi *= *reinterpret_cast<const float4v*>(A.weight + channel + 4);
                    }
                    if (A.out_fp32) {
                        float4v* const to4 = reinterpret_cast<float4v*>(static_cast<float*>(A.out) + to + channel);
                        to4[0] = lo;
                        to4[1] = hi;
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) lo[i] = half_range(lo[i]), hi[i] = half_range(hi[i]);
                        const u32x4 w = {kvq_flash::pack2(lo[0], lo[1]), kvq_flash::pack2(lo[2], lo[3]), kvq_flash::pack2(hi[0], hi[1]), kvq_flash::pack2(hi[2], hi[3])};
                        *reinterpret_cast<u32x4*>(static_cast<_Float16*>(A.out) + to + channel) = w;
                    }
                }
                if (MAPS == 1 && A.lse && h == 0)
                    A.lse[row.head * A.lse_hs + seq.row0 + row.i] = fine == 0.f ? -INFINITY : (st[0].m + __builtin_amdgcn_logf(fine)) * 0.69314718055994530942f;
            }
        }
        pos = unit_end;
    }
}

constexpr uint64_t kCounterBytes = 2ull * KVQ_P8_GROUPS * KVQ_P8_COUNTER_STRIDE * 4;

bool heads_ok(int32_t n_q, int32_t n_kv) { return n_q >= 1 && n_q % n_kv == 0 && n_q / n_kv <= KVQ_MAX_GQA; }

// The launches of a call: over ranges of tiles for sequences of few rows, of more where there may be any.  Either uses the workspace from its start.
constexpr int kFewRows = 64;  // flat rows of one map
constexpr int64_t kMostSum = 1 << 30;  // what the kernels add up, at most
struct Plan {
    int r;                  // groups of 16 rows of the first launch
    bool packed;
    int64_t groups, chunk;  // workgroups
    uint64_t bytes;
};
bool plan_of(const KvqP8& P, int gqa, int maps, Plan& plan) {
    const int64_t most = (int64_t)P.max_rows * gqa, few = std::min<int64_t>(most, kFewRows) * maps;
    plan.r = few <= 16 ? 1 : 2;
    const int64_t tiles = (int64_t)P.table_pages << (P.page_shift - 5), heads = (int64_t)P.n_seqs * P.n_kv;
    // the sums of a launch over pieces, which counts all sequences' rows as few
    if (heads && (few + 16 * plan.r - 1) / (16 * plan.r) * tiles > kMostSum / heads) return false;
    // and the line of all chunks: blocks of every sequence as if each had max_rows, or where that is too many, of the rows that there are
    const int64_t length = tiles + 2 * Line::kLead + P.max_rows / 64, of_each = (most + 255) / 256 * P.n_seqs;
    int64_t blocks = of_each;
    plan.packed = most > kFewRows && heads && of_each * length > kMostSum / P.n_kv;
    if (plan.packed) {
        blocks = std::min(of_each, (int64_t)P.n_rows * gqa / 256 + P.n_seqs);
        if (blocks * length > kMostSum / P.n_kv) return false;
    }
    // as many workgroups as pieces there can be (of few rows, or of all in a small call), and partial results of those of units that are cut
    const int64_t at_a_time = KVQ_P8_GROUPS / plan.r;
    const auto pieces = [&](int64_t flat, int64_t limit) {
        const int64_t units = std::min(limit, (flat * maps + 16 * plan.r - 1) / (16 * plan.r) * heads);
        const int64_t cuts = units * ((tiles + KVQ_P8_LEAST_SHARE - 1) / KVQ_P8_LEAST_SHARE);
        return std::min(cuts, few_units(units, at_a_time) ? at_a_time : at_a_time + units);
    };
    plan.groups = std::max(pieces(std::min<int64_t>(most, kFewRows), INT32_MAX), pieces(most, KVQ_P8_SMALL_UNITS));
    if (plan.groups > UINT32_MAX / 512) return false;  // threads of a launch
    const int64_t line = blocks * length * P.n_kv;
    plan.chunk = most > kFewRows ? std::min<int64_t>(KVQ_P8_CHUNK_GROUPS, (line / KVQ_P8_LEAST_CHUNK + 8) & ~7ll) : 0;
    plan.bytes = kCounterBytes + 2 * (uint64_t)std::max<int64_t>(std::min<int64_t>(plan.groups, at_a_time) * plan.r * KVQ_PART_BYTES, plan.chunk * 8 * maps * KVQ_P8_MAP_BYTES);
    return true;
}

kvq_status_t attend(const kvq_paged8_t* cache, const kvq_paged8_batch_t* batch, const kvq_paged8_rows_t* q, const kvq_paged8_rows_t* out,
                    int32_t n_q_heads, int32_t out_is_fp32, float softmax_scale, void* workspace, uint64_t bytes, AttnArgs& A, hipStream_t stream) {
    Plan plan;
    if (!kvq_p8_args(cache, batch, A.p) || !heads_ok(n_q_heads, cache->n_kv_heads)) return KVQ_E_INVALID;
    if (!kvq_p8_rows_ok(q, batch, 8) || !kvq_p8_rows_ok(out, batch, out_is_fp32 ? 4 : 8) || !kvq_p8_rows_apart(out, batch, n_q_heads)) return KVQ_E_INVALID;
    if (!std::isfinite(softmax_scale) || !plan_of(A.p, n_q_heads / cache->n_kv_heads, A.maps, plan)) return KVQ_E_INVALID;
    if (!A.p.n_seqs || !A.p.n_rows) return KVQ_OK;
    if (!kvq_p8_aligned(workspace, 16) || bytes < plan.bytes) return KVQ_E_INVALID;
    A.q = static_cast<const _Float16*>(q->data_dev);
    A.out = const_cast<void*>(out->data_dev);
    A.q_rs = q->row_stride; A.q_hs = q->head_stride;
    A.o_rs = out->row_stride; A.o_hs = out->head_stride;
    A.lse_hs = A.p.n_rows;
    A.gqa = n_q_heads / cache->n_kv_heads;
    A.out_fp32 = out_is_fp32 ? 1 : 0;
    const float scale = softmax_scale != 0.f ? softmax_scale : 1.0f / std::sqrt((float)(KVQ_D / A.maps));
    A.scale_log2 = std::fabs(scale) * 1.44269504088896340736f;
    A.flip = scale < 0.f ? 0x80008000u : 0u;
    A.counters = static_cast<uint32_t*>(workspace);
    A.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kCounterBytes);
    A.few_rows = kFewRows;
    A.packed = plan.packed ? 1 : 0;
    if (plan.r == 1) hipLaunchKernelGGL(kvq_paged8_ranges_kernel<1>, dim3((unsigned)plan.groups), dim3(512), 0, stream, A);
    else hipLaunchKernelGGL(kvq_paged8_ranges_kernel<2>, dim3((unsigned)plan.groups), dim3(512), 0, stream, A);
    if (hipGetLastError() != hipSuccess) return KVQ_E_HIP;
    if (!plan.chunk) return KVQ_OK;
    if (A.maps == 1) hipLaunchKernelGGL(kvq_paged8_chunk_kernel<1>, dim3((unsigned)plan.chunk), dim3(512), 0, stream, A);
    else hipLaunchKernelGGL(kvq_paged8_chunk_kernel<2>, dim3((unsigned)plan.chunk), dim3(512), 0, stream, A);
    return hipGetLastError() == hipSuccess ? KVQ_OK : KVQ_E_HIP;
}

}  // namespace

extern "C" {

uint64_t kvq_paged8_workspace_bytes(const kvq_paged8_t* cache, const kvq_paged8_batch_t* batch, int32_t n_q_heads, int32_t two_maps) {
    KvqP8 P{};
    Plan plan;
    if (!kvq_p8_args(cache, batch, P) || !heads_ok(n_q_heads, P.n_kv)) return 0;
    return plan_of(P, n_q_heads / P.n_kv, two_maps ? 2 : 1, plan) ? plan.bytes : 0;
}

kvq_status_t kvq_paged8_attention(const kvq_paged8_t* cache, const kvq_paged8_batch_t* batch, const kvq_paged8_rows_t* q_dev,
                                  const kvq_paged8_rows_t* out_dev, int32_t n_q_heads, int32_t out_is_fp32, float softmax_scale,
                                  float* lse_dev, void* workspace_dev, uint64_t workspace_bytes, void* hip_stream) {
    AttnArgs A{};
    if (reinterpret_cast<uintptr_t>(lse_dev) & 3u) return KVQ_E_INVALID;
    A.lse = lse_dev;
    A.maps = 1;
    return attend(cache, batch, q_dev, out_dev, n_q_heads, out_is_fp32, softmax_scale, workspace_dev, workspace_bytes, A,
                  static_cast<hipStream_t>(hip_stream));
}

kvq_status_t kvq_paged8_diff_attention(const kvq_paged8_t* cache, const kvq_paged8_batch_t* batch, const kvq_paged8_rows_t* q_dev,
                                       const float* lambda_dev, const kvq_paged8_rows_t* out_dev, int32_t n_q_heads, int32_t out_is_fp32,
                                       float softmax_scale, const float* norm_weight_dev, float norm_eps, float out_scale,
                                       void* workspace_dev, uint64_t workspace_bytes, void* hip_stream) {
    AttnArgs A{};
    if (!kvq_p8_aligned(lambda_dev, 4) || (norm_weight_dev && !kvq_p8_aligned(norm_weight_dev, 16))) return KVQ_E_INVALID;
    if (!std::isfinite(out_scale) || !std::isfinite(norm_eps) || norm_eps < 0.f) return KVQ_E_INVALID;
    A.lambda = lambda_dev;
    A.weight = norm_weight_dev;
    A.eps = norm_eps;
    A.out_scale = out_scale;
    A.maps = 2;
    return attend(cache, batch, q_dev, out_dev, n_q_heads, out_is_fp32, softmax_scale, workspace_dev, workspace_bytes, A,
                  static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
