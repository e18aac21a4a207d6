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

#define KVQ_P8_GROUPS 512       // workgroups of a launch over ranges of tiles, at most
#define KVQ_P8_COUNTER_STRIDE 16 // words: a line for each arrival counter
#define KVQ_P8_LEAST_SHARE 8    // tiles of a workgroup, at least
#define KVQ_P8_LEAST_CHUNK 16   // of a workgroup with a chunk
#define KVQ_P8_MOST_PIECES 128  // of a unit

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
    int32_t least_rows;            // sequences with more flat rows (of one map) are chunks
    float scale_log2, eps, out_scale;
    uint32_t flip;                 // sign bits to turn over in the queries (a negative scale)
};

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
// Values are taken times 1/2 and outputs times 2: a rounded code may stand for up to 2^16, beyond fp16.
__device__ inline float value_scale(int word) { return ldexpf(0.5f, exponent_of(word)); }

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
// are few, of the smallest share that leaves no more pieces than the device takes workgroups at a time (a workgroup that came behind them would
// have the device for itself), else of what an equal share of all tiles is, short units behind long pieces as workgroups end.
struct Piece {
    int seq, unit, tiles, pieces, piece;
    int slot;  // of the unit's first piece among those of all units that are cut
};
struct Cuts {
    struct Shape { int tiles, units; };
    const Shape* all;  // of all sequences, where they are more than lanes
    Shape mine;
    int n, per, lane, share;

    // over this lane's sequences
    template <class F>
    __device__ int sum(F f) const {
        if (per == 1) return f(mine);
        int x = 0;
        for (int k = 0; k < per; ++k)
            if (lane * per + k < n) x += f(all[lane * per + k]);
        return x;
    }
    template <class F>
    __device__ int total(F f) const { return __builtin_amdgcn_readlane(wave_scan(sum(f)), 63); }
    __device__ int cuts_of(Shape x) const { return (x.tiles + share - 1) / share; }

    __device__ Cuts(const Shape* shapes, int n_seqs, Shape own, int lane_) : all(shapes), mine(own), n(n_seqs), per((n_seqs + 63) >> 6), lane(lane_) {
        const int units = total([](Shape x) { return x.units; }), tiles = total([](Shape x) { return x.units * x.tiles; });
        int longest = 0;
        sum([&](Shape x) { longest = max(longest, x.units ? x.tiles : 0); return 0; });
        longest = wave_max(longest);
        const int wanted = KVQ_P8_GROUPS;
        int low = max(max(KVQ_P8_LEAST_SHARE, (tiles + wanted - 1) / wanted), (longest + KVQ_P8_MOST_PIECES - 1) / KVQ_P8_MOST_PIECES);
        share = low;
        if (2 * units > wanted) return;
        int high = max(low, (tiles + wanted - units - 1) / (wanted - units));  // enough: a unit has at most one piece more than its tiles by the share
        while (high - low > low >> 4) {
            share = (low + high) >> 1;
            if (total([&](Shape x) { return x.units * cuts_of(x); }) <= wanted) high = share;
            else low = share + 1;
        }
        share = high;
    }
    // Piece `id`, the same in all lanes.
    __device__ bool find(int id, Piece& p) const {
        const auto pieces = [&](Shape x) { return x.units * cuts_of(x); };
        const auto cut = [&](Shape x) { const int c = cuts_of(x); return c > 1 ? x.units * c : 0; };
        int x = sum(pieces), y = sum(cut), upto = wave_scan(x), cut_upto = wave_scan(y);
        uint64_t behind = __ballot(upto > id);
        if (!behind) return false;
        int at = __builtin_ctzll(behind);
        int before = __builtin_amdgcn_readlane(upto - x, at), slots = __builtin_amdgcn_readlane(cut_upto - y, at);
        Shape s = mine;
        p.seq = at;
        if (per > 1) {  // among that lane's sequences, one a lane
            const int i = at * per + lane;
            s = lane < per && i < n ? all[i] : Shape{1, 0};
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
        p.pieces = (p.tiles + share - 1) / share;
        p.unit = (id - before) / p.pieces;
        p.piece = id - before - p.unit * p.pieces;
        p.slot = slots + p.unit * p.pieces;
        return true;
    }
};

// A piece a workgroup; the pieces of a unit are joined by the last of them to arrive.  Eight wavefronts take a piece's tiles in turn, every one
// from memory straight into operand registers: nothing but the queries is shared before the end.
template <int R>
__global__ __launch_bounds__(512, R == 1 ? 4 : 2) void kvq_paged8_ranges_kernel(const AttnArgs A) {
    constexpr int RB = 16 * R, W = 8;
    __shared__ float4v lds_o[W][16][32];     // a wavefront's outputs of 16 rows, chunks of four channels turned by the row
    __shared__ float4v lds_ml[W][16];        // reference, sum, sum of the unrounded
    __shared__ u32x4 lds_q[R][4][64];        // queries as operands: registers are for tiles on their way
    __shared__ int lds_last;
    const KvqP8& P = A.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, n = lane & 15;
    const int rows_per_token = A.gqa * A.maps;

    // ---- which piece
    const auto shape = [&](int at) {
        const Seq q = seq_of(P, at);
        const int blocks = q.rows * A.gqa > A.least_rows ? 0 : (q.rows * rows_per_token + RB - 1) / RB;
        return Cuts::Shape{max(1, (q.tokens + 31) >> 5), blocks * P.n_kv};
    };
    Cuts::Shape* const shapes = reinterpret_cast<Cuts::Shape*>(lds_o);
    if (P.n_seqs > 64) {
        for (int at = threadIdx.x; at < P.n_seqs; at += 512) shapes[at] = shape(at);
        __syncthreads();
    }
    Cuts cuts(shapes, P.n_seqs, P.n_seqs <= 64 && lane < P.n_seqs ? shape(lane) : Cuts::Shape{1, 0}, lane);
    Piece pc;
    if (!cuts.find(blockIdx.x, pc)) return;
    const int s = pc.seq, tiles = pc.tiles, pieces = pc.pieces, piece = pc.piece;
    const Seq seq = seq_of(P, s);
    const int blocks = (seq.rows * rows_per_token + RB - 1) / RB, kv = pc.unit / blocks, block = pc.unit - kv * blocks;
    // (equal ranges: 33 tiles are 17 and 16, not 32 and 1)
    const int t0 = (int)((int64_t)tiles * piece / pieces), t1 = (int)((int64_t)tiles * (piece + 1) / pieces);
    int limit[R];
    int most = 0, least = 0x7fffffff;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int f = block * RB + 16 * r + n, i = f / rows_per_token;
        const bool real = i < seq.rows;
        limit[r] = real ? max(0, seq.tokens - seq.rows + i + 1) : seq.tokens;
        most = max(most, real ? limit[r] : 0);
        least = min(least, limit[r]);
    }
    if (wave < 4) {  // four channel groups of the rows, one a wavefront
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int f = block * RB + 16 * r + n, i = f / rows_per_token, rest = f - i * rows_per_token;
            const int h = A.maps == 2 ? rest >> 1 : rest, map = A.maps == 2 ? rest & 1 : 0;
            u32x4 w = {0, 0, 0, 0};
            if (i < seq.rows && (A.maps == 1 || (wave >> 1) == map)) {
                w = *reinterpret_cast<const u32x4*>(A.q + (seq.row0 + i) * A.q_rs + (int64_t)(kv * A.gqa + h) * A.q_hs + 32 * wave + 8 * j);
                w ^= A.flip;
            }
            lds_q[r][wave][lane] = w;
        }
    }
    __syncthreads();
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
    }
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);
    const int end = min(t1, (most + 31) >> 5);

    State<R> st;
    st.clear();
    for (int from = t0 + wave; from < end; from += 64 * W) {
        // the pages and scale words of the wavefront's next 64 tiles, one a lane
        const int mine = from + lane * W;
        const int page = mine < end ? page_of(P, s, mine >> (P.page_shift - 5)) : -1;
        u32x2 words = {0, 0};
        if (page >= 0) words = *reinterpret_cast<const u32x2*>(P.words + ((int64_t)page * P.n_kv + kv) * 2);
        const int todo = min(64, (end - from + W - 1) / W);
        u32x4 kc[4], vc[4];
        const auto at = [&](int k) {
            const int pg = max(0, __builtin_amdgcn_readlane(page, k));
            return tile_of(P, pg, kv, (from + k * W) & ((1 << (P.page_shift - 5)) - 1)) + lane * 16;
        };
        const auto load_k = [&](const uint8_t* p) {
#pragma unroll
            for (int c = 0; c < 4; ++c) kc[c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + c * 1024));
        };
        const auto load_v = [&](const uint8_t* p) {
#pragma unroll
            for (int c = 0; c < 4; ++c) vc[c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 4096 + c * 1024));
        };
        load_k(at(0));
        load_v(at(0));
        for (int k = 0; k < todo; ++k) {
            const uint8_t* const next = at(min(k + 1, todo - 1));
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
                const float vs = value_scale(vw);
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
    }

    // ---- the wavefronts' states together, then the pieces of the unit, then the rows of the output
    {
        // (the thread's index afresh: what follows from it would be kept in registers through the loop above)
        int fresh = threadIdx.x;
        asm volatile("" : "+v"(fresh));
        const int tid = fresh, lane = tid & 63, j = lane >> 4, n = lane & 15;
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
            if (lane < 16) lds_ml[wave][n] = float4v{st.m[r], sum, fine_sum, 0.f};
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
                o[r] += lds_o[w][row][(chunk + row) & 31] * weight;
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
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (16 * r + row >= real_rows) continue;
                    m[r] = -INFINITY;
                    l[r] = fine[r] = 0.f;
                    o[r] = float4v{0.f, 0.f, 0.f, 0.f};
                    for (int k = 0; k < pieces; ++k) {
                        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(slot(k), 0, R * KVQ_PART_BYTES, 0x00020000);
                        const float4v ml = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, r * KVQ_PART_BYTES + KVQ_PART_O_FLOATS * 4 + row * 16, 0, 16));
                        const float4v x = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, r * KVQ_PART_BYTES + tid * 16, 0, 16));
                        const float m_new = fmaxf(m[r], ml[0]), ref = reference_of(m_new);
                        const float a = __builtin_amdgcn_exp2f(m[r] - ref), b = __builtin_amdgcn_exp2f(ml[0] - ref);
                        o[r] = o[r] * a + x * b;
                        l[r] = l[r] * a + ml[1] * b;
                        fine[r] = fine[r] * a + ml[2] * b;
                        m[r] = m_new;
                    }
                }
            }
        }
        if (mine) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int f = block * RB + 16 * r + row, i = f / rows_per_token, rest = f - i * rows_per_token;
                float4v x = o[r] * (2.f * kvq_flash::inverse_of(l[r]));
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
                kvq_flash::store_out4(dst, A.out_fp32, 4 * chunk, x);
                if (A.lse && chunk == 0)
                    A.lse[h * A.lse_hs + seq.row0 + i] = fine[r] == 0.f ? -INFINITY : (m[r] + __builtin_amdgcn_logf(fine[r])) * 0.69314718055994530942f;
            }
        }
    }
}

// ---- Sequences with many rows: chunks of prompts

// Probabilities of TT tiles for row group r as kvq_flash.h's softmax_group, the tiles with a factor each.
template <int R, int TT>
__device__ inline void softmax_tiles(State<R>& st, int r, const float4v (&s)[TT][2], const float (&factor)[TT], bool fine, uint32_t (&p)[TT][4]) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        float most = -INFINITY;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, s[t][sub][i]);
        top = fmaxf(top, most * factor[t]);
    }
    if (__any(top > st.m[r] + (KVQ_BELOW + KVQ_FOLLOW))) {
        const float m_new = fmaxf(st.m[r], kvq_flash::quarters_max(top) - KVQ_BELOW);
        const float alpha = __builtin_amdgcn_exp2f(st.m[r] - reference_of(m_new));
        st.l[r] *= alpha;
        st.fine[r] *= alpha;
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) st.o[r][nt] *= alpha;
        st.m[r] = m_new;
    }
    const float ref = reference_of(st.m[r]);
    const half2v ones = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        float e[2][4];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int i = 0; i < 4; ++i) e[sub][i] = __builtin_amdgcn_exp2f(fmaf(s[t][sub][i], factor[t], -ref));
        if (fine) {
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.fine[r] += e[sub][i];
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            p[t][v] = kvq_flash::pack2(e[v >> 1][2 * (v & 1)], e[v >> 1][2 * (v & 1) + 1]);
            const uint32_t two = p[t][v];
            st.l[r] = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, two), ones, st.l[r], false);
        }
    }
}

// Where the work of the units lies on one line that workgroups take equal shares of.  A block's length on it is its tiles, by the tokens that its last
// row sees, and kLead for what a block costs beside them; blocks of a KV head lie one after the other, KV heads, sequences.
struct Line {
    int rows, seen0, per_token, blocks;  // flat rows, tokens that the rows of the first token see, flat rows of a token, blocks
    int length;                          // of all blocks of one KV head
    static constexpr int kLead = 4;
    template <int RB>
    __device__ int at(int b) const {  // where block b begins
        return (int)(((int64_t)b * seen0 + (int64_t)b * (b + 1) / 2 * RB / per_token) >> 5) + kLead * b;
    }
};
template <int RB>
__device__ inline Line line_of(const Seq& q, int per_token, int least_rows) {
    Line x;
    x.rows = q.rows * per_token;
    x.seen0 = max(0, q.tokens - q.rows);
    x.per_token = per_token;
    x.blocks = x.rows > least_rows ? (x.rows + RB - 1) / RB : 0;
    x.length = x.blocks ? x.at<RB>(x.blocks) : 0;
    return x;
}

// RG groups of 16 rows a wavefront, MAPS states of each; four wavefronts with rows of their own share the tiles: two an iteration, widened to fp16 once on
// their way into LDS, where the next ones are put while these are computed on.
template <int RG, int MAPS, int TT>
__global__ __launch_bounds__(256, 2) void kvq_paged8_chunk_kernel(const AttnArgs A) {
    constexpr int R = RG * MAPS, RB = 64 * RG, NT = 2, TILE = 2 * KVQ_FLASH_TILE_BYTES, STAGE = NT * TILE;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE];
    __shared__ int lds_last;
    const KvqP8& P = A.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, n = lane & 15;
    const int per_page = P.page_shift - 5;

    const auto line = [&](const Seq& q) { return line_of<RB>(q, A.gqa, A.least_rows); };
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
    first = __builtin_amdgcn_readfirstlane(first);
    Seq seq = seq_of(P, s);
    Line ln = line(seq);
    while (pos < range_end) {
        while (pos - first >= ln.length * P.n_kv) {
            first += ln.length * P.n_kv;
            seq = seq_of(P, ++s);
            ln = line(seq);
        }
        const int kv = (pos - first) / ln.length, in_head = pos - first - kv * ln.length;
        int block = 0;
        for (int step = 1 << 26; step; step >>= 1)
            if (block + step < ln.blocks && ln.at<RB>(block + step) <= in_head) block += step;
        const int unit = pos - in_head + ln.at<RB>(block), length = ln.at<RB>(block + 1) - ln.at<RB>(block);  // the unit's place on the line
        const int unit_end = min(range_end, unit + length);

        int limit[RG];
        half8 q[RG][4];
        int most = 0, least = 0x7fffffff;
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            const int f = block * RB + wave * 16 * RG + 16 * g + n, i = f / A.gqa, h = f - i * A.gqa;
            const bool real = f < ln.rows;
            limit[g] = real ? max(0, seq.tokens - seq.rows + i + 1) : seq.tokens;
            most = max(most, real ? limit[g] : 0);
            least = min(least, limit[g]);
            const _Float16* const src = A.q + (seq.row0 + (real ? i : 0)) * A.q_rs + (int64_t)(kv * A.gqa + (real ? h : 0)) * A.q_hs + 8 * j;
#pragma unroll
            for (int grp = 0; grp < 4; ++grp) {
                u32x4 w = *reinterpret_cast<const u32x4*>(src + 32 * grp);
                w ^= A.flip;
                if (!real) w = u32x4{0, 0, 0, 0};
                q[g][grp] = to_half8(w);
            }
        }
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) {
            most = max(most, __shfl_xor(most, d));
            least = min(least, __shfl_xor(least, d));
        }
        most = __builtin_amdgcn_readfirstlane(most);
        least = __builtin_amdgcn_readfirstlane(least);
        // the block's tiles: those that its last row sees
        const int last_row = min(ln.rows, (block + 1) * RB) - 1;
        const int tiles = (max(0, seq.tokens - seq.rows + last_row / A.gqa + 1) + 31) >> 5;
        const auto tile_at = [&](int x) { return __builtin_amdgcn_readfirstlane((int)((int64_t)(x - unit) * tiles / length)); };
        const int t0 = tile_at(pos), t1 = tile_at(unit_end);

        State<R> st;
        st.clear();

        // pages and scale words of 64 tiles, one a lane, and of the 64 behind them
        int batch = t0, page, page_next;
        u32x2 words, words_next;
        const auto pages_from = [&](int t) { return t + lane < t1 ? page_of(P, s, (t + lane) >> per_page) : -1; };
        const auto words_of = [&](int pg) {
            u32x2 w = {0, 0};
            if (pg >= 0) w = *reinterpret_cast<const u32x2*>(P.words + ((int64_t)pg * P.n_kv + kv) * 2);
            return w;
        };
        page = pages_from(batch);
        page_next = pages_from(batch + 64);
        words = words_of(page);
        words_next = u32x2{0, 0};

        struct Tile { int page, kw, vw; } now[NT], next[NT];
        u32x4 kr[NT], vr[NT];
        const auto load = [&](int t) {  // a quarter of every tile a wavefront
            if (t - batch >= 64) {
                page = page_next;
                words = words_next;
                batch += 64;
                page_next = pages_from(batch + 64);
            }
            if (t - batch == 32) words_next = words_of(page_next);
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                next[x].page = __builtin_amdgcn_readlane(page, t - batch + x);
                next[x].kw = __builtin_amdgcn_readlane(words[0], t - batch + x);
                next[x].vw = __builtin_amdgcn_readlane(words[1], t - batch + x);
                const uint8_t* const at = tile_of(P, max(0, next[x].page), kv, (t + x) & ((1 << per_page) - 1)) + wave * 1024 + lane * 16;
                kr[x] = *reinterpret_cast<const u32x4*>(at);
                vr[x] = *reinterpret_cast<const u32x4*>(at + 4096);
            }
        };
        const auto store = [&](int buf) {
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                uint8_t* const kt = lds + buf * STAGE + x * TILE + lane * 16;
                uint8_t* const vt = kt + KVQ_FLASH_TILE_BYTES;
                const float vs = value_scale(next[x].vw);
                u32x4 v = vr[x];
                if (next[x].page < 0) v = u32x4{0, 0, 0, 0};
                if (next[x].vw & KVQ_P8_NAN) {
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int b = 0; b < 32; b += 8)
                            if (((v[d] >> b) & 0x7fu) == 0x7fu) v[d] &= ~(0xffu << b);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // chunk `wave` of the K tile: sub-tile wave / 2, channel groups 2 (wave % 2) + h; of the V tile: channel block 2 wave + h
                    *reinterpret_cast<half8*>(kt + (4 * (wave >> 1) + 2 * (wave & 1) + h) * 1024) = widen(kr[x][2 * h], kr[x][2 * h + 1], 1.f);
                    *reinterpret_cast<half8*>(vt + (2 * wave + h) * 1024) = widen(v[2 * h], v[2 * h + 1], vs);
                }
            }
        };
        if (t0 < t1) {
            load(t0);
            store(0);
        }
        __syncthreads();
        int buf = 0;
        for (int t = t0; t < t1; t += NT) {
            const bool more = t + NT < t1;
#pragma unroll
            for (int x = 0; x < NT; ++x) now[x] = next[x];
            if (more) load(t + NT);
            if (t * 32 < most) {  // (behind what its rows see a wavefront only loads)
#pragma unroll
                for (int x0 = 0; x0 < NT; x0 += TT) {
                    const uint8_t* const kt = lds + buf * STAGE + x0 * TILE + lane * 16;
                    const uint8_t* const vt = kt + KVQ_FLASH_TILE_BYTES;
                    const int tok = (t + x0) * 32;
                    float4v sc[R][TT][2];
#pragma unroll
                    for (int x = 0; x < TT; ++x)
#pragma unroll
                        for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
                            for (int r = 0; r < R; ++r) sc[r][x][sub] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int grp = 0; grp < 4; ++grp) {
                                const half8 a = to_half8(*reinterpret_cast<const u32x4*>(kt + x * TILE + (sub * 4 + grp) * 1024));
#pragma unroll
                                for (int g = 0; g < RG; ++g) {
                                    float4v& to = sc[MAPS * g + (MAPS == 2 ? grp >> 1 : 0)][x][sub];
                                    to = mma(a, q[g][grp], to);
                                }
                            }
                        }
                    bool masked = least < tok + TT * 32;
                    float factor[TT];
#pragma unroll
                    for (int x = 0; x < TT; ++x) {
                        masked = masked || now[x0 + x].page < 0;
                        factor[x] = score_factor(A.scale_log2, now[x0 + x].kw);
                    }
                    if (masked) {
#pragma unroll
                        for (int g = 0; g < RG; ++g)
#pragma unroll
                            for (int x = 0; x < TT; ++x) {
                                const int over = (now[x0 + x].page < 0 ? 0 : limit[g] - tok - 32 * x) - 8 * j;
#pragma unroll
                                for (int m = 0; m < MAPS; ++m)
#pragma unroll
                                    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                                        for (int i = 0; i < 4; ++i)
                                            if (4 * sub + i >= over) sc[MAPS * g + m][x][sub][i] = -INFINITY;
                            }
                    }
                    uint32_t p[R][TT][4];
#pragma unroll
                    for (int r = 0; r < R; ++r) softmax_tiles<R, TT>(st, r, sc[r], factor, A.lse != nullptr, p[r]);
                    int flagged = 0;
#pragma unroll
                    for (int x = 0; x < TT; ++x) flagged |= now[x0 + x].page >= 0 ? now[x0 + x].vw : 0;
                    if (flagged & KVQ_P8_NAN) {  // (one branch in front of all products)
#pragma unroll 1
                        for (int x = 0; x < TT; ++x) {
                            const Tile& at_x = x ? now[x0 + TT - 1] : now[x0];
                            if (!(at_x.vw & KVQ_P8_NAN) || at_x.page < 0) continue;
                            const uint8_t* const at = tile_of(P, at_x.page, kv, (t + x0 + x) & ((1 << per_page) - 1)) + 4096 + lane * 16;
#pragma unroll
                            for (int nt = 0; nt < 8; ++nt) {
                                const u32x2 w = *reinterpret_cast<const u32x2*>(at + (nt >> 1) * 1024 + (nt & 1) * 8);
#pragma unroll
                                for (int r = 0; r < R; ++r) {
                                    uint32_t y[2] = {w[0], w[1]};
                                    st.o[r][nt] += nan_codes(y, tok + 32 * x + 8 * j, limit[r / MAPS]);
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int x = 0; x < TT; ++x)
#pragma unroll
                        for (int nt = 0; nt < 8; ++nt) {
                            const half8 a = to_half8(*reinterpret_cast<const u32x4*>(vt + x * TILE + nt * 1024));
#pragma unroll
                            for (int r = 0; r < R; ++r) st.o[r][nt] = mma(a, to_half8(p[r][x]), st.o[r][nt]);
                        }
                }
            }
            if (more) store(buf ^ 1);
            __syncthreads();
            buf ^= 1;
        }

        // ---- the pieces of a unit that lies in several workgroups' shares, joined by the last of them in the order of the line
        const int w0 = unit / share, w1 = (unit + length - 1) / share, pieces = w1 - w0 + 1;
        bool mine = true;
        if (pieces > 1) {
            constexpr int SLOT = 4 * R * KVQ_PART_BYTES;
            const auto slot = [&](int k) {
                return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<uint8_t*>(A.part) + (int64_t)(2 * (w0 + k) + (k == 0 ? 1 : 0)) * SLOT, 0, SLOT, 0x00020000);
            };
            const __amdgpu_buffer_rsrc_t to = slot(wg - w0);
            const int own_at = wave * R * KVQ_PART_BYTES + lane * 16;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int at = own_at + r * KVQ_PART_BYTES;
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, st.o[r][nt]), to, at + nt * 1024, 0, 16);
                const float l = quarters_sum(st.l[r]), fine = quarters_sum(st.fine[r]);
                if (j == 0) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, float4v{st.m[r], l, fine, 0.f}), to, at + 8192, 0, 16);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0) {
                uint32_t* const counter = A.counters + (int64_t)w0 * KVQ_P8_COUNTER_STRIDE;
                const uint32_t got = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                const bool last = got == (uint32_t)pieces - 1u;
                if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                lds_last = last ? 1 : 0;
            }
            __syncthreads();
            mine = lds_last != 0;
            asm volatile("" ::: "memory");
            if (mine) {
                st.clear();
                for (int k = 0; k < pieces; ++k) {
                    const __amdgpu_buffer_rsrc_t from = slot(k);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int at = own_at + r * KVQ_PART_BYTES;
                        const float4v ml = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, at - j * 256 + 8192, 0, 16));
                        float a, b;
                        kvq_flash::join_row<R>(st, r, ml[0], j == 0 ? ml[1] : 0.f, j == 0 ? ml[2] : 0.f, a, b);
#pragma unroll
                        for (int nt = 0; nt < 8; ++nt)
                            st.o[r][nt] = st.o[r][nt] * a + __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(from, at + nt * 1024, 0, 16)) * b;
                    }
                }
            }
        }
        if (mine) {
#pragma unroll
            for (int g = 0; g < RG; ++g) {
                const int f = block * RB + wave * 16 * RG + 16 * g + n, i = f / A.gqa, h = kv * A.gqa + f - i * A.gqa;
                const bool real = f < ln.rows;
                float inv[MAPS], fine = 0.f;
#pragma unroll
                for (int m = 0; m < MAPS; ++m) inv[m] = 2.f * kvq_flash::inverse_of(quarters_sum(st.l[MAPS * g + m]));
                float4v x[8];
                float square = 0.f;
                const float lam = MAPS == 2 && real ? A.lambda[h] : 0.f;
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) {
                    x[nt] = st.o[MAPS * g][nt] * inv[0];
                    if (MAPS == 2) {
                        x[nt] = x[nt] - st.o[R - 1 - (MAPS * (RG - 1 - g))][nt] * inv[MAPS - 1] * lam;
#pragma unroll
                        for (int e = 0; e < 4; ++e) square = fmaf(x[nt][e], x[nt][e], square);
                    }
                }
                if (MAPS == 2) {
                    float by = A.out_scale;
                    if (A.weight) {
                        const float mean = quarters_sum(square) * (1.f / KVQ_D) + A.eps;
                        by *= mean > 0.f ? 1.f / sqrtf(mean) : mean;
                    }
#pragma unroll
                    for (int nt = 0; nt < 8; ++nt) {
                        x[nt] *= by;
                        if (A.weight) x[nt] *= *reinterpret_cast<const float4v*>(A.weight + 16 * nt + 4 * j);
                    }
                } else {
                    fine = quarters_sum(st.fine[g]);
                }
                if (!real) continue;
                const int64_t to = (seq.row0 + i) * A.o_rs + h * A.o_hs;
                void* const dst = A.out_fp32 ? static_cast<void*>(static_cast<float*>(A.out) + to) : static_cast<void*>(static_cast<_Float16*>(A.out) + to);
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) kvq_flash::store_out4(dst, A.out_fp32, 16 * nt + 4 * j, x[nt]);
                if (MAPS == 1 && A.lse && j == 0)
                    A.lse[h * A.lse_hs + seq.row0 + i] = fine == 0.f ? -INFINITY : (st.m[g] + __builtin_amdgcn_logf(fine)) * 0.69314718055994530942f;
            }
        }
        pos = unit_end;
    }
}

constexpr uint64_t kCounterBytes = 2ull * KVQ_P8_GROUPS * KVQ_P8_COUNTER_STRIDE * 4;

bool heads_ok(int32_t n_q, int32_t n_kv) { return n_q >= 1 && n_q % n_kv == 0 && n_q / n_kv <= KVQ_MAX_GQA; }

// The launches of a call: over ranges of tiles for sequences of few rows, of more where there may be any.  Either uses the workspace from its start.
constexpr int kFewRows = 64;  // flat rows of one map
struct Plan {
    int r;                  // groups of 16 rows of the first launch
    int64_t groups, chunk;  // workgroups
    uint64_t bytes;
};
bool plan_of(const KvqP8& P, int gqa, int maps, Plan& plan) {
    const int64_t most = (int64_t)P.max_rows * gqa, rows = std::min<int64_t>(most, kFewRows) * maps;
    plan.r = rows <= 16 ? 1 : 2;
    const int64_t tiles = (int64_t)P.table_pages << (P.page_shift - 5), heads = (int64_t)P.n_seqs * P.n_kv;
    // blocks of 16 rows bound both: every number on either line stays below 2^30
    if (heads && (most * maps + 15) / 16 * (tiles + 8 + P.max_rows / 32) > (1 << 30) / heads) return false;
    // as many workgroups as pieces there can be, and partial results of those of units that are cut
    const int64_t units = (rows + 16 * plan.r - 1) / (16 * plan.r) * heads, cuts = units * ((tiles + KVQ_P8_LEAST_SHARE - 1) / KVQ_P8_LEAST_SHARE);
    plan.groups = std::min(cuts, 2 * units > KVQ_P8_GROUPS ? KVQ_P8_GROUPS + units : KVQ_P8_GROUPS);
    const int64_t line = ((most + 63) / 64) * (tiles + 8 + P.max_rows / 32) * heads;
    plan.chunk = most > kFewRows ? std::min<int64_t>(KVQ_P8_GROUPS, (line / KVQ_P8_LEAST_CHUNK + 8) & ~7ll) : 0;
    plan.bytes = kCounterBytes + 2 * (uint64_t)KVQ_PART_BYTES * std::max<uint64_t>(std::min<int64_t>(cuts, KVQ_P8_GROUPS) * plan.r, plan.chunk * 4 * (maps == 1 ? 2 : 4));
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
    A.least_rows = kFewRows;
    if (plan.r == 1) hipLaunchKernelGGL(kvq_paged8_ranges_kernel<1>, dim3((unsigned)plan.groups), dim3(512), 0, stream, A);
    else hipLaunchKernelGGL(kvq_paged8_ranges_kernel<2>, dim3((unsigned)plan.groups), dim3(512), 0, stream, A);
    if (hipGetLastError() != hipSuccess) return KVQ_E_HIP;
    if (!plan.chunk) return KVQ_OK;
    if (A.maps == 1) hipLaunchKernelGGL((kvq_paged8_chunk_kernel<2, 1, 2>), dim3((unsigned)plan.chunk), dim3(256), 0, stream, A);
    else hipLaunchKernelGGL((kvq_paged8_chunk_kernel<1, 2, 2>), dim3((unsigned)plan.chunk), dim3(256), 0, stream, A);
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
