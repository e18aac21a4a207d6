// Causal attention of whole prompts, or of chunks of them, over fp16 keys and values: packed sequences of different lengths, grouped
// heads (kvq_prompt_attention).
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdlib>
#include <type_traits>

#include "../../include/kvq.h"
#include "kvq_flash.h"
#include "kvq_append16.h"

namespace {

using namespace kvq_flash;

#define KVQ_PROMPT_SEQS 64  // sequences of one launch, whose descriptions ride in the kernel arguments
#define KVQ_PROMPT_THREADS 256

struct PromptSeq {
    int32_t q0, nq, k0, nk;  // first row and rows of queries, of keys
    int32_t item0;           // first workgroup
    int32_t blocks;          // row blocks of a KV head, those with the most keys first
    int32_t whole, splits;   // the first `whole` of them are taken whole, the others in so many ranges of keys
    int32_t flat;            // 1: the rows of all heads of a group follow one another; 0: every head has blocks of its own
    int32_t part0, merge0;   // of the blocks in ranges: first group of 16 rows in the workspace, first block that the second kernel joins
};
struct PromptArgs {
    const _Float16 *q, *k, *v;
    void* out;
    float* lse;
    float* part;
    int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs, lse_hs;
    int32_t gqa, n_kv, out_fp32, n_seqs;
    float scale_log2;
    uint32_t flip;  // sign bits to turn over in the queries (a negative scale)
    PromptSeq seq[KVQ_PROMPT_SEQS];
};
static_assert(sizeof(PromptArgs) <= 4096 - 64, "kernel arguments end at 4 KiB");

// Which workgroup does what: items of a sequence run through its KV heads first (neighbouring workgroups go to different XCDs, so the
// workgroups of one KV head meet in one L2 where the heads are eight), then through the ranges of keys, then through its row blocks.
struct Item {
    int seq, kv, block, split, splits;
};
__device__ inline Item item_of(const PromptArgs& A, int id) {
    int s = 0;
    for (int step = KVQ_PROMPT_SEQS / 2; step; step >>= 1)
        if (s + step < A.n_seqs && A.seq[s + step].item0 <= id) s += step;
    const PromptSeq& S = A.seq[s];
    const int x = id - S.item0, y = x / A.n_kv;
    if (y < S.whole) return Item{s, x - y * A.n_kv, y, 0, 1};
    const int z = (y - S.whole) / S.splits;
    return Item{s, x - y * A.n_kv, S.whole + z, y - S.whole - z * S.splits, S.splits};
}
// The partial results of a block in ranges: its first group of 16 rows, range 0.
template <int RB>
__device__ inline int64_t parts_of(const PromptSeq& S, int kv, int block) {
    return S.part0 + ((int64_t)kv * (S.blocks - S.whole) + (block - S.whole)) * S.splits * (RB / 16);
}
// Row r of a block: head inside the group and query; head < 0: no such row.
struct Row {
    int head, query;
};
template <int RB>
__device__ inline Row row_of(const PromptArgs& A, const PromptSeq& S, int block, int r) {
    if (S.flat) {
        const int at = block * RB + r, h = at / S.nq;
        return Row{h < A.gqa ? h : -1, at - h * S.nq};
    }
    const int per_head = S.blocks / A.gqa, ib = per_head - 1 - block / A.gqa, h = block % A.gqa;
    const int i = ib * RB + r;
    return Row{i < S.nq ? h : -1, i};
}

// What infinite and NaN values of the tiles t0 .. t1 - 1 add to a row that sees them, to what the same lanes have stored: a partial result or an output.
__device__ inline void add_nonfinite(const PromptArgs& A, const PromptSeq& S, int kv, Row row, int t0, int t1, float* part, int lane) {
    const int j = lane >> 4, n = lane & 15;
    const int limit = row.head >= 0 ? min(t1 * KVQ_TILE_TOKENS, row.query + 1 + S.nk - S.nq) : 0;
    const uint16_t* const v = reinterpret_cast<const uint16_t*>(A.v) + (int64_t)S.k0 * A.v_ts + (int64_t)kv * A.v_hs;
#pragma unroll 1
    for (int nt = 0; nt < 8; ++nt) {
        NonfiniteCount found;
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
            uint16_t w[8];
            half8 sees;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = t * KVQ_TILE_TOKENS + 8 * j + e;
                w[e] = key < S.nk ? v[(int64_t)key * A.v_ts + 16 * nt + n] : (uint16_t)0;
                sees[e] = key < limit ? (_Float16)1.f : (_Float16)0.f;
            }
            found.add(w, sees);
        }
        if (part) {
            reinterpret_cast<float4v*>(part)[nt * 64 + lane] += found.sum();
        } else if (row.head >= 0) {
            const int64_t at = (S.q0 + row.query) * A.o_ts + (int64_t)(kv * A.gqa + row.head) * A.o_hs;
            add_to_out4(A.out, A.out_fp32, at + 16 * nt + 4 * j, found.sum());
        }
    }
}

// One workgroup: WM * 16 R rows of one KV head against a range of keys; WT wavefronts share rows and take the tiles in turn.  An
// iteration loads NT tiles (K and V, 16 KiB each) into one half of LDS while the other is computed on.
// 32 rows a wavefront, so that an operand read from LDS serves two products, two workgroups a compute unit.  32,768 tokens x 64 heads: 16.9 to
// 18.7 ms on different cards, 940 to 1,040 TFLOP/s where an fp16 product of 8,192^3 reaches 1,290.  Matrix cores 47 % busy, vector ALUs
// 31 %, at the 2.0 GHz to which the card lowers its clock under this load; exponentials put beside products, a third wavefront a SIMD and
// wavefront priorities each changed that by 2 % or less.
template <int R, int WM, int WT, int NT>
__global__ __launch_bounds__(KVQ_PROMPT_THREADS, (R <= 2 && NT == 2 ? 2 : 1)) void kvq_prompt_kernel(const PromptArgs A) {
    constexpr int RB = 16 * R * WM, TT = NT / WT, STAGE = NT * 2 * KVQ_FLASH_TILE_BYTES;
    static_assert(WM * WT == 4 && WM * (WT / 2) * KVQ_JOIN_BYTES <= 2 * STAGE, "four wavefronts");
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE];  // [2][NT]{K tile, V tile}
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WT, wt = wave % WT;
    const int j = lane >> 4, n = lane & 15;
    const Item it = item_of(A, blockIdx.x);
    const PromptSeq& S = A.seq[it.seq];

    half8 q[R][4];
    int limit[R];  // keys that the row of this lane sees
    int most = 0, least = 0x7fffffff;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const Row row = row_of<RB>(A, S, it.block, wm * 16 * R + 16 * r + n);
        const bool real = row.head >= 0;
        limit[r] = real ? max(0, row.query + 1 + S.nk - S.nq) : S.nk;
        most = max(most, real ? limit[r] : 0);
        least = min(least, limit[r]);
        const _Float16* src = A.q + (int64_t)(S.q0 + (real ? row.query : 0)) * A.q_ts + (int64_t)(it.kv * A.gqa + (real ? row.head : 0)) * A.q_hs + 8 * j;
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) {
            u32x4 w = *reinterpret_cast<const u32x4*>(src + 32 * grp);
            w ^= A.flip;
            if (!real) w = u32x4{0, 0, 0, 0};
            q[r][grp] = to_half8(w);
        }
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
    }
    most = __builtin_amdgcn_readfirstlane(most);    // of the wavefront's rows
    least = __builtin_amdgcn_readfirstlane(least);
    // the keys of the block: those of its last row (in flat blocks, which may begin with a later head's first rows, of any row)
    int tiles;
    {
        int last = S.nk;
        if (!S.flat) {
            const int per_head = S.blocks / A.gqa, ib = per_head - 1 - it.block / A.gqa;
            last = max(0, min(S.nq, (ib + 1) * RB) + S.nk - S.nq);
        }
        // (the compiler does not see that this is the same in all lanes; without it every load of the loop was issued in a loop of its
        // own over the lanes' descriptors, and the accumulators were copied once an iteration)
        tiles = __builtin_amdgcn_readfirstlane((last + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS);
    }
    const int per = (tiles + it.splits - 1) / it.splits, t0 = __builtin_amdgcn_readfirstlane(min(tiles, it.split * per)), t1 = min(tiles, t0 + per);

    State<R> st;
    st.clear();

    // loads: a wavefront's 64 lanes take eight half rows of K or four rows of V at a time, in an order in which eight neighbouring
    // lanes write 128 consecutive bytes of the tile in LDS
    const int k_n = (tid & 7) | ((tid >> 7) & 1) << 3, k_chunk = (tid >> 3) & 15;
    const int k_token = 8 * (k_n >> 2) + (k_n & 3);  // + 4 for the odd half tiles
    const int v_token = 8 * ((tid >> 7) & 1) + 4 * ((tid >> 6) & 1) + ((tid >> 1) & 3), v_chunk = ((tid >> 3) & 7) * 2 + (tid & 1);  // + 16
    const int k_at = k_chunk_at(k_token, k_chunk), v_at = v_chunk_at(v_token, v_chunk);
    constexpr int K_HALF = 4 * 64 * 16, V_HALF = 2 * 16 * 8;
    // rows of the sequence as buffers that begin with the iteration's first key and end with the sequence's last: rows beyond read zeros
    const uint8_t* const kp = reinterpret_cast<const uint8_t*>(A.k + (int64_t)S.k0 * A.k_ts + (int64_t)it.kv * A.k_hs);
    const uint8_t* const vp = reinterpret_cast<const uint8_t*>(A.v + (int64_t)S.k0 * A.v_ts + (int64_t)it.kv * A.v_hs);
    const int k_row = (int)A.k_ts * 2, v_row = (int)A.v_ts * 2;
    const int k_off = k_token * k_row + k_chunk * 16, v_off = v_token * v_row + v_chunk * 16;
    u32x4 kr[2 * NT], vr[2 * NT];
    const auto load = [&](int t) {
        const int tok = t * KVQ_TILE_TOKENS, behind = __builtin_amdgcn_readfirstlane(S.nk - 1 - tok);
        const auto buffer = [&](const uint8_t* base, int row) {
            const int64_t bytes = (int64_t)behind * row + 2 * KVQ_D;
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base + (int64_t)tok * row), 0, (int)min(bytes, (int64_t)0x7fffffff), 0x00020000);
        };
        const __amdgpu_buffer_rsrc_t kb = buffer(kp, k_row), vb = buffer(vp, v_row);
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
            kr[i] = __builtin_amdgcn_raw_buffer_load_b128(kb, k_off, ((i >> 1) * KVQ_TILE_TOKENS + 4 * (i & 1)) * k_row, 0);
            vr[i] = __builtin_amdgcn_raw_buffer_load_b128(vb, v_off, ((i >> 1) * KVQ_TILE_TOKENS + 16 * (i & 1)) * v_row, 0);
        }
    };
    const auto store = [&](int buf) {
        uint8_t* const at = lds + buf * STAGE;
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
            *reinterpret_cast<u32x4*>(at + (i >> 1) * (2 * KVQ_FLASH_TILE_BYTES) + k_at + (i & 1) * K_HALF) = kr[i];
            *reinterpret_cast<u32x4*>(at + (i >> 1) * (2 * KVQ_FLASH_TILE_BYTES) + KVQ_FLASH_TILE_BYTES + v_at + (i & 1) * V_HALF) = vr[i];
        }
    };

    // The pass over the tiles; returns whether every sum of values is finite.  APART: a range with a sum that is not is taken a second time, with
    // zeros in the place of infinite and NaN values of V (as a branch inside one pass it costs all the others sixty registers).  Such a value
    // reaches the sums of all rows of its tile, as zero times infinity those of rows that do not see it or whose weight for it
    // is rounded to zero.
    const auto pass = [&](auto apart) {
        constexpr bool APART = decltype(apart)::value;
        if (t0 < t1) {
            load(t0);
            store(0);
        }
        __syncthreads();
        int buf = 0;
        // the tiles that this wavefront's rows see; behind them it only loads (in a loop of its own: with the products under a condition in
        // one loop the accumulators were copied once an iteration)
        int t = t0;
        const auto next = [&](bool more) {
            if (more) {
                if (APART) load(t + NT);  // (here it need not be on its way meanwhile, and there are no registers for it)
                store(buf ^ 1);
            }
            __syncthreads();
            buf ^= 1;
            t += NT;
        };
        for (const int end = min(t1, (most + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS) - wt * TT; t < end;) {
            const bool more = t + NT < t1;
            if (!APART && more) load(t + NT);
            const int tok = (t + wt * TT) * KVQ_TILE_TOKENS;  // of this wavefront's tiles
            {
                const uint8_t* const kt = lds + buf * STAGE + wt * TT * (2 * KVQ_FLASH_TILE_BYTES);
                const uint8_t* const vt = kt + KVQ_FLASH_TILE_BYTES;
                float4v s[R][TT][2];
#pragma unroll
                for (int x = 0; x < TT; ++x)
#pragma unroll
                    for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
                        for (int r = 0; r < R; ++r) s[r][x][sub] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int grp = 0; grp < 4; ++grp) {
                            const half8 a = to_half8(*reinterpret_cast<const u32x4*>(kt + x * (2 * KVQ_FLASH_TILE_BYTES) + ((sub * 4 + grp) * 64 + lane) * 16));
#pragma unroll
                            for (int r = 0; r < R; ++r) s[r][x][sub] = mma(a, q[r][grp], s[r][x][sub]);
                        }
                    }
                if constexpr (!APART) {  // operands are read four ahead of their products
                    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                    for (int g = 0; g < 8 * TT - 4; ++g) {
                        __builtin_amdgcn_sched_group_barrier(0x008, R, 0);
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    }
                    __builtin_amdgcn_sched_group_barrier(0x008, 4 * R, 0);
                }
                // behind the causal border of some row, beyond the last key or beyond the range
                const bool masked = min(least, t1 * KVQ_TILE_TOKENS) < tok + TT * KVQ_TILE_TOKENS;
                if (masked) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int end = min(limit[r], t1 * KVQ_TILE_TOKENS) - tok - 8 * j;
#pragma unroll
                        for (int x = 0; x < TT; ++x)
#pragma unroll
                            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    if (x * KVQ_TILE_TOKENS + 4 * sub + i >= end) s[r][x][sub][i] = -INFINITY;
                    }
                }
                uint32_t p[R][TT][4];
#pragma unroll
                for (int r = 0; r < R; ++r) softmax_group<R, TT, false, true>(st, r, s[r], A.scale_log2, A.lse != nullptr, p[r]);
#pragma unroll
                for (int x = 0; x < TT; ++x)
#pragma unroll
                    for (int nt = 0; nt < 8; ++nt) {
                        half8 a = read_v(vt + x * (2 * KVQ_FLASH_TILE_BYTES), nt, lane);
                        if (APART) a = to_half8(finite_only(__builtin_bit_cast(u32x4, a)));
#pragma unroll
                        for (int r = 0; r < R; ++r) st.o[r][nt] = mma(a, to_half8(p[r][x]), st.o[r][nt]);
                    }
                if constexpr (!APART) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 8, 1);
#pragma unroll
                    for (int g = 0; g < 8 * TT - 4; ++g) {
                        __builtin_amdgcn_sched_group_barrier(0x008, R, 1);
                        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
                    }
                    __builtin_amdgcn_sched_group_barrier(0x008, 4 * R, 1);
                }
            }
            next(more);
        }
        while (t < t1) {
            const bool more = t + NT < t1;
            if (!APART && more) load(t + NT);
            next(more);
        }
        float zero = 0.f;  // (times zero a sum is zero, or NaN if it is not finite)
        if (!APART) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) zero = fmaf(st.o[r][nt][i], 0.f, zero);
        }
        return zero == 0.f;
    };
    const bool apart = __builtin_amdgcn_readfirstlane(__syncthreads_or(pass(std::false_type{}) ? 0 : 1)) != 0;
    if (apart) {
        st.clear();
        pass(std::true_type{});
    }
    if constexpr (WT > 1) join_waves<R, WM, WT>(st, lds, wm, wt, lane);
    if (WT > 1 && wt > 0) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (it.splits > 1) {
            const int64_t group = parts_of<RB>(S, it.kv, it.block) + it.split * (RB / 16) + wm * R + r;
            store_partial(st, r, A.part + group * (KVQ_PART_BYTES / 4), lane);
            continue;
        }
        const float l = quarters_sum(st.l[r]), fine = quarters_sum(st.fine[r]);
        const Row row = row_of<RB>(A, S, it.block, wm * 16 * R + 16 * r + n);
        if (row.head < 0) continue;
        const float inv = inverse_of(l);
        const int head = it.kv * A.gqa + row.head;
        const int64_t tok = S.q0 + row.query, at = tok * A.o_ts + (int64_t)head * A.o_hs;
        void* const dst = A.out_fp32 ? static_cast<void*>(static_cast<float*>(A.out) + at) : static_cast<void*>(static_cast<_Float16*>(A.out) + at);
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) store_out4(dst, A.out_fp32, 16 * nt + 4 * j, st.o[r][nt] * inv);
        if (A.lse && j == 0) A.lse[(int64_t)head * A.lse_hs + tok] = fine == 0.f ? -INFINITY : (st.m[r] + __builtin_amdgcn_logf(fine)) * 0.69314718055994530942f;
    }
    if (apart) {
#pragma unroll 1
        for (int r = 0; r < R; ++r) {
            const int64_t group = parts_of<RB>(S, it.kv, it.block) + it.split * (RB / 16) + wm * R + r;
            add_nonfinite(A, S, it.kv, row_of<RB>(A, S, it.block, wm * 16 * R + 16 * r + n), t0, t1,
                          it.splits > 1 ? A.part + group * (KVQ_PART_BYTES / 4) : nullptr, lane);
        }
    }
}

// Joins the ranges of keys of one group of 16 rows, 32 channels a workgroup.  RB: rows of a block.
template <int RB>
__global__ __launch_bounds__(512) void kvq_prompt_merge_kernel(const PromptArgs A) {
    __shared__ JoinLds lds;
    const int lane = threadIdx.x & 63, j = lane >> 4, n = lane & 15;
    const int pair = blockIdx.x & 3, rg = (blockIdx.x >> 2) % (RB / 16), id = (blockIdx.x >> 2) / (RB / 16);
    int q = 0;
    for (int step = KVQ_PROMPT_SEQS / 2; step; step >>= 1)
        if (q + step < A.n_seqs && A.seq[q + step].merge0 <= id) q += step;
    const PromptSeq& S = A.seq[q];
    const int at = id - S.merge0, kv = at % A.n_kv, block = S.whole + at / A.n_kv;
    const float* part = A.part + (parts_of<RB>(S, kv, block) + rg) * (KVQ_PART_BYTES / 4);
    Joined x;
    if (!join_partials(lds, part, (int64_t)(RB / 16) * (KVQ_PART_BYTES / 4), S.splits, pair, x)) return;
    const Row row = row_of<RB>(A, S, block, rg * 16 + n);
    if (row.head < 0) return;
    const int head = kv * A.gqa + row.head;
    const int64_t tok = S.q0 + row.query, to = tok * A.o_ts + (int64_t)head * A.o_hs;
    void* const dst = A.out_fp32 ? static_cast<void*>(static_cast<float*>(A.out) + to) : static_cast<void*>(static_cast<_Float16*>(A.out) + to);
    store_out4(dst, A.out_fp32, 16 * x.nt + 4 * j, x.o * inverse_of(x.l));
    if (A.lse && x.nt == 0 && j == 0) A.lse[(int64_t)head * A.lse_hs + tok] = x.fine == 0.f ? -INFINITY : (x.m + __builtin_amdgcn_logf(x.fine)) * 0.69314718055994530942f;
}

// ---- host side: which sequences share a launch, their blocks and ranges

// Kernels by the rows of a block.  Few rows leave wavefronts over, which then share the rows and take the tiles in turn.
struct Variant {
    int rb, slots;  // slots: workgroups that the device takes at a time
    void (*kernel)(PromptArgs), (*merge)(PromptArgs);
};
#define KVQ_PROMPT_VARIANT(R, WM, WT, NT, SLOTS) {16 * R * WM, SLOTS, kvq_prompt_kernel<R, WM, WT, NT>, kvq_prompt_merge_kernel<16 * R * WM>}
const Variant kVariants[] = {KVQ_PROMPT_VARIANT(1, 1, 4, 4, 256), KVQ_PROMPT_VARIANT(2, 1, 4, 4, 256), KVQ_PROMPT_VARIANT(2, 2, 2, 4, 256),
                             KVQ_PROMPT_VARIANT(2, 4, 1, 2, 512)};
constexpr int kNumVariants = 4;
constexpr int kLeastTiles = 8;          // of a range of keys
constexpr int kMostSplits = KVQ_MOST_PARTS;
constexpr int kJoinTiles = 48;
constexpr int64_t kMostItems = (1 << 30) / KVQ_MOST_PARTS;  // row blocks x KV heads of a launch

int variant_of(int gqa, int nq) {
    const int64_t rows = (int64_t)gqa * nq;
    return rows <= 16 ? 0 : rows <= 32 ? 1 : rows <= 64 ? 2 : 3;
}
PromptSeq describe(int v, int gqa, int q0, int nq, int k0, int nk) {
    const int rb = kVariants[v].rb;
    PromptSeq s{};
    s.q0 = q0; s.nq = nq; s.k0 = k0; s.nk = nk;
    s.flat = nq <= rb ? 1 : 0;
    s.blocks = s.whole = s.flat ? (int)(((int64_t)gqa * nq + rb - 1) / rb) : gqa * ((nq + rb - 1) / rb);
    s.splits = 1;
    return s;
}

// Cuts blocks of a launch into ranges of keys where whole ones would leave the device idle: all of them if they are fewer than the
// workgroups it takes at a time, else those that are left over when it has been filled as often as they fill it, the last ones of the order
// (640 equal blocks: 512, then 128 in four ranges each, 904 -> 748 us), unless the fillings are many.
void cut_blocks(PromptArgs& A, int64_t items, int slots) {
    if (items >= 4 * (int64_t)slots) return;
    int64_t left = items % slots;
    if (2 * left > slots && items < slots) {
        // the first filling, more than half: in two where the longest blocks would take much longer than their share of all that is to do
        int64_t total = 0, longest = 0;
        for (int k = 0; k < A.n_seqs; ++k) {
            const PromptSeq& s = A.seq[k];
            const int64_t tiles = (s.nk + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS;
            total += (int64_t)A.n_kv * s.blocks * (s.flat ? tiles : std::max<int64_t>(0, tiles - s.nq / 2 / KVQ_TILE_TOKENS));
            longest = std::max(longest, tiles);
        }
        // (440 blocks of up to 219 tiles 172 -> 156 us, 275 of up to 134 118 -> 102; 448 of up to 128 110 -> 117)
        if (longest < (3 * items <= 2 * slots ? 96 : 160) || 2 * longest * slots < 3 * total) return;
        for (int k = 0; k < A.n_seqs; ++k)
            if (2 * ((A.seq[k].nk + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS) > longest) {
                A.seq[k].splits = 2;
                A.seq[k].whole = 0;
            }
        return;
    }
    if (2 * left > slots || left == 0) return;
    const int64_t want = std::min<int64_t>(slots / left, kMostSplits);
    for (int k = A.n_seqs - 1; k >= 0 && left > 0; --k) {
        PromptSeq& s = A.seq[k];
        const int64_t mine = std::min<int64_t>(s.blocks, (left + A.n_kv - 1) / A.n_kv);
        left -= mine * A.n_kv;
        const int tiles = (s.nk + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS;
        s.splits = (int)std::max<int64_t>(1, std::min<int64_t>(want, tiles / kLeastTiles));
        if (s.splits > 1) s.whole = s.blocks - (int)mine;
    }
}

// Calls launch(variant, args, workgroups, blocks in ranges) for every launch of the call, with everything in args that depends on the
// lengths; workspace: bytes there are (0: no ranges).  Returns the most bytes of workspace a launch uses, -1 if the call is
// too large, -2 if a launch fails.
template <class Launch>
int64_t plan_prompt(PromptArgs& A, const int32_t* qb, const int32_t* kb, int n_seqs, int64_t workspace, Launch launch) {
    int64_t most = 0;
    // Few sequences of few rows go with the largest ones' launch where they end before those (a launch of their own and one that joins its ranges
    // take longer than what they add there): up to kJoinTiles tiles for each workgroup that the device takes at a time.  Nine sequences of 1 to
    // 3,372 keys 41.5 -> 20.4 us, sixteen decode steps beside a prompt of 2,000 tokens 76.6 -> 59.6, 62 beside a chunk of 512 138 -> 114.
    int largest = 0, longest = 0;
    for (int i = 0; i < n_seqs; ++i) {
        const int nq = qb[i + 1] - qb[i], v = nq ? variant_of(A.gqa, nq) : 0;
        if (v > largest) longest = 0;
        largest = std::max(largest, v);
        if (nq && v == largest) longest = std::max(longest, kb[i + 1] - kb[i]);
    }
    int64_t small = 0;
    for (int i = 0; i < n_seqs; ++i) {
        const int nq = qb[i + 1] - qb[i], nk = kb[i + 1] - kb[i];
        if (nq && nk <= longest && variant_of(A.gqa, nq) < largest) small += (int64_t)A.n_kv * ((nk + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS);
    }
    const bool together = small <= kJoinTiles * (int64_t)kVariants[largest].slots;
    const auto variant = [&](int nq, int nk) {
        const int v = variant_of(A.gqa, nq);
        return together && nk <= longest ? largest : v;
    };
    for (int v = 0; v < kNumVariants; ++v) {
        for (int i = 0; i < n_seqs;) {
            A.n_seqs = 0;
            int64_t items = 0;
            for (; i < n_seqs && A.n_seqs < KVQ_PROMPT_SEQS; ++i) {
                const int nq = qb[i + 1] - qb[i], nk = kb[i + 1] - kb[i];
                if (!nq || variant(nq, nk) != v) continue;
                A.seq[A.n_seqs] = describe(v, A.gqa, qb[i], nq, kb[i], nk);
                items += (int64_t)A.n_kv * A.seq[A.n_seqs++].blocks;
            }
            if (!A.n_seqs) continue;
            if (items > kMostItems) return -1;
            // the longest first: what starts last ends last
            std::sort(A.seq, A.seq + A.n_seqs, [](const PromptSeq& a, const PromptSeq& b) { return a.nk != b.nk ? a.nk > b.nk : a.q0 < b.q0; });
            cut_blocks(A, items, kVariants[v].slots);
            for (int pass = 0;; ++pass) {  // a second time without ranges where the workspace does not hold their partial results
                int64_t at = 0, groups = 0, merges = 0;
                for (int k = 0; k < A.n_seqs; ++k) {
                    PromptSeq& s = A.seq[k];
                    if (pass) s.whole = s.blocks;
                    s.item0 = (int32_t)at;
                    s.part0 = (int32_t)groups;
                    s.merge0 = (int32_t)merges;
                    const int64_t cut = (int64_t)A.n_kv * (s.blocks - s.whole);
                    at += (int64_t)A.n_kv * s.whole + cut * s.splits;
                    groups += cut * s.splits * (kVariants[v].rb / 16);
                    merges += cut;
                }
                const int64_t bytes = groups * KVQ_PART_BYTES;
                if (bytes > workspace && !pass) continue;
                most = std::max(most, bytes);
                if (!launch(v, A, (int)at, (int)merges)) return -2;
                break;
            }
        }
    }
    return most;
}

bool lengths_ok(const int32_t* qb, const int32_t* kb, int n_seqs) {
    if (!qb || n_seqs < 1 || n_seqs > (1 << 20)) return false;
    for (const int32_t* b : {qb, kb}) {
        if (b[0] < 0 || b[n_seqs] > INT32_MAX - 4096) return false;  // (rounded up to tiles and blocks they stay below 2^31)
        for (int i = 0; i < n_seqs; ++i)
            if (b[i + 1] < b[i]) return false;
    }
    return true;
}
// Whether no two of the rows t * token + h * head, 128 long each, share an element (0 <= t < n, 0 <= h < heads; strides of 128 or more).
bool rows_apart(int64_t token, int64_t head, int64_t n, int64_t heads) {
    if (n <= 1 || heads <= 1 || token >= (heads - 1) * head + KVQ_D || head >= (n - 1) * token + KVQ_D) return true;
    for (int64_t h = 1; h < heads; ++h)  // the tokens that h heads on comes next to
        for (int64_t t = h * head / token, k = 0; k < 2; ++k, ++t)
            if (t < n && std::abs(h * head - t * token) < KVQ_D) return false;
    return true;
}
bool heads_ok(int n_q, int n_kv) { return n_kv >= 1 && n_kv <= 65535 && n_q >= 1 && n_q % n_kv == 0 && n_q / n_kv <= KVQ_MAX_GQA; }

}  // namespace

extern "C" {

uint64_t kvq_prompt_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, const int32_t* q_begin_host, const int32_t* k_begin_host,
                                    int32_t n_seqs) {
    if (!k_begin_host) k_begin_host = q_begin_host;
    if (!heads_ok(n_q_heads, n_kv_heads) || !lengths_ok(q_begin_host, k_begin_host, n_seqs)) return 0;
    PromptArgs A{};
    A.gqa = n_q_heads / n_kv_heads;
    A.n_kv = n_kv_heads;
    const int64_t most = plan_prompt(A, q_begin_host, k_begin_host, n_seqs, INT64_MAX, [](int, const PromptArgs&, int, int) { return true; });
    return most < 0 ? 0 : (uint64_t)most;
}

kvq_status_t kvq_prompt_attention(const kvq_prompt_t* d, const void* q_dev, const void* k_dev, const void* v_dev, void* out_dev,
                                  float* lse_dev, const int32_t* q_begin_host, const int32_t* k_begin_host, int32_t n_seqs,
                                  void* workspace_dev, uint64_t workspace_bytes, void* hip_stream) {
    if (!k_begin_host) k_begin_host = q_begin_host;
    if (!d || !heads_ok(d->n_q_heads, d->n_kv_heads) || !lengths_ok(q_begin_host, k_begin_host, n_seqs)) return KVQ_E_INVALID;
    if (!std::isfinite(d->softmax_scale)) return KVQ_E_INVALID;
    const bool any_q = q_begin_host[n_seqs] > q_begin_host[0], any_k = k_begin_host[n_seqs] > k_begin_host[0];
    if (!any_q) return KVQ_OK;
    if (!q_dev || !out_dev || (any_k && (!k_dev || !v_dev))) return KVQ_E_INVALID;
    for (const void* p : {q_dev, k_dev, v_dev, static_cast<const void*>(out_dev), static_cast<const void*>(workspace_dev)})
        if (reinterpret_cast<uintptr_t>(p) & 15u) return KVQ_E_INVALID;
    if (reinterpret_cast<uintptr_t>(lse_dev) & 3u) return KVQ_E_INVALID;
    // 16-byte loads and stores; rows of the output must not share memory
    for (int64_t s : {d->q_token_stride, d->q_head_stride, d->k_token_stride, d->k_head_stride, d->v_token_stride, d->v_head_stride,
                      d->out_token_stride, d->out_head_stride})
        if (s < 0 || s % 8 != 0 || s >= (1ll << 40)) return KVQ_E_INVALID;
    // the kernel addresses the rows of an iteration with 32 bits, and rows beyond the last key by where they would begin
    for (int64_t s : {d->k_token_stride, d->v_token_stride})
        if (s < KVQ_D || s >= (1ll << 22)) return KVQ_E_INVALID;
    if (d->out_token_stride < KVQ_D || (d->n_q_heads > 1 && d->out_head_stride < KVQ_D)) return KVQ_E_INVALID;
    if (!rows_apart(d->out_token_stride, d->out_head_stride, q_begin_host[n_seqs] - q_begin_host[0], d->n_q_heads)) return KVQ_E_INVALID;

    PromptArgs A{};
    A.q = static_cast<const _Float16*>(q_dev);
    A.k = static_cast<const _Float16*>(k_dev);
    A.v = static_cast<const _Float16*>(v_dev);
    A.out = out_dev;
    A.lse = lse_dev;
    A.part = static_cast<float*>(workspace_dev);
    A.q_ts = d->q_token_stride; A.q_hs = d->q_head_stride;
    A.k_ts = d->k_token_stride; A.k_hs = d->k_head_stride;
    A.v_ts = d->v_token_stride; A.v_hs = d->v_head_stride;
    A.o_ts = d->out_token_stride; A.o_hs = d->out_head_stride;
    A.lse_hs = q_begin_host[n_seqs];
    A.gqa = d->n_q_heads / d->n_kv_heads;
    A.n_kv = d->n_kv_heads;
    A.out_fp32 = d->out_is_fp32 ? 1 : 0;
    const float scale = d->softmax_scale != 0.f ? d->softmax_scale : 1.0f / std::sqrt((float)KVQ_D);
    A.scale_log2 = std::fabs(scale) * 1.44269504088896340736f;
    A.flip = scale < 0.f ? 0x80008000u : 0u;
    // nothing is enqueued of a call whose last launches would be too large
    int64_t items = 0;
    for (int i = 0; i < n_seqs; ++i) {
        const int nq = q_begin_host[i + 1] - q_begin_host[i];
        if (nq) items += (int64_t)A.n_kv * describe(variant_of(A.gqa, nq), A.gqa, 0, nq, 0, 0).blocks;
    }
    if (items > kMostItems && plan_prompt(A, q_begin_host, k_begin_host, n_seqs, 0, [](int, const PromptArgs&, int, int) { return true; }) < 0) return KVQ_E_INVALID;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int64_t got = plan_prompt(A, q_begin_host, k_begin_host, n_seqs, workspace_dev ? (int64_t)std::min<uint64_t>(workspace_bytes, INT64_MAX) : 0,
                                    [&](int v, const PromptArgs& args, int wgs, int merges) {
        const Variant& V = kVariants[v];
        hipLaunchKernelGGL(V.kernel, dim3((unsigned)wgs), dim3(KVQ_PROMPT_THREADS), 0, s, args);
        if (hipGetLastError() != hipSuccess) return false;
        if (!merges) return true;
        hipLaunchKernelGGL(V.merge, dim3((unsigned)merges * (unsigned)(V.rb / 16 * 4)), dim3(512), 0, s, args);
        return hipGetLastError() == hipSuccess;
    });
    return got == -1 ? KVQ_E_INVALID : got < 0 ? KVQ_E_HIP : KVQ_OK;
}

}  // extern "C"
