// Attention of drafted tokens (a tree of them, or any set with a mask among themselves) over a block's cache and over one another
// (kvq_tree_attention).
//
// The rows of one (sequence, KV head) unit are its g query heads times the nodes.  A workgroup takes a block of rows and a range of the
// cache's tiles.  Four wavefronts fetch a tile each, unpack it once and leave it in LDS in operand order, from where every wavefront of the
// block multiplies it: K as its codes, V as code * S + Z in one fused step, rounded to fp16.  Many rows share the work of one
// unpacking, which the decode kernel, with at most 16 rows, avoids instead.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "../../include/kvq.h"
#include "kvq_cache.h"
#include "kvq_attention_body.h"
#include "kvq_flash.h"

namespace {

using namespace kvq_flash;

#define KVQ_TREE_V KVQ_FLASH_TILE_BYTES                 // one tile in LDS: K operands, V operands,
#define KVQ_TREE_K_LOW (2 * KVQ_FLASH_TILE_BYTES)       // in the integer 16-bit tier the low bytes of K

struct TreeArgs {
    const uint8_t* arena;
    const KvqPageDesc* table;
    const _Float16 *q, *k, *v;
    const uint32_t* mask;   // [sequence or 1][node][words]
    const float* lambda;    // [n_kv_heads][128] or null
    void* out;
    float* part;            // [unit][block][split][16 rows of it]
    int64_t mask_seq;       // words from one sequence's mask to the next's, 0: one for all
    int32_t n_tokens, n_tiles, tpp;
    uint32_t tpp_magic;
    int32_t units, n_kv, gqa, nodes, words, rows;
    int32_t blocks, splits;  // row blocks of a unit, ranges (partial results of a block, if more than one)
    int32_t per;             // tiles of a range
    int32_t node_tiles;      // what the nodes count for, in tiles: they come first in the line that is cut into ranges, in range 0
    int32_t groups;          // of 16 rows in a block
    int32_t out_fp32;
    float scale_log2;
    uint32_t flip;
};

// Eight 16-bit values in order -> the pairs (v, v + 4) in which codes are unpacked.
__device__ inline u32x4 paired(u32x4 w) {
    return u32x4{__builtin_amdgcn_perm(w.z, w.x, 0x05040100u), __builtin_amdgcn_perm(w.z, w.x, 0x07060302u),
                 __builtin_amdgcn_perm(w.w, w.y, 0x05040100u), __builtin_amdgcn_perm(w.w, w.y, 0x07060302u)};
}
__device__ inline uint32_t fma2(uint32_t c, uint32_t s, uint32_t z) {
    const half2v x = __builtin_elementwise_fma(__builtin_bit_cast(half2v, c), __builtin_bit_cast(half2v, s), __builtin_bit_cast(half2v, z));
    return __builtin_bit_cast(uint32_t, x);
}
// Whether the largest code of some group of a tile overflows (or its S or Z is not finite).  meta: the lane's 16 bytes of the
// tile's metadata, of which rows 0 and 2 of 16 lanes hold scales and rows 1 and 3 the zero points that belong to them.
__device__ inline bool overflows(u32x4 meta, int levels) {
    const half2v top = {(_Float16)(float)levels, (_Float16)(float)levels}, zero = {(_Float16)0.f, (_Float16)0.f};
    half2v seen = zero;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const auto r = __builtin_amdgcn_permlane16_swap(meta[e], meta[e], false, false);
        const uint32_t s = r[0], z = r[1];
        seen += __builtin_elementwise_fma(top, __builtin_bit_cast(half2v, s), __builtin_bit_cast(half2v, z)) * zero;
    }
    return __any((__builtin_bit_cast(uint32_t, seen) & 0x7fff7fffu) != 0);
}

// Behind such a tile's values: what the rounded scale has carried beyond the largest fp16 becomes the largest, as every other value stays
// within half a step of its scale of what was stored.  to: the lane's values of V; meta: scales and zero points of V.
__device__ inline void clamp_values(uint8_t* to, const uint8_t* meta, int lane) {
#pragma unroll 1
    for (int nt = 0; nt < 8; ++nt) {
        const u32x4 s = *reinterpret_cast<const u32x4*>(meta + (nt >> 1) * 64 + (lane >> 4) * 16), z = *reinterpret_cast<const u32x4*>(meta + 256 + (nt >> 1) * 64 + (lane >> 4) * 16);
        u32x4 y = *reinterpret_cast<const u32x4*>(to + (nt * 64 + lane) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < 32; h += 16) {
                const uint32_t inf = 0x7c00u << h;
                if ((y[e] & (0x7fffu << h)) == inf && (s[e] & inf) != inf && (z[e] & inf) != inf) y[e] -= 1u << h;
            }
        *reinterpret_cast<u32x4*>(to + (nt * 64 + lane) * 16) = y;
    }
}
// One tile on its way through registers: the packed strings of a lane and its share of the metadata.
struct Fetched {
    uint32_t k[32], v[32];
    u32x4 meta;
    uint32_t bits;
};

template <int NDW>
__device__ inline void fetch_string(const uint8_t* tile, uint32_t lane_off, uint32_t (&w)[32]) {
#pragma unroll
    for (int c = 0; c < NDW / 4; ++c) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(tile + lane_off + c * 1024);
        w[4 * c] = x.x; w[4 * c + 1] = x.y; w[4 * c + 2] = x.z; w[4 * c + 3] = x.w;
    }
}
template <int B>
__device__ inline void fetch_codes(Fetched& f, const uint8_t* code, uint32_t lane_off) {
    fetch_string<2 * B>(code, lane_off, f.k);
    fetch_string<2 * B>(code + 512u * B, lane_off, f.v);
}
// The page entry of a tile.  It is asked for an iteration ahead of its use: a trip to memory in front of the tile's own.
// (By scalar loads: nothing writes the table while the kernel runs, and a vector load under way holds up what reuses its registers.)
__device__ inline KvqPageDesc entry_of(const TreeArgs& A, int tile) {
    typedef const __attribute__((address_space(4))) uint32_t* constant;
    const constant e = reinterpret_cast<constant>(reinterpret_cast<uintptr_t>(A.table)) +
                       4 * __builtin_amdgcn_readfirstlane(kvq_dev::div_magic(tile, A.tpp, A.tpp_magic));
    return KvqPageDesc{e[0], e[1], e[2], e[3]};
}
template <bool I16>
__device__ inline void fetch_tile(Fetched& f, const TreeArgs& A, const KvqPageDesc& d, int unit, int tile, uint32_t lane_off) {
    const int page = kvq_dev::div_magic(tile, A.tpp, A.tpp_magic), tip = tile - page * A.tpp;
    const uint32_t bits = __builtin_amdgcn_readfirstlane(d.bits);
    const uint64_t slot = (uint64_t)unit * A.tpp + tip;
    const uint8_t* code = A.arena + (uint64_t)__builtin_amdgcn_readfirstlane(d.code_off256) * 256u + slot * (1024u * bits);
    const uint8_t* meta = A.arena + (uint64_t)__builtin_amdgcn_readfirstlane(d.meta_off256) * 256u + slot * KVQ_META_TILE_BYTES;
    f.bits = bits;
    if (I16 || bits < 16) f.meta = *reinterpret_cast<const u32x4*>(meta + lane_off);
    if (bits == 2) fetch_codes<2>(f, code, lane_off);
    else if (bits == 4) fetch_codes<4>(f, code, lane_off);
    else if (bits == 8) fetch_codes<8>(f, code, lane_off);
    else fetch_codes<16>(f, code, lane_off);
}

// The values of a fetched tile into a slot of LDS, operands in (v, v + 4) pairs.  meta_lds: 1 KiB of the wavefront's own.
// K stays codes (exact in fp16, in (v, v + 4) pairs): its scales and zero points are applied to the sums of 32 channels, in fp32.
// (With K_hat rounded to fp16 as V_hat is, keys with channels 20 times the others moved scores by 5e-4, three times what all else does.)
template <int B>
__device__ inline void expand_v(const Fetched& f, uint8_t* slot, const uint8_t* meta_lds, int lane) {
    const int j = lane >> 4;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const u32x4 s = *reinterpret_cast<const u32x4*>(meta_lds + 512 + g * 64 + j * 16), z = *reinterpret_cast<const u32x4*>(meta_lds + 768 + g * 64 + j * 16);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 c = __builtin_bit_cast(u32x4, dq_piece<B>(f.v, 2 * g + h));
            *reinterpret_cast<u32x4*>(slot + KVQ_TREE_V + ((2 * g + h) * 64 + lane) * 16) =
                u32x4{fma2(c.x, s.x, z.x), fma2(c.y, s.y, z.y), fma2(c.z, s.z, z.z), fma2(c.w, s.w, z.w)};
        }
    }
}
template <int B>
__device__ inline void expand_codes(const Fetched& f, uint8_t* slot, const uint8_t* meta_lds, int lane) {
#pragma unroll
    for (int p = 0; p < 8; ++p) *reinterpret_cast<u32x4*>(slot + (p * 64 + lane) * 16) = __builtin_bit_cast(u32x4, dq_piece<B>(f.k, p));
    expand_v<B>(f, slot, meta_lds, lane);
    if (overflows(f.meta, (1 << B) - 1)) clamp_values(slot + KVQ_TREE_V, meta_lds + 512, lane);
}
// Integer 16-bit tier: of K both byte planes as integers and as 256ths of them (both exact); of V the values, whose product needs 32 bits.
__device__ inline uint32_t value16(uint32_t hi, uint32_t lo, int byte, float s, float z) {
    const float x = fmaf((float)(((hi >> (8 * byte)) & 255u) << 8 | ((lo >> (8 * byte)) & 255u)), s, z);
    return (uint32_t)kvq_dev::f2h_rn(fabsf(x) < INFINITY ? fminf(fmaxf(x, -65504.f), 65504.f) : x);  // (as clamp_values)
}
__device__ inline void values_of_planes(const uint32_t (&v)[32], const uint8_t* meta, uint8_t* to, int lane) {  // meta: scales and zero points of V
    const int j = lane >> 4;
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
        const u32x4 s = *reinterpret_cast<const u32x4*>(meta + (nt >> 1) * 64 + j * 16), z = *reinterpret_cast<const u32x4*>(meta + 256 + (nt >> 1) * 64 + j * 16);
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = value16(v[2 * nt], v[16 + 2 * nt], e, mixf(s[e], 0), mixf(z[e], 0)) |
                   value16(v[2 * nt + 1], v[17 + 2 * nt], e, mixf(s[e], 1), mixf(z[e], 1)) << 16;
        *reinterpret_cast<u32x4*>(to + (nt * 64 + lane) * 16) = w;
    }
}
__device__ inline void expand_planes(const Fetched& f, uint8_t* slot, const uint8_t* meta_lds, int lane) {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        *reinterpret_cast<u32x4*>(slot + (p * 64 + lane) * 16) = __builtin_bit_cast(u32x4, dq_piece<8>(f.k, p));
        *reinterpret_cast<u32x4*>(slot + KVQ_TREE_K_LOW + (p * 64 + lane) * 16) = __builtin_bit_cast(u32x4, dq_piece_frac(f.k + 16, p));
    }
    values_of_planes(f.v, meta_lds + 512, slot + KVQ_TREE_V, lane);
}
// A raw tile has scales of one and zero points of zero.
template <bool I16>
__device__ inline void expand_tile(const Fetched& f, uint8_t* slot, uint8_t* meta_lds, int lane) {
    u32x4 meta = f.meta;
    if (!I16 && f.bits == 16) meta = lane < 16 ? u32x4{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u} : u32x4{0u, 0u, 0u, 0u};
    *reinterpret_cast<u32x4*>(meta_lds + lane * 16) = meta;
    wave_lds_sync();
    if (f.bits == 2) {
        expand_codes<2>(f, slot, meta_lds, lane);
    } else if (f.bits == 4) {
        expand_codes<4>(f, slot, meta_lds, lane);
    } else if (f.bits == 8) {
        expand_codes<8>(f, slot, meta_lds, lane);
    } else if constexpr (I16) {
        expand_planes(f, slot, meta_lds, lane);
    } else {
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            *reinterpret_cast<u32x4*>(slot + (p * 64 + lane) * 16) = paired(u32x4{f.k[4 * p], f.k[4 * p + 1], f.k[4 * p + 2], f.k[4 * p + 3]});
            *reinterpret_cast<u32x4*>(slot + KVQ_TREE_V + (p * 64 + lane) * 16) = paired(u32x4{f.v[4 * p], f.v[4 * p + 1], f.v[4 * p + 2], f.v[4 * p + 3]});
        }
    }
}

// Query operands in pairs.  For the cache they are multiplied by the block's key factors (fp32 product, rounded to fp16, as for a decode
// step); against the nodes' own keys they are what they are.  The rows of a wavefront's groups are `step` rows apart.
template <int R>
__device__ inline void ask_queries(u32x4 (&w)[R][4], const TreeArgs& A, int unit, int row0, int step, int lane) {  // (all loads first: they are the start of a chain)
    const int j = lane >> 4, n = lane & 15;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + step * r + n;
        const _Float16* src = A.q + ((int64_t)unit * A.rows + min(row, A.rows - 1)) * KVQ_D + 8 * j;
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) w[r][grp] = *reinterpret_cast<const u32x4*>(src + 32 * grp);
    }
}
template <int R>
__device__ inline void set_queries(half8 (&q)[R][4], u32x4 (&w)[R][4], const TreeArgs& A, int unit, int row0, int step, bool factors, int lane) {
    const int j = lane >> 4, n = lane & 15;
    if (factors && A.lambda) {
        const float* lam = A.lambda + (size_t)(unit % A.n_kv) * KVQ_D + 8 * j;
        kvq_dev::f32x4 l[4][2];
#pragma unroll
        for (int grp = 0; grp < 4; ++grp)
#pragma unroll
            for (int h = 0; h < 2; ++h) l[grp][h] = *reinterpret_cast<const kvq_dev::f32x4_any*>(lam + 32 * grp + 4 * h);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int grp = 0; grp < 4; ++grp)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[r][grp][e] = kvq_dev::scale_pair(w[r][grp][e], l[grp][e >> 1][(2 * e) & 3], l[grp][e >> 1][(2 * e + 1) & 3]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool real = row0 + step * r + n < A.rows;
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) q[r][grp] = to_half8(real ? paired(w[r][grp] ^ A.flip) : u32x4{0, 0, 0, 0});
    }
}
template <int R>
__device__ inline void load_queries(half8 (&q)[R][4], const TreeArgs& A, int unit, int row0, int step, bool factors, int lane) {
    u32x4 w[R][4];
    ask_queries<R>(w, A, unit, row0, step, lane);
    set_queries<R>(q, w, A, unit, row0, step, factors, lane);
}
// Sums of q over the channels of each group, for the zero points: a high part in lane quarter 0, what it leaves in quarter 1, the B operand
// of a product with 16 channels whose A operand repeats a token's four zero points.  A query so large that a sum passes the fp16
// range is made smaller by 2^10, and its scale, of the lane's row, grows by that (rows have scales of their own: the small components of other
// queries would become subnormal).
template <int R>
__device__ inline void sum_queries(half8 (&q)[R][4], half4 (&qs)[R], float (&scale)[R], float scale_log2, int lane) {
    const int j = lane >> 4;
    half8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (_Float16)1.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float sum[4];
        bool large = false;
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) {
            sum[grp] = mma(ones, q[r][grp], float4v{0.f, 0.f, 0.f, 0.f})[0];  // (the same for every row of the result)
            large |= fabsf(sum[grp]) >= 65504.f;
        }
        scale[r] = scale_log2;
        if (__any(large)) {
            const float less = large ? 1.f / 1024.f : 1.f;
            if (large) scale[r] *= 1024.f;
#pragma unroll
            for (int grp = 0; grp < 4; ++grp) {
                sum[grp] *= less;
                q[r][grp] *= (_Float16)less;
            }
        }
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) {
            const _Float16 high = (_Float16)sum[grp], low = (_Float16)(sum[grp] - (float)high);
            qs[r][grp] = j == 0 ? high : j == 1 ? low : (_Float16)0.f;
        }
    }
}

// Scores of one tile of the cache in LDS for the first RR groups of a wavefront: sums of codes times queries over the channels of a scale, times it, plus
// the zero points' part.  SCALES: groups of channels of a token, 4, 2 or 1.
template <int RR, bool I16, int SCALES, int R>
__device__ inline void cache_scores(float4v (&s)[R][1][2], const half8 (&q)[R][4], const half4 (&qs)[R], const uint8_t* slot, const uint8_t* meta,
                                    bool planes, int lane) {
    const int j = lane >> 4, n = lane & 15;
    const float4v zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
        __builtin_amdgcn_sched_barrier(0);
        const int t = 8 * (n >> 2) + 4 * sub + (n & 3);
        const half4 z = __builtin_bit_cast(half4, *reinterpret_cast<const u32x2*>(meta + 256 + t * 8));
        uint32_t scale[8];  // of the quarter's four tokens of this half: two words of two groups each
        const u32x4 a0 = *reinterpret_cast<const u32x4*>(meta + j * 64 + sub * 32), a1 = *reinterpret_cast<const u32x4*>(meta + j * 64 + sub * 32 + 16);
        scale[0] = a0.x; scale[1] = a0.y; scale[2] = a0.z; scale[3] = a0.w;
        scale[4] = a1.x; scale[5] = a1.y; scale[6] = a1.z; scale[7] = a1.w;
        if (I16 && planes) {  // (times 256: the low bytes are 256ths; a scale is at most 2)
#pragma unroll
            for (int e = 0; e < 8; ++e) scale[e] = pk_mul(scale[e], 0x5c005c00u);
        }
#pragma unroll
        for (int r = 0; r < RR; ++r) s[r][0][sub] = mma16(z, qs[r], zero);
#pragma unroll
        for (int g = 0; g < SCALES; ++g) {
            float4v part[RR];
#pragma unroll
            for (int r = 0; r < RR; ++r) part[r] = zero;
#pragma unroll
            for (int grp = g * (4 / SCALES); grp < (g + 1) * (4 / SCALES); ++grp) {
                const half8 a = to_half8(*reinterpret_cast<const u32x4*>(slot + ((sub * 4 + grp) * 64 + lane) * 16));
#pragma unroll
                for (int r = 0; r < RR; ++r) part[r] = mma(a, q[r][grp], part[r]);
                if (I16 && planes) {
                    const half8 b = to_half8(*reinterpret_cast<const u32x4*>(slot + KVQ_TREE_K_LOW + ((sub * 4 + grp) * 64 + lane) * 16));
#pragma unroll
                    for (int r = 0; r < RR; ++r) part[r] = mma(b, q[r][grp], part[r]);
                }
            }
            constexpr int last = 4 / SCALES - 1;  // (the four scales of a token are equal within a group)
            const int at = g * (4 / SCALES) + last;
#pragma unroll
            for (int r = 0; r < RR; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[r][0][sub][i] = fmaf(mixf(scale[2 * i + (at >> 1)], at & 1), part[r][i], s[r][0][sub][i]);
        }
    }
}
// Scores of one tile of the nodes' keys.
template <int R>
__device__ inline void node_scores(float4v (&s)[R][1][2], const half8 (&q)[R][4], const uint8_t* slot, int lane) {
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][0][sub] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) {
            const half8 a = to_half8(*reinterpret_cast<const u32x4*>(slot + ((sub * 4 + grp) * 64 + lane) * 16));
#pragma unroll
            for (int r = 0; r < R; ++r) s[r][0][sub] = mma(a, q[r][grp], s[r][0][sub]);
        }
    }
}
template <int RR, int R>
__device__ inline void tile_products(State<R>& st, const uint32_t (&p)[R][1][4], const uint8_t* slot, int lane) {
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
        const half8 a = to_half8(*reinterpret_cast<const u32x4*>(slot + KVQ_TREE_V + (nt * 64 + lane) * 16));
#pragma unroll
        for (int r = 0; r < RR; ++r) st.o[r][nt] = mma(a, to_half8(p[r][0]), st.o[r][nt]);
    }
}

// What infinite and NaN values of the nodes add to a row that sees them, to what the same lanes have stored: a partial result or an output.
__device__ inline void add_nonfinite(const TreeArgs& A, int unit, int row, float* part, int lane) {
    const int j = lane >> 4, n = lane & 15, at_row = min(row, A.rows - 1);
    const uint32_t* const mask = A.mask + (int64_t)(unit / A.n_kv) * A.mask_seq + (int64_t)(at_row % A.nodes) * A.words;
    const uint16_t* const v = reinterpret_cast<const uint16_t*>(A.v) + (int64_t)unit * A.nodes * KVQ_D;
#pragma unroll 1
    for (int nt = 0; nt < 8; ++nt) {
        NonfiniteCount found;
#pragma unroll 1
        for (int node0 = 0; node0 < A.nodes; node0 += KVQ_TILE_TOKENS) {
            const uint32_t word = mask[node0 / KVQ_TILE_TOKENS];
            uint16_t w[8];
            half8 sees;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int node = node0 + 8 * j + e;
                w[e] = node < A.nodes ? v[(int64_t)node * KVQ_D + 16 * nt + n] : (uint16_t)0;
                sees[e] = ((word >> (8 * j + e)) & 1u) ? (_Float16)1.f : (_Float16)0.f;
            }
            found.add(w, sees);
        }
        if (part) reinterpret_cast<float4v*>(part)[nt * 64 + lane] += found.sum();
        else if (row < A.rows) add_to_out4(A.out, A.out_fp32, ((int64_t)unit * A.rows + row) * KVQ_D + 16 * nt + 4 * j, found.sum());
    }
}

// ---- many rows: wavefronts that share the unpacked tiles

// One of the operands of a tile on its way to the workgroup's staging area in LDS, past the registers: the lanes' packed strings of K or of V
// and 512 bytes of metadata (scales, zero points).  Strings of 16 bits are not staged, there is no room for them: they are
// loaded when they are unpacked.
#define KVQ_TREE_STAGE (KVQ_FLASH_TILE_BYTES / 2 + KVQ_META_TILE_BYTES / 2)
#define KVQ_TREE_STAGE_META (KVQ_FLASH_TILE_BYTES / 2)
struct Staged {
    const uint8_t* code;  // of 16 bits: where the strings are
    uint32_t bits;
};
__device__ inline void stage16(const uint8_t* from, uint8_t* to) {  // to: the wavefront's address, lane l writes 16 bytes at 16 l
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(reinterpret_cast<uintptr_t>(from)),
                                     (__attribute__((address_space(3))) uint32_t*)to, 16, 0, 0);
}
__device__ inline Staged stage_tile(const TreeArgs& A, const KvqPageDesc& d, int unit, int tile, int part, uint8_t* to, int lane) {
    const int page = kvq_dev::div_magic(tile, A.tpp, A.tpp_magic), tip = tile - page * A.tpp;
    const uint32_t bits = __builtin_amdgcn_readfirstlane(d.bits);
    const uint64_t slot = (uint64_t)unit * A.tpp + tip;
    const uint8_t* code = A.arena + (uint64_t)__builtin_amdgcn_readfirstlane(d.code_off256) * 256u + slot * (1024u * bits) + (uint32_t)part * 512u * bits;
    const uint8_t* meta = A.arena + (uint64_t)__builtin_amdgcn_readfirstlane(d.meta_off256) * 256u + slot * KVQ_META_TILE_BYTES + part * (KVQ_META_TILE_BYTES / 2);
    if (bits < 16)
        for (uint32_t c = 0; c < bits / 2; ++c) stage16(code + c * 1024 + lane * 16, to + c * 1024);
    if ((bits < 16 || __builtin_amdgcn_readfirstlane(d.int16)) && lane < 32) stage16(meta + lane * 16, to + KVQ_TREE_STAGE_META);
    return Staged{code, bits};
}
// Waits for what the wavefront has under way to LDS; a barrier that does not (it orders LDS alone).
__device__ inline void wait_staged() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int NDW>
__device__ inline void staged_string(const uint8_t* from, int lane, uint32_t (&w)[NDW]) {
#pragma unroll
    for (int c = 0; c < NDW / 4; ++c) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(from + (c * 64 + lane) * 16);
        w[4 * c] = x.x; w[4 * c + 1] = x.y; w[4 * c + 2] = x.z; w[4 * c + 3] = x.w;
    }
}
template <int B>
__device__ inline void unpack_k(const uint8_t* from, uint8_t* to, int lane) {
    uint32_t w[2 * B];
    staged_string<2 * B>(from, lane, w);
#pragma unroll
    for (int p = 0; p < 8; ++p) *reinterpret_cast<u32x4*>(to + (p * 64 + lane) * 16) = __builtin_bit_cast(u32x4, dq_piece<B>(w, p));
}
template <int B>
__device__ inline void unpack_v(const uint8_t* from, uint8_t* to, int lane) {
    const uint8_t* const meta = from + KVQ_TREE_STAGE_META + (lane >> 4) * 16;
    uint32_t w[2 * B];
    staged_string<2 * B>(from, lane, w);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const u32x4 s = *reinterpret_cast<const u32x4*>(meta + g * 64), z = *reinterpret_cast<const u32x4*>(meta + 256 + g * 64);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 c = __builtin_bit_cast(u32x4, dq_piece<B>(w, 2 * g + h));
            *reinterpret_cast<u32x4*>(to + ((2 * g + h) * 64 + lane) * 16) =
                u32x4{fma2(c.x, s.x, z.x), fma2(c.y, s.y, z.y), fma2(c.z, s.z, z.z), fma2(c.w, s.w, z.w)};
        }
    }
}
__device__ inline void unpack_raw(const uint8_t* from, uint8_t* to, int lane) {
#pragma unroll
    for (int p = 0; p < 8; ++p) *reinterpret_cast<u32x4*>(to + (p * 64 + lane) * 16) = paired(*reinterpret_cast<const u32x4*>(from + (p * 64 + lane) * 16));
}
// A staged operand into its place in a slot (slot: K operands, V operands, and the low bytes of K in the integer 16-bit tier); meta: where
// the scales and zero points of K go, ones and zeros for a raw tile.
template <bool I16>
__device__ __attribute__((always_inline)) inline void unpack_staged(const Staged& f, const uint8_t* from, uint8_t* slot, uint8_t* meta, int part, int lane) {
    const uint32_t bits = f.bits;
    if (part == 0) {
        u32x4 m = *reinterpret_cast<const u32x4*>(from + KVQ_TREE_STAGE_META + (lane & 31) * 16);
        if (!I16 && bits == 16) m = lane < 16 ? u32x4{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u} : u32x4{0u, 0u, 0u, 0u};
        if (lane < 32) *reinterpret_cast<u32x4*>(meta + lane * 16) = m;
        if (bits == 2) unpack_k<2>(from, slot, lane);
        else if (bits == 4) unpack_k<4>(from, slot, lane);
        else if (bits == 8) unpack_k<8>(from, slot, lane);
        else if constexpr (I16) {
            uint32_t w[32];
            staged_string<32>(f.code, lane, w);
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                *reinterpret_cast<u32x4*>(slot + (p * 64 + lane) * 16) = __builtin_bit_cast(u32x4, dq_piece<8>(w, p));
                *reinterpret_cast<u32x4*>(slot + KVQ_TREE_K_LOW + (p * 64 + lane) * 16) = __builtin_bit_cast(u32x4, dq_piece_frac(w + 16, p));
            }
        } else unpack_raw(f.code, slot, lane);
        return;
    }
    uint8_t* const to = slot + KVQ_TREE_V;
    if (bits == 16) {
        if constexpr (!I16) {
            unpack_raw(f.code, to, lane);
        } else {
            uint32_t w[32];
            staged_string<32>(f.code, lane, w);
            values_of_planes(w, from + KVQ_TREE_STAGE_META, to, lane);
        }
        return;
    }
    if (bits == 2) unpack_v<2>(from, to, lane);
    else if (bits == 4) unpack_v<4>(from, to, lane);
    else unpack_v<8>(from, to, lane);
    const u32x4 m = *reinterpret_cast<const u32x4*>(from + KVQ_TREE_STAGE_META + (lane & 31) * 16);  // (twice: rows 0 and 2 scales, 1 and 3 zero points)
    if (overflows(m, (1 << bits) - 1)) clamp_values(to, from + KVQ_TREE_STAGE_META, lane);
}

// The nodes' own keys or values of one tile as operands in a slot (part 0: K, 1: V), infinite and NaN values as zeros; true if there were any.
__device__ inline bool lay_out_k(const TreeArgs& A, int unit, int first, uint8_t* to, int lane) {
    const int j = lane >> 4, n = lane & 15;
    const _Float16* const kn = A.k + (int64_t)unit * A.nodes * KVQ_D;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int node = min(first + 8 * (n >> 2) + 4 * (p >> 2) + (n & 3), A.nodes - 1);
        *reinterpret_cast<u32x4*>(to + (p * 64 + lane) * 16) = paired(*reinterpret_cast<const u32x4*>(kn + (int64_t)node * KVQ_D + 32 * (p & 3) + 8 * j));
    }
    return false;
}
__device__ inline bool lay_out_v(const TreeArgs& A, int unit, int first, uint8_t* to, int lane) {
    const _Float16* const vn = A.v + (int64_t)unit * A.nodes * KVQ_D;
    const int k = (lane >> 1) & 3, chunk = (lane >> 3) * 2 + (lane & 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int token = 8 * (i >> 1) + 4 * (i & 1) + k;
        u32x4 w = *reinterpret_cast<const u32x4*>(vn + (int64_t)min(first + token, A.nodes - 1) * KVQ_D + chunk * 8);
        if (first + token >= A.nodes) w = u32x4{0, 0, 0, 0};
        *reinterpret_cast<u32x4*>(to + v_chunk_at(token, chunk)) = w;
    }
    wave_lds_sync();
    uint32_t bad = 0;
    u32x4 vo[8];
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
        const half8 a = read_v(to, nt, lane);
        watch_nonfinite(a, bad);
        vo[nt] = paired(__builtin_bit_cast(u32x4, a));
    }
    wave_lds_sync();
    const bool any = __any(bad != 0);
    if (any) {  // what is not finite is added at the very end, to the rows that see it
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) vo[nt] = finite_only(vo[nt]);
    }
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) *reinterpret_cast<u32x4*>(to + (nt * 64 + lane) * 16) = vo[nt];
    return any;
}

// The cache's tiles of a range.
__device__ inline void range_of(const TreeArgs& A, int split, int& t0, int& t1) {
    t0 = min(A.n_tiles, max(0, split * A.per - A.node_tiles));
    t1 = min(A.n_tiles, max(0, (split + 1) * A.per - A.node_tiles));
}
// Masks what lies behind the cache's last token.
template <int RR, int R>
__device__ inline void mask_end(float4v (&s)[R][1][2], int end) {
#pragma unroll
    for (int r = 0; r < RR; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= end) s[r][0][e >> 2][e & 3] = -INFINITY;
}
// One tile of nodes that is laid out in a slot, for a wavefront's rows.
template <int R>
__device__ inline void take_nodes(State<R>& st, const half8 (&q)[R][4], const TreeArgs& A, const uint32_t* mask, const uint8_t* slot, int row0, int step,
                                  int tile, int lane) {
    const int j = lane >> 4, n = lane & 15;
    float4v s[R][1][2];
    node_scores<R>(s, q, slot, lane);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = min(row0 + step * r + n, A.rows - 1);
        const int here = A.nodes - tile * KVQ_TILE_TOKENS;
        uint32_t w = mask[(int64_t)(row % A.nodes) * A.words + tile];
        if (here < KVQ_TILE_TOKENS) w &= (1u << here) - 1u;
        w >>= 8 * j;  // the quarter's eight nodes
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!((w >> e) & 1u)) s[r][0][e >> 2][e & 3] = -INFINITY;
    }
    uint32_t p[R][1][4];
#pragma unroll
    for (int r = 0; r < R; ++r) softmax_group<R, 1, true, false>(st, r, s[r], A.scale_log2, false, p[r]);
    tile_products<R, R>(st, p, slot, lane);
}
// A wavefront's results (its groups of 16 rows `apart` groups apart): partial ones beyond one range, else the output.
template <int R>
__device__ inline void store_rows(const State<R>& st, const TreeArgs& A, int unit, int block, int split, int group0, int apart, bool nonfinite, int lane) {
    const int j = lane >> 4, n = lane & 15;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = (block * A.groups + group0 + apart * r) * 16 + n;
        if (group0 + apart * r >= A.groups || row - n >= A.rows) continue;  // (another block's, or nobody's)
        if (A.splits > 1) {
            const int64_t group = ((int64_t)(unit * A.blocks + block) * A.splits + split) * A.groups + group0 + apart * r;
            store_partial(st, r, A.part + group * (KVQ_PART_BYTES / 4), lane);
            continue;
        }
        const float inv = inverse_of(quarters_sum(st.l[r]));
        if (row >= A.rows) continue;
        const int64_t at = ((int64_t)unit * A.rows + row) * KVQ_D;
        void* const dst = A.out_fp32 ? static_cast<void*>(static_cast<float*>(A.out) + at) : static_cast<void*>(static_cast<_Float16*>(A.out) + at);
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) store_out4(dst, A.out_fp32, 16 * nt + 4 * j, st.o[r][nt] * inv);
    }
    if (nonfinite) {
#pragma unroll 1
        for (int r = 0; r < R; ++r) {
            if (group0 + apart * r >= A.groups || (block * A.groups + group0 + apart * r) * 16 >= A.rows) continue;
            const int64_t group = ((int64_t)(unit * A.blocks + block) * A.splits + split) * A.groups + group0 + apart * r;
            add_nonfinite(A, unit, (block * A.groups + group0 + apart * r) * 16 + n, A.splits > 1 ? A.part + group * (KVQ_PART_BYTES / 4) : nullptr, lane);
        }
    }
}

// Many rows: 16 R for each of W wavefronts or, WT == 2, for each of W / 2 pairs, which take an iteration's tiles in turn.  An iteration unpacks
// W / 2 tiles, K and V of each in a wavefront of its own, while the next ones are on their way into the staging area.  Twelve
// wavefronts fit a compute unit, three on every SIMD: in three workgroups or, where rows are enough, in one, which unpacks a tile for all of them.
// What it spends its time on (64 drafted tokens x 40 heads over 4 x 32,768 tokens at all widths, 244 us with the joining kernel, 705 TFLOP/s
// where an fp16 product of 8,192^3 reaches 1,290; with scales for 64 or 128 channels 219 us): issuing.  A tile of two groups of rows takes 36
// products, 64 multiply-adds with the scales of K, some 70 instructions of softmax, and unpacking its share of a tile 150; products and vector
// instructions of the wavefronts on a SIMD hardly overlap, no wavefront waits for memory (8 ns an iteration) and little for barriers.
// Four wavefronts, three workgroups a compute unit: 288 us.
template <int R, bool I16, int SCALES, int WT, int W>
__global__ __launch_bounds__(64 * W, I16 ? 2 : 3) void kvq_tree_shared_kernel(const TreeArgs A) {
    constexpr int NT = W / 2, SLOT = (I16 ? 3 : 2) * KVQ_FLASH_TILE_BYTES;
    static_assert((WT == 1 && W % 4 == 0) || (W == 4 && 2 * KVQ_JOIN_BYTES <= NT * SLOT), "two pairs of wavefronts");
    // (the staging area is an object of its own: reads of the others then do not wait for what is on its way into it)
    __shared__ __attribute__((aligned(16))) uint8_t lds[NT * SLOT + NT * 512];
    __shared__ __attribute__((aligned(16))) uint8_t staging[W * KVQ_TREE_STAGE];
    __shared__ uint32_t widths[NT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WT, wt = wave % WT;
    const int part = wave & 1, own = wave >> 1;  // what this wavefront unpacks
    uint8_t* const slot = lds + own * SLOT;
    uint8_t* const stage = staging + wave * KVQ_TREE_STAGE;
    uint8_t* const meta = lds + NT * SLOT;
    // neighbouring workgroups are different units (and go to different XCDs); the row blocks of a range follow closely
    const int unit = blockIdx.x % A.units, x = blockIdx.x / A.units, block = x % A.blocks, split = x / A.blocks;
    constexpr int apart = W / WT, step = 16 * apart;  // the wavefronts take turns at the groups of rows
    const int row0 = (block * A.groups + wm) * 16;
    int t0, t1;
    range_of(A, split, t0, t1);
    State<R> st;
    st.clear();
    half8 q[R][4];
    if (t0 < t1) {
        const KvqPageDesc first = entry_of(A, min(t0 + own, t1 - 1));
        KvqPageDesc next = entry_of(A, min(t0 + NT + own, t1 - 1));
        u32x4 w[R][4];
        ask_queries<R>(w, A, unit, row0, step, lane);
        Staged f = stage_tile(A, first, unit, min(t0 + own, t1 - 1), part, stage, lane);
        set_queries<R>(q, w, A, unit, row0, step, true, lane);
        half4 qs[R];
        float scale[R];
        sum_queries<R>(q, qs, scale, A.scale_log2, lane);
        // rows that do not fill a block leave wavefronts with fewer groups (RR), in a loop of their own (not in pairs, where the length of
        // the chain counts and not what there is to do)
        const auto pass = [&](auto groups) {
        constexpr int RR = decltype(groups)::value;
        for (int t = t0; t < t1; t += NT) {
            wait_staged();
            int l = lane;  // (addresses derived from it are not to be kept over the loop: there are no registers for them)
            asm volatile("" : "+v"(l));
            unpack_staged<I16>(f, stage, slot, meta + own * 512, part, l);
            if (I16 && part == 0 && lane == 0) widths[own] = f.bits;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the staging area has been read
            if (t + NT < t1) {
                f = stage_tile(A, next, unit, min(t + NT + own, t1 - 1), part, stage, lane);
                next = entry_of(A, min(t + 2 * NT + own, t1 - 1));
            }
            lds_barrier();
#pragma unroll 1
            for (int i = wt; i < NT; i += WT) {
                const int tile = t + i;
                if (tile >= t1) break;
                int l = lane;
                asm volatile("" : "+v"(l));
                float4v s[R][1][2];
                cache_scores<RR, I16, SCALES, R>(s, q, qs, lds + i * SLOT, meta + i * 512, I16 && __builtin_amdgcn_readfirstlane(widths[i]) == 16, l);
                if ((tile + 1) * KVQ_TILE_TOKENS > A.n_tokens) {
                    asm volatile("" ::: "memory");  // keep this a branch: the selects must not run for every tile
                    mask_end<RR, R>(s, A.n_tokens - tile * KVQ_TILE_TOKENS - 8 * (lane >> 4));
                }
                uint32_t p[R][1][4];
#pragma unroll
                for (int r = 0; r < RR; ++r) softmax_group<R, 1, true, false>(st, r, s[r], scale[r], false, p[r]);
                tile_products<RR, R>(st, p, lds + i * SLOT, l);
            }
            lds_barrier();
        }
        };
        if (WT == 2 || (wm + apart < A.groups && row0 + step < A.rows)) pass(std::integral_constant<int, R>{});
        else pass(std::integral_constant<int, 1>{});
    }
    // the nodes among themselves
    bool nonfinite = false;
    if (split == 0) {
        const uint32_t* const mask = A.mask + (int64_t)(unit / A.n_kv) * A.mask_seq;
        const int tiles = (A.nodes + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS;
        for (int t = 0; t < tiles; t += NT) {
            if (t + own < tiles)
                nonfinite |= part == 0 ? lay_out_k(A, unit, (t + own) * KVQ_TILE_TOKENS, slot, lane)
                                       : lay_out_v(A, unit, (t + own) * KVQ_TILE_TOKENS, slot + KVQ_TREE_V, lane);
            __syncthreads();
            load_queries<R>(q, A, unit, row0, step, false, lane);  // (here, where they do not take registers from the lines above)
#pragma unroll 1
            for (int i = wt; i < NT && t + i < tiles; i += WT) take_nodes<R>(st, q, A, mask, lds + i * SLOT, row0, step, t + i, lane);
            __syncthreads();
        }
        nonfinite = __syncthreads_or(nonfinite ? 1 : 0) != 0;
    }
    if constexpr (WT == 2) {
        join_waves<R, 2, 2>(st, lds, wm, wt, lane);
        if (wt > 0) return;
    }
    store_rows<R>(st, A, unit, block, split, wm, apart, nonfinite, lane);
}

// Few rows, 16 R: four wavefronts that all have them and take a tile each, unpacked for themselves alone.
// 4 drafted tokens x 8 heads over 4,096 tokens: 7.8 us and 2.9 to join 17 ranges, a chain of trips to memory (arguments, page entry, tile) and of
// two tiles' work.
template <int R, bool I16>
__global__ __launch_bounds__(256, I16 ? 1 : 2) void kvq_tree_kernel(const TreeArgs A) {
    constexpr int SLOT = (I16 ? 3 : 2) * KVQ_FLASH_TILE_BYTES;
    static_assert(2 * KVQ_JOIN_BYTES <= 4 * SLOT, "four wavefronts");
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * SLOT + 4 * KVQ_META_TILE_BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lane_off = 16u * lane;
    uint8_t* const slot = lds + wave * SLOT;
    uint8_t* const meta_lds = lds + 4 * SLOT + wave * KVQ_META_TILE_BYTES;
    const int unit = blockIdx.x % A.units, x = blockIdx.x / A.units, block = x % A.blocks, split = x / A.blocks;
    const int row0 = block * A.groups * 16;
    int t0, t1;
    range_of(A, split, t0, t1);
    State<R> st;
    st.clear();
    half8 q[R][4];
    if (t0 + wave < t1) {
        const KvqPageDesc first = entry_of(A, t0 + wave);
        KvqPageDesc next = entry_of(A, min(t0 + wave + 4, t1 - 1));
        u32x4 w[R][4];
        Fetched f;
        fetch_tile<I16>(f, A, first, unit, t0 + wave, lane_off);
        ask_queries<R>(w, A, unit, row0, 16, lane);
        set_queries<R>(q, w, A, unit, row0, 16, true, lane);
        half4 qs[R];
        float scale[R];
        sum_queries<R>(q, qs, scale, A.scale_log2, lane);
        for (int tile = t0 + wave; tile < t1; tile += 4) {
            expand_tile<I16>(f, slot, meta_lds, lane);
            const bool planes = I16 && f.bits == 16;
            if (tile + 4 < t1) {
                fetch_tile<I16>(f, A, next, unit, tile + 4, lane_off);
                next = entry_of(A, min(tile + 8, t1 - 1));
            }
            wave_lds_sync();
            float4v s[R][1][2];
            cache_scores<R, I16, 4, R>(s, q, qs, slot, meta_lds, planes, lane);
            if ((tile + 1) * KVQ_TILE_TOKENS > A.n_tokens) {
                asm volatile("" ::: "memory");  // keep this a branch: the selects must not run for every tile
                mask_end<R, R>(s, A.n_tokens - tile * KVQ_TILE_TOKENS - 8 * (lane >> 4));
            }
            uint32_t p[R][1][4];
#pragma unroll
            for (int r = 0; r < R; ++r) softmax_group<R, 1, true, false>(st, r, s[r], scale[r], false, p[r]);
            tile_products<R, R>(st, p, slot, lane);
            wave_lds_sync();
        }
    }
    // the nodes among themselves
    bool nonfinite = false;
    if (split == 0) {
        load_queries<R>(q, A, unit, row0, 16, false, lane);
        const uint32_t* const mask = A.mask + (int64_t)(unit / A.n_kv) * A.mask_seq;
        const int tiles = (A.nodes + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS;
        for (int t = wave; t < tiles; t += 4) {
            lay_out_k(A, unit, t * KVQ_TILE_TOKENS, slot, lane);
            nonfinite |= lay_out_v(A, unit, t * KVQ_TILE_TOKENS, slot + KVQ_TREE_V, lane);
            wave_lds_sync();
            take_nodes<R>(st, q, A, mask, slot, row0, 16, t, lane);
            wave_lds_sync();
        }
        nonfinite = __syncthreads_or(nonfinite ? 1 : 0) != 0;
    }
    join_waves<R, 1, 4>(st, lds, 0, wave, lane);
    if (wave > 0) return;
    store_rows<R>(st, A, unit, block, split, 0, 1, nonfinite, lane);
}

// Joins the ranges of one group of 16 rows, 32 channels a workgroup.
__global__ __launch_bounds__(512) void kvq_tree_merge_kernel(const TreeArgs A) {
    __shared__ JoinLds lds;
    const int lane = threadIdx.x & 63, j = lane >> 4, n = lane & 15;
    const int pair = blockIdx.x & 3, rg = (blockIdx.x >> 2) % A.groups, ub = (blockIdx.x >> 2) / A.groups, block = ub % A.blocks, unit = ub / A.blocks;
    const int row0 = (block * A.groups + rg) * 16;
    if (row0 >= A.rows) return;
    const float* part = A.part + ((int64_t)ub * A.splits * A.groups + rg) * (KVQ_PART_BYTES / 4);
    Joined x;
    if (!join_partials(lds, part, (int64_t)A.groups * (KVQ_PART_BYTES / 4), A.splits, pair, x)) return;
    const int row = row0 + n;
    if (row >= A.rows) return;
    const int64_t at = ((int64_t)unit * A.rows + row) * KVQ_D;
    void* const dst = A.out_fp32 ? static_cast<void*>(static_cast<float*>(A.out) + at) : static_cast<void*>(static_cast<_Float16*>(A.out) + at);
    store_out4(dst, A.out_fp32, 16 * x.nt + 4 * j, x.o * inverse_of(x.l));
}

// ---- host side

constexpr int kMostSplits = KVQ_MOST_PARTS;
constexpr int kNodeTiles = 4;   // what the nodes cost beside their tiles, in tiles: their queries and their layout
constexpr int kLeastTiles = 8;  // of a range: two a wavefront of the kernel for few rows, or four iterations of the other
struct TreePlan {
    bool many;
    int waves, groups, wt, blocks, splits, per, node_tiles;  // groups of 16 rows in a block
    uint64_t bytes;  // of the partial results, no more than `most`: those of as many ranges as this kernel may take for a cache that is not longer
    uint64_t most;
};
// workspace: bytes there are for partial results
TreePlan plan_tree(const kvq_cache* c, int nodes, int n_tiles, uint64_t workspace) {
    TreePlan p;
    const int rows = c->gqa * nodes;
    p.many = rows > 32;
    if (p.many) {
        // pairs where rows are few or there is so little to do that the length of the chain counts: 112 rows x 282 tiles x 4 units 27.4 us
        // and 24.7 in pairs, 256 x 128 x 2 21.4 and 18.7; 200 x 938 x 8 70 and 78, 448 x 256 x 16 77 and 83
        p.wt = rows <= 64 || (int64_t)c->units * ((rows + 127) / 128) * n_tiles <= 4096 ? 2 : 1;
        // a tile is unpacked once a block: twelve wavefronts where they have enough rows (320 rows x 1,026 tiles x 32 units 288 us with four and
        // 247 with twelve, 272 x 938 x 32 257 and 216, 256 x 938 x 32 196 and 195, 200 x 4,096 x 8 205 and 212) and iterations
        // of six tiles (320 x 94 x 32 49 and 52, 288 x 157 x 32 65 and 61)
        const int groups = (rows + 15) / 16, large = (groups + 23) / 24;
        const bool twelve = p.wt == 1 && !c->int16() && groups > 16 * large && (int64_t)n_tiles * c->units * large >= 18 * (int64_t)c->target_workgroups;
        p.waves = twelve ? 12 : 4;
        p.groups = twelve ? (groups + large - 1) / large : 8 / p.wt;
        p.blocks = (rows + 16 * p.groups - 1) / (16 * p.groups);
    } else {
        p.groups = rows <= 16 ? 1 : 2;
        p.blocks = p.wt = 1;
        p.waves = 4;
    }
    const int64_t wgs = (int64_t)c->units * p.blocks;
    const int64_t want = std::max<int64_t>(1, (p.many && !c->int16() ? 12 / p.waves : 2) * c->target_workgroups / wgs);
    const uint64_t one = (uint64_t)wgs * p.groups * KVQ_PART_BYTES;  // a range's partial results
    const int64_t room = (int64_t)std::min<uint64_t>(workspace / one, kMostSplits);
    p.node_tiles = ((nodes + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS + kNodeTiles + kLeastTiles - 1) / kLeastTiles * kLeastTiles;
    // half as many tiles a range as long as the ranges are not too many to be joined: 40 rows x 64 tiles x 8 units 17.4 us in 8 and 14.7 in
    // 16, 16 x 128 x 2 11.5 in 16 and 10.3 in 32; 7 x 282 x 4 14.1 in 35 and 15.7 in 65
    const int64_t tiles = n_tiles + p.node_tiles, cut = std::max<int64_t>(tiles / kLeastTiles, std::min<int64_t>(2 * tiles / kLeastTiles, 32));
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, kMostSplits), std::min<int64_t>(cut, room)));
    if (n_tiles < kLeastTiles) p.splits = 1;
    p.most = p.splits > 1 ? one * (uint64_t)p.splits : 0;
    const int round = p.many ? p.waves / 2 : 4;  // (in whole iterations: half a tile a wavefront, or one)
    p.per = ((int)((tiles + p.splits - 1) / p.splits) + round - 1) / round * round;
    p.splits = p.splits > 1 ? (int)((tiles + p.per - 1) / p.per) : 1;
    p.bytes = p.splits > 1 ? one * (uint64_t)p.splits : 0;
    return p;
}
using Kernel = void (*)(TreeArgs);
template <bool I16, int SCALES>
Kernel kernel_of(const TreePlan& p) {
    if (p.many && p.wt == 2) return kvq_tree_shared_kernel<2, I16, 4, 2, 4>;
    if constexpr (!I16)
        if (p.many && p.waves == 12) return kvq_tree_shared_kernel<2, I16, SCALES, 1, 12>;
    if (p.many) return kvq_tree_shared_kernel<2, I16, SCALES, 1, 4>;
    return p.groups > 1 ? kvq_tree_kernel<2, I16> : kvq_tree_kernel<1, I16>;
}
template <bool I16>
Kernel kernel_of(const TreePlan& p, int group) {
    return group == 32 ? kernel_of<I16, 4>(p) : kernel_of<I16, 2>(p);
}
bool nodes_ok(const kvq_cache* c, int nodes) { return c && nodes >= 1 && nodes <= KVQ_MAX_TREE_NODES; }

}  // namespace

extern "C" {

uint64_t kvq_tree_workspace_bytes(const kvq_cache_t* c, int32_t n_nodes) {
    if (!nodes_ok(c, n_nodes)) return 0;
    // A shorter cache may take another kernel, and fewer tiles may be cut into more ranges, which are of whole iterations.  Before that rounding
    // ranges only become more with the tiles, so the longest cache of each kernel decides; kernels change at no more than two lengths.
    const auto plan = [&](int n_tiles) { return plan_tree(c, n_nodes, n_tiles, UINT64_MAX); };
    const auto same = [](const TreePlan& a, const TreePlan& b) { return a.wt == b.wt && a.waves == b.waves && a.groups == b.groups; };
    uint64_t most = 0;
    for (int n_tiles = (c->cfg.max_tokens + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS; n_tiles > 0;) {
        const TreePlan p = plan(n_tiles);
        most = std::max(most, p.most);
        int shorter = 0, longer = n_tiles;  // the longest cache that takes another kernel, 0: none
        while (longer - shorter > 1) {
            const int middle = shorter + (longer - shorter) / 2;
            (same(plan(middle), p) ? longer : shorter) = middle;
        }
        n_tiles = shorter;
    }
    return most;
}

kvq_status_t kvq_tree_attention(kvq_cache_t* c, int32_t layer, const void* q_dev, const void* k_dev, const void* v_dev, int32_t n_nodes,
                                const uint32_t* mask_dev, int32_t mask_per_sequence, void* out_dev, int32_t out_is_fp32, float softmax_scale,
                                void* workspace_dev, uint64_t workspace_bytes, void* hip_stream) {
    if (!nodes_ok(c, n_nodes) || layer < 0 || layer >= c->cfg.n_layers) return KVQ_E_INVALID;
    if (!q_dev || !k_dev || !v_dev || !mask_dev || !out_dev || !std::isfinite(softmax_scale)) return KVQ_E_INVALID;
    for (const void* p : {q_dev, k_dev, v_dev, static_cast<const void*>(out_dev), static_cast<const void*>(workspace_dev)})
        if (reinterpret_cast<uintptr_t>(p) & 15u) return KVQ_E_INVALID;
    if (reinterpret_cast<uintptr_t>(mask_dev) & 3u) return KVQ_E_INVALID;
    if (c->dry) return KVQ_E_STATE;
    const kvq_host::Layer& L = c->layers[(size_t)layer];
    if (L.poisoned) return KVQ_E_STATE;
    TreeArgs A{};
    A.n_tokens = L.T;
    A.n_tiles = (L.T + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS;
    const TreePlan plan = plan_tree(c, n_nodes, A.n_tiles, workspace_dev ? workspace_bytes : 0);
    A.arena = c->arena;
    A.table = c->table_dev(layer);
    A.q = static_cast<const _Float16*>(q_dev);
    A.k = static_cast<const _Float16*>(k_dev);
    A.v = static_cast<const _Float16*>(v_dev);
    A.mask = mask_dev;
    A.words = (n_nodes + 31) / 32;
    A.mask_seq = mask_per_sequence ? (int64_t)n_nodes * A.words : 0;
    A.lambda = L.reparam ? c->lambda_dev(layer) : nullptr;
    A.out = out_dev;
    A.part = static_cast<float*>(workspace_dev);
    A.tpp = c->tpp;
    A.tpp_magic = c->tpp > 1 ? (uint32_t)(((1ull << 32) + (uint64_t)c->tpp - 1) / (uint64_t)c->tpp) : 0u;
    A.units = c->units;
    A.n_kv = c->cfg.n_kv_heads;
    A.gqa = c->gqa;
    A.nodes = n_nodes;
    A.rows = c->gqa * n_nodes;
    A.blocks = plan.blocks;
    A.splits = plan.splits;
    A.per = plan.per;
    A.node_tiles = plan.node_tiles;
    A.out_fp32 = out_is_fp32 ? 1 : 0;
    const float scale = softmax_scale != 0.f ? softmax_scale : 1.0f / std::sqrt((float)KVQ_D);
    A.scale_log2 = std::fabs(scale) * 1.44269504088896340736f;
    A.flip = scale < 0.f ? 0x80008000u : 0u;
    A.groups = plan.groups;
    const hipStream_t s = kvq_host::as_stream(hip_stream);
    const unsigned row_blocks = (unsigned)(c->units * plan.blocks);
    const Kernel kernel = c->int16() ? kernel_of<true>(plan, c->cfg.group) : kernel_of<false>(plan, c->cfg.group);
    hipLaunchKernelGGL(kernel, dim3(row_blocks * (unsigned)plan.splits),
                       dim3(64u * (unsigned)plan.waves), 0, s, A);
    if (hipGetLastError() != hipSuccess) return KVQ_E_HIP;
    if (plan.splits > 1) {
        hipLaunchKernelGGL(kvq_tree_merge_kernel, dim3(row_blocks * (unsigned)plan.groups * 4), dim3(512), 0, s, A);
        if (hipGetLastError() != hipSuccess) return KVQ_E_HIP;
    }
    return KVQ_OK;
}

}  // extern "C"
