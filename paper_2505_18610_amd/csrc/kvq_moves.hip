// Cached states that move: one block's sequences into another cache or another order (kvq_cache_fork), its newest tokens taken away
// (kvq_cache_truncate), its tokens read back as values (kvq_cache_read).
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "../../include/kvq.h"
#include "kvq_append16.h"
#include "kvq_cache.h"

namespace {

using kvq_dev::div_magic;
using kvq_dev::f2h_rn;
using kvq_dev::h2f;
using kvq_dev::u32x4;
using kvq_host::Layer;
using kvq_host::Page;
using kvq_host::as_stream;
using kvq_host::order_of_bits;

uint32_t magic_of(int d) { return d > 1 ? (uint32_t)(((1ull << 32) + (uint64_t)d - 1) / (uint64_t)d) : 0u; }

// ---------------------------------------------------------------------------------------------------------------- fork
#define KVQ_FORK_ARG_PAGES 192  // pages whose new places ride in the kernel arguments
#define KVQ_FORK_TILES 4        // tiles a workgroup copies
struct ForkArgs {
    const uint8_t* src;
    uint8_t* dst;
    const KvqPageDesc* src_table;
    KvqPageDesc* dst_table;      // written, in another cache by the copy itself
    const int32_t* map;          // [dst batch] or null
    const float* src_lambda;     // the block's key factors and their reciprocals, or null
    float* dst_lambda;
    KvqVMark src_mark, dst_mark;
    int32_t n_lambda;
    int32_t src_batch, dst_batch, n_kv, tpp, n_pages, last_tiles;  // last_tiles: tiles of the last page that hold tokens
    int32_t groups;              // of KVQ_FORK_TILES tiles in a page
    int32_t page0, n_here;       // the pages of this launch
    int32_t in_place;            // the table is the one that the copy reads: kvq_fork_table_kernel writes it behind the copy
    uint32_t code_off256[KVQ_FORK_ARG_PAGES], meta_off256[KVQ_FORK_ARG_PAGES];
};
static_assert(sizeof(ForkArgs) <= 4096 - 64, "kernel arguments end at 4 KiB");

// Forks that write more than the device's last-level cache holds go past it (sixteen samples of 32,768 tokens, 361 MB, 90 -> 75 us);
// what fits is left there for the attention that follows (eight beams of 2,500 tokens, 45 MB: the same 16.5 us, but the next
// kernel reads them in 21.6 us and not in 32).
#define KVQ_FORK_STREAM_BYTES (256ull << 20)
template <bool STREAM>
__device__ inline void store16(uint8_t* to, u32x4 w) {
    if (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(to));
    else *reinterpret_cast<u32x4*>(to) = w;
}
// Copies `bytes` (a multiple of 1 KiB, 1 KiB or more) with 256 threads, four loads in flight a thread.
template <bool STREAM>
__device__ inline void copy_bytes(uint8_t* dst, const uint8_t* src, uint32_t bytes, int tid) {
    uint32_t at = 16u * tid;
    for (; at + 3 * 4096 < bytes; at += 4 * 4096) {
        u32x4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const u32x4*>(src + at + i * 4096);
#pragma unroll
        for (int i = 0; i < 4; ++i) store16<STREAM>(dst + at + i * 4096, w[i]);
    }
    for (; at < bytes; at += 4096) store16<STREAM>(dst + at, *reinterpret_cast<const u32x4*>(src + at));
}

// One workgroup: up to four neighbouring tiles of one page, KV head and sequence, codes and metadata.  Workgroups of one place follow
// one another over the sequences, so that sequences with the same parent read it while it is in the caches.
template <bool STREAM>
__global__ __launch_bounds__(256) void kvq_fork_kernel(const ForkArgs A) {
    const int tid = threadIdx.x;
    int x = blockIdx.x;
    const int b = x % A.dst_batch;
    x /= A.dst_batch;
    const int h = x % A.n_kv;
    x /= A.n_kv;
    const int group = x % A.groups, here = x / A.groups, page = A.page0 + here;
    if (blockIdx.x == 0 && A.page0 == 0 && !A.in_place) {
        if (tid == 0 && kvq_v_marked(*A.src_mark.word, A.src_mark.epoch, false))
            *A.dst_mark.word = A.dst_mark.epoch;
        if (A.dst_lambda)
            for (int i = tid; i < A.n_lambda; i += 256) A.dst_lambda[i] = A.src_lambda[i];
    }
    KvqPageDesc from = A.src_table[page], to = from;
    to.code_off256 = A.code_off256[here];
    to.meta_off256 = A.meta_off256[here];
    if (!A.in_place && b == 0 && h == 0 && group == 0 && tid == 0) A.dst_table[page] = to;
    const int tiles = min(page + 1 == A.n_pages ? A.last_tiles : A.tpp, (group + 1) * KVQ_FORK_TILES) - group * KVQ_FORK_TILES;
    if (tiles <= 0) return;
    const int parent = A.map ? min(max(A.map[b], 0), A.src_batch - 1) : A.src_batch == 1 ? 0 : b;
    const uint64_t src_slot = (uint64_t)(parent * A.n_kv + h) * A.tpp + group * KVQ_FORK_TILES;
    const uint64_t dst_slot = (uint64_t)(b * A.n_kv + h) * A.tpp + group * KVQ_FORK_TILES;
    const uint32_t tile_bytes = 1024u * from.bits;
    copy_bytes<STREAM>(A.dst + (uint64_t)to.code_off256 * 256u + dst_slot * tile_bytes, A.src + (uint64_t)from.code_off256 * 256u + src_slot * tile_bytes,
               (uint32_t)tiles * tile_bytes, tid);
    if (from.bits < 16 || from.int16)
        copy_bytes<STREAM>(A.dst + (uint64_t)to.meta_off256 * 256u + dst_slot * KVQ_META_TILE_BYTES,
                   A.src + (uint64_t)from.meta_off256 * 256u + src_slot * KVQ_META_TILE_BYTES, (uint32_t)tiles * KVQ_META_TILE_BYTES, tid);
}

__global__ __launch_bounds__(256) void kvq_fork_table_kernel(const ForkArgs A) {
    if ((int)threadIdx.x >= A.n_here) return;
    KvqPageDesc& d = A.dst_table[A.page0 + threadIdx.x];
    d.code_off256 = A.code_off256[threadIdx.x];
    d.meta_off256 = A.meta_off256[threadIdx.x];
}

// ------------------------------------------------------------------------------------------------------------ truncate
// Clears the tokens from `first` on in one tile of every unit: slots that hold no token are zero, codes and metadata, so that what
// they held cannot reach a sum that multiplies it by zero.  One wavefront a unit.
__global__ __launch_bounds__(64) void kvq_clear_tail_kernel(uint8_t* arena, const KvqPageDesc d, int tpp, int tile, int first) {
    const int lane = threadIdx.x, j = lane >> 4, n = lane & 15;
    const uint64_t slot = (uint64_t)blockIdx.x * tpp + tile;
    uint8_t* const code = arena + (uint64_t)d.code_off256 * 256u + slot * (1024u * d.bits);
    const bool planes = d.bits == 16 && d.int16;
    const int bits = planes ? 8 : (int)d.bits;  // of a slot of a string
    const int strings = planes ? 2 : 1;
    // A lane's string of K: slots 0..31 one token, 32..63 the token four later; of V: slot s is token 8 j + s % 8.
    for (int which = 0; which < 2; ++which)
        for (int plane = 0; plane < strings; ++plane) {
            uint32_t* const words = reinterpret_cast<uint32_t*>(code + which * 512u * d.bits + plane * 4096u);
            for (int w = 0; w < 2 * bits; ++w) {
                uint32_t keep = 0;
                for (int e = 0; e < 32 / bits; ++e) {
                    const int s = w * (32 / bits) + e;
                    const int token = which == 0 ? 8 * (n >> 2) + 4 * (s >> 5) + (n & 3) : 8 * j + (s & 7);
                    if (token < first) keep |= ((1u << bits) - 1u) << (e * bits);
                }
                if (keep != 0xffffffffu) words[((w >> 2) * 64 + lane) * 4 + (w & 3)] &= keep;
            }
        }
    if (d.bits == 16 && !d.int16) return;
    uint16_t* const meta = reinterpret_cast<uint16_t*>(arena + (uint64_t)d.meta_off256 * 256u + slot * KVQ_META_TILE_BYTES);
    for (int i = lane; i < KVQ_TILE_TOKENS * KVQ_NGRP; i += 64) {
        const int token = i >> 2, g = i & 3;
        if (token < first) continue;
        meta[i] = meta[128 + i] = 0;
        const int v = kvq_vmeta_index(token, g);
        meta[256 + v] = meta[384 + v] = 0;
    }
}

// ---------------------------------------------------------------------------------------------------------------- read
struct ReadArgs {
    const uint8_t* arena;
    const KvqPageDesc* table;
    const float* lambda;  // [n_kv_heads][128] or null
    void *k_out, *v_out;
    int32_t begin, n_tokens;  // tokens begin .. n_tokens - 1 are read
    int32_t tpp;
    uint32_t tpp_magic;
    int32_t n_kv, first_tile, n_tiles, fp32;
    int64_t items;            // units * n_tiles
};
#define KVQ_READ_PITCH 68  // floats of a row of 64 channels in LDS

__device__ inline uint32_t slot_code(const uint32_t* w, int bits, int s) {  // slot s of a lane's packed string (bits <= 8)
    return (w[s * bits >> 5] >> (s * bits & 31)) & ((1u << bits) - 1u);
}
// Eight consecutive channels of one token.
__device__ inline void store8(void* out, int fp32, int64_t at, const float (&x)[8]) {
    if (fp32) {
        kvq_dev::f32x4* p = reinterpret_cast<kvq_dev::f32x4*>(static_cast<float*>(out) + at);
        __builtin_nontemporal_store(kvq_dev::f32x4{x[0], x[1], x[2], x[3]}, p);
        __builtin_nontemporal_store(kvq_dev::f32x4{x[4], x[5], x[6], x[7]}, p + 1);
    } else {
        __builtin_nontemporal_store(u32x4{kvq_dev::pack_rn2(x[0], x[1]), kvq_dev::pack_rn2(x[2], x[3]), kvq_dev::pack_rn2(x[4], x[5]),
                                          kvq_dev::pack_rn2(x[6], x[7])}, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + at));
    }
}
// What a rounded scale (or a key's factor) has carried beyond the largest fp16 value becomes it, as in tree attention: no value that was
// appended is larger.  Infinities and NaNs stay.
__device__ inline float within_fp16(float x) { return fabsf(x) < INFINITY ? fminf(fmaxf(x, -65504.f), 65504.f) : x; }
__device__ inline float largest(float most, const float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
    return most;
}

// Values of the eight slots 8 p .. 8 p + 7 of a lane; B: 2, 4, 8, 16 (raw) or 17 (integer 16-bit tier, two byte planes).  s and z of
// each slot: one pair for K, a token each for V.
template <int B>
__device__ inline void piece_values(const uint8_t* tile, int lane, int p, const float (&s)[8], const float (&z)[8], float (&x)[8]) {
    if constexpr (B == 16) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(tile + (p * 64 + lane) * 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t word = w[i >> 1];
            x[i] = h2f((uint16_t)(i & 1 ? word >> 16 : word));
        }
    } else {
        constexpr int W = B == 17 ? 8 : B;                  // bits of a slot of a string
        uint32_t a[2] = {}, b[2] = {};
        const auto word = [&](const uint8_t* at, int i) {   // dword i of the lane's string
            return *reinterpret_cast<const uint32_t*>(at + ((i >> 2) * 64 + lane) * 16 + (i & 3) * 4);
        };
        const int first = p * 8 * W >> 5;
#pragma unroll
        for (int i = 0; i < (W == 8 ? 2 : 1); ++i) {
            a[i] = word(tile, first + i);
            if (B == 17) b[i] = word(tile + 4096, first + i);
        }
        if (W == 2 && (p & 1)) a[0] >>= 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t c = slot_code(a, W, i);
            if (B == 17) c = c << 8 | slot_code(b, 8, i);
            x[i] = fmaf((float)c, s[i], z[i]);
        }
    }
}
// Rows of 64 channels that the wavefront has put together in LDS: eight lanes store 128 consecutive bytes of a row (256 of fp32).
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// most: the largest size among the lane's values (looked at once for all rows: every value on its own cost a block of 4 x 32,768 tokens 8 %).
__device__ inline void store_rows(const ReadArgs& A, void* out, int unit, int tile, int half, float* lds, float most, int lane) {
    const int64_t rows = A.n_tokens - A.begin;
    if (!A.fp32 && __any(most > 65504.f)) {
        wave_sync();
        for (int i = lane; i < KVQ_TILE_TOKENS * 64; i += 64) {
            float* const x = lds + (i >> 6) * KVQ_READ_PITCH + (i & 63);
            *x = within_fp16(*x);
        }
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 8 * i + (lane >> 3), c = 8 * (lane & 7), tok = tile * KVQ_TILE_TOKENS + t;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = lds[t * KVQ_READ_PITCH + c + e];
        if (tok >= A.begin && tok < A.n_tokens) store8(out, A.fp32, ((int64_t)unit * rows + (tok - A.begin)) * KVQ_D + 64 * half + c, x);
    }
    wave_sync();
}
// A lane holds eight channels of a token ...
template <int B>
__device__ inline void read_k(const ReadArgs& A, const uint8_t* code, const uint16_t* meta, int unit, int tile, float* lds, int lane) {
    const int j = lane >> 4, n = lane & 15;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float most = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int sub = q >> 1, grp = 2 * half + (q & 1);
            const int t = 8 * (n >> 2) + 4 * sub + (n & 3), channel = 32 * grp + 8 * j;
            float s[8] = {}, z[8] = {}, x[8];
            if (B != 16) {
                const float s1 = h2f(meta[t * 4 + grp]), z1 = h2f(meta[128 + t * 4 + grp]);
#pragma unroll
                for (int i = 0; i < 8; ++i) { s[i] = s1; z[i] = z1; }
            }
            piece_values<B>(code, lane, sub * 4 + grp, s, z, x);
            if (A.lambda) {
                const float* l = A.lambda + (size_t)(unit % A.n_kv) * KVQ_D + channel;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= l[i];
            }
            most = largest(most, x);
            kvq_dev::f32x4* const to = reinterpret_cast<kvq_dev::f32x4*>(lds + t * KVQ_READ_PITCH + (channel & 63));
            to[0] = kvq_dev::f32x4{x[0], x[1], x[2], x[3]};
            to[1] = kvq_dev::f32x4{x[4], x[5], x[6], x[7]};
        }
        store_rows(A, A.k_out, unit, tile, half, lds, most, lane);
    }
}
// ... or eight tokens of a channel.
template <int B>
__device__ inline void read_v(const ReadArgs& A, const uint8_t* code, const uint16_t* meta, int unit, int tile, float* lds, int lane) {
    const int j = lane >> 4, n = lane & 15;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float most = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int nt = 4 * half + q;
            float s[8] = {}, z[8] = {}, x[8];
            if (B != 16) {  // the quarter's eight tokens, in pairs (v, v + 4)
                const u32x4 sw = *reinterpret_cast<const u32x4*>(meta + 256 + (nt >> 1) * 32 + j * 8), zw = *reinterpret_cast<const u32x4*>(meta + 384 + (nt >> 1) * 32 + j * 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t sp = sw[i & 3], zp = zw[i & 3];
                    s[i] = h2f((uint16_t)(i < 4 ? sp : sp >> 16));
                    z[i] = h2f((uint16_t)(i < 4 ? zp : zp >> 16));
                }
            }
            piece_values<B>(code, lane, nt, s, z, x);
            if (B != 16) most = largest(most, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) lds[(8 * j + i) * KVQ_READ_PITCH + 16 * q + n] = x[i];
        }
        store_rows(A, A.v_out, unit, tile, half, lds, most, lane);
    }
}
// A wavefront takes K or V of one tile of one unit.  Rows are put together in LDS because a lane holds eight channels of a token or eight tokens of
// a channel, and stores of whole lines are what bounds it: a block of 4 x 32,768 tokens at all widths, 706 MB read and written, 155 us from
// memory (4.6 TB/s; a copy reaches 5.1).  2,372 tokens of 8 heads 6.4 us, one launch's chain of trips.
__global__ __launch_bounds__(256) void kvq_read_kernel(const ReadArgs A) {
    __shared__ __attribute__((aligned(16))) float lds[4][KVQ_TILE_TOKENS * KVQ_READ_PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * 2 + (wave >> 1);
    if (item >= A.items) return;
    const int unit = (int)(item / A.n_tiles), tile = A.first_tile + (int)(item % A.n_tiles);
    const int page = div_magic(tile, A.tpp, A.tpp_magic), tip = tile - page * A.tpp;
    const KvqPageDesc d = A.table[page];
    const uint64_t slot = (uint64_t)unit * A.tpp + tip;
    const uint8_t* code = A.arena + (uint64_t)d.code_off256 * 256u + slot * (1024u * d.bits);
    const uint16_t* meta = reinterpret_cast<const uint16_t*>(A.arena + (uint64_t)d.meta_off256 * 256u + slot * KVQ_META_TILE_BYTES);
    const int width = d.bits == 16 && d.int16 ? 17 : (int)d.bits;
    float* const own = lds[wave];
    if (!(wave & 1)) {
        if (width == 2) read_k<2>(A, code, meta, unit, tile, own, lane);
        else if (width == 4) read_k<4>(A, code, meta, unit, tile, own, lane);
        else if (width == 8) read_k<8>(A, code, meta, unit, tile, own, lane);
        else if (width == 16) read_k<16>(A, code, meta, unit, tile, own, lane);
        else read_k<17>(A, code, meta, unit, tile, own, lane);
    } else {
        code += 512u * d.bits;
        if (width == 2) read_v<2>(A, code, meta, unit, tile, own, lane);
        else if (width == 4) read_v<4>(A, code, meta, unit, tile, own, lane);
        else if (width == 8) read_v<8>(A, code, meta, unit, tile, own, lane);
        else if (width == 16) read_v<16>(A, code, meta, unit, tile, own, lane);
        else read_v<17>(A, code, meta, unit, tile, own, lane);
    }
}

// ----------------------------------------------------------------------------------------------------------- host side

constexpr int64_t kMostWorkgroups = ((1ll << 32) - 1) / 256;  // of 256 threads: a launch has less than 2^32

void release_pages(kvq_cache* c, const std::vector<Page>& pages, size_t from, size_t to) {
    for (size_t i = from; i < to; ++i) {
        c->buddy.release(pages[i].code_unit, order_of_bits(pages[i].bits));
        if (c->has_meta(pages[i].bits)) c->buddy.release(pages[i].meta_unit, 0);
    }
}
// Whether the first n tokens of a block of `from` would leave cache c with a last page that is partly filled below 16 bits while c's policy
// appends at 16: no token could follow.  (A copy of all of a block that no token can follow either is what was asked for.)
bool strands_page(const kvq_cache* c, const kvq_cache* from, const Layer& L, int n) {
    if (n % c->cfg.page_tokens == 0 || !kvq_host::appends_at_16(c) || L.pages[(size_t)(n / c->cfg.page_tokens)].bits == 16) return false;
    return n < L.T || !kvq_host::appends_at_16(from);
}
hipError_t clear_tail(const kvq_cache* c, const Page& p, int n, hipStream_t s) {
    const int in_page = n % c->cfg.page_tokens;  // (not 0)
    if (in_page % KVQ_TILE_TOKENS == 0) return hipSuccess;
    hipLaunchKernelGGL(kvq_clear_tail_kernel, dim3((unsigned)c->units), dim3(64), 0, s, c->arena, c->desc(p), c->tpp, in_page / KVQ_TILE_TOKENS,
                       in_page % KVQ_TILE_TOKENS);
    return hipGetLastError();
}
void set_pages(kvq_cache* c, Layer& L, int n) {  // the block's pages hold n tokens
    const int P = c->cfg.page_tokens;
    for (size_t i = 0; i < L.pages.size(); ++i) L.pages[i].n = std::min(P, n - (int)i * P);
    L.T = n;
    L.resumed = n % P ? n / P : -1;
    L.version++;
    L.plan_tiles = -1;
}

kvq_status_t fork_impl(kvq_cache* dst, kvq_cache* src, int32_t layer, const int32_t* map, int32_t n_tokens, hipStream_t s) {
    const kvq_config_t &a = src->cfg, &b = dst->cfg;
    if (layer < 0 || layer >= a.n_layers || layer >= b.n_layers || n_tokens < -1) return KVQ_E_INVALID;
    if (a.n_kv_heads != b.n_kv_heads || a.page_tokens != b.page_tokens || a.group != b.group || src->tier16 != dst->tier16 || src->dry != dst->dry)
        return KVQ_E_INVALID;
    if (!map && a.batch != b.batch && a.batch != 1) return KVQ_E_INVALID;
    if (reinterpret_cast<uintptr_t>(map) & 3u) return KVQ_E_INVALID;
    Layer &S = src->layers[(size_t)layer], &D = dst->layers[(size_t)layer];
    if (S.poisoned || D.poisoned) return KVQ_E_STATE;
    const int held = S.T, n = n_tokens < 0 ? held : n_tokens, P = a.page_tokens;
    if (n > held || n > b.max_tokens || strands_page(dst, src, S, n)) return KVQ_E_STATE;
    const size_t n_pages = (size_t)((n + P - 1) / P);
    uint64_t bytes = 0;
    for (size_t i = 0; i < n_pages; ++i)
        bytes += (uint64_t)std::min(P, n - (int)i * P) * dst->units * dst->bpth(S.pages[i].bits);
    if (bytes > D.budget) return KVQ_E_BUDGET;
    if (n == 0) {
        kvq_host::empty_block(dst, D);  // (its factors stay, as after kvq_cache_reset)
        kvq_host::start_over_if_empty(dst);
        return KVQ_OK;
    }
    // places for all pages before anything changes: where the old block has a page of the same width it is written over (in another cache;
    // in the same one the old pages are what is read), the others are taken from the arena
    std::vector<Page> pages(S.pages.begin(), S.pages.begin() + (std::ptrdiff_t)n_pages);
    std::vector<uint8_t> used(D.pages.size(), 0);
    std::vector<size_t> fresh;
    fresh.reserve(n_pages);
    size_t next[17] = {};  // by width: where the search for an old page goes on
    for (size_t i = 0; i < n_pages; ++i) {
        Page& p = pages[i];
        bool found = false;
        if (src != dst) {
            size_t& k = next[p.bits];
            while (k < D.pages.size() && D.pages[k].bits != p.bits) ++k;
            if (k < D.pages.size()) {
                p.code_unit = D.pages[k].code_unit;
                p.meta_unit = D.pages[k].meta_unit;
                used[k++] = 1;
                found = true;
            }
        }
        if (found) continue;
        const bool ok = dst->buddy.alloc(order_of_bits(p.bits), &p.code_unit);
        if (!ok || (dst->has_meta(p.bits) && !dst->buddy.alloc(0, &p.meta_unit))) {
            if (ok) dst->buddy.release(p.code_unit, order_of_bits(p.bits));
            for (size_t k : fresh) release_pages(dst, pages, k, k + 1);
            return KVQ_E_OOM;
        }
        fresh.push_back(i);
    }
    kvq_status_t st = kvq_host::ensure_device(dst, s);
    if (st == KVQ_OK) st = kvq_host::ensure_device(src, s);
    if (st != KVQ_OK) {
        for (size_t k : fresh) release_pages(dst, pages, k, k + 1);
        return st;
    }
    // from here on the old block of dst is gone; its pages are reused by work that is enqueued later
    D.pages.swap(pages);
    for (size_t i = 0; i < pages.size(); ++i)
        if (src == dst || !used[i]) release_pages(dst, pages, i, i + 1);
    set_pages(dst, D, n);
    const bool factors = src != dst && S.reparam;
    D.reparam = S.reparam;
    if (dst->dry) return KVQ_OK;
    ForkArgs A;
    A.src = src->arena;
    A.dst = dst->arena;
    A.src_table = src->table_dev(layer);
    A.dst_table = dst->table_dev(layer);
    A.map = map;
    A.src_lambda = src->lambda_dev(layer);
    A.dst_lambda = factors ? dst->lambda_dev(layer) : nullptr;
    A.n_lambda = 2 * a.n_kv_heads * KVQ_D;
    A.src_mark = src->v_mark();
    A.dst_mark = dst->v_mark();
    A.src_batch = a.batch;
    A.dst_batch = b.batch;
    A.n_kv = a.n_kv_heads;
    A.tpp = src->tpp;
    A.n_pages = (int)n_pages;
    A.last_tiles = (n - (int)(n_pages - 1) * P + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS;
    A.groups = (src->tpp + KVQ_FORK_TILES - 1) / KVQ_FORK_TILES;
    A.in_place = src == dst ? 1 : 0;
    const int64_t per_page = (int64_t)A.groups * dst->units;  // (at most 256 x 65,535 workgroups)
    const int most = (int)std::min<int64_t>(KVQ_FORK_ARG_PAGES, kMostWorkgroups / per_page);
    const bool stream = bytes > KVQ_FORK_STREAM_BYTES;
    hipError_t e = hipSuccess;
    for (int at = 0; at < A.n_pages && e == hipSuccess; at += most) {
        A.page0 = at;
        A.n_here = std::min(most, A.n_pages - at);
        for (int i = 0; i < A.n_here; ++i) {
            const KvqPageDesc d = dst->desc(D.pages[(size_t)(at + i)]);
            A.code_off256[i] = d.code_off256;
            A.meta_off256[i] = d.meta_off256;
        }
        hipLaunchKernelGGL(stream ? kvq_fork_kernel<true> : kvq_fork_kernel<false>, dim3((unsigned)(per_page * A.n_here)), dim3(256), 0, s, A);
        e = hipGetLastError();
        if (e == hipSuccess && A.in_place) {
            hipLaunchKernelGGL(kvq_fork_table_kernel, dim3(1), dim3(256), 0, s, A);
            e = hipGetLastError();
        }
    }
    if (e == hipSuccess && n < held && n % P) e = clear_tail(dst, D.pages.back(), n, s);
    if (e != hipSuccess) {
        D.poisoned = true;
        return KVQ_E_HIP;
    }
    return KVQ_OK;
}

}  // namespace

extern "C" {

kvq_status_t kvq_cache_fork(kvq_cache_t* dst, kvq_cache_t* src, int32_t layer, const int32_t* seq_map_dev, int32_t n_tokens,
                            void* hip_stream) {
    if (!dst || !src) return KVQ_E_INVALID;
    try {
        return fork_impl(dst, src, layer, seq_map_dev, n_tokens, as_stream(hip_stream));
    } catch (const std::bad_alloc&) {  // of the host's lists, all of which are made before anything changes
        return KVQ_E_OOM;
    }
}

kvq_status_t kvq_cache_truncate(kvq_cache_t* c, int32_t layer, int32_t n_tokens, void* hip_stream) {
    if (!c || layer < 0 || layer >= c->cfg.n_layers || n_tokens < 0) return KVQ_E_INVALID;
    Layer& L = c->layers[(size_t)layer];
    if (L.poisoned || n_tokens > L.T || strands_page(c, c, L, n_tokens)) return KVQ_E_STATE;
    if (n_tokens == L.T) return KVQ_OK;
    const int P = c->cfg.page_tokens;
    const size_t n_pages = (size_t)((n_tokens + P - 1) / P);
    release_pages(c, L.pages, n_pages, L.pages.size());
    L.pages.resize(n_pages);  // (fewer: nothing is allocated)
    set_pages(c, L, n_tokens);
    if (n_tokens == 0) kvq_host::start_over_if_empty(c);
    if (!c->dry && n_tokens % P && clear_tail(c, L.pages.back(), n_tokens, as_stream(hip_stream)) != hipSuccess) {
        L.poisoned = true;
        return KVQ_E_HIP;
    }
    return KVQ_OK;
}

kvq_status_t kvq_cache_read(kvq_cache_t* c, int32_t layer, int32_t token_begin, int32_t n_tokens, void* k_out_dev, void* v_out_dev,
                            int32_t out_is_fp32, void* hip_stream) {
    if (!c || layer < 0 || layer >= c->cfg.n_layers || token_begin < 0 || n_tokens < 0) return KVQ_E_INVALID;
    if (n_tokens > 0 && (!k_out_dev || !v_out_dev)) return KVQ_E_INVALID;
    for (const void* p : {static_cast<const void*>(k_out_dev), static_cast<const void*>(v_out_dev)})
        if (reinterpret_cast<uintptr_t>(p) & 15u) return KVQ_E_INVALID;
    if (c->dry) return KVQ_E_STATE;
    const Layer& L = c->layers[(size_t)layer];
    if (L.poisoned || (int64_t)token_begin + n_tokens > L.T) return KVQ_E_STATE;
    if (n_tokens == 0) return KVQ_OK;
    ReadArgs A;
    A.arena = c->arena;
    A.table = c->table_dev(layer);
    A.lambda = L.reparam ? c->lambda_dev(layer) : nullptr;
    A.k_out = k_out_dev;
    A.v_out = v_out_dev;
    A.begin = token_begin;
    A.n_tokens = token_begin + n_tokens;
    A.tpp = c->tpp;
    A.tpp_magic = magic_of(c->tpp);
    A.n_kv = c->cfg.n_kv_heads;
    A.first_tile = token_begin / KVQ_TILE_TOKENS;
    A.n_tiles = (A.n_tokens + KVQ_TILE_TOKENS - 1) / KVQ_TILE_TOKENS - A.first_tile;
    A.fp32 = out_is_fp32 ? 1 : 0;
    A.items = (int64_t)c->units * A.n_tiles;
    const int64_t wgs = (A.items + 1) / 2;
    if (wgs > kMostWorkgroups) return KVQ_E_INVALID;
    hipLaunchKernelGGL(kvq_read_kernel, dim3((unsigned)wgs), dim3(256), 0, as_stream(hip_stream), A);
    return hipGetLastError() == hipSuccess ? KVQ_OK : KVQ_E_HIP;
}

}  // extern "C"
