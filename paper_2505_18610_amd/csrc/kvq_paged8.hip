// The paged cache of 8-bit floating point: appends, with the rotation of the keys on the way, and read-back.
#include <cmath>
#include <cstdint>

#include "../../include/kvq.h"
#include "kvq_paged8.h"
#include "kvq_paged8_host.h"

namespace {

using namespace kvq_p8;
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));

struct AppendArgs {
    KvqP8 p;
    const _Float16 *k, *v;
    const float* angles;
    int64_t k_ts, k_hs, v_ts, v_hs;
    int32_t pair;       // 64 or 32: channel i of a run of 2 pair channels is rotated with channel i + pair; 0: ready keys
    int32_t per_seq;    // pages of a sequence that the grid counts with, 0: the workgroup finds its page among all that are touched
};
struct ReadArgs {
    KvqP8 p;
    void *k, *v;
    int64_t k_ts, k_hs, v_ts, v_hs;
    int32_t fp32, per_seq;
};

// The page of a sequence that a workgroup works on: those that rows of the call touch, one after the other.
struct Touched {
    int s, at, page;     // sequence, page of the sequence, page of the cache
    int first, row0;     // the sequence's token that its first row is, and that row
    int begin, end;      // tokens of rows, relative to the page's first token
};
__device__ inline bool touched_page(const KvqP8& P, int per_seq, int id, Touched& T) {
    const auto pages = [&](const Seq& q) {
        const int first = max(0, q.end - q.rows);
        return first < min(q.tokens, first + q.rows) ? ((q.tokens - 1) >> P.page_shift) - (first >> P.page_shift) + 1 : 0;
    };
    int number;
    if (per_seq) {
        T.s = id / per_seq;
        if (T.s >= P.n_seqs) return false;
        number = id - T.s * per_seq;
    } else {
        const auto count = [&](int s) { return pages(seq_of(P, s)); };
        const Census<decltype(count)> census(count, P.n_seqs);
        if (id >= census.total) return false;
        int before;
        T.s = census.find(id, before);
        if (T.s < 0) return false;
        number = id - before;
    }
    const Seq q = seq_of(P, T.s);
    if (number >= pages(q)) return false;
    T.first = q.end - q.rows;
    T.row0 = q.row0;
    T.at = (max(0, T.first) >> P.page_shift) + number;
    T.page = page_of(P, T.s, T.at);
    if (T.page < 0) return false;
    const int token0 = T.at << P.page_shift;
    T.begin = max(0, max(0, T.first) - token0);
    T.end = min(1 << P.page_shift, q.tokens - token0);
    return true;
}

// The smallest e >= KVQ_P8_LOW with x <= 448 2^e, for finite x >= 0: 448 = 7/8 2^9.
__device__ inline int exponent_for(float x) {
    const uint32_t b = __float_as_uint(x);
    const int e = (int)(b >> 23) - 126 - 9 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, KVQ_P8_LOW);
}
__device__ inline float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
// What is not finite becomes NaN (infinity times zero); finite values stay.
__device__ inline float finite_or_nan(float x) { return fmaf(x, 0.f, x); }
__device__ inline uint32_t codes4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Four codes multiplied by a power of two of at most one, rounded again.
__device__ inline uint32_t lower_codes(uint32_t w, float factor) {
    const float2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return codes4(a[0] * factor, a[1] * factor, b[0] * factor, b[1] * factor);
}
// Bytes that belong to set bits of an 8-bit mask, for four codes.
__device__ inline uint32_t byte_mask(uint32_t bits) {
    return ((bits & 1u) | (bits & 2u) << 7 | (bits & 4u) << 14 | (bits & 8u) << 21) * 0xffu;
}

// Between rows and tiles codes pass through LDS, a tile of a wavefront's own.  A lane (j, m) of the row side has channels 8 m .. 8 m + 7 of tokens
// 8 j .. 8 j + 7, and reads or writes eight bytes at a time: keys of one token, values of one channel.  Chunks lie a little turned, so that
// the 64 lanes of such an access meet every bank as often (as in memory 16 lanes met one).
template <bool KEYS>
__device__ inline int chunk_in_lds(int c, int j, int n) {
    return (c * 64 + 16 * j + (KEYS ? (n & 12) | ((n + j) & 3) : (n & 8) | ((n + j + 4 * c) & 7))) * 16;
}
template <bool KEYS>
__device__ inline int eight_in_lds(int j, int m, int i) {  // KEYS: token 8 j + i; else channel 8 m + i
    if (KEYS) return chunk_in_lds<true>((i >> 2) * 2 + (m >> 3), m & 3, 4 * j + (i & 3)) + ((m >> 2) & 1) * 8;
    return chunk_in_lds<false>(m >> 2, j, 8 * (m & 1) + i) + ((m >> 1) & 1) * 8;
}
// (written and read by one wavefront, whose LDS accesses stay in order)
__device__ inline void lds_written() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// The value of lane m ^ 8, or of lane m ^ 4, of the 16 lanes of a row.
__device__ inline float partner(float x, int m, bool eight) {
    const int v = __float_as_int(x);
    const int by8 = __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);                                                          // row_ror:8
    const int up = __builtin_amdgcn_mov_dpp(v, 0x124, 0xf, 0xf, true), down = __builtin_amdgcn_mov_dpp(v, 0x12c, 0xf, 0xf, true);  // row_ror:4, 12
    return __int_as_float(eight ? by8 : m & 4 ? up : down);
}

// One page's keys or values of one head a workgroup, a tile a wavefront, in three steps: load (and rotate) the new tokens and take the
// largest magnitude, over all wavefronts; settle the scale; round and store.  The new values stay in registers in between.
// Rows are loaded whole, by 16 lanes; the channel that one is rotated with is 8 or 4 lanes on.  Memory bounds it: four prompts of 32,768 tokens x 8 heads
// 190 us = 4.6 TB/s (248 with keys loaded in the tile's order, 64 bytes of a row by four lanes, and values scattered into the tile).  95 registers:
// with more than 96 a SIMD holds four wavefronts instead of five, 210 us.
template <bool KEYS>
__device__ inline void append_page(const AppendArgs& A, const Touched& T, int kv, uint8_t* lds, uint32_t* wave_max) {
    const KvqP8& P = A.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, n = lane & 15;
    const int tok0 = wave * 32;  // of the page
    const bool any_new = tok0 < T.end && tok0 + 32 > T.begin, any_old = tok0 < T.begin;
    int32_t* const word = P.words + ((int64_t)T.page * P.n_kv + kv) * 2 + (KEYS ? 0 : 1);
    const int old_word = T.begin > 0 ? *word : 0;
    uint8_t* const tile = tile_of(P, T.page, kv, wave) + (KEYS ? 0 : KVQ_P8_TILE_BYTES / 2);
    const int64_t row = (int64_t)T.row0 + ((T.at << P.page_shift) - T.first) + tok0 + 8 * j;  // of the lane's first token
    const auto is_new = [&](int t) { return tok0 + t >= T.begin && tok0 + t < T.end; };       // t: token of the tile

    float x[8][8];  // token 8 j + i, channel 8 n + e
    float largest = 0.f;
    bool nan = false;
    if (any_new) {
        half8 w[8];
        const _Float16* const src = KEYS ? A.k + row * A.k_ts + kv * A.k_hs + 8 * n : A.v + row * A.v_ts + kv * A.v_hs + 8 * n;
        const int64_t step = KEYS ? A.k_ts : A.v_ts;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = half8{};
            if (is_new(8 * j + i)) w[i] = __builtin_nontemporal_load(reinterpret_cast<const half8*>(src + i * step));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = (float)w[i][e];
            if (!__any(is_new(8 * j + i))) continue;  // (of a decode step one of eight)
            if (KEYS && A.pair) {
                float c[8] = {}, s[8] = {};
                if (is_new(8 * j + i)) {
                    const float* const at = A.angles + (row + i) * (2 * A.pair) + ((8 * n) & (A.pair - 1));
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        const float4v cc = *reinterpret_cast<const float4v*>(at + e), ss = *reinterpret_cast<const float4v*>(at + A.pair + e);
#pragma unroll
                        for (int d = 0; d < 4; ++d) c[e + d] = cc[d], s[e + d] = ss[d];
                    }
                }
                const bool eight = A.pair == 64, upper = n & (eight ? 8 : 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // (each product and the sum rounded by itself, as elsewhere in the library)
                    const float other = __fmul_rn(partner(x[i][e], n, eight), s[e]), own = __fmul_rn(x[i][e], c[e]);
                    x[i][e] = upper ? __fadd_rn(other, own) : __fsub_rn(own, other);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[i][e] = finite_or_nan(x[i][e]);
                largest = fmaxf(largest, fabsf(x[i][e]));  // (passes over NaN)
                nan = nan || x[i][e] != x[i][e];
            }
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));
    const bool wave_nan = __any(nan);
    if (lane == 0) wave_max[wave] = __float_as_uint(largest) | (wave_nan ? 1u << 31 : 0u);  // (the sign: whether any is NaN)
    __syncthreads();
    const int waves = blockDim.x >> 6;
    uint32_t any_nan = 0;
    largest = 0.f;
    for (int w = 0; w < waves; ++w) {
        const uint32_t x = wave_max[w];
        largest = fmaxf(largest, __uint_as_float(x & 0x7fffffffu));
        any_nan |= x >> 31;
    }
    int e = exponent_for(largest);
    const int e_old = exponent_of(old_word);
    if (T.begin > 0) e = max(e, e_old);
    if (threadIdx.x == 0) *word = (e + KVQ_P8_BIAS) | (any_nan ? KVQ_P8_NAN : 0) | (old_word & KVQ_P8_NAN);

    const bool lowered = any_old && e != e_old;  // the wavefront's held codes are rounded to the new scale
    if (!any_new && !lowered) return;
    const float factor = lowered ? power_of_two(max(e_old - e, -126)) : 1.f;
    const auto code4 = [&](float a, float b, float c, float d) {
        return codes4(__builtin_ldexpf(a, -e), __builtin_ldexpf(b, -e), __builtin_ldexpf(c, -e), __builtin_ldexpf(d, -e));
    };
    u32x4 held[4] = {};  // the tile's strings, where tokens are held that change or share a word with new ones
    if (any_old) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            held[c] = *reinterpret_cast<const u32x4*>(tile + (c * 64 + lane) * 16);
            if (lowered)
#pragma unroll
                for (int d = 0; d < 4; ++d) held[c][d] = lower_codes(held[c][d], factor);
        }
    }
    u32x4 fresh[4] = {};
    if (any_new) {
        uint8_t* const at = lds + wave * 4096;
#pragma unroll
        for (int k = 0; k < 8; ++k) {  // KEYS: token 8 j + k; else channel 8 n + k
            u32x2 w;
            if (KEYS) w = u32x2{code4(x[k][0], x[k][1], x[k][2], x[k][3]), code4(x[k][4], x[k][5], x[k][6], x[k][7])};
            else w = u32x2{code4(x[0][k], x[1][k], x[2][k], x[3][k]), code4(x[4][k], x[5][k], x[6][k], x[7][k])};
            *reinterpret_cast<u32x2*>(at + eight_in_lds<KEYS>(j, n, k)) = w;
        }
        lds_written();
#pragma unroll
        for (int c = 0; c < 4; ++c) fresh[c] = *reinterpret_cast<const u32x4*>(at + chunk_in_lds<KEYS>(c, j, n));
    }
    // A tile that held no token is written whole: slots that hold none are zero.
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        u32x4 w = fresh[c];
        if (any_old) {
            if (KEYS) {
                if (!is_new(8 * (n >> 2) + 4 * (c >> 1) + (n & 3))) {
                    if (!lowered) continue;
                    w = held[c];
                }
            } else {
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) bits |= (is_new(8 * j + i) ? 1u : 0u) << i;
                const u32x4 mask = {byte_mask(bits), byte_mask(bits >> 4), byte_mask(bits), byte_mask(bits >> 4)};
                w = (fresh[c] & mask) | (held[c] & ~mask);
                if (bits == 0 && !lowered) continue;
            }
        }
        *reinterpret_cast<u32x4*>(tile + (c * 64 + lane) * 16) = w;
    }
}

// What a workgroup works on: the heads and kinds of eight pages in turn, so that those of one page, which read the same angles, are on one XCD.
struct Job {
    int page, kv, kind;
};
__device__ inline Job job_of(int n_kv) {
    const int of_page = blockIdx.x >> 3, page8 = of_page / (2 * n_kv), at = of_page - page8 * 2 * n_kv;
    return Job{page8 * 8 + ((int)blockIdx.x & 7), at >> 1, at & 1};
}

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void kvq_paged8_append_kernel(const AppendArgs A) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[WAVES * 4096];
    __shared__ uint32_t wave_max[WAVES];
    Touched T;
    const Job job = job_of(A.p.n_kv);
    if (!touched_page(A.p, A.per_seq, job.page, T)) return;
    if (job.kind == 0) append_page<true>(A, T, job.kv, lds, wave_max);
    else append_page<false>(A, T, job.kv, lds, wave_max);
}

// Cached tokens as values, a tile of keys or values a wavefront; rows are stored whole, by 16 lanes.  4 x 32,768 tokens x 8 heads into fp16 145 us = 5.5 TB/s (203
// with half lines of keys and eight bytes at a time of values).
template <bool FP32>
__device__ inline void store_values(void* to, int64_t at, const float (&x)[8]) {
    if (FP32) {
        float* const f = static_cast<float*>(to) + at;
        __builtin_nontemporal_store(float4v{x[0], x[1], x[2], x[3]}, reinterpret_cast<float4v*>(f));
        __builtin_nontemporal_store(float4v{x[4], x[5], x[6], x[7]}, reinterpret_cast<float4v*>(f + 4));
    } else {
        half8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (_Float16)half_range(x[e]);
        __builtin_nontemporal_store(h, reinterpret_cast<half8*>(static_cast<_Float16*>(to) + at));
    }
}
__device__ inline float byte_value(uint32_t w, int byte) {
    return byte == 0 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 0) : byte == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 1)
         : byte == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 2) : __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}
template <bool FP32, bool KEYS>
__device__ inline void read_page(const ReadArgs& A, const Touched& T, int kv, uint8_t* lds) {
    const KvqP8& P = A.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, n = lane & 15;
    const int tok0 = wave * 32;
    if (tok0 >= T.end || tok0 + 32 <= T.begin) return;
    const uint8_t* const tile = tile_of(P, T.page, kv, wave) + (KEYS ? 0 : KVQ_P8_TILE_BYTES / 2);
    uint8_t* const in = lds + wave * 4096;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *reinterpret_cast<u32x4*>(in + chunk_in_lds<KEYS>(c, j, n)) = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(tile + (c * 64 + lane) * 16));
    const float scale = ldexpf(1.f, exponent_of(P.words[((int64_t)T.page * P.n_kv + kv) * 2 + (KEYS ? 0 : 1)]));
    lds_written();
    u32x2 w[8];  // KEYS: token 8 j + k; else channel 8 n + k
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const u32x2*>(in + eight_in_lds<KEYS>(j, n, k));
    const int64_t row = (int64_t)T.row0 + ((T.at << P.page_shift) - T.first) + tok0 + 8 * j;
    void* const to = KEYS ? A.k : A.v;
    const int64_t step = KEYS ? A.k_ts : A.v_ts, at = row * step + kv * (KEYS ? A.k_hs : A.v_hs) + 8 * n;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int t = tok0 + 8 * j + i;
        if (t < T.begin || t >= T.end) continue;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (KEYS ? byte_value(w[i][e >> 2], e & 3) : byte_value(w[e][i >> 2], i & 3)) * scale;
        store_values<FP32>(to, at + i * step, x);
    }
}
template <bool FP32, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void kvq_paged8_read_kernel(const ReadArgs A) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[WAVES * 4096];
    Touched T;
    const Job job = job_of(A.p.n_kv);
    if (!touched_page(A.p, A.per_seq, job.page, T)) return;
    if (job.kind == 0) read_page<FP32, true>(A, T, job.kv, lds);
    else read_page<FP32, false>(A, T, job.kv, lds);
}

// Workgroups that a call over the pages that rows touch needs, and pages of a sequence to count with (0: workgroups find theirs): straight
// where every sequence touches few, else as many as rows and sequences allow for.
int64_t touched_pages(const KvqP8& P, int32_t& per_seq) {
    const int64_t page = 1ll << P.page_shift, each = std::min<int64_t>((P.max_rows + page - 2) / page + 1, P.table_pages);
    const int64_t straight = each * P.n_seqs, found = P.n_rows / page + 2ll * P.n_seqs;
    per_seq = P.n_seqs == 1 || straight <= found ? (int32_t)each : 0;
    return per_seq ? straight : found;
}

template <class Args, class Kernel>
kvq_status_t launch(Kernel const (&kernels)[4], Args& A, hipStream_t stream) {
    const int64_t groups = ((touched_pages(A.p, A.per_seq) + 7) & ~7ll) * A.p.n_kv * 2;
    if (groups > INT32_MAX / (32 << (A.p.page_shift - 4))) return KVQ_E_INVALID;  // threads of a launch stay below 2^32
    const int waves = 1 << (A.p.page_shift - 5);
    hipLaunchKernelGGL(kernels[A.p.page_shift - 5], dim3((unsigned)groups), dim3(64 * waves), 0, stream, A);
    return hipGetLastError() == hipSuccess ? KVQ_OK : KVQ_E_HIP;
}

}  // namespace

extern "C" {

kvq_status_t kvq_paged8_append(const kvq_paged8_t* cache, const kvq_paged8_batch_t* batch, const kvq_paged8_rows_t* k_dev,
                               const kvq_paged8_rows_t* v_dev, const float* cos_sin_dev, int32_t pair, void* hip_stream) {
    AppendArgs A{};
    if (!kvq_p8_args(cache, batch, A.p)) return KVQ_E_INVALID;
    if (!kvq_p8_rows_ok(k_dev, batch, 8) || !kvq_p8_rows_ok(v_dev, batch, 8)) return KVQ_E_INVALID;
    if (cos_sin_dev && pair != 64 && pair != 32) return KVQ_E_INVALID;
    if (reinterpret_cast<uintptr_t>(cos_sin_dev) & 15u) return KVQ_E_INVALID;
    if (!A.p.n_seqs || !A.p.n_rows) return KVQ_OK;
    A.k = static_cast<const _Float16*>(k_dev->data_dev);
    A.v = static_cast<const _Float16*>(v_dev->data_dev);
    A.k_ts = k_dev->row_stride; A.k_hs = k_dev->head_stride;
    A.v_ts = v_dev->row_stride; A.v_hs = v_dev->head_stride;
    A.angles = cos_sin_dev;
    A.pair = cos_sin_dev ? pair : 0;
    void (*const kernels[4])(AppendArgs) = {kvq_paged8_append_kernel<1>, kvq_paged8_append_kernel<2>, kvq_paged8_append_kernel<4>,
                                            kvq_paged8_append_kernel<8>};
    return launch(kernels, A, static_cast<hipStream_t>(hip_stream));
}

kvq_status_t kvq_paged8_read(const kvq_paged8_t* cache, const kvq_paged8_batch_t* batch, const kvq_paged8_rows_t* k_out_dev,
                             const kvq_paged8_rows_t* v_out_dev, int32_t out_is_fp32, void* hip_stream) {
    ReadArgs A{};
    if (!kvq_p8_args(cache, batch, A.p)) return KVQ_E_INVALID;
    const int align = out_is_fp32 ? 4 : 8;
    for (const kvq_paged8_rows_t* r : {k_out_dev, v_out_dev})
        if (!kvq_p8_rows_ok(r, batch, align) || !kvq_p8_rows_apart(r, batch, cache->n_kv_heads)) return KVQ_E_INVALID;
    if (!A.p.n_seqs || !A.p.n_rows) return KVQ_OK;
    A.k = const_cast<void*>(k_out_dev->data_dev);
    A.v = const_cast<void*>(v_out_dev->data_dev);
    A.k_ts = k_out_dev->row_stride; A.k_hs = k_out_dev->head_stride;
    A.v_ts = v_out_dev->row_stride; A.v_hs = v_out_dev->head_stride;
    A.fp32 = out_is_fp32 ? 1 : 0;
    void (*const half[4])(ReadArgs) = {kvq_paged8_read_kernel<false, 1>, kvq_paged8_read_kernel<false, 2>, kvq_paged8_read_kernel<false, 4>,
                                       kvq_paged8_read_kernel<false, 8>};
    void (*const full[4])(ReadArgs) = {kvq_paged8_read_kernel<true, 1>, kvq_paged8_read_kernel<true, 2>, kvq_paged8_read_kernel<true, 4>,
                                       kvq_paged8_read_kernel<true, 8>};
    return launch(out_is_fp32 ? full : half, A, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
