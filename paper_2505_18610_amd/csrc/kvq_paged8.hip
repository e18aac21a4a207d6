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
        const int first = max(0, q.tokens - q.rows);
        return q.rows && q.tokens ? ((q.tokens - 1) >> P.page_shift) - (first >> P.page_shift) + 1 : 0;
    };
    int number;
    if (per_seq) {
        T.s = id / per_seq;
        number = id - T.s * per_seq;
    } else {
        const auto count = [&](int s) { return pages(seq_of(P, s)); };
        const Census<decltype(count)> census(count, P.n_seqs);
        if (id >= census.total) return false;
        int before;
        T.s = census.find(id, before);
        number = id - before;
    }
    const Seq q = seq_of(P, T.s);
    if (number >= pages(q)) return false;
    T.first = q.tokens - q.rows;
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

// One page's keys or values of one head a workgroup, a tile a wavefront, in three steps: load (and rotate) the new tokens and take the
// largest magnitude, over all wavefronts; settle the scale; round and store.  The new values stay in registers in between.
// Keys are loaded where the tile's layout wants them, 64 bytes of a row by four lanes; values as whole rows by 16 lanes, eight tokens
// a lane, which makes the four codes of a word four tokens of one channel; they pass through LDS into the layout's order.
template <bool KEYS>
__device__ inline void append_page(const AppendArgs& A, const Touched& T, int kv, uint8_t* lds, float* wave_max) {
    const KvqP8& P = A.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, n = lane & 15;
    const int tok0 = wave * 32;  // of the page
    const bool any_new = tok0 < T.end && tok0 + 32 > T.begin, any_old = tok0 < T.begin;
    int32_t* const word = P.words + ((int64_t)T.page * P.n_kv + kv) * 2 + (KEYS ? 0 : 1);
    const int old_word = T.begin > 0 ? *word : 0;
    uint8_t* const tile = tile_of(P, T.page, kv, wave) + (KEYS ? 0 : KVQ_P8_TILE_BYTES / 2);
    const int64_t row = (int64_t)T.row0 + ((T.at << P.page_shift) - T.first);  // the row that the page's first token would be

    // slots: KEYS: x[4 sub + grp][i], token 8 (n / 4) + 4 sub + n % 4, channel 32 grp + 8 j + i; else x[i][e], token 8 j + i, channel 8 n + e
    float x[8][8];
    float largest = 0.f;
    bool nan = false;
    const auto slot_token = [&](int a) { return tok0 + (KEYS ? 8 * (n >> 2) + 4 * (a >> 2) + (n & 3) : 8 * j + a); };
    const auto is_new = [&](int a) { const int t = slot_token(a); return t >= T.begin && t < T.end; };
    if (any_new) {
#pragma unroll
        for (int a = 0; a < 8; ++a) {
            half8 w = {};
            if (is_new(a)) {
                const int64_t r = row + slot_token(a);
                w = KEYS ? *reinterpret_cast<const half8*>(A.k + r * A.k_ts + kv * A.k_hs + 32 * (a & 3) + 8 * j)
                         : *reinterpret_cast<const half8*>(A.v + r * A.v_ts + kv * A.v_hs + 8 * n);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[a][e] = (float)w[e];
        }
        if (KEYS && A.pair) {
            // a pair's channels are 64 or 32 apart: groups of 32 channels of one lane
            const int step = A.pair >> 5;  // groups between them
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                if (!is_new(4 * sub)) continue;
                const float* const angles = A.angles + (row + slot_token(4 * sub)) * (2 * A.pair);
#pragma unroll
                for (int g = 0; g < 2; ++g) {  // the pair's number among the lane's
                    const float* const at = angles + (step == 2 ? 32 * g : 0) + 8 * j;
                    float c[8], s[8];
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        const float4v cc = *reinterpret_cast<const float4v*>(at + e), ss = *reinterpret_cast<const float4v*>(at + A.pair + e);
#pragma unroll
                        for (int d = 0; d < 4; ++d) c[e + d] = cc[d], s[e + d] = ss[d];
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = step == 2 ? x[4 * sub + g][e] : x[4 * sub + 2 * g][e];
                        const float b = step == 2 ? x[4 * sub + g + 2][e] : x[4 * sub + 2 * g + 1][e];
                        // (each product and the sum rounded by itself, as elsewhere in the library)
                        const float lo = __fsub_rn(__fmul_rn(a, c[e]), __fmul_rn(b, s[e]));
                        const float hi = __fadd_rn(__fmul_rn(a, s[e]), __fmul_rn(b, c[e]));
                        if (step == 2) x[4 * sub + g][e] = lo, x[4 * sub + g + 2][e] = hi;
                        else x[4 * sub + 2 * g][e] = lo, x[4 * sub + 2 * g + 1][e] = hi;
                    }
                }
            }
        }
#pragma unroll
        for (int a = 0; a < 8; ++a)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[a][e] = finite_or_nan(x[a][e]);
                largest = fmaxf(largest, fabsf(x[a][e]));  // (passes over NaN)
                nan = nan || x[a][e] != x[a][e];
            }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));
    if (lane == 0) wave_max[wave] = largest;
    const int any_nan = __syncthreads_or(nan ? 1 : 0);
    const int waves = blockDim.x >> 6;
    largest = 0.f;
    for (int w = 0; w < waves; ++w) largest = fmaxf(largest, wave_max[w]);
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
        if (KEYS) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const float* const y = &x[2 * c + (d >> 1)][4 * (d & 1)];
                    fresh[c][d] = code4(y[0], y[1], y[2], y[3]);
                }
        } else {
            uint8_t* const at = lds + wave * 4096;
#pragma unroll
            for (int c = 0; c < 8; ++c) {  // channel 8 n + c: its eight tokens
                const int ch = 8 * n + c;
                const u32x2 w = {code4(x[0][c], x[1][c], x[2][c], x[3][c]), code4(x[4][c], x[5][c], x[6][c], x[7][c])};
                *reinterpret_cast<u32x2*>(at + ((ch >> 5) * 64 + 16 * j + (ch & 15)) * 16 + ((ch >> 4) & 1) * 8) = w;
            }
            // (written and read by one wavefront, whose LDS accesses stay in order)
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int c = 0; c < 4; ++c) fresh[c] = *reinterpret_cast<const u32x4*>(at + (c * 64 + lane) * 16);
        }
    }
    // A tile that held no token is written whole: slots that hold none are zero.
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        u32x4 w = fresh[c];
        if (any_old) {
            if (KEYS) {
                const bool take = is_new(4 * (c >> 1));
                if (!take) {
                    if (!lowered) continue;
                    w = held[c];
                }
            } else {
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) bits |= (is_new(i) ? 1u : 0u) << i;
                const u32x4 mask = {byte_mask(bits), byte_mask(bits >> 4), byte_mask(bits), byte_mask(bits >> 4)};
                w = (fresh[c] & mask) | (held[c] & ~mask);
                if (bits == 0 && !lowered) continue;
            }
        }
        *reinterpret_cast<u32x4*>(tile + (c * 64 + lane) * 16) = w;
    }
}

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void kvq_paged8_append_kernel(const AppendArgs A) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[WAVES * 4096];
    __shared__ float wave_max[WAVES];
    Touched T;
    const int kind = blockIdx.x & 1, at = blockIdx.x >> 1, kv = at % A.p.n_kv;
    if (!touched_page(A.p, A.per_seq, at / A.p.n_kv, T)) return;
    if (kind == 0) append_page<true>(A, T, kv, lds, wave_max);
    else append_page<false>(A, T, kv, lds, wave_max);
}

// Cached tokens as values, a tile of keys or values a wavefront.
template <bool FP32>
__device__ inline void store_values(void* to, int64_t at, const float (&x)[8]) {
    if (FP32) {
        float* const f = static_cast<float*>(to) + at;
        *reinterpret_cast<float4v*>(f) = float4v{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<float4v*>(f + 4) = float4v{x[4], x[5], x[6], x[7]};
    } else {
        half8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // a rounded code may lie beyond the largest value; NaN stays
            const float y = fabsf(x[e]) > 65504.f ? copysignf(65504.f, x[e]) : x[e];
            h[e] = (_Float16)y;
        }
        *reinterpret_cast<half8*>(static_cast<_Float16*>(to) + at) = h;
    }
}
__device__ inline float byte_value(uint32_t w, int byte) {
    return byte == 0 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 0) : byte == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 1)
         : byte == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)w, 2) : __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}
template <bool FP32, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void kvq_paged8_read_kernel(const ReadArgs A) {
    const KvqP8& P = A.p;
    Touched T;
    const int kind = blockIdx.x & 1, at = blockIdx.x >> 1, kv = at % P.n_kv;
    if (!touched_page(P, A.per_seq, at / P.n_kv, T)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, n = lane & 15;
    const int tok0 = wave * 32;
    if (tok0 >= T.end || tok0 + 32 <= T.begin) return;
    const uint8_t* const tile = tile_of(P, T.page, kv, wave) + kind * (KVQ_P8_TILE_BYTES / 2);
    const float scale = ldexpf(1.f, exponent_of(P.words[((int64_t)T.page * P.n_kv + kv) * 2 + kind]));
    const int64_t row = (int64_t)T.row0 + ((T.at << P.page_shift) - T.first);
    if (kind == 0) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(tile + (c * 64 + lane) * 16);
            const int t = tok0 + 8 * (n >> 2) + 4 * (c >> 1) + (n & 3);
            if (t < T.begin || t >= T.end) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = byte_value(w[2 * h + (e >> 2)], e & 3) * scale;
                store_values<FP32>(A.k, (row + t) * A.k_ts + kv * A.k_hs + 64 * (c & 1) + 32 * h + 8 * j, x);
            }
        }
    } else {
        u32x2 w[8];  // channel 8 n + e: eight tokens
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int ch = 8 * n + e;
            w[e] = *reinterpret_cast<const u32x2*>(tile + ((ch >> 5) * 64 + 16 * j + (ch & 15)) * 16 + ((ch >> 4) & 1) * 8);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = tok0 + 8 * j + i;
            if (t < T.begin || t >= T.end) continue;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = byte_value(w[e][i >> 2], i & 3) * scale;
            store_values<FP32>(A.v, (row + t) * A.v_ts + kv * A.v_hs + 8 * n, x);
        }
    }
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
    const int64_t groups = touched_pages(A.p, A.per_seq) * A.p.n_kv * 2;
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
