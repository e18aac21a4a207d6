// Device code shared by prompt attention and tree attention (gfx950): attention of many query rows over 32-token tiles of fp16
// keys and values, one pass with a running maximum and sum.
//
// Both contractions are taken transposed, with v_mfma_f32_16x16x32_f16 and the rows in its N dimension:
//   S^T[token, row] = K q^T,   O^T[channel, row] += V^T P^T.
// lane = 16 j + n.  The K operand's rows are dealt so that lane quarter j receives the scores of tokens 8j .. 8j + 7 of row n, which
// after exponentiation are the B operand of the second product as they stand: nothing crosses lanes between the products.  A
// wavefront carries R groups of 16 rows, so an operand read from LDS serves R products.
//
// Statistics, in 32 bits: a reference per row in log2 units, which is set 2^KVQ_BELOW below the row's maximum and follows it when that is more
// than 2^KVQ_FOLLOW above where it was (a rescaling of the accumulators then; with every new maximum 38 % of the tiles of 128 had one, 20
// instructions a tile and group of rows), and the sum of the probabilities as rounded to fp16 for the second product, so that a row
// that one key dominates gets its values back as they are.  Where the caller asks for the log of the sum it is taken from the unrounded ones
// beside it.  Probabilities so lie below 2^(KVQ_BELOW + KVQ_FOLLOW) = 2^15, within fp16, and what the rounding of a small one loses, 2^-25 at
// most, is 2^-(25 + KVQ_BELOW) of the weight of the row's leading key (with the reference at the maximum 131,072 equal keys 17 nats below
// a leading one were 44 % too heavy and 18 nats below it lost; 0.1 % and 0.9 % now).  Half a per cent of a prompt's time, 1 % of a tree's.
#ifndef KVQ_FLASH_H
#define KVQ_FLASH_H

#include <hip/hip_runtime.h>
#include "kvq_layout.h"

namespace kvq_flash {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));

#define KVQ_FLASH_TILE_BYTES 8192  // one fp16 K or V tile in LDS
#define KVQ_BELOW 7.f
#define KVQ_FOLLOW 8.f

#ifdef KVQ_NO_ARITHMETIC  // the measurement build (build.py) loads tiles and computes on none
__device__ inline float4v mma(half8, half8, float4v c) { return c; }
__device__ inline float4v mma16(half4, half4, float4v c) { return c; }
#else
__device__ inline float4v mma(half8 a, half8 b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline float4v mma16(half4 a, half4 b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0); }
#endif
__device__ inline uint32_t pack2(float a, float b) {
    const half2v h = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, h);
}
// over the four lane quarters, in every lane
__device__ inline float quarters_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float quarters_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <int R>
struct State {
    float4v o[R][8];  // o[r][nt][i]: channel 16 nt + 4 j + i of row n of group r
    float m[R];       // the reference (log2 units), equal in the four quarters
    float l[R];       // this quarter's share of the sum
    float fine[R];    // the same of the unrounded probabilities
    __device__ void clear() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -INFINITY;
            l[r] = fine[r] = 0.f;
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) o[r][nt] = float4v{0.f, 0.f, 0.f, 0.f};
        }
    }
};

// What is subtracted from a score: the reference, or zero while nothing has been seen (exp2(-inf - -inf) would be NaN).
__device__ inline float reference_of(float m) { return m == -INFINITY ? 0.f : m; }

// Probabilities of TT tiles for row group r from raw scores s (before the scale), masked ones at -inf; p in the order of the V
// operand: natural, or (v, v + 4) pairs of a quarter's eight tokens.  FINE: whether `fine` may be asked for.
template <int R, int TT, bool PAIRED, bool FINE>
__device__ inline void softmax_group(State<R>& st, int r, const float4v (&s)[TT][2], float scale_log2, bool fine, uint32_t (&p)[TT][4]) {
    float lmax = -INFINITY;
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int i = 0; i < 4; ++i) lmax = fmaxf(lmax, s[t][sub][i]);
    lmax *= scale_log2;
    if (__any(lmax > st.m[r] + (KVQ_BELOW + KVQ_FOLLOW))) {
        const float m_new = fmaxf(st.m[r], quarters_max(lmax) - KVQ_BELOW);
        const float alpha = __builtin_amdgcn_exp2f(st.m[r] - reference_of(m_new));  // 0 for the first scores
        st.l[r] *= alpha;
        if (FINE) st.fine[r] *= alpha;
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
            for (int i = 0; i < 4; ++i) e[sub][i] = __builtin_amdgcn_exp2f(fmaf(s[t][sub][i], scale_log2, -ref));
        if (FINE && fine) {
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.fine[r] += e[sub][i];
        }
        if constexpr (PAIRED) {
#pragma unroll
            for (int v = 0; v < 4; ++v) p[t][v] = pack2(e[0][v], e[1][v]);
        } else {
            p[t][0] = pack2(e[0][0], e[0][1]);
            p[t][1] = pack2(e[0][2], e[0][3]);
            p[t][2] = pack2(e[1][0], e[1][1]);
            p[t][3] = pack2(e[1][2], e[1][3]);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const uint32_t two = p[t][v];
            st.l[r] = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, two), ones, st.l[r], false);
        }
    }
}

__device__ inline half8 to_half8(const uint32_t (&w)[4]) {
    const u32x4 v = {w[0], w[1], w[2], w[3]};
    return __builtin_bit_cast(half8, v);
}
__device__ inline half8 to_half8(u32x4 v) { return __builtin_bit_cast(half8, v); }

// A V tile in LDS, row-major in blocks that the transposing read takes whole: token 8 j + 4 h + k, channel 16 nt + c at byte
// ((2 nt + h) 64 + 16 j + 4 k) 8 + 2 c.  A read covers 512 consecutive bytes; of 16 lanes, lane n receives channel n of four tokens.
__device__ inline half8 read_v(const uint8_t* tile, int nt, int lane) {
    typedef __attribute__((address_space(3))) short4v lds_short4;
    const uint8_t* at = tile + (nt * 128 + lane) * 8;
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(at));
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(at + 512));
    const auto both = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(half8, both);
}
// Where the 16 bytes of (token, chunk of 8 channels) go in such a tile, and in a K tile (operand order).
__device__ inline int v_chunk_at(int token, int chunk) {
    return ((chunk >> 1) * 128 + ((token >> 2) & 1) * 64 + (token >> 3) * 16 + (token & 3) * 4 + (chunk & 1) * 2) * 8;
}
__device__ inline int k_chunk_at(int token, int chunk) {
    return ((((token >> 2) & 1) * 4 + (chunk >> 2)) * 64 + (chunk & 3) * 16 + (token >> 3) * 4 + (token & 3)) * 16;
}

// A lane's eight values of one V operand added to `seen` times zero: 0 stays 0 unless one of them is infinite or NaN.
__device__ inline void watch_nonfinite(half8 v, uint32_t& seen) {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    half2v acc = __builtin_bit_cast(half2v, seen);
    const half2v zero = {(_Float16)0.f, (_Float16)0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t two = w[e];  // (a bit cast of a vector's element itself takes its first one)
        acc += __builtin_bit_cast(half2v, two) * zero;
    }
    seen = __builtin_bit_cast(uint32_t, acc) & 0x7fff7fffu;
}

// Infinite and NaN values of V: a key that a row does not see must not reach it, not even as zero times infinity.  Where there are any they
// are taken as zeros, and their number among the keys that each row sees is counted apart, by products: infinities of either sign
// and NaNs.  What they add to a row is added behind everything else, to what has been stored: nothing takes an infinity or a NaN out
// of a sum again.  Slow, and rare.
__device__ inline u32x4 finite_only(u32x4 v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t w = v[e];
        if ((w & 0x7c00u) == 0x7c00u) w &= 0xffff0000u;
        if ((w & 0x7c000000u) == 0x7c000000u) w &= 0x0000ffffu;
        v[e] = w;
    }
    return v;
}
struct NonfiniteCount {
    float4v count[3] = {};
    // v: the lane's eight values of a V operand; sees: 1 for the tokens that row n sees, 0 for the others
    __device__ void add(const uint16_t (&v)[8], half8 sees) {
        half8 kind[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            kind[0][e] = v[e] == 0x7c00u ? (_Float16)1.f : (_Float16)0.f;
            kind[1][e] = v[e] == 0xfc00u ? (_Float16)1.f : (_Float16)0.f;
            kind[2][e] = (v[e] & 0x7fffu) > 0x7c00u ? (_Float16)1.f : (_Float16)0.f;
        }
#pragma unroll
        for (int c = 0; c < 3; ++c) count[c] = mma(kind[c], sees, count[c]);
    }
    __device__ float4v sum() const {
        float4v x;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = (count[0][i] > 0.f ? INFINITY : 0.f) + (count[1][i] > 0.f ? -INFINITY : 0.f) + (count[2][i] > 0.f ? __builtin_nanf("") : 0.f);
        return x;
    }
};
// x to four consecutive values of an output
__device__ inline void add_to_out4(void* out, int fp32, int64_t at, float4v x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (fp32) static_cast<float*>(out)[at + i] += x[i];
        else static_cast<_Float16*>(out)[at + i] = (_Float16)((float)static_cast<_Float16*>(out)[at + i] + x[i]);
    }
}

// Joins the states of two wavefronts that saw different tokens of the same rows: x of the other one.
template <int R>
__device__ inline void join_row(State<R>& st, int r, float m_x, float l_x, float fine_x, float& w_mine, float& w_x) {
    const float m_new = fmaxf(st.m[r], m_x), ref = reference_of(m_new);
    w_mine = __builtin_amdgcn_exp2f(st.m[r] - ref);
    w_x = __builtin_amdgcn_exp2f(m_x - ref);
    st.l[r] = st.l[r] * w_mine + l_x * w_x;
    st.fine[r] = st.fine[r] * w_mine + fine_x * w_x;
    st.m[r] = m_new;
}

// Bytes of LDS that join_waves needs for each of half of a workgroup's wavefronts.
#define KVQ_JOIN_BYTES (8 * 64 * 16 + 3 * 64 * 4)
// The WT wavefronts wt = 0 .. WT - 1 that share rows (the same wm) hand their states to wt = 0, halving by halving, a group of rows after
// the other.  lds: WM * WT / 2 times KVQ_JOIN_BYTES.  Every wavefront of the workgroup takes part.
template <int R, int WM, int WT>
__device__ inline void join_waves(State<R>& st, uint8_t* lds, int wm, int wt, int lane) {
#pragma unroll
    for (int half = WT / 2; half >= 1; half /= 2) {
        uint8_t* const at = lds + (wm * (WT / 2) + (wt % half)) * KVQ_JOIN_BYTES;
        float4v* const o = reinterpret_cast<float4v*>(at);
        float* const ml = reinterpret_cast<float*>(at + 8 * 64 * 16);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            __syncthreads();
            if (wt >= half && wt < 2 * half) {
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) o[nt * 64 + lane] = st.o[r][nt];
                ml[lane] = st.m[r];
                ml[64 + lane] = st.l[r];
                ml[128 + lane] = st.fine[r];
            }
            __syncthreads();
            if (wt < half) {
                float a, b;
                join_row<R>(st, r, ml[lane], ml[64 + lane], ml[128 + lane], a, b);
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) st.o[r][nt] = st.o[r][nt] * a + o[nt * 64 + lane] * b;
            }
        }
    }
}

// Partial results of one group of 16 rows and one split, 32 bits, as the lanes hold them: 8 KiB of un-normalised outputs
// [nt][lane][4] and of each of the 16 rows the reference, the sum and the sum of the unrounded probabilities.
#define KVQ_PART_O_FLOATS (8 * 64 * 4)
#define KVQ_PART_ML_FLOATS 64
#define KVQ_PART_BYTES ((KVQ_PART_O_FLOATS + KVQ_PART_ML_FLOATS) * 4)

template <int R>
__device__ inline void store_partial(const State<R>& st, int r, float* part, int lane) {
    float4v* const o = reinterpret_cast<float4v*>(part);
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) o[nt * 64 + lane] = st.o[r][nt];
    const float l = quarters_sum(st.l[r]), fine = quarters_sum(st.fine[r]);
    if (lane < 16) reinterpret_cast<float4v*>(part + KVQ_PART_O_FLOATS)[lane] = float4v{st.m[r], l, fine, 0.f};
}

// Joins n_parts (at most KVQ_MOST_PARTS) partial results of one group of 16 rows, `step` floats apart.  A workgroup of eight wavefronts
// takes 32 of the 128 channels: two blocks of 16 in four slices of the parts each, so that the loads of a thread are few and all in
// flight together; `pair` says which two blocks.  True in the wavefronts that hold the result: the lane's four channels of block nt of row n, and the
// row's statistics.  (One wavefront a block and the parts one after the other: 20 us for 36 parts.)
#define KVQ_MOST_PARTS 65
struct Joined {
    float4v o;
    float m, l, fine;
    int nt;
};
struct JoinLds {
    float w[KVQ_MOST_PARTS][16];  // references
    float l[KVQ_MOST_PARTS][16], fine[KVQ_MOST_PARTS][16];
    float4v o[6][64];
};
__device__ inline bool join_partials(JoinLds& lds, const float* part, int64_t step, int n_parts, int pair, Joined& x) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15;
    const int slice = wave >> 1;
    x.nt = 2 * pair + (wave & 1);
    for (int i = tid; i < n_parts * 16; i += 512) {
        const float4v at = reinterpret_cast<const float4v*>(part + (i >> 4) * step + KVQ_PART_O_FLOATS)[i & 15];
        lds.w[i >> 4][i & 15] = at[0];
        lds.l[i >> 4][i & 15] = at[1];
        lds.fine[i >> 4][i & 15] = at[2];
    }
    // the slice's first eight parts are on their way meanwhile
    float4v o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int s = min(slice + 4 * k, n_parts - 1);
        o[k] = *reinterpret_cast<const float4v*>(part + s * step + (x.nt * 64 + lane) * 4);
    }
    __syncthreads();
    x.m = -INFINITY;
    for (int s = 0; s < n_parts; ++s) x.m = fmaxf(x.m, lds.w[s][n]);
    const float ref = reference_of(x.m);
    // (never zero: an infinity among the values that a row sees stays one, whatever its range weighs; of finite sums 2^-126 leaves nothing)
    const auto weight = [&](int s) { return fmaxf(__builtin_amdgcn_exp2f(lds.w[s][n] - ref), 0x1p-126f); };
    x.o = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int s = slice + 4 * k;
        if (s < n_parts) x.o += o[k] * weight(s);
    }
    for (int s = slice + 32; s < n_parts; s += 4)
        x.o += *reinterpret_cast<const float4v*>(part + s * step + (x.nt * 64 + lane) * 4) * weight(s);
    if (slice) lds.o[wave - 2][lane] = x.o;
    __syncthreads();
    if (slice) return false;
#pragma unroll
    for (int k = 0; k < 3; ++k) x.o += lds.o[2 * k + wave][lane];
    x.l = x.fine = 0.f;
    for (int s = 0; s < n_parts; ++s) {
        const float w = __builtin_amdgcn_exp2f(lds.w[s][n] - ref);
        x.l += lds.l[s][n] * w;
        x.fine += lds.fine[s][n] * w;
    }
    return true;
}

// What the sum of a row's weights divides by: a row that saw nothing gives zeros.
__device__ inline float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }

// Four channels of an output row.
__device__ inline void store_out4(void* row, int fp32, int channel, float4v x) {
    if (fp32) {
        *reinterpret_cast<float4v*>(static_cast<float*>(row) + channel) = x;
    } else {
        const u32x2 h = {pack2(x[0], x[1]), pack2(x[2], x[3])};
        *reinterpret_cast<u32x2*>(static_cast<_Float16*>(row) + channel) = h;
    }
}

}  // namespace kvq_flash

#endif
