// Kernel of attention over whole prompts (etf_prompt_attend).  Included by etf_prompt.hip, inside its anonymous namespace.
#pragma once

#include "etf_kv_types.hip.h"

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t qs[2], ks[2], vs[2];  // strides of token, head
    Packed seq;
    uint16_t *out;
    float *lse;
    float *part_o, *part_ml;  // partial results of ranges: [tile][head][range][128][D], [tile][head][range][128][2]
    float scale2;  // softmax scale times log2 e, finite
    int heads, g;
    int ranges, per;  // most ranges of a tile's blocks, and blocks of one
};

// ------------------------------------------------------------------------------------------------
// Attention of prompts in 16 bits.  Rows are pairs (token, query head of the group) of one sequence and key/value head, 128 to
// a workgroup, 32 to a wave.  s^T = K q^T and o^T = V^T p^T on v_mfma_f32_32x32x16: a lane's column is a row, so the running
// maximum and sum are the lane's own (and its neighbour's 32 lanes up), and p^T stands in its registers as the second product wants
// it: of 16 tokens, those 8 (j / 4) + 4 (lane / 32) + j % 4.  Blocks of 64 tokens go straight from memory to LDS, the next one while this
// one is worked on; values are read transposed (ds_read_b64_tr_b16: 16 lanes exchange 4 x 4 numbers).  Pieces of 16 bytes are
// exchanged within a row of LDS, so that lanes that read together hit all banks (no conflicts are counted).  A weight is rounded to the rows' type
// for its product, as in k_kv_attend; its sum takes it unrounded.
// Bound by the clock, which falls to 1.9 GHz of 2.4 under it, and by phases that wait for each other: the matrix cores are busy 52 % of the time and vector issue 50 % (128
// dimensions; 64: 49 % and 79 %, the exponentials).  Two prompts of 4096 tokens, 32 heads of 128 dimensions: 279 to 293 us = 940 to 985 TFLOP/s, where a matrix product
// of 8192^3 reaches 1230.  One prompt of 8192, 64 dimensions: 298 to 318 us = 865 to 920 TFLOP/s; 34 356 tokens in 24 prompts of 1 to 2500, five query heads of 96
// dimensions to each: 305 to 315 us = 750 to 775 TFLOP/s.  Tried for the first of these, 289 us at that time: the next block's first product and the block before's second one between the
// exponentials 484 (registers: one wave to a unit); 64 rows a wave 403 (likewise); eight waves of which four multiply while four take exponentials 304 to 366;
// loads into LDS spread between the products 298 to 312; values transposed on their way into LDS and read 16 bytes at a time 311; wave priorities 300 to 310;
// maxima only where a sum of weights asks for them 854 (registers); half of a wave's last block left out where it sees no more than the other, 293 -> 311, and 314 -> 353 for
// the 24 prompts (registers: 162 -> 197 with 96 dimensions).
// ------------------------------------------------------------------------------------------------
// 16 bytes to a lane from offset `at` of the `bytes` bytes at `from` (nothing is read behind them) to the 1 KB of LDS at `to`, in the
// order of the lanes.  `from`, `bytes` and `to` are the same for all lanes.
__device__ __forceinline__ void buffer_to_lds(const void *from, int bytes, uint32_t at, void *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void *)from, 0, bytes, 0x00020000), (__attribute__((address_space(3))) void *)to, 16, at, 0, 0, 0);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int D>
struct PromptTile {
    static constexpr int PT = D / 8;  // pieces of a row
    // place in its row of LDS of piece `at` of a token's keys, values; BACK: the piece that stands at place `at`
    template <bool BACK>
    static __device__ __forceinline__ int k_place(int token, int at)
    {
        if constexpr (D == 96) return (at + (BACK ? 12 - (token >> 2 & 7) : token >> 2 & 7)) % 12;
        return at ^ (D == 128 ? token & 15 : token >> 1 & 7);
    }
    static __device__ __forceinline__ int v_place(int token, int at) { return at ^ (D == 128 ? (token & 3) << 2 : D == 64 ? (token >> 1 & 1) << 2 : 0); }
};

// Rows whose sums of weighted values float32 does not hold have weights smaller by 2^prompt_down: a weight is 2^(TILE_UP + TILE_LAG) at most, so that
// sums of as many as a row sees are no larger than its largest value.  Such a row's dimensions lose what is smaller than float32's smallest
// normal number times that.
template <typename T>
__device__ __forceinline__ int prompt_down(int sees) { return T::TILE_UP + T::TILE_LAG + 32 - __builtin_clz(sees); }

// o times f = 1 / l.  What rounded weights put past the type's largest number becomes that one.
template <typename T>
__device__ __forceinline__ float held_mean(float o, float f)
{
    const float x = o * f;
    return fabsf(x) > T::MOST && fabsf(o) < INFINITY ? copysignf(T::MOST, x) : x;
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void k_prompt(PromptArgs a)
{
    using Tile = PromptTile<D>;
    constexpr int ROWS = 128, PT = Tile::PT, LOADS = PT / 4, DT = D / 32, ST = D / 16;
    __shared__ __attribute__((aligned(1024))) uint8_t s_k0[KB * D * 2], s_v0[KB * D * 2], s_k1[KB * D * 2], s_v1[KB * D * 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), x = lane & 31, half = lane >> 5;
    const int H = a.heads, g = a.g;
    // A prompt's last tiles, the longest ones, first; where all workgroups run at once, two to a compute unit (of 64 and 96 dimensions it holds three; the
    // limit is that of 128, with which it was measured), the second ones from the other end, so that
    // a long tile has a short one beside it (two prompts of 950 tokens, 8 heads, four query heads to each: 32 us instead of 36; one of 2000: 50 instead of 51).
    // Cutting a tile's blocks between two groups of waves of a larger workgroup as well: 25 us instead of 27 for 1000 tokens, nothing for 600 and
    // 1500; left out, since a row's sums would then depend on the call that it is in.
    const int h = blockIdx.x % H, range = blockIdx.x / H % a.ranges, unit = blockIdx.x / (H * a.ranges), units = gridDim.x / (H * a.ranges), paired = 256 / H;
    const int number = gridDim.x <= 512 && a.ranges == 1 && unit >= paired ? unit - paired : units - 1 - unit;
    const int b = packed_of_tile<ROWS>(a.seq, g, number);
    const int begin = __builtin_amdgcn_readfirstlane(packed_start(a.seq, b)), n = __builtin_amdgcn_readfirstlane(packed_start(a.seq, b + 1)) - begin;
    const int tile = number - __builtin_amdgcn_readfirstlane(packed_base<ROWS>(a.seq, b, g));
    if (n <= 0 || tile < 0 || (int64_t)tile * ROWS >= (int64_t)n * g) return;
    const int64_t rows = (int64_t)n * g, row0 = (int64_t)tile * ROWS, row = row0 + 32 * wave + x;
    const bool valid = row < rows;
    const int qi = (int)(min(row, rows - 1) / g), hg = valid ? (int)(row % g) : 0;
    const int sees = qi + 1;
    const int wleast = __builtin_amdgcn_readfirstlane(sees), wmost = __builtin_amdgcn_readfirstlane((int)(min(row0 + 32 * wave + 31, rows - 1) / g) + 1);
    const bool wlive = row0 + 32 * wave < rows;
    const int most = (int)(min(row0 + ROWS - 1, rows - 1) / g) + 1, all = (most + KB - 1) / KB;
    const bool alone = all <= a.per;  // one range
    const int from = alone ? 0 : range * a.per, blocks = min(from + a.per, all);
    if (range > 0 && (alone || from >= all)) return;

    typename T::x8 q[ST];
    const uint16_t *qp = a.q + (begin + qi) * a.qs[0] + ((int64_t)h * g + hg) * a.qs[1];
#pragma unroll
    for (int i = 0; i < ST; ++i) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (valid) w = *reinterpret_cast<const uint4 *>(qp + 16 * i + 8 * half);
        q[i] = query8<T>(__builtin_bit_cast(typename T::x8, w));
    }

    // where this lane's pieces of a block come from, in bytes from the block's first key or value
    uint32_t k_from[LOADS], v_from[LOADS];
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
        const int p = (wave * LOADS + l) * 64 + lane, t = p / PT, at = p % PT;
        k_from[l] = t * (uint32_t)a.ks[0] * 2 + Tile::template k_place<true>(t, at) * 16;
        v_from[l] = t * (uint32_t)a.vs[0] * 2 + Tile::v_place(t, at) * 16;
    }
    const uint16_t *kp = a.k + begin * a.ks[0] + h * a.ks[1], *vp = a.v + begin * a.vs[0] + h * a.vs[1];
    auto load = [&](int j, uint8_t *to_k, uint8_t *to_v) __attribute__((always_inline)) {
        const int last = min(KB, n - j * KB) - 1;  // rows behind the sequence's end are out of the buffers' range
        const void *fk = kp + (int64_t)j * KB * a.ks[0], *fv = vp + (int64_t)j * KB * a.vs[0];
        const int nk = last * (int)a.ks[0] * 2 + D * 2, nv = last * (int)a.vs[0] * 2 + D * 2;
#pragma unroll
        for (int l = 0; l < LOADS; ++l) buffer_to_lds(fk, nk, k_from[l], to_k + (wave * LOADS + l) * 1024);
#pragma unroll
        for (int l = 0; l < LOADS; ++l) buffer_to_lds(fv, nv, v_from[l], to_v + (wave * LOADS + l) * 1024);
    };

    f32x16 o[DT];
    float m, l;
    int down = 0;
    const int l16 = lane & 15, quad = l16 >> 2;
    const int v_at = (4 * half + quad) * D * 2 + (lane >> 4 & 1) * 32 + (l16 & 3) * 8;  // of the dimensions from 0 on, before exchange
    // four tokens from 16 u + 8 c + 4 half on of dimension 32 i + x
    auto value4 = [&](const uint8_t *s_v, int u, int c, int i) __attribute__((always_inline)) {
        const int seg = D == 128 ? i ^ quad : D == 64 ? i ^ (quad >> 1) : i;
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(s_v + v_at + seg * 64 + (16 * u + 8 * c) * D * 2));
    };
    auto value8 = [&](const uint8_t *s_v, int u, int i) __attribute__((always_inline)) {
        const s16x4 v0 = value4(s_v, u, 0, i), v1 = value4(s_v, u, 1, i);
        return (u32x4){__builtin_bit_cast(uint2, v0).x, __builtin_bit_cast(uint2, v0).y, __builtin_bit_cast(uint2, v1).x, __builtin_bit_cast(uint2, v1).y};
    };

    auto block = [&](auto careful, int j, const uint8_t *s_k, const uint8_t *s_v) __attribute__((always_inline)) {
        f32x16 s[2];
        s[0] = s[1] = (f32x16)(0.f);
#pragma unroll
        for (int i = 0; i < ST; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int at = (32 * t + x) * D * 2 + Tile::template k_place<false>(x, 2 * i + half) * 16;
                s[t] = T::mfma(*reinterpret_cast<const typename T::x8 *>(s_k + at), q[i], s[t]);
            }
        float scale = a.scale2;
        if (j * KB + KB > wleast) {
            asm volatile("");  // a branch: few blocks need the comparisons
            const int left = sees - j * KB - 4 * half;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * t + 8 * (i / 4) + i % 4 >= left) s[t][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);  // and what the lane 32 up or down has
        top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * scale;
        // z is s * scale less the reference with one rounding, as long as what rounding the largest z has left out matters no more than the others'
        // roundings; from there on, with one more, no z is above the largest: exponentials stay within the type.  Here and below a row goes by
        // its own numbers alone, so that its result does not depend on the rows beside it.
        const bool far = fabsf(top) > 0x1p20f;
        if (__any(far)) {
            asm volatile("");  // a branch: few blocks need it
            const float now = far ? scale : 1.f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] *= now;
            scale = far ? 1.f : scale;
        }
        top = reference<T::TILE_UP>(top);
        // the reference in use may lag behind by a factor of 2^TILE_LAG in the weights, which changes nothing but spares the scaling
        const bool more = top - m > T::TILE_LAG;
        if (__any(more)) {
            const float fade = more ? __builtin_amdgcn_exp2f(m - top) : 1.f;
            m = more ? top : m;
            l *= fade;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[i] *= fade;
        }
        const float base = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], scale, -base));
                if constexpr (T::WIDE && decltype(careful)::value) s[t][i] = __builtin_amdgcn_ldexpf(s[t][i], -down);
                sum += s[t][i];
            }
        l += sum;
        typename T::x8 p[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const f32x16 &w = s[u / 2];
            const int at = 8 * (u % 2);
            const typename T::x2 p0 = T::narrow(w[at], w[at + 1]), p1 = T::narrow(w[at + 2], w[at + 3]);
            const typename T::x2 p2 = T::narrow(w[at + 4], w[at + 5]), p3 = T::narrow(w[at + 6], w[at + 7]);
            p[u] = (typename T::x8){p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
        }
        if constexpr (!decltype(careful)::value) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < DT; ++i) o[i] = T::mfma(__builtin_bit_cast(typename T::x8, value8(s_v, u, i)), p[u], o[i]);
        } else {
            // values that are not finite go to the rows that see them, and to no other: zeros in the product, then added
            uint32_t some = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    u32x4 w = value8(s_v, u, i);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t lo = (w[y] & T::EXP) == T::EXP ? 0xFFFFu : 0u, hi = (w[y] >> 16 & T::EXP) == T::EXP ? 0xFFFF0000u : 0u;
                        some |= lo | hi;
                        w[y] &= ~(lo | hi);
                    }
                    o[i] = T::mfma(__builtin_bit_cast(typename T::x8, w), p[u], o[i]);
                }
            if (!__any(some != 0)) return;
#pragma unroll 1
            for (int t = 0; t < min(KB, n - j * KB); ++t) {
                const bool see = j * KB + t < sees;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int y = 0; y < 16; ++y) {
                        const int d = 32 * i + 8 * (y / 4) + 4 * half + y % 4;
                        const uint16_t u = *reinterpret_cast<const uint16_t *>(s_v + t * D * 2 + Tile::v_place(t, d / 8) * 16 + d % 8 * 2);
                        o[i][y] += see && (u & T::EXP) == T::EXP ? T::wide(u) : 0.f;
                    }
            }
        }
    };

    auto clear = [&]() __attribute__((always_inline)) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = (f32x16)(0.f);
    };
    // the wave's loads into LDS have arrived: the compiler does not wait for them at a barrier
    auto arrived = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
    clear();
    load(from, s_k0, s_v0);
    for (int j = from; j < blocks; j += 2) {
        arrived();
        __syncthreads();  // this block is there, and everyone is done with the one before it
        if (j + 1 < blocks) load(j + 1, s_k1, s_v1);
        if (wlive && j * KB < wmost) block(std::false_type(), j, s_k0, s_v0);
        if (j + 1 >= blocks) break;
        arrived();
        __syncthreads();
        if (j + 2 < blocks) load(j + 2, s_k0, s_v0);
        if (wlive && (j + 1) * KB < wmost) block(std::false_type(), j + 1, s_k1, s_v1);
    }
    // A value that is not finite makes whole tiles so, whether or not their rows see it, through products with weights of 0: such
    // tiles are worked out again.  Rows that are not finite then have such values themselves or sums that float32 does not hold: they
    // are worked out once more, with smaller weights.
    auto not_finite = [&]() __attribute__((always_inline)) {
        float zero = 0.f * l;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int y = 0; y < 16; ++y) zero = __builtin_fmaf(0.f, o[i][y], zero);
        return zero != 0.f;
    };
    auto once_more = [&]() __attribute__((always_inline)) {
        clear();
        for (int j = from; j < blocks; ++j) {
            load(j, s_k0, s_v0);
            arrived();
            __syncthreads();
            if (wlive && j * KB < wmost) block(std::true_type(), j, s_k0, s_v0);
            __syncthreads();
        }
    };
    if (__syncthreads_or(valid && not_finite())) {
        once_more();
        if constexpr (T::WIDE) {
            int more = not_finite();
            more |= __shfl_xor(more, 32);
            if (more) down = prompt_down<T>(sees);
            if (__syncthreads_or(valid && more)) once_more();
            if (more) l = -l;  // tells that weights are smaller
        }
    }
    // the compiler keeps what follows apart for rows that come from here and from there, at 40 registers and more, unless something hides where they come from
    if (T::WIDE) asm volatile("" : "+v"(l));
    l += __shfl_xor(l, 32);
    if (!valid) return;

    const int64_t at = (int64_t)(begin + qi) * H * g + h * g + hg;
    if (alone) {
        float f = 1.f / fabsf(l);
        T::hold(f);
        uint16_t *to = a.out + at * D + 4 * half;
        auto store = [&](auto mean) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const typename T::x2 p0 = T::narrow(mean(o[i][4 * y]), mean(o[i][4 * y + 1])), p1 = T::narrow(mean(o[i][4 * y + 2]), mean(o[i][4 * y + 3]));
                    *reinterpret_cast<uint2 *>(to + 32 * i + 8 * y) = make_uint2(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1));
                }
        };
        if (T::WIDE && __any(l < 0.f)) {
            store([&](float x) { return held_mean<T>(x, f); });
            if (l < 0.f) l = __builtin_amdgcn_ldexpf(-l, prompt_down<T>(sees));
        } else {
            store([&](float x) { return x * f; });
        }
        if (half == 0 && a.lse) a.lse[at] = (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
        return;
    }
    const int64_t part = (((int64_t)number * H + h) * a.ranges + range) * ROWS + row - row0;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int y = 0; y < 4; ++y)
            *reinterpret_cast<f32x4 *>(a.part_o + part * D + 32 * i + 8 * y + 4 * half) = (f32x4){o[i][4 * y], o[i][4 * y + 1], o[i][4 * y + 2], o[i][4 * y + 3]};
    if (half == 0) *reinterpret_cast<float2 *>(a.part_ml + part * 2) = make_float2(m, l);
}

// Joins the ranges of tiles that have several: 32 lanes to a row, eight rows to a workgroup.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_prompt_join(PromptArgs a)
{
    constexpr int ROWS = 128, PARTS = ROWS / 8;
    const int H = a.heads, g = a.g, lane = threadIdx.x & 31, y = blockIdx.x % PARTS * 8 + threadIdx.x / 32;
    const int h = blockIdx.x / PARTS % H, number = blockIdx.x / (PARTS * H);
    const int b = packed_of_tile<ROWS>(a.seq, g, number), tile = number - packed_base<ROWS>(a.seq, b, g);
    const int begin = packed_start(a.seq, b), n = packed_start(a.seq, b + 1) - begin;
    const int64_t rows = (int64_t)max(0, n) * g, row = (int64_t)tile * ROWS + y;
    if (tile < 0 || row >= rows) return;
    const int most = (int)(min((int64_t)(tile + 1) * ROWS - 1, rows - 1) / g) + 1, all = (most + KB - 1) / KB;
    if (all <= a.per) return;
    const int many = (all + a.per - 1) / a.per;
    const int64_t first = ((int64_t)number * H + h) * a.ranges * ROWS + y;
    float m = -INFINITY, l = 0.f;
    for (int s = 0; s < many; ++s) m = fmaxf(m, a.part_ml[(first + s * ROWS) * 2]);
    const float base = m == -INFINITY ? 0.f : m;
    const float down = ldexpf(1.f, -prompt_down<T>((int)(row / g) + 1));
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    // `of`: the sums are of weights that are smaller by it
    auto add = [&](float of) __attribute__((always_inline)) {
        o = (f32x4){0.f, 0.f, 0.f, 0.f};
        l = 0.f;
        for (int s = 0; s < many; ++s) {
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + (first + s * ROWS) * 2);
            float weight = __builtin_amdgcn_exp2f(ml.x - base);
            if constexpr (T::WIDE) weight *= __builtin_signbit(ml.y) ? of / down : of;
            l += fabsf(ml.y) * weight;
            if (lane < D / 4) o += *reinterpret_cast<const f32x4 *>(a.part_o + (first + s * ROWS) * D + 4 * lane) * weight;
        }
    };
    add(1.f);
    const float lse = (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
    bool wide = false;
    if constexpr (T::WIDE) {
        wide = 0.f * o[0] + 0.f * o[1] + 0.f * o[2] + 0.f * o[3] != 0.f;
        if (wide) add(down);
    }
    float f = 1.f / l;
    T::hold(f);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = T::WIDE && wide ? held_mean<T>(o[i], f) : o[i] * f;
    const int64_t at = (int64_t)(begin + (int)(row / g)) * H * g + h * g + row % g;
    const typename T::x2 p0 = T::narrow(o[0], o[1]), p1 = T::narrow(o[2], o[3]);
    if (lane < D / 4) *reinterpret_cast<uint2 *>(a.out + at * D + 4 * lane) = make_uint2(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1));
    if (lane == 0 && a.lse) a.lse[at] = lse;
}
