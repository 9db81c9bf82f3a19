// Kernels of the attention cache in 8 bits (etf_kv_*): what fills it, what reads it, what picks blocks of it and what
// thins it out.  Included by etf_kv.hip, inside its anonymous namespace.
#pragma once

constexpr int KB = 64;  // tokens of a block

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// The 16-bit type of queries, outputs and open blocks.  Codes become operands of the matrix cores exactly: four bits of
// significand fit either type.  Keys are multiplied unscaled (their scale goes into the logits, in float32), values are
// multiplied by a power of two on the way (`bring`).
struct TBf {
    typedef bf16x2 x2;
    typedef bf16x8 x8;
    static constexpr uint32_t EXP = 0x7F80u;  // exponent bits: all ones where a number is not finite
    static constexpr uint16_t NOT = 0x7FC0u;
    static __device__ __forceinline__ x2 bring(uint32_t w, float scale, bool high)
    {
        return high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    }
    static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float wide(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
    static __device__ __forceinline__ x2 narrow(float a, float b) { return __builtin_convertvector((f32x2){a, b}, x2); }
    static constexpr bool NARROW = false;
    static constexpr int UP = 0, TILE_UP = 0, TILE_LAG = 8;
};
struct THf {
    typedef f16x2 x2;
    typedef f16x8 x8;
    static constexpr uint32_t EXP = 0x7C00u;
    static constexpr uint16_t NOT = 0x7E00u;
    static __device__ __forceinline__ x2 bring(uint32_t w, float scale, bool high)
    {
        return high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false);
    }
    static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float wide(uint16_t u) { return (float)__builtin_bit_cast(_Float16, u); }
    static __device__ __forceinline__ x2 narrow(float a, float b) { return __builtin_convertvector((f32x2){a, b}, x2); }
    // A value near the type's largest may round up past it in 8 bits, 65504 to 256 codes of 256 = 65536: where values have that scale, half
    // of it goes to the weights.  A code times any smaller scale is a number of the type: a multiple of its smallest, like the
    // values that it was rounded from.
    static constexpr bool NARROW = true;
    // Softmax weights are taken 2^UP times as large (2^TILE_UP and up to 2^TILE_LAG more in k_kv_tile), the sums of them too: next to a
    // weight of 1 those below 2^-14 would lose bits and those below 2^-25 be gone, of which a long cache can have many.  So a weight is off
    // by 2^-39 of the largest at most (2^-31), besides its rounding.  2^10 and 2^4 in k_kv_tile: 135.7 instead of 134.7 us for pieces of
    // three prompts of up to 1000 tokens over caches of up to 10 001, 96 dimensions.
    static constexpr int UP = 14, TILE_UP = 6, TILE_LAG = 8;
};

// What weights 2^(z - reference) are taken against where `top` is the largest z: `up` bits below it.  Where float32 does not resolve
// that, none: a weight above 2^up could pass the type's largest.
template <int UP>
__device__ __forceinline__ float reference(float top)
{
    if (UP == 0) return top;
    const float ref = top - UP;
    return top - ref > UP ? top : ref;
}

// eight codes (two words) as an operand
template <typename T>
__device__ __forceinline__ typename T::x8 bring8(uint32_t w0, uint32_t w1, float scale)
{
    const typename T::x2 a = T::bring(w0, scale, false), b = T::bring(w0, scale, true), c = T::bring(w1, scale, false), d = T::bring(w1, scale, true);
    return (typename T::x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

struct KvView {
    uint8_t *k, *v, *bounds;
    float *scales;
    uint16_t *tail_k, *tail_v;
    const int32_t *table, *lens, *evicted;
    int32_t batch, heads, blocks, pages;
};

// tokens of sequence b, within what the table has room for
__device__ __forceinline__ int kv_len(const KvView &c, int b) { return min(max(c.lens[b], 0), c.blocks * KB + KB - 1); }
__device__ __forceinline__ int kv_count(const int32_t *counts, int b, int n) { return counts ? min(max(counts[b], 0), n) : n; }
// page of block j, or -1: none, or no page of the pool
__device__ __forceinline__ int kv_page(const KvView &c, int64_t bh, int j)
{
    if (j < 0 || j >= c.blocks) return -1;
    const int p = c.table[bh * c.blocks + j];
    return p >= 0 && p < c.pages ? p : -1;
}
// buffer of the open block, number j
__device__ __forceinline__ int64_t kv_tail(const KvView &c, int64_t bh, int b, int j, int D)
{
    return (bh * 2 + ((j + c.evicted[b]) & 1)) * (int64_t)(KB * D);
}

// ------------------------------------------------------------------------------------------------
// Append.  A workgroup takes one block of one (sequence, head): where the new tokens complete it, it is sealed: the
// smallest power of two s with amax <= 448 s, codes round_e4m3(x / s) (the division is exact), the values transposed
// through LDS so that a row of a page is one dimension's 64 tokens, and every dimension's smallest and largest key code.
// The workgroup of the first block reads the open block's earlier tokens; it also writes what is left over into the open
// block, afterwards, because both may be the same buffer.  A token that is not finite has keys that are not numbers
// and values of zero: rows that see it become not a number, others do not.
// Bound by vector issue and memory alike: four prompts of 8192 tokens, 8 heads of 128 dimensions (202 MB) 48 us = 4.2 TB/s; with maxima and
// bounds number by number instead of two to an operation 53 us.
// ------------------------------------------------------------------------------------------------
struct KvAppendArgs {
    KvView c;
    const uint16_t *k, *v;
    int64_t ks[3], vs[3];  // strides of sequence, token, head
    const int32_t *counts;
    int n, per;  // per: workgroups of a (sequence, head), the most blocks that n tokens can complete
};

// Largest size of eight numbers, as the bits without the sign, which are in the order of the sizes; from T::EXP on: one of them is not finite
__device__ __forceinline__ uint32_t size8(const uint4 &w)
{
    constexpr uint32_t mask = 0x7FFF7FFFu;
    const u16x2 a = __builtin_bit_cast(u16x2, w.x & mask), b = __builtin_bit_cast(u16x2, w.y & mask);
    const u16x2 c = __builtin_bit_cast(u16x2, w.z & mask), d = __builtin_bit_cast(u16x2, w.w & mask);
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(a, b), __builtin_elementwise_max(c, d));
    return max((uint32_t)m[0], (uint32_t)m[1]);
}

// A piece of a query: one that is not finite is made NaN, so that its row becomes not a number even where all products would be -inf
template <typename T>
__device__ __forceinline__ typename T::x8 query8(typename T::x8 q)
{
    uint4 w = __builtin_bit_cast(uint4, q);
    if (size8(w) >= T::EXP) w.x = T::NOT | (uint32_t)T::NOT << 16;
    return __builtin_bit_cast(typename T::x8, w);
}

// Codes in the order of their values, two to a word: 16-bit numbers whose low byte is the code, its lower bits turned where it is
// negative (so that -0 stands below +0).  Its own inverse.
__device__ __forceinline__ i16x2 code_order(i16x2 code) { return code ^ ((code >> 15) & (int16_t)0x7F); }

// eight values times `inverse`, a power of two, as codes
template <typename T>
__device__ __forceinline__ uint2 codes8(const uint4 &w, float inverse)
{
    uint32_t o[2];
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    for (int i = 0; i < 2; ++i) {
        float f[4];
        // beyond 448 only where the scale is the largest: the code of the largest value then
        for (int j = 0; j < 4; ++j) f[j] = __builtin_amdgcn_fmed3f(T::wide((uint16_t)(in[2 * i + j / 2] >> (16 * (j & 1)))) * inverse, -448.f, 448.f);
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
        o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
    }
    return make_uint2(o[0], o[1]);
}

// exponent of the smallest power of two s with amax <= 448 s, within what a float's normal numbers hold
__device__ __forceinline__ int scale_exponent(float amax)
{
    if (!(amax > 0.f)) return 0;
    int e;
    const float m = frexpf(amax, &e);  // amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    return min(max(e - (m <= 0.875f ? 9 : 8), -126), 119);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void k_kv_append(KvAppendArgs a)
{
    constexpr int PT = D / 8;                // 16-byte pieces of a token
    constexpr int NP = KB * PT / 256;        // pieces of a thread
    static_assert(KB * PT % 256 == 0, "pieces divide among the threads");
    constexpr int VROW = KB + 4;             // LDS row of one dimension's value codes, padded
    __shared__ __attribute__((aligned(16))) uint8_t s_v[D * VROW];
    __shared__ __attribute__((aligned(16))) uint8_t s_k[KB * D];
    __shared__ uint32_t s_amax[2][4];
    __shared__ int s_bad[KB];
    constexpr int BW = D / 4, BG = 256 / BW, BT = (KB + BG - 1) / BG;  // bounds: words of a row, groups of tokens, tokens of a group
    __shared__ __attribute__((aligned(8))) int16_t s_edge[2][BG][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t bh = blockIdx.x / a.per;
    const int h = (int)(bh % a.c.heads), b = (int)(bh / a.c.heads), blk = blockIdx.x % a.per;
    const int len = kv_len(a.c, b), count = min(kv_count(a.counts, b, a.n), a.c.blocks * KB + KB - 1 - len);  // as many as lens can count
    const int first = len / KB, begin = len % KB;
    const int full = (begin + count) / KB, left = (begin + count) % KB;
    if (blk > 0 && blk >= full) return;
    const uint16_t *nk = a.k + b * a.ks[0] + h * a.ks[2], *nv = a.v + b * a.vs[0] + h * a.vs[2];
    if (tid < KB) s_bad[tid] = 0;
    __syncthreads();
    if (blk < full) {
        const int64_t old = kv_tail(a.c, bh, b, first, D);
        uint4 kw[NP], vw[NP];
        uint32_t ks[NP], vs[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int p = tid + 256 * i, t = p / PT, d = p % PT * 8;
            const int at = blk * KB + t - begin;  // among the new tokens
            if (at >= 0) {
                kw[i] = *reinterpret_cast<const uint4 *>(nk + at * a.ks[1] + d);
                vw[i] = *reinterpret_cast<const uint4 *>(nv + at * a.vs[1] + d);
            } else {
                kw[i] = *reinterpret_cast<const uint4 *>(a.c.tail_k + old + t * D + d);
                uint16_t x[8];
                for (int j = 0; j < 8; ++j) x[j] = a.c.tail_v[old + (d + j) * KB + t];
                vw[i] = make_uint4(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16, x[4] | (uint32_t)x[5] << 16, x[6] | (uint32_t)x[7] << 16);
            }
            ks[i] = size8(kw[i]);
            vs[i] = size8(vw[i]);
            if (max(ks[i], vs[i]) >= T::EXP) s_bad[t] = 1;
        }
        __syncthreads();
        uint32_t mk = 0, mv = 0;
        bool bad[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            bad[i] = s_bad[(tid + 256 * i) / PT] != 0;
            if (!bad[i]) {
                mk = max(mk, ks[i]);
                mv = max(mv, vs[i]);
            }
        }
        for (int o = 32; o; o >>= 1) {
            mk = max(mk, (uint32_t)__shfl_xor((int)mk, o));
            mv = max(mv, (uint32_t)__shfl_xor((int)mv, o));
        }
        if (lane == 0) {
            s_amax[0][wave] = mk;
            s_amax[1][wave] = mv;
        }
        __syncthreads();
        const int ek = scale_exponent(T::wide((uint16_t)max(max(s_amax[0][0], s_amax[0][1]), max(s_amax[0][2], s_amax[0][3]))));
        const int ev = scale_exponent(T::wide((uint16_t)max(max(s_amax[1][0], s_amax[1][1]), max(s_amax[1][2], s_amax[1][3]))));
        const float ik = ldexpf(1.f, -ek), iv = ldexpf(1.f, -ev);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int p = tid + 256 * i, t = p / PT, d = p % PT * 8;
            uint2 ck = codes8<T>(kw[i], ik), cv = codes8<T>(vw[i], iv);
            if (bad[i]) {
                ck = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
                cv = make_uint2(0, 0);
            }
            *reinterpret_cast<uint2 *>(s_k + t * D + d) = ck;
            for (int j = 0; j < 8; ++j) s_v[(d + j) * VROW + t] = (uint8_t)((j < 4 ? cv.x : cv.y) >> (8 * (j & 3)));
        }
        __syncthreads();
        const int page = kv_page(a.c, bh, first + blk);
        if (page >= 0) {
            for (int p = tid; p < KB * D / 16; p += 256) {
                reinterpret_cast<uint4 *>(a.c.k + (int64_t)page * (KB * D))[p] = reinterpret_cast<const uint4 *>(s_k)[p];
                const uint32_t *r = reinterpret_cast<const uint32_t *>(s_v + p / 4 * VROW + p % 4 * 16);
                reinterpret_cast<uint4 *>(a.c.v + (int64_t)page * (KB * D))[p] = make_uint4(r[0], r[1], r[2], r[3]);
            }
            // smallest and largest codes: four dimensions and a group of tokens to a thread, then the groups
            if (tid < BW * BG) {
                const int w = tid % BW, grp = tid / BW;
                i16x2 lo[2], hi[2];  // of bytes 0 and 2, of bytes 1 and 3
                lo[0] = lo[1] = 0x7F;
                hi[0] = hi[1] = -0x80;
                for (int t = grp * BT; t < min(KB, (grp + 1) * BT); ++t) {
                    if (s_bad[t]) continue;
                    const i16x2 u = *reinterpret_cast<const i16x2 *>(s_k + t * D + 4 * w);
                    const i16x2 even = code_order((i16x2)(u << 8) >> 8), odd = code_order(u >> 8);
                    lo[0] = __builtin_elementwise_min(lo[0], even);
                    lo[1] = __builtin_elementwise_min(lo[1], odd);
                    hi[0] = __builtin_elementwise_max(hi[0], even);
                    hi[1] = __builtin_elementwise_max(hi[1], odd);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s_edge[0][grp][4 * w + i] = lo[i & 1][i >> 1];
                    s_edge[1][grp][4 * w + i] = hi[i & 1][i >> 1];
                }
            }
            if (tid < 2) a.c.scales[(int64_t)page * 2 + tid] = ldexpf(1.f, tid ? ev : ek);
        }
        __syncthreads();
        if (page >= 0 && tid < 2 * BW) {
            const int e = tid / BW, d = tid % BW * 4;
            uint32_t out = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int lo = 0x7F, hi = -0x80;
                for (int y = 0; y < BG; ++y) {
                    lo = min(lo, (int)s_edge[0][y][d + i]);
                    hi = max(hi, (int)s_edge[1][y][d + i]);
                }
                const i16x2 o = {(int16_t)(lo > hi ? 0 : e ? hi : lo), 0};
                const uint32_t code = (uint32_t)(uint16_t)code_order(o)[0] & 0xFF;
                out |= (code == 0x80 ? 0 : code) << (8 * i);  // no -0
            }
            *reinterpret_cast<uint32_t *>(a.c.bounds + ((int64_t)page * 2 + e) * D + d) = out;
        }
    }
    if (blk > 0) return;
    // what is left over: tokens [from, left) of the open block
    const int from = full ? 0 : begin;
    const int64_t now = kv_tail(a.c, bh, b, first + full, D);
    if (tid < KB) s_bad[tid] = 0;
    __syncthreads();
    const int np = (left - from) * PT;
    for (int pass = 0; pass < 2; ++pass) {
        for (int p = tid; p < np; p += 256) {
            const int t = from + p / PT, d = p % PT * 8;
            const int at = full * KB + t - begin;
            uint4 kw = *reinterpret_cast<const uint4 *>(nk + at * a.ks[1] + d), vw = *reinterpret_cast<const uint4 *>(nv + at * a.vs[1] + d);
            if (pass == 0) {
                if (max(size8(kw), size8(vw)) >= T::EXP) s_bad[t] = 1;
                continue;
            }
            if (s_bad[t]) {
                constexpr uint32_t two = T::NOT | (uint32_t)T::NOT << 16;
                kw = make_uint4(two, two, two, two);
                vw = make_uint4(0, 0, 0, 0);
            }
            *reinterpret_cast<uint4 *>(a.c.tail_k + now + t * D + d) = kw;
            const uint32_t w[4] = {vw.x, vw.y, vw.z, vw.w};
            for (int j = 0; j < 8; ++j) a.c.tail_v[now + (d + j) * KB + t] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------
// Attention.  Rows are pairs (query token, query head of the group), 16 of them to a tile, which share the keys and values
// of one key/value head.  s^T = K q^T and o^T = V^T p^T on v_mfma_f32_16x16x32: a lane's column is a row of the tile, so
// the running maximum and sum are the lane's own and the tile of s^T is, register for register, the operand p^T of the
// second product (which token of the block stands in which row of s^T is chosen so: row m of tile t is token
// 16 (m / 4) + 4 t + m % 4).  Keys and values go straight from memory to LDS, 1 KB contiguous to a load, and from there as operands
// into registers (loaded as operands, whose neighbouring lanes lie a row apart, every lane of a load is an access of its own:
// 10.7 instead of 13.2 TB/s from the second-level cache); the next block's keys are asked for as soon as this one's are in
// registers, the values likewise, so that a wave always has a block on its way.  A wave takes every fourth block of its workgroup's
// range; the four join through LDS, ranges of a long cache through memory (k_kv_join).
// Bound by memory: 820 MB of cache (four sequences of 100 000 tokens) at 5.5 TB/s, 545 MB (64 sequences of up to 8192) at 4.9; listed blocks of
// many tokens by the second-level caches, 14.6 TB/s.
// ------------------------------------------------------------------------------------------------
struct KvAttendArgs {
    KvView c;
    const uint16_t *q;
    int64_t qs[3];  // strides of sequence, token, head
    const int32_t *counts, *lists;
    uint16_t *out;
    float *lse;
    float *part_o, *part_ml;  // partial results of ranges: [slot][rows of a tile][D], [slot][rows of a tile][2]
    int4 *plan;               // [b]: what k_kv_join needs of the sequence's ranges
    float *row_lse, *block_lse;  // logarithms (base 2) for the blocks' weights: [b][h][row], [b][h][blocks + 1][row]
    float scale2;  // softmax scale times log2 e, finite
    int n, g, w, splits;
    int tiles;        // row tiles of a (sequence, head): of all tokens, or of one token where blocks are listed
    int64_t units;    // listed: (sequence, token, tile, head) units
    bool split;       // whole caches: into ranges
};

constexpr int KV_LEAST = 4;    // blocks of a range, one to a wave
// Workgroups that the card holds at once: two to a compute unit, as many as 128 dimensions leave room for (64 KB of LDS in k_kv_attend, registers in
// k_kv_tile).  The same number is planned with for 64 and 96 dimensions, of which more would fit.
constexpr int KV_ROUND = 512;
constexpr int KV_ROUNDS = 3;   // most rounds of them that ranges are made for

// A sequence's workgroups: `live` tiles of `tiles` have rows that are no padding; first the ranges of those, heads innermost, then one to
// each (tile, head) of padding.
struct KvRange {
    int b, live, splits, per;  // sequence; its tiles; ranges of its blocks; blocks of a range
    int first;                 // number of its first workgroup
};

// Sums over the lanes up to each one
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_from(int x)
{
    return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int sum_upto(int x)
{
    x = add_from<0x111, 0xf>(x);  // one, two, four and eight lanes up within rows of 16
    x = add_from<0x112, 0xf>(x);
    x = add_from<0x114, 0xf>(x);
    x = add_from<0x118, 0xf>(x);
    x = add_from<0x142, 0xa>(x);  // a row's last lane into the next row, of the first half into the second
    return add_from<0x143, 0xc>(x);
}

// Workgroup numbers of a call over whole caches: every sequence gets ranges of up to `per` blocks for each of its live tiles of ROWS rows and
// heads, of one length within the sequence, and `per` comes from the blocks of all sequences, so that the lengths on the device decide
// the split and long sequences get more workgroups.  Of the splits into one to three rounds of workgroups the one is taken whose rounds times
// blocks of a range, with four more for a range's start and its join, are the least.  The sequence that workgroup `find` works for
// (b = batch: none); its first workgroup leaves the ranges for k_kv_join (planning there again: 29 us instead of 15 for pieces of three
// prompts).  Every lane of the wave calls it.
template <int ROWS>
__device__ __forceinline__ KvRange kv_plan(const KvAttendArgs &a, int find)
{
    constexpr int LEAST = ROWS == 16 ? KV_LEAST : 1;  // the waves of a tile of 128 rows take the same blocks
    const int lane = threadIdx.x & 63, batch = a.c.batch, H = a.c.heads;
    auto blocks_of = [&](int i) { return i < batch ? (kv_len(a.c, i) + KB - 1) / KB : 0; };
    auto live_of = [&](int i) { return i < batch ? (kv_count(a.counts, i, a.n) * a.g + ROWS - 1) / ROWS : 0; };
    KvRange r;
    r.per = 1 << 30;  // no splits
    if (a.split) {
        const int blocks0 = blocks_of(lane), live0 = live_of(lane);  // of the first 64 sequences, as a rule all
        int units = 0;
        double total = 0;  // whole numbers below 2^53
        for (int i0 = 0; i0 < batch; i0 += 64) {
            const int blocks = i0 ? blocks_of(i0 + lane) : blocks0, live = i0 ? live_of(i0 + lane) : live0;
            units += __builtin_amdgcn_readlane(sum_upto(live), 63) * H;
            const uint64_t both = (uint64_t)blocks * live;  // below 2^48: added up in two halves
            total += (16777216.0 * __builtin_amdgcn_readlane(sum_upto((int)(both >> 24)), 63) + __builtin_amdgcn_readlane(sum_upto((int)(both & 0xFFFFFF)), 63)) * H;
        }
        int64_t least = INT64_MAX;
        for (int rounds = 1; rounds <= KV_ROUNDS; ++rounds) {
            // ranges come to no more than the divisor and one for each unit
            const int room = rounds * KV_ROUND - units;
            if (room <= 0 && rounds < KV_ROUNDS) continue;
            const int per = max(LEAST, (int)min(1073741824.0, ceil(total / (room > 0 ? room : 2 * KV_ROUND))));
            int many = 0;
            for (int i0 = 0; i0 < batch; i0 += 64) {
                const int blocks = i0 ? blocks_of(i0 + lane) : blocks0, live = i0 ? live_of(i0 + lane) : live0;
                many += __builtin_amdgcn_readlane(sum_upto(max(1, (blocks + per - 1) / per) * live), 63) * H;
            }
            const int64_t cost = (int64_t)((many + KV_ROUND - 1) / KV_ROUND) * (per + 4);
            if (cost < least) {
                least = cost;
                r.per = per;
            }
            if (per == LEAST) break;
        }
        r.per = __builtin_amdgcn_readfirstlane(r.per);
    }
    int base = 0;
    for (int i0 = 0; i0 < batch; i0 += 64) {
        const int i = i0 + lane, blocks = blocks_of(i), live = live_of(i), s = i < batch ? max(1, (blocks + r.per - 1) / r.per) : 0;
        const int upto = base + sum_upto(i < batch ? (s - 1) * live + a.tiles : 0) * H;
        const uint64_t hit = __ballot(i < batch && upto > find);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            r.b = i0 + l;
            r.splits = __builtin_amdgcn_readlane(s, l);
            r.live = __builtin_amdgcn_readlane(live, l);
            r.first = __builtin_amdgcn_readlane(upto, l) - ((r.splits - 1) * r.live + a.tiles) * H;
            const int even = (__builtin_amdgcn_readlane(blocks, l) + r.splits - 1) / r.splits;
            r.per = min(r.per, (even + LEAST - 1) / LEAST * LEAST);
            if (a.split && r.first == find && threadIdx.x == 0) a.plan[r.b] = make_int4(r.live, r.splits, r.first, 0);
            return r;
        }
        base = __builtin_amdgcn_readlane(upto, 63);
    }
    r.b = batch;
    r.live = r.splits = r.first = 0;
    return r;
}

// what a block's products are multiplied by, its key scale times the softmax scale: neither 0, which masked places (-inf) turn into not a number, nor
// infinite, which products of 0 do
__device__ __forceinline__ float logit_factor(float key_scale, float scale2) { return __builtin_amdgcn_fmed3f(key_scale * scale2, 0x1p-149f, 3.402823466e38f); }

__device__ __forceinline__ float row_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Where the 16-byte piece `at` of a row of keys (a token's) or values (a dimension's) stands in its row of LDS: lanes that read
// together hit all banks.  Its own inverse but for rows of six pieces (BACK: which piece stands at `at`).
template <int D, bool BACK>
__device__ __forceinline__ int k_place(int token, int at)
{
    if constexpr (D == 96) return (at + (BACK ? 6 - (token >> 4) : token >> 4)) % 6;
    return at ^ (D == 128 ? (token >> 1 & 1) | (token >> 4) << 1 : token >> 4);
}
__device__ __forceinline__ int v_place(int d, int at) { return at ^ (d >> 2 & 3); }

// 16 bytes to a lane from `from` to the 1 KB of LDS at `to`, in the order of the lanes
__device__ __forceinline__ void load_lds(const void *from, void *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
// waits until no more than `left` of the wave's loads are on their way
#define KV_WAIT_LOADS(left) asm volatile("s_waitcnt vmcnt(" #left ")" ::: "memory")
__device__ __forceinline__ void wait_loads(int left)
{
    switch (left) {
        case 8: KV_WAIT_LOADS(8); break;
        case 6: KV_WAIT_LOADS(6); break;
        case 4: KV_WAIT_LOADS(4); break;
        default: KV_WAIT_LOADS(0);
    }
}
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// Reads of LDS that have arrived when the block ends (the compiler, which does not see that the loads into LDS and these
// reads are ordered by the waits above, would wait for every load on its way before each of them).
// Eight rows of 1 KB apart, or six, or four: the values of a lane.
template <int N>
__device__ __forceinline__ void read_v(uint32_t at, u32x4 (&v)[N])
{
    if constexpr (N == 8)
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:1024\n\tds_read_b128 %2, %8 offset:2048\n\tds_read_b128 %3, %8 offset:3072\n\t"
                     "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %8 offset:5120\n\tds_read_b128 %6, %8 offset:6144\n\tds_read_b128 %7, %8 offset:7168\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
                     : "v"(at)
                     : "memory");
    else if constexpr (N == 6)
        asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %1, %6 offset:1024\n\tds_read_b128 %2, %6 offset:2048\n\tds_read_b128 %3, %6 offset:3072\n\t"
                     "ds_read_b128 %4, %6 offset:4096\n\tds_read_b128 %5, %6 offset:5120\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5])
                     : "v"(at)
                     : "memory");
    else
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:1024\n\tds_read_b128 %2, %4 offset:2048\n\tds_read_b128 %3, %4 offset:3072\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
                     : "v"(at)
                     : "memory");
}
// The keys of a lane: four tokens, four apart; of each the pieces at `at` and (128 dimensions) `more`, or half a piece at `more` (96).
template <int D>
struct KvKeys {
    u32x4 wide[4][D / 64];
    uint2 odd[4];
};
template <int D>
__device__ __forceinline__ void read_k(uint32_t at, uint32_t more, KvKeys<D> &k)
{
    if constexpr (D == 128) {
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %8 offset:512\n\tds_read_b128 %3, %9 offset:512\n\t"
                     "ds_read_b128 %4, %8 offset:1024\n\tds_read_b128 %5, %9 offset:1024\n\tds_read_b128 %6, %8 offset:1536\n\tds_read_b128 %7, %9 offset:1536\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(k.wide[0][0]), "=&v"(k.wide[0][1]), "=&v"(k.wide[1][0]), "=&v"(k.wide[1][1]), "=&v"(k.wide[2][0]), "=&v"(k.wide[2][1]),
                       "=&v"(k.wide[3][0]), "=&v"(k.wide[3][1])
                     : "v"(at), "v"(more)
                     : "memory");
    } else if constexpr (D == 96) {
        uint64_t o[4];
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b64 %1, %9\n\tds_read_b128 %2, %8 offset:384\n\tds_read_b64 %3, %9 offset:384\n\t"
                     "ds_read_b128 %4, %8 offset:768\n\tds_read_b64 %5, %9 offset:768\n\tds_read_b128 %6, %8 offset:1152\n\tds_read_b64 %7, %9 offset:1152\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(k.wide[0][0]), "=&v"(o[0]), "=&v"(k.wide[1][0]), "=&v"(o[1]), "=&v"(k.wide[2][0]), "=&v"(o[2]), "=&v"(k.wide[3][0]), "=&v"(o[3])
                     : "v"(at), "v"(more)
                     : "memory");
        for (int t = 0; t < 4; ++t) k.odd[t] = make_uint2((uint32_t)o[t], (uint32_t)(o[t] >> 32));
    } else {
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:256\n\tds_read_b128 %2, %4 offset:512\n\tds_read_b128 %3, %4 offset:768\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(k.wide[0][0]), "=&v"(k.wide[1][0]), "=&v"(k.wide[2][0]), "=&v"(k.wide[3][0])
                     : "v"(at)
                     : "memory");
    }
}

// SOLO: every wave of a workgroup has a unit of its own (listed blocks, enough units for the card): nothing to join.
template <typename T, int D, bool LIST, bool MASS, bool SOLO>
__global__ __launch_bounds__(256, 2) void k_kv_attend(KvAttendArgs a)
{
    static_assert(!SOLO || (LIST && !MASS), "units of a wave are listed ones");
    constexpr int KS = D / 32;  // steps of the first product
    constexpr int DT = D / 16;  // tiles of the second
    constexpr int WIDE = D / 64, ODD = D % 64 / 32;
    constexpr int OROW = D + 4;
    constexpr int HALF = KB * D;            // bytes of a block's keys, of its values
    constexpr int LOADS = HALF / 1024;      // loads for either
    constexpr int JOIN = 4 * 16 * (OROW + 2) * 4;
    // a wave's block on its way; afterwards the waves' results
    __shared__ __attribute__((aligned(1024))) uint8_t s_all[8 * HALF > JOIN || SOLO ? 8 * HALF : JOIN];
    float(*s_o)[16][OROW] = reinterpret_cast<float(*)[16][OROW]>(s_all);
    float(*s_ml)[16][2] = reinterpret_cast<float(*)[16][2]>(s_all + 4 * 16 * OROW * 4);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), x = lane & 15, hq = lane >> 4;
    const int H = a.c.heads, g = a.g;
    int b, h, tile, token = 0, splits, from, to;
    int64_t slot;
    if (LIST) {
        splits = a.splits;
        slot = blockIdx.x;
        int64_t unit;  // of its head
        int split = 0;
        if (SOLO) {
            // a head's tokens to every H-th workgroup: consecutive ones go to the XCDs in turn, so that with 8 heads (or 4, 2, 1) an XCD's
            // second-level cache serves few of them (1000 tokens, 8 heads with 4.2 MB each: 40 % of the reads missed it)
            h = (int)(blockIdx.x % H);
            unit = (int64_t)(blockIdx.x / H) * 4 + wave;
            if (unit >= a.units / H) return;
        } else {
            unit = blockIdx.x % a.units;
            split = (int)(blockIdx.x / a.units);
            h = (int)(unit % H);
            unit /= H;
        }
        tile = (int)(unit % a.tiles);
        token = (int)(unit / a.tiles % a.n);
        b = (int)(unit / ((int64_t)a.tiles * a.n));
        const int per = (a.w + 1 + splits - 1) / splits;
        from = split * per;
        to = min(a.w + 1, from + per);
    } else {
        const KvRange r = kv_plan<16>(a, blockIdx.x);
        if (r.b >= a.c.batch) return;
        b = r.b;
        const int local = (int)blockIdx.x - r.first, units = r.live * H, pad = local - units * r.splits;
        slot = blockIdx.x;
        h = (pad < 0 ? local : pad) % H;
        if (pad < 0) {
            splits = r.splits;
            tile = local / H % r.live;
            from = local / units * r.per;
            to = from + r.per;
        } else {  // rows of padding: zeros
            splits = 1;
            tile = r.live + pad / H;
            from = to = 0;
        }
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const int64_t bh = (int64_t)b * H + h;
    const int len = kv_len(a.c, b), count = kv_count(a.counts, b, a.n), nb = len / KB;
    // this lane's row, and what it sees
    const int row = LIST ? token * g + tile * 16 + x : tile * 16 + x;
    const int qi = LIST ? token : row / g, hg = LIST ? tile * 16 + x : row % g;
    const bool valid = LIST ? hg < g : row < a.n * g;
    const bool live = valid && qi < count;
    const int sees = live ? max(0, len - count + qi + 1) : 0;
    // what all rows of the tile see, and what any does
    int least, most;
    if (LIST) {
        least = most = token < count ? max(0, len - count + token + 1) : 0;
    } else {
        const int i0 = tile * 16 / g, i1 = min(min(tile * 16 + 15, a.n * g - 1) / g, count - 1);
        least = max(0, len - count + i0 + 1);
        most = i1 >= i0 ? max(0, len - count + i1 + 1) : 0;
        if (MASS)
            to = min(to, (len + KB - 1) / KB);
        else
            to = min(to, (most + KB - 1) / KB);
    }
    const int whole = most / KB;  // listed: blocks that the token sees all of

    typename T::x8 q[KS];
    const uint16_t *qp = a.q + b * a.qs[0] + (valid ? qi : 0) * a.qs[1] + ((int64_t)h * g + (valid ? hg : 0)) * a.qs[2];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = ks < 2 * WIDE ? 64 * (ks / 2) + 16 * hq + 8 * (ks % 2) : 64 * WIDE + 8 * hq;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (live) w = *reinterpret_cast<const uint4 *>(qp + d);
        q[ks] = __builtin_bit_cast(typename T::x8, w);
    }

    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    // A wave's items, every STEPth of the range: number u of them is block j of the cache and the page it lies in (-1: none, -2: the
    // open block).  64 of them are looked up together, one to a lane.
    constexpr int STEP = SOLO ? 1 : 4;
    const int start = SOLO ? from : from + wave, many = start < to ? (to - start + STEP - 1) / STEP : 0;
    int js = 0, ps = -1;
    f32x2 ss = {0.f, 0.f};
    auto look = [&](int u0) {
        const int u = start + (u0 + lane) * STEP;
        js = 0;
        ps = -1;
        if (u >= to) return;
        bool open = false;
        if (LIST) {
            if (u == a.w) {  // the block that the token sees a part of
                js = whole;
                if (most % KB == 0) return;
                open = js == nb;
            } else {
                js = a.lists[(((int64_t)b * a.n + token) * H + h) * a.w + u];
                if (js < 0 || js >= whole) return;
            }
        } else {
            js = u;
            open = js == nb;
        }
        ps = open ? -2 : kv_page(a.c, bh, js);
        if (ps >= 0) ss = *reinterpret_cast<const f32x2 *>(a.c.scales + (int64_t)ps * 2);
    };

    const int kt = 16 * (x / 4) + x % 4;  // this lane's token of key tile 0
    uint8_t *s_k = s_all + wave * (2 * HALF), *s_v = s_k + HALF;
    const uint32_t k_at = lds_address(s_k) + kt * D + 16 * k_place<D, false>(kt, hq);
    const uint32_t k_more = D == 128 ? k_at ^ 64 : lds_address(s_k) + kt * D + 16 * k_place<D, false>(kt, 4 + hq / 2) + 8 * (hq & 1);
    const uint32_t v_at = lds_address(s_v) + x * KB + 16 * v_place(x, hq);
    auto load_k = [&](int page) {
        const uint8_t *p = a.c.k + (int64_t)page * HALF;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = 64 * i + lane, token = at / (D / 16);
            load_lds(p + token * D + 16 * k_place<D, true>(token, at % (D / 16)), s_k + 1024 * i);
        }
    };
    auto load_v = [&](int page) {
        const uint8_t *p = a.c.v + (int64_t)page * HALF;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = 64 * i + lane, d = at / 4;
            load_lds(p + d * KB + 16 * v_place(d, at % 4), s_v + 1024 * i);
        }
    };

    // logits of a block become weights: z in, p out, reference and sum kept
    auto softmax = [&](f32x4 (&s)[4], float scale, int j, bool all) {
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float z = s[t][i] * scale;
                if (!all && j * KB + 16 * hq + 4 * t + i >= sees) z = -INFINITY;
                s[t][i] = z;
                top = fmaxf(top, z);
            }
        top = fmaxf(m, reference<T::UP>(row_max(top)));
        const float base = top == -INFINITY ? 0.f : top;
        const float fade = __builtin_amdgcn_exp2f(m - base);
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(s[t][i] - base);
                sum += s[t][i];
            }
        if (__any(top != m)) {
#pragma unroll
            for (int i = 0; i < DT; ++i) o[i] *= fade;
        }
        m = top;
        l = l * fade + sum;
        if (MASS) {
            const float all_sum = row_sum(sum);
            if (hq == 0 && valid) a.block_lse[(bh * (a.c.blocks + 1) + j) * a.n * g + row] = base + __builtin_amdgcn_logf(all_sum);
        }
    };
    // The matrix cores' second operand has 16 bits: a weight is rounded to the type, off by half a unit of it at most, while its sum is
    // not.  Two operands for each weight would keep 32 bits and double the second product.
    auto pack = [&](const f32x4 (&s)[4], int e) {
        const typename T::x2 p0 = T::narrow(s[2 * e][0], s[2 * e][1]), p1 = T::narrow(s[2 * e][2], s[2 * e][3]);
        const typename T::x2 p2 = T::narrow(s[2 * e + 1][0], s[2 * e + 1][1]), p3 = T::narrow(s[2 * e + 1][2], s[2 * e + 1][3]);
        return (typename T::x8){p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    };

    look(0);
    bool open = false;
    int page = __builtin_amdgcn_readlane(ps, 0);
    if (many > 0 && page >= 0) {
        load_k(page);
        load_v(page);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = query8<T>(q[ks]);  // behind the first block's loads
    for (int u = 0; u < many; ++u) {
        const int j = __builtin_amdgcn_readlane(js, u & 63);
        const float ks = logit_factor(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ss[0]), u & 63)), a.scale2);
        float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ss[1]), u & 63));
        if ((u & 63) == 63) look(u + 1);
        const int pn = u + 1 < many ? __builtin_amdgcn_readlane(ps, (u + 1) & 63) : -1;
        if (page >= 0) {
            // on their way: this block's keys, then its values
            wait_loads(LOADS);
            f32x4 s[4];
            {
                KvKeys<D> k;
                read_k<D>(k_at, k_more, k);
                if (pn >= 0) load_k(pn);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    s[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < WIDE; ++i) {
                        s[t] = T::mfma(bring8<T>(k.wide[t][i].x, k.wide[t][i].y, 1.f), q[2 * i], s[t]);
                        s[t] = T::mfma(bring8<T>(k.wide[t][i].z, k.wide[t][i].w, 1.f), q[2 * i + 1], s[t]);
                    }
                    if (ODD) s[t] = T::mfma(bring8<T>(k.odd[t].x, k.odd[t].y, 1.f), q[KS - 1], s[t]);
                }
            }
            softmax(s, ks, j, (j + 1) * KB <= least);
            typename T::x8 p0 = pack(s, 0), p1 = pack(s, 1);
            if (T::NARROW && vs > 128.f) {
                vs *= 0.5f;
                p0 = p0 + p0;
                p1 = p1 + p1;
            }
            // this block's values, then the next one's keys
            if (pn >= 0)
                wait_loads(LOADS);
            else
                wait_loads(0);
            u32x4 v[DT];
            read_v<DT>(v_at, v);
            if (pn >= 0) load_v(pn);
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                o[i] = T::mfma(bring8<T>(v[i].x, v[i].y, vs), p0, o[i]);
                o[i] = T::mfma(bring8<T>(v[i].z, v[i].w, vs), p1, o[i]);
            }
        } else {
            if (page == -2)
                open = true;
            else if (MASS && hq == 0 && valid)
                a.block_lse[(bh * (a.c.blocks + 1) + j) * a.n * g + row] = -INFINITY;
            if (pn >= 0) {
                load_k(pn);
                load_v(pn);
            }
        }
        page = pn;
    }
    if (open) {  // the last block of the wave that has it
        const int64_t tail = kv_tail(a.c, bh, b, nb, D);
        const uint16_t *tk = a.c.tail_k + tail, *tv = a.c.tail_v + tail;
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = ks < 2 * WIDE ? 64 * (ks / 2) + 16 * hq + 8 * (ks % 2) : 64 * WIDE + 8 * hq;
                s[t] = T::mfma(*reinterpret_cast<const typename T::x8 *>(tk + (kt + 4 * t) * D + d), q[ks], s[t]);
            }
        }
        softmax(s, a.scale2, nb, false);
        const typename T::x8 p0 = pack(s, 0), p1 = pack(s, 1);
        // what no token has written yet may be anything: its values count as zero
        const int held = len - nb * KB - 16 * hq;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            __builtin_amdgcn_sched_barrier(0);  // few of these loads at once: two waves' registers have to fit
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                typename T::x8 v = *reinterpret_cast<const typename T::x8 *>(tv + (i * 16 + x) * KB + 16 * hq + 8 * e);
#pragma unroll
                for (int y = 0; y < 8; ++y) v[y] = 8 * e + y < held ? v[y] : 0;
                o[i] = T::mfma(v, e ? p1 : p0, o[i]);
            }
        }
    }

    // the four waves' results into one
    l = row_sum(l);
    if (!live) {  // a row of padding: nothing seen
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    if constexpr (SOLO) {
        if (!valid) return;
        const int64_t at = ((int64_t)b * a.n + qi) * H * g + h * g + hg;
        const float f = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const typename T::x2 p0 = T::narrow(o[i][0] * f, o[i][1] * f), p1 = T::narrow(o[i][2] * f, o[i][3] * f);
            *reinterpret_cast<uint2 *>(a.out + at * D + 16 * i + 4 * hq) = make_uint2(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1));
        }
        if (a.lse && hq == 0) a.lse[at] = (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
        return;
    }
    __syncthreads();  // no wave reads its block any more
    if (hq == 0) {
        s_ml[wave][x][0] = m;
        s_ml[wave][x][1] = l;
    }
#pragma unroll
    for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4 *>(&s_o[wave][x][16 * i + 4 * hq]) = o[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * D / 4; e += 256) {
        const int y = e / (D / 4), d = e % (D / 4) * 4;
        const int yrow = LIST ? token * g + tile * 16 + y : tile * 16 + y;
        const int yi = LIST ? token : yrow / g, yh = LIST ? tile * 16 + y : yrow % g;
        if (LIST ? yh >= g : yrow >= a.n * g) continue;
        const float top = fmaxf(fmaxf(s_ml[0][y][0], s_ml[1][y][0]), fmaxf(s_ml[2][y][0], s_ml[3][y][0]));
        const float base = top == -INFINITY ? 0.f : top;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = __builtin_amdgcn_exp2f(s_ml[i][y][0] - base);
            all += s_ml[i][y][1] * f;
            sum += *reinterpret_cast<const f32x4 *>(&s_o[i][y][d]) * f;
        }
        if (splits > 1) {
            *reinterpret_cast<f32x4 *>(a.part_o + (slot * 16 + y) * D + d) = sum;
            if (d == 0) {
                a.part_ml[(slot * 16 + y) * 2] = top;
                a.part_ml[(slot * 16 + y) * 2 + 1] = all;
            }
        } else {
            const float f = all != 0.f ? 1.f / all : 0.f;
            const int64_t at = ((int64_t)b * a.n + yi) * H * g + h * g + yh;
            const typename T::x2 p0 = T::narrow(sum[0] * f, sum[1] * f), p1 = T::narrow(sum[2] * f, sum[3] * f);
            *reinterpret_cast<uint2 *>(a.out + at * D + d) = make_uint2(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1));
            if (d == 0) {
                const float y2 = top + __builtin_amdgcn_logf(all);
                if (a.lse) a.lse[at] = y2 * 0.69314718055994531f;
                if (MASS) a.row_lse[bh * a.n * g + yrow] = y2;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Attention of many rows: prompts.  128 rows to a workgroup, 32 to a wave; a block's codes are staged in LDS once for all of them
// and become operands as they are read.  s^T = K q^T and o^T = V^T p^T on v_mfma_f32_32x32x16, again so that a lane's column is a
// row and p^T stands in its registers as the second product wants it: row m of a tile of s^T is token
// 16 (m / 4 % 2) + 8 (m / 16) + 4 (m / 8 % 2) + m % 4 of its 32.  The next block is on its way from memory to registers while this one
// is worked on.  Pieces of 16 bytes are exchanged within a row of LDS, so that eight lanes that read together hit all banks.
// Bound by vector issue beside the matrix cores (64 % and 42 % of the time): two prompts of 4096 tokens, 32 heads of 128 dimensions 302
// to 332 us from card to card = 830 to 910 TFLOP/s.  Making operands of the codes once a workgroup, on their way into LDS, instead of in every wave: 306 us
// where that is 302.
// ------------------------------------------------------------------------------------------------
template <typename T, int D, bool MASS>
__global__ __launch_bounds__(256, 2) void k_kv_tile(KvAttendArgs a)
{
    constexpr int ROWS = 128;
    constexpr int PAIRS = D / 32;               // steps of the first product, two by two: 16 dimensions of each half of the wave
    constexpr int DT = D / 32;                  // tiles of the second product
    constexpr int KP = D / 16;                  // pieces of a row of keys
    constexpr int LOADS = KB * D / 16 / 256 + (KB * D / 16 % 256 ? 1 : 0);  // pieces of a thread, of keys and of values
    __shared__ u32x4 s_k[2][KB * D / 16], s_v[2][KB * D / 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), x = lane & 31, half = lane >> 5;
    const int H = a.c.heads, g = a.g;
    const KvRange r = kv_plan<128>(a, blockIdx.x);
    if (r.b >= a.c.batch) return;
    const int b = __builtin_amdgcn_readfirstlane(r.b), units = r.live * H;
    const int local = __builtin_amdgcn_readfirstlane((int)blockIdx.x - r.first), pad = local - units * r.splits;
    const int h = (pad < 0 ? local : pad) % H, splits = pad < 0 ? r.splits : 1;
    const int tile = pad < 0 ? r.live - 1 - local / H % r.live : r.live + pad / H;  // the longest ones first; rows of padding last
    const int range = pad < 0 ? local / units : 0;
    const int64_t bh = (int64_t)b * H + h, slot = r.first + range * units + tile * H + h;
    const int len = kv_len(a.c, b), count = kv_count(a.counts, b, a.n), nb = len / KB;
    auto seen_by = [&](int row) {  // what the row sees; rows past the last one like it
        const int i = min(row, a.n * g - 1) / g;
        return i < count ? max(0, len - count + i + 1) : 0;
    };
    const int row0 = tile * ROWS, wrow = row0 + 32 * wave, row = wrow + x;
    const bool valid = row < a.n * g;
    const int qi = min(row, a.n * g - 1) / g, hg = valid ? row % g : 0;
    const bool live = valid && qi < count;
    const int sees = live ? seen_by(row) : 0;
    // the rows of one tile see no less from one to the next, up to the last one that is not padding
    auto most_of = [&](int from, int rows) {
        const int i0 = from / g, i1 = min(min(from + rows, a.n * g) - 1, count * g - 1) / g;
        return from < a.n * g && i0 < count ? max(0, len - count + i1 + 1) : 0;
    };
    const int most = most_of(row0, ROWS), wmost = most_of(wrow, 32), wleast = wrow < a.n * g ? seen_by(wrow) : 0;
    const int from = range * r.per;
    const int to = pad < 0 ? min(from + r.per, MASS ? (len + KB - 1) / KB : (most + KB - 1) / KB) : 0;

    typename T::x8 q[2 * PAIRS];
    const uint16_t *qp = a.q + b * a.qs[0] + (int64_t)qi * a.qs[1] + ((int64_t)h * g + hg) * a.qs[2];
#pragma unroll
    for (int i = 0; i < 2 * PAIRS; ++i) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (live) w = *reinterpret_cast<const uint4 *>(qp + 16 * (i / 2 * 2 + half) + 8 * (i % 2));
        q[i] = query8<T>(__builtin_bit_cast(typename T::x8, w));
    }
    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = (f32x16)(0.f);
    float m = -INFINITY, l = 0.f;

    // piece p of the keys lies at p of LDS; the piece of the row that it holds:
    auto k_piece = [](int token, int at) { return KP == 8 ? at ^ ((token & 3) | (token >> 4 & 1) << 2) : KP == 4 ? at ^ (token & 3) : at; };
    auto v_piece = [](int d, int at) { return at ^ (d >> 2 & 3); };
    u32x4 next_k[LOADS], next_v[LOADS];
    f32x2 next_scales = {0.f, 0.f};
    auto fetch = [&](int page) {
        const u32x4 *pk = reinterpret_cast<const u32x4 *>(a.c.k + (int64_t)page * (KB * D)), *pv = reinterpret_cast<const u32x4 *>(a.c.v + (int64_t)page * (KB * D));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = tid + 256 * i;
            if (KB * D / 16 % 256 && p >= KB * D / 16) continue;
            next_k[i] = pk[p / KP * KP + k_piece(p / KP, p % KP)];
            next_v[i] = pv[p / 4 * 4 + v_piece(p / 4, p % 4)];
        }
        next_scales = *reinterpret_cast<const f32x2 *>(a.c.scales + (int64_t)page * 2);
    };
    auto stage = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = tid + 256 * i;
            if (KB * D / 16 % 256 && p >= KB * D / 16) continue;
            s_k[buf][p] = next_k[i];
            s_v[buf][p] = next_v[i];
        }
    };
    const int kt = 16 * (x >> 2 & 1) + 8 * (x >> 4) + 4 * (x >> 3 & 1) + (x & 3);  // this lane's token of tile 0

    // logits of a block become weights; z = s * scale
    auto softmax = [&](f32x16 (&s)[2], float scale, int j, bool all) {
        if (!all) {
            asm volatile("");  // a branch: few blocks need the comparisons
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j * KB + 32 * t + 16 * half + i >= sees) s[t][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
        top = fmaxf(top, __shfl_xor(top, 32)) * scale;
        // z is s * scale less the reference with one rounding, as long as what rounding the largest z has left out matters no more than the others'
        // roundings; from there on, with one more, no z is above the largest: exponentials stay within the type
        if (__any(fabsf(top) > 0x1p20f)) {
            asm volatile("");  // a branch: few blocks need it
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] *= scale;
            scale = 1.f;
        }
        top = reference<T::TILE_UP>(top);
        // the reference in use may lag behind by a factor of 2^TILE_LAG in the weights, which changes nothing but spares the scaling
        if (__any(top - m > T::TILE_LAG)) {
            const float was = m;
            m = fmaxf(m, top);
            const float fade = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(was - m);
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
                sum += s[t][i];
            }
        l += sum;
        if (MASS) {
            sum += __shfl_xor(sum, 32);
            if (half == 0 && valid) a.block_lse[(bh * (a.c.blocks + 1) + j) * a.n * g + row] = base + __builtin_amdgcn_logf(sum);
        }
    };
    // operand p^T of step u of tile t, rounded to the type as in k_kv_attend
    auto pack = [&](const f32x16 &s, int u) {
        const typename T::x2 p0 = T::narrow(s[8 * u], s[8 * u + 1]), p1 = T::narrow(s[8 * u + 2], s[8 * u + 3]);
        const typename T::x2 p2 = T::narrow(s[8 * u + 4], s[8 * u + 5]), p3 = T::narrow(s[8 * u + 6], s[8 * u + 7]);
        return (typename T::x8){p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    };

    const int paged = min(to, nb);  // the open block comes last, on its own
    int page = from < paged ? __builtin_amdgcn_readfirstlane(kv_page(a.c, bh, from)) : -1;
    int after = from + 1 < paged ? kv_page(a.c, bh, from + 1) : -1;
    if (page >= 0) {
        fetch(page);
        stage(0);
    }
    __syncthreads();
    int buf = 0;
    for (int j = from; j < paged; ++j) {
        const int next = __builtin_amdgcn_readfirstlane(after);
        after = j + 2 < paged ? kv_page(a.c, bh, j + 2) : -1;
        const float ks = next_scales[0];
        float vs = next_scales[1];
        if (next >= 0) fetch(next);
        if (page >= 0 && (MASS || j * KB < wmost)) {
            f32x16 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = (f32x16)(0.f);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const u32x4 w = s_k[buf][(kt + 32 * t) * KP + k_piece(kt + 32 * t, 2 * i + half)];
                    s[t] = T::mfma(bring8<T>(w.x, w.y, 1.f), q[2 * i], s[t]);
                    s[t] = T::mfma(bring8<T>(w.z, w.w, 1.f), q[2 * i + 1], s[t]);
                }
            }
            softmax(s, logit_factor(ks, a.scale2), j, (j + 1) * KB <= wleast);
            typename T::x8 p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = pack(s[i / 2], i % 2);
            if (T::NARROW && __builtin_amdgcn_readfirstlane(__float_as_uint(vs)) > 0x43000000u) {  // above 128
                asm volatile("");  // a branch: few blocks need it
                vs *= 0.5f;
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = p[i] + p[i];
            }
            if (next >= 0) stage(buf ^ 1);  // ahead of the second product rather than after it: 302 us instead of 309
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 w = s_v[buf][(32 * i + x) * 4 + v_piece(32 * i + x, 2 * t + half)];
                    o[i] = T::mfma(bring8<T>(w.x, w.y, vs), p[2 * t], o[i]);
                    o[i] = T::mfma(bring8<T>(w.z, w.w, vs), p[2 * t + 1], o[i]);
                }
        } else {
            if (MASS && page < 0 && half == 0 && valid) a.block_lse[(bh * (a.c.blocks + 1) + j) * a.n * g + row] = -INFINITY;
            if (next >= 0) stage(buf ^ 1);
        }
        __syncthreads();
        buf ^= 1;
        page = next;
    }
    if (nb >= from && nb < to && (MASS || nb * KB < wmost)) {
        const int64_t tail = kv_tail(a.c, bh, b, nb, D);
        const uint16_t *tk = a.c.tail_k + tail, *tv = a.c.tail_v + tail;
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = (f32x16)(0.f);
#pragma unroll
            for (int i = 0; i < 2 * PAIRS; ++i)
                s[t] = T::mfma(*reinterpret_cast<const typename T::x8 *>(tk + (kt + 32 * t) * D + 16 * (i / 2 * 2 + half) + 8 * (i % 2)), q[i], s[t]);
        }
        softmax(s, a.scale2, nb, false);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const typename T::x8 p = pack(s[y / 2], y % 2);
            // what no token has written yet may be anything: its values count as zero
            const int at = 32 * (y / 2) + 16 * half + 8 * (y % 2), held = len - nb * KB - at;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                typename T::x8 v = *reinterpret_cast<const typename T::x8 *>(tv + (32 * i + x) * KB + at);
#pragma unroll
                for (int z = 0; z < 8; ++z) v[z] = z < held ? v[z] : 0;
                o[i] = T::mfma(v, p, o[i]);
            }
        }
    }

    l += __shfl_xor(l, 32);
    if (!valid) return;
    if (!live) {  // padding: nothing seen
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = (f32x16)(0.f);
    }
    const int64_t at = ((int64_t)b * a.n + qi) * H * g + h * g + hg, part = slot * ROWS + row - row0;
    const float f = splits > 1 ? 1.f : l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int d = 32 * i + 8 * y + 4 * half;
            const f32x4 v = {o[i][4 * y] * f, o[i][4 * y + 1] * f, o[i][4 * y + 2] * f, o[i][4 * y + 3] * f};
            if (splits > 1) {
                *reinterpret_cast<f32x4 *>(a.part_o + part * D + d) = v;
            } else {
                const typename T::x2 p0 = T::narrow(v[0], v[1]), p1 = T::narrow(v[2], v[3]);
                *reinterpret_cast<uint2 *>(a.out + at * D + d) = make_uint2(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1));
            }
        }
    if (half == 0) {
        if (splits > 1) {
            a.part_ml[part * 2] = m;
            a.part_ml[part * 2 + 1] = l;
        } else {
            const float y2 = m + __builtin_amdgcn_logf(l);
            if (a.lse) a.lse[at] = y2 * 0.69314718055994531f;
            if (MASS) a.row_lse[bh * a.n * g + row] = y2;
        }
    }
}

// Joins the ranges of a long cache: 32 lanes to a row, eight rows to a workgroup.  A lane weighs one range at a time for its
// row, then all of them add up four dimensions each; the loads of a round do not wait for one another.
template <typename T, int D, int ROWS, bool LIST, bool MASS>
__global__ __launch_bounds__(256) void k_kv_join(KvAttendArgs a)
{
    constexpr int PARTS = ROWS / 8;  // workgroups of a tile
    const int H = a.c.heads, g = a.g, lane = threadIdx.x & 31, y = blockIdx.x % PARTS * 8 + threadIdx.x / 32;
    const int64_t unit = blockIdx.x / PARTS;
    const int h = (int)(unit % H), tile = (int)(unit / H % a.tiles);
    int b, token = 0, splits;
    int64_t slot, step;
    if (LIST) {
        token = (int)(unit / ((int64_t)H * a.tiles) % a.n);
        b = (int)(unit / ((int64_t)H * a.tiles * a.n));
        splits = a.splits;
        slot = unit;
        step = a.units;
    } else {
        b = (int)(unit / (a.tiles * H));
        const int4 r = a.plan[b];  // live tiles, ranges, first workgroup
        splits = tile < r.x ? r.y : 1;
        slot = r.z + tile * H + h;
        step = r.x * H;
    }
    if (splits < 2) return;
    const int row = LIST ? token * g + tile * ROWS + y : tile * ROWS + y;
    const int qi = LIST ? token : row / g, hg = LIST ? tile * ROWS + y : row % g;
    if (LIST ? hg >= g : row >= a.n * g) return;
    const int64_t first = slot * ROWS + y, next = step * ROWS;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < splits; s0 += 32) {
        const int s = s0 + lane;
        const float2 ml = s < splits ? *reinterpret_cast<const float2 *>(a.part_ml + (first + s * next) * 2) : make_float2(-INFINITY, 0.f);
        float top = ml.x;
        for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
        top = fmaxf(top, m);
        const float base = top == -INFINITY ? 0.f : top, fade = __builtin_amdgcn_exp2f(m - base), weight = __builtin_amdgcn_exp2f(ml.x - base);
        float sum = ml.y * weight;
        for (int i = 16; i; i >>= 1) sum += __shfl_xor(sum, i);
        l = l * fade + sum;
        o *= fade;
        m = top;
        const int many = min(32, splits - s0);
        const float *from = a.part_o + (first + s0 * next) * D + 4 * (lane < D / 4 ? lane : 0);
        for (int i0 = 0; i0 < many; i0 += 8) {
            f32x4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i0 + i < many ? *reinterpret_cast<const f32x4 *>(from + (i0 + i) * next * D) : (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i) o += v[i] * __shfl(weight, (threadIdx.x & 32) + i0 + i);
        }
    }
    const float f = l != 0.f ? 1.f / l : 0.f;
    const int64_t at = ((int64_t)b * a.n + qi) * H * g + h * g + hg;
    const typename T::x2 p0 = T::narrow(o[0] * f, o[1] * f), p1 = T::narrow(o[2] * f, o[3] * f);
    if (lane < D / 4) *reinterpret_cast<uint2 *>(a.out + at * D + 4 * lane) = make_uint2(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1));
    if (lane == 0) {
        const float y2 = m + __builtin_amdgcn_logf(l);
        if (a.lse) a.lse[at] = y2 * 0.69314718055994531f;
        if (MASS) a.row_lse[((int64_t)b * H + h) * a.n * g + row] = y2;
    }
}

// Weight of every block in this call, summed over the rows of a (sequence, head): 2^(block's logarithm - row's logarithm).
// `width` lanes to a block, a power of two: with few rows a workgroup has many blocks (4 rows of 16 x 8 x 128 blocks: 12.6 us with one
// to a workgroup).  Sums in 64 bits, in an order that does not depend on the launch.
__global__ __launch_bounds__(256) void k_kv_mass(KvView c, const float *__restrict__ row_lse, const float *__restrict__ block_lse, int rows, int width,
                                                 const float *mass_in, float *mass_out)
{
    __shared__ double s_sum[4];
    const int64_t at = (int64_t)blockIdx.x * (256 / width) + threadIdx.x / width, bh = at / c.blocks;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = threadIdx.x & (width - 1), j = (int)(at % c.blocks);
    const bool there = bh < (int64_t)c.batch * c.heads;
    double sum = 0;
    if (there && j < (kv_len(c, (int)(bh / c.heads)) + KB - 1) / KB)
        for (int r = first; r < rows; r += width) {
            const float lr = row_lse[bh * rows + r];
            // a row that sees nothing adds nothing
            if (lr != -INFINITY) sum += (double)__builtin_amdgcn_exp2f(block_lse[(bh * (c.blocks + 1) + j) * rows + r] - lr);
        }
    for (int o = min(width, 64) / 2; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (width > 64) {
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        const int w0 = threadIdx.x / width * (width / 64);
        sum = s_sum[w0] + s_sum[w0 + 1];
        if (width == 256) sum += s_sum[2] + s_sum[3];
    }
    if (there && first == 0) mass_out[at] = (mass_in ? mass_in[at] : 0.f) + (float)sum;
}

// ------------------------------------------------------------------------------------------------
// Selection of blocks.  score(token, head, block) = largest over the group's query heads of
//     key scale * sum_d max(q_d lo_d, q_d hi_d)  =  key scale * ( <max(q, 0), hi> + <min(q, 0), lo> ),
// which no logit of the block exceeds (before the softmax scale).  k_kv_score takes it on the matrix cores: products of a query's
// element and a code are exact in float32, D of them are not zero, and their float32 additions, rounded or truncated, are off by at most
// D 2^-23 of the sum of the terms' sizes, a second product of the same shape.  k_kv_pick takes the choice from these scores and bounds, and evaluates
// the blocks that they leave open in float64, where products of at most 15 bits add up to the same sum in any order
// unless a query's elements differ by more than 2^20 in size.  Chains of dependent loads and counts bound both: 13 and 14 us for 256 rows of up to 512
// blocks, 16 and 34 for 8 rows of 15 625 (a row's keys on one compute unit), 30 and 29 for 8000 rows of 256.
// ------------------------------------------------------------------------------------------------
struct KvSelectArgs {
    KvView c;
    const uint16_t *q;
    int64_t qs[3];
    const int32_t *counts;
    uint64_t *scores;  // [b][n][h][blocks]: score and bound on its error, a float each; a bound below zero: a block that is not there
    int32_t *lists;
    int n, g, w, sink, recent;
    int gp, tokens;  // columns of a token (its heads, the last one repeated up to a power of two), tokens of a tile of 16 columns
    int tiles, turns;  // tiles of a sequence's tokens, tiles that a wave goes through
};

__device__ __forceinline__ uint64_t key_of(double x)
{
    if (x != x) return 1;  // not a number: after everything else
    const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ double code_value(uint32_t u)
{
    const f32x2 f = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false);
    return (double)f[0];
}

__device__ __forceinline__ uint32_t positive16(uint32_t w)  // both halves: the number if its sign is plus, else 0
{
    const uint32_t neg = (w >> 15 & 0x00010001u) * 0xFFFFu;
    return w & ~neg;
}

// A wave takes 16 blocks (rows of the product) and goes through tiles of 16 (token, head) columns.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_kv_score(KvSelectArgs a)
{
    constexpr int KS = D / 32, WIDE = D / 64, ODD = D % 64 / 32;
    const int H = a.c.heads, lane = threadIdx.x & 63, x = lane & 15, hq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunks = (a.c.blocks + 63) / 64, turns = (a.tiles + a.turns - 1) / a.turns;
    const int h = blockIdx.x % H, turn = blockIdx.x / H % turns, chunk = blockIdx.x / H / turns % chunks, b = blockIdx.x / H / turns / chunks;
    const int64_t bh = (int64_t)b * H + h;
    const int len = kv_len(a.c, b), count = kv_count(a.counts, b, a.n);
    const int j0 = (chunk * 4 + wave) * 16;
    const int last = min(count, (turn + 1) * a.turns * a.tokens);  // tokens from there on see no less than the others
    if (last <= turn * a.turns * a.tokens || j0 >= min(max(0, len - count + last) / KB, a.c.blocks)) return;
    const int page = kv_page(a.c, bh, j0 + x);
    uint4 edge[2][KS];  // lo, hi
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint8_t *p = a.c.bounds + ((int64_t)max(page, 0) * 2 + e) * D;
#pragma unroll
        for (int s = 0; s < WIDE; ++s) {
            const uint4 w = *reinterpret_cast<const uint4 *>(p + 64 * s + 16 * hq);
            edge[e][2 * s] = __builtin_bit_cast(uint4, bring8<T>(w.x, w.y, 1.f));
            edge[e][2 * s + 1] = __builtin_bit_cast(uint4, bring8<T>(w.z, w.w, 1.f));
        }
        if (ODD) {
            const uint2 w = *reinterpret_cast<const uint2 *>(p + 64 * WIDE + 8 * hq);
            edge[e][KS - 1] = __builtin_bit_cast(uint4, bring8<T>(w.x, w.y, 1.f));
        }
    }
    auto sizes = [](uint4 w) {
        constexpr uint32_t mask = 0x7FFF7FFFu;
        return __builtin_bit_cast(typename T::x8, make_uint4(w.x & mask, w.y & mask, w.z & mask, w.w & mask));
    };
    const float own = page >= 0 ? a.c.scales[(int64_t)page * 2] : -1.f;
    float scale[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) scale[i] = __shfl(own, 4 * hq + i);

    for (int tile = turn * a.turns; tile < min(a.tiles, (turn + 1) * a.turns); ++tile) {
        const int token = tile * a.tokens + x / a.gp;
        const bool live = x / a.gp < a.tokens && token < count;
        f32x4 best = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        f32x4 size = {0.f, 0.f, 0.f, 0.f};  // largest sum of the terms' sizes
        bool odd = false;  // not a number anywhere
        for (int g0 = 0; g0 < a.g; g0 += 16) {
            const uint16_t *qp = a.q + b * a.qs[0] + (live ? token : 0) * a.qs[1] + ((int64_t)h * a.g + min(a.g - 1, g0 + x % a.gp)) * a.qs[2];
            f32x4 s = {0.f, 0.f, 0.f, 0.f}, terms = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = ks < 2 * WIDE ? 64 * (ks / 2) + 16 * hq + 8 * (ks % 2) : 64 * WIDE + 8 * hq;
                uint4 w = make_uint4(0, 0, 0, 0);
                if (live) w = *reinterpret_cast<const uint4 *>(qp + d);
                uint4 p;
                p.x = positive16(w.x);
                p.y = positive16(w.y);
                p.z = positive16(w.z);
                p.w = positive16(w.w);
                s = T::mfma(__builtin_bit_cast(typename T::x8, edge[1][ks]), __builtin_bit_cast(typename T::x8, p), s);
                terms = T::mfma(sizes(edge[1][ks]), __builtin_bit_cast(typename T::x8, p), terms);
                p.x ^= w.x;
                p.y ^= w.y;
                p.z ^= w.z;
                p.w ^= w.w;
                s = T::mfma(__builtin_bit_cast(typename T::x8, edge[0][ks]), __builtin_bit_cast(typename T::x8, p), s);
                terms = T::mfma(sizes(edge[0][ks]), sizes(p), terms);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                odd = odd || s[i] != s[i] || terms[i] != terms[i];
                best[i] = fmaxf(best[i], s[i]);
                size[i] = fmaxf(size[i], terms[i]);
            }
        }
        for (int o = a.gp / 2; o; o >>= 1) {
            odd = __shfl_xor((int)odd, o) || odd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                best[i] = fmaxf(best[i], __shfl_xor(best[i], o));
                size[i] = fmaxf(size[i], __shfl_xor(size[i], o));
            }
        }
        if (live && x % a.gp == 0) {
            uint64_t *to = a.scores + (((int64_t)b * a.n + token) * H + h) * a.c.blocks + j0 + 4 * hq;
            // some more than D: the sum of sizes is as far off, and score plus bound are rounded once more
            constexpr float off = (D + 16) * 1.1920929e-7f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 v = make_float2(best[i] * scale[i], off * size[i] * scale[i]);
                if (scale[i] < 0.f)
                    v = make_float2(0.f, -1.f);
                else if (odd || !(fabsf(v.x) < INFINITY) || !(v.y < INFINITY))
                    v = make_float2(0.f, INFINITY);  // whatever it is: k_kv_pick looks
                if (j0 + 4 * hq + i < a.c.blocks) to[i] = (uint64_t)__float_as_uint(v.y) << 32 | __float_as_uint(v.x);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// The largest of a wave's numbers, in all lanes
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_from(uint32_t x)
{
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max_from<0x111, 0xf>(x);  // one, two, four and eight lanes up within rows of 16
    x = max_from<0x112, 0xf>(x);
    x = max_from<0x114, 0xf>(x);
    x = max_from<0x118, 0xf>(x);
    x = max_from<0x142, 0xa>(x);  // a row's last lane into the next row, of the first half into the second
    x = max_from<0x143, 0xc>(x);
    return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t x)
{
    const uint32_t top = wave_max((uint32_t)(x >> 32));
    return (uint64_t)top << 32 | wave_max(x >> 32 == top ? (uint32_t)x : 0u);
}

// The `w` largest of `n` keys that are not zero, ties to the lower index.  WAVES waves take one row together; a wave holds up to 64 KPT
// consecutive keys in registers.  The w-th largest key is found by counting, with ballots, how many keys reach a number between two
// bounds; where it would lie among evenly spread keys is tried first.  The walk ends once exactly w keys reach a number, or no more than 64
// lie between the bounds (some four counts for scores, two for a bit at most): those are ranked against one another.  Rows longer
// than the registers read their keys again for every count (KPT = 0).
// ------------------------------------------------------------------------------------------------
template <typename U, int WAVES, int KPT>
struct Pick {
    static constexpr int KEYS = KPT ? KPT : 1;
    U keys[KEYS];
    U cut = 0;  // chosen: keys above it, and the first `ties` of those that equal it
    int ties = 0;
    int n, from;       // keys of the row; first of this wave's
    int span;          // keys of a wave, a multiple of 64

    static __device__ __forceinline__ int wave() { return WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    static __device__ __forceinline__ int lane() { return threadIdx.x & 63; }

    template <typename Key>
    __device__ __forceinline__ U at(int i, Key key) const
    {
        if (KPT) return keys[i];
        const int j = from + 64 * i + lane();
        return j < n ? key(j) : 0;
    }

    // keys that reach x, over all waves
    template <typename Key>
    __device__ __forceinline__ int reach(U x, Key key, int (&s_sum)[2][WAVES], int turn) const
    {
        int c = 0;
        if constexpr (KPT >= 8) {  // a lane counts its own keys (those past the row are 0), then the lanes' counts are added bit by bit
            static_assert(KPT % 4 == 0 && KPT < 32, "in groups of four, counts of five bits");
            int mine = 0;
#pragma unroll
            for (int i = 0; i < KPT; i += 4)
                if (from + 64 * i < n)
#pragma unroll
                    for (int y = 0; y < 4; ++y) mine += keys[i + y] >= x;
#pragma unroll
            for (int y = 0; y < 5; ++y) c += __popcll(__ballot(mine >> y & 1)) << y;
        } else if constexpr (KPT > 0) {
#pragma unroll
            for (int i = 0; i < KPT; ++i)
                if (from + 64 * i < n) c += __popcll(__ballot(keys[i] >= x));
        } else {
            for (int k = 0; k < span && from + k < n; k += 64) c += __popcll(__ballot(at(k / 64, key) >= x));
        }
        if (WAVES == 1) return c;
        if (lane() == 0) s_sum[turn][wave()] = c;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) all += s_sum[turn][i];
        return __builtin_amdgcn_readfirstlane(all);
    }

    // a row of n keys; key number i of this lane is the row's place(i)
    __device__ __forceinline__ void row(int n_)
    {
        n = n_;
        span = KPT ? 64 * KPT : (n + 64 * WAVES - 1) / (64 * WAVES) * 64;
        from = wave() * span;
    }
    __device__ __forceinline__ int place(int i) const { return from + 64 * i + lane(); }
    template <typename Key>
    __device__ __forceinline__ void load(int n_, Key key)
    {
        row(n_);
#pragma unroll
        for (int i = 0; i < KEYS; ++i) keys[i] = KPT && place(i) < n ? key(place(i)) : 0;
    }

    static __device__ __forceinline__ uint32_t of_lane(uint32_t x, int l) { return __builtin_amdgcn_readlane(x, l); }
    static __device__ __forceinline__ uint64_t of_lane(uint64_t x, int l)
    {
        return (uint64_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, l);
    }

    // The w-th largest of the up to 64 keys in [l, r), `many` of them
    __device__ __forceinline__ void rank(U l, U r, int w, int many)
    {
        __shared__ U s_few[WAVES == 1 ? 4 : 1][64];
        __shared__ int s_count;
        U *few = s_few[WAVES == 1 ? threadIdx.x >> 6 : 0];
        int c = 0;
        uint64_t in[KEYS];
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            in[i] = __ballot(keys[i] >= l && keys[i] < r);
            c += __popcll(in[i]);
        }
        if (WAVES > 1) {
            if (threadIdx.x == 0) s_count = 0;
            __syncthreads();
            int at = 0;
            if (c > 0 && lane() == 0) at = atomicAdd(&s_count, c);
            c = __builtin_amdgcn_readfirstlane(at);
        } else {
            c = 0;
        }
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int at = c + __popcll(in[i] & ((1ull << lane()) - 1));
            if (in[i] >> lane() & 1) few[at & 63] = keys[i];
            c += __popcll(in[i]);
        }
        if (WAVES > 1) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        const U own = lane() < many ? few[lane()] : 0;
        int above = 0, same = 0;
        for (int z = 0; z < many; ++z) {
            const U other = of_lane(own, z);
            above += other > own;
            same += other == own;
        }
        const uint64_t hit = __ballot(lane() < many && above < w && above + same >= w);
        const int at = __ffsll((unsigned long long)hit) - 1;
        cut = of_lane(own, at);
        ties = w - __builtin_amdgcn_readlane(above, at);
    }

    // after the keys are there; turn: the buffer of the row's last count
    template <typename Key>
    __device__ __forceinline__ void find(int w, Key key, int (&s_sum)[2][WAVES], int &turn)
    {
        int cl = reach(1, key, s_sum, turn ^= 1);
        if (cl <= w) return;  // no more than asked for: all of them
        // more than w keys reach l, fewer than w reach r
        const U all = (U)~(U)0;
        int cr = reach(all, key, s_sum, turn ^= 1);  // those that are always chosen
        if (cr >= w) {
            cut = all;
            ties = w;
            return;
        }
        U l = all, r = 0;  // smallest and largest of the others
        auto ends = [&](U k) {
            if (k != 0 && k != all) {
                l = k < l ? k : l;
                r = k > r ? k : r;
            }
        };
        if constexpr (KPT > 0) {
#pragma unroll
            for (int i = 0; i < KPT; ++i) ends(keys[i]);
        } else {
            for (int k = 0; k < span && from + k < n; k += 64) ends(at(k / 64, key));
        }
        l = ~wave_max((U)~l);
        r = wave_max(r);
        if (WAVES > 1) {
            __shared__ U s_ends[2][WAVES];
            if (lane() == 0) {
                s_ends[0][wave()] = l;
                s_ends[1][wave()] = r;
            }
            __syncthreads();
            for (int i = 0; i < WAVES; ++i) {
                l = s_ends[0][i] < l ? s_ends[0][i] : l;
                r = s_ends[1][i] > r ? s_ends[1][i] : r;
            }
            l = of_lane(l, 0);
            r = of_lane(r, 0);
        }
        ++r;
        for (int turns = 0; r - l > 1; ++turns) {
            if constexpr (KPT > 0) {
                if (cl - cr <= 64) {
                    rank(l, r, w - cr, cl - cr);
                    return;
                }
            }
            // where the w-th key would lie if they were spread evenly, and the middle, in turn
            const U gap = r - l;
            U step = gap / 2;
            if (turns % 2 == 0) step = (U)((float)gap * ((cl - w + 0.5f) / (float)(cl - cr)));
            step = step < 1 ? 1 : step > gap - 1 ? gap - 1 : step;
            const U x = of_lane((U)(l + step), 0);
            const int c = reach(x, key, s_sum, turn ^= 1);
            if (c == w) {
                cut = x - 1;
                return;
            }
            if (c > w) {
                l = x;
                cl = c;
            } else {
                r = x;
                cr = c;
            }
        }
        // l is the w-th largest key, and more than one equals it
        cut = l;
        ties = w - cr;
    }

    // Calls put(j, place, chosen) for every j < n (ALL) or every chosen one, place = how many of its kind come before it; returns the
    // number of chosen ones.
    template <bool ALL, typename Key, typename Put>
    __device__ __forceinline__ int walk(Key key, Put put) const
    {
        __shared__ int s_kind[2][WAVES];
        int over = 0, same = 0, all = 0;
        if (WAVES > 1) {
            if constexpr (KPT > 0) {
#pragma unroll
                for (int i = 0; i < KPT; ++i)
                    if (from + 64 * i < n) {
                        over += __popcll(__ballot(keys[i] > cut));
                        same += __popcll(__ballot(keys[i] != 0 && keys[i] == cut));
                    }
            } else {
                for (int k = 0; k < span && from + k < n; k += 64) {
                    const U v = at(k / 64, key);
                    over += __popcll(__ballot(v > cut));
                    same += __popcll(__ballot(v != 0 && v == cut));
                }
            }
            if (lane() == 0) {
                s_kind[0][wave()] = over;
                s_kind[1][wave()] = same;
            }
            __syncthreads();
            over = same = 0;
            for (int i = 0; i < wave(); ++i) {
                over += s_kind[0][i];
                same += s_kind[1][i];
            }
            int so = 0, ss = 0;
            for (int i = 0; i < WAVES; ++i) {
                so += s_kind[0][i];
                ss += s_kind[1][i];
            }
            all = so + min(ss, ties);
        }
        const uint64_t below = (1ull << lane()) - 1;
        auto round = [&](int k, U v) {
            const int j = from + k + lane();
            const uint64_t bo = __ballot(v > cut), bs = __ballot(v != 0 && v == cut);
            if (!ALL && (bo | bs) == 0) return;
            const int os = same + __popcll(bs & below);
            const bool take = v > cut || (v != 0 && v == cut && os < ties);
            const int place = over + __popcll(bo & below) + min(os, ties);
            if (j < n) put(j, take ? place : j - place, take);
            over += __popcll(bo);
            same += __popcll(bs);
        };
        if constexpr (KPT > 0) {
#pragma unroll
            for (int i = 0; i < KPT; ++i)
                if (from + 64 * i < n) round(64 * i, keys[i]);
        } else {
            for (int k = 0; k < span && from + k < n; k += 64) round(k, at(k / 64, key));
        }
        return WAVES == 1 ? over + min(same, ties) : all;
    }
};

// The score of one block in float64, by 16 lanes together: lane `part` of them has D / 16 dimensions in a row.
template <typename T, int D>
__device__ __forceinline__ double exact_score(const KvSelectArgs &a, const uint16_t *q, int page, int part)
{
    constexpr int N = D / 16;
    const uint8_t *lo = a.c.bounds + (int64_t)page * (2 * D) + part * N, *hi = lo + D;
    uint32_t codes[N];  // lo, and hi 16 bits higher
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const uint32_t x = reinterpret_cast<const uint16_t *>(lo)[i], y = reinterpret_cast<const uint16_t *>(hi)[i];
        codes[2 * i] = (x & 0xFF) | (y & 0xFF) << 16;
        codes[2 * i + 1] = x >> 8 | (y >> 8) << 16;
    }
    const float scale = a.c.scales[(int64_t)page * 2];
    double best = -INFINITY;
    bool odd = false;
    for (int h0 = 0; h0 < a.g; h0 += 4) {  // four heads at a time, the last one again where there are fewer
        uint32_t w[4][N / 2];
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int i = 0; i < N / 2; ++i) w[y][i] = reinterpret_cast<const uint32_t *>(q + min(h0 + y, a.g - 1) * a.qs[2] + part * N)[i];
        double sum[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            sum[y] = 0;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float x0 = T::wide((uint16_t)w[y][i]), x1 = T::wide((uint16_t)(w[y][i] >> 16));
                sum[y] += (double)x0 * code_value(x0 > 0.f ? codes[2 * i] >> 16 : codes[2 * i]);
                sum[y] += (double)x1 * code_value(x1 > 0.f ? codes[2 * i + 1] >> 16 : codes[2 * i + 1]);
            }
        }
        for (int o = 8; o; o >>= 1)
#pragma unroll
            for (int y = 0; y < 4; ++y) sum[y] += __shfl_xor(sum[y], o);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            odd = odd || sum[y] != sum[y];
            best = fmax(best, sum[y]);
        }
    }
    return odd ? NAN : best * (double)scale;
}

// ROWS rows to a workgroup, WAVES waves to a row (one of the two is 1).  From the scores' intervals: no block below the w-th largest
// lower end can be chosen, and any whose lower end lies above the (w + 1)-th largest upper end is; the rest are
// evaluated, as a rule none or two.
template <typename T, int D, int ROWS, int WAVES, int KPT>
__global__ __launch_bounds__(64 * ROWS * WAVES) void k_kv_pick(KvSelectArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);  // (sequence, token, head)
    const int H = a.c.heads, b = (int)(row / H / a.n), i = (int)(row / H % a.n), h = (int)(row % H);
    if (b >= a.c.batch) return;
    const int len = kv_len(a.c, b), count = kv_count(a.counts, b, a.n);
    const int whole = __builtin_amdgcn_readfirstlane(i < count ? min(max(0, len - count + i + 1) / KB, a.c.blocks) : 0);
    __shared__ int s_sum[2][WAVES];
    int turn = 0;
    uint64_t *scores = a.scores + row * a.c.blocks;
    int32_t *out = a.lists + row * a.w;
    auto forced = [&](int j) { return j < a.sink || j >= whole - a.recent; };
    auto low_of = [&](int j, uint64_t u) -> uint32_t {
        const float v = __uint_as_float((uint32_t)u), off = __uint_as_float((uint32_t)(u >> 32));
        if (off < 0.f) return 0;
        return forced(j) ? ~0u : off == INFINITY ? 1 : key_of(v - off);
    };
    auto high_of = [&](int j, uint64_t u) -> uint32_t {
        const float v = __uint_as_float((uint32_t)u), off = __uint_as_float((uint32_t)(u >> 32));
        if (off < 0.f) return 0;
        return forced(j) ? ~0u : off == INFINITY ? ~0u - 1 : key_of(v + off);
    };
    auto low = [&](int j) { return low_of(j, scores[j]); };
    auto high = [&](int j) { return high_of(j, scores[j]); };
    auto put = [&](int j, int place, bool take) {
        if (take) out[place] = j;
    };
    const int lane = threadIdx.x & 63, wave = Pick<uint32_t, WAVES, KPT>::wave();
    const uint16_t *q = a.q + b * a.qs[0] + i * a.qs[1] + (int64_t)h * a.g * a.qs[2];
    int got = -1;
    Pick<uint32_t, WAVES, KPT> lower, upper;
    lower.row(whole);
    upper.row(whole);
    float widest = 0.f;  // interval of those that are not forced
    if constexpr (KPT > 0) {
        uint64_t raw[KPT];  // all on their way together
#pragma unroll
        for (int y = 0; y < KPT; ++y) raw[y] = scores[min(lower.place(y), a.c.blocks - 1)];
#pragma unroll
        for (int y = 0; y < KPT; ++y) {
            const int j = lower.place(y);
            lower.keys[y] = j < whole ? low_of(j, raw[y]) : 0;
            upper.keys[y] = j < whole ? high_of(j, raw[y]) : 0;
            if (j < whole && !forced(j)) widest = fmaxf(widest, __uint_as_float((uint32_t)(raw[y] >> 32)));
        }
    }
    lower.find(a.w, low, s_sum, turn);
    // w blocks reach `least` with their lower ends: one whose upper end does not cannot be chosen
    const uint32_t least = lower.ties ? lower.cut : lower.cut + 1;
    if (upper.reach(least, high, s_sum, turn ^= 1) <= a.w) {
        upper.cut = least - 1;
        got = upper.template walk<false>(high, put);
    } else if constexpr (KPT > 0) {
        // No more than w blocks have a lower end above `least` (or w have one from there on), so no more than w an upper end that lies
        // by the widest interval above it: a block whose lower end does is chosen.  The few between, up to 64 of a wave, are
        // evaluated and ranked against one another.
        __shared__ float s_widest[WAVES];
        __shared__ uint64_t s_open[ROWS * WAVES][64];
        __shared__ int s_found[2][WAVES];
        int *list = reinterpret_cast<int *>(s_open[threadIdx.x >> 6]);  // the wave's open blocks
        widest = __uint_as_float(wave_max(__float_as_uint(widest)));  // not negative: ordered like its bits
        if (WAVES > 1) {
            if (lane == 0) s_widest[wave] = widest;
            __syncthreads();
            for (int y = 0; y < WAVES; ++y) widest = fmaxf(widest, s_widest[y]);
        }
        const uint32_t bits = least >> 31 ? least & 0x7FFFFFFFu : ~least;  // the number whose key `least` is
        const float edge = __uint_as_float(bits) + 2.5f * widest;
        const bool firm = least < 0xFF800000u && least > 0x007FFFFFu && edge < INFINITY;  // a finite number, plus a finite one
        const uint32_t sure = firm ? key_of(edge) : ~0u;
        int sures = 0, opens = 0;
#pragma unroll
        for (int y = 0; y < KPT; ++y) {
            const bool chosen = upper.keys[y] >= least && upper.keys[y] != 0 && (lower.keys[y] > sure || lower.keys[y] == ~0u);
            const uint64_t open = __ballot(upper.keys[y] >= least && !chosen);
            const int nth = opens + __popcll(open & ((1ull << lane) - 1));
            if ((open >> lane & 1) && nth < 64) list[nth] = lower.from + 64 * y + lane;
            // from here on: 0, 1 chosen, 2 open
            upper.keys[y] = chosen ? 1 : open >> lane & 1 ? 2 : 0;
            sures += __popcll(__ballot(chosen));
            opens += __popcll(open);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        bool fits = opens <= 64;
        int need = a.w - sures, ahead = 0;
        uint64_t own = 0;  // key of the wave's lane-th open block
        if (fits) {
            const int mine = lane < opens ? list[lane] : -1;
            for (int z = 0; z < opens; z += 4) {  // four blocks at a time, 16 lanes to each
                const int j = __shfl(mine, min(z + lane / 16, 63));
                const int page = j >= 0 && z + lane / 16 < opens ? kv_page(a.c, (int64_t)b * H + h, j) : 0;
                const uint64_t key = key_of(exact_score<T, D>(a, q, max(page, 0), lane & 15));
                const uint64_t here = __shfl(key, (lane - z) * 16 & 63);
                if (lane >= z && lane < z + 4) own = here;
            }
        }
        if (WAVES > 1) {
            __syncthreads();
            if (lane == 0) {
                s_found[0][wave] = sures;
                s_found[1][wave] = opens;
            }
            if (lane < opens) s_open[wave][lane] = own;
            __syncthreads();
            need = a.w;
            for (int y = 0; y < WAVES; ++y) {
                need -= s_found[0][y];
                fits = fits && s_found[1][y] <= 64;
            }
            if (fits && opens > 0)
                for (int y = 0; y < WAVES; ++y) {
                    const int found = __builtin_amdgcn_readfirstlane(s_found[1][y]);
                    if (found == 0) continue;
                    const uint64_t others = s_open[y][lane];
                    for (int z = 0; z < found; ++z) {
                        const uint64_t other = Pick<uint64_t, WAVES, KPT>::of_lane(others, z);
                        ahead += other > own || (other == own && (y < wave || (y == wave && z < lane)));
                    }
                }
        } else if (fits) {
            for (int z = 0; z < opens; ++z) {
                const uint64_t other = Pick<uint64_t, WAVES, KPT>::of_lane(own, z);
                ahead += other > own || (other == own && z < lane);
            }
        }
        if (fits) {
            const uint64_t wins = __ballot(lane < opens && ahead < need);  // bit n: the wave's n-th open block
            int before = 0;
#pragma unroll
            for (int y = 0; y < KPT; ++y) {
                const uint64_t open = __ballot(upper.keys[y] == 2);
                const int nth = before + __popcll(open & ((1ull << lane) - 1));
                if (upper.keys[y] == 2) upper.keys[y] = wins >> (nth & 63) & 1;
                before += __popcll(open);
            }
            upper.cut = 0;
            upper.ties = 0;
            got = upper.template walk<false>(high, put);
        }
    }
    if (got < 0) {  // many blocks alike: the exact scores of all that may be chosen, in the place of their bounds
        for (int k = 0; k < lower.span && lower.from + k < whole; k += 64) {
            const int j = lower.from + k + lane;
            uint64_t key = 0;
            if (j < whole) key = high(j) < least ? 0 : forced(j) ? ~0ull : 2;
            if (key == 2 && scores[j] >> 32 == 0) key = key_of((double)__uint_as_float((uint32_t)scores[j]));  // a query of zeros
            uint64_t open = __ballot(key == 2);
            while (open) {  // four blocks at a time, 16 lanes to each
                int bit[4], mine = -1;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    bit[y] = __ffsll((unsigned long long)open) - 1;  // -1: none left
                    if (lane / 16 == y) mine = bit[y];
                    open &= open - 1;
                }
                const int page = mine >= 0 ? kv_page(a.c, (int64_t)b * H + h, lower.from + k + mine) : 0;
                const uint64_t score = key_of(exact_score<T, D>(a, q, max(page, 0), lane & 15));
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const uint64_t one = __shfl(score, 16 * y);
                    if (lane == bit[y]) key = one;
                }
            }
            if (j < whole) scores[j] = key;
        }
        auto key = [&](int j) { return scores[j]; };
        Pick<uint64_t, WAVES, KPT> last;
        last.load(whole, key);
        last.find(a.w, key, s_sum, turn);
        got = last.template walk<false>(key, put);
    }
    for (int j = got + threadIdx.x % (64 * WAVES); j < a.w; j += 64 * WAVES) out[j] = -1;
}

// ------------------------------------------------------------------------------------------------
// Eviction: of every (sequence, head) with more than `budget` blocks the first `sink`, the last `recent` and those of
// the others with the largest weight stay, in their order.  Lengths that are changed in place change in a launch of their own
// (k_kv_evict_lens), since every workgroup here reads them; into other arrays (lens_out not null) they are written here.
// Bound by latency: 7 us for 128 rows of 128 blocks, 10 for 16 rows of 313.
// ------------------------------------------------------------------------------------------------
// Everything is read before anything is written, since the outputs may be the inputs; with more blocks than the registers hold a launch
// of one workgroup per row has to write apart from what it reads (KPT = 0: `table_out` and `mass_out` are not the inputs).
template <int WAVES, int KPT>
__global__ __launch_bounds__(64 * WAVES) void k_kv_evict(KvView c, const float *mass, int budget, int sink, int recent, int32_t *table_out, float *mass_out,
                                                         int32_t *freed, int32_t *lens_out, int32_t *evicted_out)
{
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / c.heads), tid = threadIdx.x;
    const int nb = __builtin_amdgcn_readfirstlane(min(kv_len(c, b) / KB, c.blocks)), stay = min(nb, budget);
    const int32_t *table = c.table + bh * c.blocks;
    mass += bh * c.blocks;
    table_out += bh * c.blocks;
    mass_out += bh * c.blocks;
    freed += bh * c.blocks;
    const float open = nb < c.blocks ? mass[nb] : 0.f;  // the open block's weight moves along
    if (lens_out && bh % c.heads == 0 && tid == 0) {
        const int len = kv_len(c, b), gone = max(0, len / KB - budget);
        lens_out[b] = len - gone * KB;
        evicted_out[b] = c.evicted[b] + gone;
    }
    auto key = [&](int j) -> uint64_t {
        if (j < sink || j >= nb - recent) return ~0ull;
        return key_of((double)mass[j]);
    };
    __shared__ int s_sum[2][WAVES];
    int turn = 0;
    Pick<uint64_t, WAVES, KPT> pick;
    int32_t page[KPT ? KPT : 1];
    float weight[KPT ? KPT : 1];
    pick.row(nb);
    if constexpr (KPT > 0) {  // all on their way together
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int j = min(pick.place(i), c.blocks - 1);
            page[i] = table[j];
            weight[i] = mass[j];
        }
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int j = pick.place(i);
            pick.keys[i] = j >= nb ? 0 : j < sink || j >= nb - recent ? ~0ull : key_of((double)weight[i]);
        }
    }
    pick.find(budget, key, s_sum, turn);
    if (KPT) __syncthreads();
    pick.template walk<true>(key, [&](int j, int place, bool take) {
        int32_t p;
        float w;
        if (KPT) {
            p = 0;
            w = 0.f;
#pragma unroll
            for (int i = 0; i < KPT; ++i)
                if (j == pick.place(i)) {
                    p = page[i];
                    w = weight[i];
                }
        } else {
            p = table[j];
            w = mass[j];
        }
        if (take) {
            table_out[place] = p;
            mass_out[place] = w;
        } else {
            freed[place] = p;
        }
    });
    __syncthreads();
    for (int j = tid; j < c.blocks; j += 64 * WAVES) {
        if (j >= stay) {
            table_out[j] = -1;
            mass_out[j] = j == stay && nb < c.blocks ? open : 0.f;
        }
        if (j >= nb - stay) freed[j] = -1;
    }
}

__global__ __launch_bounds__(64) void k_kv_evict_lens(KvView c, int budget, int32_t *lens_out, int32_t *evicted_out)
{
    const int b = blockIdx.x * 64 + threadIdx.x;
    if (b >= c.batch) return;
    const int len = kv_len(c, b), gone = max(0, len / KB - budget);
    lens_out[b] = len - gone * KB;
    evicted_out[b] = c.evicted[b] + gone;
}
