// What the kernels of the attention cache and of prompts' attention share: the 16-bit types with their matrix products, sizes of
// numbers, what softmax weights are taken against, and the numbering of packed sequences' tiles.  Included inside an anonymous namespace.
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
    // As large as float32's numbers: sums of weighted values may not be finite where their mean is one of the type's (k_prompt).
    static constexpr bool WIDE = true;
    static constexpr float MOST = 0x1.FEp127f;
    static __device__ __forceinline__ void hold(float &) {}
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
    static constexpr bool WIDE = false;
    static constexpr float MOST = 65504.f;
    // From here on what is rounded past the type's largest number becomes that one, infinities stay (FP16_OVFL, bit 23 of MODE).  What comes of f
    // is worked out behind it.  No matrix product may follow: with it a query that is not a number gave ordinary results.
    static __device__ __forceinline__ void hold(float &f)
    {
        __builtin_amdgcn_s_setreg(1 | 23 << 6, 1);
        asm volatile("" : "+v"(f));
    }
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

// Sequences that lie packed: sequence b has the tokens [starts[b], starts[b + 1]) of `tokens`; starts ascend.
struct Packed {
    const int32_t *starts;
    int tokens, batch;
};
// first token of sequence b (b = batch: the end of the last), within the tokens that there are
__device__ __forceinline__ int packed_start(const Packed &p, int b) { return min(max(p.starts[b], 0), p.tokens); }

// All sequences share one numbering of tiles of ROWS rows, g rows to a token, that needs no counting: sequence b's tiles begin at number
// floor(starts[b] g / ROWS) + b, since it has at most floor(n g / ROWS) + 1 of them.  Where starts descend, these overlap and a number may be another
// sequence's: tiles are left out, but none is given to two numbers, and none is outside of its sequence.
template <int ROWS>
__device__ __forceinline__ int packed_base(const Packed &p, int b, int g) { return (int)((int64_t)packed_start(p, b) * g / ROWS) + b; }
// The last sequence whose tiles begin at or before number `find`, or 0, by a search of 64 places at a time.  Every lane of the wave calls it.
template <int ROWS>
__device__ __forceinline__ int packed_of_tile(const Packed &p, int g, int find)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, many = p.batch;  // it is one of [lo, lo + many)
    while (many > 1) {
        const int step = (many + 63) / 64, i = lane * step;
        const uint64_t before = __ballot(i < many && packed_base<ROWS>(p, min(lo + i, p.batch - 1), g) <= find);
        const int last = before ? 63 - __builtin_clzll(before) : 0;
        lo += last * step;
        many = min(step, many - last * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
