// Dropout's mask, computed wherever it is needed and stored nowhere.
//
// The bits come from Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011), a bijection of 128-bit counters under a 64-bit key.  The key is the caller's seed; the counter is (column / 8, row,
// offset), so every value of a matrix has bits of its own that depend on its place alone: not on strides, tiles or launches.  One
// counter gives 128 bits, 16 for each of eight neighbouring columns.  16 bits and not 32 because the multiplications are what
// such a kernel computes most: two per round and counter are 2.5 a value (32 bits: 5), which stay under the memory's time.
#pragma once
#include <cmath>

#include "pairs.cuh"

namespace scar {

struct DropRule {
    unsigned key[20];  // of the ten rounds, two each: operands from the kernel's parameters
    int on;          // something is dropped
    unsigned above;  // 65536 cut - 1: a value is kept if its 16 bits, as the upper half of a word, are above this
    float scale;     // of what is kept
    unsigned long long offset;
    const unsigned long long *d_offset;  // added to it, or nullptr
    __device__ __forceinline__ unsigned long long at() const { return offset + (d_offset ? *d_offset : 0ull); }
};

// SCAR_OK, or what is wrong with the caller's rule (nullptr: nothing is dropped).  The probability is taken to the nearest
// multiple of 2^-16 that is neither 0 nor 1 unless it is 0 or 1 itself; the scale is of the one taken, so means are kept.
inline int make_rule(const scar_dropout *d, DropRule *out) {
    *out = DropRule{};
    out->scale = 1.f;
    if (!d) return SCAR_OK;
    if (!(d->p >= 0. && d->p <= 1.) || (uintptr_t)d->d_offset % 8) return SCAR_ERR_INVALID_ARG;
    unsigned cut = (unsigned)std::floor(d->p * 65536. + 0.5);
    if (d->p > 0. && cut == 0) cut = 1;
    if (d->p < 1. && cut == 65536) cut = 65535;
    for (unsigned i = 0; i < 10; ++i) {
        out->key[2 * i] = (unsigned)d->seed + i * 0x9E3779B9u;
        out->key[2 * i + 1] = (unsigned)(d->seed >> 32) + i * 0xBB67AE85u;
    }
    out->on = cut != 0;
    out->above = cut * 65536u - 1u;
    out->scale = cut == 65536 ? 0.f : 65536.f / (float)(65536 - cut);
    out->offset = d->offset;
    out->d_offset = reinterpret_cast<const unsigned long long *>(d->d_offset);
    return SCAR_OK;
}

// The 16-bit values of columns 8 * block .. 8 * block + 7 of a row, two per word, the lower column in the lower half.
__device__ __forceinline__ uint4 mask_bits(const DropRule &r, unsigned long long offset, unsigned row, unsigned block) {
    uint4 c = make_uint4(block, row, (unsigned)offset, (unsigned)(offset >> 32));
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long a = (unsigned long long)c.x * 0xD2511F53u, b = (unsigned long long)c.z * 0xCD9E8D57u;
        c = make_uint4((unsigned)(b >> 32) ^ c.y ^ r.key[2 * i], (unsigned)b, (unsigned)(a >> 32) ^ c.w ^ r.key[2 * i + 1], (unsigned)a);
    }
    return c;
}
__device__ __forceinline__ bool mask_keeps(const DropRule &r, const uint4 &bits, int j) {
    const unsigned w = j < 2 ? bits.x : j < 4 ? bits.y : j < 6 ? bits.z : bits.w;
    return !r.on || (j & 1 ? w : w << 16) > r.above;
}
// Eight neighbours as the mask leaves them: what is dropped is 0 whatever it was.
__device__ __forceinline__ void mask_apply(const DropRule &r, const uint4 &bits, float2 (&x)[4]) {
    const unsigned w[4] = {bits.x, bits.y, bits.z, bits.w};
    const float2 scale = both(r.scale);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 y = mul2(x[j], scale);
        x[j].x = (w[j] << 16) > r.above ? y.x : 0.f;
        x[j].y = w[j] > r.above ? y.y : 0.f;
    }
}
// Bit j of the result: column j is kept.
__device__ __forceinline__ unsigned mask_byte(const DropRule &r, const uint4 &bits) {
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m |= (unsigned)mask_keeps(r, bits, j) << j;
    return m;
}

}  // namespace scar
