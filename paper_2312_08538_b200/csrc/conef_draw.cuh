// Counter-based 16-bit variates for matrices: a word of the library's 64-bit hash serves four consecutive columns of
// a row, so a hash costs a quarter of an element, and nothing has to be stored: whoever has (seed, worker, tensor, step) has
// every number again.  16 bits: a probability is a multiple of 2^-16, a rounding is up with a probability off by 2^-17 at most.
#pragma once
#include "conef_hash.cuh"

namespace conef {

enum { kDrawDropout = 0, kDrawRounding = 1 };   // the two words of a group of four columns

__host__ __device__ __forceinline__ uint64_t draw_stream(uint64_t seed, int64_t worker, int64_t tensor, int64_t step)
{
    return stream_key(mix64(seed + (uint64_t)worker + 1u), (uint64_t)tensor, (uint64_t)step);
}
// the word of columns 4 g .. 4 g + 3 of a row, group = row * ceil(cols / 4) + g; column 4 g + i has bits 16 i to 16 i + 15
__device__ __forceinline__ uint64_t draw_word(uint64_t stream, uint64_t group, int which) { return h64(stream, 2u * group + (unsigned)which); }
__device__ __forceinline__ uint32_t draw_of(uint64_t word, uint32_t col) { return (uint32_t)(word >> (16u * (col & 3u))) & 0xFFFFu; }

// The same for runs of groups: the mixer's argument for group 0, to which a group adds kDrawStep
constexpr uint64_t kDrawStep = 2u * kGolden;
__host__ __device__ __forceinline__ uint64_t draw_base(uint64_t stream, int which) { return stream + kGolden * (uint64_t)(which + 1); }

// A dropout: an element is kept where its number is at least `off` (the probability in 65536ths, 0 to 65536)
struct Dropout {
    uint32_t off;
    float scale;     // 65536 / (65536 - off)
    uint32_t limit;  // (off << 16) - 1: what the number, as the upper half of a word, is compared with (off > 0)
    uint32_t all;    // ones where off is 0: everything is kept
};
// bits 0 to 3: whether the columns of a word are kept
__device__ __forceinline__ uint32_t dropout_kept(uint64_t word, const Dropout &d)
{
    const uint32_t lo = (uint32_t)word, hi = (uint32_t)(word >> 32);
    return ((lo << 16) > d.limit ? 1u : 0u) | (lo > d.limit ? 2u : 0u) | ((hi << 16) > d.limit ? 4u : 0u) | (hi > d.limit ? 8u : 0u);
}
inline Dropout dropout_of(double p)
{
    Dropout d;
    d.off = (uint32_t)__builtin_rint(p * 65536.0);
    d.scale = (float)(65536.0 / (d.off < 65536u ? 65536u - d.off : 1u));
    d.limit = (d.off << 16) - 1u;
    d.all = d.off ? 0u : 0xFFFFFFFFu;
    return d;
}

}  // namespace conef
