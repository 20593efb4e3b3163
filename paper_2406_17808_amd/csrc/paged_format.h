// The paged cache in 4 bits: its geometry, where its bytes sit and what they stand for.  Host and device: the same routines decide which byte a
// kernel touches and are run on the host over arrays of any content.
#pragma once

#include "internal.h"

namespace ckv {

// ------------------------------------------------------------------ geometry
struct PagedGeom {
    int Hq, Hkv, G, d;
    int page_size;          // tokens; a multiple of 32
    int groups;             // page_size / 32
    int group_bytes;
    int64_t n_pages;
    float scale;            // of the logits
    int window;             // 0: none
    uint8_t* pages;
    const double2* rope;    // null: keys are stored as they come
    int64_t rope_positions;
};

// The arrays are the caller's and are read when a kernel runs: the kernels rely on nothing in them (SeqView, paged_group).
struct PagedBatch {
    int n_seqs, n_tokens, max_new, max_length;
    const int32_t* lengths;
    const int32_t* offsets;
    const int32_t* table;
    int64_t table_stride;
};

constexpr int kGroupTokens = 32;
__host__ __device__ constexpr int paged_group_bytes(int d) { return (33 * d + 64 + 127) / 128 * 128; }

// ------------------------------------------------------------------ places
// One sequence of a batch, with everything that a caller's arrays may hold forced into the ranges the host knows.
struct SeqView {
    int len;      // tokens before the new ones: 0 .. max_length
    int first;    // row of the first new token: 0 .. n_tokens
    int n;        // new tokens: 0 .. min(max_new, n_tokens - first)
};
__host__ __device__ inline SeqView seq_view(const PagedBatch& b, int s)
{
    SeqView v;
    const int len = b.lengths[s], first = b.offsets[s], last = b.offsets[s + 1];
    v.len = len < 0 ? 0 : len > b.max_length ? b.max_length : len;
    v.first = first < 0 ? 0 : first > b.n_tokens ? b.n_tokens : first;
    const int end = last > b.n_tokens ? b.n_tokens : last;
    v.n = end <= v.first ? 0 : end - v.first > b.max_new ? b.max_new : end - v.first;
    return v;
}

// Number of the group of 32 tokens that holds position p of sequence s for KV head 0 (head h: + h * groups), or -1 where the position is behind
// max_length or the table, or the page does not exist.
__host__ __device__ inline int64_t paged_group(const PagedGeom& g, const PagedBatch& b, int s, int p)
{
    if (p < 0 || p >= b.max_length) return -1;
    const int slot = p / g.page_size;
    if (slot >= b.table_stride) return -1;
    const int page = b.table[(int64_t)s * b.table_stride + slot];
    if (page < 0 || page >= g.n_pages) return -1;
    return (int64_t)page * g.Hkv * g.groups + (p - slot * g.page_size) / kGroupTokens;
}

// Bytes inside a group, for token r (0 .. 31).  K codes of 32 channels are 16 contiguous bytes: what one lane of an MFMA takes
// as its part of the contraction, with one scale.  A byte of V holds two channels of ONE token, so that a token is written without reading its
// neighbours; the order of the bytes is that of the probabilities of 32 keys in the accumulators of S^T = K Q^T (keys 4q + b and
// 16 + 4q + b in a lane), so that V fragments are loaded as they are used.
__host__ __device__ inline int k_code_byte(int c, int r) { return (c >> 5) * 512 + r * 16 + ((c & 31) >> 1); }                  // channels c, c + 1 (c even)
__host__ __device__ inline int v_slot(int r) { return ((r >> 2) & 3) * 8 + (r >> 4) * 4 + (r & 3); }
__host__ __device__ inline int v_code_byte(int d, int u, int m, int r)                                                          // channels 32 u + m and 32 u + 16 + m
{
    return 16 * d + (u >> 1) * 1024 + ((r >> 2) & 3) * 256 + m * 16 + (u & 1) * 8 + (r >> 4) * 4 + (r & 3);
}
__host__ __device__ inline int k_exp_byte(int d, int block, int r) { return 32 * d + block * 32 + (r & 15) * 2 + (r >> 4); }
__host__ __device__ inline int v_scale_byte(int d, int r) { return 33 * d + v_slot(r) * 2; }

// ------------------------------------------------------------------ numbers
__host__ __device__ inline float f32_from_bits(uint32_t u)
{
    union { uint32_t u; float f; } c;
    c.u = u;
    return c.f;
}

// The value of a code (low four bits of x).
__host__ __device__ inline float fp4_value(uint32_t x)
{
    const uint32_t e = (x >> 1) & 3u, m = x & 1u;
    const float a = e == 0 ? 0.5f * (float)m : f32_from_bits(((e + 126u) << 23) | (m << 22));
    return x & 8u ? -a : a;
}

// The scale of a K block: 2^(byte - 127); 255 stands for NaN.
__host__ __device__ inline float k_scale(uint32_t byte) { return byte == 255u ? f32_from_bits(0x7FC00000u) : byte == 0u ? 0.f : f32_from_bits(byte << 23); }

// The code of y: the nearest value, ties to the even code, at most 6.  The borders 0.25 ... 5 have three bits.
template <typename F> __host__ __device__ inline uint32_t fp4_code(F y, F unit)
{
    const F a = y < (F)0 ? -y : y;
    const uint32_t code = (uint32_t)(a > (F)0.25 * unit) + (uint32_t)(a >= (F)0.75 * unit) + (uint32_t)(a > (F)1.25 * unit) +
                          (uint32_t)(a >= (F)1.75 * unit) + (uint32_t)(a > (F)2.5 * unit) + (uint32_t)(a >= (F)3.5 * unit) + (uint32_t)(a > (F)5 * unit);
    return code | (y < (F)0 ? 8u : 0u);
}

// |y| of a 64-bit number in 32 bits, for comparisons with numbers of at most 19 mantissa bits: the upper word, with the last bit set where the lower word
// is not zero.  Which side of such a number y lies on is kept.
__host__ __device__ inline uint32_t k_key(double y)
{
    union { double d; uint64_t u; } c;
    c.d = y;
    return ((uint32_t)(c.u >> 32) & 0x7FFFFFFFu) | ((uint32_t)c.u != 0u ? 1u : 0u);
}

// Byte of the smallest scale 2^e with top <= 7 * 2^e, top the largest key of a block; 0 for zeros, 255 where it is an infinity or NaN.
__host__ __device__ inline uint32_t k_exponent_of_key(uint32_t top)
{
    const int biased = (int)(top >> 20);
    if (biased == 0x7FF) return 255u;
    if (biased < 1023 - 400) return 0u;      // zero, or far below the smallest scale
    int e = biased - 1023 - 2 + ((top & 0xFFFFFu) > 0xC0000u ? 1 : 0);      // 1.m * 2^(biased - 1023); 1.75 * 4 = 7
    e = e < -126 ? -126 : e > 127 ? 127 : e;
    return (uint32_t)(e + 127);
}
__host__ __device__ inline uint32_t k_exponent(double top) { return k_exponent_of_key(k_key(top)); }

// The bits of a float next to |y| / scale of `byte`, on the same side of every number with few bits: rounding it to a code rounds y.  0 for the byte 255.
__host__ __device__ inline uint32_t k_scaled_bits(uint32_t key, uint32_t byte)
{
    const int d = (int)key - ((1023 - 127 + (int)byte - 127) << 20);      // exponents: of y / 2^(byte - 127), with a float's bias
    return byte == 255u || d < 0 ? 0u : (uint32_t)d << 3;
}

// Scale of a V row (bf16 bits): top / 6; 0 below 2^-100.  A NaN or infinity in the row gives NaN.
__host__ __device__ inline bf16_t v_scale_bits(float top)
{
    if (!(top < f32_from_bits(0x7F800000u))) return 0x7FC0;
    const float s = top / 6.f;
    return s < f32_from_bits(27u << 23) ? (bf16_t)0 : f32_to_bf16(s);
}

}  // namespace ckv
