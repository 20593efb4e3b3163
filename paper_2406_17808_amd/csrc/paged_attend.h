// Device helpers that the attention kernels of the paged cache share.
#pragma once

#include "mfma_util.h"
#include "paged.h"

namespace ckv {

typedef __attribute__((ext_vector_type(4))) float f32x4_t;

constexpr int kFewWaves = 4;        // waves of a workgroup for few rows
constexpr int kFewRows = 32;        // rows of a sequence and KV head that it takes in any case
constexpr int kFewMaxSplits = 512;

struct FewPlan {
    int groups_per_split, splits;
    int max_rows;      // rows of a sequence and KV head: more are left to the other kernel
    int block_rows;    // rows of a workgroup: 16 or 32
};

constexpr int kChunkPartRows = 512 * 256;      // rows of partial results that a split launch may have

struct ChunkPlan {
    int units;         // at least the row blocks of all sequences
    int splits;
    int few_rows;      // sequences with at most this many rows are the other kernel's
};
ChunkPlan chunk_plan(const PagedGeom& g, const PagedBatch& b, int few_rows, int block_rows);
void launch_attend_chunk(const PagedGeom& g, const PagedBatch& b, int few_rows, const void* q, int64_t q_stride, void* out, void* scratch, int dtype, hipStream_t s);

// Row block `unit` of a batch, counted over the sequences that have more rows than the other kernel takes.
__device__ inline bool find_row_block(const PagedGeom& g, const PagedBatch& b, const ChunkPlan& plan, int unit, int block_rows, int& seq, int& block)
{
    return find_unit(b, [&](const SeqView& v) {
        const int rows = v.n * g.G;
        return rows > plan.few_rows ? (rows + block_rows - 1) / block_rows : 0;
    }, unit, seq, block);
}

// Groups of 32 keys that the new tokens i0 .. i1 of a sequence see: [first, last)
struct KeySpan {
    int first, last;
};
__device__ inline KeySpan key_span(const PagedGeom& g, const PagedBatch& b, const SeqView& v, int i0, int i1)
{
    KeySpan k;
    const int from = g.window && v.len + i0 >= g.window ? v.len + i0 - g.window + 1 : 0, to = min(v.len + i1 + 1, b.max_length);
    k.first = from / kGroupTokens;
    k.last = max(k.first, (to + kGroupTokens - 1) / kGroupTokens);
    return k;
}

// What the running maximum of a row (in units of log2) begins with: finite, so that a row that has seen nothing, or only logits of -infinity, gets exponentials of 0
// and factors of 1 without a test.
constexpr float kNoLogit = -3.4028234663852886e38f;

// An exponential of fma(logit, scale, -maximum) is off by what the maximum was rounded by, the same for all keys of a row: nothing for ordinary logits, a factor of up to 2
// where the maximum (in units of log2) is 2^24, an overflow from 2^31 on.  A wave that has come by a maximum of this size rounds its products with the scale before
// it subtracts.
constexpr float kFarLogit = 16777216.f;
__device__ inline bool is_far(float top) { return fabsf(top) >= kFarLogit && top != kNoLogit; }

// Whether the query at `pos` sees a key that exists in groups [first, last): what tells a row of logits of -infinity, whose softmax is NaN, from a row without keys, which
// gives zeros.
__device__ inline bool sees_a_key(const PagedGeom& g, const PagedBatch& b, int s, int pos, int first, int last)
{
    const int from = max(first * kGroupTokens, g.window ? pos - g.window + 1 : 0), to = min(last * kGroupTokens, min(pos + 1, b.max_length));
    for (int p = from; p < to; p = (p / kGroupTokens + 1) * kGroupTokens)
        if (paged_group(g, b, s, p) >= 0) return true;
    return false;
}

// One over the sum of a row's probabilities.  Where there is no logit, all of them are 0 and `total` counts the parts of the row that see a key (or is NaN).
__device__ inline float row_factor(float top, float total)
{
    return top != kNoLogit ? 1.f / total : total == 0.f ? 0.f : __uint_as_float(0x7FC00000u);
}

// The larger of two numbers, NaN if one is: an instruction of its own on gfx950 (fmaxf first makes its operands canonical, one instruction each).
__device__ inline float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The scale of a K block as the conversion takes it; NaN for byte 255.
__device__ inline float scale_of_byte(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23); }

// Eight codes -> bf16 times scale (a power of two): exact.
__device__ inline Frag bf16_of_codes(uint32_t codes, float scale)
{
    Frag f;
    f.u[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    f.u[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    f.u[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    f.u[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return f;
}

// Two floats as sums of three bf16 terms (8 + 8 + 8 bits): put(term, the two terms packed).
template <typename F> __device__ inline void split_terms(float a, float b, F put)
{
    const uint32_t x = cvt_pk_bf16(a, b);
    const float a1 = a - __uint_as_float(x << 16), b1 = b - __uint_as_float(x & 0xFFFF0000u);
    const uint32_t y = cvt_pk_bf16(a1, b1);
    put(0, x);
    put(1, y);
    put(2, cvt_pk_bf16(a1 - __uint_as_float(y << 16), b1 - __uint_as_float(y & 0xFFFF0000u)));
}

__device__ inline void store4(float* p, float a, float b, float c, float d) { *(float4*)p = make_float4(a, b, c, d); }
__device__ inline void store4(bf16_t* p, float a, float b, float c, float d) { *(uint2*)p = make_uint2(cvt_pk_bf16(a, b), cvt_pk_bf16(c, d)); }

}  // namespace ckv
