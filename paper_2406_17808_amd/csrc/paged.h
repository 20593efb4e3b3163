// Device helpers and launchers of the paged cache in 4 bits and of the per-head norms.
#pragma once

#include "paged_format.h"

namespace ckv {

// ------------------------------------------------------------------ rotation table
// lo[256][d/2] for the offsets 0 .. 255, then hi[ceil(n/256)][d/2] for the positions 0, 256, ...: (cos, sin) in 64 bits.
__device__ inline double2 rope_entry(const double2* __restrict__ rope, int half, uint32_t p, int i)
{
    const double2 a = rope[(size_t)(p & 255u) * half + i];
    const double2 b = rope[((size_t)(p >> 8) + 256) * half + i];
    return make_double2(__builtin_fma(a.x, b.x, -(a.y * b.y)), __builtin_fma(a.y, b.x, a.x * b.y));
}

// ------------------------------------------------------------------ work of ragged batches
// The last sequence whose first row is at or before row t.  Called by whole waves, t the same in all lanes.
__device__ inline int seq_of_row(const PagedBatch& b, int t)
{
    const int l = threadIdx.x & 63;
    int lo = 0, n = b.n_seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = l * step;
        const uint64_t in = __ballot(i < n && b.offsets[lo + (i < n ? i : 0)] <= t);
        const int k = max(0, __builtin_popcountll(in) - 1);
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Unit `unit` of a batch whose sequences have count(SeqView) units each: its sequence and its number there; false behind the last.  Called by whole
// waves, unit the same in all lanes.
template <typename F> __device__ inline bool find_unit(const PagedBatch& b, F count, int unit, int& seq, int& number)
{
    const int l = threadIdx.x & 63;
    if (b.n_seqs == 1) {
        seq = 0;
        number = unit;
        return unit < count(seq_view(b, 0));
    }
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
        const int n = s0 + l < b.n_seqs ? count(seq_view(b, s0 + l)) : 0;
        int upto = n;      // units of the sequences up to this lane's
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            if (l >= o) upto += x;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (unit < all) {
            const int at = __builtin_popcountll(__ballot(upto <= unit));
            seq = s0 + at;
            number = unit - __builtin_amdgcn_readlane(upto - n, at);
            return true;
        }
        unit -= all;
    }
    return false;
}

// ------------------------------------------------------------------ launchers
// f(PagedForm<element type, head size>{}) for the context's.
template <typename T, int D> struct PagedForm {
    typedef T Elt;
    static constexpr int d = D;
};
template <typename F> inline void with_paged_form(int dtype, int d, F f)
{
    if (dtype == CASCADE_BF16) {
        if (d == 64) f(PagedForm<bf16_t, 64>{});
        else f(PagedForm<bf16_t, 128>{});
    } else {
        if (d == 64) f(PagedForm<float, 64>{});
        else f(PagedForm<float, 128>{});
    }
}

struct NormRope {
    int d, n_tokens, Hq, Hk, norm;
    float eps;
    const void *q, *k;
    void *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const void *q_weight, *k_weight;
    const int32_t* positions;
    const double2* rope;
    int64_t rope_positions;
    bool vectors;     // every row is made of whole 16-byte pieces at 16-byte aligned places
};
size_t rope_pair_table_bytes(int64_t n_positions, int head_dim);
void launch_rope_pair_table(double2* rope, int64_t n_positions, int head_dim, double base, hipStream_t s);
void launch_norm_rope(const NormRope& a, int dtype, hipStream_t s);

struct PagedRows {
    const void *k, *v, *q;
    void* q_out;
    int64_t k_stride, v_stride, q_stride;
};
void launch_paged_append(const PagedGeom& g, const PagedBatch& b, const PagedRows& x, int dtype, hipStream_t s);
void launch_paged_read(const PagedGeom& g, const PagedBatch& b, void* k_out, void* v_out, int dtype, hipStream_t s);

size_t paged_scratch_bytes(const PagedGeom& g);
void launch_paged_attend(const PagedGeom& g, const PagedBatch& b, const void* q, int64_t q_stride, void* out, void* scratch, int dtype, hipStream_t s);

}  // namespace ckv
