// Rows into and out of the paged cache: appending with the rotation on the way, and reading back as values.
#include "row_pieces.h"

namespace ckv {

// One half of a K block: 8 rotated channels of a thread, the 32 of the block in four neighbouring threads.
__device__ inline void write_k8(uint8_t* group, int d, int c, int r, const double (&y)[8])
{
    double top = 0.0;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double a = fabs(y[e]);
        top = fmax(top, a);
        bad |= !(a < __builtin_huge_val());
    }
    if (bad) top = __builtin_huge_val();
    top = fmax(top, __shfl_xor(top, 1));
    top = fmax(top, __shfl_xor(top, 2));
    const uint32_t byte = k_exponent(top);
    const double unit = byte == 255u ? __builtin_nan("") : pow2_f64((int)byte - 127);      // no comparison holds: codes of zeros
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) codes |= fp4_code(y[e], unit) << (4 * e);
    *(uint32_t*)(group + k_code_byte(c, r)) = codes;
    if ((c & 31) == 0) group[k_exp_byte(d, c >> 5, r)] = (uint8_t)byte;
}

// A workgroup per new token.  Rows are the KV heads' keys, their values and the query heads, D / 16 threads a row: the cosines and
// sines are made once per token, in 64 bits, and every row is read in 16-byte pieces.  Keys are rotated and
// rounded to codes in 64 bits: their codes then depend on nothing but the row and its position.
template <typename T, int D> __global__ __launch_bounds__(1024) void append_token_kernel(PagedGeom g, PagedBatch b, PagedRows x)
{
    constexpr int kTpr = D / 16, half = D / 2;
    __shared__ double2 cs[half];
    const int t = blockIdx.x;
    const int s = seq_of_row(b, t);
    const SeqView v = seq_view(b, s);
    const int i = t - v.first, p = v.len + i;
    if (i < 0 || i >= v.n) return;      // a row of no sequence
    if (g.rope) {
        for (int k = threadIdx.x; k < half; k += blockDim.x)
            cs[k] = p < g.rope_positions ? rope_entry(g.rope, half, (uint32_t)p, k) : make_double2(__builtin_nan(""), __builtin_nan(""));
        __syncthreads();
    }
    const int64_t at = paged_group(g, b, s, p);
    const int r = p & 31, j = threadIdx.x % kTpr;
    const int rows = 2 * g.Hkv + (x.q ? g.Hq : 0);
    for (int row = threadIdx.x / kTpr; row < rows; row += blockDim.x / kTpr) {      // the threads of a row leave together
        float lo[8], hi[8];
        if (row >= 2 * g.Hkv) {
            const int h = row - 2 * g.Hkv;
            const T* q = (const T*)x.q + t * x.q_stride + h * D;
            load8(q + 8 * j, lo);
            load8(q + half + 8 * j, hi);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double2 w = cs[8 * j + e];
                const float c = (float)w.x, sn = (float)w.y, a = lo[e], h2 = hi[e];
                lo[e] = rot_lo(a, h2, c, sn);
                hi[e] = rot_hi(a, h2, c, sn);
            }
            T* out = (T*)x.q_out + ((int64_t)t * g.Hq + h) * D;
            store8(out + 8 * j, lo);
            store8(out + half + 8 * j, hi);
            continue;
        }
        if (at < 0) continue;
        const int h = row < g.Hkv ? row : row - g.Hkv;
        uint8_t* group = g.pages + (at + (int64_t)h * g.groups) * g.group_bytes;
        if (row < g.Hkv) {
            const T* k = (const T*)x.k + t * x.k_stride + h * D;
            load8(k + 8 * j, lo);
            load8(k + half + 8 * j, hi);
            double ylo[8], yhi[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double a = lo[e], c = hi[e];
                if (g.rope) {
                    const double2 w = cs[8 * j + e];
                    ylo[e] = __builtin_fma(a, w.x, -(c * w.y));
                    yhi[e] = __builtin_fma(c, w.x, a * w.y);
                } else {
                    ylo[e] = a;
                    yhi[e] = c;
                }
            }
            write_k8(group, D, 8 * j, r, ylo);
            write_k8(group, D, half + 8 * j, r, yhi);
        } else {
            const int u = j >> 1, m0 = (j & 1) * 8;
            const T* val = (const T*)x.v + t * x.v_stride + h * D + 32 * u + m0;
            load8(val, lo);
            load8(val + 16, hi);
            float top = 0.f;
            bool bad = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                top = fmaxf(top, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
                bad |= !(fabsf(lo[e]) < __builtin_huge_valf() && fabsf(hi[e]) < __builtin_huge_valf());
            }
            if (bad) top = __builtin_huge_valf();
#pragma unroll
            for (int o = 1; o < kTpr; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
            const bf16_t bits = v_scale_bits(top);
            const float unit = bf16_to_f32(bits);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t byte = bits == 0 ? 0u : fp4_code(lo[e], unit) | fp4_code(hi[e], unit) << 4;
                group[v_code_byte(D, u, m0 + e, r)] = (uint8_t)byte;
            }
            if (j == 0) *(bf16_t*)(group + v_scale_byte(D, r)) = bits;
        }
    }
}

template <typename T, int D> __global__ __launch_bounds__(1024) void read_token_kernel(PagedGeom g, PagedBatch b, void* k_out, void* v_out)
{
    constexpr int kTpr = D / 16;
    const int t = blockIdx.x;
    const int s = seq_of_row(b, t);
    const SeqView v = seq_view(b, s);
    const int i = t - v.first, p = v.len + i;
    if (i < 0 || i >= v.n) return;
    const int64_t at = paged_group(g, b, s, p);
    const int r = p & 31, j = threadIdx.x % kTpr;
    for (int row = threadIdx.x / kTpr; row < 2 * g.Hkv; row += blockDim.x / kTpr) {
        const bool is_k = row < g.Hkv;
        const int h = is_k ? row : row - g.Hkv;
        if (!(is_k ? k_out : v_out)) continue;
        const uint8_t* group = g.pages + ((at < 0 ? 0 : at) + (int64_t)h * g.groups) * g.group_bytes;
        T* out = (T*)(is_k ? k_out : v_out) + ((int64_t)t * g.Hkv + h) * D;
        float a[8] = {}, c[8] = {};
        const int u = j >> 1, m0 = (j & 1) * 8;
        if (at >= 0 && is_k) {
            const uint2 codes = *(const uint2*)(group + k_code_byte(16 * j, r));
            const float scale = k_scale(group[k_exp_byte(D, j >> 1, r)]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] = fp4_value(codes.x >> (4 * e)) * scale;
                c[e] = fp4_value(codes.y >> (4 * e)) * scale;
            }
        } else if (at >= 0) {
            const float scale = bf16_to_f32(*(const bf16_t*)(group + v_scale_byte(D, r)));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t byte = group[v_code_byte(D, u, m0 + e, r)];
                a[e] = fp4_value(byte) * scale;
                c[e] = fp4_value(byte >> 4) * scale;
            }
        }
        store8(out + (is_k ? 16 * j : 32 * u + m0), a);
        store8(out + (is_k ? 16 * j + 8 : 32 * u + 16 + m0), c);
    }
}

static int row_threads(int rows, int d)
{
    const int n = (rows * (d / 16) + 63) / 64 * 64;
    return n > 1024 ? 1024 : n;
}

void launch_paged_append(const PagedGeom& g, const PagedBatch& b, const PagedRows& x, int dtype, hipStream_t s)
{
    const dim3 grid(b.n_tokens), block(row_threads(2 * g.Hkv + (x.q ? g.Hq : 0), g.d));
    with_paged_form(dtype, g.d, [&](auto f) {
        hipLaunchKernelGGL((append_token_kernel<typename decltype(f)::Elt, decltype(f)::d>), grid, block, 0, s, g, b, x);
    });
}

void launch_paged_read(const PagedGeom& g, const PagedBatch& b, void* k_out, void* v_out, int dtype, hipStream_t s)
{
    const dim3 grid(b.n_tokens), block(row_threads(2 * g.Hkv, g.d));
    with_paged_form(dtype, g.d, [&](auto f) {
        hipLaunchKernelGGL((read_token_kernel<typename decltype(f)::Elt, decltype(f)::d>), grid, block, 0, s, g, b, k_out, v_out);
    });
}

}  // namespace ckv
