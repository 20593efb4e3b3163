// Rows into and out of the paged cache: appending with the rotation on the way, and reading back as values.
#include "row_pieces.h"

namespace ckv {

// One half of a K block: 8 rotated channels of a thread, the 32 of the block in four neighbouring threads.  The numbers are rounded to codes from 32-bit
// keys: seven comparisons of 64-bit numbers a channel took longer than everything else.
__device__ inline void write_k8(uint8_t* group, int d, int c, int r, const double (&y)[8])
{
    uint32_t key[8], top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        key[e] = k_key(y[e]);
        top = max(top, key[e]);
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t byte = k_exponent_of_key(top);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(k_scaled_bits(key[e], byte) | (y[e] < 0.0 ? 0x80000000u : 0u));
    uint32_t codes = 0;      // rounds to the nearest code, ties to even, at most 6
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], 1.f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], 1.f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], 1.f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], 1.f, 3);
    *(uint32_t*)(group + k_code_byte(c, r)) = codes;
    if ((c & 31) == 0) group[k_exp_byte(d, c >> 5, r)] = (uint8_t)byte;
}

// Channels 16 j .. 16 j + 15 of key r.
__device__ inline void k_values(const uint8_t* group, int d, int j, int r, float (&a)[8], float (&c)[8])
{
    const uint2 codes = *(const uint2*)(group + k_code_byte(16 * j, r));
    const float scale = k_scale(group[k_exp_byte(d, j >> 1, r)]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        a[e] = fp4_value(codes.x >> (4 * e)) * scale;
        c[e] = fp4_value(codes.y >> (4 * e)) * scale;
    }
}

// A thread's part of a key, in 64 bits: 8 channels of the lower half and their partners, rotated or as they come.
struct KeyPart {
    double lo[8], hi[8];
};
template <typename F> __device__ inline KeyPart key_part(const float (&lo)[8], const float (&hi)[8], bool rotated, F cs)
{
    KeyPart y;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double a = lo[e], c = hi[e];
        if (rotated) {
            const double2 w = cs(e);
            y.lo[e] = __builtin_fma(a, w.x, -(c * w.y));
            y.hi[e] = __builtin_fma(c, w.x, a * w.y);
        } else {
            y.lo[e] = a;
            y.hi[e] = c;
        }
    }
    return y;
}

// The scale of a V row of which a thread has lo and hi, the row in TPR neighbouring threads; then its 8 bytes: put(e, byte).
template <int TPR, typename F> __device__ inline bf16_t value_part(const float (&lo)[8], const float (&hi)[8], F put)
{
    float top = 0.f;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
        bad |= !(fabsf(lo[e]) < __builtin_huge_valf() && fabsf(hi[e]) < __builtin_huge_valf());
    }
    if (bad) top = __builtin_huge_valf();
#pragma unroll
    for (int o = 1; o < TPR; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const bf16_t bits = v_scale_bits(top);
    const float unit = bf16_to_f32(bits);
#pragma unroll
    for (int e = 0; e < 8; ++e) put(e, bits == 0 ? 0u : fp4_code(lo[e], unit) | fp4_code(hi[e], unit) << 4);
    return bits;
}

// A row of queries: rotated in 32 bits.
template <typename T, typename F> __device__ inline void rotate_row(const T* q, T* out, int half, int j, F cs)
{
    float lo[8], hi[8];
    load8(q + 8 * j, lo);
    load8(q + half + 8 * j, hi);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 c = cs(e);
        const float x = lo[e], z = hi[e];
        lo[e] = rot_lo(x, z, c.x, c.y);
        hi[e] = rot_hi(x, z, c.x, c.y);
    }
    store8(out + 8 * j, lo);
    store8(out + half + 8 * j, hi);
}

__device__ inline double2 rope_or_nan(const PagedGeom& g, int half, int p, int i)
{
    return p < g.rope_positions ? rope_entry(g.rope, half, (uint32_t)p, i) : make_double2(__builtin_nan(""), __builtin_nan(""));
}

// A workgroup per new token.  Rows are the KV heads' keys, their values and the query heads, D / 16 threads a row: the cosines and
// sines are made once per token, in 64 bits, and every row is read in 16-byte pieces.  Keys are rotated and
// rounded to codes in 64 bits: their codes then depend on nothing but the row and its position.  32 single tokens of 32 + 8 + 8 heads (0.8 MB): 4.8 us on
// the device, the latency of arrays, table and row one after the other.
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
            cs[k] = rope_or_nan(g, half, p, k);
        __syncthreads();
    }
    const int64_t at = paged_group(g, b, s, p);
    const int r = p & 31, j = threadIdx.x % kTpr;
    const int rows = 2 * g.Hkv + (x.q ? g.Hq : 0);
    for (int row = threadIdx.x / kTpr; row < rows; row += blockDim.x / kTpr) {      // the threads of a row leave together
        if (row >= 2 * g.Hkv) {
            const int h = row - 2 * g.Hkv;
            rotate_row((const T*)x.q + t * x.q_stride + h * D, (T*)x.q_out + ((int64_t)t * g.Hq + h) * D, half, j,
                       [&](int e) { return make_float2((float)cs[8 * j + e].x, (float)cs[8 * j + e].y); });
            continue;
        }
        if (at < 0) continue;
        float lo[8], hi[8];
        const int h = row < g.Hkv ? row : row - g.Hkv;
        uint8_t* group = g.pages + (at + (int64_t)h * g.groups) * g.group_bytes;
        if (row < g.Hkv) {
            const T* k = (const T*)x.k + t * x.k_stride + h * D;
            load8(k + 8 * j, lo);
            load8(k + half + 8 * j, hi);
            const KeyPart y = key_part(lo, hi, g.rope != nullptr, [&](int e) { return cs[8 * j + e]; });
            write_k8(group, D, 8 * j, r, y.lo);
            write_k8(group, D, half + 8 * j, r, y.hi);
        } else {
            const int u = j >> 1, m0 = (j & 1) * 8;
            const T* val = (const T*)x.v + t * x.v_stride + h * D + 32 * u + m0;
            load8(val, lo);
            load8(val + 16, hi);
            const bf16_t bits = value_part<kTpr>(lo, hi, [&](int e, uint32_t byte) { group[v_code_byte(D, u, m0 + e, r)] = (uint8_t)byte; });
            if (j == 0) *(bf16_t*)(group + v_scale_byte(D, r)) = bits;
        }
    }
}

// ------------------------------------------------------------------ groups
// The groups of 32 tokens that a sequence's new tokens reach, and the tokens of one of them.
__device__ inline int groups_of(const SeqView& v) { return v.n ? (v.len + v.n - 1) / kGroupTokens - v.len / kGroupTokens + 1 : 0; }
struct GroupRows {
    int from, to;      // tokens of the group: [from, to)
    int p0, t0;        // position of its token 0, and the row that token 0 would have
};
__device__ inline GroupRows group_rows(const SeqView& v, int number)
{
    GroupRows x;
    x.p0 = (v.len / kGroupTokens + number) * kGroupTokens;
    x.from = max(0, v.len - x.p0);
    x.to = min(kGroupTokens, v.len + v.n - x.p0);
    x.t0 = v.first + x.p0 - v.len;
    return x;
}

// Many tokens of a sequence: a workgroup per group of 32 tokens and KV head, D / 16 threads a row, one half of the workgroup on keys and the other on
// values.  V bytes are gathered in LDS and leave in 16-byte pieces (a group that is not filled: in words of four tokens, or bytes); written
// token by token they are bytes 16 apart.  Workgroups behind the groups rotate queries, a row of D / 16 threads each.  4096 tokens of 8 KV heads, d 128, bf16: 23.0 us with the
// queries of 32 heads (88 MB, 3.8 TB/s), 15 without: 4200 vector instructions a workgroup, most of them for the keys in 64 bits (loading the cosines ahead costs half of the
// waves: 28 us); a workgroup per token takes 27.
template <typename T, int D> __global__ __launch_bounds__(4 * D) void append_group_kernel(PagedGeom g, PagedBatch b, PagedRows x, unsigned group_blocks)
{
    constexpr int kTpr = D / 16, half = D / 2, kHalf = 2 * D;      // threads of a half of the workgroup: 32 rows
    __shared__ __attribute__((aligned(16))) uint8_t v_img[16 * D];
    __shared__ float2 cs_q[half];
    const int j = threadIdx.x % kTpr;
    if (blockIdx.x >= group_blocks) {      // queries of a token
        const int t = blockIdx.x - group_blocks;
        const int s = seq_of_row(b, t);
        const SeqView v = seq_view(b, s);
        const int i = t - v.first, p = v.len + i;
        if (i < 0 || i >= v.n) return;
        if (threadIdx.x < half) {
            const double2 w = rope_or_nan(g, half, p, threadIdx.x);
            cs_q[threadIdx.x] = make_float2((float)w.x, (float)w.y);
        }
        __syncthreads();
        for (int h = threadIdx.x / kTpr; h < g.Hq; h += 2 * kHalf / kTpr)
            rotate_row((const T*)x.q + t * x.q_stride + h * D, (T*)x.q_out + ((int64_t)t * g.Hq + h) * D, half, j, [&](int e) { return cs_q[8 * j + e]; });
        return;
    }
    int s, number;
    const int h = blockIdx.x % g.Hkv;
    if (!find_unit(b, groups_of, blockIdx.x / g.Hkv, s, number)) return;
    const SeqView v = seq_view(b, s);
    const GroupRows rows = group_rows(v, number);
    const bool keys = threadIdx.x < kHalf;      // whole waves
    const int tid = threadIdx.x % kHalf, r = tid / kTpr, p = rows.p0 + r, to = min(rows.to, b.max_length - rows.p0);
    const bool on = r >= rows.from && r < to;      // the threads of a row agree
    const int u = j >> 1, m0 = (j & 1) * 8;
    float lo[8], hi[8];
    if (on) {      // on their way while the place is looked up
        const T* y = keys ? (const T*)x.k + (rows.t0 + r) * x.k_stride + h * D + 8 * j : (const T*)x.v + (rows.t0 + r) * x.v_stride + h * D + 32 * u + m0;
        load8(y, lo);
        load8(y + (keys ? half : 16), hi);
    }
    const int64_t at = paged_group(g, b, s, rows.p0);
    if (at < 0) return;
    uint8_t* group = g.pages + (at + (int64_t)h * g.groups) * g.group_bytes;
    if (on && keys) {
        const KeyPart y = key_part(lo, hi, g.rope != nullptr, [&](int e) { return rope_or_nan(g, half, p, 8 * j + e); });
        write_k8(group, D, 8 * j, r, y.lo);
        write_k8(group, D, half + 8 * j, r, y.hi);
    } else if (on) {
        const bf16_t bits = value_part<kTpr>(lo, hi, [&](int e, uint32_t byte) { v_img[v_code_byte(D, u, m0 + e, r) - 16 * D] = (uint8_t)byte; });
        if (j == 0) *(bf16_t*)(group + v_scale_byte(D, r)) = bits;
    }
    __syncthreads();
    if (keys) return;
    uint8_t* v_codes = group + 16 * D;
    if (rows.from == 0 && to == kGroupTokens) {
        if (tid < D) *(u32x4_t*)(v_codes + 16 * tid) = *(const u32x4_t*)(v_img + 16 * tid);
        return;
    }
    for (int w = tid; w < 4 * D; w += kHalf) {      // word w: tokens r0 .. r0 + 3
        const int r0 = ((w >> 6) & 3) * 4 + (w & 1) * 16;
        if (r0 >= rows.from && r0 + 4 <= to) *(uint32_t*)(v_codes + 4 * w) = *(const uint32_t*)(v_img + 4 * w);
        else
            for (int e = 0; e < 4; ++e)
                if (r0 + e >= rows.from && r0 + e < to) v_codes[4 * w + e] = v_img[4 * w + e];
    }
}

// Reading many tokens of a sequence: the same workgroups the other way round (4096 tokens, 21 MB: 9.2 us, twice what the bytes take: codes are expanded one by one by integer
// instructions, V bytes read from LDS one by one; a workgroup per token 11.6).
template <typename T, int D> __global__ __launch_bounds__(4 * D) void read_group_kernel(PagedGeom g, PagedBatch b, void* k_out, void* v_out)
{
    constexpr int kTpr = D / 16, kHalf = 2 * D;
    __shared__ __attribute__((aligned(16))) uint8_t v_img[16 * D];
    const bool keys = threadIdx.x < kHalf;
    const int tid = threadIdx.x % kHalf, j = tid % kTpr, r = tid / kTpr, h = blockIdx.y;
    int s, number;
    if (!find_unit(b, groups_of, blockIdx.x, s, number)) return;
    const SeqView v = seq_view(b, s);
    const GroupRows rows = group_rows(v, number);
    const int64_t at = paged_group(g, b, s, rows.p0);
    const uint8_t* group = g.pages + ((at < 0 ? 0 : at) + (int64_t)h * g.groups) * g.group_bytes;
    const bool on = r >= rows.from && r < rows.to, there = at >= 0 && rows.p0 + r < b.max_length;
    float a[8] = {}, c[8] = {};
    const int64_t row = ((int64_t)(rows.t0 + r) * g.Hkv + h) * D;
    if (keys && on && k_out) {
        if (there) k_values(group, D, j, r, a, c);
        store8((T*)k_out + row + 16 * j, a);
        store8((T*)k_out + row + 16 * j + 8, c);
    }
    const float scale = !keys && there ? bf16_to_f32(*(const bf16_t*)(group + v_scale_byte(D, r))) : 0.f;
    if (!keys && at >= 0 && tid < D) *(u32x4_t*)(v_img + 16 * tid) = *(const u32x4_t*)(group + 16 * D + 16 * tid);
    __syncthreads();
    if (keys || !on || !v_out) return;
    const int u = j >> 1, m0 = (j & 1) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t byte = there ? v_img[v_code_byte(D, u, m0 + e, r) - 16 * D] : 0u;
        a[e] = fp4_value(byte) * scale;
        c[e] = fp4_value(byte >> 4) * scale;
    }
    store8((T*)v_out + row + 32 * u + m0, a);
    store8((T*)v_out + row + 32 * u + 16 + m0, c);
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
            k_values(group, D, j, r, a, c);
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

// Calls with a sequence of at least this many new tokens go group by group: a launch is one kernel for all its sequences, by max_new (a group with a few
// tokens leaves most of its workgroup idle).  Append with queries, us token by token and by groups: bf16, 8 KV heads, d 128, one sequence with 16 new tokens 4.3, 5.3, with 256 4.7,
// 5.8; 32 sequences with 16 each 6.2, 6.8, with 32 10.3, 8.2, with 256 43.3, 42.2 (read 22.5, 15.8); 4096 of one 27, 23; fp32, 2 KV heads, d 64, 16 of one 5.9, 5.1, 32 of 32
// sequences 9.7, 6.4.  So 16 tokens of one bf16 sequence are 1 us slower than they could be.
constexpr int kGroupFormTokens = 16;

// At least the groups that all sequences reach.
static int group_units(const PagedBatch& b)
{
    const int64_t n = (int64_t)b.n_tokens / kGroupTokens + 2 * (int64_t)b.n_seqs;
    return (int)(n < b.n_tokens ? n : b.n_tokens);
}

void launch_paged_append(const PagedGeom& g, const PagedBatch& b, const PagedRows& x, int dtype, hipStream_t s)
{
    with_paged_form(dtype, g.d, [&](auto f) {
        typedef typename decltype(f)::Elt T;
        constexpr int D = decltype(f)::d;
        if (b.max_new >= kGroupFormTokens) {
            const int units = group_units(b);
            const unsigned group_blocks = (unsigned)units * g.Hkv;
            hipLaunchKernelGGL((append_group_kernel<T, D>), dim3(group_blocks + (x.q ? b.n_tokens : 0)), dim3(4 * D), 0, s, g, b, x, group_blocks);
        } else {
            hipLaunchKernelGGL((append_token_kernel<T, D>), dim3(b.n_tokens), dim3(row_threads(2 * g.Hkv + (x.q ? g.Hq : 0), D)), 0, s, g, b, x);
        }
    });
}

void launch_paged_read(const PagedGeom& g, const PagedBatch& b, void* k_out, void* v_out, int dtype, hipStream_t s)
{
    with_paged_form(dtype, g.d, [&](auto f) {
        typedef typename decltype(f)::Elt T;
        constexpr int D = decltype(f)::d;
        if (b.max_new >= kGroupFormTokens)
            hipLaunchKernelGGL((read_group_kernel<T, D>), dim3(group_units(b), g.Hkv), dim3(4 * D), 0, s, g, b, k_out, v_out);
        else
            hipLaunchKernelGGL((read_token_kernel<T, D>), dim3(b.n_tokens), dim3(row_threads(2 * g.Hkv, D)), 0, s, g, b, k_out, v_out);
    });
}

}  // namespace ckv
