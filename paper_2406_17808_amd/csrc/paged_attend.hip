// Attention over the paged cache in 4 bits: a few query rows per KV head (single tokens, a few of them) against a long cache.
#include "mfma_util.h"
#include "paged_attend.h"

namespace ckv {

// ------------------------------------------------------------------ few rows
// out = softmax(scale Q K^T) V for at most 16 * NT rows (new tokens x query heads of one KV head), bound by the bytes of the cache.
//
// v_mfma_f32_16x16x32_bf16: S^T = K Q^T, keys are rows and queries columns.  A lane (m = l % 16, q = l / 16) takes key m of 16
// and a quarter of the channels, D/4 consecutive ones: one 16-byte piece of codes (D = 128) with one scale, turned into bf16 by
// v_cvt_scalef32_pk_bf16_fp4 without error (a code has two significant bits).  The accumulators of two such tiles are the logits of keys
// 4q + b and 16 + 4q + b; V bytes lie in that order, so the probabilities are the B operand of O^T = V^T P^T as they stand.  V codes
// go in unscaled; a key's scale is a factor of its probability.  fp32: the queries and the scaled probabilities are sums of three bf16 terms
// (24 bits), with a product each.
//
// A workgroup has kFewWaves waves; wave w takes groups w, w + kFewWaves, ... of the workgroup's share, with the next group's codes on their way
// while one is worked on.  The running maximum is raised only when a logit exceeds it by 2^8 (in 32 bits
// nothing is lost below 2^127): a vote instead of an exchange between lanes for most groups.
template <int D> struct GroupCodes {
    u32x4_t k[2];            // D = 64: the first two words
    u32x4_t v[D / 64];
    u32x4_t scales;          // V scales of keys 4q + b, then 16 + 4q + b
    uint32_t exps;           // K bytes of keys m and 16 + m
};

template <int D> __device__ inline void load_group(GroupCodes<D>& c, const uint8_t* __restrict__ group, int m, int q)
{
    if constexpr (D == 128) {
        c.k[0] = *(const u32x4_t*)(group + q * 512 + m * 16);
        c.k[1] = *(const u32x4_t*)(group + q * 512 + 256 + m * 16);
        c.exps = *(const uint16_t*)(group + 32 * D + q * 32 + m * 2);
    } else {
        const uint2 a = *(const uint2*)(group + (q >> 1) * 512 + m * 16 + (q & 1) * 8), b = *(const uint2*)(group + (q >> 1) * 512 + 256 + m * 16 + (q & 1) * 8);
        c.k[0][0] = a.x; c.k[0][1] = a.y; c.k[1][0] = b.x; c.k[1][1] = b.y;
        c.exps = *(const uint16_t*)(group + 32 * D + (q >> 1) * 32 + m * 2);
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i) c.v[i] = *(const u32x4_t*)(group + 16 * D + i * 1024 + (q * 16 + m) * 16);
    c.scales = *(const u32x4_t*)(group + 33 * D + q * 16);
}

// max and sum over the four lanes that share column l % 16
__device__ inline float max_quarters(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max_xor32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float sum_quarters(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

template <typename T, int D, int NT> __global__ __launch_bounds__(kFewWaves * 64) void attend_few_kernel(PagedGeom g, PagedBatch b, FewPlan plan, const T* __restrict__ q, int64_t q_stride,
                                                                                                        T* __restrict__ out, float* __restrict__ part)
{
    constexpr int kTerms = sizeof(T) == 2 ? 1 : 3, kSteps = D / 32;
    __shared__ float o_wave[kFewWaves][16][D + 4], m_wave[kFewWaves][16], l_wave[kFewWaves][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, qq = lane >> 4;
    const int split = blockIdx.x, hk = blockIdx.y, s = blockIdx.z;
    const SeqView v = seq_view(b, s);
    const int rows = v.n * g.G;
    if (rows == 0 || rows > plan.max_rows) return;
    const KeySpan span = key_span(g, b, v);
    const int per = plan.groups_per_split, first = span.first + split * per, last = min(first + per, span.last);
    if (split > 0 && first >= span.last) return;      // split 0 also stands for a sequence that sees nothing

    // queries: column m + 16 n, the channels that this lane's keys have
    Frag qf[NT][kTerms][kSteps];
    int pos[NT];      // of the column's token; columns without a row stand for row 0
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = m + 16 * n, i = c < rows ? c / g.G : 0, h = c < rows ? c - i * g.G : 0;
        pos[n] = v.len + i;
        const T* x = q + (v.first + i) * q_stride + (hk * g.G + h) * D + D / 4 * qq;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            if constexpr (kTerms == 1) {
                qf[n][0][st].u = *(const u32x4_t*)(x + 8 * st);
            } else {
                float y[8];
                *(float4*)y = *(const float4*)(x + 8 * st);
                *(float4*)(y + 4) = *(const float4*)(x + 8 * st + 4);
#pragma unroll
                for (int e = 0; e < 8; e += 2) split_terms(y[e], y[e + 1], [&](int term, uint32_t pair) { qf[n][term][st].u[e / 2] = pair; });
            }
        }
    }

    f32x4_t o[NT][D / 16];
    float top[NT], sum[NT];      // running maximum (in units of log2) and the lane's part of the row sum
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) o[n][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float scale = g.scale * 1.44269504088896341f;
    // groups that every column sees whole
    const int whole_from = g.window ? v.len + v.n - g.window : 0, whole_to = min(v.len + 1, b.max_length);

    const int count = (last - first - wave + kFewWaves - 1) / kFewWaves;      // groups of this wave
    int numbers = -1;      // lane l: place of the wave's group 64 * k + l
    GroupCodes<D> cur, next;
    bool have = false;
    auto fetch = [&](int i, GroupCodes<D>& c) -> bool {
        if (i >= count) return false;
        if ((i & 63) == 0) {
            const int mine = i + lane;
            const int64_t at = mine < count ? paged_group(g, b, s, (first + wave + mine * kFewWaves) * kGroupTokens) : -1;
            numbers = (int)at;
        }
        const int at = __builtin_amdgcn_readlane(numbers, i & 63);
        if (at < 0) return false;
        load_group<D>(c, g.pages + ((int64_t)at + hk * g.groups) * g.group_bytes, m, qq);
        return true;
    };
    have = fetch(0, cur);
    for (int i = 0; i < count; ++i) {
        const bool have_next = fetch(i + 1, next);
        if (have) {
            const int key0 = (first + wave + i * kFewWaves) * kGroupTokens;
            const bool whole = key0 >= whole_from && key0 + 32 <= whole_to;
            f32x4_t st[NT][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float ks = scale_of_byte((cur.exps >> (8 * t)) & 255u);
#pragma unroll
                for (int n = 0; n < NT; ++n) st[n][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < kSteps; ++x) {
                    const Frag a = bf16_of_codes(cur.k[t][x], ks);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int y = 0; y < kTerms; ++y) st[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, qf[n][y][x].v, st[n][t], 0, 0, 0);
                }
            }
            Frag pf[NT][kTerms];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t seen = 255;
                if (!whole) {
                    const int to = min(pos[n] + 1, b.max_length), from = g.window ? pos[n] - g.window + 1 : 0;
                    seen = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int key = key0 + 16 * (j >> 2) + 4 * qq + (j & 3);
                        if (key >= from && key < to) seen |= 1u << j;
                        else st[n][j >> 2][j & 3] = -INFINITY;
                    }
                }
                float mx = st[n][0][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) mx = fmaxf(mx, st[n][j >> 2][j & 3]);
                mx *= scale;
                if (__ballot(mx > top[n] + kRescaleLog2)) {
                    const float now = fmaxf(top[n], max_quarters(mx));
                    const float shrink = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[n] - now);
                    top[n] = now;
                    sum[n] *= shrink;
#pragma unroll
                    for (int t = 0; t < D / 16; ++t) o[n][t] *= shrink;
                }
                float p[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[n][j >> 2][j & 3], scale, -top[n]));
                    if (!whole && !(seen >> j & 1u)) e = 0.f;
                    sum[n] += e;
                    const uint32_t w = cur.scales[j >> 1];
                    const float vs = __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
                    p[j] = !whole && !(seen >> j & 1u) ? 0.f : e * vs;      // what is not seen may hold any scale
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if constexpr (kTerms == 1) pf[n][0].u[x] = cvt_pk_bf16(p[x], p[4 + x]);
                    else split_terms(p[x], p[4 + x], [&](int term, uint32_t pair) { pf[n][term].u[x] = pair; });
                }
            }
#pragma unroll
            for (int u = 0; u < D / 32; ++u) {
                // four bytes of keys 4q + b and of keys 16 + 4q + b, two channels each -> eight keys of one channel
                const uint32_t x = cur.v[u >> 1][(u & 1) * 2], y = cur.v[u >> 1][(u & 1) * 2 + 1];
                const uint32_t lo = (x & 0x0F0F0F0Fu) | ((y << 4) & 0xF0F0F0F0u), hi = ((x >> 4) & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u);
                const Frag a = bf16_of_codes(lo, 1.f), c = bf16_of_codes(hi, 1.f);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int z = 0; z < kTerms; ++z) {
                        o[n][2 * u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, pf[n][z].v, o[n][2 * u], 0, 0, 0);
                        o[n][2 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c.v, pf[n][z].v, o[n][2 * u + 1], 0, 0, 0);
                    }
            }
        }
        cur = next;
        have = have_next;
    }

    // the waves' results together: a row's channels by 16 threads
    const bool alone = span.last - span.first <= per;      // no other split has keys
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n) __syncthreads();
        const float whole_sum = sum_quarters(sum[n]);
        if (qq == 0) {
            m_wave[wave][m] = top[n];
            l_wave[wave][m] = whole_sum;
        }
#pragma unroll
        for (int t = 0; t < D / 16; ++t) *(f32x4_t*)&o_wave[wave][m][16 * t + 4 * qq] = o[n][t];
        __syncthreads();
        constexpr int kEach = D / 16;
        const int c = threadIdx.x / 16, at = threadIdx.x % 16 * kEach, row = c + 16 * n;
        if (row < rows) {
            float all = m_wave[0][c];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) all = fmaxf(all, m_wave[w][c]);
            float l = 0.f, x[kEach] = {};
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                const float f = m_wave[w][c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_wave[w][c] - all);
                l += f * l_wave[w][c];
#pragma unroll
                for (int e = 0; e < kEach; ++e) x[e] += f * o_wave[w][c][at + e];
            }
            const int i = row / g.G, h = row - i * g.G;
            if (alone) {
                T* y = out + ((int64_t)(v.first + i) * g.Hq + hk * g.G + h) * D + at;
                const float r = all == -INFINITY ? 0.f : 1.f / l;
#pragma unroll
                for (int e = 0; e < kEach; e += 4) store4(y + e, x[e] * r, x[e + 1] * r, x[e + 2] * r, x[e + 3] * r);
            } else {
                float* y = part + (((int64_t)(s * g.Hkv + hk) * plan.splits + split) * plan.max_rows + row) * (D + 2);
#pragma unroll
                for (int e = 0; e < kEach; ++e) y[at + e] = x[e];
                if (at == 0) {
                    y[D] = all;
                    y[D + 1] = l;
                }
            }
        }
    }
}

// Joins the splits of a row: D/4 threads on four channels each, the splits over the rest of the workgroup.
template <typename T, int D> __global__ __launch_bounds__(256) void merge_few_kernel(PagedGeom g, PagedBatch b, FewPlan plan, const float* __restrict__ part, T* __restrict__ out)
{
    constexpr int kLanes = D / 4, kParts = 256 / kLanes;
    __shared__ float o_part[kParts][D], l_part[kParts], m_part[kParts];
    const int row = blockIdx.x, hk = blockIdx.y, s = blockIdx.z;
    const SeqView v = seq_view(b, s);
    if (row >= v.n * g.G || v.n * g.G > plan.max_rows) return;
    const KeySpan span = key_span(g, b, v);
    const int splits = (span.last - span.first + plan.groups_per_split - 1) / plan.groups_per_split;
    if (splits <= 1) return;      // written by its only split
    const float* x = part + ((int64_t)(s * g.Hkv + hk) * plan.splits * plan.max_rows + row) * (D + 2);
    const int64_t step = (int64_t)plan.max_rows * (D + 2);
    const int p = threadIdx.x / kLanes, c = threadIdx.x % kLanes * 4;
    float top = -INFINITY;
    for (int i = p; i < splits; i += kParts) top = fmaxf(top, x[i * step + D]);
    if (c == 0) m_part[p] = top;
    __syncthreads();
    top = m_part[0];
#pragma unroll
    for (int i = 1; i < kParts; ++i) top = fmaxf(top, m_part[i]);
    float l = 0.f, o[4] = {};
    for (int i = p; i < splits; i += kParts) {
        const float m = x[i * step + D], f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        l += f * x[i * step + D + 1];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += f * x[i * step + c + e];
    }
    if (c == 0) l_part[p] = l;
#pragma unroll
    for (int e = 0; e < 4; ++e) o_part[p][c + e] = o[e];
    __syncthreads();
    if (p) return;
    l = 0.f;
    for (int i = 0; i < kParts; ++i) l += l_part[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o[e] = 0.f;
        for (int i = 0; i < kParts; ++i) o[e] += o_part[i][c + e];
    }
    const int i = row / g.G, h = row - i * g.G;
    const float r = top == -INFINITY ? 0.f : 1.f / l;
    store4(out + ((int64_t)(v.first + i) * g.Hq + hk * g.G + h) * D + c, o[0] * r, o[1] * r, o[2] * r, o[3] * r);
}

// ------------------------------------------------------------------ launches
// Splits of a launch for few rows.  A share is a whole number of rounds of the workgroup's waves: at least one, at most 8, and
// between them what makes about 1024 workgroups (four for each compute unit); more than 8 only where there would be more than kFewParts.
static FewPlan few_plan(const PagedGeom& g, const PagedBatch& b)
{
    FewPlan p;
    const int64_t pairs = (int64_t)b.n_seqs * g.Hkv;
    const int longest = g.window && g.window < b.max_length - b.max_new ? g.window + b.max_new + 31 : b.max_length;
    const int64_t groups = longest / kGroupTokens + 1;
    int64_t rounds = groups * pairs / (1024 * kFewWaves);
    rounds = rounds < 1 ? 1 : rounds > 8 ? 8 : rounds;
    int64_t splits = (groups + rounds * kFewWaves - 1) / (rounds * kFewWaves);
    const int64_t most = kFewParts / pairs < 1 ? 1 : kFewParts / pairs;
    if (splits > most) {
        splits = most;
        rounds = (groups + splits * kFewWaves - 1) / (splits * kFewWaves);
    }
    p.groups_per_split = (int)(rounds * kFewWaves);
    p.splits = (int)splits;
    const int rows = b.max_new * g.G;
    p.max_rows = rows < kFewRows ? rows : kFewRows;
    return p;
}

static_assert(kFewParts * kFewRows <= kChunkPartRows, "one scratch for both");
size_t paged_scratch_bytes(const PagedGeom& g) { return (size_t)kChunkPartRows * (g.d + 2) * 4; }

void launch_paged_attend(const PagedGeom& g, const PagedBatch& b, const void* q, int64_t q_stride, void* out, void* scratch, int dtype, hipStream_t s)
{
    const FewPlan p = few_plan(g, b);
    const int64_t rows = (int64_t)b.max_new * g.G;
    with_paged_form(dtype, g.d, [&](auto f) {
        typedef typename decltype(f)::Elt T;
        constexpr int D = decltype(f)::d;
        const dim3 grid(p.splits, g.Hkv, b.n_seqs);
        if (p.max_rows <= 16)
            hipLaunchKernelGGL((attend_few_kernel<T, D, 1>), grid, dim3(kFewWaves * 64), 0, s, g, b, p, (const T*)q, q_stride, (T*)out, (float*)scratch);
        else
            hipLaunchKernelGGL((attend_few_kernel<T, D, 2>), grid, dim3(kFewWaves * 64), 0, s, g, b, p, (const T*)q, q_stride, (T*)out, (float*)scratch);
        if (p.splits > 1)
            hipLaunchKernelGGL((merge_few_kernel<T, D>), dim3(p.max_rows, g.Hkv, b.n_seqs), dim3(256), 0, s, g, b, p, (const float*)scratch, (T*)out);
        if (rows > kFewRows)
            launch_attend_chunk(g, b, p.max_rows, q, q_stride, out, scratch, dtype, s);
    });
}

}  // namespace ckv
