// Attention over the paged cache in 4 bits: blocks of a few query rows per KV head (single tokens, a few of them, short chunks) against a long cache.
#include <type_traits>

#include "async_copy.h"
#include "paged_attend.h"

namespace ckv {

// ------------------------------------------------------------------ few rows
// out = softmax(scale Q K^T) V for blocks of 16 * NT rows (new tokens x query heads of one KV head), bound by the bytes of the cache.
//
// v_mfma_f32_16x16x32_bf16: S^T = K Q^T, keys are rows and queries columns.  A lane (m = l % 16, q = l / 16) takes key m of 16
// and a quarter of the channels, D/4 consecutive ones: one 16-byte piece of codes (D = 128) with one scale, turned into bf16 by
// v_cvt_scalef32_pk_bf16_fp4 without error (a code has two significant bits).  The accumulators of two such tiles are the logits of keys
// 4q + b and 16 + 4q + b; V bytes lie in that order, so the probabilities are the B operand of O^T = V^T P^T as they stand.  V codes
// go in unscaled; a key's scale is a factor of its probability.  bf16: that product is rounded to bf16, which the matrix instruction takes, with the sum of probabilities from
// before the rounding: outputs of 131072 keys are off by 0.0023 of their size (root mean square) where the rounding of the outputs alone makes 0.0017; a second term would double
// the products.  fp32: the queries and the scaled probabilities are sums of three bf16 terms
// (24 bits), with a product each.
//
// A workgroup has kFewWaves waves; wave w takes groups w, w + kFewWaves, ... of the workgroup's share.  A wave has kFewStages groups of its own in
// LDS, filled by asynchronous copies (a group is contiguous), and waits only for its own.  A group takes a wave 1 to 2 us from its first LDS read to its last product, most of it
// waiting for itself, so waves a SIMD count for more than bytes on their way: 32 sequences of 16384 keys (562 MB) take 104 us with two
// stages, 106 with three stages, 114 with four and two workgroups; 132 with the next group's
// loads in registers.  One token on 131072 keys (140 MB): 26 us and 4 for the join of 94 splits, 5.4 and 4.6 TB/s; a large copy reaches 4.74, reads alone 6.5 to 6.9.  The running maximum is raised only when a logit exceeds it by 2^8 (in 32 bits nothing is lost below 2^127): a
// vote instead of an exchange between lanes for most groups.
template <int D> struct GroupCodes {
    u32x4_t k[2];            // D = 64: the first two words
    u32x4_t v[D / 64];
    u32x4_t scales;          // V scales of keys 4q + b, then 16 + 4q + b
    uint32_t exps;           // K bytes of keys m and 16 + m
};

constexpr int kFewStages = 2;
template <int D> constexpr int few_stage_bytes() { return 32 * D + 256; }      // the codes, and 256 bytes from the scales on
template <int D> constexpr int few_copies() { return D / 32 + 1; }             // copies of 1 KB, and one of 256 bytes

// One group, to LDS.  The last copy's lanes behind the group (D = 64) read its last word again.  A group that one workgroup reads is streamed past the caches (32 sequences of
// 16384 keys take 104 us, 117 without); one that other blocks of rows read too is not (33 new tokens on 60000 keys: 83 us, streamed 97).
template <int D> __device__ inline void copy_group(const uint8_t* group, uint32_t lds, int lane, bool once)
{
    if (once) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) async_copy_1k_stream(group, (uint32_t)(i * 1024 + lane * 16), __builtin_amdgcn_readfirstlane(lds + i * 1024u));
    } else {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) async_copy_1k(group, (uint32_t)(i * 1024 + lane * 16), __builtin_amdgcn_readfirstlane(lds + i * 1024u));
    }
    async_copy_256(group, (uint32_t)(32 * D + min(lane * 4, paged_group_bytes(D) - 32 * D - 4)), __builtin_amdgcn_readfirstlane(lds + 32u * D));
}

// At most `behind` groups (0 .. MOST) of C copies each on their way.
template <int MOST, int C> __device__ inline void wait_behind(int behind)
{
    if constexpr (MOST == 0) {
        wait_vm_fenced<0>();
    } else {
        if (behind == MOST) wait_vm_fenced<MOST * C>();
        else wait_behind<MOST - 1, C>(behind);
    }
}

template <int D> __device__ inline void load_group(GroupCodes<D>& c, const uint8_t* group, int m, int q)
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

template <typename T, int D, int NT> __global__ __launch_bounds__(kFewWaves * 64, sizeof(T) == 4 && NT == 2 ? 1 : 2) void attend_few_kernel(PagedGeom g, PagedBatch b, FewPlan plan, const T* __restrict__ q, int64_t q_stride,
                                                                                                        T* __restrict__ out, float* __restrict__ part)
{
    constexpr int kTerms = sizeof(T) == 2 ? 1 : 3, kSteps = D / 32;
    constexpr int kStage = few_stage_bytes<D>(), kCopies = few_copies<D>();
    typedef float WaveRows[16][D + 4];
    __shared__ __attribute__((aligned(1024))) uint8_t ring[kFewWaves * kFewStages * kStage];      // afterwards: the waves' outputs
    __shared__ float m_wave[kFewWaves][16], l_wave[kFewWaves][16];
    static_assert(sizeof(WaveRows) <= kFewStages * kStage, "outputs fit the stages");
    WaveRows* o_wave = (WaveRows*)ring;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, qq = lane >> 4;
    const int split = blockIdx.x, hk = blockIdx.y % g.Hkv, row0 = (gridDim.y - 1 - blockIdx.y) / g.Hkv * (16 * NT), s = blockIdx.z;
    const bool once = NT == 1 || (int)gridDim.y == g.Hkv;      // (known to the compiler for up to 16 rows: a test of it in the loop costs 32 ragged sequences 60 -> 71 us)
    const SeqView v = seq_view(b, s);
    const int rows = v.n * g.G;
    if (row0 >= rows || rows > plan.max_rows) return;
    const int i0 = row0 / g.G, i1 = (min(row0 + 16 * NT, rows) - 1) / g.G;      // the block's tokens
    const KeySpan span = key_span(g, b, v, i0, i1);
    const int per = plan.groups_per_split, first = span.first + split * per, last = min(first + per, span.last);
    if (split > 0 && first >= span.last) return;      // split 0 also stands for a sequence that sees nothing

    // queries: column m + 16 n, the channels that this lane's keys have
    Frag qf[NT][kTerms][kSteps];
    int pos[NT];      // of the column's token; columns without a row stand for the block's first
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + m + 16 * n < rows ? row0 + m + 16 * n : row0, i = row / g.G, h = row - i * g.G;
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
    bool far = false;            // a column of the wave has come by a maximum of kFarLogit
    bool saw_whole = false, saw[NT];      // whether a group that every column sees whole, or a key that the lane's column sees, was there
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = kNoLogit;
        saw[n] = false;
        sum[n] = 0.f;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) o[n][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float scale = g.scale * 1.44269504088896341f;
    // groups that every column sees whole
    const int whole_from = g.window ? v.len + i1 + 1 - g.window : 0, whole_to = min(v.len + i0 + 1, b.max_length);

    const int count = (last - first - wave + kFewWaves - 1) / kFewWaves;      // groups of this wave
    int numbers = -1;      // lane l: place of the wave's group 64 * k + l
    uint32_t missing = 0;      // bit: stage holds a group that does not exist (what was copied is page 0's)
    const uint8_t* stages = ring + wave * kFewStages * kStage;
    const uint32_t stages_lds = lds_address(stages);
    auto issue = [&](int i) {
        if ((i & 63) == 0) {
            const int mine = i + lane;
            numbers = mine < count ? (int)paged_group(g, b, s, (first + wave + mine * kFewWaves) * kGroupTokens) : -1;
        }
        const int at = __builtin_amdgcn_readlane(numbers, i & 63), stage = i % kFewStages;
        missing = at < 0 ? missing | 1u << stage : missing & ~(1u << stage);
        copy_group<D>(g.pages + ((int64_t)max(at, 0) + hk * g.groups) * g.group_bytes, stages_lds + stage * kStage, lane, once);
    };
    for (int i = 0; i < min(count, kFewStages - 1); ++i) issue(i);
    for (int i = 0; i < count; ++i) {
        wait_lds_reads();      // the stage that is filled now has been read
        if (i + kFewStages - 1 < count) issue(i + kFewStages - 1);
        const int behind = min(count - 1 - i, kFewStages - 1);      // groups on their way behind this one
        wait_behind<kFewStages - 1, kCopies>(behind);
        if (!(missing >> (i % kFewStages) & 1u)) {
            GroupCodes<D> cur;
            load_group<D>(cur, stages + i % kFewStages * kStage, m, qq);
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
            // SOME: there may be keys that a column does not see
            auto probabilities = [&](auto some) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    bool seen[8];
                    if (decltype(some)::value) {
                        const int to = min(pos[n] + 1, b.max_length), from = g.window ? pos[n] - g.window + 1 : 0;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int key = key0 + 16 * (j >> 2) + 4 * qq + (j & 3);
                            seen[j] = key >= from && key < to;
                            if (!seen[j]) st[n][j >> 2][j & 3] = -INFINITY;
                            saw[n] |= seen[j];
                        }
                    }
                    float mx = st[n][0][0];
#pragma unroll
                    for (int j = 1; j < 8; ++j) mx = max_of(mx, st[n][j >> 2][j & 3]);
                    mx *= scale;
                    if (__ballot(mx > top[n] + kRescaleLog2)) {
                        const float now = max_of(top[n], max_quarters(mx));
                        far |= __ballot(is_far(now)) != 0;
                        const float shrink = __builtin_amdgcn_exp2f(top[n] - now);
                        top[n] = now;
                        sum[n] *= shrink;
#pragma unroll
                        for (int t = 0; t < D / 16; ++t) o[n][t] *= shrink;
                    }
                    // (16 rows: without a branch, with which the compiler keeps the outputs twice and a SIMD has one wave fewer, 32 sequences 56 -> 69 us; fp32: 1 to 2 % either way)
                    const float unit = far ? 1.f : scale;
                    if (NT == 1 || sizeof(T) == 4 || __builtin_expect(far, 0))
#pragma unroll
                        for (int j = 0; j < 8; ++j) st[n][j >> 2][j & 3] *= far ? scale : 1.f;
                    float p[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[n][j >> 2][j & 3], unit, -top[n]));
                        sum[n] += e;
                        const uint32_t w = cur.scales[j >> 1];
                        p[j] = e * __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
                        if (decltype(some)::value) p[j] = seen[j] ? p[j] : 0.f;      // what is not seen may hold any scale
                    }
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if constexpr (kTerms == 1) pf[n][0].u[x] = cvt_pk_bf16(p[x], p[4 + x]);
                        else split_terms(p[x], p[4 + x], [&](int term, uint32_t pair) { pf[n][term].u[x] = pair; });
                    }
                }
            };
            saw_whole |= whole;
            if (whole) probabilities(std::false_type());
            else probabilities(std::true_type());
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
    }
    __syncthreads();      // every wave has read its last stage

    // the waves' results together: a row's channels by 16 threads
    const bool alone = span.last - span.first <= per;      // no other split has keys
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n) __syncthreads();
        const float whole_sum = sum_quarters(top[n] == kNoLogit && (saw_whole || saw[n]) ? sum[n] + 1.f : sum[n]);      // (row_factor)
        if (qq == 0) {
            m_wave[wave][m] = top[n];
            l_wave[wave][m] = whole_sum;
        }
#pragma unroll
        for (int t = 0; t < D / 16; ++t) *(f32x4_t*)&o_wave[wave][m][16 * t + 4 * qq] = o[n][t];
        __syncthreads();
        constexpr int kEach = D / 16;
        const int c = threadIdx.x / 16, at = threadIdx.x % 16 * kEach, row = row0 + c + 16 * n;
        if (row < rows) {
            float all = m_wave[0][c];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) all = fmaxf(all, m_wave[w][c]);
            float l = 0.f, x[kEach] = {};
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(m_wave[w][c] - all);
                l += f * l_wave[w][c];
#pragma unroll
                for (int e = 0; e < kEach; ++e) x[e] += f * o_wave[w][c][at + e];
            }
            const int i = row / g.G, h = row - i * g.G;
            if (alone) {
                T* y = out + ((int64_t)(v.first + i) * g.Hq + hk * g.G + h) * D + at;
                const float r = row_factor(all, l);
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

// Joins the splits of a row: the splits' maxima and sums a thread each, then D/4 threads on four channels with the splits over the rest of the workgroup.
template <typename T, int D> __global__ __launch_bounds__(256) void merge_few_kernel(PagedGeom g, PagedBatch b, FewPlan plan, const float* __restrict__ part, T* __restrict__ out)
{
    constexpr int kLanes = D / 4, kParts = 256 / kLanes, kFirst = 12;
    __shared__ float o_part[kParts][D], weight[kFewMaxSplits], m_wave[4], l_wave[4];
    const int row = blockIdx.x, hk = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
    const int p = tid / kLanes, c = tid % kLanes * 4;
    const float* x = part + ((int64_t)(s * g.Hkv + hk) * plan.splits * plan.max_rows + row) * (D + 2);
    const int64_t step = (int64_t)plan.max_rows * (D + 2);
    // what a launch of plan.splits may hold is on its way before the sequence is looked up: one token on 131072 keys 33.4 -> 32.3 us, on 16384 11.6 -> 11.2
    float2 ml[2];      // of at most kFewMaxSplits, two a thread
#pragma unroll
    for (int i = 0; i < 2; ++i) ml[i] = tid + 256 * i < plan.splits ? *(const float2*)(x + (tid + 256 * i) * step + D) : make_float2(kNoLogit, 0.f);
    float2 first[kFirst][2];
#pragma unroll
    for (int n = 0; n < kFirst; ++n) {
        if (n * kParts >= plan.splits) break;
        const float* y = x + min(p + n * kParts, plan.splits - 1) * step + c;
        first[n][0] = *(const float2*)y;
        first[n][1] = *(const float2*)(y + 2);
    }
    const SeqView v = seq_view(b, s);
    if (row >= v.n * g.G || v.n * g.G > plan.max_rows) return;
    const int row0 = row / plan.block_rows * plan.block_rows;
    const KeySpan span = key_span(g, b, v, row0 / g.G, (min(row0 + plan.block_rows, v.n * g.G) - 1) / g.G);
    const int splits = (span.last - span.first + plan.groups_per_split - 1) / plan.groups_per_split;
    if (splits <= 1) return;      // written by its only split
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (tid + 256 * i >= splits) ml[i] = make_float2(kNoLogit, 0.f);
    float top = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
    for (int w = 32; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    if ((tid & 63) == 0) m_wave[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(m_wave[0], m_wave[1]), fmaxf(m_wave[2], m_wave[3]));
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float f = __builtin_amdgcn_exp2f(ml[i].x - top);
        weight[tid + 256 * i] = f;
        l += f * ml[i].y;
    }
#pragma unroll
    for (int w = 32; w; w >>= 1) l += __shfl_xor(l, w);
    if ((tid & 63) == 0) l_wave[tid >> 6] = l;
    __syncthreads();
    float o[4] = {};
    const auto add = [&](float f, const float2& a, const float2& e) {
        o[0] += f * a.x;
        o[1] += f * a.y;
        o[2] += f * e.x;
        o[3] += f * e.y;
    };
#pragma unroll
    for (int n = 0; n < kFirst; ++n)
        if (p + n * kParts < splits) add(weight[p + n * kParts], first[n][0], first[n][1]);
#pragma unroll 8
    for (int i = p + kFirst * kParts; i < splits; i += kParts) add(weight[i], *(const float2*)(x + i * step + c), *(const float2*)(x + i * step + c + 2));
    *(float4*)&o_part[p][c] = make_float4(o[0], o[1], o[2], o[3]);
    __syncthreads();
    if (p) return;
    l = l_wave[0] + l_wave[1] + l_wave[2] + l_wave[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o[e] = 0.f;
#pragma unroll
        for (int i = 0; i < kParts; ++i) o[e] += o_part[i][c + e];
    }
    const int i = row / g.G, h = row - i * g.G;
    const float r = row_factor(top, l);
    store4(out + ((int64_t)(v.first + i) * g.Hq + hk * g.G + h) * D + c, o[0] * r, o[1] * r, o[2] * r, o[3] * r);
}

// The same for a few splits of many rows: D/4 threads a row, one split after the other.
template <typename T, int D> __global__ __launch_bounds__(256) void merge_rows_kernel(PagedGeom g, PagedBatch b, FewPlan plan, const float* __restrict__ part, T* __restrict__ out)
{
    constexpr int kLanes = D / 4;
    const int row = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes, hk = blockIdx.y, s = blockIdx.z, c = threadIdx.x % kLanes * 4;
    const SeqView v = seq_view(b, s);
    if (row >= v.n * g.G || v.n * g.G > plan.max_rows) return;
    const int row0 = row / plan.block_rows * plan.block_rows;
    const KeySpan span = key_span(g, b, v, row0 / g.G, (min(row0 + plan.block_rows, v.n * g.G) - 1) / g.G);
    const int splits = (span.last - span.first + plan.groups_per_split - 1) / plan.groups_per_split;
    if (splits <= 1) return;
    const float* x = part + ((int64_t)(s * g.Hkv + hk) * plan.splits * plan.max_rows + row) * (D + 2);
    const int64_t step = (int64_t)plan.max_rows * (D + 2);
    float top = kNoLogit;
#pragma unroll 4
    for (int i = 0; i < splits; ++i) top = fmaxf(top, x[i * step + D]);
    float l = 0.f, o[4] = {};
#pragma unroll 4
    for (int i = 0; i < splits; ++i) {
        const float2 a = *(const float2*)(x + i * step + c), e = *(const float2*)(x + i * step + c + 2), ml = *(const float2*)(x + i * step + D);
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        l += f * ml.y;
        o[0] += f * a.x;
        o[1] += f * a.y;
        o[2] += f * e.x;
        o[3] += f * e.y;
    }
    const int i = row / g.G, h = row - i * g.G;
    const float r = row_factor(top, l);
    store4(out + ((int64_t)(v.first + i) * g.Hq + hk * g.G + h) * D + c, o[0] * r, o[1] * r, o[2] * r, o[3] * r);
}

// ------------------------------------------------------------------ launches
// The longest range of keys of a batch's sequences.
static int64_t longest_span(const PagedGeom& g, const PagedBatch& b)
{
    return g.window && g.window < b.max_length - b.max_new ? (int64_t)g.window + b.max_new : b.max_length;
}

// Splits of a launch for few rows: a share is a whole number of rounds of the workgroup's waves.  Workgroups that a compute unit runs at once: with 16 rows, bound by
// memory, three are enough (registers would allow four: one token on 131072 keys 32.3 us, with four 34.7; at D = 64 four); with 32 rows two (three at D
// = 64), fp32 one (two).  That many times 256 a launch (16 new tokens of four sequences on 16000 keys: 41 us, with three workgroups a unit 47; fp32 on 2000 keys
// 18, with two 24), or as many times that as leave a workgroup at most 24 rounds (sequences of different lengths even out over them: 32 of up to 16384 keys take 60
// us, with 48 rounds 90, with 12 77).
constexpr int kFewRounds = 24;
// Joins of at least 2048 rows of at most 16 splits go to merge_rows_kernel (16 new tokens of four sequences on 16000 keys, 2048 rows of 16 splits: 39 us in all, with
// a workgroup a row 42; 1024 rows of 9 splits 61 and 60; 512 of 16 21 and 20; 32 7.8 and 7.5).
static bool rows_share_workgroups(int64_t rows, int64_t splits) { return rows >= 2048 && splits <= 16; }
static double join_cost(int64_t rows, int64_t splits) { return 5 + rows / 1024.0 * (rows_share_workgroups(rows, splits) ? 0.2 * splits : 1 + 0.25 * splits); }      // us
static FewPlan few_plan(const PagedGeom& g, const PagedBatch& b, int limit, int dtype)
{
    FewPlan p;
    const int64_t rows = (int64_t)b.max_new * g.G;
    p.max_rows = rows < limit ? (int)rows : limit;
    p.block_rows = p.max_rows <= 16 ? 16 : 32;
    const int64_t pairs = (int64_t)b.n_seqs * g.Hkv, blocks = pairs * ((p.max_rows + p.block_rows - 1) / p.block_rows);
    const int64_t rounds = (longest_span(g, b) / kGroupTokens + 2 + kFewWaves - 1) / kFewWaves;      // of the longest sequence (its first and last group may be begun)
    const int at_once = p.block_rows == 16 ? 3 : dtype == CASCADE_F32 ? 1 : 2;
    const int64_t fill = 256 * (g.d == 64 ? at_once + 1 : at_once), most = kChunkPartRows / (pairs * p.max_rows);      // (the partial results have to fit)
    int64_t splits = fill / blocks;
    for (int64_t k = 2; splits < most && rounds > kFewRounds * (splits < 1 ? 1 : splits) && k <= 64; ++k) splits = fill * k / blocks;
    if (splits > most) splits = most;
    if (splits > rounds) splits = rounds;
    if (splits > kFewMaxSplits) splits = kFewMaxSplits;
    // (a round takes about 1 us: 24 new tokens of 4 heads each on 300 keys, 16 sequences, 38 us with two splits, 12 without)
    if (splits < 1 || rounds - rounds / splits < join_cost(pairs * p.max_rows, splits)) splits = 1;
    const int64_t each = (rounds + splits - 1) / splits;
    p.groups_per_split = (int)(each * kFewWaves);
    p.splits = (int)((rounds + each - 1) / each);
    return p;
}

// Whether the kernel for few rows takes sequences of more than kFewRows rows of a KV head too: where it is the cheaper one for the whole batch.  Its workgroups have 32 rows and
// go over the keys again for each of them; the other kernel's have 256 (fp32: 128), one on a compute unit, begin late and take a tile of 64 keys after the other.  us, from
// measurements of both: here 6 and 0.28 for 32 rows by 32 keys on a compute unit; there 4, 12 for a workgroup and 2 for a tile; fp32 has three times the
// products.  us here and there, 8 KV heads of 4 query heads, on 16000 keys, 48 | 200 | 400 new tokens of one sequence: bf16, d 128 35, 57 | 102, 103 | 178, 147; d 64 29, 46 | 75, 77 |
// 127, 107; fp32, d 128 67, 106 | 225, 224 | 442, 431; d 64 39, 81 | 123, 169 | 210, 322; 16 of four sequences in bf16 38, 128.  Of 198 calls (both types and head sizes, 2 and 8 KV
// heads, 1 and 4 sequences, 500 to 16000 keys, 16 to 1000 new tokens) the estimate takes the kernel that is more than 5 % slower in 17, by 1.34 at most (fp32, d 64, 1000 on
// 16000: 483, 647).
static bool few_rows_take_all(const PagedGeom& g, const PagedBatch& b, int dtype)
{
    const int64_t most = (int64_t)b.max_new * g.G, rows = ((int64_t)b.n_tokens * g.G + b.n_seqs - 1) / b.n_seqs;      // of a sequence: the most, the mean
    if (most <= kFewRows) return true;
    // (a workgroup per 32 of the most rows: not where nearly all of them would be empty, nor more than a launch can have)
    const int64_t pairs = (int64_t)b.n_seqs * g.Hkv, blocks = pairs * ((rows + 31) / 32), grid = pairs * ((most + 31) / 32);
    if (grid > 4096 + 2 * blocks || grid > (1 << 23) || grid / b.n_seqs > 65535 || most > kChunkPartRows) return false;
    const bool f32 = dtype == CASCADE_F32;
    const int block_rows = f32 ? 128 : 256;
    // keys of the last row, and of the mean one
    const int64_t longest = longest_span(g, b), mean = g.window && g.window < b.max_length - b.max_new ? g.window + 32 : b.max_length - b.max_new / 2;
    const FewPlan few = few_plan(g, b, (int)most, dtype);
    const double here = 6 + 0.28 * (f32 ? 3 : 1) * g.d / 128 * blocks * (mean / kGroupTokens + 1) / 256 + (few.splits > 1 ? join_cost(pairs * rows, few.splits) : 0.0);
    const ChunkPlan many = chunk_plan(g, b, 0, block_rows);
    const double waves = ceil(pairs * ((rows + block_rows - 1) / block_rows) * many.splits / 256.0), tile = (f32 ? 3.8 : 2.0) * (g.d == 64 ? 0.75 : 1.0);
    const double there = 4 + waves * (12 + tile * ((waves > 1 ? mean : longest) / 64.0 / many.splits + 1)) + (many.splits > 1 ? 6 : 0);
    return here <= there;
}

size_t paged_scratch_bytes(const PagedGeom& g) { return (size_t)kChunkPartRows * (g.d + 2) * 4; }

void launch_paged_attend(const PagedGeom& g, const PagedBatch& b, const void* q, int64_t q_stride, void* out, void* scratch, int dtype, hipStream_t s)
{
    const int64_t rows = (int64_t)b.max_new * g.G;
    const bool all = few_rows_take_all(g, b, dtype);
    // one sequence with more: the other kernel takes it, however many of the rows there are in the end
    const bool none = !all && b.n_seqs == 1;
    const FewPlan p = few_plan(g, b, all ? (int)rows : kFewRows, dtype);
    with_paged_form(dtype, g.d, [&](auto f) {
        typedef typename decltype(f)::Elt T;
        constexpr int D = decltype(f)::d;
        const dim3 grid(p.splits, g.Hkv * ((p.max_rows + p.block_rows - 1) / p.block_rows), b.n_seqs);
        if (none)
            ;
        else if (p.block_rows == 16)
            hipLaunchKernelGGL((attend_few_kernel<T, D, 1>), grid, dim3(kFewWaves * 64), 0, s, g, b, p, (const T*)q, q_stride, (T*)out, (float*)scratch);
        else
            hipLaunchKernelGGL((attend_few_kernel<T, D, 2>), grid, dim3(kFewWaves * 64), 0, s, g, b, p, (const T*)q, q_stride, (T*)out, (float*)scratch);
        if (!none && p.splits > 1 && rows_share_workgroups((int64_t)b.n_seqs * g.Hkv * p.max_rows, p.splits))
            hipLaunchKernelGGL((merge_rows_kernel<T, D>), dim3((p.max_rows * D / 4 + 255) / 256, g.Hkv, b.n_seqs), dim3(256), 0, s, g, b, p, (const float*)scratch, (T*)out);
        else if (!none && p.splits > 1)
            hipLaunchKernelGGL((merge_few_kernel<T, D>), dim3(p.max_rows, g.Hkv, b.n_seqs), dim3(256), 0, s, g, b, p, (const float*)scratch, (T*)out);
        if (!all)
            launch_attend_chunk(g, b, none ? 0 : p.max_rows, q, q_stride, out, scratch, dtype, s);
    });
}

}  // namespace ckv
