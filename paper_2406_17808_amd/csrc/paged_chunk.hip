// Attention over the paged cache in 4 bits: many query rows per KV head (chunks of prompts), bound by the matrix cores.
#include <type_traits>

#include "async_copy.h"
#include "paged_attend.h"

namespace ckv {

// out = softmax(scale Q K^T) V for a block of 32 * NW rows (token, query head of the group) of one sequence and KV head.
//
// v_mfma_f32_32x32x16_bf16, S^T = K Q^T (keys are rows, one lane holds half of a query's 64 keys of a tile), O^T = V^T P^T.  The
// codes of a tile of 64 keys (two groups) are turned into bf16 once per workgroup, on their way from registers to LDS: every
// value is exact.  K: rows of D channels.  V: rows of 64 keys, in the order that the groups store them and the accumulators of S^T have them
// (a lane's keys 8s + 4h + b and 16 + 8s + 4h + b are piece 2s + h of a group); a key's V scale multiplies its probability.
//
// NW = 8: the two waves of a SIMD work in opposite phase, one on products (a matrix block: P V of tile t, then K Q^T of tile
// t + 1) while the other takes exponentials and converts codes (a vector block), with a barrier between phases.  Set x in LDS is K of
// tile x + 1 and V of tile x: what matrix block x reads.  The early waves (0 - 3) run matrix block x in phase 2x and write K in the vector block before
// it, phase 2x - 1; the late waves (4 - 7) run it in phase 2x + 1 and write V in phase 2x - 2.  Nobody reads set x after phase
// 2x + 1, and set x + 2 is written from phase 2x + 2 on: two stages do.
// What bounds it: 2048 tokens of 32 heads on 63500 cached ones, d 128, bf16, 2.0 ms: 1.08 PFLOP/s (a large library product in bf16: 1.27); the matrix cores are busy 51 % of the
// cycles, and a wave issues an instruction every five to six cycles: its vector block (exponentials, codes, maxima) takes 2300 cycles, its matrix block
// 1650, so that the vector blocks set the pace and each matrix block waits for one.  4096 tokens on none: 153 us, 0.90 PFLOP/s (the tiles at the diagonal,
// and about 10 us before a workgroup's first product).
// bf16: a probability times its V scale is rounded to bf16 for the product (the sum takes it before); outputs are off by 0.0021 to 0.0023 of their size (root mean square)
// where the rounding of the outputs alone makes 0.0016 to 0.0017.
// d 64, bf16: 2048 on 16000 386 us, 0.74 PFLOP/s, 4096 on none 111 us, 0.62: a tile has half of the products of d 128 and the same exponentials, so that the vector blocks
// weigh twice as much.
// NW = 4 (fp32: queries and scaled probabilities are sums of three bf16 terms, three times the products and the query registers): all waves are early and convert
// K and V; one wave a SIMD, so that products and exponentials take turns.  2048 on 16000 1.73 ms, 330 TFLOP/s (three products each: 424 at most).

// What a thread converts: N words of codes, and the K byte or a V scale.
template <int N> struct Piece {
    uint32_t w[N], extra;
    bool gone;      // the group is missing: this is page 0's
    __device__ void load(const uint8_t* p)
    {
        if constexpr (N == 4) {
            const u32x4_t c = *(const u32x4_t*)p;
            w[0] = c[0]; w[1] = c[1]; w[2] = c[2]; w[3] = c[3];
        } else {
            const uint2 c = *(const uint2*)p;
            w[0] = c.x; w[1] = c.y;
        }
    }
};

// Positions of 16-byte pieces in the rows of a tile: sixteen lanes that read or write one column of sixteen rows meet all banks once (256 bytes).
template <int D> __device__ inline int k_place(int r, int piece) { return r * D + (piece ^ (D == 128 ? r & 15 : (r >> 1) & 7)) * 8; }
__device__ inline int v_place(int ch, int piece) { return ch * kBN + (piece ^ ((ch >> 1) & 7)) * 8; }

template <typename T, int D, int NW> __global__ __launch_bounds__(NW * 64, 1) void attend_chunk_kernel(PagedGeom g, PagedBatch b, ChunkPlan plan, const T* __restrict__ q, int64_t q_stride,
                                                                                                   T* __restrict__ out, float* __restrict__ part)
{
    constexpr int kTerms = sizeof(T) == 2 ? 1 : 3, KS = D / 16, DB = D / 32, kRows = 32 * NW;
    constexpr int kItems = 8 / NW;                     // K and / or V pieces that a thread converts
    constexpr int kWords = D / 32;                     // words of codes a piece has: 8 * kWords channels of a key, or 8 keys of kWords channels
    __shared__ __attribute__((aligned(16))) bf16_t k_lds[2][kBN * D], v_lds[2][kBN * D];
    __shared__ __attribute__((aligned(16))) float vs_lds[2][kBN];
    __shared__ uint32_t special_lds;
    __shared__ float sees_lds[kRows];      // 1: the row sees a key of this range
    __shared__ uint32_t odd_lds[2][2], gone_lds[2][2];      // of a group: bits of V slots whose scale is an infinity or NaN; whether the group is missing

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, l32 = l & 31, half = l >> 5;
    const bool late = NW == 8 && wave >= 4;
    // consecutive workgroups: different KV heads; the blocks of a sequence from its end, which see most keys
    const int hk = blockIdx.x % g.Hkv, split = blockIdx.y;
    int s, block;
    if (!find_row_block(g, b, plan, gridDim.x / g.Hkv - 1 - blockIdx.x / g.Hkv, kRows, s, block)) return;
    const SeqView v = seq_view(b, s);
    const int rows = v.n * g.G, row0 = block * kRows;

    // positions that a row sees: [from, to)
    auto pos_of = [&](int row) { return v.len + min(row, rows - 1) / g.G; };
    auto from_of = [&](int pos) { return g.window ? max(0, pos - g.window + 1) : 0; };
    auto to_of = [&](int pos) { return min(pos + 1, b.max_length); };
    const int row = row0 + wave * 32 + l32, pos = pos_of(row), from = from_of(pos), to = to_of(pos);
    const int wave_first = pos_of(row0 + wave * 32), wave_last = pos_of(row0 + wave * 32 + 31);
    const int whole_from = from_of(wave_last), whole_to = to_of(wave_first), any_from = from_of(wave_first), any_to = to_of(wave_last);
    int tile0 = from_of(pos_of(row0)) / kBN, tile1 = (to_of(pos_of(row0 + kRows - 1)) + kBN - 1) / kBN;
    tile1 = max(tile1, tile0);
    if (plan.splits > 1) {
        const int n = tile1 - tile0;
        tile1 = tile0 + (int)((int64_t)n * (split + 1) / plan.splits);
        tile0 += (int)((int64_t)n * split / plan.splits);
    }
    const int NT = tile1 - tile0;

    // ---- codes -> LDS
    // item i of a wave is pieces 64 (w % 2) .. of group w / 2 % 2, w = wave + NW * i; K for w < 4 (of a thread: the same piece of K and V)
    const int n = (wave & 1) * 64 + l, gi = (wave & 3) >> 1;
    // K, D = 128: block n / 32 of key n % 32; D = 64: half n % 2 of block n / 64 of key n / 2 % 32.  Its scale's byte stands next to that of the key 16 apart.
    const int key = D == 128 ? n & 31 : (n >> 1) & 31, k_block = D == 128 ? n >> 5 : n >> 6;
    const int k_to = k_place<D>(32 * gi + key, D == 128 ? 4 * k_block : 4 * k_block + 2 * (n & 1)) * 2;      // bytes; its pieces of 8 channels: XOR 16 e
    // V, D = 128: chunk n / 64, keys 4q + b, 16 + 4q + b with q = n / 16 % 4, channels n % 16 + 16 (0 .. 3) of 64; D = 64: half of that
    const int c16 = D == 128 ? n : n >> 1, v_to = v_place((D == 128 ? 64 * (n >> 6) : 32 * (n & 1)) + (c16 & 15), 4 * gi + ((c16 >> 4) & 3)) * 2;
    auto tile_of = [&](int item, int set) { return wave + NW * item < 4 ? set + 1 : set; };
    Piece<kWords> held[kItems];
    // lane l: place of the item's group in tile 64 * k + l, in units of 128 bytes; ~0: the group is missing
    uint32_t places[kItems];
    bool missing = false;      // a group that some row sees is
    constexpr uint32_t kGroupUnits = paged_group_bytes(D) / 128;
    const uint32_t last_place = (uint32_t)(g.n_pages * g.Hkv * g.groups - 1) * kGroupUnits;
    auto find_places = [&](int i, int t) {
        const int64_t at = t + l < NT ? paged_group(g, b, s, ((tile0 + t + l) * 2 + gi) * kGroupTokens) : -1;
        places[i] = at < 0 ? ~0u : (uint32_t)(at + (int64_t)hk * g.groups) * kGroupUnits;
    };
    auto load_tile = [&](int i, int t, auto plain) {
        if (__builtin_expect((t & 63) == 0 && t > 0, 0)) find_places(i, t);
        const bool is_k = wave + NW * i < 4;
        uint32_t at = __builtin_amdgcn_readlane(places[i], t & 63);
        held[i].gone = !decltype(plain)::value && at == ~0u;
        at = min(at, last_place);      // a group that is missing: any other's bytes, which nobody sees
        const uint8_t* group = g.pages + ((uint64_t)at << 7);
        held[i].load(group + (is_k ? 0 : 16 * D) + n * (4 * kWords));
        held[i].extra = *(const uint16_t*)(group + (is_k ? 32 * D + k_block * 32 + (key & 15) * 2 : 33 * D + 2 * l32));
    };
    auto load_set = [&](int set) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int t = tile_of(i, set);
            if (t >= 0 && t < NT) load_tile(i, t, std::false_type());
        }
    };
    // The first loads are on their way together with the queries: the places of 64 tiles, then this wave's piece of tile 0.
    const int lead = late ? 2 : 1;      // a wave converts set t + lead in vector block t + 1
    find_places(0, 0);
    places[kItems - 1] = places[0];
    load_set(lead - 2);
    Frag qf[kTerms][KS];
    {
        const int r = min(row, rows - 1), i = r / g.G, h = r - i * g.G;
        const T* x = q + (v.first + i) * q_stride + (hk * g.G + h) * D + 8 * half;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if constexpr (kTerms == 1) {
                qf[0][ks].u = *(const u32x4_t*)(x + 16 * ks);
            } else {
                float y[8];
                *(float4*)y = *(const float4*)(x + 16 * ks);
                *(float4*)(y + 4) = *(const float4*)(x + 16 * ks + 4);
#pragma unroll
                for (int e = 0; e < 8; e += 2) split_terms(y[e], y[e + 1], [&](int term, uint32_t pair) { qf[term][ks].u[e / 2] = pair; });
            }
        }
    }
    wait_vm_fenced<0>();      // (or the products wait for the codes on their way as well)
    f32x16_t o[DB], st[2];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[db][j] = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < 16; ++j) st[kb][j] = 0.f;
    bool far = false;      // a row of the wave has come by a maximum of kFarLogit
    float top = kNoLogit, sum = 0.f;
    const float scale = g.scale * 1.44269504088896341f;

    // Whether anything in the range needs the careful form of a tile: a group that is missing (looked for here), a V row of NaN (seen when it is
    // converted).  It stays set: the fast form ends for the rest.
    auto absent = [&](int i, bool there) {      // group i of the range, seen by some row
        const int p = (2 * tile0 + i) * kGroupTokens;
        return i < 2 * NT && p < to_of(pos_of(row0 + kRows - 1)) && p + kGroupTokens > from_of(pos_of(row0)) && !there;
    };
    missing = absent(2 * l + gi, places[0] != ~0u);      // (the waves have both groups of 64 tiles)
    for (int i = 128 + tid; i < 2 * NT; i += NW * 64) missing |= absent(i, paged_group(g, b, s, (2 * tile0 + i) * kGroupTokens) >= 0);
    missing = __syncthreads_or(missing);
    if (tid == 0) special_lds = missing;
    {      // kept until the end, where a row without a logit asks for it
        bool sees = max(from, tile0 * kBN) < min(to, tile1 * kBN);
        if (missing && sees) sees = sees_a_key(g, b, s, pos, 2 * tile0, 2 * tile1);
        sees_lds[wave * 32 + l32] = sees ? 1.f : 0.f;
    }

    // (what no row sees is masked anyway, and the fast form leaves gone_lds as it is)
    auto is_gone = [&](int i, auto plain) { return !decltype(plain)::value && missing && held[i].gone; };
    auto write_codes = [&](int i, int stage, auto plain) {
        const Piece<kWords>& x = held[i];
        if (wave + NW * i < 4) {
            const float ks = scale_of_byte(x.extra >> (key >> 4) * 8 & 255u);
            char* to = (char*)&k_lds[0][0] + stage * (kBN * D * 2);
#pragma unroll
            for (int e = 0; e < kWords; ++e) *(u32x4_t*)(to + (k_to ^ (16 * e))) = bf16_of_codes(x.w[e], ks).u;
            return;
        }
        char* to = (char*)&v_lds[0][0] + stage * (kBN * D * 2) + v_to;
#pragma unroll
        for (int e = 0; e < kWords; e += 2) {
            const uint32_t a = x.w[e], c = x.w[e + 1];
            *(u32x4_t*)(to + 32 * e * kBN) = bf16_of_codes((a & 0x0F0F0F0Fu) | ((c << 4) & 0xF0F0F0F0u), 1.f).u;
            *(u32x4_t*)(to + 32 * (e + 1) * kBN) = bf16_of_codes(((a >> 4) & 0x0F0F0F0Fu) | (c & 0xF0F0F0F0u), 1.f).u;
        }
        if (wave & 1) return;
        // a NaN must not reach rows that do not see the key (0 * NaN): the scale becomes 0, and rows that do see it are marked
        const bool finite = (x.extra & 0x7F80u) != 0x7F80u, gone = is_gone(i, plain);
        vs_lds[stage][32 * gi + l32] = finite && !gone ? __uint_as_float(x.extra << 16) : 0.f;
        const uint32_t odd = gone ? 0u : (uint32_t)__ballot(!finite);      // lanes 32 .. 63 have the same scales
        if (__builtin_expect(odd != 0u, 0)) special_lds = 1;
        if (!decltype(plain)::value || __builtin_expect(odd != 0u, 0)) odd_lds[stage][gi] = odd;      // (0 as long as nothing was special)
    };
    auto write_set = [&](int set) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int t = tile_of(i, set);
            if (t < 0 || t >= NT) continue;
            write_codes(i, set & 1, std::false_type());
            if (wave + NW * i < 4 && !(wave & 1) && l == 0) gone_lds[set & 1][gi] = is_gone(i, std::false_type());
        }
    };

    // ---- blocks
    // tiles of whose keys all rows of the wave see all (that exist)
    const int w0 = (whole_from + kBN - 1) / kBN - tile0, w1 = whole_to / kBN - tile0;
    // Fragments of a matrix block, in the order of its products: 4 DB of V (16 keys of 32 channels), then 2 KS of K (16 channels of 32 keys).  Each
    // is read kAhead products before it is used, the first ones (of V) in the vector block before.
    constexpr int NV = 4 * DB, NF = NV + 2 * KS, kAhead = 6;
    // (Pieces two apart lie 32 bytes apart but for the row's XOR: one place for all.)
    const int v_lane = v_place(l32, half) * 2, k_lane = k_place<D>(l32, half) * 2;      // bytes
    auto read_frag = [&](int stage, int i) {
        Frag f;
        const char* v = (const char*)&v_lds[0][0] + stage * (kBN * D * 2);
        const char* k = (const char*)&k_lds[0][0] + stage * (kBN * D * 2);
        if (i < NV) f.u = *(const u32x4_t*)(v + (v_lane ^ (32 * (i / DB))) + (i % DB) * (64 * kBN));      // (rows 32 apart have the same order)
        else f.u = *(const u32x4_t*)(k + (k_lane ^ (32 * ((i - NV) >> 1))) + ((i - NV) & 1) * (64 * D));
        return f;
    };
    Frag fr[kAhead];
    float4 scales[2];      // V scales of the lane's keys 16 x .. of the tile, in the order of V's pieces
    uint32_t special = missing;
    auto read_scales = [&](int stage, int x) {
        scales[0] = *(const float4*)&vs_lds[stage][8 * (2 * x + half)];
        scales[1] = *(const float4*)&vs_lds[stage][8 * (2 * x + half) + 4];
    };
    auto read_ahead = [&](int stage) {
        if (NW == 8) special = special_lds;
        read_scales(stage, 0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fr[i] = read_frag(stage, i);
    };
    // probabilities of keys 16 x .. of the tile times their V scales, and their part of the row sum: here, between products, because the vector
    // block is the longer one
    auto scaled = [&](int x, Frag (&pf)[kTerms]) {
        const float a[4] = {scales[0].x, scales[0].y, scales[0].z, scales[0].w}, c[4] = {scales[1].x, scales[1].y, scales[1].z, scales[1].w};
        const int gi = x >> 1, sx = x & 1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p0 = st[gi][4 * sx + e] * a[e], p1 = st[gi][8 + 4 * sx + e] * c[e];
            sum += st[gi][4 * sx + e];
            sum += st[gi][8 + 4 * sx + e];
            if constexpr (kTerms == 1) pf[0].u[e] = cvt_pk_bf16(p0, p1);
            else split_terms(p0, p1, [&](int term, uint32_t pair) { pf[term].u[e] = pair; });
        }
    };
    // P V of tile t (its first fragments and scales are there), K Q^T of tile t + 1, from the stage of set t.  One form for all tiles: before a wave's
    // first tile the probabilities are 0 and V finite, behind its last nobody looks at the logits.  (Forms without the one or the other cost
    // copies of all outputs where they meet.)  Scales are asked for three products before they are used: LDS answers in order, so a wait for
    // them is a wait for all fragments asked for before.
    auto matrix_block = [&](int stage) {
        Frag pf[kTerms];
        scaled(0, pf);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const Frag f = fr[i % kAhead];
            if (i < NV) {
                const int x = i / DB;
                if (i % DB == 0 && x < 3) read_scales(stage, x + 1);
#pragma unroll
                for (int y = 0; y < kTerms; ++y) o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, pf[y].v, o[i % DB], 0, 0, 0);
                if (i % DB == DB - 1 && x < 3) scaled(x + 1, pf);
            } else {
                const int ks = (i - NV) >> 1, kb = (i - NV) & 1;
                if (ks == 0)
#pragma unroll
                    for (int j = 0; j < 16; ++j) st[kb][j] = 0.f;
#pragma unroll
                for (int y = 0; y < kTerms; ++y) st[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, qf[y][ks].v, st[kb], 0, 0, 0);
            }
            if (i + kAhead < NF) fr[i % kAhead] = read_frag(stage, i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // a row that sees a key whose V row is NaN
    auto mark_odd = [&](int t) {
        const uint32_t odd[2] = {odd_lds[t & 1][0], odd_lds[t & 1][1]};
        if (!__builtin_amdgcn_readfirstlane(odd[0] | odd[1])) return;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
            for (int r = 4 * half; r < 32; r += (r & 3) == 3 ? 5 : 1) {      // the lane's keys
                const int key = (tile0 + t) * kBN + 32 * kb + r;
                if ((odd[kb] >> v_slot(r) & 1u) && key >= from && key < to) sum = __uint_as_float(0x7FC00000u);
            }
    };
    auto mask = [&](int t) {      // what a row does not see
        const uint32_t gone[2] = {gone_lds[(t + 1) & 1][0], gone_lds[(t + 1) & 1][1]};      // (K of tile t is in set t - 1)
        if (t >= w0 && t < w1 && !__builtin_amdgcn_readfirstlane(gone[0] | gone[1])) return;
        const int key0 = (tile0 + t) * kBN;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int key = key0 + 32 * kb + 8 * (j >> 2) + 4 * half + (j & 3);
                if (gone[kb] || key < from || key >= to) st[kb][j] = -INFINITY;
            }
    };
    auto softmax = [&]() {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 16; ++j) mx = max_of(mx, st[kb][j]);
        mx *= scale;
        if (__ballot(mx > top + kRescaleLog2)) {
            const float now = max_of(top, max_xor32(mx));
            far |= __ballot(is_far(now)) != 0;
            const float shrink = __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= shrink;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[db][j] *= shrink;
        }
        if (__builtin_expect(far, 0))
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int j = 0; j < 16; ++j) st[kb][j] *= scale;
        const float unit = far ? 1.f : scale;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 16; ++j) st[kb][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][j], unit, -top));
    };

    // ---- the tiles
    for (int i = tid; i < kBN * D / 8; i += NW * 64) *(u32x4_t*)&v_lds[1][8 * i] = u32x4_t{0, 0, 0, 0};      // matrix block -1 multiplies them with 0
    if (tid < kBN) vs_lds[1][tid] = 0.f;
    if (tid < 2) odd_lds[1][tid] = 0;
    wait_lds_reads();
    wg_barrier();      // (special_lds as well: a wave that converts may set it)
    write_set(lead - 2);
    load_set(lead - 1);
    // the tiles that some row of the wave sees
    const int a0 = max(any_from / kBN - tile0, 0), a1 = min((any_to + kBN - 1) / kBN - tile0, NT);
    wait_lds_reads();
    wg_barrier();
    if (late) wg_barrier();
    if (NW == 8 && a0 == 0) read_ahead(1);
    // Tiles of whose successor all rows of the wave see all keys, with all keys of tile t + 3 there (the last tile may end in a group that does not exist): nothing
    // to test but whether something special came up.  (A wave
    // issues an instruction every five to six cycles whatever it is, and the vector block is the longer one.)
    const int plain0 = max(max(a0, w0) - 1, 0), plain1 = min(min(a1, w1) - 1, NT - 4);
    int t = -1;
    while (t < NT) {
        if (NW == 8 && t >= plain0 && t < plain1 && !__builtin_amdgcn_readfirstlane(special)) {
            do {
                __builtin_amdgcn_s_setprio(1);
                matrix_block(t & 1);
                __builtin_amdgcn_s_setprio(0);
                wg_barrier();
                write_codes(0, (t + lead) & 1, std::true_type());
                load_tile(0, t + 3, std::true_type());
                softmax();
                wait_lds_reads();
                ++t;
                read_ahead(t & 1);
                wg_barrier();
            } while (t < plain1 && !__builtin_amdgcn_readfirstlane(special));
        }
        if (t >= a0 - 1 && t < a1) {
            if (NW == 4) read_ahead(t & 1);      // (V of the tile is written in the vector block before)
            mark_odd(t);
            matrix_block(t & 1);
        }
        wg_barrier();      // (all that this wave has read from LDS is in the products)
        if (t + 1 < NT) {
            write_set(t + lead);
            load_set(t + lead + 1);
        }
        if (t + 1 >= a0 && t + 1 < a1) {
            mask(t + 1);
            softmax();
        }
        wait_lds_reads();      // what this wave has written is there
        ++t;
        if (NW == 8) read_ahead(t & 1);
        wg_barrier();
    }
    if (!late && NW == 8) wg_barrier();

    // ---- rows out: lane l has channels 32 db + 8 (j / 4) + 4 half + j % 4 of its row
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    float total = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    if (row >= rows) return;
    if (total == 0.f) total = sees_lds[wave * 32 + l32];      // (row_factor)
    if (plan.splits == 1) {
        const int i = row / g.G, h = row - i * g.G;
        T* y = out + ((int64_t)(v.first + i) * g.Hq + hk * g.G + h) * D + 4 * half;
        const float r = row_factor(top, total);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int j = 0; j < 16; j += 4) store4(y + 32 * db + 2 * j, o[db][j] * r, o[db][j + 1] * r, o[db][j + 2] * r, o[db][j + 3] * r);
    } else {
        const int64_t unit = (int64_t)(gridDim.x / g.Hkv - 1 - blockIdx.x / g.Hkv) * g.Hkv + hk;
        float* y = part + ((unit * plan.splits + split) * kRows + wave * 32 + l32) * (D + 2);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int j = 0; j < 16; j += 2) *(float2*)(y + 32 * db + 8 * (j >> 2) + 4 * half + (j & 3)) = make_float2(o[db][j], o[db][j + 1]);
        if (half == 0) *(float2*)(y + D) = make_float2(top, total);
    }
}

// Joins the splits: D/4 threads a row, four channels each.
template <typename T, int D> __global__ __launch_bounds__(256) void merge_chunk_kernel(PagedGeom g, PagedBatch b, ChunkPlan plan, int block_rows, const float* __restrict__ part, T* __restrict__ out)
{
    constexpr int kLanes = D / 4, kRowsHere = 256 / kLanes;
    const int unit = blockIdx.x, hk = blockIdx.y;
    int s, block;
    if (!find_row_block(g, b, plan, unit, block_rows, s, block)) return;
    const SeqView v = seq_view(b, s);
    const int in_block = blockIdx.z * kRowsHere + threadIdx.x / kLanes, row = block * block_rows + in_block, c = threadIdx.x % kLanes * 4;
    if (row >= v.n * g.G) return;
    const float* x = part + ((int64_t)(unit * g.Hkv + hk) * plan.splits * block_rows + in_block) * (D + 2);
    const int64_t step = (int64_t)block_rows * (D + 2);
    float top = kNoLogit;
    for (int i = 0; i < plan.splits; ++i) top = fmaxf(top, x[i * step + D]);
    float l = 0.f, o[4] = {};
    for (int i = 0; i < plan.splits; ++i) {
        const float m = x[i * step + D], f = __builtin_amdgcn_exp2f(m - top);
        const float2 a = *(const float2*)(x + i * step + c), e = *(const float2*)(x + i * step + c + 2);
        l += f * x[i * step + D + 1];
        o[0] += f * a.x;
        o[1] += f * a.y;
        o[2] += f * e.x;
        o[3] += f * e.y;
    }
    const int i = row / g.G, h = row - i * g.G;
    const float r = row_factor(top, l);
    store4(out + ((int64_t)(v.first + i) * g.Hq + hk * g.G + h) * D + c, o[0] * r, o[1] * r, o[2] * r, o[3] * r);
}

// Splits of a launch that has fewer row blocks than compute units: as many workgroups as there are of those, eight tiles each at least.
ChunkPlan chunk_plan(const PagedGeom& g, const PagedBatch& b, int few_rows, int block_rows)
{
    ChunkPlan p;
    p.few_rows = few_rows;
    // a sequence's last block may be short
    p.units = (int)(((int64_t)b.n_tokens * g.G + block_rows - 1) / block_rows) + b.n_seqs;
    const int64_t longest = g.window && g.window < b.max_length - b.max_new ? g.window + b.max_new + kBN : b.max_length;
    const int64_t tiles = longest / kBN + 1, pairs = (int64_t)(p.units - b.n_seqs + (b.n_seqs + 1) / 2) * g.Hkv;
    int64_t n = 256 / pairs;
    if (n > tiles / 8) n = tiles / 8;
    const int64_t most = (int64_t)kChunkPartRows / ((int64_t)p.units * g.Hkv * block_rows);
    if (n > most) n = most;
    p.splits = n < 1 ? 1 : (int)n;
    return p;
}

void launch_attend_chunk(const PagedGeom& g, const PagedBatch& b, int few_rows, const void* q, int64_t q_stride, void* out, void* scratch, int dtype, hipStream_t s)
{
    with_paged_form(dtype, g.d, [&](auto f) {
        typedef typename decltype(f)::Elt T;
        constexpr int D = decltype(f)::d, NW = sizeof(T) == 2 ? 8 : 4;
        const ChunkPlan p = chunk_plan(g, b, few_rows, 32 * NW);
        hipLaunchKernelGGL((attend_chunk_kernel<T, D, NW>), dim3(p.units * g.Hkv, p.splits), dim3(NW * 64), 0, s, g, b, p, (const T*)q, q_stride, (T*)out, (float*)scratch);
        if (p.splits > 1)
            hipLaunchKernelGGL((merge_chunk_kernel<T, D>), dim3(p.units, g.Hkv, 32 * NW * D / 1024), dim3(256), 0, s, g, b, p, 32 * NW, (const float*)scratch, (T*)out);
    });
}

}  // namespace ckv
