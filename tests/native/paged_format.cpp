// The places and numbers of the paged cache (csrc/paged_format.h) on the host: every byte that a token of a valid page takes is inside its group and its own, batches of any
// content lead to no access outside the arrays, and the numbers obey their definitions.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <random>
#include <vector>

#include "../../paper_2406_17808_amd/csrc/paged_format.h"

using namespace ckv;

static int g_failed = 0;
#define CHECK(x)                                                       \
    do {                                                               \
        if (!(x)) {                                                    \
            if (g_failed++ < 10) printf("line %d: %s\n", __LINE__, #x); \
        }                                                              \
    } while (0)

static void bytes_of_a_group(int d)
{
    std::vector<int> owner(paged_group_bytes(d), -1);
    auto take = [&](int at, int r) {
        CHECK(at >= 0 && at < (int)owner.size());
        if (at < 0 || at >= (int)owner.size()) return;
        CHECK(owner[at] == -1);      // no byte has two tokens, or two uses
        owner[at] = r;
    };
    for (int r = 0; r < 32; ++r) {
        for (int c = 0; c < d; c += 2) take(k_code_byte(c, r), r);
        for (int u = 0; u < d / 32; ++u)
            for (int m = 0; m < 16; ++m) take(v_code_byte(d, u, m, r), r);
        for (int blk = 0; blk < d / 32; ++blk) take(k_exp_byte(d, blk, r), r);
        take(v_scale_byte(d, r), r);
        take(v_scale_byte(d, r) + 1, r);
    }
    CHECK(paged_group_bytes(d) % 128 == 0);
}

static int any_int(std::mt19937& rng)
{
    switch (rng() % 6) {
    case 0: return (int)(rng() % 8);
    case 1: return -(int)(rng() % 8);
    case 2: return 0x7FFFFFFF - (int)(rng() % 3);
    case 3: return (int)0x80000000u + (int)(rng() % 3);
    case 4: return (int)(rng() % 2000);
    default: return (int)rng();
    }
}

static void batches_of_any_content(int seed)
{
    std::mt19937 rng(seed);
    PagedGeom g;
    memset(&g, 0, sizeof(g));
    g.d = rng() % 2 ? 64 : 128;
    g.Hkv = 1 + rng() % 4;
    g.groups = 1 + rng() % 5;
    g.page_size = 32 * g.groups;
    g.group_bytes = paged_group_bytes(g.d);
    g.n_pages = 1 + rng() % 9;
    PagedBatch b;
    b.n_seqs = 1 + rng() % 5;
    b.n_tokens = 1 + rng() % 50;
    b.max_new = 1 + rng() % b.n_tokens;
    b.max_length = rng() % 3 ? rng() % 500 : 0x7FFFFFFF - (1 << 20);
    b.table_stride = rng() % 7;
    std::vector<int32_t> lengths(b.n_seqs), offsets(b.n_seqs + 1), table(b.n_seqs * b.table_stride);
    for (auto& x : lengths) x = any_int(rng);
    for (auto& x : offsets) x = any_int(rng);
    for (auto& x : table) x = any_int(rng);
    b.lengths = lengths.data();
    b.offsets = offsets.data();
    b.table = table.data();
    std::vector<uint8_t> pages((size_t)g.n_pages * g.Hkv * g.groups * g.group_bytes);
    for (int s = 0; s < b.n_seqs; ++s) {
        const SeqView v = seq_view(b, s);
        CHECK(v.len >= 0 && v.len <= b.max_length);
        CHECK(v.n >= 0 && v.n <= b.max_new && v.first >= 0 && v.first + v.n <= b.n_tokens);
        for (int i = 0; i < v.n; ++i) {
            const int p = v.len + i;      // no overflow: max_length leaves room for the tokens of a call
            const int64_t at = paged_group(g, b, s, p);
            CHECK(at >= -1);
            if (at < 0) continue;
            for (int h = 0; h < g.Hkv; ++h) {
                const int64_t group = (at + (int64_t)h * g.groups) * g.group_bytes;
                CHECK(group >= 0 && group + g.group_bytes <= (int64_t)pages.size());
                if (group >= 0 && group + g.group_bytes <= (int64_t)pages.size()) pages[group + v_scale_byte(g.d, p & 31) + 1] = 1;
            }
        }
        CHECK(paged_group(g, b, s, -1) == -1 && paged_group(g, b, s, b.max_length) == -1);
    }
}

static void numbers()
{
    const double mag[8] = {0, .5, 1, 1.5, 2, 3, 4, 6};
    for (uint32_t c = 0; c < 16; ++c) CHECK(fp4_value(c) == (c & 8 ? -mag[c & 7] : mag[c & 7]) && fp4_value(c | 0xF0u) == fp4_value(c));
    std::mt19937_64 rng(7);
    for (int i = 0; i < 200000; ++i) {
        double y = ldexp((double)(int64_t)rng(), -63) * 8.0;
        if (i % 3 == 0) y = rint(y * 8) / 8;      // on the borders
        const uint32_t c = fp4_code(y, 1.0);
        const double a = fabs(y), off = fabs(a - mag[c & 7]);
        for (int k = 0; k < 8; ++k) CHECK(off < fabs(a - mag[k]) || k == (int)(c & 7) || (off == fabs(a - mag[k]) && c % 2 == 0));
        CHECK((c >> 3) == (y < 0 ? 1u : 0u));
        CHECK(fp4_code((float)y, 1.f) == fp4_code((double)(float)y, 1.0));
        const double top = ldexp(fabs(y) + 0.01, (int)(rng() % 200) - 100);
        const uint32_t byte = k_exponent(top);
        CHECK(byte >= 1 && byte <= 254 && top <= 7 * ldexp(1, (int)byte - 127) && top > 7 * ldexp(1, (int)byte - 128));
        CHECK(k_exponent(7 * ldexp(1, (int)byte - 127)) == byte && k_exponent(nextafter(7 * ldexp(1, (int)byte - 127), 1e300)) == byte + 1);
    }
    CHECK(k_exponent(0.0) == 0 && k_exponent(INFINITY) == 255 && k_exponent(NAN) == 255 && k_exponent(1e-60) == 1 && k_exponent(3.4e38) == 127 + 126);
    CHECK(k_scale(0) == 0.f && k_scale(127) == 1.f && k_scale(1) == ldexpf(1, -126) && isnan(k_scale(255)));
    CHECK(v_scale_bits(0.f) == 0 && v_scale_bits(6.f) == 0x3F80 && v_scale_bits(INFINITY) == 0x7FC0 && v_scale_bits(NAN) == 0x7FC0 && v_scale_bits(1e-35f) == 0);
    // what the kernels round to a code: a float on the same side of every border as the 64-bit number
    for (int i = 0; i < 200000; ++i) {
        const int e = (int)(rng() % 253) - 126;
        const double border = rint(ldexp((double)(rng() >> 1), -63) * 28) / 4;
        const double y = i % 4 == 0 ? border : i % 4 == 1 ? nextafter(border, 9) : i % 4 == 2 ? nextafter(border, -1) : ldexp((double)(rng() >> 1), -63) * 7;
        const uint32_t bits = k_scaled_bits(k_key(ldexp(y, e)), (uint32_t)(e + 127));
        CHECK(y < 0 || fp4_code((double)f32_from_bits(bits), 1.0) == fp4_code(y, 1.0));
    }
    CHECK(k_scaled_bits(k_key(INFINITY), 255) == 0 && k_scaled_bits(k_key(0.0), 0) == 0 && k_scaled_bits(k_key(1e-300), 200) == 0);
}

int main()
{
    bytes_of_a_group(64);
    bytes_of_a_group(128);
    for (int seed = 0; seed < 3000; ++seed) batches_of_any_content(seed);
    numbers();
    printf("%d failed\n", g_failed);
    return g_failed != 0;
}
