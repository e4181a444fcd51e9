// esb_attention.cu -- attention over a cache of 4-bit codes: which kernel a
// call takes, and its arguments.
#include <cmath>

#include "esb_attention.cuh"

namespace esb {

namespace {

// Eights of rows in a tile: those of an average sequence, as far as their sums fit the registers.
int eights_of(int64_t tokens, int64_t seqs, int group, int most)
{
    const int64_t rows = (tokens + seqs - 1) / seqs * group;
    return rows <= 8 || most == 1 ? 1 : (rows <= 16 || most == 2 ? 2 : 4);
}
// Planes of queries and weights, 11 bits each.  One for bf16 queries: it puts outputs
// 4e-4 of their size off, a quarter of what rounding them to bf16 does (1.7e-3, root mean
// squares over 4 x 131072 places and 24 x 10000), and bf16 outputs 1.1e-3 from those of
// fp32 arithmetic: some differ in their last place.  Two planes leave 4e-5 of that,
// but take 171 us for 4 x 131072 places (134 with one), 55 for a draft of four tokens
// (45), 975 for a prompt's part (614): they are for queries of more bits.
int planes(int q_type) { return q_type == ESB_BF16 ? 1 : 2; }

// High bytes of the fp16 numbers of codes 0..7 of a 4-bit set.
uint2 lut_of(int k)
{
    uint32_t w[2] = {0u, 0u};
    const int n = (1 << (3 - k)) - 1;
    for (int c = 0; c < 8; c++) {
        const int e = (c >> k) & n, f = c & ((1 << k) - 1);
        const double v = e == n ? std::ldexp((double)f, -k) : std::ldexp(1.0 + std::ldexp((double)f, -k), e);
        uint32_t h = 0u;
        if (v > 0.0) {
            int x;
            const double m = std::frexp(v, &x) * 2.0 - 1.0;     // v = (1 + m) 2^(x - 1)
            h = (uint32_t)((x - 1 + 15) << 2) | (uint32_t)(m * 4.0);
        }
        w[c / 4] |= h << (8 * (c % 4));
    }
    return make_uint2(w[0], w[1]);
}

}  // namespace

size_t attention_workspace_bytes(int64_t tokens, int64_t seqs, int q_heads, int heads, int head_dim, int q_type)
{
    const int p = planes(q_type), group = q_heads / heads;
    if (head_dim <= 64) return attention_bytes_64(eights_of(tokens, seqs, group, attention_most_64(p)), p);
    if (head_dim <= 128) return attention_bytes_128(eights_of(tokens, seqs, group, attention_most_128(p)), p);
    return attention_bytes_256(eights_of(tokens, seqs, group, attention_most_256(p)), p);
}

cudaError_t launch_attention(int64_t tokens, const esb_kv_cache& c, const esb_attention& n, void* workspace, cudaStream_t st)
{
    AttnArgs a = {};
    auto rows16 = [](const void* p, int64_t ld, int type) {
        return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
    };
    a.q = n.q; a.ldq = n.ldq; a.out = n.out; a.ldo = n.ldo; a.lse = n.lse;
    a.starts = n.starts; a.lens = n.lens; a.pages = n.pages; a.ld_pages = n.ld_pages; a.tokens = tokens;
    a.kc = c.k_codes; a.vc = c.v_codes; a.ks = c.k_scales; a.vs = c.v_scales;
    a.npages = c.pages; a.page16 = (uint32_t)(c.page_ld / 4); a.page_lds = (uint32_t)c.page_lds;
    const bool lin = c.k_fmt.k >= 2 && c.v_fmt.k >= 2;
    // places of k = 2 are their codes with the top bit changed; a place counts 2^-16, and stands for 2^-k
    a.klut = lin ? make_uint2(c.k_fmt.k == 2 ? 0x04040404u : 0u, 0u) : lut_of(c.k_fmt.k);
    a.vlut = lin ? make_uint2(c.v_fmt.k == 2 ? 0x04040404u : 0u, 0u) : lut_of(c.v_fmt.k);
    a.vunit = (lin ? (float)(1 << (16 - c.v_fmt.k)) : 1.0f) / kWeightUp;
    a.seqs = n.seqs; a.max_pages = n.max_pages; a.heads = c.heads; a.group = n.q_heads / c.heads; a.D = c.head_dim;
    a.chunks = (c.head_dim + 31) / 32; a.page_size = c.page_size;
    a.group_shift = -1;
    for (int i = 0; i < 24; i++)
        if (a.group == 1 << i) a.group_shift = i;
    a.window = n.window; a.q_type = n.q_type; a.out_type = n.out_type;
    a.qvec = rows16(n.q, n.ldq, n.q_type); a.ovec = rows16(n.out, n.ldo, n.out_type);
    a.scale2 = (float)std::frexp((double)n.scale * 1.4426950408889634, &a.scale_up);
    a.scale_up += lin ? 16 - c.k_fmt.k : 0;
    a.rot = make_rot(n.rotation, c.head_dim);
    const int p = planes(n.q_type);
    if (a.D <= 64) return attention_run_64(a, eights_of(tokens, n.seqs, a.group, attention_most_64(p)), p, lin, workspace, st);
    if (a.D <= 128) return attention_run_128(a, eights_of(tokens, n.seqs, a.group, attention_most_128(p)), p, lin, workspace, st);
    return attention_run_256(a, eights_of(tokens, n.seqs, a.group, attention_most_256(p)), p, lin, workspace, st);
}

}  // namespace esb
