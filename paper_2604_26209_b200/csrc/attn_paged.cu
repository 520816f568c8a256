// hpd_attn_decode_paged: one warp per (row, query head) over the document's pages and the branch's page, online softmax in fp32.
#include "common.cuh"
#include "paged.cuh"

namespace hpd {

namespace {

template <int D>
__global__ void __launch_bounds__(256)
attn_paged_kernel(const PagedArgs p, float scale)
{
    constexpr int E = D / 32;
    const int Hq = p.a.g.Hq, Hkv = p.a.g.Hkv, G = Hq / Hkv, lane = threadIdx.x & 31;
    const int64_t w = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (w >= static_cast<int64_t>(min(*p.a.n_active, p.a.max_rows)) * Hq) return;
    const int r = static_cast<int>(w / Hq), h = static_cast<int>(w % Hq), kh = h / G;
    float q[E], acc[E], m = -INFINITY, l = 0.f;
    bool bad = false;
    for (int e = 0; e < E; ++e) {
        q[e] = __bfloat162float(p.a.q[w * D + lane * E + e]);
        acc[e] = 0.f;
        bad |= !(fabsf(q[e]) < INFINITY);
    }
    bad = __any_sync(0xffffffffu, bad);
    auto token = [&](const uint8_t* k, const uint8_t* v, float ks, float vs) {
        float s = 0.f;
        for (int e = 0; e < E; ++e) s = fmaf(q[e], e4m3x2_value(k[lane * E + e]).x, s);
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        s *= ks * scale;
        const float mn = fmaxf(m, s), f = m == -INFINITY ? 0.f : exp2f((m - mn)), pr = exp2f(s - mn);
        l = l * f + pr;
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + pr * e4m3x2_value(v[lane * E + e]).x * vs;
        m = mn;
    };
    const int d = p.a.doc_id[r];
    int status = 0;
    for (int t = 0; t < p.a.doc_prefix_len[d]; ++t) {
        const int i = t / p.page_size;
        const int page = i < p.pages_per_doc ? p.page_table[static_cast<int64_t>(d) * p.pages_per_doc + i] : -1;
        if (page < 0 || page >= p.n_pages) { status = HPD_S_BAD_TABLE; bad = true; break; }
        const int64_t ph = static_cast<int64_t>(page) * Hkv + kh, at = (ph * p.page_size + t % p.page_size) * D;
        token(p.page_k + at, p.page_v + at, e8m0_value(p.scale_k[ph]), e8m0_value(p.scale_v[ph]));
    }
    const int n = max(0, min(p.a.suffix_len[r] + p.a.suffix_extra, p.a.g.suffix_cap));
    const int slot = p.a.active_slot[r];
    const int page = slot >= 0 && slot < p.a.n_slots ? p.slot_page[slot] : -1;
    if (n > 0 && (page < 0 || page >= p.n_branch_pages)) {
        status = HPD_S_BAD_TABLE;
    } else {
        const int64_t ph = static_cast<int64_t>(page) * Hkv + kh;
        for (int t = 0; t < n; ++t) {
            const int64_t at = (ph * p.a.g.suffix_cap + t) * D;
            bool nan = false;
            for (int e = 0; e < E; ++e) nan |= (p.branch_v[at + lane * E + e] & 0x7f) == 0x7f;
            bad |= __any_sync(0xffffffffu, nan) != 0;
            token(p.branch_k + at, p.branch_v + at, e8m0_value(p.branch_scale_k[ph]), e8m0_value(p.branch_scale_v[ph]));
        }
    }
    if (status && lane == 0 && p.a.dev_status) atomicOr(p.a.dev_status, status);
    for (int e = 0; e < E; ++e) p.a.o[w * D + lane * E + e] = __float2bfloat16(bad ? NAN : l > 0.f || l != l ? acc[e] / l : 0.f);
    if (p.a.lse && lane == 0) p.a.lse[w] = bad ? NAN : l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

int launch_attn_paged(const PagedArgs& p)
{
    const unsigned blocks = static_cast<unsigned>((static_cast<long long>(p.a.max_rows) * p.a.g.Hq + 7) / 8);
    const float scale = p.a.g.sm_scale * 1.4426950408889634f;
    if (p.a.g.D == 128) attn_paged_kernel<128><<<blocks, 256, 0, p.a.stream>>>(p, scale);
    else attn_paged_kernel<64><<<blocks, 256, 0, p.a.stream>>>(p, scale);
    HPD_CUDA_TRY(cudaGetLastError());
    return HPD_OK;
}

}  // namespace hpd
