// hpd_append_paged: new keys and values into pages of 8-bit codes, with the rotary embedding on the way.
//
// For the tokens that one call puts into one page, per kv head and for K and V each:
//     a = largest finite magnitude of the new tokens' elements (keys: rotated and rounded to bf16, the bits of hpd_rope)
//     n = smallest integer >= -126 with a <= 448 * 2^n
//     e = n for a page that held no token, else max(n, e of before); codes held before become e4m3(code * 2^(e_before - e))
//     new codes = e4m3(x * 2^-e)
// With powers of two as scales the growth of a scale is exact for every code that stays a normal number, so a page that fills up
// token by token ends with the codes of one that is filled at once, but for elements below 2^-14 of the largest.
//
// HBM bound: a token's q, k and v are read once, the codes written once; what a page holds is read only where its scale grows.
// Ordinary launches: the kernels before have ended when these start.
#include <algorithm>

#include "common.cuh"
#include "paged.cuh"
#include "rotary.cuh"

namespace hpd {

namespace {

struct PageArgs {
    int n_seqs, max_rows, table_rows, pages_per_seq, n_pages, page_size;
    const int32_t *n_rows, *row_seq, *seq_row_start, *seq_id, *seq_len, *page_table, *pos_id;
    const __nv_bfloat16* q;
    __nv_bfloat16* q_rot;
    const __nv_bfloat16 *k_new, *v_new;
    uint8_t *page_k, *page_v, *scale_k, *scale_v;
    int32_t* dev_status;
};

// a chunk pair: 8 elements of the low half of a head and their 8 partners of the high half
struct Chunk { uint4 lo, hi; };

template <int D> __device__ __forceinline__ Chunk load_chunk(const __nv_bfloat16* head, int ch)
{
    const uint4* p = reinterpret_cast<const uint4*>(head) + ch;
    return {p[0], p[D / 16]};
}
template <int D> __device__ __forceinline__ void store_chunk(__nv_bfloat16* head, int ch, const Chunk& c)
{
    uint4* p = reinterpret_cast<uint4*>(head) + ch;
    p[0] = c.lo; p[D / 16] = c.hi;
}
// the operations of hpd_rope in its order: the same bits
__device__ __forceinline__ void rotate_chunk(Chunk& c, const float* cs, const float* sn)
{
    uint32_t* l = reinterpret_cast<uint32_t*>(&c.lo);
    uint32_t* h = reinterpret_cast<uint32_t*>(&c.hi);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int i = w * 2;
        const float a0 = bf16lo(l[w]), a1 = bf16hi(l[w]);
        const float b0 = bf16lo(h[w]), b1 = bf16hi(h[w]);
        l[w] = pack_bf16(fmaf(a0, cs[i], -b0 * sn[i]), fmaf(a1, cs[i + 1], -b1 * sn[i + 1]));
        h[w] = pack_bf16(fmaf(b0, cs[i], a0 * sn[i]), fmaf(b1, cs[i + 1], a1 * sn[i + 1]));
    }
}
__device__ __forceinline__ int chunk_top(const Chunk& c)
{
    int top = 0;
    const uint32_t* l = reinterpret_cast<const uint32_t*>(&c.lo);
    const uint32_t* h = reinterpret_cast<const uint32_t*>(&c.hi);
#pragma unroll
    for (int w = 0; w < 4; ++w) { top = max_finite(top, l[w]); top = max_finite(top, h[w]); }
    return top;
}
__device__ __forceinline__ uint2 codes8(const uint4& x, float inv)
{
    return make_uint2(e4m3x4(bf16lo(x.x) * inv, bf16hi(x.x) * inv, bf16lo(x.y) * inv, bf16hi(x.y) * inv),
                      e4m3x4(bf16lo(x.z) * inv, bf16hi(x.z) * inv, bf16lo(x.w) * inv, bf16hi(x.w) * inv));
}
template <int D> __device__ __forceinline__ void store_codes(uint8_t* token, int ch, const Chunk& c, float inv)
{
    *reinterpret_cast<uint2*>(token + ch * 8) = codes8(c.lo, inv);
    *reinterpret_cast<uint2*>(token + D / 2 + ch * 8) = codes8(c.hi, inv);
}
// codes held before, 16 at a time, for a scale that has grown from `was` to `now`
__device__ __forceinline__ void rescale16(uint8_t* p, int was, int now)
{
    const float f = now - was < 127 ? __uint_as_float(static_cast<uint32_t>(127 - (now - was)) << 23) : 0.f;
    uint4 w = *reinterpret_cast<const uint4*>(p);
    w.x = e4m3x4_times(w.x, f); w.y = e4m3x4_times(w.y, f); w.z = e4m3x4_times(w.z, f); w.w = e4m3x4_times(w.w, f);
    *reinterpret_cast<uint4*>(p) = w;
}

// Page of token `index` of table row `entry`: -1 and a status bit where there is none.
__device__ __forceinline__ int page_of(const PageArgs& p, int entry, int64_t index, bool report)
{
    int bits = 0, page = -1;
    if (entry < 0 || entry >= p.table_rows || index < 0) {
        bits = HPD_S_BAD_TABLE;
    } else if (index >= static_cast<int64_t>(p.pages_per_seq) * p.page_size) {
        bits = HPD_S_OVERFLOW;
    } else {
        page = p.page_table[static_cast<int64_t>(entry) * p.pages_per_seq + index / p.page_size];
        if (page < 0 || page >= p.n_pages) { page = -1; bits = HPD_S_BAD_TABLE; }
    }
    if (bits && report && p.dev_status) atomicOr(p.dev_status, bits);
    return page;
}

// ------------------------------------------------------------------------------------------------
// One token per sequence: the decode step.  Row r is sequence r's token.
// ------------------------------------------------------------------------------------------------
constexpr int kStepThreads = 128, kStepRows = 2, kStepBatch = 3;

template <int D>
__global__ void __launch_bounds__(kStepThreads)
append_step_kernel(int Hq /* 0: no queries */, int Hkv, const InvFreq inv_freq, const PageArgs p)
{
    constexpr int HALF = D / 2, CH = D / 16;         // chunk pairs of a head: CH consecutive lanes
    __shared__ float cs[kStepRows][HALF], sn[kStepRows][HALF];
    __shared__ int s_page[kStepRows], s_slot[kStepRows];
    const int r0 = blockIdx.x * kStepRows;
    const int part = blockIdx.y, parts = gridDim.y;  // the CTAs of a row pair take turns at its batches of kStepThreads chunk pairs
    const int n = min(*p.n_rows, min(p.max_rows, p.n_seqs));
    if (r0 >= n) return;
    const int nr = min(kStepRows, n - r0);
    const int items = (2 * Hkv + Hq) * CH;           // of one row: its keys, its values, its queries
    const int total = nr * items;
    auto source = [&](int it, int& row, int& head, int& ch) -> const __nv_bfloat16* {
        row = it / items;
        const int local = it - row * items;
        head = local / CH; ch = local - head * CH;
        const int64_t r = r0 + row;
        if (head < Hkv) return p.k_new + (r * Hkv + head) * D;
        if (head < 2 * Hkv) return p.v_new + (r * Hkv + head - Hkv) * D;
        return p.q + (r * Hq + head - 2 * Hkv) * D;
    };
    Chunk c[kStepBatch];
    auto fetch = [&](int base) {
#pragma unroll
        for (int k = 0; k < kStepBatch; ++k) {
            const int it = base + threadIdx.x + (k * parts + part) * kStepThreads;
            if (it < total) {
                int row, head, ch;
                const __nv_bfloat16* src = source(it, row, head, ch);
                c[k] = load_chunk<D>(src, ch);
            }
        }
    };
    fetch(0);
    if (threadIdx.x < nr) {
        const int r = r0 + threadIdx.x;
        const int entry = p.seq_id ? p.seq_id[r] : r;
        const int index = p.seq_len[r];
        s_page[threadIdx.x] = page_of(p, entry, index, part == 0);
        s_slot[threadIdx.x] = index % p.page_size;
    }
    const int ar = threadIdx.x / HALF, ai = threadIdx.x % HALF;
    if (p.pos_id && ar < nr) rotary_angle(p.pos_id[r0 + ar], inv_freq.f[ai], cs[ar][ai], sn[ar][ai]);
    __syncthreads();
    for (int base = 0; base < total; base += kStepBatch * parts * kStepThreads) {
        if (base > 0) fetch(base);
#pragma unroll
        for (int k = 0; k < kStepBatch; ++k) {
            const int it = base + threadIdx.x + (k * parts + part) * kStepThreads;
            if (it >= total) continue;
            int row, head, ch;
            (void)source(it, row, head, ch);
            const bool is_v = head >= Hkv && head < 2 * Hkv;
            if (p.pos_id && !is_v) rotate_chunk(c[k], cs[row] + ch * 8, sn[row] + ch * 8);
            if (head >= 2 * Hkv) {
                store_chunk<D>(p.q_rot + (static_cast<int64_t>(r0 + row) * Hq + head - 2 * Hkv) * D, ch, c[k]);
                continue;
            }
            // a head's CH lanes, a group inside the warp, agree on its scale
            const unsigned group = (CH == 32 ? 0xffffffffu : ((1u << CH) - 1u)) << (threadIdx.x & 31 & ~(CH - 1));
            int top = chunk_top(c[k]);
#pragma unroll
            for (int s = 1; s < CH; s <<= 1) top = max(top, __shfl_xor_sync(group, top, s));
            const int page = s_page[row], slot = s_slot[row];
            if (page < 0) continue;
            const int64_t ph = static_cast<int64_t>(page) * Hkv + (is_v ? head - Hkv : head);
            uint8_t* scale = (is_v ? p.scale_v : p.scale_k) + ph;
            uint8_t* codes = (is_v ? p.page_v : p.page_k) + ph * p.page_size * D;
            int now = e8m0_needed(top);
            if (slot > 0) {
                const int was = *scale;
                if (now > was) {
                    // 16 codes a lane: token by token, D/16 = CH lanes each
                    for (int t = 0; t < slot; ++t) rescale16(codes + static_cast<int64_t>(t) * D + ch * 16, was, now);
                } else {
                    now = was;
                }
                __syncwarp(group);                   // every lane of the group has the old scale
            }
            store_codes<D>(codes + static_cast<int64_t>(slot) * D, ch, c[k], e8m0_inverse(now));
            if (ch == 0) *scale = static_cast<uint8_t>(now);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Any number of tokens per sequence: prompts and chunks.  The rows of a sequence that go into one page are a segment; a CTA takes
// the segments that begin in its window of page_size rows, for every gridDim.y-th kv head and that head's queries.
// ------------------------------------------------------------------------------------------------
constexpr int kTokThreads = 256, kTokRows = 64, kTokQueries = 4;

template <int D>
__global__ void __launch_bounds__(kTokThreads)
append_tokens_kernel(int Hq /* 0: no queries */, int Hkv, const InvFreq inv_freq, const PageArgs p)
{
    constexpr int HALF = D / 2, CH = D / 16;
    constexpr int B = kTokRows * CH / kTokThreads;   // chunk pairs of one head's keys (or values) a thread holds
    __shared__ float cs[kTokRows][HALF], sn[kTokRows][HALF];
    __shared__ int s_top[2][kTokThreads / 32];
    const int n = min(*p.n_rows, p.max_rows);
    const int P = p.page_size, G = Hq / Hkv;
    const int64_t lo = static_cast<int64_t>(blockIdx.x) * P;
    const int end = static_cast<int>(min(lo + P, static_cast<int64_t>(n)));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int r = static_cast<int>(min(lo, static_cast<int64_t>(n))), stop; r < end; r = stop) {
        // ---- the segment that begins at row r, or the rest of one that another window has ----
        const int seq = p.row_seq[r];
        int page = -1, slot = 0;
        stop = r + 1;
        if (seq < 0 || seq >= p.n_seqs || r < p.seq_row_start[seq] || r >= p.seq_row_start[seq + 1]) {
            if (threadIdx.x == 0 && blockIdx.y == 0 && p.dev_status) atomicOr(p.dev_status, HPD_S_BAD_TABLE);
        } else {
            const int first = p.seq_row_start[seq], past = min(p.seq_row_start[seq + 1], n);
            const int64_t index = static_cast<int64_t>(p.seq_len[seq]) + (r - first);
            slot = static_cast<int>(index < 0 ? 0 : index % P);
            stop = min(past, r + P - slot);
            if (r != first && slot != 0) continue;
            page = page_of(p, p.seq_id ? p.seq_id[seq] : seq, index, threadIdx.x == 0 && blockIdx.y == 0);
        }
        const int rows = stop - r;
        if (p.pos_id) {
            __syncthreads();                         // the angles of the segment before have been used
            for (int i = threadIdx.x; i < rows * HALF; i += kTokThreads) {
                const int t = i / HALF, a = i % HALF;
                rotary_angle(p.pos_id[r + t], inv_freq.f[a], cs[t][a], sn[t][a]);
            }
            __syncthreads();
        }
        for (int h = blockIdx.y; h < Hkv; h += gridDim.y) {
            if (page >= 0) {
                Chunk k[B], v[B];
                bool mine[B];                        // rows that the two tables agree on
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const int it = threadIdx.x + b * kTokThreads, t = it / CH;
                    mine[b] = t < rows && p.row_seq[r + t] == seq;
                    if (t < rows && !mine[b] && h == 0 && p.dev_status) atomicOr(p.dev_status, HPD_S_BAD_TABLE);
                    if (t < rows) {
                        const int64_t at = (static_cast<int64_t>(r + t) * Hkv + h) * D;
                        k[b] = load_chunk<D>(p.k_new + at, it % CH);
                        v[b] = load_chunk<D>(p.v_new + at, it % CH);
                    }
                }
                const int64_t ph = static_cast<int64_t>(page) * Hkv + h;
                const int was_k = slot > 0 ? p.scale_k[ph] : 0, was_v = slot > 0 ? p.scale_v[ph] : 0;
                int top_k = 0, top_v = 0;
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const int it = threadIdx.x + b * kTokThreads, t = it / CH;
                    if (mine[b]) {
                        if (p.pos_id) rotate_chunk(k[b], cs[t] + it % CH * 8, sn[t] + it % CH * 8);
                        top_k = max(top_k, chunk_top(k[b]));
                        top_v = max(top_v, chunk_top(v[b]));
                    }
                }
                top_k = __reduce_max_sync(0xffffffffu, top_k);
                top_v = __reduce_max_sync(0xffffffffu, top_v);
                if (lane == 0) { s_top[0][warp] = top_k; s_top[1][warp] = top_v; }
                __syncthreads();                     // ... and everybody has the scales of before
#pragma unroll
                for (int w = 0; w < kTokThreads / 32; ++w) { top_k = max(top_k, s_top[0][w]); top_v = max(top_v, s_top[1][w]); }
                const int now_k = max(e8m0_needed(top_k), was_k), now_v = max(e8m0_needed(top_v), was_v);
                uint8_t* codes_k = p.page_k + ph * P * D;
                uint8_t* codes_v = p.page_v + ph * P * D;
                if (now_k > was_k)
                    for (int i = threadIdx.x; i < slot * (D / 16); i += kTokThreads) rescale16(codes_k + i * 16, was_k, now_k);
                if (now_v > was_v)
                    for (int i = threadIdx.x; i < slot * (D / 16); i += kTokThreads) rescale16(codes_v + i * 16, was_v, now_v);
                const float inv_k = e8m0_inverse(now_k), inv_v = e8m0_inverse(now_v);
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const int it = threadIdx.x + b * kTokThreads, t = it / CH;
                    if (mine[b]) {
                        store_codes<D>(codes_k + (slot + t) * D, it % CH, k[b], inv_k);
                        store_codes<D>(codes_v + (slot + t) * D, it % CH, v[b], inv_v);
                    }
                }
                if (threadIdx.x == 0) { p.scale_k[ph] = static_cast<uint8_t>(now_k); p.scale_v[ph] = static_cast<uint8_t>(now_v); }
                __syncthreads();                     // s_top is free again
            }
            // ---- the queries of this kv head ----
            const int per_row = G * CH, total = rows * per_row;
            for (int base = 0; base < total; base += kTokQueries * kTokThreads) {
                Chunk c[kTokQueries];
                auto at = [&](int it) { return (static_cast<int64_t>(r + it / per_row) * Hq + h * G + it % per_row / CH) * D; };
#pragma unroll
                for (int b = 0; b < kTokQueries; ++b) {
                    const int it = base + threadIdx.x + b * kTokThreads;
                    if (it < total) c[b] = load_chunk<D>(p.q + at(it), it % CH);
                }
#pragma unroll
                for (int b = 0; b < kTokQueries; ++b) {
                    const int it = base + threadIdx.x + b * kTokThreads;
                    if (it < total) {
                        const int t = it / per_row;
                        rotate_chunk(c[b], cs[t] + it % CH * 8, sn[t] + it % CH * 8);
                        store_chunk<D>(p.q_rot + at(it), it % CH, c[b]);
                    }
                }
            }
        }
    }
}

}  // namespace

int launch_append_paged(const hpd_geom& g, const AppendPagedArgs& a)
{
    const PageArgs p{a.n_seqs, a.max_rows, a.table_rows, a.pages_per_seq, a.n_pages, a.page_size, a.n_rows, a.row_seq, a.seq_row_start, a.seq_id,
                     a.seq_len, a.page_table, a.pos_id, a.q, a.q_rot, a.k_new, a.v_new, a.page_k, a.page_v, a.scale_k, a.scale_v, a.dev_status};
    const int Hq = a.q ? g.Hq : 0;
    const bool wide = g.D == 128;
    const InvFreq& f = inv_freq_table(g);
    if (!a.row_seq) {
        const unsigned blocks = (static_cast<unsigned>(std::min(a.max_rows, a.n_seqs)) + kStepRows - 1) / kStepRows;
        if (blocks == 0) return HPD_OK;
        // few rows: several CTAs to a pair of them, as many as there are batches and SMs
        const unsigned batches = static_cast<unsigned>(kStepRows * (Hq + 2 * g.Hkv) * (g.D / 16) + kStepThreads - 1) / kStepThreads;
        const dim3 grid(blocks, std::max(1u, std::min(8u * sm_count() / blocks, batches)));
        if (wide) append_step_kernel<128><<<grid, kStepThreads, 0, a.stream>>>(Hq, g.Hkv, f, p);
        else append_step_kernel<64><<<grid, kStepThreads, 0, a.stream>>>(Hq, g.Hkv, f, p);
    } else {
        const unsigned windows = (static_cast<unsigned>(a.max_rows) + a.page_size - 1) / a.page_size;
        const dim3 grid(windows, static_cast<unsigned>(g.Hkv));
        if (wide) append_tokens_kernel<128><<<grid, kTokThreads, 0, a.stream>>>(Hq, g.Hkv, f, p);
        else append_tokens_kernel<64><<<grid, kTokThreads, 0, a.stream>>>(Hq, g.Hkv, f, p);
    }
    HPD_CUDA_TRY(cudaGetLastError());
    return HPD_OK;
}

}  // namespace hpd
