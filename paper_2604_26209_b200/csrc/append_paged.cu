// hpd_append_paged: new keys and values into pages of 8-bit codes, with the rotary embedding on the way.
//
// For the tokens that one call puts into one page, per kv head and for K and V each:
//     a = largest finite magnitude of the new tokens' elements (keys: rotated and rounded to bf16, the bits of hpd_rope)
//     n = smallest integer >= -126 with a <= 448 * 2^n
//     e = n for a page that held no token, else max(n, e of before); codes held before become e4m3(code * 2^(e_before - e))
//     new codes = e4m3(x * 2^-e)
// Roundings: the key to bf16 (2^-8 of it), the code (2^-4 of the value, 2^-10 of the scale below 2^-6 of it), codes held before that fall below 2^-6 of a
// grown scale once more (2^-10 of that scale each time, 2^-9 of the last one in all).  The angle is reduced in 64 bits and rounded to 32 as hpd_rope does it, so that keys
// that hpd_rope has rotated and keys rotated here give the same codes; against a rotation in 64 bits up to some ten in 3.5 million codes lie on the
// other side of a border, one step off (with sines and cosines rounded once: up to four).
// With powers of two as scales the growth of a scale is exact for every code that stays a normal number, so a page that fills up
// token by token ends with the codes of one that is filled at once, but for infinities and for elements below 2^-6 of the final scale (up to 2^-13.8 of the
// page's largest element, which is above 224 scales).
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
    const uint32_t w[8] = {c.lo.x, c.lo.y, c.lo.z, c.lo.w, c.hi.x, c.hi.y, c.hi.z, c.hi.w};
    uint32_t two = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) two = __vmaxu2(two, w[i] & 0x7fff7fffu);
    int top = static_cast<int>(max(two & 0xffffu, two >> 16));
    if (top >= 0x7f80) {                             // infinities or NaN among them, which do not count: element by element
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max_finite(top, w[i]);
    }
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

// the same for units u, u + 32, u + 64 and u + 96 of `units`, their loads together
__device__ __forceinline__ void rescale16x4(uint8_t* p, int u, int units, int was, int now)
{
    const float f = now - was < 127 ? __uint_as_float(static_cast<uint32_t>(127 - (now - was)) << 23) : 0.f;
    uint4* q = reinterpret_cast<uint4*>(p);
    uint4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (u + 32 * i < units) w[i] = q[u + 32 * i];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (u + 32 * i < units)
            q[u + 32 * i] = make_uint4(e4m3x4_times(w[i].x, f), e4m3x4_times(w[i].y, f), e4m3x4_times(w[i].z, f), e4m3x4_times(w[i].w, f));
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
// One token per sequence: the decode step.  Row r is sequence r's token.  6144 rows (32 / 8 heads of 128, pages of 16): 37 us, 3.8 TB/s; without the
// rotation 33, without the held codes' rescaling 35, without the angles or the conversions 37: what is left is two batches of loads one after the
// other per CTA.  (One batch in 256 threads 40.5, six chunks a thread 45.4, ten CTAs an SM 39.1.)
// ------------------------------------------------------------------------------------------------
constexpr int kStepThreads = 128, kStepRows = 2, kStepBatch = 3, kStepResident = 8;

template <int D>
__global__ void __launch_bounds__(kStepThreads, kStepResident)
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
        static_assert(kStepRows == 2, "row by comparison");
        row = it >= items;
        const int local = row ? it - items : it;
        head = local / CH; ch = local % CH;
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
        int was[kStepBatch];                         // scales of before, asked for together; 0: the page is new (or it is a query)
#pragma unroll
        for (int k = 0; k < kStepBatch; ++k) {
            const int it = base + threadIdx.x + (k * parts + part) * kStepThreads;
            was[k] = 0;
            if (it < total) {
                int row, head, ch;
                (void)source(it, row, head, ch);
                if (head < 2 * Hkv && s_page[row] >= 0 && s_slot[row] > 0)
                    was[k] = head < Hkv ? p.scale_k[static_cast<int64_t>(s_page[row]) * Hkv + head] : p.scale_v[static_cast<int64_t>(s_page[row]) * Hkv + head - Hkv];
            }
        }
#pragma unroll
        for (int k = 0; k < kStepBatch; ++k) {
            const int it = base + threadIdx.x + (k * parts + part) * kStepThreads;
            const bool have = it < total;
            int row = 0, head = 2 * Hkv, ch = 0;
            if (have) (void)source(it, row, head, ch);
            const bool is_v = head >= Hkv && head < 2 * Hkv;
            if (have && p.pos_id && !is_v) rotate_chunk(c[k], cs[row] + ch * 8, sn[row] + ch * 8);
            if (have && head >= 2 * Hkv) store_chunk<D>(p.q_rot + (static_cast<int64_t>(r0 + row) * Hq + head - 2 * Hkv) * D, ch, c[k]);
            // a head's CH lanes agree on its scale
            const bool kept = have && head < 2 * Hkv && s_page[row] >= 0;
            int top = kept ? chunk_top(c[k]) : 0;
#pragma unroll
            for (int s = 1; s < CH; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
            const int slot = s_slot[row], now = max(e8m0_needed(top), was[k]);
            const long long ph = kept ? static_cast<long long>(s_page[row]) * Hkv + (is_v ? head - Hkv : head) : 0;
            uint8_t* codes = (is_v ? p.page_v : p.page_k) + ph * p.page_size * D;
            // Codes held under a smaller scale: by the whole warp, four loads of 16 bytes in flight a lane; the head's own lanes would have one
            // round trip to memory for every token.
            for (unsigned m = __ballot_sync(0xffffffffu, kept && ch == 0 && slot > 0 && now > was[k]); m; m &= m - 1) {
                const int from = __ffs(m) - 1;
                uint8_t* at = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(codes), from));
                const int units = __shfl_sync(0xffffffffu, slot, from) * CH, was_m = __shfl_sync(0xffffffffu, was[k], from), now_m = __shfl_sync(0xffffffffu, now, from);
                for (int u = threadIdx.x & 31; u < units; u += 128) rescale16x4(at, u, units, was_m, now_m);
            }
            if (kept) {
                store_codes<D>(codes + static_cast<int64_t>(slot) * D, ch, c[k], e8m0_inverse(now));
                if (ch == 0) (is_v ? p.scale_v : p.scale_k)[ph] = static_cast<uint8_t>(now);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Any number of tokens per sequence: prompts and chunks.  The rows of a sequence that go into one page are a segment.  A CTA has the
// segments that begin in its window of rows and takes them in groups of up to 64 rows, for every gridDim.y-th kv head and those heads' queries:
// the angles of a group's rows are computed once, each thread those of one frequency (its frequency and the rows' position IDs fetched with the
// tables: 586 -> 575 us and 22.6 -> 18.5; from the table of parameters lane by lane and from memory row by row they were a third of a small call).
// 64 prompts of 2288 tokens (32 / 8 heads of 128, pages of 64): 577 to 591 us from box to box, 5.5 to 5.7 TB/s.  What few rows cost is a group's chain --
// tables, pages, scales, then two round trips per head: 7.5 to 8.2 us for one prompt without rotation, 18.5 to 20.5 for 37 ragged chunks.
// ------------------------------------------------------------------------------------------------
constexpr int kTokThreads = 256, kTokRows = 64, kTokQueries = 2;
template <int D> constexpr int kTokResident = D == 128 ? 3 : 4;       // CTAs of an SM

template <int D>
__global__ void __launch_bounds__(kTokThreads, kTokResident<D>)
append_tokens_kernel(int Hq /* 0: no queries */, int Hkv, int window, const InvFreq inv_freq, const PageArgs p)
{
    constexpr int HALF = D / 2, CH = D / 16;
    constexpr int B = kTokRows * CH / kTokThreads;   // chunk pairs of one head's keys (or values) a thread holds
    __shared__ float cs[kTokRows][HALF], sn[kTokRows][HALF];
    __shared__ int s_seg[kTokRows], s_slot[kTokRows], s_pos[kTokRows];       // per row: its segment in the group, its place in the page, its position ID
    __shared__ int g_page[kTokRows], g_held[kTokRows];                       // per segment: page (-1: none), tokens that it held
    __shared__ int g_top[2][2][kTokRows], g_was[2][2][kTokRows];             // per parity of the head, K / V and segment: largest magnitude, scale of before
    __shared__ uint32_t s_starts[4];
    __shared__ int s_end;
    const int n = min(*p.n_rows, p.max_rows);
    const int P = p.page_size, G = Hq / Hkv, q_shift = 31 - __clz(max(G, 1) * CH);
    const int64_t lo = static_cast<int64_t>(blockIdx.x) * window;
    const int end = static_cast<int>(min(lo + window, static_cast<int64_t>(n)));
    const int t0 = threadIdx.x;
    const double freq = p.pos_id ? inv_freq.f[t0 % HALF] : 0.;               // of the angles that this thread computes
    for (int r = static_cast<int>(min(lo, static_cast<int64_t>(n))); r < end;) {
        // ---- the group's rows: where they go, where segments begin ----
        __syncthreads();                             // the tables of the group before have been used
        if (t0 == 0) s_end = r;
        __syncthreads();
        int entry = -1, slot = 0, stop = 0;
        int64_t index = 0;
        bool start = false;
        if (t0 < 2 * kTokRows) {
            const int row = r + t0;
            if (row < n) {
                const int seq = p.row_seq[row];
                const int first = seq >= 0 && seq < p.n_seqs ? p.seq_row_start[seq] : 0, past = seq >= 0 && seq < p.n_seqs ? p.seq_row_start[seq + 1] : 0;
                if (row < first || row >= past) {    // of no sequence: a segment of its own without a page
                    start = true; stop = row + 1;
                } else {
                    index = static_cast<int64_t>(p.seq_len[seq]) + (row - first);
                    slot = static_cast<int>(index < 0 ? 0 : index % P);
                    start = row == first || slot == 0;
                    stop = min(min(past, n), row + P - slot);
                    entry = p.seq_id ? p.seq_id[seq] : seq;
                    if (index < 0 || entry < 0) entry = -1;
                }
            }
            const unsigned starts = __ballot_sync(0xffffffffu, start);
            if ((t0 & 31) == 0) s_starts[t0 >> 5] = starts;
        }
        __syncthreads();
        // Behind the rows of a segment that another window has: 64 rows from the first segment on that begins here.
        const uint64_t near = s_starts[0] | static_cast<uint64_t>(s_starts[1]) << 32, far = s_starts[2] | static_cast<uint64_t>(s_starts[3]) << 32;
        const int skip = near ? __ffsll(static_cast<long long>(near)) - 1 : kTokRows;
        const uint64_t starts = !near ? 0 : skip ? near >> skip | far << (64 - skip) : near;
        r += skip;
        const int t = t0 - skip;
        if (t >= 0 && t < kTokRows) {
            if (p.pos_id && r + t < n) s_pos[t] = p.pos_id[r + t];
            const int seg = __popcll(starts & (~0ull >> (63 - t))) - 1;
            s_seg[t] = seg; s_slot[t] = slot;
            if (starts >> t & 1) {
                int page = -1;
                if (entry >= 0) page = page_of(p, entry, index, blockIdx.y == 0);
                else if (blockIdx.y == 0 && p.dev_status) atomicOr(p.dev_status, HPD_S_BAD_TABLE);
                g_page[seg] = page; g_held[seg] = page < 0 ? 0 : slot;
                if (r + t < end && stop - r <= kTokRows) atomicMax(&s_end, stop);        // later ones are another window's
            }
        }
        __syncthreads();
        const int rows = s_end - r;                  // whole segments only
        if (rows <= 0) break;                        // none begins in the window
        const int segs = __popcll(starts & (~0ull >> (64 - rows)));
        if (p.pos_id)
            for (int t = t0 / HALF; t < rows; t += kTokThreads / HALF) rotary_angle(s_pos[t], freq, cs[t][t0 % HALF], sn[t][t0 % HALF]);
        // ---- head by head: while the keys and values are on their way, the head's queries ----
        for (int h = blockIdx.y, par = 0; h < Hkv; h += gridDim.y, par ^= 1) {
            Chunk k[B], v[B];
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int it = t0 + b * kTokThreads, t = it / CH;
                if (t < rows) {
                    const int64_t at = (static_cast<int64_t>(r + t) * Hkv + h) * D;
                    k[b] = load_chunk<D>(p.k_new + at, it % CH);
                    v[b] = load_chunk<D>(p.v_new + at, it % CH);
                }
            }
            if (t0 < 2 * kTokRows && t0 % kTokRows < segs) {
                const int seg = t0 % kTokRows, is_v = t0 / kTokRows;
                g_top[par][is_v][seg] = 0;
                g_was[par][is_v][seg] = g_held[seg] > 0 ? (is_v ? p.scale_v : p.scale_k)[static_cast<int64_t>(g_page[seg]) * Hkv + h] : 0;
            }
            __syncthreads();
            const int per_row = G * CH, total = rows * per_row;      // a power of two: G is 1, 2, 4 or 8
            auto at = [&](int it) { return (static_cast<int64_t>(r + (it >> q_shift)) * Hq + h * G + (it & (per_row - 1)) / CH) * D; };
            for (int base = t0; base < total; base += kTokQueries * kTokThreads) {
                Chunk c[kTokQueries];
#pragma unroll
                for (int b = 0; b < kTokQueries; ++b) {
                    const int it = base + b * kTokThreads;
                    if (it < total) c[b] = load_chunk<D>(p.q + at(it), it % CH);
                }
#pragma unroll
                for (int b = 0; b < kTokQueries; ++b) {
                    const int it = base + b * kTokThreads;
                    if (it < total) {
                        rotate_chunk(c[b], cs[it >> q_shift] + it % CH * 8, sn[it >> q_shift] + it % CH * 8);
                        store_chunk<D>(p.q_rot + at(it), it % CH, c[b]);
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int it = t0 + b * kTokThreads, t = it / CH, ch = it % CH;
                int top_k = 0, top_v = 0;
                if (t < rows) {
                    if (p.pos_id) rotate_chunk(k[b], cs[t] + ch * 8, sn[t] + ch * 8);
                    top_k = chunk_top(k[b]);
                    top_v = chunk_top(v[b]);
                }
                // a token's CH lanes, then the segment's tokens
#pragma unroll
                for (int s = 1; s < CH; s <<= 1) {
                    top_k = max(top_k, __shfl_xor_sync(0xffffffffu, top_k, s));
                    top_v = max(top_v, __shfl_xor_sync(0xffffffffu, top_v, s));
                }
                if (t < rows && ch == 0) { atomicMax(&g_top[par][0][s_seg[t]], top_k); atomicMax(&g_top[par][1][s_seg[t]], top_v); }
            }
            __syncthreads();
            auto now_of = [&](int is_v, int seg) { return max(e8m0_needed(g_top[par][is_v][seg]), g_was[par][is_v][seg]); };
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int it = t0 + b * kTokThreads, t = it / CH, ch = it % CH;
                if (t < rows) {
                    const int seg = s_seg[t];
                    if (g_page[seg] >= 0) {
                        const int64_t at = ((static_cast<int64_t>(g_page[seg]) * Hkv + h) * P + s_slot[t]) * D;
                        store_codes<D>(p.page_k + at, ch, k[b], e8m0_inverse(now_of(0, seg)));
                        store_codes<D>(p.page_v + at, ch, v[b], e8m0_inverse(now_of(1, seg)));
                    }
                }
            }
            // pages that held tokens under a smaller scale: few, at most the first of each sequence
            for (int seg = 0; seg < segs; ++seg) {
                const int held = g_held[seg];
                if (held == 0) continue;
                const int64_t ph = static_cast<int64_t>(g_page[seg]) * Hkv + h;
                for (int is_v = 0; is_v < 2; ++is_v) {
                    const int was = g_was[par][is_v][seg], now = now_of(is_v, seg);
                    uint8_t* codes = (is_v ? p.page_v : p.page_k) + ph * P * D;
                    if (now > was)
                        for (int i = t0; i < held * (D / 16); i += kTokThreads) rescale16(codes + i * 16, was, now);
                }
            }
            if (t0 < 2 * kTokRows && t0 % kTokRows < segs) {
                const int seg = t0 % kTokRows, is_v = t0 / kTokRows;
                if (g_page[seg] >= 0) (is_v ? p.scale_v : p.scale_k)[static_cast<int64_t>(g_page[seg]) * Hkv + h] = static_cast<uint8_t>(now_of(is_v, seg));
            }
        }
        r = s_end;
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
        // A window's segments should be one group of up to 64 rows: windows of 48, but 64 for large pages while every window and head has a CTA at the
        // same time.  In us with windows of 64 / 48 / 32 rows: 37 ragged chunks in pages of 16 24.6 / 18.5 / 21.8, of 32 23.3 / 23.0 / 20.7, of 64
        // 24.7 / 25.5 / 32.6; 64 prompts of 2288 tokens in pages of 16 572 / 560 / 596, of 32 576 / 572 / 593, of 64 590 / 575 / 571; one
        // prompt in pages of 64 7.6 / 8.1 / 10.1.  (The chunks with 8 / 4 heads of 64, the rest with 32 / 8 of 128.  With heads of 64 the rule is not the best
        // everywhere: 8 prompts in pages of 16 22.7 / 28.6 / 26.9, 64 prompts 132 / 142 / 144 in pages of 16, 129 / 141 / 142 of 32, 129 / 132 / 120 of 64.)
        const unsigned resident = static_cast<unsigned>(wide ? kTokResident<128> : kTokResident<64>) * sm_count();
        const unsigned rows = static_cast<unsigned>(a.max_rows), all = static_cast<unsigned>(kTokRows), heads = static_cast<unsigned>(g.Hkv);
        const unsigned window = a.page_size > 32 && (rows + all - 1) / all * heads <= resident ? all : 48;
        const unsigned windows = (rows + window - 1) / window;
        // The heads of a window go to several CTAs, each with tables and angles of its own: as many as fit the GPU at once, and no more than three heads to
        // a CTA until the windows alone are several rounds of it.  Prompts of 2288 tokens, 1 / 2 / 4 / 8 / 16 / 32 / 64 of them, in us: one CTA
        // 57 / 62 / 94 / 113 / 194 / 317 / 574, two 35 / 42 / 64 / 102 / 167 / 311 / 575, three 29 / 35 / 55 / 88 / 161 / 307 / 586,
        // four 25 / 33 / 62 / 94 / 170 / 320 / 609, eight 20.6 / 35 / 59 / 102 / 190 / 367 / 710.  That is with 8 heads of 128.  4 of 128, 8 / 16 / 64 / 72
        // prompts: one CTA 82 / 161 / 492 / 529, two (the rule's up to 54 prompts) 89 / 140 / 493 / 548, three 76 / 140 / 511 / 571.  Below the
        // threshold and above, 54 and 72 prompts: 8 of 128 one 487 / 612, three (the rule's at 54) 497 / 656; 4 of 128 one 421 / 529, two 417 / 548.  With heads
        // of 64 one CTA would be faster from 16 prompts on: 8 heads, 16 / 64 prompts, one 60 / 204, three (the rule's) 67 / 234; 4 heads 36 / 113 against 40 / 129.
        const unsigned fit = std::max(1u, resident / windows), few = windows < 6 * resident ? (heads + 2) / 3 : 1;
        const dim3 grid(windows, std::min(heads, std::max(fit, few)));
        if (wide) append_tokens_kernel<128><<<grid, kTokThreads, 0, a.stream>>>(Hq, g.Hkv, static_cast<int>(window), f, p);
        else append_tokens_kernel<64><<<grid, kTokThreads, 0, a.stream>>>(Hq, g.Hkv, static_cast<int>(window), f, p);
    }
    HPD_CUDA_TRY(cudaGetLastError());
    return HPD_OK;
}

}  // namespace hpd
