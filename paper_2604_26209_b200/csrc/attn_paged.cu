// hpd_attn_decode_paged on the 5th-generation tensor cores: decode attention over paged caches of e4m3 codes.
//
// The structure is that of hpd_attn_decode: one persistent CTA per SM, two independent pipelines, each walking units of its own (up
// to 128/G branches of a document x G query heads against a chunk of its prefix, for one kv head) in tiles of 64 keys, the
// branches' own tokens first, packed back to back.  What differs is where the bytes are made into operands:
//
//   S = Q K^T    K tiles go from the pages to the tensor core as they are (kind::f8f6f4).  A row of q is scaled by a power of two, its
//                largest magnitude to [128, 256), and split into two e4m3 terms, q = hi + lo: a bf16 has eight significant bits, two
//                terms of four hold them all (below 2^-8 of the largest magnitude some are lost, at most 2^-17 of it).  Twice the
//                k-steps at twice the rate of bf16, and no conversion of K.
//   scales       a page's K scale multiplies its 16-column part of S inside the softmax's multiply-add, its V scale 2^e moves the
//                exponent of its probabilities there: no instruction per element for either.
//   O += P V     two warps of each pipeline widen V tiles from e4m3 to fp16 (exact) in shared memory; P is fp16 with its largest elements
//                between 2^7 and 2^15, so that what is flushed is below 2^-31 of them.  They zero what lies behind a tile's last
//                token; they also fetch Q and write its two terms in its place.
//
// Two references per row.  With s the scaled score (log2) and e the V exponent of its page, R >= s + e - 8 is what the products P V are
// relative to (rescaled when it grows by more than 8), M >= s is what the sum is relative to.  A part of 16 columns whose products
// stay below 2^-60 of R takes part in the sum alone: its probabilities are raised to there, where fp16 flushes them.
//
// NaN.  The pages of a document are all its rows' in any case.  Branches share tiles, and 0 * NaN would reach the others: a NaN among a branch's V
// codes is zeroed and noted, and its rows become NaN in the epilogue; one among its K codes stays in its own columns, which others' rows mask.
//
// What bounds it.  64 prompts (256 documents of 512 tokens with 24 branches each, 32 / 8 heads of 128): 166 us for 72.7 us of bytes at the copy rate
// and 146 us of hpd_attn_decode over an unpaged bf16 cache of twice the bytes; 192 documents of 1024 to 4096 tokens with 12 branches: 290 for 165,
// and 369 in bf16 (after a second of it, at the clock that the power cap leaves, 172 to 178 and 330 to 344).  The copies and matrix products alone take 105 of the 166 us
// (a product of 128 x 64 x 16 or 32 takes the tensor core 48 to 64 cycles here whatever its type: 12 of them per tile); the softmax of a tile
// is a chain of 1.9 k cycles for its warp, 2.3 k with both pipelines' on the SM's issue slots (41 % used), which is why units of few rows
// are taken apart (ways_of); a unit's turn costs 8 k cycles (Q fetched and split 5 k, epilogue 3 k), of which the other pipeline covers about half.
//
// Warps: 0 / 3 scheduler and copies of pipeline 0 / 1, 1 / 2 MMA issuers, 4-7 / 8-11 softmax, 12-13 / 14-15 conversion.
// TMEM columns as in hpd_attn_decode: S0 [0,64) S1 [64,128) O [128,256) of a pipeline, P over the first half of its scores.
// All waits are bounded: a wait that gives up raises HPD_S_TIMEOUT in the status word and the CTA drains and exits.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include <cuda_fp16.h>

#include "common.cuh"
#include "paged.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace hpd {

namespace {

constexpr int kThreads = 512;
constexpr int kM = 128;                    // rows of a tile
constexpr int kN = 64;                     // keys of a tile
constexpr int kPart = 16;                  // keys of a page at least: columns of S with one scale
constexpr int kVHalf = kN * 128;           // one 64-element half of a widened V tile: 64 keys x 128 B
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRescaleSlack = 8.0f;      // tolerated growth of the reference (log2 units) before O is rescaled
constexpr float kUp = 7.0f;                // probabilities are 2^7 larger: 2^15 at most, fp16 holds 65504
constexpr float kFaint = 60.0f;            // products below 2^-60 of the reference are dropped
constexpr uint32_t kColPipe = 256, kColS = 0, kColO = 128;
struct Regs { static constexpr int IO = 104, SOFTMAX = 160, CONVERT = 88; };
static_assert(Regs::IO + 2 * Regs::SOFTMAX + Regs::CONVERT <= 4 * 128, "registers traded between the warpgroups exceed the CTA's allocation");
constexpr int kRounds = 4;                 // a unit has at most 128 branches: 4 rounds of 32 lanes
constexpr int kDescReaders = 7;            // MMA thread, four softmax warps, two conversion warps

template <int D> struct Cfg {
    static constexpr int Q_BYTES = kM * 2 * D;                   // two e4m3 terms of every element
    static constexpr int KV_BYTES = kN * D;                      // one tile of codes
    static constexpr int WIDE_BYTES = kN * 2 * D;                // one V tile in fp16
    static constexpr int NK = D == 128 ? 3 : 4;                               // K stages of a pipeline
    static constexpr int NC = 4;                  // V stages as codes
    static constexpr int NV = D == 128 ? 1 : 2;                  // V stages in fp16
    static constexpr int PAD = D == 128 ? 1 : 2;                 // a branch begins at a multiple of PAD columns (a copy's destination: 128 bytes)
    static constexpr int OFF_Q = 0;
    static constexpr int OFF_STAGE = OFF_Q + 2 * Q_BYTES;        // output transpose, 1 KB per softmax warp
    static constexpr int OFF_K = OFF_STAGE + 8 * 1024;
    static constexpr int OFF_C = OFF_K + 2 * NK * KV_BYTES;
    static constexpr int OFF_V = OFF_C + 2 * NC * KV_BYTES;
    static constexpr int OFF_MISC = OFF_V + 2 * NV * WIDE_BYTES;
    static constexpr int SMEM = OFF_MISC + 8192;
    static_assert(OFF_V % 1024 == 0 && OFF_K % 1024 == 0, "swizzled tiles");
    static_assert(NK + 2 < 8, "a batch of pages has at least eight tiles");
};
static_assert(Cfg<128>::SMEM <= 232448, "shared memory budget");

struct Maps {
    CUtensorMap q;                         // bf16: boxes of 128/G rows x G heads x 64 elements
    CUtensorMap page;                      // K codes of the documents: boxes of one page
    CUtensorMap branch[16];                // K codes of the branches: boxes of 1 .. 16 tokens (of a page at most)
};

struct Params {
    PagedArgs a;
    const WsHeader* hdr;
    const WorkItem* work;
    float *part_ml, *part_o;
    float scale_log2;
    int G;
};

struct UnitDesc {
    int nt;                                // tiles of the unit (branches' and document's); -1: no more units
    int np;                                // document's tiles
    int stot;                              // packed columns of the branches
    int head, key_count, part_base, row_begin, nb /*branches*/, row0 /*first global row*/;
    int nb_cached;                         // branches whose tokens the unit visits: entries below
    int pad[6];
    uint16_t cs[kM];                       // per branch: packed column of its first token
    uint16_t len[kM];                      // per branch: tokens visible
    uint8_t ks[kM], vs[kM];                // per branch: scale bytes of its page
};
static_assert(sizeof(UnitDesc) == 64 + 6 * kM, "descriptor size");

constexpr int kMaxStages = 4;
struct Misc {
    unsigned long long q_raw[2], q_full[2], q_empty[2];          // q as it is has come; its two terms are there; the tile is free
    unsigned long long k_full[2][kMaxStages], k_empty[2][kMaxStages], c_full[2][kMaxStages], c_empty[2][kMaxStages], v_empty[2][kMaxStages];
    unsigned long long s_full[2][2], pv_full[2][2], o_full[2], o_free[2];        // pv: the probabilities and the widened V tile
    unsigned long long desc_full[2], desc_empty[2], batch_full[2], meet[2];
    uint32_t tmem_base;
    int abort_flag;
    int pad[2];
    float2 page_scale[2][2][64];           // pipeline, unit's parity: K scale and V exponent of the document's pages, two batches of 32
    float q_factor[2][kM];                 // what the scaled rows of q have to be multiplied by
    float2 way_ml[2][kM];                  // reference and sum of every row of the tile, where they are two ways' (see ways_of)
    uint32_t nan_branch[2][2][2][4];       // pipeline, unit's parity, conversion warp: branches with a NaN among their values
    UnitDesc desc[2];
};
static_assert(sizeof(Misc) <= 8192, "misc block");

// tcgen05.mma on two operands of e4m3 codes in shared memory (descriptors' low and high words)
__device__ __forceinline__ void tc_mma_codes(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
                 "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %6};\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(a_hi), "r"(b_hi) : "memory");
}
// Descriptors' high words: SBO (bytes of eight rows / 16), version 1, swizzle mode: rows of 128 bytes (mode 2) or of 64 bytes (mode 4).
constexpr uint32_t kRows128 = 0x40004040u, kRows64 = 0x80004020u;
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr) { return (saddr >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_lo_mnmajor(uint32_t saddr) { return (saddr >> 4) | (static_cast<uint32_t>(kVHalf >> 4) << 16); }
// Instruction descriptors, fp32 accumulation, M = 128: e4m3 x e4m3 with both K-major, fp16 x fp16 with B MN-major.
__device__ __forceinline__ uint32_t idesc_codes(int N) { return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(kM >> 4) << 24); }
__device__ __forceinline__ uint32_t idesc_wide(int N) { return idesc_codes(N) | (1u << 16); }

// Units of up to 64 rows and at least kTwoTiles tiles have their rows twice in the tile: rows 0-63 take the first half of every tile's keys, rows 64-127 the
// second, each with references and sums of their own; the epilogue adds them up.  A tile's softmax is then half as long, and that is
// what most of a tile's time is (192 documents of 1024 to 4096 tokens, 12 branches of 4 heads: 337 -> 285 us).
// In a kernel of its own, for steps whose documents have 64 rows or fewer on average: the code for both in one cost the others 4 %.
constexpr int kTwoTiles = 8;
template <bool TWO> __device__ __forceinline__ int ways_of(int nrows, int nt) { return TWO && nrows <= kM / 2 && nt >= kTwoTiles ? 2 : 1; }

// power of two that a V scale byte stands for; NaN for NaN
__device__ __forceinline__ float v_exponent(int byte) { return byte == 255 ? __uint_as_float(0x7fffffffu) : static_cast<float>(byte - 127); }

struct Unit { int nt, np, stot, head, key_count, part_base, row_begin, nb, row0; };
__device__ __forceinline__ Unit read_unit(const UnitDesc& d) {
    return {d.nt, d.np, d.stot, d.head, d.key_count, d.part_base, d.row_begin, d.nb, d.row0};
}

template <int D, bool TWO>
__global__ void __launch_bounds__(kThreads, 1)
attn_paged_kernel(const __grid_constant__ Maps maps, const Params p)
{
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    Misc* misc = reinterpret_cast<Misc*>(smem + C::OFF_MISC);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.G, g_shift = 31 - __clz(G), Hkv = p.a.a.g.Hkv;       // G: 1, 2, 4 or 8
    int32_t* status = p.a.a.dev_status;
    if ((smem_u32(smem) & 1023u) != 0) {                 // swizzled tiles need 1024-byte alignment: refuse rather than misread
        if (threadIdx.x == 0 && status) atomicOr(status, HPD_S_BAD_TABLE);
        return;
    }
    // The merge kernel may come now: this is an ordinary launch, what wrote the plan that it looks at has ended, and it waits for this kernel's end itself.
    start_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&misc->q_raw[i], 1);   mbar_init(&misc->q_full[i], 2);  mbar_init(&misc->q_empty[i], 5);
            for (int b = 0; b < 2; ++b) { mbar_init(&misc->s_full[i][b], 1); mbar_init(&misc->pv_full[i][b], 6); }
            mbar_init(&misc->o_full[i], 1);  mbar_init(&misc->o_free[i], 4);
            mbar_init(&misc->desc_full[i], 1); mbar_init(&misc->desc_empty[i], kDescReaders);
            for (int k = 0; k < kMaxStages; ++k) {
                mbar_init(&misc->k_full[i][k], 1); mbar_init(&misc->k_empty[i][k], 1);
                mbar_init(&misc->c_full[i][k], 1); mbar_init(&misc->c_empty[i][k], 2);
                mbar_init(&misc->v_empty[i][k], 1);
            }
            mbar_init(&misc->batch_full[i], 1); mbar_init(&misc->meet[i], 4);
        }
        misc->abort_flag = 0;
        fence_mbar_init();
    }
    // stale contents of widened tiles are multiplied by zero probabilities: they must be finite from the start
    for (int i = threadIdx.x; i < (C::OFF_MISC - C::OFF_V) / 16; i += kThreads)
        reinterpret_cast<uint4*>(smem + C::OFF_V)[i] = make_uint4(0, 0, 0, 0);
    fence_async_smem();
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&misc->tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&misc->tmem_base);

    if (warp == 0 || warp == 3) {
        // ============================ scheduler and copies of one pipeline =====================
        // Units are drawn as in hpd_attn_decode: six fixed ones per pipeline, then from the step's ticket counter.  What a unit needs to
        // know is a chain of loads -- item, row tables, pages, scales -- of which the unit before issues one link after another between
        // its first tiles.
        reg_dealloc<Regs::IO>();
        const int x = warp == 0 ? 0 : 1;
        // Few units: each becomes two of half the rows (their keys come from L2 the second time), on SMs that would be idle.  One prompt of 4 documents
        // of 512 tokens and 96 branches 24.8 -> 22.7 us.
        const int n_work = p.hdr->n_work, halves = TWO && 2 * n_work * Hkv <= static_cast<int>(gridDim.x) ? 2 : 1;
        const int n_units = n_work * Hkv * halves;
        const bool alternate = p.hdr->longest_first != 0;
        const int P = p.a.page_size, shift = 31 - __clz(P);          // tokens of a page: 2^shift
        const int per_tile = kN >> shift, per_batch = 32 / per_tile; // pages of a tile; tiles whose pages the lanes hold (8, 16 or 32)
        uint32_t* ticket = const_cast<uint32_t*>(&p.hdr->ticket);
        UnitDesc& d = misc->desc[x];
        uint8_t* k_ring = smem + C::OFF_K + x * C::NK * C::KV_BYTES;
        uint8_t* c_ring = smem + C::OFF_C + x * C::NC * C::KV_BYTES;
        if (n_units == 0) {
            if (lane == 0) { d.nt = -1; mbar_arrive(&misc->desc_full[x]); }
        } else {
            constexpr int kStatic = 6;
            const bool spread = n_units < 4 * 2 * static_cast<int>(gridDim.x);
            const uint32_t first_dynamic = static_cast<uint32_t>(kStatic) * 2u * gridDim.x;
            auto next = [&](int i) {                                     // the pipeline's i-th unit
                uint32_t t = 0;
                if (i < kStatic) {
                    const uint32_t j = spread ? blockIdx.x + static_cast<uint32_t>(x) * gridDim.x : 2u * blockIdx.x + static_cast<uint32_t>(x);
                    t = (((i & 1) && alternate) ? 2u * gridDim.x - 1u - j : j) + static_cast<uint32_t>(i) * 2u * gridDim.x;
                } else {
                    if (lane == 0) t = atomicAdd(ticket, 1u);
                    t = __shfl_sync(0xffffffffu, t, 0) + first_dynamic;
                }
                return static_cast<int>(min(t, static_cast<uint32_t>(n_units)));
            };
            auto item_of = [&](int w) {
                const int i = min(w, n_units - 1);
                WorkItem it = p.work[i / Hkv / halves];
                if (TWO && halves == 2) {
                    const int first = (it.row_count + 1) / 2;
                    if (i / Hkv & 1) { it.row_begin += first; it.row_count -= first; } else { it.row_count = first; }
                    if (it.row_count == 0) { it.key_count = 0; it.with_suffix = 0; }      // a single row: nothing is left for the other half
                }
                return it;
            };
            // ---- the links of a unit's chain: row tables and page numbers; branches' pages; scales ----
            int len[kRounds], page[kRounds], ks[kRounds], vs[kRounds];   // per branch; page: slot, then page, then first row of its codes
            int bad;                                                     // a table entry out of range
            // per lane: one of 32 pages of the document: its number (-2: not needed), then first row of its codes (-1: none) and scale bytes
            int id, row, sk, sv;
            auto branches_of = [&](int w, const WorkItem& it) { return w < n_units && it.with_suffix ? it.row_count : 0; };
            auto page_id = [&](const WorkItem& it, int i) {
                const int at = (it.key_begin >> shift) + i;
                if (i << shift >= it.key_count) return -2;
                return at < p.a.pages_per_doc ? p.a.page_table[static_cast<int64_t>(it.doc) * p.a.pages_per_doc + at] : -1;
            };
            auto page_scales = [&](int id_, int head, int& row_, int& sk_, int& sv_) {
                row_ = -1; sk_ = 127; sv_ = 127;
                if (id_ == -2) return;
                if (id_ < 0 || id_ >= p.a.n_pages) { sk_ = 255; bad = 1; return; }      // NaN for the document's rows
                const int64_t ph = static_cast<int64_t>(id_) * Hkv + head;
                row_ = static_cast<int>(ph << shift);
                sk_ = p.a.scale_k[ph]; sv_ = p.a.scale_v[ph];
            };
            int first_row;                                               // the document's, as the tables passed have it
            auto row_tables = [&](int w, const WorkItem& it, int row0) {
                const int nb = branches_of(w, it);
#pragma unroll
                for (int r = 0; r < kRounds; ++r) {
                    const int b = lane + 32 * r;
                    len[r] = 0; page[r] = -1;
                    if (b < nb) {
                        len[r] = p.a.a.suffix_len[row0 + it.row_begin + b];
                        page[r] = p.a.a.active_slot[row0 + it.row_begin + b];
                    }
                }
            };
            // The item names its document's first row, so that the rows are asked for together with the table's entry; where that says another (tables
            // moved after the list was made), it decides.
            auto link_rows = [&](int w, const WorkItem& it) {
                first_row = p.a.a.doc_active_start[it.doc];
                row_tables(w, it, it.doc_row);
                id = w < n_units ? page_id(it, lane) : -2;
            };
            auto link_pages = [&](int w, WorkItem& it) {
                if (first_row != it.doc_row) {
                    it.doc_row = first_row;
                    row_tables(w, it, first_row);
                }
                bad = 0;
#pragma unroll
                for (int r = 0; r < kRounds; ++r) {
                    const int n = len[r] + p.a.a.suffix_extra;
                    len[r] = n < 0 ? 0 : n > p.a.a.g.suffix_cap ? p.a.a.g.suffix_cap : n;
                    if (page[r] < 0) len[r] = 0;
                    if (len[r] > 0) page[r] = page[r] < p.a.a.n_slots ? p.a.slot_page[page[r]] : -1;
                }
            };
            auto link_scales = [&](int w) {
                const int head = w % Hkv;
#pragma unroll
                for (int r = 0; r < kRounds; ++r) {
                    ks[r] = vs[r] = 127;
                    if (len[r] > 0) {
                        if (page[r] < 0 || page[r] >= p.a.n_branch_pages) {
                            bad = 1; len[r] = 0;
                        } else {
                            const int64_t ph = static_cast<int64_t>(page[r]) * Hkv + head;
                            ks[r] = p.a.branch_scale_k[ph]; vs[r] = p.a.branch_scale_v[ph];
                            page[r] = static_cast<int>(ph * p.a.a.g.suffix_cap);
                        }
                    }
                }
                page_scales(id, head, row, sk, sv);
            };
            auto report = [&]() { if (__any_sync(0xffffffffu, bad) && lane == 0 && status) atomicOr(status, HPD_S_BAD_TABLE); };
            // unit ui is w0, the next one w1; before the first there is one without tiles, so that the links stand in one place
            int w0 = n_units, w1 = next(0);
            WorkItem it1 = item_of(w1), it0 = it1;
            int st = 0, sc = 0;                                          // stages of the next tile's copies, and the parities of their barriers
            uint32_t k_par = 1, c_par = 1;
            bool ok = true;
            for (int ui = -1; ok; ++ui) {
                int nt = 0, ns = 0, np = 0, head = 0, row0 = 0, key_count = 0, carry = 0, nb = 0;
                int cs[kRounds], blen[kRounds], brow[kRounds];           // per branch: first column, tokens, first row of its codes
                float2* scales = misc->page_scale[x][ui & 1];
                auto put_scales = [&](int batch, int k, int v) {
                    scales[(batch & 1) * 32 + lane] = make_float2(e8m0_value(k), v_exponent(v));
                };
                int cur_row = -1, nxt_id = -2, nxt_row = -1, nxt_sk = 127, nxt_sv = 127;       // this unit's batch of 32 pages, and the next
                if (ui >= 0) {
                    // ---- scan and publish unit ui ----
                    if (ui >= 1) {
                        ok = mbar_wait_warp(&misc->desc_empty[x], (ui - 1) & 1, misc);
                        if (!ok) break;
                    }
                    const bool live = w0 < n_units;
                    report();
                    nb = branches_of(w0, it0);
#pragma unroll
                    for (int r = 0; r < kRounds; ++r) {
                        cs[r] = 0; blen[r] = 0; brow[r] = 0;
                        if (32 * r < nb) {
                            const int b = lane + 32 * r;
                            const int occ = (len[r] + C::PAD - 1) / C::PAD * C::PAD;
                            int incl = occ;
#pragma unroll
                            for (int s = 1; s < 32; s <<= 1) {
                                const int v = __shfl_up_sync(0xffffffffu, incl, s);
                                if (lane >= s) incl += v;
                            }
                            cs[r] = carry + incl - occ; blen[r] = len[r]; brow[r] = page[r];
                            d.cs[b] = static_cast<uint16_t>(cs[r]);
                            d.len[b] = static_cast<uint16_t>(len[r]);
                            d.ks[b] = static_cast<uint8_t>(ks[r]);
                            d.vs[b] = static_cast<uint8_t>(vs[r]);
                            carry += __shfl_sync(0xffffffffu, incl, 31);
                        }
                    }
                    ns = (carry + kN - 1) / kN; np = live ? (it0.key_count + kN - 1) / kN : 0;
                    nt = live ? ns + np : -1; head = w0 % Hkv; row0 = it0.doc_row + it0.row_begin; key_count = it0.key_count;
                    if (lane == 0) {
                        d.nt = nt; d.np = np; d.stot = carry; d.head = head; d.key_count = key_count; d.part_base = it0.part_base;
                        d.row_begin = it0.row_begin; d.nb = it0.row_count; d.row0 = row0; d.nb_cached = nb;
                    }
                    put_scales(0, sk, sv);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&misc->desc_full[x]);
                    if (!live) break;
                    cur_row = row;
                    nxt_id = page_id(it0, 32 + lane);
                }
                const int w2 = next(ui + 2);
                const WorkItem it2 = item_of(w2);
                link_rows(w1, it1);
                for (int t = 0; t < max(nt, 2) && ok; ++t) {
                    if (t < nt) {
                        uint8_t* kt = k_ring + st * C::KV_BYTES;
                        uint8_t* ct = c_ring + sc * C::KV_BYTES;
                        unsigned long long *kf = &misc->k_full[x][st], *cf = &misc->c_full[x][sc];
                        ok = mbar_wait_warp(&misc->k_empty[x][st], k_par, misc) && mbar_wait_warp(&misc->c_empty[x][sc], c_par, misc);
                        if (!ok) break;
                        if (t < ns) {
                            // pieces of the branches that fall into the tile; a box has the exact height of the piece
                            const int c_lo = t * kN, c_hi = min(carry, c_lo + kN);
                            int mine = 0;
#pragma unroll
                            for (int r = 0; r < kRounds; ++r)
                                if (32 * r < nb) mine += max(0, min(cs[r] + blen[r], c_hi) - max(cs[r], c_lo));
                            const uint32_t bytes = __reduce_add_sync(0xffffffffu, mine) * D;
                            if (lane == 0) { mbar_expect_tx(kf, bytes); mbar_expect_tx(cf, bytes); }
#pragma unroll
                            for (int r = 0; r < kRounds; ++r) {
                                if (32 * r >= nb) break;
                                const int lo = max(cs[r], c_lo);
                                int n = min(cs[r] + blen[r], c_hi) - lo, from = brow[r] + (lo - cs[r]), col = lo - c_lo;
                                if (n > 0) bulk_load(ct + col * D, p.a.branch_v + static_cast<int64_t>(from) * D, cf, static_cast<uint32_t>(n) * D);
                                while (n > 0) {
                                    const int hb = min(n, 16);
                                    tma_load_2d(kt + col * D, &maps.branch[hb - 1], kf, 0, from);
                                    from += hb; col += hb; n -= hb;
                                }
                            }
                        } else {
                            // the lanes that hold the tile's pages copy them
                            const int tp = t - ns, in_batch = tp & (per_batch - 1);
                            if (tp > 0 && in_batch == 0) {                   // the next 32 pages; ask for the ones behind them
                                cur_row = nxt_row;
                                nxt_id = page_id(it0, (tp / per_batch + 1) * 32 + lane);
                            }
                            const int pages = (min(kN, key_count - tp * kN) + P - 1) >> shift, j = lane - in_batch * per_tile;
                            const bool copies = j >= 0 && j < pages && cur_row >= 0;
                            const uint32_t bytes = static_cast<uint32_t>(__popc(__ballot_sync(0xffffffffu, copies))) * P * D;
                            if (lane == 0) { mbar_expect_tx(kf, bytes); mbar_expect_tx(cf, bytes); }
                            if (copies) {
                                tma_load_2d(kt + j * P * D, &maps.page, kf, 0, cur_row);
                                bulk_load(ct + j * P * D, p.a.page_v + static_cast<int64_t>(cur_row) * D, cf, static_cast<uint32_t>(P) * D);
                            }
                            if (in_batch == 1) {
                                const int was = bad;
                                bad = 0;
                                page_scales(nxt_id, head, nxt_row, nxt_sk, nxt_sv);
                                report();
                                bad = was;
                            }
                            // The next batch's scales, over those of the batch before this one: the softmax is at most NK + 2 tiles behind, so it has left it.
                            if (in_batch == per_batch - 1 && tp + 1 < np) {
                                put_scales(tp / per_batch + 1, nxt_sk, nxt_sv);
                                __syncwarp();
                                if (lane == 0) mbar_arrive(&misc->batch_full[x]);
                            }
                        }
                        __syncwarp();
                        if (++st == C::NK) { st = 0; k_par ^= 1; }
                        if (++sc == C::NC) { sc = 0; c_par ^= 1; }
                    }
                    if (t == 0) link_pages(w1, it1);
                    if (t == 1) link_scales(w1);
                }
                if (!ok) break;
                w0 = w1; w1 = w2; it0 = it1; it1 = it2;
            }
        }
    } else if (warp < 3) {
        // ================================ MMA issuers (one per pipeline) =============================
        reg_dealloc<Regs::IO>();
        if (elect_one()) {
            const int x = warp - 1;
            uint32_t qc = 0, tiles = 0;                   // units with tiles so far; tiles of earlier units
            bool ok = true;
            constexpr uint32_t kHi = D == 128 ? kRows128 : kRows64;
            const uint32_t q_lo = desc_lo(smem_u32(smem + C::OFF_Q + x * C::Q_BYTES));
            const uint32_t k_lo0 = desc_lo(smem_u32(smem + C::OFF_K + x * C::NK * C::KV_BYTES));
            const uint32_t v_lo0 = desc_lo_mnmajor(smem_u32(smem + C::OFF_V + x * C::NV * C::WIDE_BYTES));
            const uint32_t tmem_s = tmem + x * kColPipe + kColS, tmem_o = tmem + x * kColPipe + kColO;
            const uint32_t idesc_pv = idesc_wide(D);
            for (uint32_t ui = 0; ok; ++ui) {
                ok = mbar_wait(&misc->desc_full[x], ui & 1, misc);
                if (!ok) break;
                const Unit u = read_unit(misc->desc[x]);
                mbar_arrive(&misc->desc_empty[x]);
                if (u.nt < 0) break;
                const int nt = u.nt;
                if (nt == 0) continue;
                const int ns = nt - u.np;
                const int last_s = u.stot - (ns - 1) * kN, last_p = u.key_count - (u.np - 1) * kN;
                auto cols16 = [&](int j) {                // sixteens of columns of tile j
                    int c = kN;
                    if (j == ns - 1) c = last_s;
                    else if (j == nt - 1) c = last_p;
                    return (c + 15) >> 4;
                };
                ok = mbar_wait(&misc->q_full[x], qc & 1, misc);
                ++qc;
                auto issue_qk = [&](int j) {
                    const uint32_t kt = tiles + j;
                    const int ks = kt % C::NK, sb = kt & 1;
                    const uint32_t idesc = idesc_codes(cols16(j) << 4);
                    const uint32_t k_lo = k_lo0 + ks * (C::KV_BYTES >> 4);
                    if (!mbar_wait(&misc->k_full[x][ks], (kt / C::NK) & 1, misc)) return false;
                    tc_fence_after();
                    // k-steps of 32 codes; the low terms of q are a tile (D = 128) or half a row (D = 64) behind the high ones
#pragma unroll
                    for (int k = 0; k < 2 * D / 32; ++k) {
                        const uint32_t kk = (k % (D / 32)) * 2;
                        const uint32_t qk = k < D / 32 ? kk : (D == 128 ? (kM * 128 >> 4) + kk : 4 + kk);
                        tc_mma_codes(tmem_s + sb * kN, q_lo + qk, kRows128, k_lo + kk, kHi, idesc, k > 0);
                    }
                    tc_commit(&misc->s_full[x][sb]);
                    tc_commit(&misc->k_empty[x][ks]);
                    if (j + 1 >= nt) tc_commit(&misc->q_empty[x]);
                    return true;
                };
                // Scores run two tiles ahead: S(j+2) overwrites the tile in which S(j) was computed and P(j) was read, and the tensor core
                // executes this thread's instructions in the order of issue.  (One tile of scores, handed back as soon as the softmax has them in
                // registers, and two of P measured 12 % slower.)
                if (ok) ok = issue_qk(0);
                if (ok && nt > 1) ok = issue_qk(1);
                for (int j = 0; j < nt && ok; ++j) {
                    const uint32_t vt = tiles + j;
                    const int vs = vt % C::NV, pb = vt & 1;
                    const uint32_t v_lo = v_lo0 + vs * (C::WIDE_BYTES >> 4);
                    const int nk = cols16(j);
                    const uint32_t acc0 = j >= 1;
                    if (j == 0 && qc > 1) ok = mbar_wait(&misc->o_free[x], (qc - 2) & 1, misc);       // the epilogue of the unit before has read O
                    if (ok) ok = mbar_wait(&misc->pv_full[x][pb], (vt >> 1) & 1, misc);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < kN / 16; ++k)
                        if (k < nk) tc_mma_ts(tmem_o, tmem_s + pb * kN + k * 8, v_lo + k * 128, idesc_pv, k > 0 ? 1u : acc0);
                    tc_commit(&misc->v_empty[x][vs]);
                    if (j + 1 >= nt) tc_commit(&misc->o_full[x]);
                    if (j + 2 < nt) ok = issue_qk(j + 2);
                }
                tiles += nt;
            }
        }
    } else if (warp >= 12) {
        // ======================= conversion: the two terms of Q, V tiles from e4m3 to fp16 ===================
        reg_dealloc<Regs::CONVERT>();
        const int x = (warp - 12) >> 1, half = warp & 1, tid = half * 32 + lane;
        uint8_t* q_tile = smem + C::OFF_Q + x * C::Q_BYTES;
        uint8_t* c_ring = smem + C::OFF_C + x * C::NC * C::KV_BYTES;
        uint8_t* v_ring = smem + C::OFF_V + x * C::NV * C::WIDE_BYTES;
        uint32_t tiles = 0, qc = 0;
        bool ok = true;
        for (uint32_t ui = 0; ok; ++ui) {
            ok = mbar_wait_warp(&misc->desc_full[x], ui & 1, misc);
            if (!ok) break;
            const UnitDesc& d = misc->desc[x];
            const Unit u = read_unit(d);
            uint32_t cols[kRounds];                       // of this lane's branches: first column and length, for NaN codes
#pragma unroll
            for (int r = 0; r < kRounds; ++r) cols[r] = lane + 32 * r < d.nb_cached ? d.cs[lane + 32 * r] | static_cast<uint32_t>(d.len[lane + 32 * r]) << 16 : 0u;
            __syncwarp();
            if (lane == 0) mbar_arrive(&misc->desc_empty[x]);
            if (u.nt < 0) break;
            if (u.nt == 0) continue;
            // ---- Q in place: 16 elements a lane, D/16 lanes a row; a row's 2 D bytes of bf16 become D bytes of high terms and D of low ones ----
            constexpr int LANES = D / 16, ROWS = 32 / LANES, BATCH = 2;
            const int nrows = u.nb * G, ways = ways_of<TWO>(nrows, u.nt), part = lane % LANES;
            if (half == 0) {
                ok = mbar_wait_warp(&misc->q_empty[x], (qc & 1) ^ 1, misc);
                if (!ok) break;
                if (elect_one()) {
                    mbar_expect_tx(&misc->q_raw[x], C::Q_BYTES);
                    for (int h = 0; h < D / 64; ++h) tma_load_4d(q_tile + h * (kM * 128), &maps.q, &misc->q_raw[x], h * 64, 0, u.head, u.row0);
                }
                __syncwarp();
            }
            ok = mbar_wait_warp(&misc->q_raw[x], qc & 1, misc);
            if (!ok) break;
            if (lane < 4) misc->nan_branch[x][qc & 1][half][lane] = 0u;
            for (int r0 = half * (BATCH * ROWS); r0 < nrows; r0 += 2 * BATCH * ROWS) {
                // rows of 128 bytes, 16-byte pieces exchanged by the row's number in its group of eight (rows behind the unit's last: whatever is there)
                auto piece = [&](int r, int c) { return reinterpret_cast<uint4*>(q_tile + (c >> 3) * (kM * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)); };
                uint32_t w[BATCH][8], top[BATCH];         // pairs of elements; largest magnitude of the row (bits)
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int r = r0 + i * ROWS + lane / LANES;
                    const uint4 a = *piece(r, 2 * part), b = *piece(r, 2 * part + 1);
                    w[i][0] = a.x; w[i][1] = a.y; w[i][2] = a.z; w[i][3] = a.w; w[i][4] = b.x; w[i][5] = b.y; w[i][6] = b.z; w[i][7] = b.w;
                    uint32_t t2 = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) t2 = __vmaxu2(t2, w[i][k] & 0x7fff7fffu);
                    top[i] = max(t2 & 0xffffu, t2 >> 16);
                }
#pragma unroll
                for (int s = 1; s < LANES; s <<= 1)
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], s));
                __syncwarp();                             // every row of the batch has been read
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int r = r0 + i * ROWS + lane / LANES;
                    const uint32_t e = min(max(top[i] >> 7, 15u), 254u);  // exponent byte of the largest; q * 2^(134 - e) is below 256
                    const float up = __uint_as_float((261u - e) << 23);
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t h2[2], l2[2];            // pairs of codes
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t e2 = w[i][2 * k + j];
                            const __half2 v = __floats2half2_rn(bf16lo(e2) * up, bf16hi(e2) * up);        // exact, below 2^-16 to 2^-25
                            h2[j] = half2_e4m3x2(v);
                            const uint32_t back = e4m3x2_half2(h2[j]);
                            l2[j] = half2_e4m3x2(__hsub2(v, *reinterpret_cast<const __half2*>(&back)));
                        }
                        hi[k] = h2[0] | h2[1] << 16;
                        lo[k] = l2[0] | l2[1] << 16;
                    }
                    const float factor = top[i] >= 0x7f80u ? __uint_as_float(0x7fffffffu) : __uint_as_float((e - 7u) << 23);
                    for (int w = 0; w < ways; ++w) {
                        *piece(r + w * (kM / 2), part) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        *piece(r + w * (kM / 2), (D == 128 ? 8 : 4) + part) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                        if (part == 0) misc->q_factor[x][r + w * (kM / 2)] = factor;
                    }
                }
                __syncwarp();
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&misc->q_full[x]);
            // ---- V tiles ----
            const int ns = u.nt - u.np;
            for (int t = 0; t < u.nt; ++t, ++tiles) {
                const int sc = tiles % C::NC, sv = tiles % C::NV;
                const bool own = t < ns;
                const int rows = min(kN, own ? u.stot - t * kN : u.key_count - (t - ns) * kN);       // what lies behind is zero
                uint8_t* src = c_ring + sc * C::KV_BYTES;
                uint8_t* dst = v_ring + sv * C::WIDE_BYTES;
                ok = mbar_wait_warp(&misc->c_full[x][sc], (tiles / C::NC) & 1, misc);
                if (!ok) break;
                ok = mbar_wait_warp(&misc->v_empty[x][sv], ((tiles / C::NV) & 1) ^ 1, misc);
                // the epilogue of the unit before may be using the tile's memory
                if (TWO && ok && t == 0 && qc > 0) ok = mbar_wait_warp(&misc->o_free[x], (qc - 1) & 1, misc);
                if (!ok) break;
                // pieces of 8 codes: 16 bytes of fp16 each, one below another for a thread (rows of 128 bytes, exchanged like q's)
                constexpr int PIECES = D / 8, STEP = 64 / PIECES, BATCH_V = 8;
                const int c = tid % PIECES, row = tid / PIECES;
                uint8_t* from = src + row * D + c * 8;
                uint8_t* to = dst + (c >> 3) * kVHalf + row * 128 + (((c & 7) ^ row) << 4);
                const int odd = STEP == 4 ? ((c & 4) ^ (row & 4)) == 0 ? 64 : -64 : 0;                 // where the row's number gains a 4
                if (own) {
                    // A NaN code must not meet the zero probabilities of other branches' rows: it becomes zero, its branch is noted.  (What
                    // lies between branches, stale, is no branch's.)
                    uint32_t any = 0;
                    auto nan_of = [](uint32_t v) { return ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };
#pragma unroll
                    for (int i = 0; i < kN / STEP; ++i) {
                        const uint2 v = *reinterpret_cast<const uint2*>(from + i * STEP * D);
                        any |= nan_of(v.x) | nan_of(v.y);
                    }
                    if (__any_sync(0xffffffffu, any != 0)) {
#pragma unroll 1
                        for (int i = 0; i < kN / STEP; ++i) {
                            uint2* at = reinterpret_cast<uint2*>(from + i * STEP * D);
                            const uint32_t n0 = nan_of(at->x), n1 = nan_of(at->y);
                            if (n0 | n1) *at = make_uint2(at->x & ~((n0 >> 7) * 0xffu), at->y & ~((n1 >> 7) * 0xffu));
                            for (unsigned hit = __ballot_sync(0xffffffffu, (n0 | n1) != 0); hit; hit &= hit - 1) {
                                const int col = t * kN + (i * 64 + half * 32 + __ffs(hit) - 1) / PIECES;
#pragma unroll
                                for (int r = 0; r < kRounds; ++r) {
                                    const bool in = static_cast<uint32_t>(col - static_cast<int>(cols[r] & 0xffff)) < cols[r] >> 16;
                                    const unsigned who = __ballot_sync(0xffffffffu, in);
                                    if (lane == 0) misc->nan_branch[x][qc & 1][half][r] |= who;
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int i0 = 0; i0 < kN / STEP; i0 += BATCH_V) {
                    uint2 w[BATCH_V];
#pragma unroll
                    for (int i = 0; i < BATCH_V; ++i) w[i] = *reinterpret_cast<const uint2*>(from + (i0 + i) * STEP * D);
                    if (rows < kN)
#pragma unroll
                        for (int i = 0; i < BATCH_V; ++i)
                            if (row + (i0 + i) * STEP >= rows) w[i] = make_uint2(0u, 0u);
#pragma unroll
                    for (int i = 0; i < BATCH_V; ++i) {
                        const uint4 v = make_uint4(e4m3x2_half2(w[i].x), e4m3x2_half2(w[i].x >> 16), e4m3x2_half2(w[i].y), e4m3x2_half2(w[i].y >> 16));
                        *reinterpret_cast<uint4*>(to + (i0 + i) * STEP * 128 + ((i0 + i) & 1) * odd) = v;
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) { mbar_arrive(&misc->pv_full[x][tiles & 1]); mbar_arrive(&misc->c_empty[x][sc]); }
            }
            ++qc;
        }
    } else {
        // ======================================= softmax =======================================
        reg_alloc<Regs::SOFTMAX>();
        const int x = warp >= 8 ? 1 : 0;                 // pipeline
        const int quad = warp & 3;                       // TMEM lane quadrant this warp may access
        const int row = quad * 32 + lane;                // tile row = TMEM lane
        const uint32_t lane_base = static_cast<uint32_t>(quad * 32) << 16;
        const uint32_t tmem_s0 = tmem + lane_base + x * kColPipe + kColS;
        const uint32_t tmem_o = tmem + lane_base + x * kColPipe + kColO;
        uint8_t* stg = smem + C::OFF_STAGE + (x * 4 + quad) * 1024;      // this warp's output staging
        const int shift = 31 - __clz(p.a.page_size);
        uint32_t pw = 0, qc = 0, batches = 0, meets = 0; // tiles done (S read, P written), units with tiles, batches of pages beyond the first, meetings
        bool ok = true;
        for (uint32_t unit_idx = 0; ok; ++unit_idx) {
            ok = mbar_wait_warp(&misc->desc_full[x], unit_idx & 1, misc);
            if (!ok) break;
            const UnitDesc& d = misc->desc[x];
            const Unit u = read_unit(d);
            const int nrows = u.nb * G, ways = ways_of<TWO>(nrows, u.nt), way = ways == 2 ? quad >> 1 : 0;
            const int u_row = row - way * (kM / 2);      // row of the unit
            const int b_row = u_row >> g_shift;          // its branch inside the unit
            const bool cached = b_row < d.nb_cached;
            const int my_cs = cached ? d.cs[b_row] : 0, my_len = cached ? d.len[b_row] : 0;
            const float my_k = e8m0_value(cached ? d.ks[b_row] : 127), my_e = cached ? v_exponent(d.vs[b_row]) : 0.f;
            __syncwarp();
            if (lane == 0) mbar_arrive(&misc->desc_empty[x]);
            if (u.nt < 0) break;
            const int nt = u.nt, ns = nt - u.np;
            const bool row_valid = u_row < nrows;
            const bool warp_active = quad * 32 - way * (kM / 2) < nrows;
            float q_factor = 0.f;
            if (nt > 0) {
                ok = mbar_wait_warp(&misc->q_full[x], qc & 1, misc);
                if (!ok) break;
                // rows behind the unit's last hold anything: their scores are made zero, or they would have the warp rescale O in every tile
                q_factor = row_valid ? misc->q_factor[x][row] * p.scale_log2 : 0.f;
                __syncwarp();
                if (lane == 0) mbar_arrive(&misc->q_empty[x]);
            }
            float R = -INFINITY, M = -INFINITY, l = 0.f;
            const int j_full = ns + u.key_count / kN;    // tiles [ns, j_full): every row sees them whole
            // References of the row from a tile's largest score and largest product (log2): taken as they are by a row that has seen nothing so far,
            // moved when one has grown by more than the slack (probabilities and sums are at most 2^8 larger until then).  False: gave up.
            auto refer = [&](float top_s, float top_r) {
                const bool fresh = R == -INFINITY;       // O row is still exactly zero
                if (fresh) { R = top_r; M = top_s; }
                const bool grow = top_r > R + kRescaleSlack || top_s > M + kRescaleSlack;
                if (__any_sync(0xffffffffu, grow)) {
                    // O must be rescaled: wait until the previous P V product has landed in TMEM.  (In a unit's first tile all rows are fresh.)
                    if (!mbar_wait_warp(&misc->v_empty[x][(pw - 1) % C::NV], ((pw - 1) / C::NV) & 1, misc)) return false;
                    tc_fence_after();
                    const float r_new = grow ? fmaxf(R, top_r) : R, m_new = grow ? fmaxf(M, top_s) : M;
                    const float f = grow ? ex2(R - r_new) : 1.f;
                    if (grow) l *= ex2(M - m_new);
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 32) {
                        uint32_t ov[32];
                        tmem_ld32(tmem_o + c0, ov);
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < 32; ++c) ov[c] = __float_as_uint(__uint_as_float(ov[c]) * f);
                        tmem_st32(tmem_o + c0, ov);
                    }
                    tmem_st_wait();
                    R = r_new;
                    M = m_new;
                }
                return true;
            };
            auto factor = [&](float k) {                 // of raw scores; not zero: masked scores are -inf (NaN stays)
                k *= q_factor;
                return k < 1.17549435e-38f ? 1.17549435e-38f : k;
            };
            auto largest16 = [](const uint32_t* s) {
                float a = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])), b = fmaxf(__uint_as_float(s[2]), __uint_as_float(s[3]));
#pragma unroll
                for (int k = 4; k < kPart; k += 4) {
                    a = fmax3(a, __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
                    b = fmax3(b, __uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
                }
                return fmaxf(a, b);
            };
            // V exponent less the reference, raised for a part whose products stay below 2^-60 of it: ms is the part's largest score
            auto exponent = [&](float ev, float ms) {
                const float ref = R == -INFINITY ? 0.f : R;
                return fminf(fmaxf(ev, ref - kFaint - ms), 400.f) - ref + (ev - ev);       // NaN stays
            };
            // The probabilities of 16 columns of one scale as fp16 pairs, and their share of the sum.
            auto probabilities = [&](const uint32_t* s, float k, float e, uint32_t* pk) {
                const uint64_t k2 = pair(k, k), e2 = pair(e + kUp, e + kUp);
                uint64_t sum = pair(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < kPart / 2; ++i) {
                    const uint64_t y = fma2(pair(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), k2, e2);
                    float y0, y1;
                    unpair(y, y0, y1);
                    const float e0 = ex2(y0), e1 = ex2(y1);
                    sum = add2(sum, pair(e0, e1));
                    const __half2 two = __floats2half2_rn(e0, e1);
                    pk[i] = *reinterpret_cast<const uint32_t*>(&two);
                }
                float a0, a1;
                unpair(sum, a0, a1);
                l = fmaf(a0 + a1, ex2(-e - kUp - (M == -INFINITY ? 0.f : M)), l);
            };
            // A document's tile that every row sees whole: PARTS parts of it from `first` on (four, or the half of this way's rows; the other half's
            // probabilities are zero).
            auto whole = [&](auto parts, int first, uint32_t tmem_s, auto& scale_of) {
                constexpr int PARTS = decltype(parts)::value;
                uint32_t sv[PARTS * kPart];
#pragma unroll
                for (int h = 0; h < PARTS / 2; ++h) tmem_ld32(tmem_s + (first + 2 * h) * kPart, sv + h * 32);
                float k[PARTS], ev[PARTS], ms[PARTS];    // of the parts: factor of the scores, V exponent, largest score
#pragma unroll
                for (int c = 0; c < PARTS; ++c) { const float2 sc = scale_of(first + c); k[c] = factor(sc.x); ev[c] = sc.y; }
                tmem_ld_wait();
                float top_s = -INFINITY, top_r = -INFINITY, low_r = INFINITY;
#pragma unroll
                for (int c = 0; c < PARTS; ++c) {
                    ms[c] = largest16(sv + c * kPart) * k[c];
                    top_s = fmaxf(top_s, ms[c]);
                    top_r = fmaxf(top_r, ms[c] + ev[c]);
                    low_r = fminf(low_r, ms[c] + ev[c]);
                }
                if (!refer(top_s, top_r)) return false;
                if (__any_sync(0xffffffffu, row_valid && !(low_r >= R - kFaint))) {
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) ev[c] = exponent(ev[c], ms[c]);
                } else {
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) ev[c] -= R;
                }
                // to tensor memory, over the first half of the row's own scores: 32 keys = 16 columns of pairs per store
#pragma unroll
                for (int h = 0; h < PARTS / 2; ++h) {
                    uint32_t pk[16];
#pragma unroll
                    for (int c = 0; c < 2; ++c) probabilities(sv + (2 * h + c) * kPart, k[2 * h + c], ev[2 * h + c], pk + c * 8);
                    tmem_st16(tmem_s + (first + 2 * h) * (kPart / 2), pk);
                }
                if (PARTS < 4) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) pk[i] = 0u;
                    tmem_st16(tmem_s + (first ^ 2) * (kPart / 2), pk);
                }
                tmem_st_wait();
                return true;
            };
            for (int j = 0; j < nt && ok; ++j) {
                const int pb = pw & 1;                   // the tile's S / P buffer
                const uint32_t tmem_s = tmem_s0 + pb * kN;
                // K scale and V exponent of the tile's c-th part
                const int first_page = (j - ns) << (6 - shift);
                auto scale_of = [&](int c) {
                    return j < ns ? make_float2(my_k, my_e) : misc->page_scale[x][unit_idx & 1][(first_page + (c * kPart >> shift)) & 63];
                };
                if (j > ns && (first_page & 31) == 0) {  // the next 32 pages
                    ok = mbar_wait_warp(&misc->batch_full[x], batches & 1, misc);
                    if (!ok) break;
                    ++batches;
                }
                ok = mbar_wait_warp(&misc->s_full[x][pb], (pw >> 1) & 1, misc);
                if (!ok) break;
                tc_fence_after();
                if (!warp_active) {                      // no rows: nobody reads its probabilities' products
                } else if (j >= ns && j < j_full) {
                    if (TWO && ways == 2) ok = whole(std::integral_constant<int, 2>(), 2 * way, tmem_s, scale_of);
                    else ok = whole(std::integral_constant<int, 4>(), 0, tmem_s, scale_of);
                    if (!ok) break;
                } else {
                    // A tile of branches' tokens, or a document's last: columns [lo, hi) of this row, parts [c_lo, c_hi) of the warp's rows; the other parts'
                    // probabilities are zero.
                    int lo = 0, hi = u.key_count - (j - ns) * kN;
                    if (j < ns) {
                        lo = max(0, my_cs - j * kN);
                        hi = min(kN, my_cs + my_len - j * kN);
                    }
                    if (ways == 2) { lo = max(lo, way * (kN / 2)); hi = min(hi, (way + 1) * (kN / 2)); }
                    const bool sees = row_valid && hi > lo;
                    const int c_lo = __reduce_min_sync(0xffffffffu, sees ? lo : kN) / kPart;
                    const int c_hi = (__reduce_max_sync(0xffffffffu, sees ? hi : 0) + kPart - 1) / kPart;
                    // Part by part, twice: the largest score first.  (P of a part lies over scores that have been used.)
                    auto part = [&](int c, uint32_t (&sv)[kPart]) {
                        tmem_ld16(tmem_s + c * kPart, sv);
                        const int from = lo - c * kPart;
                        const unsigned span = sees ? static_cast<unsigned>(hi - lo) : 0u;
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < kPart; ++i)
                            if (static_cast<unsigned>(i - from) >= span) sv[i] = 0xff800000u;       // -inf
                    };
                    float top_s = -INFINITY, top_r = -INFINITY;
#pragma unroll 1
                    for (int c = c_lo; c < c_hi; ++c) {
                        uint32_t sv[kPart];
                        part(c, sv);
                        const float2 sc = scale_of(c);
                        const float ms = largest16(sv) * factor(sc.x);
                        top_s = fmaxf(top_s, ms);
                        top_r = fmaxf(top_r, ms + sc.y);
                    }
                    ok = c_hi <= c_lo || refer(top_s, top_r);
                    if (!ok) break;
#pragma unroll 1
                    for (int c = 0; c < kN / kPart; ++c) {
                        uint32_t pk[8];
                        if (c >= c_lo && c < c_hi) {
                            uint32_t sv[kPart];
                            part(c, sv);
                            const float2 sc = scale_of(c);
                            const float k = factor(sc.x);
                            probabilities(sv, k, exponent(sc.y, largest16(sv) * k), pk);
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i) pk[i] = 0u;
                        }
                        tmem_st8(tmem_s + c * 8, pk);
                    }
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&misc->pv_full[x][pb]);
                ++pw;
            }
            if (!ok) break;

            // ------------------------------------ epilogue ------------------------------------
            if (nt > 0) {                                // the unit's last P V product has landed (and the P tile is free)
                ok = mbar_wait_warp(&misc->o_full[x], qc & 1, misc);
                if (!ok) break;
                const volatile uint32_t* nan = &misc->nan_branch[x][qc & 1][0][0];
                if (ns > 0 && (nan[b_row >> 5] | nan[4 + (b_row >> 5)]) >> (b_row & 31) & 1) l = __uint_as_float(0x7fffffffu);
                ++qc;
            }
            tc_fence_after();
            const int grow_row = u.row0 + b_row;
            const int hq = u.head * G + (u_row & (G - 1));
            const bool store = row_valid && grow_row < p.a.a.max_rows;
            const bool final_out = u.part_base < 0;
            // The pipeline's four warps meet (bounded, as all waits are).
            auto meet = [&]() {
                __syncwarp();
                if (lane == 0) mbar_arrive(&misc->meet[x]);
                return mbar_wait_warp(&misc->meet[x], meets++ & 1, misc);
            };
            float l_row = l, M_row = M;                  // of the row, both ways together
            if (ways == 2) {
                misc->way_ml[x][row] = make_float2(M, l);
                ok = meet();
                if (!ok) break;
                const float2 other = misc->way_ml[x][row ^ (kM / 2)];
                M_row = fmaxf(M, other.x);
                l_row = (M == -INFINITY ? l : l * ex2(M - M_row)) + (other.x == -INFINITY ? other.y : other.y * ex2(other.x - M_row));
            }
            // o = O 2^(R - 7 - M) / l, the power in two steps: it may be that of any V scale.  So are partial results: without the division, values of one
            // sign above 2^(119 - log2 of the chunk's tokens) could leave fp32 before the merge divides.
            const float two = R == -INFINITY ? 0.f : ex2(0.5f * (R - kUp - M_row));
            const float inv = two * (l_row == 0.f ? 0.f : 1.f / l_row);
            const int64_t pr = (static_cast<int64_t>(final_out ? 0 : u.part_base) + u.row_begin + b_row) * p.a.a.g.Hq + hq;
            float* po = p.part_o + pr * D;
            // the accumulator, 32 columns at a time; rolled: the code runs once per unit, out of a cold instruction cache
            auto read_o = [&](int c0, float (&acc)[32]) {
                if (warp_active && nt > 0) {
                    uint32_t ov[32];
                    tmem_ld32(tmem_o + c0, ov);
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 32; ++c) acc[c] = two * __uint_as_float(ov[c]) * inv;
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) acc[c] = 0.f;
                }
                if (c0 + 32 >= D && nt > 0) {            // all TMEM reads of this unit are done
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&misc->o_free[x]);
                }
            };
            if (ways == 2) {
                // Each way finishes half of the columns: it hands the other's over, 32 at a time and column by column, in the memory of the widened V
                // tile, which the conversion leaves alone until O is free.  (16 columns at a time from the second way to the first, in the staging
                // memory, took 5.7 k cycles of the unit.)
                static_assert(C::NV * C::WIDE_BYTES == 2 * 32 * (kM / 2) * 4, "two ways' 32 columns of 64 rows");
                float* hand = reinterpret_cast<float*>(smem + C::OFF_V + x * C::NV * C::WIDE_BYTES) + u_row;
                float *mine = hand + way * 32 * (kM / 2), *theirs = hand + (way ^ 1) * 32 * (kM / 2);
#pragma unroll 1
                for (int c0 = 0; c0 < D / 2 && ok; c0 += 32) {
                    uint32_t ov[32];
                    tmem_ld32(tmem_o + (way ^ 1) * (D / 2) + c0, ov);
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 32; ++c) mine[c * (kM / 2)] = two * __uint_as_float(ov[c]) * inv;
                    const int own = way * (D / 2) + c0;
                    tmem_ld32(tmem_o + own, ov);
                    ok = meet();
                    tmem_ld_wait();
                    if (!ok) break;
                    float acc[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) acc[c] = two * __uint_as_float(ov[c]) * inv + theirs[c * (kM / 2)];
                    if (store && final_out) {
                        uint4* to = reinterpret_cast<uint4*>(p.a.a.o + (static_cast<int64_t>(grow_row) * p.a.a.g.Hq + hq) * D + own);
#pragma unroll
                        for (int c = 0; c < 32; c += 8)
                            to[c / 8] = make_uint4(pack_bf16(acc[c], acc[c + 1]), pack_bf16(acc[c + 2], acc[c + 3]), pack_bf16(acc[c + 4], acc[c + 5]), pack_bf16(acc[c + 6], acc[c + 7]));
                    } else if (store) {
#pragma unroll
                        for (int c = 0; c < 32; c += 4) *reinterpret_cast<float4*>(po + own + c) = make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]);
                    }
                    if (c0 + 32 < D / 2) ok = meet();
                }
                if (!ok) break;
                tc_fence_before();                       // all TMEM reads of this unit are done (it has tiles), and what was handed over has been read
                __syncwarp();
                if (lane == 0) mbar_arrive(&misc->o_free[x]);
            } else if (final_out) {
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    float acc[32];
                    read_o(c0, acc);
                    // transpose through this warp's 1 KB of shared memory, 16 columns at a time: a row's go out as one 32-byte
                    // piece, 16 rows per store instruction
#pragma unroll
                    for (int c1 = 0; c1 < 32; c1 += 16) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float* a = acc + c1 + 8 * c;
                            *reinterpret_cast<uint4*>(stg + lane * 32 + (((c ^ (lane >> 2)) & 1) << 4)) =
                                make_uint4(pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(a[4], a[5]), pack_bf16(a[6], a[7]));
                        }
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int rl = 16 * i + (lane >> 1), ch = lane & 1;  // row inside the warp's 32, 16-byte piece
                            const uint4 pk = *reinterpret_cast<const uint4*>(stg + rl * 32 + (((ch ^ (rl >> 2)) & 1) << 4));
                            const int trow = quad * 32 + rl, tb = trow >> g_shift, grow = u.row0 + tb;
                            if (trow < nrows && grow < p.a.a.max_rows)
                                *reinterpret_cast<uint4*>(p.a.a.o + (static_cast<int64_t>(grow) * p.a.a.g.Hq + u.head * G + (trow & (G - 1))) * D + c0 + c1 + ch * 8) = pk;
                        }
                        __syncwarp();
                    }
                }
            } else {
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    float acc[32];
                    read_o(c0, acc);
                    if (store) {
#pragma unroll
                        for (int c = 0; c < 32; c += 4)
                            *reinterpret_cast<float4*>(po + c0 + c) = make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]);
                    }
                }
            }
            if (store && way == 0) {
                if (final_out) {
                    if (p.a.a.lse) p.a.a.lse[static_cast<int64_t>(grow_row) * p.a.a.g.Hq + hq] = l_row == 0.f ? -INFINITY : (M_row + log2f(l_row)) * kLn2;
                } else {
                    p.part_ml[pr * 2] = M_row; p.part_ml[pr * 2 + 1] = l_row;
                }
            }
        }
    }

    // ---------------------------------------- teardown ----------------------------------------
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (misc->abort_flag) {
        if (threadIdx.x == 0 && status) atomicOr(status, HPD_S_TIMEOUT);
        // give copies that may still be in flight time to land before the shared memory is released
        const long long t0 = clock64();
        while (clock64() - t0 < 20000000ll) { }
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// codes [rows, D]: boxes of box_rows rows, swizzled in rows of D bytes
bool make_codes_map(CUtensorMap* m, const void* base, int D, long long rows, int box_rows)
{
    auto fn = tensor_map_encoder();
    if (!fn) return false;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(rows)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(D)};
    cuuint32_t box[2] = {static_cast<cuuint32_t>(D), static_cast<cuuint32_t>(box_rows)};
    cuuint32_t es[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool TWO>
int launch_d(const PagedArgs& a)
{
    using C = Cfg<D>;
    // the dynamic shared-memory limit is an attribute of the kernel on ONE device: set it once per device
    static std::atomic<bool> attr_set[kMaxDevices];
    const int dev = current_device();
    if (dev < 0 || dev >= kMaxDevices || !attr_set[dev].load(std::memory_order_acquire)) {
        HPD_CUDA_TRY(cudaFuncSetAttribute(attn_paged_kernel<D, TWO>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM));
        if (dev >= 0 && dev < kMaxDevices) attr_set[dev].store(true, std::memory_order_release);
    }
    const hpd_geom& g = a.a.g;
    // an empty pool's map still needs an address: any will do, nothing is fetched through it
    const long long page_rows = static_cast<long long>(a.n_pages) * g.Hkv * a.page_size, branch_rows = static_cast<long long>(a.n_branch_pages) * g.Hkv * g.suffix_cap;
    const void* pages = page_rows > 0 ? static_cast<const void*>(a.page_k) : a.a.q;
    const void* branches = branch_rows > 0 ? static_cast<const void*>(a.branch_k) : a.a.q;
    Maps maps{};
    bool ok = make_q_map(&maps.q, a.a.q, D, g.Hq / g.Hkv, g.Hkv, a.a.max_rows) && make_codes_map(&maps.page, pages, D, std::max(page_rows, 1ll), a.page_size);
    for (int i = 0; i < std::min(16, g.suffix_cap) && ok; ++i) ok = make_codes_map(&maps.branch[i], branches, D, std::max(branch_rows, 1ll), i + 1);
    if (!ok) {
        set_last_cuda_error(cudaErrorInvalidValue);
        return HPD_E_CUDA;
    }
    Params p{};
    p.a = a;
    char* ws = static_cast<char*>(a.a.workspace);
    p.hdr = reinterpret_cast<const WsHeader*>(ws);
    p.work = reinterpret_cast<const WorkItem*>(ws + a.a.lay.off_work);
    p.part_ml = reinterpret_cast<float*>(ws + a.a.lay.off_ml);
    p.part_o = reinterpret_cast<float*>(ws + a.a.lay.off_o);
    p.scale_log2 = g.sm_scale * kLog2e;
    p.G = g.Hq / g.Hkv;
    attn_paged_kernel<D, TWO><<<sm_count(), kThreads, C::SMEM, a.a.stream>>>(maps, p);
    HPD_CUDA_TRY(cudaGetLastError());
    return launch_paged_merge(a.a);
}

}  // namespace

int launch_attn_paged(const PagedArgs& a)
{
    // Few rows to a document on average, or few documents (whose units are halved then).  By the rows that there may be: how many of them are live only
    // the device knows, so a step whose branches have mostly retired keeps the kernel of the full one.
    const long long rows = static_cast<long long>(a.a.max_rows) * (a.a.g.Hq / a.a.g.Hkv);
    const bool two = rows <= static_cast<long long>(a.a.n_docs) * (kM / 2) || 2ll * a.a.n_docs * a.a.g.Hkv <= sm_count();
    if (a.a.g.D == 128) return two ? launch_d<128, true>(a) : launch_d<128, false>(a);
    return two ? launch_d<64, true>(a) : launch_d<64, false>(a);
}

}  // namespace hpd
