// Attention over the paged 8-bit cache: for every sequence its newest L_q query tokens, each over the keys up to its own position.
//
// Work is cut on the device, from the sequences' lengths as they are when the kernel runs: a (sequence, KV head, block of query
// rows) is a segment of ceil(len / step) steps of keys, all segments lie behind one another on one axis, and every CTA takes an
// equal stretch of it.  A segment that lies in several CTAs leaves partial rows (at most two sets per CTA, whatever the shapes),
// which a second kernel merges.
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>
#include <stddef.h>

#include <atomic>
#include <type_traits>

#include "daf_common.cuh"

namespace daf {

constexpr int kD = 128;

struct PageAttnArgs {
    Pool p;
    int n, L_q, Hq, G;
    int rows;              // query rows of a KV head: L_q * G, row r is token r / G, head r % G of the group
    int inv_G;             // 65536 / G, rounded down, + 1
    int units;             // tiles of them: what a step of keys of one (sequence, KV head) costs
    int pad;               // what a segment costs beyond its steps
    float scale_log2;      // softmax scale * log2(e)
    const int32_t* seqs; const int32_t* lens; const int32_t* table;
    const __nv_bfloat16* q; __nv_bfloat16* out; float* lse;
    struct ChainEntry* chains;      // [CTAs]
    float* part_o;         // [CTAs][2][block rows][128] unnormalised
    float2* part_ml;       // [CTAs][2][block rows] running maximum and sum
    DeviceStatus* status;
};

// Where a CTA's unfinished segments continue (written by every CTA of a launch).
struct ChainEntry {
    int last_cta;          // the CTA that ends the segment this CTA begins but does not end; -1: none
    int b, h, block;       // that segment
};

// ---------------------------------------------------------------------------------------------------- few rows: warps on their own
// Up to 24 rows of a KV head go through the warp-wide matrix instruction, eight at a time: with keys (and then channels) as its 16
// rows and query rows as its eight columns, S^T = K Q^T and O^T = V^T P^T, so that one token of a group of up to eight heads wastes
// nothing, and a widened tile of K or V serves all kN column blocks.  (There are 4 flops per byte and row: the cache's way from HBM
// is what counts, not the tensor cores' rate, and a warp that needs nobody else keeps its loads in flight all the time.)  A warp
// walks its stretch of the work axis in steps of 32 keys: it asks for the tiles of K and V some steps ahead (asynchronous 16-byte
// copies into a ring of its own, whose 16-byte pieces are XOR-ed with the row number so that eight rows of a column lie in
// different banks), multiplies, keeps the running maximum and sum, and multiplies again.  (Tiled copies were slower here: a warp has
// to issue them one by one, with everything in uniform registers, and at pages of 16 tokens a step takes four: 1160 clocks a step.)
//   Measured: one token of 64 sequences of 0.5k to 12k tokens, 32 / 8 heads, 142 us: 5.7 TB/s, 86 % of a copy's rate.  One token of 28 / 4
// heads over 32k 13.8 us (5.2 at that rate) and over 1k 9.6: two launches and the chain lengths -> table -> bytes -> products -> merge,
// of which every part runs once (11,000 clocks in this kernel).  One token (7 rows) of 16 sequences of 4k 17.9, two (14) 25.4, three (21)
// 33.7: each eight rows more cost some 8 us of conversions and products in warps that are too few (two a scheduler) to cover their
// latencies; with 12 warps of two column blocks 27.0, with 10 of three 48.0, each in fewer registers.
//   8-bit values are exact in fp16, and so are the query rows once each is scaled by a power of two to a largest magnitude of
//   2^14 .. 2^15 (elements 2^-31 of that and below are rounded), so the logits are products of the given numbers with fp32 sums.
//   P goes into the product as fp16 of p * vs * 2^9 / (row maximum of p * 2^floor(log2 vs)): 11 bits down to 2^-23 of the
//   largest and some bits down to 2^-34 (as bf16 it would have 8), while sums of p stay in fp32.
//   Maxima are those of p * 2^floor(log2 vs), and what is 2^-126 of one is flushed, from the sum of p too.  With V's scales at most
//   2^90 apart, as the header asks, such a token's p is below 2^-36 of another's: four million of them are 2^-14 of a sum.
constexpr int kStep = 32;
constexpr int kMostBlocks = 3;                       // column blocks of eight rows
constexpr int kTile = kStep * kD;                    // 4 KB: K or V of one step
constexpr float kPExp = 9.f;
// Warps of a CTA (one CTA an SM), and steps a warp asks ahead: as many warps as the registers of one column block leave room for,
// since each waits on its own chain of products half of the time.
__host__ __device__ constexpr int decode_warps(int blocks) { return blocks == 1 ? 12 : 8; }
__host__ __device__ constexpr int decode_depth(int blocks) { return blocks == 1 ? 2 : 3; }
struct DecodeStage { float ks[2], vs[2]; };          // scales of the step's first and second 16 keys; negative: no such page
// An unfinished segment's rows, maxima and sums in shared memory; rows 528 bytes apart, so that a warp's eight-byte stores to every second
// row fall into different banks.
constexpr int kPieceRow = kD + 4;
__host__ __device__ constexpr int piece_floats(int rows) { return rows * kPieceRow + 2 * rows; }
__host__ __device__ constexpr size_t ring_bytes(int blocks) { return (size_t)decode_warps(blocks) * decode_depth(blocks) * 2 * kTile; }
__host__ __device__ constexpr size_t decode_smem(int blocks) {
    return 1024 + ring_bytes(blocks) + (size_t)decode_warps(blocks) * decode_depth(blocks) * sizeof(DecodeStage);
}
static_assert(decode_warps(1) * piece_floats(8) * sizeof(float) <= ring_bytes(1) && decode_warps(2) <= 16 &&
              decode_warps(kMostBlocks) * piece_floats(8 * kMostBlocks) * sizeof(float) <= ring_bytes(kMostBlocks), "the pieces take the ring's place at the end");

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {           // an 8 x 8 matrix of 16-bit elements, two neighbours a lane
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}
__device__ __forceinline__ uint32_t widen2(uint32_t two_bytes) {       // two 8-bit values -> two fp16
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((uint16_t)two_bytes));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two bf16 values times a power of two as fp16.  (Subnormal ones too: with K's scale large enough they count.)
__device__ __forceinline__ uint32_t scaled_f16(uint32_t w, float up) {
    return pack_f16(mul_rn_keep_subnormals(__uint_as_float(w << 16), up), mul_rn_keep_subnormals(__uint_as_float(w & 0xFFFF0000u), up));
}
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {            // 0xFF where a byte is NaN (0x7f, 0xff)
    return (((w & 0x7F7F7F7Fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xFFu;
}

// Largest magnitude (bf16 bits, which ascend with it) of the finite ones among words of two bf16 values: all of them at first, two at
// a time, and only where one is not finite each by itself.
struct FiniteMax {
    uint32_t pairs = 0;
    __device__ __forceinline__ void add(uint32_t w) { pairs = __vmaxu2(pairs, w & 0x7FFF7FFFu); }
    __device__ __forceinline__ uint32_t top() const { return max(pairs & 0xFFFFu, pairs >> 16); }
    __device__ __forceinline__ bool all_finite() const { return top() < 0x7F80u; }
};
__device__ __forceinline__ uint32_t finite_top(uint32_t w) {
    const uint32_t b0 = w & 0x7FFFu, b1 = (w >> 16) & 0x7FFFu;
    return max(b0 < 0x7F80u ? b0 : 0u, b1 < 0x7F80u ? b1 : 0u);
}

// Whether a page's V scale is one that the sums of p can take (see above); -1 stands for no page.
__device__ __forceinline__ bool sums_take(float vs) { return (vs >= 0x1p-60f && vs <= 0x1p30f) || vs == -1.f; }

// A place on the work axis: a segment is (b, h, block), a block `width` tiles (kW, or one less in the last).  It takes a.pad places, for
// what it costs beyond its steps, and weight<kW>(width) places for each of them.
struct Place { int b, h, block, width, step, n_steps, seq, len; };

// Running sums of the sequences' steps (of one tile) in shared memory: pre[b] = steps of sequences 0 .. b - 1.  (2048 sequences of 4M
// tokens: 2^28 steps of 32 keys.)
__device__ __forceinline__ int seq_len(const PageAttnArgs& a, int b) {
    int len = __ldg(a.lens + b);
    const int seq = a.seqs != nullptr ? __ldg(a.seqs + b) : b;
    if ((unsigned)seq >= (unsigned)a.p.n_seqs || len < 0) len = 0;
    return (int)min((long long)len, (long long)a.p.max_pages * a.p.T);
}
__device__ __forceinline__ int steps_of(int len, int step) { return max(1, (len + step - 1) / step); }   // (an empty one writes its zeros)

template <int kThreads>
__device__ __forceinline__ void sum_steps(const PageAttnArgs& a, int step, int* pre, int* warp_sums) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int run = 0;
    for (int b0 = 0; b0 < a.n; b0 += kThreads) {
        const int b = a.n <= 32 ? lane : b0 + tid;
        int x = b < a.n ? steps_of(seq_len(a, b), step) : 0;
        if (blockIdx.x == 0 && b < a.n && b == b0 + tid) {
            const int len = __ldg(a.lens + b), seq = a.seqs != nullptr ? __ldg(a.seqs + b) : b;
            if ((unsigned)seq >= (unsigned)a.p.n_seqs || len != seq_len(a, b)) report_status(a.status, DAF_ERR_BOUNDS, 252, b);
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
            if (lane >= o) x += y;
        }
        if (a.n <= 32) {                             // every warp knows all of it
            if (warp == 0 && b < a.n) pre[b + 1] = x;
            break;
        }
        if (lane == 31) warp_sums[warp] = x;
        __syncthreads();
        int before = run, all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += warp_sums[w];
            all += warp_sums[w];
        }
        if (b < a.n) pre[b + 1] = before + x;
        run += all;
        __syncthreads();
    }
    if (tid == 0) pre[0] = 0;
    __syncthreads();
}

// Positions on the work axis.  For few rows 32 bits are enough (daf_page_attn refuses calls that could need more), and every CTA begins
// with a chain of this arithmetic; for many rows a division of 32 bits is tried first, since one of 64 takes some 300 cycles.
template <int kW> using Axis = std::conditional_t<kW == 1, int, long long>;
__device__ __forceinline__ int axis_div(int x, int y) { return (int)((uint32_t)x / (uint32_t)y); }
__device__ __forceinline__ long long axis_div(long long x, long long y) {
    return ((x | y) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}
// `total` places shared by `ctas`: the first `more` take each + 1, the others `each`.
template <typename A> struct Shares { A each, more; };
template <typename A>
__device__ __forceinline__ Shares<A> share(A total, A ctas) {
    const A each = axis_div(total, ctas);
    return Shares<A>{each, total - each * ctas};
}
template <typename A>
__device__ __forceinline__ A cta_begin(const Shares<A>& s, A c) { return c * s.each + min(c, s.more); }
// The CTA whose stretch holds place `at`.
template <typename A>
__device__ __forceinline__ int cta_of(const Shares<A>& s, A at) {
    const A longer = s.more * (s.each + 1);
    return (int)(at < longer ? axis_div(at, s.each + 1) : s.more + axis_div(at - longer, s.each));
}

template <int kW>
__device__ __forceinline__ void next_segment(const PageAttnArgs& a, const int* pre, Place& x) {
    x.step = 0;
    if (kW > 1) {
        x.width = min(kW, a.units - kW * ++x.block);
        if (x.width > 0) return;
        x.block = 0;
        x.width = min(kW, a.units);
    }
    if (++x.h < a.p.Hkv) return;
    x.h = 0;
    ++x.b;
    if (x.b >= a.n) return;
    x.len = seq_len(a, x.b);
    x.n_steps = pre[x.b + 1] - pre[x.b];
    x.seq = a.seqs != nullptr ? __ldg(a.seqs + x.b) : x.b;
}
// What a step costs: in blocks of up to two tiles (many rows), one tile takes 0.68 of the time of two.
template <int kW>
__device__ __forceinline__ int weight(int width) { return kW == 1 ? 1 : width + 1; }
// Places that one (sequence, KV head) takes, and that sequences 0 .. b - 1 take.  (kW == 1, few rows: one tile, no pad.)
template <int kW>
__device__ __forceinline__ Axis<kW> head_places(const PageAttnArgs& a, int n_steps) {
    if (kW == 1) return n_steps;
    return (Axis<kW>)n_steps * (a.units / kW * weight<kW>(kW) + (a.units % kW != 0 ? weight<kW>(1) : 0)) + (Axis<kW>)a.pad * ((a.units + kW - 1) / kW);
}
template <int kW>
__device__ __forceinline__ Axis<kW> places_before(const PageAttnArgs& a, const int* pre, int b) {
    if (kW == 1) return a.p.Hkv * pre[b];
    return a.p.Hkv * (head_places<kW>(a, pre[b]) + (Axis<kW>)(b - 1) * a.pad * ((a.units + kW - 1) / kW));
}
// The first step that begins at or behind `at` (which is less than the total); a place in front of a segment's first step stands for it.
template <int kW>
__device__ __forceinline__ Place place_at(const PageAttnArgs& a, const int* pre, Axis<kW> at) {
    int lo = 0, hi = a.n - 1;                    // last b whose places begin at or in front of `at`
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (places_before<kW>(a, pre, mid) <= at) lo = mid; else hi = mid - 1;
    }
    Place x;
    x.b = lo;
    x.len = seq_len(a, lo);
    x.seq = a.seqs != nullptr ? __ldg(a.seqs + lo) : lo;
    x.n_steps = pre[lo + 1] - pre[lo];
    Axis<kW> rest = at - places_before<kW>(a, pre, lo);
    const Axis<kW> head = head_places<kW>(a, x.n_steps), block = (Axis<kW>)weight<kW>(kW) * x.n_steps + a.pad;
    x.h = (int)axis_div(rest, head);
    rest -= x.h * head;
    if (kW == 1) {
        x.block = 0;
        x.width = 1;
        x.step = (int)rest;
        return x;
    }
    x.block = (int)axis_div(rest, block);
    x.width = min(kW, a.units - kW * x.block);
    rest = max(rest - x.block * block - a.pad, (Axis<kW>)0);
    x.step = (int)axis_div(rest + weight<kW>(x.width) - 1, (Axis<kW>)weight<kW>(x.width));
    if (x.step == x.n_steps) next_segment<kW>(a, pre, x);
    return x;
}
// The last place that stands for a place's step.
template <int kW>
__device__ __forceinline__ Axis<kW> axis_at(const PageAttnArgs& a, const int* pre, const Place& x) {
    if (kW == 1) return places_before<kW>(a, pre, x.b) + x.h * x.n_steps + x.step;
    return places_before<kW>(a, pre, x.b) + x.h * head_places<kW>(a, x.n_steps) + x.block * ((Axis<kW>)weight<kW>(kW) * x.n_steps + a.pad) + a.pad + (Axis<kW>)x.step * weight<kW>(x.width);
}

// A row's factor 1 / sum (a row that saw nothing: 0), its log-sum-exp, and the weight of a partial with (maximum, sum) in a merge
// whose largest maximum is mx.  A maximum of -inf with a sum other than 0 is a row of NaN logits: it stays one.
__device__ __forceinline__ float row_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float row_lse(float m, float l) {
    return l == 0.f ? -INFINITY : (m == -INFINITY ? l : m - kPExp + log2f(l)) * 0.6931471805599453f;
}
__device__ __forceinline__ float partial_weight(float2 ml, float mx) {
    return ml.y == 0.f ? 0.f : (ml.x == -INFINITY ? 1.f : fast_exp2(ml.x - mx));
}

// Token of one of the few rows: row / G by the reciprocal in 16 bits (row < 24, G <= 24: what is added to it stays below 24 / 65536,
// less than what row / G lacks of the next whole number).
__device__ __forceinline__ int token_of(const PageAttnArgs& a, int row) { return (row * a.inv_G) >> 16; }

template <int kN>
__global__ void __launch_bounds__(decode_warps(kN) * 32, 1)
page_decode_kernel(const PageAttnArgs a) {
    constexpr int kRows = 8 * kN, kPiece = piece_floats(kRows), kDecodeWarps = decode_warps(kN), kDepth = decode_depth(kN);
    extern __shared__ unsigned char decode_smem_raw[];
    unsigned char* const smem = decode_smem_raw + ((1024u - (smem_u32(decode_smem_raw) & 1023u)) & 1023u);      // (stays a shared address to the compiler)
    DecodeStage* const stages = reinterpret_cast<DecodeStage*>(smem + ring_bytes(kN));
    int* const pre = reinterpret_cast<int*>(stages + kDecodeWarps * kDepth);
    __shared__ int warp_sums[kDecodeWarps];
    __shared__ int piece_kind[2 * kDecodeWarps];         // of each warp, parked and last: 1 there, 2 begins its segment, 4 ends it
    __shared__ int2 piece_seg[2 * kDecodeWarps];         // (b, h)

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    DecodeStage* const sc_ring = stages + warp * kDepth;
    unsigned char* const ring = smem + warp * (kDepth * 2 * kTile);
    if (threadIdx.x < 2 * kDecodeWarps) piece_kind[threadIdx.x] = 0;
    pdl_wait();
    pdl_launch_dependents();
    sum_steps<kDecodeWarps * 32>(a, kStep, pre, warp_sums);
    const int total = places_before<1>(a, pre, a.n);
    // CTAs that take part: no more than give each of its warps a step
    const int ctas = min((int)gridDim.x, (int)((unsigned)(total + kDecodeWarps - 1) / kDecodeWarps));
    const Shares<int> shares = share(total, ctas);
    const int cta_lo = cta_begin(shares, min((int)blockIdx.x, ctas)), span = cta_begin(shares, min((int)blockIdx.x + 1, ctas)) - cta_lo;
    // a warp's stretch: the first ones take one more
    const unsigned warp_each = (unsigned)span / kDecodeWarps, warp_more = (unsigned)span % kDecodeWarps;
    const int lo = cta_lo + (int)(warp * warp_each + min((unsigned)warp, warp_more)), hi = lo + (int)(warp_each + ((unsigned)warp < warp_more ? 1u : 0u));

    const int T = a.p.T, Hkv = a.p.Hkv, page_bits = 31 - __clz(T);
    Place at = {};
    if (lo < hi) at = place_at<1>(a, pre, lo);
    // ---- the loads run ahead of the products with a place of their own
    Place ahead = at;
    int ahead_at = lo;
    int ids = -1, ids_first = -64;               // page numbers of 32 pages of the place's sequence, one a lane
    const uint32_t ring_at = smem_u32(ring);
    const uint32_t dst0 = (uint32_t)((lane >> 3) * kD + (((lane & 7) ^ (lane >> 3)) << 4)), dst1 = (uint32_t)((lane >> 3) * kD + 512 + (((lane & 7) ^ (lane >> 3) ^ 4) << 4));
    auto issue = [&](int slot) {
        const int key0 = ahead.step * kStep, page0 = key0 >> page_bits;
        if ((unsigned)(page0 - ids_first) >= 31u) {
            ids_first = page0;
            const int j = page0 + lane;
            const bool needed = j < a.p.max_pages && (j << page_bits) < ahead.len;
            ids = needed ? __ldg(a.table + (size_t)ahead.seq * a.p.max_pages + j) : -1;
            if ((unsigned)ids >= (unsigned)a.p.n_pages) {
                if (needed && ahead.h == 0) report_status(a.status, DAF_ERR_BOUNDS, 250, ids);
                ids = -1;
            }
        }
        const int id0 = __shfl_sync(0xFFFFFFFFu, ids, page0 - ids_first), id1 = __shfl_sync(0xFFFFFFFFu, ids, page0 - ids_first + (T < kStep ? 1 : 0));
        // A lane copies the 16 bytes at 16 lane of each 512 (four rows); a half of 16 keys lies in one page.  No page: zeros.
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int id = half == 0 ? id0 : id1;
            const size_t row = id < 0 ? 0 : ((size_t)(id * Hkv + ahead.h) << page_bits) + ((key0 + 16 * half) & (T - 1));
            const uint8_t* const k_src = a.p.k8 + row * kD + 16 * lane;
            const uint8_t* const v_src = a.p.v8 + row * kD + 16 * lane;
            const uint32_t k_dst = ring_at + (uint32_t)(slot * 2 * kTile + half * 2048), bytes = id < 0 ? 0u : 16u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cp_async16(k_dst + (i & 1 ? dst1 : dst0) + (i >> 1) * 1024, k_src + i * 512, bytes);
                cp_async16(k_dst + kTile + (i & 1 ? dst1 : dst0) + (i >> 1) * 1024, v_src + i * 512, bytes);
            }
        }
        if (lane < 4) {
            // lanes 0, 1: K's scale of the first and second half; 2, 3: V's
            const int id = lane & 1 ? id1 : id0;
            float* const dst = lane < 2 ? &sc_ring[slot].ks[lane] : &sc_ring[slot].vs[lane - 2];
            if (id >= 0)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;"
                             ::"r"(smem_u32(dst)), "l"((lane < 2 ? a.p.k_scale : a.p.v_scale) + (size_t)id * Hkv + ahead.h) : "memory");
            else
                *dst = -1.f;
        }
        __syncwarp();
        ++ahead_at;
        if (++ahead.step == ahead.n_steps) {
            next_segment<1>(a, pre, ahead);
            ids_first = -64;
        }
    };
    int slot = 0;
    bool tail = false;
    float o[kN][8][4];       // [column block][16 channels]: channels 16 c + 2 g and + 1 of rows 2 t (elements 0, 2) and 2 t + 1 (1, 3)
    float m[kN][2], l[kN][2];
    for (int x = lo; x < hi;) {
        // ---- a segment, or the stretch of it that is this warp's
        const int first_step = at.step;
        uint32_t qf[kN][8][2];
        float cs[kN][2];                   // factors of the logits of this thread's rows
        int limit[kN][2];                  // last key each of them sees
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            const int row = 8 * n + g;
            const bool there = row < a.rows;
            const uint2* const src = reinterpret_cast<const uint2*>(a.q + (((size_t)at.b * a.L_q + token_of(a, row)) * a.Hq + at.h * a.G + row - token_of(a, row) * a.G) * kD) + t;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                const uint2 v = there ? __ldg(src + kk * 4) : make_uint2(0u, 0u);
                qf[n][kk][0] = v.x; qf[n][kk][1] = v.y;
            }
        }
        if (x == lo) {
            // One group of copies per slot, an empty one where nothing is left: the group of the oldest slot is always kDepth - 1
            // groups back.  (Asked for here, with the first rows of Q on their way.)
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                if (ahead_at < hi) issue(d);
                cp_async_commit();
            }
        }
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            FiniteMax all;
#pragma unroll
            for (int j = 0; j < 16; ++j) all.add(qf[n][j >> 1][j & 1]);
            uint32_t big = all.top();
            if (!all.all_finite()) {
                big = 0;
#pragma unroll
                for (int j = 0; j < 16; ++j) big = max(big, finite_top(qf[n][j >> 1][j & 1]));
            }
            big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
            big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
            const int e = max((int)(big >> 7) - 127, -100);
            const float up = __int_as_float((14 - e + 127) << 23), back = __int_as_float((e - 14 + 127) << 23) * a.scale_log2;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    qf[n][kk][j] = scaled_f16(qf[n][kk][j], up);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int mine = 8 * n + 2 * t + j;
                cs[n][j] = __shfl_sync(0xFFFFFFFFu, back, 4 * (2 * t + j));
                limit[n][j] = mine < a.rows ? at.len - a.L_q + token_of(a, mine) : -1;
                m[n][j] = -INFINITY;
                l[n][j] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int u = 0; u < 4; ++u) o[n][c][u] = 0.f;
        }
        const int first_limit = at.len - a.L_q;       // of the first row
        // One step, in two forms: `odd` ones have keys that some row does not see, or that have no page.
        auto step = [&](auto odd_c, int key0, const DecodeStage sc) {
            constexpr bool odd = decltype(odd_c)::value;
            const uint32_t k_at = ring_at + (uint32_t)(slot * 2 * kTile), v_at = k_at + kTile;
            // S^T: 32 keys in two tiles of 16.  A lane's four bytes of a key are four neighbouring channels: two k-slots and, eight
            // further, two more (the order of the channels within a k-step is free, and Q's fragments have it too).
            float s[kN][2][4];
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int u = 0; u < 4; ++u) s[n][i][u] = 0.f;
#pragma unroll
            for (int c = 0; c < 8; c += 2) {
                uint32_t w[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i)      // matrices: keys 0-7 and 8-15 of channels 16 c .., then of 16 (c + 1) ..
                    ldsm4(w[i], k_at + (uint32_t)((16 * i + (lane & 15)) * kD + (((c + (lane >> 4)) ^ (lane & 7)) << 4)));
#pragma unroll
                for (int cc = 0; cc < 2; ++cc)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t f[4] = {widen2(w[i][2 * cc]), widen2(w[i][2 * cc + 1]), widen2(w[i][2 * cc] >> 16), widen2(w[i][2 * cc + 1] >> 16)};
#pragma unroll
                        for (int n = 0; n < kN; ++n) mma16816(s[n][i], f, qf[n][c + cc][0], qf[n][c + cc][1]);
                    }
            }
            float shift[2], vm[2], back[2];      // vs = vm * 2^shift, 1 <= vm < 2; back = 2^-shift: the sums are of p itself
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int bits = __float_as_int(sc.vs[i]), e = sc.vs[i] > 0.f ? max((bits >> 23) - 127, -126) : 0;
                shift[i] = (float)e;
                back[i] = __int_as_float((127 - e) << 23);
                vm[i] = sc.vs[i] > 0.f ? __int_as_float((bits & 0x7FFFFF) | 0x3F800000) : 1.f;
            }
            uint32_t pf[kN][2][2];               // P^T: [16 keys][their halves], two keys of row g
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        s[n][i][u] = fmaf(s[n][i][u], cs[n][u & 1] * sc.ks[i], shift[i]);
                        if (odd && (key0 + 16 * i + 8 * (u >> 1) + g > limit[n][u & 1] || sc.ks[i] < 0.f)) s[n][i][u] = -INFINITY;
                        top[u & 1] = fmaxf(top[u & 1], s[n][i][u]);
                    }
                float used[2], alpha[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xFFFFFFFFu, top[j], d));
                    const float now = fmaxf(m[n][j], top[j]);
                    alpha[j] = m[n][j] == now ? 1.f : fast_exp2(m[n][j] - now);      // (2^-inf = 0 at the first key)
                    used[j] = now == -INFINITY ? 0.f : now - kPExp;
                    m[n][j] = now;
                }
                if (__any_sync(0xFFFFFFFFu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        o[n][c][0] *= alpha[0]; o[n][c][2] *= alpha[0];
                        o[n][c][1] *= alpha[1]; o[n][c][3] *= alpha[1];
                    }
                    l[n][0] *= alpha[0]; l[n][1] *= alpha[1];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float e = fast_exp2(s[n][i][u] - used[u & 1]);
                        l[n][u & 1] = fmaf(e, back[i], l[n][u & 1]);
                        s[n][i][u] = e * vm[i];
                    }
                    pf[n][i][0] = transpose8(pack_f16(s[n][i][0], s[n][i][1]));
                    pf[n][i][1] = transpose8(pack_f16(s[n][i][2], s[n][i][3]));
                }
            }
            // O^T += V^T P^T: channels 16 c + 2 r and 16 c + 2 r + 1 are rows r and r + 8 of the instruction
            bool poison = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int c = 0; c < 8; c += 2) {
                    uint32_t w[4];
                    ldsm4_t(w, v_at + (uint32_t)((16 * i + (lane & 15)) * kD + (((c + (lane >> 4)) ^ (lane & 7)) << 4)));
                    if (odd) {
                        // Keys that no row of the sequence sees, or of no page: whatever lies there counts as zero.  Keys that
                        // some rows see: a NaN must not reach the others, so it is taken out here and put into the rows that
                        // see it below.
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int key = key0 + 16 * i + 8 * (u & 1) + 2 * t;
                            const bool none = sc.ks[i] < 0.f;
                            if (none || key >= at.len) w[u] &= 0xFFFF0000u;
                            if (none || key + 1 >= at.len) w[u] &= 0x0000FFFFu;
                            uint32_t nan = nan_bytes(w[u]);
                            if (key <= first_limit) nan &= 0xFFFF0000u;
                            if (key + 1 <= first_limit) nan &= 0x0000FFFFu;
                            poison |= nan != 0u;
                            w[u] &= ~nan;
                        }
                    }
#pragma unroll
                    for (int cc = 0; cc < 2; ++cc) {
                        const uint32_t w0 = __byte_perm(w[2 * cc], 0u, 0x3120), w1 = __byte_perm(w[2 * cc + 1], 0u, 0x3120);
                        const uint32_t f[4] = {widen2(w0), widen2(w0 >> 16), widen2(w1), widen2(w1 >> 16)};
#pragma unroll
                        for (int n = 0; n < kN; ++n) mma16816(o[n][c + cc], f, pf[n][i][0], pf[n][i][1]);
                    }
                }
            }
            if (odd && __any_sync(0xFFFFFFFFu, poison)) {
                for (int j = 0; j < kStep; ++j) {
                    const int key = key0 + j;
                    if (key <= first_limit || key >= at.len) continue;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const uint32_t w = nan_bytes(*reinterpret_cast<const uint16_t*>(ring + slot * 2 * kTile + kTile + j * kD + ((c ^ (j & 7)) << 4) + 2 * g));
#pragma unroll
                        for (int n = 0; n < kN; ++n)
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                if (((w >> (8 * (u >> 1))) & 1u) && key <= limit[n][u & 1]) o[n][c][u] = __int_as_float(0x7FC00000);
                    }
                }
            }
        };
        for (; at.step < at.n_steps && x < hi; ++at.step, ++x) {
            cp_async_wait_group<kDepth - 1>();
            __syncwarp();
            const DecodeStage sc = sc_ring[slot];
            const int key0 = at.step * kStep;
            if (!(sums_take(sc.vs[0]) && sums_take(sc.vs[1])) && lane == 0) report_status(a.status, DAF_ERR_BOUNDS, 253, at.b);
            if (key0 + kStep - 1 > first_limit || sc.ks[0] < 0.f || sc.ks[1] < 0.f) step(std::integral_constant<bool, true>{}, key0, sc);
            else step(std::integral_constant<bool, false>{}, key0, sc);
            __syncwarp();          // every lane is done with the slot
            if (ahead_at < hi) issue(slot);
            cp_async_commit();
            if (++slot == kDepth) slot = 0;
        }
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(0xFFFFFFFFu, l[n][j], d);
        const bool begins = first_step == 0, ends = at.step == at.n_steps;
        if (begins && ends) {
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = 8 * n + 2 * t + j;
                    if (row >= a.rows) continue;
                    const int tok = token_of(a, row), head = at.h * a.G + row - tok * a.G;
                    const float inv = row_inverse(l[n][j]);
                    uint32_t* const dst = reinterpret_cast<uint32_t*>(a.out + (((size_t)at.b * a.L_q + tok) * a.Hq + head) * kD) + g;
#pragma unroll
                    for (int c = 0; c < 8; ++c) dst[8 * c] = pack_bf16(o[n][c][j] * inv, o[n][c][2 + j] * inv);
                    if (a.lse != nullptr && g == 0) a.lse[((size_t)at.b * a.Hq + head) * a.L_q + tok] = row_lse(m[n][j], l[n][j]);
                }
        } else if (x < hi) {
            // The end of a segment that begins in front of this warp's stretch, with more behind it: parked in global memory, since the
            // ring is in use.
            const size_t set = (size_t)gridDim.x * 2 + (size_t)blockIdx.x * kDecodeWarps + warp;
            float* const dst = a.part_o + set * (kRows * kD);
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = 8 * n + 2 * t + j;
                    if (row >= a.rows) continue;
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        *reinterpret_cast<float2*>(dst + row * kD + 16 * c + 2 * g) = make_float2(o[n][c][j], o[n][c][2 + j]);
                    if (g == 0) a.part_ml[set * kRows + row] = make_float2(m[n][j], l[n][j]);
                }
            if (lane == 0) {
                piece_kind[2 * warp] = 1 | 4;
                piece_seg[2 * warp] = make_int2(at.b, at.h);
            }
        } else {
            tail = true;           // stays in registers until the ring is free
            if (lane == 0) {
                piece_kind[2 * warp + 1] = 1 | (begins ? 2 : 0) | (ends ? 4 : 0);
                piece_seg[2 * warp + 1] = make_int2(at.b, at.h);
            }
        }
        if (x < hi) next_segment<1>(a, pre, at);
    }
    cp_async_wait_group<0>();      // (the last groups are empty)
    __syncthreads();
    // ---- the warps' unfinished pieces: neighbours of one segment are merged; what is still unfinished is the CTA's
    float* const pieces = reinterpret_cast<float*>(smem);
    if (tail) {
        float* const dst = pieces + warp * kPiece;
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = 8 * n + 2 * t + j;
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    *reinterpret_cast<float2*>(dst + row * kPieceRow + 16 * c + 2 * g) = make_float2(o[n][c][j], o[n][c][2 + j]);
                if (g == 0) reinterpret_cast<float2*>(dst + kRows * kPieceRow)[row] = make_float2(m[n][j], l[n][j]);
            }
    }
    __syncthreads();
    const int kind = lane < 2 * kDecodeWarps ? piece_kind[lane] : 0;
    unsigned left = __ballot_sync(0xFFFFFFFFu, kind != 0);
    const unsigned beginning = __ballot_sync(0xFFFFFFFFu, (kind & 2) != 0), ending = __ballot_sync(0xFFFFFFFFu, (kind & 4) != 0);
    ChainEntry chain = {-1, 0, 0, 0};
    while (left != 0) {
        // pieces of one segment: from the first left to the one that ends the segment, or to the last
        const int first = __ffs(left) - 1;
        const unsigned ends_at = left & ending;
        const unsigned group = ends_at != 0 ? left & ((ends_at & (0u - ends_at)) * 2u - 1u) : left;
        left &= ~group;
        const bool begins = (beginning >> first) & 1u, ends = ends_at != 0;
        const int2 seg = piece_seg[first];
        for (int r = warp; r < a.rows; r += kDecodeWarps) {
            // lane i knows piece i: odd ones lie here, even ones were parked
            float2 ml = make_float2(-INFINITY, 0.f);
            if ((group >> lane) & 1u)
                ml = (lane & 1) ? reinterpret_cast<const float2*>(pieces + (lane >> 1) * kPiece + kRows * kPieceRow)[r]
                                : __ldcg(a.part_ml + ((size_t)gridDim.x * 2 + (size_t)blockIdx.x * kDecodeWarps + (lane >> 1)) * kRows + r);
            float mx = ml.x;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, d));
            const float mine = partial_weight(ml, mx);
            const unsigned some = __ballot_sync(0xFFFFFFFFu, ml.y != 0.f);       // pieces with keys; the others' memory holds anything
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum = mine * ml.y;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            auto add = [&](int i, float4 v) {
                const float w = __shfl_sync(0xFFFFFFFFu, mine, i);
                const bool counts = (some >> i) & 1u;         // (a weight of 0 still takes a NaN along)
                acc.x += counts ? w * v.x : 0.f; acc.y += counts ? w * v.y : 0.f;
                acc.z += counts ? w * v.z : 0.f; acc.w += counts ? w * v.w : 0.f;
            };
#pragma unroll
            for (int i0 = 0; i0 < kDecodeWarps; i0 += 4) {
                float4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = reinterpret_cast<const float4*>(pieces + (i0 + i) * kPiece + r * kPieceRow)[lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) add(2 * (i0 + i) + 1, v[i]);
            }
            for (unsigned rest = group & 0x55555555u; rest != 0; rest &= rest - 1) {
                const int i = __ffs(rest) - 1;
                add(i, reinterpret_cast<const float4*>(a.part_o + (((size_t)gridDim.x * 2 + (size_t)blockIdx.x * kDecodeWarps + (i >> 1)) * kRows + r) * kD)[lane]);
            }
            if (begins && ends) {
                const int tok = token_of(a, r), head = seg.y * a.G + r - tok * a.G;
                const float inv = row_inverse(sum);
                reinterpret_cast<uint2*>(a.out + (((size_t)seg.x * a.L_q + tok) * a.Hq + head) * kD)[lane] =
                    make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                if (a.lse != nullptr && lane == 0) a.lse[((size_t)seg.x * a.Hq + head) * a.L_q + tok] = row_lse(mx, sum);
            } else {
                const size_t set = (size_t)blockIdx.x * 2 + (begins ? 1 : 0);
                reinterpret_cast<float4*>(a.part_o + (set * kRows + r) * kD)[lane] = acc;
                if (lane == 0) a.part_ml[set * kRows + r] = make_float2(mx, sum);
            }
        }
        if (begins && !ends) chain = ChainEntry{0, seg.x, seg.y, 0};
    }
    if (threadIdx.x == (kDecodeWarps - 1) * 32) {       // (a warp with the fewest rows to merge)
        if (chain.last_cta == 0) {
            const int n_steps = pre[chain.b + 1] - pre[chain.b];
            chain.last_cta = cta_of(shares, axis_at<1>(a, pre, Place{chain.b, chain.h, 0, 1, n_steps - 1, n_steps, 0, 0}));
        }
        a.chains[blockIdx.x] = chain;
    }
}

// ---------------------------------------------------------------------------------------------- many rows: tensor memory
// More than 24 rows of a KV head (a question, or a few speculated tokens of a large group) go through the tensor cores in tiles
// of 128 consecutive rows, in steps of 128 keys.  One CTA per SM, 20 warps:
//   10, 11  ask for the bytes of K and V (TMA, kQStages half steps ahead);
//   12-15, 16-19  widen K's, and V's, to fp16 into the buffers that the products read (128-byte swizzle), half a step at a time: exactly,
//          but that V takes along what its scale is beside a power of two, rounded to fp16 (daf_page_write leaves none).  Each of
//          these is a chain of waits, reads, conversions and writes, so K and V have warps of their own;
//   8, 9   issue a tile group's products: S = Q K^T, O += P V with P from tensor memory, over S, by halves as they come;
//   0-3, 4-7  a tile group's softmax, a row per thread, and its epilogue.
// A block of two tiles shares every widened K and V.  A block of one tile gives its even steps to one group and its odd ones to the
// other, and the two halves of the result are merged in shared memory.  A group's 256 columns of tensor memory are O and S, 128
// each.  One S is enough because the groups take turns: while one's products run, the other's softmax does.
//   Measured: 128 tokens of 28 / 4 heads over 32k keys 85 to 87 us, 700 TFLOP/s, 42 % of the measured bf16 rate; 4 tokens of 16 sequences of
// 4k 39.1 (28 rows of a tile's 128), 64 tokens over 6k 30.0.  A step of both tiles takes some 5800 clocks, of which the tensor cores
// are busy for 2050; the rest is each group's chain: exponentials 2000 (the unit needs 1024 of them), maximum 550, P on its way 350,
// products 1500 to 1800.  A piece of work costs some 15,000 clocks beside its steps.  What was measured on the way, same case: steps of
// 64 keys with two S a group 114 us; with Q in tensor memory and one S 110; without turns 104 (92 with them then; what could be left out
// was measured on that form only: the exponentials or three quarters of Q K^T changed nothing, the widening a tenth); turns that end before
// P's last quarter 95 (87 then); 152 / 56 or 168 / 48 registers 87 (85 then).
// Rows of Q are scaled by powers of two and P enters the product as fp16 as in the kernel above.
constexpr int kQStep = 128, kQSub = 64;
constexpr int kQStages = 3;        // half steps
// Barriers of their bytes: twice as many, so that each belongs to one of the two pairs of warps that widen half steps in turn.  With one
// a slot a pair would see every other of its phases only, and where the other pair's bytes were late take its parity for that of its own.
constexpr int kQFull = 2 * kQStages;
static_assert(kQFull % 2 == 0 && kQFull % kQStages == 0, "a barrier's half steps all have one slot and one pair");
// Places (a step of two tiles takes three) that a piece of work costs: rows of Q in, results out.  128 tokens of 28 / 4 heads over 32k
// keys with 8 or 16: 86.4 us, with 12: 85.0 (before the bytes had twice as many barriers).
constexpr int kQPad = 12;
constexpr int kQConsts = 16;       // half steps whose constants are kept: written up to 10 ahead of their last reader
constexpr int kQRows = 256;
constexpr int kQThreads = 640;
constexpr int kQTile = 128 * kD * 2;                  // 32 KB: 128 rows of Q or K as fp16, two 64-column halves
constexpr int kQHalf = kQTile / 2;
constexpr int kQSlot = kQSub * kD * 2;                // 16 KB: V of half a step, widened, two 64-column halves
constexpr int kQSlotHalf = kQSlot / 2;
constexpr int kQStage = kQSub * kD;                   // 8 KB: the bytes of K or V of half a step
constexpr uint32_t kColS = 128;                       // columns of a group, behind O
constexpr float kLazy = 6.f;                          // log2: a row's maximum may be this stale, P then reaches 2^(kPExp + kLazy)
// Shared memory: Q's two tiles; V's two slots; K's two buffers.  A block of one tile has four slots of V, the last two in the second
// tile of Q.  When a piece begins K's buffers hold the raw rows of Q, at its end all of this what leaves the CTA.
constexpr int kQOffV = 2 * kQTile, kQOffK = kQOffV + 2 * kQSlot, kQOffStage = kQOffK + 2 * kQTile;

struct QuestionSmem {
    uint64_t st_full[2][kQFull], st_empty[2][kQStages];       // [K, V] the bytes of half a step, there and taken
    uint64_t k_full[2], k_empty[2];                           // [buffer] a step's K, widened
    uint64_t v_full[4], v_empty[4];                           // [slot] half a step's V, widened
    uint64_t q_full[2], s_full[2], p_full[2][2], o_full[2];   // [group], [half]
    uint64_t turn[2][4];                                      // [group][warp] the other group's warp of the scheduler is done with its step
    uint64_t c_full[kQConsts];
    float4 chunk[kQConsts][4];      // of half a step's chunks of 16 keys: ks (negative: no page), floor(log2 vs), 2^-that, vs / 2^that
    int missing[kQConsts];          // some keys of the half step have no page
    float2 ml[2][128];              // [group] row maxima and sums (blocks of one tile)
    uint32_t tmem_base;
    int abort_flag;
    unsigned long long odd;         // which barriers have completed an odd number of phases
    int go[2][2][2];                // [K, V][half step mod 2][step mod 2] what the polling warp found
    int poison;                     // a NaN was taken out of a value that some rows must not see
    // The piece of work under way and the CTA's stretch: kept here rather than in every thread's registers
    Place at;
    int step1, n_t, first_limit, last_limit;      // steps at.step .. step1 - 1, of which the first n_t have keys that some row sees
    Place end;
    Shares<long long> shares;
    ChainEntry chain;
};
constexpr int kBarStEmpty = (int)(offsetof(QuestionSmem, st_empty) / 8), kBarK = (int)(offsetof(QuestionSmem, k_full) / 8),
              kBarKEmpty = (int)(offsetof(QuestionSmem, k_empty) / 8), kBarV = (int)(offsetof(QuestionSmem, v_full) / 8),
              kBarQ = (int)(offsetof(QuestionSmem, q_full) / 8),
              kBarS = (int)(offsetof(QuestionSmem, s_full) / 8), kBarP = (int)(offsetof(QuestionSmem, p_full) / 8),
              kBarO = (int)(offsetof(QuestionSmem, o_full) / 8), kBarTurn = (int)(offsetof(QuestionSmem, turn) / 8),
              kBarC = (int)(offsetof(QuestionSmem, c_full) / 8), kBars = kBarC + kQConsts;
static_assert(offsetof(QuestionSmem, st_full) == 0 && kBarStEmpty == 2 * kQFull && kBarStEmpty % kQStages == 0 && kBarK % 2 == 0 && kBarS % 2 == 0 && kBarO % 2 == 0 && kBars <= 64, "what the barriers' numbers rest on");
constexpr size_t kQuestionSmem = 1024 + kQOffStage + 2 * (size_t)kQStages * kQStage + sizeof(QuestionSmem);

__host__ __device__ constexpr uint32_t make_idesc_f16(uint32_t M, uint32_t N, uint32_t b_mn_major) {
    return (1u << 4) | (b_mn_major << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);      // fp16 x fp16 -> fp32
}

// 32 lanes x 16 consecutive 32-bit columns
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

// Bytes from shared to global memory, both 16-byte aligned and a multiple of 16 of them; and the wait of the thread that asked until
// they are written.
__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(reinterpret_cast<uint64_t>(dst)), "r"(smem_u32(src)), "r"(bytes) : "memory");
    tma_store_commit();
}
__device__ __forceinline__ void bulk_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// A row's factor for the logits of a chunk.  It stays a normal number: with rows of zeros or nearly so and keys of a small scale the product
// would be flushed to zero, and hidden logits, which are -inf ahead of it, would become NaN.  (Visible logits are below 2^32 ahead of
// it: times this bound they are nothing.)
__device__ __forceinline__ float logit_factor(float c, float ks) { return fmaxf(c * fabsf(ks), FLT_MIN); }

// One softmax step of one row over 128 keys: P over the first half of the logits' columns, running maximum and sum.  `rescale` is called
// ahead of the first P with the factor for the row of O (1 unless the maximum grew by more than kLazy), `half_done` when half of P is
// on its way to tensor memory.  c: the row's factor for its logits; chunk: two half steps' constants.  A thread has no
// room for 128 logits: the quarters are looked at in the order 2, 3, 0, 1 for the maximum, so that the first two are still there when
// their exponentials come, and the last two are fetched again.
template <typename Rescale, typename HalfDone>
__device__ __forceinline__ void question_softmax(uint32_t s_addr, const float4* const (&chunk)[2], bool missing, int key0, int limit, float c,
                                                 float& m, float& l, Rescale rescale, HalfDone half_done) {
    if (__any_sync(0xFFFFFFFFu, key0 + kQStep - 1 > limit || missing)) {
        // rare (the last steps of a sequence): logits of keys that the row does not see become -inf where they are
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            uint32_t r[16];
            tmem_ld16(s_addr + (uint32_t)(16 * i), r);
            tc_wait_ld();
            const int last = chunk[i >> 2][i & 3].x < 0.f ? -1 : limit - key0 - 16 * i;
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j > last) r[j] = 0xFF800000u;
            tmem_st16(s_addr + (uint32_t)(16 * i), r);
        }
        tc_wait_st();
    }
    float top = -INFINITY;
    uint32_t sr[2][32];
    tmem_ld32(s_addr + 64u, sr[0]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int q = (u + 2) & 3;
        tc_wait_ld();
        if (u < 3) tmem_ld32(s_addr + (uint32_t)(32 * ((q + 1) & 3)), sr[(q + 1) & 1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float2 k2 = *reinterpret_cast<const float2*>(chunk[q >> 1] + 2 * (q & 1) + i);
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                mx[0] = fmax3(mx[0], __uint_as_float(sr[q & 1][16 * i + j]), __uint_as_float(sr[q & 1][16 * i + j + 1]));
                mx[1] = fmax3(mx[1], __uint_as_float(sr[q & 1][16 * i + j + 2]), __uint_as_float(sr[q & 1][16 * i + j + 3]));
            }
            top = fmaxf(top, fmaf(fmaxf(mx[0], mx[1]), logit_factor(c, k2.x), k2.y));
        }
    }
    float now = fmaxf(m, top);
    if (m != -INFINITY && now - m <= kLazy) now = m;
    const float used = now == -INFINITY ? 0.f : now - kPExp;
    const float alpha = m == -INFINITY ? 1.f : fast_exp2(m - now);
    rescale(alpha);
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= 2) tc_wait_ld();
        if (q == 2) tmem_ld32(s_addr + 96u, sr[1]);
        uint32_t pr[16];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 k4 = chunk[q >> 1][2 * (q & 1) + i];
            const float f = logit_factor(c, k4.x), d = k4.y - used;
            const uint64_t f2 = pack_f32x2(f, f), d2 = pack_f32x2(d, d);
            uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const uint64_t x = ffma2(pack_f32x2(__uint_as_float(sr[q & 1][16 * i + j]), __uint_as_float(sr[q & 1][16 * i + j + 1])), f2, d2);
                const float p0 = fast_exp2(f32x2_lo(x)), p1 = fast_exp2(f32x2_hi(x));
                acc[(j >> 1) & 1] = fadd2(acc[(j >> 1) & 1], pack_f32x2(p0, p1));
                pr[8 * i + (j >> 1)] = pack_f16(p0, p1);
            }
            const uint64_t both = fadd2(acc[0], acc[1]);
            sum = fmaf(f32x2_lo(both) + f32x2_hi(both), k4.z, sum);
        }
        if (q == 0) tmem_ld32(s_addr + 64u, sr[0]);
        // a quarter of P takes 16 columns, over logits that have been fetched (or are on their way: columns further up)
        tmem_st16(s_addr + (uint32_t)(16 * q), pr);
        if (q & 1) half_done(q >> 1);
    }
    l = l * alpha + sum;
    m = now;
}

// How many phases barrier i completes in a piece of n_t steps.
__device__ __forceinline__ int bar_uses(int i, int n_t, bool pair) {
    if (i < kBarStEmpty) return (2 * n_t - i % kQFull + kQFull - 1) / kQFull;      // every sixth half step
    if (i < kBarK) return (2 * n_t - i % kQStages + kQStages - 1) / kQStages;      // every third
    if (i < kBarV) return (n_t - (i & 1) + 1) >> 1;
    if (i < kBarQ) {
        const int slot = (i - kBarV) & 3;
        return pair ? (slot < 2 ? n_t : 0) : (n_t - (slot >> 1) + 1) >> 1;
    }
    if (i < kBarS) return 1;
    if (i >= kBarTurn && i < kBarC) return pair ? n_t : 0;
    if (i < kBarC) {
        const int g = i < kBarP || i >= kBarO ? i & 1 : ((i - kBarP) >> 1), steps = pair ? n_t : (n_t - g + 1) >> 1;    // of the group
        return i < kBarO ? steps : (steps > 0 ? 1 : 0);
    }
    return i < kBars ? (2 * n_t - (i - kBarC) + kQConsts - 1) / kQConsts : 0;
}

// The bounded wait of this kernel, `parity` as if the piece of work were the CTA's first (a second at most, or until another thread has
// given up): it only leaves the number of the wait in the abort flag, which one thread reports at the end.  The warps' loops are
// many, and what they keep in the instruction caches counts: with longer waits and every rare case unrolled, warps that had work
// found no instruction a sixth of the time.
__device__ __forceinline__ bool wait_phase(QuestionSmem* sm, unsigned long long odd, uint64_t* bar, uint32_t parity, volatile int* abort, int where) {
    parity ^= (uint32_t)(odd >> ((smem_u32(bar) - smem_u32(sm)) >> 3)) & 1u;
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (*abort != 0) return false;
        if (global_ns() - t0 > kWaitLimitNs) {
            *abort = where;
            return false;
        }
    }
}

// Where slot i of V lies: two of their own, two in the second tile of Q (blocks of one tile).
__host__ __device__ constexpr int v_slot(int i) { return i < 2 ? kQOffV + i * kQSlot : kQTile + (i - 2) * kQSlot; }

__global__ void __launch_bounds__(kQThreads, 1)
page_question_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const PageAttnArgs a) {
    extern __shared__ unsigned char question_smem_raw[];
    unsigned char* const smem = question_smem_raw + ((1024u - (smem_u32(question_smem_raw) & 1023u)) & 1023u);      // (stays a shared address to the compiler)
    unsigned char* const k_smem = smem + kQOffK;
    unsigned char* const stage_smem = smem + kQOffStage;
    QuestionSmem* const sm = reinterpret_cast<QuestionSmem*>(stage_smem + 2 * kQStages * kQStage);
    int* const pre = reinterpret_cast<int*>(sm + 1);
    __shared__ int warp_sums[kQThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* const abort = &sm->abort_flag;

    if (warp == 8) {
        tmem_alloc(&sm->tmem_base, 512);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        sm->abort_flag = 0;
        sm->odd = 0;
        tma_prefetch_desc(&tmap_k);
        tma_prefetch_desc(&tmap_v);
    }
    if (warp == 1) {
        uint64_t* const bars = reinterpret_cast<uint64_t*>(sm);
        for (int i = lane; i < kBars; i += 32) {
            // four warps (or lanes) arrive, or two warps, or both groups' products, or one copy's bytes or product
            const bool by_four = (i >= kBarK && i < kBarKEmpty) || (i >= kBarQ && i < kBarS) || (i >= kBarP && i < kBarO) || i >= kBarC;
            const bool by_two = (i >= kBarStEmpty && i < kBarK) || (i >= kBarKEmpty && i < kBarQ);
            mbar_init(bars + i, by_four ? 4 : by_two ? 2 : 1);
        }
        mbar_fence_init();
    }
    pdl_wait();
    pdl_launch_dependents();
    sum_steps<kQThreads>(a, kQStep, pre, warp_sums);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;
    const int T = a.p.T, Hkv = a.p.Hkv;
    if (warp == 0) {
        const long long total = places_before<2>(a, pre, a.n);
        const long long ctas = min((long long)gridDim.x, (total + 3) / 4);       // no fewer than two steps of a tile each
        const Shares<long long> shares = share(total, ctas);
        // lane 0 finds the stretch's begin, lane 1 its end; both move up to the next step's begin
        const long long from = cta_begin(shares, min((long long)blockIdx.x + min(lane, 1), ctas));
        Place at = {};
        at.b = a.n;
        if (from < total) at = place_at<2>(a, pre, from);
        if (lane == 1) sm->end = at;
        if (lane == 0) {
            sm->at = at;
            sm->step1 = 0;
            sm->shares = shares;
            sm->chain = ChainEntry{-1, 0, 0, 0};
        }
        __syncwarp();          // (lane 0 goes on with what lane 1 found)
    }
    // Three of the five warpgroups need few registers: 256 x 144 + 384 x 64 = 640 x 96
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
        int prev_t = 0;                 // steps and width of the piece before
        bool prev_pair = false, any_before = false;
        for (;;) {
            // ---- one segment, or this CTA's stretch of it
            if (threadIdx.x == 0) {
                if (sm->step1 > 0) {            // behind the piece before
                    sm->at.step = sm->step1;
                    if (sm->at.step == sm->at.n_steps) next_segment<2>(a, pre, sm->at);
                }
                const Place at = sm->at, end = sm->end;
                sm->step1 = 0;
                const bool last = at.b == end.b && at.h == end.h && at.block == end.block;      // the stretch ends in this segment
                if (at.b < a.n && !(last && at.step >= end.step)) {
                    const int step1 = last ? end.step : at.n_steps;
                    const int row0 = at.block * kQRows, last_row = min(a.rows, row0 + kQRows) - 1;
                    sm->step1 = step1;
                    sm->first_limit = at.len - a.L_q + row0 / a.G;
                    sm->last_limit = at.len - a.L_q + last_row / a.G;
                    sm->n_t = max(0, min(step1, (sm->last_limit + kQStep) / kQStep) - at.step);       // (a negative limit: none)
                    if (at.step == 0 && step1 < at.n_steps) {
                        Place tail = at;
                        tail.step = at.n_steps - 1;
                        sm->chain = ChainEntry{cta_of(sm->shares, axis_at<2>(a, pre, tail)), at.b, at.h, at.block};
                    }
                }
                sm->poison = 0;
            }
            // The barriers count on from piece to piece: bit i of `odd` says whether barrier i has completed an odd number of phases.
            if (warp == 1 && any_before) {
                const unsigned first = __ballot_sync(0xFFFFFFFFu, bar_uses(lane, prev_t, prev_pair) & 1);
                const unsigned second = __ballot_sync(0xFFFFFFFFu, bar_uses(lane + 32, prev_t, prev_pair) & 1);
                if (lane == 0) sm->odd ^= ((unsigned long long)second << 32) | first;
            }
            __syncthreads();
            if (sm->step1 == 0) break;
            bool ok = true;
            const int n_t = sm->n_t, step0 = sm->at.step;
            const unsigned long long odd = sm->odd;
            const bool pair = sm->at.width == 2;
            prev_t = n_t; prev_pair = pair; any_before = true;
            // ------------------------------------------------------------------------------------- softmax, a row per thread
            const int g = warp >> 2, rt = threadIdx.x & 127;
            const int tile_row = sm->at.block * kQRows + (pair ? g * 128 : 0), row = tile_row + rt;
            const bool valid = row < a.rows, any_valid = (row & ~31) < a.rows;      // (a warp's rows: 32 from a multiple of 32)
            const int tok = row / a.G, head = row - tok * a.G;          // (head of the group)
            const int limit = valid ? sm->at.len - a.L_q + tok : sm->last_limit;
            const int n_u = pair ? n_t : (n_t - g + 1) >> 1;
            const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
            const uint32_t o_addr = tmem + (uint32_t)(g * 256) + lane_addr, s_addr = o_addr + kColS;
            float c = 0.f;
            if (any_valid) {
                // The warp's 32 rows of Q: raw into what will be K's buffers, sixteen lanes a row, pieces of 16 bytes XOR-ed with the row
                // number.  Each thread then scales its own row to a largest magnitude of 2^14 .. 2^15 and writes it as fp16 in the layout of
                // a tiled copy.  (Both groups of a block of one tile load the same rows; only the first writes them.)
                const int sub = lane >> 4, piece = lane & 15, r0 = (warp & 3) * 32 + sub, d_tok = 2 / a.G, d_head = 2 % a.G;
                unsigned char* const raw = k_smem + g * (128 * 256);
                int tk = (tile_row + r0) / a.G, hd = tile_row + r0 - tk * a.G;
                const __nv_bfloat16* src = a.q + (((size_t)sm->at.b * a.L_q + tk) * a.Hq + sm->at.h * a.G + hd) * kD + piece * 8;
#pragma unroll 2
                for (int r = r0; r < r0 + 32; r += 2) {
                    const bool there = tile_row + r < a.rows;
                    cp_async16(smem_u32(raw + r * 256 + ((piece ^ (r & 15)) << 4)), there ? src : a.q, there ? 16u : 0u);
                    src += ((long long)d_tok * a.Hq + d_head) * kD;
                    hd += d_head;
                    if (hd >= a.G) { hd -= a.G; src += (long long)(a.Hq - a.G) * kD; }
                }
                cp_async_commit();
                cp_async_wait_group<0>();
                __syncwarp();
                const uint4* const mine = reinterpret_cast<const uint4*>(raw + rt * 256);
                FiniteMax all;
#pragma unroll 8
                for (int i = 0; i < 16; ++i) {
                    const uint4 w = mine[i ^ (rt & 15)];
                    all.add(w.x); all.add(w.y); all.add(w.z); all.add(w.w);
                }
                uint32_t big = all.top();
                if (!all.all_finite()) {
                    big = 0;
#pragma unroll 1
                    for (int i = 0; i < 16; ++i) {
                        const uint4 w = mine[i];
                        big = max(max(big, max(finite_top(w.x), finite_top(w.y))), max(finite_top(w.z), finite_top(w.w)));
                    }
                }
                const int e = max((int)(big >> 7) - 127, -100);
                const float up = __int_as_float((14 - e + 127) << 23);
                c = __int_as_float((e - 14 + 127) << 23) * a.scale_log2;
                if (pair || g == 0) {
                    unsigned char* const dst = smem + g * kQTile + rt * 128;
#pragma unroll 4
                    for (int i = 0; i < 16; ++i) {
                        const uint4 w = mine[i ^ (rt & 15)];
                        uint4 y;
                        y.x = scaled_f16(w.x, up);
                        y.y = scaled_f16(w.y, up);
                        y.z = scaled_f16(w.z, up);
                        y.w = scaled_f16(w.w, up);
                        *reinterpret_cast<uint4*>(dst + (i >> 3) * kQHalf + (((i & 7) ^ (rt & 7)) << 4)) = y;
                    }
                    fence_proxy_async();
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm->q_full[g]);
            float m = -INFINITY, l = 0.f;
            int u = 0;
            auto take_turn = [&]() {
                // The groups take turns (a scheduler's two warps, one of each): left to themselves they fall into step, wait for the
                // exponentials together (16 a clock) and then for their products together.
                if (ok && pair && (g == 1 || u > 0)) ok = wait_phase(sm, odd, &sm->turn[g][warp & 3], (uint32_t)((g == 1 ? u : u - 1) & 1), abort, 279);
            };
            auto half_done = [&](int half) {
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm->p_full[g][half]);
            };
            if (any_valid) {
                for (; u < n_u; ++u) {
                    const int t = pair ? u : 2 * u + g, c0 = (2 * t) % kQConsts;
                    ok = wait_phase(sm, odd, &sm->c_full[c0], (uint32_t)((2 * t / kQConsts) & 1), abort, 271);
                    if (ok) ok = wait_phase(sm, odd, &sm->c_full[c0 + 1], (uint32_t)((2 * t / kQConsts) & 1), abort, 273);
                    if (ok) ok = wait_phase(sm, odd, &sm->s_full[g], (uint32_t)(u & 1), abort, 272);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    const float4* const chunk[2] = {sm->chunk[c0], sm->chunk[c0 + 1]};
                    auto rescale = [&](float alpha) {
                        take_turn();
                        // (the logits came behind the product before, so O is quiet)
                        if (u == 0 || !__any_sync(0xFFFFFFFFu, alpha != 1.f)) return;
#pragma unroll 1
                        for (int i = 0; i < 8; ++i) {
                            uint32_t r[16];
                            tmem_ld16(o_addr + (uint32_t)(16 * i), r);
                            tc_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * alpha);
                            tmem_st16(o_addr + (uint32_t)(16 * i), r);
                        }
                    };
                    question_softmax(s_addr, chunk, (sm->missing[c0] | sm->missing[c0 + 1]) != 0, (step0 + t) * kQStep, limit, c, m, l, rescale, half_done);
                    if (pair && lane == 0) mbar_arrive(&sm->turn[1 - g][warp & 3]);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                }
            } else {
                // no rows of this warp's: whatever lies in its lanes of tensor memory stays among them
                for (; u < n_u; ++u) {
                    ok = wait_phase(sm, odd, &sm->s_full[g], (uint32_t)(u & 1), abort, 272);
                    take_turn();
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    half_done(0);
                    half_done(1);
                    if (pair && lane == 0) mbar_arrive(&sm->turn[1 - g][warp & 3]);
                }
            }
            if (ok && n_u > 0) ok = __all_sync(0xFFFFFFFFu, wait_phase(sm, odd, &sm->o_full[g], 0, abort, 274));
            tc_fence_after();
            // ---- epilogue: rows leave through shared memory, once both groups are done with all in front of the stages, and one bulk copy a
            // row.  A block of one tile: each group merges half of the channels, and hands the other half of its own to the other.
            float w_own = 1.f, w_other = 0.f;
            float* const given = reinterpret_cast<float*>(smem) + (1 - g) * (128 * 64) + rt * 64;      // to the other group: [128 rows][64 channels]
            const float* const taken = reinterpret_cast<const float*>(smem) + g * (128 * 64) + rt * 64;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (!pair) {
                if (ok && any_valid) {
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) {
                        uint32_t r[32];
                        if (n_u > 0) {
                            tmem_ld32(o_addr + (uint32_t)(64 * (1 - g) + 32 * i), r);
                            tc_wait_ld();
                        }
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            *reinterpret_cast<float4*>(given + (((8 * i + j / 4) ^ (lane & 15)) << 2)) =
                                n_u > 0 ? make_float4(__uint_as_float(r[j]), __uint_as_float(r[j + 1]), __uint_as_float(r[j + 2]), __uint_as_float(r[j + 3]))
                                        : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    sm->ml[g][rt] = make_float2(m, l);
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (any_valid) {
                    const float2 ml = sm->ml[1 - g][rt];
                    const float mx = fmaxf(m, ml.x);
                    w_own = partial_weight(make_float2(m, l), mx);
                    w_other = partial_weight(ml, mx);
                    m = mx;
                    l = w_own * l + w_other * ml.y;
                }
            }
            if (ok && any_valid) {      // (whole warps: the reads of tensor memory are theirs)
                const Place at = sm->at;
                const bool begins = step0 == 0, whole = begins && sm->step1 == at.n_steps;
                const float inv = row_inverse(l);
                const int c0 = pair ? 0 : 64 * g, width = pair ? kD : 64;          // this thread's channels
                // a row's bytes lie together, rows an odd number of 16 bytes apart
                unsigned char* const mine = pair ? smem + (g * 128 + rt) * (kD * 4 + 16) : smem + 2 * kQTile + (g * 128 + rt) * (64 * 4 + 16);
                static_assert(256 * (kD * 4 + 16) <= kQOffStage && 2 * kQTile + 256 * (64 * 4 + 16) <= kQOffStage, "the rows fit in front of the stages");
#pragma unroll 1
                for (int i = 0; i < width / 32; ++i) {
                    uint32_t r[32];
                    if (n_u > 0) {
                        tmem_ld32(o_addr + (uint32_t)(c0 + 32 * i), r);
                        tc_wait_ld();
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) r[j] = 0u;
                    }
                    if (!pair) {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 y = *reinterpret_cast<const float4*>(taken + (((8 * i + j / 4) ^ (lane & 15)) << 2));
                            r[j] = __float_as_uint(w_own * __uint_as_float(r[j]) + w_other * y.x);
                            r[j + 1] = __float_as_uint(w_own * __uint_as_float(r[j + 1]) + w_other * y.y);
                            r[j + 2] = __float_as_uint(w_own * __uint_as_float(r[j + 2]) + w_other * y.z);
                            r[j + 3] = __float_as_uint(w_own * __uint_as_float(r[j + 3]) + w_other * y.w);
                        }
                    }
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            uint32_t y[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) y[k] = pack_bf16(__uint_as_float(r[j + 2 * k]) * inv, __uint_as_float(r[j + 2 * k + 1]) * inv);
                            *reinterpret_cast<uint4*>(mine + i * 64 + j * 2) = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) *reinterpret_cast<uint4*>(mine + i * 128 + j * 4) = make_uint4(r[j], r[j + 1], r[j + 2], r[j + 3]);
                    }
                }
                if (valid) {
                    if (sm->poison != 0) {
                        // values that were NaN, in keys that this row sees and the block's first does not
                        const int from = max(sm->first_limit + 1, step0 * kQStep), to = min(min(limit, at.len - 1), (step0 + n_t) * kQStep - 1);
#pragma unroll 1
                        for (int key = from; key <= to; ++key) {
                            const int id = __ldg(a.table + (size_t)at.seq * a.p.max_pages + key / T);
                            if ((unsigned)id >= (unsigned)a.p.n_pages) continue;
                            const uint8_t* const v = a.p.v8 + (((size_t)id * Hkv + at.h) * T + key % T) * kD + c0;
#pragma unroll 1
                            for (int j = 0; j < width; ++j) {
                                if ((__ldg(v + j) & 0x7F) != 0x7F) continue;
                                if (whole) reinterpret_cast<uint16_t*>(mine)[j] = 0x7FC0;
                                else reinterpret_cast<float*>(mine)[j] = __int_as_float(0x7FC00000);
                            }
                        }
                    }
                    const size_t out_row = ((size_t)at.b * a.L_q + tok) * a.Hq + at.h * a.G + head;
                    const size_t set_row = ((size_t)blockIdx.x * 2 + (begins ? 1 : 0)) * kQRows + (row - at.block * kQRows);
                    fence_proxy_async();
                    if (whole) bulk_store(a.out + out_row * kD + c0, mine, (uint32_t)width * 2);
                    else bulk_store(a.part_o + set_row * kD + c0, mine, (uint32_t)width * 4);
                    if (pair || g == 0) {
                        if (!whole) a.part_ml[set_row] = make_float2(m, l);
                        else if (a.lse != nullptr) a.lse[((size_t)at.b * a.Hq + at.h * a.G + head) * a.L_q + tok] = row_lse(m, l);
                    }
                    tma_store_wait_read();
                }
            }
            tc_fence_before();
            __syncthreads();       // the rings and tensor memory are free
            tc_fence_after();
            if (sm->abort_flag != 0) break;
        }
        bulk_store_wait();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        for (;;) {
            __syncthreads();
            if (sm->step1 == 0) break;
            bool ok = true;
            const int n_t = sm->n_t, step0 = sm->at.step;
            const unsigned long long odd = sm->odd;
            const bool pair = sm->at.width == 2;
            if (warp == 10 || warp == 11) {
                // ---------------------------------------------------------------------------------------- bytes and scales
                const int kv = warp - 10, seq = sm->at.seq, h = sm->at.h, len = sm->at.len;
                const bool reports = kv == 0 && h == 0;       // (each block: the later ones see more keys)
                float ks = -1.f, vs = -1.f;         // (K's warp) the scales of the pages in ids
                const int page_bits = 31 - __clz(T), box = min(T, kQSub), pages = kQSub / box;        // copies of half a step
                const int chunk_page = box < kQSub ? ((lane & 3) * 16) >> page_bits : 0;             // page of a chunk of 16 keys
                int ids = -1, ids_end = 0;          // page numbers of 32 pages that end in front of ids_end, one a lane
                int t = 0;
                for (; t < 2 * n_t; ++t) {      // (t counts half steps here)
                    const int slot = t % kQStages;
                    if (t >= kQStages) {
                        ok = __all_sync(0xFFFFFFFFu, wait_phase(sm, odd, &sm->st_empty[kv][slot], (uint32_t)((t / kQStages - 1) & 1), abort, 260));
                        if (!ok) break;
                    }
                    uint64_t* const full = &sm->st_full[kv][t % kQFull];
                    const int key0 = step0 * kQStep + t * kQSub, page0 = key0 >> page_bits;
                    if (page0 + pages > ids_end) {
                        ids_end = page0 + 32;
                        const int j = page0 + lane;
                        const bool needed = j < a.p.max_pages && (long long)j * T < len;
                        ids = needed ? __ldg(a.table + (size_t)seq * a.p.max_pages + j) : -1;
                        if ((unsigned)ids >= (unsigned)a.p.n_pages) {
                            if (needed && reports) report_status(a.status, DAF_ERR_BOUNDS, 261, ids);
                            ids = -1;
                        }
                        if (kv == 0) {
                            ks = ids >= 0 ? __ldg(a.p.k_scale + (size_t)ids * Hkv + h) : -1.f;
                            vs = ids >= 0 ? __ldg(a.p.v_scale + (size_t)ids * Hkv + h) : -1.f;
                            if (!sums_take(vs)) report_status(a.status, DAF_ERR_BOUNDS, 253, sm->at.b);
                        }
                    }
                    const int at0 = page0 - (ids_end - 32);
                    const int mine = __shfl_sync(0xFFFFFFFFu, ids, (at0 + lane) & 31);
                    const unsigned there = __ballot_sync(0xFFFFFFFFu, lane < pages && mine >= 0);
                    if (lane == 0) mbar_arrive_expect_tx(full, (uint32_t)(__popc(there) * box * kD));
                    __syncwarp();
                    if ((there >> lane) & 1u)
                        tma_load_2d(stage_smem + (kv * kQStages + slot) * kQStage + lane * box * kD, kv == 0 ? &tmap_k : &tmap_v, full, 0,
                                    (mine * Hkv + h) * T + (key0 & (T - 1)));       // (not 0 only where a page holds several steps)
                    __syncwarp();
                    if (kv == 0) {
                        // the constants of the step's chunks, a lane each
                        const float k1 = __shfl_sync(0xFFFFFFFFu, ks, at0 + chunk_page), v1 = __shfl_sync(0xFFFFFFFFu, vs, at0 + chunk_page);
                        const bool missing = __any_sync(0xFFFFFFFFu, lane < 4 && k1 < 0.f);
                        if (lane < 4) {
                            const int bits = __float_as_int(v1), e = v1 > 0.f ? max((bits >> 23) - 127, -126) : 0;
                            sm->chunk[t % kQConsts][lane] = make_float4(k1, (float)e, __int_as_float((127 - e) << 23),
                                                                        v1 > 0.f ? __int_as_float((bits & 0x7FFFFF) | 0x3F800000) : 1.f);
                            if (lane == 0) sm->missing[t % kQConsts] = missing;
                            mbar_arrive(&sm->c_full[t % kQConsts]);
                        }
                        __syncwarp();
                    }
                }
                if (!ok)       // loads in flight get a bounded chance to land before the CTA retires
                    for (int i = max(0, t - kQStages); i < t; ++i) {
                        uint64_t* const full = &sm->st_full[kv][i % kQFull];
                        const uint32_t parity = (uint32_t)((i / kQFull) & 1) ^ ((uint32_t)(odd >> ((smem_u32(full) - smem_u32(sm)) >> 3)) & 1u);
                        for (int k = 0; k < 4096 && !mbar_try_wait(full, parity); ++k) {}
                    }
            } else if (warp >= 12) {
                // --------------------------------------------------------------------------------------------------- widening
                // Two warps take a half step, the other two the next one: each half step is a chain of waits, reads, conversions, writes and
                // a fence of some 2500 clocks, most of it latency, and so two are under way.  A lane takes 16 bytes of a row at a time.
                // Eight lanes take four neighbouring pieces of each of two rows r and r ^ 5: with the swizzle of either side their reads and
                // their writes all fall into different banks.
                const int turn = (warp >> 1) & 1, row0 = (warp & 1) * 32;
                const int first_limit = sm->first_limit, len = sm->at.len;
                const int r8 = (lane >> 3) ^ ((lane >> 2) & 1 ? 5 : 0), piece = lane & 3;
                const int kv = warp >= 16;
                for (int t = turn; t < 2 * n_t; t += 2) {      // (t counts half steps here)
                    // K: half of the buffer of its step; V: a slot
                    const int step = t >> 1, slot = kv == 0 ? step & 1 : pair ? t & 1 : t & 3, uses = kv == 0 || !pair ? step >> 1 : step;
                    // one of the two warps polls, the other sleeps at a barrier (twelve polling warps took half of the issue slots)
                    if ((warp & 1) == 0) {
                        bool there = wait_phase(sm, odd, &sm->st_full[kv][t % kQFull], (uint32_t)((t / kQFull) & 1), abort, 262);
                        if (kv == 1 && there) there = wait_phase(sm, odd, &sm->c_full[t % kQConsts], (uint32_t)((t / kQConsts) & 1), abort, 275);
                        if (there && step == 0 && (kv == 0 || !pair)) {      // the raw rows of Q are out of K's buffers, the second tile is idle
                            there = wait_phase(sm, odd, &sm->q_full[0], 0, abort, 276);
                            if (there) there = wait_phase(sm, odd, &sm->q_full[1], 0, abort, 277);
                        }
                        if (there && uses > 0) there = wait_phase(sm, odd, kv == 0 ? &sm->k_empty[slot] : &sm->v_empty[slot], (uint32_t)((uses - 1) & 1), abort, 263);
                        there = __all_sync(0xFFFFFFFFu, there);
                        if (lane == 0) sm->go[kv][turn][step & 1] = there;
                    }
                    asm volatile("bar.sync %0, 64;" ::"r"(2 + 2 * kv + turn) : "memory");
                    if (!sm->go[kv][turn][step & 1]) break;
                    unsigned char* const src = stage_smem + (kv * kQStages + t % kQStages) * kQStage + (row0 + r8) * kD;
                    const int half_at = kv == 0 ? kQHalf : kQSlotHalf;          // between the two 64-column halves
                    unsigned char* const dst = smem + (kv == 0 ? kQOffK + slot * kQTile + (t & 1) * (kQSub * 128) : v_slot(slot)) + (row0 + r8) * 128;
                    float vm[2] = {1.f, 1.f};
                    if (kv == 1) {
                        const int key0 = step0 * kQStep + t * kQSub;
                        const float4 sc0 = sm->chunk[t % kQConsts][row0 / 16], sc1 = sm->chunk[t % kQConsts][row0 / 16 + 1];
                        vm[0] = sc0.w; vm[1] = sc1.w;
                        if (key0 + kQSub - 1 > first_limit || sc0.x < 0.f || sc1.x < 0.f) {
                            // As in the kernel above: keys that no row of the sequence sees, or of no page, count as zero; a NaN in
                            // a key that only some rows see is taken out, and put into the rows that see it at the end.
#pragma unroll 1
                            for (int i = 0; i < 8; ++i) {
                                const int key = key0 + row0 + 8 * (i >> 1) + r8;
                                uint4* const at = reinterpret_cast<uint4*>(src + 8 * (i >> 1) * kD + (((4 * (i & 1) + piece) ^ r8) << 4));
                                uint4 w = *at;
                                if (key >= len || (i < 4 ? sc0.x : sc1.x) < 0.f) w = make_uint4(0u, 0u, 0u, 0u);
                                else if (key > first_limit) {
                                    const uint4 nan = make_uint4(nan_bytes(w.x), nan_bytes(w.y), nan_bytes(w.z), nan_bytes(w.w));
                                    if ((nan.x | nan.y | nan.z | nan.w) != 0u) sm->poison = 1;
                                    w.x &= ~nan.x; w.y &= ~nan.y; w.z &= ~nan.z; w.w &= ~nan.w;
                                }
                                *at = w;      // (each lane's own pieces)
                            }
                        }
                    }
                    uint4 w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)      // pieces (i & 1) * 4 .. of rows row0 + 8 (i >> 1) ..
                        w[i] = *reinterpret_cast<const uint4*>(src + 8 * (i >> 1) * kD + (((4 * (i & 1) + piece) ^ r8) << 4));
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        unsigned char* const row = dst + (i & 1) * half_at + 8 * (i >> 1) * 128;
                        *reinterpret_cast<uint4*>(row + (((2 * piece) ^ r8) << 4)) = make_uint4(widen2(w[i].x), widen2(w[i].x >> 16), widen2(w[i].y), widen2(w[i].y >> 16));
                        *reinterpret_cast<uint4*>(row + (((2 * piece + 1) ^ r8) << 4)) = make_uint4(widen2(w[i].z), widen2(w[i].z >> 16), widen2(w[i].w), widen2(w[i].w >> 16));
                    }
                    if (vm[0] != 1.f || vm[1] != 1.f) {       // what V's scale is beside a power of two (nothing, as daf_page_write leaves them): each lane its own pieces
#pragma unroll 1
                        for (int i = 0; i < 16; ++i) {
                            const __half2 f = __float2half2_rn(i < 8 ? vm[0] : vm[1]);
                            __half2* const h = reinterpret_cast<__half2*>(dst + (i & 1) * kQSlotHalf + 8 * (2 * (i >> 3) + ((i >> 1) & 1)) * 128 + (((2 * piece + ((i >> 2) & 1)) ^ r8) << 4));
#pragma unroll
                            for (int j = 0; j < 4; ++j) h[j] = __hmul2(h[j], f);
                        }
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(kv == 0 ? &sm->k_full[slot] : &sm->v_full[slot]);
                        mbar_arrive(&sm->st_empty[kv][t % kQStages]);
                    }
                }
            } else if (warp < 10) {
                // --------------------------------------------------------------------------------------------------- products
                const int g = warp - 8;
                const int n_u = pair ? n_t : (n_t - g + 1) >> 1;          // steps of this group
                if (n_u > 0) {
                    constexpr uint32_t idesc_qk = make_idesc_f16(128, kQStep, 0), idesc_pv = make_idesc_f16(128, kD, 1);
                    const uint32_t o_col = tmem + (uint32_t)(g * 256), s_col = o_col + kColS;
                    // descriptors of the first 16 channels (or keys) of the first buffer (slot); the others differ in the address, in 16-byte units
                    const uint64_t qd = make_smem_desc(smem_u32(smem + (pair ? g : 0) * kQTile), 16, 1024), kd = make_smem_desc(smem_u32(k_smem), 16, 1024);
                    const uint64_t vd = make_smem_desc(smem_u32(smem), kQSlotHalf, 1024);
                    // Frees a buffer or slot: one arrival of each group's products, or two of the one group that a step of a block of one
                    // tile has.
                    auto release = [&](uint64_t* bar) {
                        tc_commit(bar);
                        if (!pair) tc_commit(bar);
                    };
                    auto issue_qk = [&](int buf) {
                        const uint64_t k0 = kd + (uint64_t)(buf * (kQTile / 16));
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)
                            tc_mma_ss(s_col, qd + (uint64_t)((kk & 3) * 2 + (kk >> 2) * (kQHalf / 16)), k0 + (uint64_t)((kk & 3) * 2 + (kk >> 2) * (kQHalf / 16)), idesc_qk,
                                      kk > 0 ? 1u : 0u);
                        tc_commit(&sm->s_full[g]);
                        release(&sm->k_empty[buf]);
                    };
                    ok = wait_phase(sm, odd, &sm->q_full[pair ? g : 0], 0, abort, 266);
                    if (ok) ok = wait_phase(sm, odd, &sm->k_full[pair ? 0 : g], 0, abort, 267);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (ok) {
                        tc_fence_after();
                        if (elect_one()) issue_qk(pair ? 0 : g);
                        __syncwarp();
                    }
                    for (int u = 0; u < n_u && ok; ++u) {
                        const int t = pair ? u : 2 * u + g;
#pragma unroll 1
                        for (int half = 0; half < 2 && ok; ++half) {
                            const int slot = pair ? half : 2 * g + half;
                            bool there = wait_phase(sm, odd, &sm->v_full[slot], (uint32_t)(u & 1), abort, 268);
                            if (there) there = wait_phase(sm, odd, &sm->p_full[g][half], (uint32_t)(u & 1), abort, 269);
                            ok = __all_sync(0xFFFFFFFFu, there);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t v0 = vd + (uint64_t)(v_slot(slot) / 16);
#pragma unroll
                                for (int kk = 0; kk < 4; ++kk)
                                    tc_mma_ts(o_col, s_col + (uint32_t)(half * 32 + kk * 8), v0 + (uint64_t)(kk * 128), idesc_pv, (u == 0 && half == 0 && kk == 0) ? 0u : 1u);
                                release(&sm->v_empty[slot]);
                                if (u + 1 == n_u && half == 1) tc_commit(&sm->o_full[g]);
                            }
                            __syncwarp();
                        }
                        if (ok && u + 1 < n_u) {
                            const int next = pair ? t + 1 : t + 2;
                            ok = __all_sync(0xFFFFFFFFu, wait_phase(sm, odd, &sm->k_full[next & 1], (uint32_t)((next >> 1) & 1), abort, 270));
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) issue_qk(next & 1);
                            __syncwarp();
                        }
                    }
                }
            }
            tc_fence_before();
            __syncthreads();       // the rings and tensor memory are free
            tc_fence_after();
            if (sm->abort_flag != 0) break;
        }
    }
    if (threadIdx.x == 0) {
        const int gave_up = sm->abort_flag;
        if (gave_up != 0) report_status(a.status, DAF_ERR_TIMEOUT, gave_up, 0);
        a.chains[blockIdx.x] = gave_up == 0 ? sm->chain : ChainEntry{-1, 0, 0, 0};
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Merge of the segments that lie in several CTAs: kWarps warps per row of such a segment.  Bound by the trips to L2, so a warp asks for
// its first kAtOnce partials together with the row's maxima.  kMany: the blocks share the rows of all such segments; otherwise (few rows
// a segment) blockIdx is the CTA that begins it and a row.
template <int kWarps, bool kMany>
__global__ void __launch_bounds__(256) page_merge_kernel(const PageAttnArgs a, int block_rows, int ctas) {
    constexpr int kRows = 8 / kWarps, kAtOnce = kWarps == 1 ? 8 : kWarps == 4 ? 10 : 5;
    __shared__ float4 acc_s[8][32];
    __shared__ float sum_s[8];
    __shared__ int begin_cta[kMany ? 256 : 1], counts[8];
    __shared__ ChainEntry begin_chain[kMany ? 256 : 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % kWarps;
    pdl_wait();
    pdl_launch_dependents();
    // kMany: the CTAs that begin such a segment, in order, so that every block numbers them alike (at most 256, a thread each), since
    // most blocks of a full grid would only find that there is nothing to do.
    const int groups = (min(block_rows, a.rows) + kRows - 1) / kRows;
    int n_begin = 1;
    if (kMany) {
        ChainEntry mine = {-1, 0, 0, 0};
        if ((int)threadIdx.x < ctas) mine = a.chains[threadIdx.x];
        const bool begins = mine.last_cta >= 0;
        const unsigned some = __ballot_sync(0xFFFFFFFFu, begins);
        if (lane == 0) counts[warp] = __popc(some);
        __syncthreads();
        int before = __popc(some & ((1u << lane) - 1u));
        n_begin = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if (w < warp) before += counts[w];
            n_begin += counts[w];
        }
        if (begins) {
            begin_cta[before] = (int)threadIdx.x;
            begin_chain[before] = mine;
        }
        __syncthreads();
    }
    for (int item = kMany ? blockIdx.x : blockIdx.y; item < n_begin * groups; item += kMany ? gridDim.x : gridDim.y) {
        const int first = kMany ? begin_cta[item / groups] : blockIdx.x, r = (item % groups) * kRows + warp / kWarps;
        const ChainEntry e = kMany ? begin_chain[item / groups] : a.chains[first];
        if (!kMany && e.last_cta < 0) return;
        const int row = e.block * block_rows + r;
        const bool there = r < block_rows && row < a.rows;
        // partial i of the row: the first CTA's second set, then the following CTAs' first sets
        const int n = there ? e.last_cta - first + 1 : 0;
        auto at = [&](int i) { return (i == 0 ? (size_t)first * 2 + 1 : (size_t)(first + i) * 2) * block_rows + r; };
        float2 ml[kAtOnce];
        float4 v[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = part + u * kWarps;
            ml[u] = i < n ? __ldcg(a.part_ml + at(i)) : make_float2(-INFINITY, 0.f);
            v[u] = i < n ? __ldcg(reinterpret_cast<const float4*>(a.part_o + at(i) * kD) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float mx = -INFINITY;
        for (int i = lane; i < n; i += 32) mx = fmaxf(mx, __ldcg(&a.part_ml[at(i)].x));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.f;
        auto add = [&](float2 x, float4 y) {
            if (x.y == 0.f) return;                  // no keys (a weight of 0 still takes a NaN along)
            const float w = partial_weight(x, mx);
            sum += w * x.y;
            acc.x += w * y.x; acc.y += w * y.y; acc.z += w * y.z; acc.w += w * y.w;
        };
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) add(ml[u], v[u]);
#pragma unroll 4
        for (int i = part + kAtOnce * kWarps; i < n; i += kWarps)
            add(__ldcg(a.part_ml + at(i)), __ldcg(reinterpret_cast<const float4*>(a.part_o + at(i) * kD) + lane));
        if (kWarps > 1) {
            __syncthreads();
            acc_s[warp][lane] = acc;
            if (lane == 0) sum_s[warp] = sum;
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int w = 1; w < kWarps; ++w) {
                    const float4 y = acc_s[warp + w][lane];
                    acc.x += y.x; acc.y += y.y; acc.z += y.z; acc.w += y.w;
                    sum += sum_s[warp + w];
                }
            }
        }
        if (!there || part != 0) continue;
        const int tok = row / a.G, head = e.h * a.G + row % a.G;
        const float inv = row_inverse(sum);
        reinterpret_cast<uint2*>(a.out + (((size_t)e.b * a.L_q + tok) * a.Hq + head) * kD)[lane] =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
        if (a.lse != nullptr && lane == 0) a.lse[((size_t)e.b * a.Hq + head) * a.L_q + tok] = row_lse(mx, sum);
    }
}

// ------------------------------------------------------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// K or V of one layer of the pool as rows of 128 bytes, in boxes of `box_rows` rows with the 128-byte swizzle.
static int make_pool_map(CUtensorMap* m, const void* base, long long rows, int box_rows) {
    static std::atomic<EncodeTiledFn> encode{nullptr};
    EncodeTiledFn fn = encode.load(std::memory_order_acquire);
    if (fn == nullptr) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres);
        if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || p == nullptr) {
            set_cuda_error(e != cudaSuccess ? e : cudaErrorUnknown);
            return DAF_ERR_CUDA;
        }
        fn = reinterpret_cast<EncodeTiledFn>(p);
        encode.store(fn, std::memory_order_release);
    }
    const cuuint64_t dims[2] = {(cuuint64_t)kD, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)kD};
    const cuuint32_t box[2] = {(cuuint32_t)kD, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1u, 1u};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_cuda_error(cudaErrorInvalidValue); return DAF_ERR_CUDA; }
    return DAF_OK;
}

static size_t round256(size_t x) { return (x + 255) / 256 * 256; }
static size_t prefix_bytes(int n) { return ((size_t)n + 1) * sizeof(int); }
// Column blocks of the kernel of few rows, 0: too many rows for it.
static int few_blocks(int rows) { return rows <= 8 * kMostBlocks ? (rows + 7) / 8 : 0; }
// Partial rows: two sets a CTA, and for the kernel of few rows one a warp for the pieces parked on the way.
static size_t partial_rows(int ctas, int blocks) {
    return blocks > 0 ? (size_t)ctas * (2 + decode_warps(blocks)) * 8 * blocks : (size_t)ctas * 2 * kQRows;
}
template <int kN>
static cudaError_t prepare_decode() {
    return cudaFuncSetAttribute(page_decode_kernel<kN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(decode_smem(kN) + prefix_bytes(kPageMaxSeqs)));
}
template <int kN>
static cudaError_t launch_decode(const PageAttnArgs& a, int ctas, cudaStream_t stream) {
    return launch_kernel(page_decode_kernel<kN>, dim3(ctas), dim3(decode_warps(kN) * 32), decode_smem(kN) + prefix_bytes(a.n), stream, a);
}

// One CTA an SM (the merge keeps the numbers of up to 256 of them).
static int page_ctas() { return num_sms() < 256 ? num_sms() : 256; }

size_t page_attn_scratch_bytes(int n, int L_q, int Hq, int Hkv) {
    (void)n;
    const int ctas = page_ctas();
    const size_t rows = partial_rows(ctas, few_blocks(L_q * (Hq / Hkv)));
    return round256((size_t)ctas * sizeof(ChainEntry)) + round256(rows * sizeof(float2)) + rows * kD * sizeof(float);
}

int launch_page_attn(const Pool& pool, int n, const int32_t* seqs, const int32_t* lens, int L_q, int Hq, float scale, const void* q,
                     const int32_t* table, void* out, float* lse, DeviceStatus* status, void* scratch, cudaStream_t stream) {
    const int ctas = page_ctas();
    PageAttnArgs a;
    a.p = pool; a.n = n; a.L_q = L_q; a.Hq = Hq; a.G = Hq / pool.Hkv;
    a.rows = L_q * a.G; a.inv_G = 65536 / a.G + 1;
    const int blocks = few_blocks(a.rows);
    const bool few = blocks > 0;
    a.units = few ? 1 : (a.rows + 127) / 128;
    a.pad = few ? 0 : kQPad;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.seqs = seqs; a.lens = lens; a.table = table;
    a.q = reinterpret_cast<const __nv_bfloat16*>(q); a.out = reinterpret_cast<__nv_bfloat16*>(out); a.lse = lse;
    char* at = reinterpret_cast<char*>(scratch);
    a.chains = reinterpret_cast<ChainEntry*>(at); at += round256((size_t)ctas * sizeof(ChainEntry));
    a.part_ml = reinterpret_cast<float2*>(at); at += round256(partial_rows(ctas, blocks) * sizeof(float2));
    a.part_o = reinterpret_cast<float*>(at);
    a.status = status;
    static std::atomic<bool> attr_done[64];
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_done[dev].load(std::memory_order_acquire)) {
        cudaError_t e = prepare_decode<1>();
        if (e == cudaSuccess) e = prepare_decode<2>();
        if (e == cudaSuccess) e = prepare_decode<3>();
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(page_question_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kQuestionSmem + prefix_bytes(kPageMaxSeqs)));
        // the question kernel's warpgroups trade registers: their shares add up to what 96 a thread give the block at launch
        cudaFuncAttributes fa = {};
        if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, page_question_kernel);
        if (e == cudaSuccess && fa.numRegs < 96) e = cudaErrorLaunchOutOfResources;
        if (e != cudaSuccess) { set_cuda_error(e); return DAF_ERR_CUDA; }
        if (dev >= 0 && dev < 64) attr_done[dev].store(true, std::memory_order_release);
    }
    cudaError_t e;
    if (few) {
        e = blocks == 1 ? launch_decode<1>(a, ctas, stream) : blocks == 2 ? launch_decode<2>(a, ctas, stream)
          : launch_decode<3>(a, ctas, stream);
    } else {
        const long long rows = (long long)pool.n_pages * pool.Hkv * pool.T;
        CUtensorMap mk, mv;
        if (int rc = make_pool_map(&mk, pool.k8, rows, pool.T < kQSub ? pool.T : kQSub)) return rc;
        if (int rc = make_pool_map(&mv, pool.v8, rows, pool.T < kQSub ? pool.T : kQSub)) return rc;
        e = launch_kernel(page_question_kernel, dim3(ctas), dim3(kQThreads), kQuestionSmem + prefix_bytes(n), stream, mk, mv, a);
    }
    count_launch();
    if (e != cudaSuccess) { set_cuda_error(e); return DAF_ERR_CUDA; }
    // Few long segments leave many partials of a row: with four warps a row instead of one, 28 rows of 4 heads over 8k keys (37 partials)
    // take 18.1 us instead of 30.5 with the attention itself, 132 rows of 8 heads over 16k (18) 37.1 instead of 40.5.  Where there are
    // more rows than warps one is better: 448 rows of 4 heads over 6k, 29.7 us against 31.0.  (The rule lies between these three.)
    const long long heads = (long long)n * pool.Hkv, segments = heads * ((a.rows + kQRows - 1) / kQRows);
    const bool four = ctas > 10 * segments && heads * a.rows <= 10 * ctas;
    e = few ? launch_kernel(page_merge_kernel<8, false>, dim3(ctas, a.rows), dim3(256), 0, stream, a, 8 * blocks, ctas)
      : four ? launch_kernel(page_merge_kernel<4, true>, dim3(3 * ctas), dim3(256), 0, stream, a, (int)kQRows, ctas)
             : launch_kernel(page_merge_kernel<1, true>, dim3(3 * ctas), dim3(256), 0, stream, a, (int)kQRows, ctas);
    count_launch();
    if (e != cudaSuccess) { set_cuda_error(e); return DAF_ERR_CUDA; }
    return check_launch();
}

}  // namespace daf
