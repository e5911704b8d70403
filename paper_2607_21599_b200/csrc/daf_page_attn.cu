// Attention over the paged 8-bit cache: for every sequence its newest L_q query tokens, each over the keys up to its own position.
//
// Work is cut on the device, from the sequences' lengths as they are when the kernel runs: a (sequence, KV head, block of query
// rows) is a segment of ceil(len / step) steps of keys, all segments lie behind one another on one axis, and every CTA takes an
// equal stretch of it.  A segment that lies in several CTAs leaves partial rows (at most two sets per CTA, whatever the shapes),
// which a second kernel merges.
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>
#include <vector>

#include "daf_common.cuh"

namespace daf {

constexpr int kD = 128;

struct PageAttnArgs {
    Pool p;
    int n, L_q, Hq, G;
    int rows;              // query rows of a KV head: L_q * G, row r is token r / G, head r % G of the group
    int row_blocks;        // blocks of them
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
// Rows of a KV head go through the warp-wide matrix instruction in blocks of 16.  (With one token and seven heads a group there
// are two flops per byte and row: the cache's way from HBM is what counts, not the tensor cores' rate, and a warp that needs
// nobody else keeps its loads in flight all the time.)  A warp walks its stretch of the work axis in steps of 32 keys: it asks for
// the tiles of K and V kDepth steps ahead (TMA into a ring of its own, rows of 128 bytes with the 128-byte swizzle), multiplies
// Q K^T, keeps the running maximum and sum, and multiplies P V.
//   8-bit values are exact in fp16, and so are the query rows once each is scaled by a power of two to a largest magnitude of
//   2^14 .. 2^15 (elements 2^-31 of that and below are rounded), so the logits are products of the given numbers with fp32 sums.
//   P goes into the product as fp16 of p * vs * 2^13 / (row maximum of p * 2^floor(log2 vs)): 11 bits down to 2^-27 of the
//   largest and some bits down to 2^-37 (as bf16 it would have 8), while sums of p stay in fp32.
constexpr int kStep = 32;
constexpr int kDecodeWarps = 8, kDepth = 3;
constexpr int kBlockRows = 16;
constexpr int kTile = kStep * kD;                    // 4 KB: K or V of one step
constexpr float kPExp = 13.f;

struct DecodeStage { float ks[2], vs[2]; };          // scales of the step's first and second 16 keys; negative: no such page
struct DecodeWarp {
    uint64_t full[kDepth];
    DecodeStage sc[kDepth];
};
constexpr int kPieceFloats = kBlockRows * kD + 2 * kBlockRows;       // an unfinished segment's rows, maxima and sums
constexpr size_t kRingBytes = (size_t)kDecodeWarps * kDepth * 2 * kTile;
constexpr size_t kDecodeSmem = 1024 + kRingBytes + sizeof(DecodeWarp) * kDecodeWarps;
static_assert(kDecodeWarps * kPieceFloats * sizeof(float) <= kRingBytes, "the pieces take the ring's place at the end");

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
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {            // 0xFF where a byte is NaN (0x7f, 0xff)
    return (((w & 0x7F7F7F7Fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xFFu;
}

// A place on the work axis: segment (b, h, block) and the step in it.
struct Place { int b, h, block, step, n_steps, seq, len; };

// Running sums of the sequences' steps (per head and block) in shared memory: pre[b] = steps of sequences 0 .. b - 1.
__device__ __forceinline__ int seq_len(const PageAttnArgs& a, int b) {
    int len = __ldg(a.lens + b);
    const int seq = a.seqs != nullptr ? __ldg(a.seqs + b) : b;
    if ((unsigned)seq >= (unsigned)a.p.n_seqs || len < 0) len = 0;
    return (int)min((long long)len, (long long)a.p.max_pages * a.p.T);
}
__device__ __forceinline__ int steps_of(int len, int step) { return max(1, (len + step - 1) / step); }   // (an empty one writes its zeros)

template <int kThreads>
__device__ __forceinline__ void sum_steps(const PageAttnArgs& a, int step, long long* pre, long long* warp_sums) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    long long run = 0;
    for (int b0 = 0; b0 < a.n; b0 += kThreads) {
        const int b = b0 + tid;
        long long x = b < a.n ? steps_of(seq_len(a, b), step) : 0;
        if (blockIdx.x == 0 && b < a.n) {
            const int len = __ldg(a.lens + b), seq = a.seqs != nullptr ? __ldg(a.seqs + b) : b;
            if ((unsigned)seq >= (unsigned)a.p.n_seqs || len != seq_len(a, b)) report_status(a.status, DAF_ERR_BOUNDS, 252, b);
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_sums[warp] = x;
        __syncthreads();
        long long before = run, all = 0;
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

__device__ __forceinline__ Place place_at(const PageAttnArgs& a, int step, const long long* pre, long long at) {
    const long long per = (long long)a.p.Hkv * a.row_blocks;
    int lo = 0, hi = a.n - 1;                    // last b with pre[b] * per <= at
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (pre[mid] * per <= at) lo = mid; else hi = mid - 1;
    }
    Place x;
    x.b = lo;
    x.len = seq_len(a, lo);
    x.n_steps = (int)(pre[lo + 1] - pre[lo]);
    const long long rest = at - pre[lo] * per;
    const int sub = (int)(rest / x.n_steps);
    x.step = (int)(rest - (long long)sub * x.n_steps);
    x.h = sub / a.row_blocks;
    x.block = sub - x.h * a.row_blocks;
    x.seq = a.seqs != nullptr ? __ldg(a.seqs + lo) : lo;
    return x;
}
__device__ __forceinline__ void next_segment(const PageAttnArgs& a, const long long* pre, Place& x) {
    x.step = 0;
    if (++x.block < a.row_blocks) return;
    x.block = 0;
    if (++x.h < a.p.Hkv) return;
    x.h = 0;
    ++x.b;
    if (x.b >= a.n) return;
    x.len = seq_len(a, x.b);
    x.n_steps = (int)(pre[x.b + 1] - pre[x.b]);
    x.seq = a.seqs != nullptr ? __ldg(a.seqs + x.b) : x.b;
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

__global__ void __launch_bounds__(kDecodeWarps * 32, 1)
page_decode_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const PageAttnArgs a) {
    extern __shared__ unsigned char decode_smem_raw[];
    unsigned char* const smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(decode_smem_raw) + 1023) & ~(uintptr_t)1023);
    DecodeWarp* const warps = reinterpret_cast<DecodeWarp*>(smem + kRingBytes);
    long long* const pre = reinterpret_cast<long long*>(warps + kDecodeWarps);
    __shared__ long long warp_sums[kDecodeWarps];
    __shared__ int abort_flag;
    __shared__ int piece_kind[2 * kDecodeWarps];         // see below
    __shared__ int4 piece_seg[2 * kDecodeWarps];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    DecodeWarp& me = warps[warp];
    unsigned char* const ring = smem + (size_t)warp * (kDepth * 2 * kTile);
    if (lane == 0) {
        for (int s = 0; s < kDepth; ++s) mbar_init(&me.full[s], 5);      // one arrival with the byte count, four with the scales
        mbar_fence_init();
    }
    if (threadIdx.x == 0) {
        abort_flag = 0;
        tma_prefetch_desc(&tmap_k);
        tma_prefetch_desc(&tmap_v);
    }
    if (threadIdx.x < 2 * kDecodeWarps) piece_kind[threadIdx.x] = 0;
    pdl_wait();
    pdl_launch_dependents();
    sum_steps<kDecodeWarps * 32>(a, kStep, pre, warp_sums);
    const long long total = pre[a.n] * a.p.Hkv * a.row_blocks;
    // CTAs that take part: no more than give each of its warps a step
    const long long ctas = min((long long)gridDim.x, (total + kDecodeWarps - 1) / kDecodeWarps);
    const long long cta_lo = min((long long)blockIdx.x, ctas) * total / ctas, cta_hi = min((long long)blockIdx.x + 1, ctas) * total / ctas;
    const long long span = cta_hi - cta_lo;
    const long long lo = cta_lo + warp * span / kDecodeWarps, hi = cta_lo + (warp + 1) * span / kDecodeWarps;

    const int T = a.p.T, Hkv = a.p.Hkv;
    const int box = min(T, kStep);               // keys of one copy
    volatile int* const abort = &abort_flag;
    // ---- the loads run ahead of the products with a place of their own
    Place ahead = {};
    long long ahead_at = lo;
    int ids = -1, ids_first = -1;                // page numbers of 32 pages of the place's sequence, one a lane
    auto issue = [&](int slot) {
        const int key0 = ahead.step * kStep;
        const int page0 = key0 / T;
        if (ids_first < 0 || page0 < ids_first || page0 + 1 >= ids_first + 32) {
            ids_first = page0;
            const int j = page0 + lane;
            ids = j < a.p.max_pages && (long long)j * T < ahead.len ? __ldg(a.table + (size_t)ahead.seq * a.p.max_pages + j) : -1;
            if ((unsigned)ids >= (unsigned)a.p.n_pages) {
                if ((long long)j * T < ahead.len && ahead.h == 0 && ahead.block == 0) report_status(a.status, DAF_ERR_BOUNDS, 250, ids);
                ids = -1;
            }
        }
        const int id0 = __shfl_sync(0xFFFFFFFFu, ids, page0 - ids_first);
        const int id1 = T >= kStep ? id0 : __shfl_sync(0xFFFFFFFFu, ids, page0 - ids_first + 1);
        unsigned char* const k_dst = ring + slot * 2 * kTile;
        unsigned char* const v_dst = k_dst + kTile;
        if (lane < 4) {
            // lanes 0, 1: K's scale of the first and second half; 2, 3: V's
            const int id = lane & 1 ? id1 : id0;
            float* const dst = lane < 2 ? &me.sc[slot].ks[lane] : &me.sc[slot].vs[lane - 2];
            if (id >= 0) {
                const float* const src = (lane < 2 ? a.p.k_scale : a.p.v_scale) + (size_t)id * Hkv + ahead.h;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&me.full[slot])) : "memory");
            } else {
                *dst = -1.f;
                mbar_arrive(&me.full[slot]);
            }
        }
        if (lane == 0) {
            const int copies = (id0 >= 0 ? 1 : 0) + (T < kStep && id1 >= 0 ? 1 : 0);
            mbar_arrive_expect_tx(&me.full[slot], (uint32_t)(copies * 2 * box * kD));
            if (id0 >= 0) {
                const int row = (id0 * Hkv + ahead.h) * T + key0 % T;
                tma_load_2d(k_dst, &tmap_k, &me.full[slot], 0, row);
                tma_load_2d(v_dst, &tmap_v, &me.full[slot], 0, row);
            }
            if (T < kStep && id1 >= 0) {
                const int row = (id1 * Hkv + ahead.h) * T;
                tma_load_2d(k_dst + box * kD, &tmap_k, &me.full[slot], 0, row);
                tma_load_2d(v_dst + box * kD, &tmap_v, &me.full[slot], 0, row);
            }
        }
        __syncwarp();
        ++ahead_at;
        if (++ahead.step == ahead.n_steps) {
            next_segment(a, pre, ahead);
            ids_first = -1;
        }
    };
    Place at = {};
    if (lo < hi) {
        at = place_at(a, kStep, pre, lo);
        ahead = at;
        for (int s = 0; s < kDepth && ahead_at < hi; ++s) issue(s);
    }
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    bool tail = false;
    float o[16][4], m[2], l[2];
    for (long long x = lo; x < hi && ok;) {
        // ---- a segment, or the stretch of it that is this warp's
        const int first_step = at.step;
        const int r0 = at.block * kBlockRows, n_rows = min(kBlockRows, a.rows - r0);
        const int rg[2] = {r0 + g, r0 + g + 8};
        int limit[2];                      // last key each of this thread's two rows sees
        uint32_t qf[8][4];
        float cs[2];
        {
            uint32_t w[2][16];             // four consecutive channels of each k-step
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool there = rg[i] < a.rows;
                const int tok = rg[i] / a.G, head = at.h * a.G + rg[i] % a.G;
                limit[i] = there ? at.len - a.L_q + tok : -1;
                const uint2* const src = reinterpret_cast<const uint2*>(a.q + (((size_t)at.b * a.L_q + tok) * a.Hq + head) * kD) + t;
                uint32_t big = 0;
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint2 v = there ? __ldg(src + kk * 4) : make_uint2(0u, 0u);
                    w[i][2 * kk] = v.x; w[i][2 * kk + 1] = v.y;
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const uint32_t bits = ((u & 2 ? v.y : v.x) >> (16 * (u & 1))) & 0x7FFFu;
                        big = max(big, bits < 0x7F80u ? bits : 0u);
                    }
                }
                big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
                big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
                const int e = max((int)(big >> 7) - 127, -100);
                const float up = __int_as_float((14 - e + 127) << 23);
                cs[i] = __int_as_float((e - 14 + 127) << 23) * a.scale_log2;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    w[i][j] = pack_f16(__uint_as_float(w[i][j] << 16) * up, __uint_as_float(w[i][j] & 0xFFFF0000u) * up);
            }
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                qf[kk][0] = w[0][2 * kk]; qf[kk][1] = w[1][2 * kk]; qf[kk][2] = w[0][2 * kk + 1]; qf[kk][3] = w[1][2 * kk + 1];
            }
        }
        const int first_limit = at.len - a.L_q + r0 / a.G;       // of the block's rows
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
        for (; at.step < at.n_steps && x < hi; ++at.step, ++x) {
            ok = mbar_wait(&me.full[slot], phase, abort, a.status, 251);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            const uint32_t k_at = smem_u32(ring + slot * 2 * kTile), v_at = k_at + kTile;
            const DecodeStage sc = me.sc[slot];
            const int key0 = at.step * kStep;
            // logits: 32 keys in four tiles of eight
            float s[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int u = 0; u < 4; ++u) s[j][u] = 0.f;
                const uint32_t row = k_at + (uint32_t)((8 * j + (lane & 7)) * kD);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t w[4];
                    ldsm4(w, row + (uint32_t)((((lane >> 3) + 4 * half) ^ (lane & 7)) << 4));
#pragma unroll
                    for (int u = 0; u < 4; ++u) mma16816(s[j], qf[4 * half + u], widen2(w[u]), widen2(w[u] >> 16));
                }
            }
            // a step with keys that some row does not see, or without a page
            const bool odd = key0 + kStep - 1 > first_limit || sc.ks[0] < 0.f || sc.ks[1] < 0.f;
            float top[2] = {-INFINITY, -INFINITY};
            int ve[2];
            float vm[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {      // vs = vm * 2^ve, 1 <= vm < 2
                const int bits = __float_as_int(sc.vs[j]);
                ve[j] = sc.vs[j] > 0.f ? (bits >> 23) - 127 : 0;
                vm[j] = sc.vs[j] > 0.f ? __int_as_float((bits & 0x7FFFFF) | 0x3F800000) : 1.f;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float ks = sc.ks[j >> 1], shift = (float)ve[j >> 1];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    s[j][u] = s[j][u] * (cs[u >> 1] * ks) + shift;
                    if (odd && (key0 + 8 * j + 2 * t + (u & 1) > limit[u >> 1] || ks < 0.f)) s[j][u] = -INFINITY;
                    top[u >> 1] = fmaxf(top[u >> 1], s[j][u]);
                }
            }
            float used[2], alpha[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 2));
                const float now = fmaxf(m[i], top[i]);
                alpha[i] = m[i] == now ? 1.f : fast_exp2(m[i] - now);      // (2^-inf = 0 at the first key)
                used[i] = now == -INFINITY ? 0.f : now - kPExp;
                m[i] = now;
            }
            if (__any_sync(0xFFFFFFFFu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    o[i][0] *= alpha[0]; o[i][1] *= alpha[0];
                    o[i][2] *= alpha[1]; o[i][3] *= alpha[1];
                }
                l[0] *= alpha[0]; l[1] *= alpha[1];
            }
            uint32_t pf[2][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float back = __int_as_float((127 - max(ve[j >> 1], -126)) << 23);     // 2^-ve: the sums are of p itself
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float e = fast_exp2(s[j][u] - used[u >> 1]);
                    l[u >> 1] += e * back;
                    s[j][u] = e * vm[j >> 1];
                }
                pf[j >> 1][2 * (j & 1)] = pack_f16(s[j][0], s[j][1]);
                pf[j >> 1][2 * (j & 1) + 1] = pack_f16(s[j][2], s[j][3]);
            }
            // O += P V: channels 16 c + 2 n and 16 c + 2 n + 1 are columns n of two products
            bool poison = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int c = 0; c < 8; c += 2) {
                    const int row = 16 * i + 8 * ((lane >> 3) & 1) + (lane & 7);
                    uint32_t w[4];
                    ldsm4_t(w, v_at + (uint32_t)(row * kD + (((c + (lane >> 4)) ^ (lane & 7)) << 4)));
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
                        mma16816(o[2 * (c + cc)], pf[i], widen2(w0), widen2(w1));
                        mma16816(o[2 * (c + cc) + 1], pf[i], widen2(w0 >> 16), widen2(w1 >> 16));
                    }
                }
            }
            if (odd && __any_sync(0xFFFFFFFFu, poison)) {
                for (int j = 0; j < kStep; ++j) {
                    const int key = key0 + j;
                    if (key <= first_limit || key >= at.len) continue;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const uint32_t w = nan_bytes(*reinterpret_cast<const uint32_t*>(ring + slot * 2 * kTile + kTile + j * kD + ((c ^ (j & 7)) << 4) + 4 * t));
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if ((w >> (8 * u)) & 1u) {
                                if (key <= limit[0]) o[2 * c + (u & 1)][u >> 1] = __int_as_float(0x7FC00000);
                                if (key <= limit[1]) o[2 * c + (u & 1)][2 + (u >> 1)] = __int_as_float(0x7FC00000);
                            }
                    }
                }
            }
            __syncwarp();          // every lane is done with the slot
            if (ahead_at < hi) issue(slot);
            if (++slot == kDepth) { slot = 0; phase ^= 1u; }
        }
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 1);
            l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 2);
        }
        const bool begins = first_step == 0, ends = at.step == at.n_steps;
        if (begins && ends) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (rg[i] >= a.rows) continue;
                const int tok = rg[i] / a.G, head = at.h * a.G + rg[i] % a.G;
                const float inv = row_inverse(l[i]);
                uint2* const dst = reinterpret_cast<uint2*>(a.out + (((size_t)at.b * a.L_q + tok) * a.Hq + head) * kD) + t;
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    dst[c * 4] = make_uint2(pack_bf16(o[2 * c][2 * i] * inv, o[2 * c + 1][2 * i] * inv),
                                            pack_bf16(o[2 * c][2 * i + 1] * inv, o[2 * c + 1][2 * i + 1] * inv));
                if (a.lse != nullptr && t == 0)
                    a.lse[((size_t)at.b * a.Hq + head) * a.L_q + tok] = row_lse(m[i], l[i]);
            }
        } else if (ends) {
            // the end of a segment that begins in front of this warp's stretch: parked in global memory, since the ring is in use
            float* const dst = a.part_o + ((size_t)gridDim.x * 2 + (size_t)blockIdx.x * kDecodeWarps + warp) * (kBlockRows * kD);
            float2* const ml = a.part_ml + ((size_t)gridDim.x * 2 + (size_t)blockIdx.x * kDecodeWarps + warp) * kBlockRows;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (g + 8 * i >= n_rows) continue;
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    *reinterpret_cast<float4*>(dst + (g + 8 * i) * kD + c * 16 + 4 * t) =
                        make_float4(o[2 * c][2 * i], o[2 * c + 1][2 * i], o[2 * c][2 * i + 1], o[2 * c + 1][2 * i + 1]);
                if (t == 0) ml[g + 8 * i] = make_float2(m[i], l[i]);
            }
            if (lane == 0) {
                piece_kind[2 * warp] = 1 | 4;
                piece_seg[2 * warp] = make_int4(at.b, at.h, at.block, at.n_steps);
            }
        } else {
            tail = true;           // stays in registers until the ring is free
            if (lane == 0) {
                piece_kind[2 * warp + 1] = 1 | (begins ? 2 : 0);
                piece_seg[2 * warp + 1] = make_int4(at.b, at.h, at.block, at.n_steps);
            }
            break;
        }
        if (x < hi) next_segment(a, pre, at);
    }
    if (!ok) {      // loads in flight get a bounded chance to land before the CTA retires
        for (int s = 0; s < kDepth; ++s)
            for (int i = 0; i < 4096 && !mbar_try_wait(&me.full[s], 0) && !mbar_try_wait(&me.full[s], 1); ++i) {}
    }
    __syncthreads();
    if (abort_flag != 0) {
        if (threadIdx.x == 0) a.chains[blockIdx.x] = ChainEntry{-1, 0, 0, 0};
        return;
    }
    // ---- the warps' unfinished pieces: neighbours of one segment are merged; what is still unfinished is the CTA's
    float* const pieces = reinterpret_cast<float*>(smem);
    if (tail) {
        float* const dst = pieces + warp * kPieceFloats;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                *reinterpret_cast<float4*>(dst + (g + 8 * i) * kD + c * 16 + 4 * t) =
                    make_float4(o[2 * c][2 * i], o[2 * c + 1][2 * i], o[2 * c][2 * i + 1], o[2 * c + 1][2 * i + 1]);
            if (t == 0) reinterpret_cast<float2*>(dst + kBlockRows * kD)[g + 8 * i] = make_float2(m[i], l[i]);
        }
    }
    __syncthreads();
    int chain_kind = 0;            // 1: the CTA begins a segment that it does not end
    int4 chain_seg = make_int4(0, 0, 0, 0);
    for (int i0 = 0; i0 < 2 * kDecodeWarps;) {
        if (piece_kind[i0] == 0) { ++i0; continue; }
        // pieces i0 .. i1 - 1 are of one segment: the first begins it or lies first in the CTA, the last ends it or lies last
        int i1 = i0, last = i0;
        for (;;) {
            last = i1++;
            if (piece_kind[last] & 4) break;
            while (i1 < 2 * kDecodeWarps && piece_kind[i1] == 0) ++i1;
            if (i1 == 2 * kDecodeWarps) break;
        }
        const bool begins = (piece_kind[i0] & 2) != 0, ends = (piece_kind[last] & 4) != 0;
        const int4 seg = piece_seg[i0];
        const int r0 = seg.z * kBlockRows, n_rows = min(kBlockRows, a.rows - r0);
        for (int r = warp; r < n_rows; r += kDecodeWarps) {
            float mx = -INFINITY;
            auto ml_of = [&](int i) {
                return (i & 1) ? reinterpret_cast<const float2*>(pieces + (i >> 1) * kPieceFloats + kBlockRows * kD)[r]
                               : __ldcg(a.part_ml + ((size_t)gridDim.x * 2 + (size_t)blockIdx.x * kDecodeWarps + (i >> 1)) * kBlockRows + r);
            };
            for (int i = i0; i < i1; ++i)
                if (piece_kind[i] != 0) mx = fmaxf(mx, ml_of(i).x);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum = 0.f;
            for (int i = i0; i < i1; ++i) {
                if (piece_kind[i] == 0) continue;
                const float2 ml = ml_of(i);
                const float w = partial_weight(ml, mx);
                const float4 v = (i & 1) ? reinterpret_cast<const float4*>(pieces + (i >> 1) * kPieceFloats + r * kD)[lane]
                                         : __ldcg(reinterpret_cast<const float4*>(a.part_o + (((size_t)gridDim.x * 2 + (size_t)blockIdx.x * kDecodeWarps + (i >> 1)) * kBlockRows + r) * kD) + lane);
                sum += w * ml.y;
                acc.x += w * v.x; acc.y += w * v.y; acc.z += w * v.z; acc.w += w * v.w;
            }
            if (begins && ends) {
                const int row = r0 + r, tok = row / a.G, head = seg.y * a.G + row % a.G;
                const float inv = row_inverse(sum);
                reinterpret_cast<uint2*>(a.out + (((size_t)seg.x * a.L_q + tok) * a.Hq + head) * kD)[lane] =
                    make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                if (a.lse != nullptr && lane == 0)
                    a.lse[((size_t)seg.x * a.Hq + head) * a.L_q + tok] = row_lse(mx, sum);
            } else {
                const size_t set = (size_t)blockIdx.x * 2 + (begins ? 1 : 0);
                reinterpret_cast<float4*>(a.part_o + (set * kBlockRows + r) * kD)[lane] = acc;
                if (lane == 0) a.part_ml[set * kBlockRows + r] = make_float2(mx, sum);
            }
        }
        if (begins && !ends) { chain_kind = 1; chain_seg = seg; }
        i0 = i1;
    }
    if (threadIdx.x == 0) {
        ChainEntry e = {-1, 0, 0, 0};
        if (chain_kind != 0) {
            const long long seg_end = (pre[chain_seg.x] * Hkv + 0) * a.row_blocks + ((long long)chain_seg.y * a.row_blocks + chain_seg.z + 1) * chain_seg.w;
            // the CTA whose stretch holds step seg_end - 1
            long long c = min(((seg_end - 1) * ctas) / total, ctas - 1);
            while (c + 1 < ctas && (c + 1) * total / ctas <= seg_end - 1) ++c;
            while (c > 0 && c * total / ctas > seg_end - 1) --c;
            e = ChainEntry{(int)c, chain_seg.x, chain_seg.y, chain_seg.z};
        }
        a.chains[blockIdx.x] = e;
    }
}

// Merge of the segments that lie in several CTAs: one CTA of four warps per (CTA that begins such a segment, row).
__global__ void __launch_bounds__(128) page_merge_kernel(const PageAttnArgs a, int block_rows) {
    __shared__ float4 acc_s[4][32];
    __shared__ float sum_s[4], mx_s[4];
    pdl_wait();
    pdl_launch_dependents();
    const ChainEntry e = a.chains[blockIdx.x];
    const int first = blockIdx.x, last = e.last_cta, r = blockIdx.y;
    if (last < 0) return;
    const int row = e.block * block_rows + r;
    if (row >= a.rows) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // partial i of the row: the first CTA's second set, then the following CTAs' first sets
    auto set_of = [&](int i) { return i == 0 ? (size_t)first * 2 + 1 : (size_t)(first + i) * 2; };
    const int n = last - first + 1;
    float mx = -INFINITY;
    for (int i = threadIdx.x; i < n; i += 128) mx = fmaxf(mx, __ldcg(&a.part_ml[set_of(i) * block_rows + r].x));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
    if (lane == 0) mx_s[warp] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(mx_s[0], mx_s[1]), fmaxf(mx_s[2], mx_s[3]));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int i = warp; i < n; i += 4) {
        const float2 ml = __ldcg(&a.part_ml[set_of(i) * block_rows + r]);
        const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part_o + (set_of(i) * block_rows + r) * kD) + lane);
        const float w = partial_weight(ml, mx);
        sum += w * ml.y;
        acc.x += w * v.x; acc.y += w * v.y; acc.z += w * v.z; acc.w += w * v.w;
    }
    acc_s[warp][lane] = acc;
    if (lane == 0) sum_s[warp] = sum;
    __syncthreads();
    if (warp != 0) return;
    sum = (sum_s[0] + sum_s[1]) + (sum_s[2] + sum_s[3]);
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        const float4 v = acc_s[w][lane];
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
    }
    const int tok = row / a.G, head = e.h * a.G + row % a.G;
    const float inv = row_inverse(sum);
    reinterpret_cast<uint2*>(a.out + (((size_t)e.b * a.L_q + tok) * a.Hq + head) * kD)[lane] =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    if (a.lse != nullptr && lane == 0)
        a.lse[((size_t)e.b * a.Hq + head) * a.L_q + tok] = row_lse(mx, sum);
}

// ------------------------------------------------------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// K or V of one layer of the pool as rows of 128 bytes, in boxes of `box_rows` rows with the 128-byte swizzle.  Each host thread
// keeps the maps it encoded last, keyed by everything that goes into them.
static int make_pool_map(CUtensorMap* m, const void* base, long long rows, int box_rows) {
    struct Slot { const void* base; long long rows; int box; CUtensorMap map; };
    static thread_local std::vector<Slot> cache;
    if (cache.empty()) cache.resize(256, Slot{nullptr, 0, 0, {}});
    Slot& slot = cache[((reinterpret_cast<uintptr_t>(base) >> 8) * 1000003u + (size_t)rows * 31u + (size_t)box_rows) % 256];
    if (slot.base == base && slot.rows == rows && slot.box == box_rows) { *m = slot.map; return DAF_OK; }
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
    slot = Slot{base, rows, box_rows, *m};
    return DAF_OK;
}

static size_t round256(size_t x) { return (x + 255) / 256 * 256; }
// Partial rows: two sets a CTA, and one a warp for the pieces parked on the way.
static size_t decode_sets(int ctas) { return (size_t)ctas * (2 + kDecodeWarps); }
static size_t decode_smem(int n) { return kDecodeSmem + ((size_t)n + 1) * sizeof(long long); }

size_t page_attn_scratch_bytes(int n, int L_q, int Hq, int Hkv) {
    (void)n; (void)L_q; (void)Hq; (void)Hkv;
    const int ctas = num_sms();
    return round256((size_t)ctas * sizeof(ChainEntry)) + round256(decode_sets(ctas) * kBlockRows * sizeof(float2)) +
           decode_sets(ctas) * kBlockRows * kD * sizeof(float);
}

int launch_page_attn(const Pool& pool, int n, const int32_t* seqs, const int32_t* lens, int L_q, int Hq, float scale, const void* q,
                     const int32_t* table, void* out, float* lse, DeviceStatus* status, void* scratch, cudaStream_t stream) {
    const int ctas = num_sms();
    PageAttnArgs a;
    a.p = pool; a.n = n; a.L_q = L_q; a.Hq = Hq; a.G = Hq / pool.Hkv;
    a.rows = L_q * a.G;
    a.row_blocks = (a.rows + kBlockRows - 1) / kBlockRows;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.seqs = seqs; a.lens = lens; a.table = table;
    a.q = reinterpret_cast<const __nv_bfloat16*>(q); a.out = reinterpret_cast<__nv_bfloat16*>(out); a.lse = lse;
    char* at = reinterpret_cast<char*>(scratch);
    a.chains = reinterpret_cast<ChainEntry*>(at); at += round256((size_t)ctas * sizeof(ChainEntry));
    a.part_ml = reinterpret_cast<float2*>(at); at += round256(decode_sets(ctas) * kBlockRows * sizeof(float2));
    a.part_o = reinterpret_cast<float*>(at);
    a.status = status;
    const long long rows = (long long)pool.n_pages * pool.Hkv * pool.T;
    CUtensorMap mk, mv;
    const int box = pool.T < kStep ? pool.T : kStep;
    if (int rc = make_pool_map(&mk, pool.k8, rows, box)) return rc;
    if (int rc = make_pool_map(&mv, pool.v8, rows, box)) return rc;
    static std::atomic<bool> attr_done[64];
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_done[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(page_decode_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)decode_smem(kPageMaxSeqs));
        if (e != cudaSuccess) { set_cuda_error(e); return DAF_ERR_CUDA; }
        if (dev >= 0 && dev < 64) attr_done[dev].store(true, std::memory_order_release);
    }
    cudaError_t e = launch_kernel(page_decode_kernel, dim3(ctas), dim3(kDecodeWarps * 32), decode_smem(n), stream, mk, mv, a);
    count_launch();
    if (e != cudaSuccess) { set_cuda_error(e); return DAF_ERR_CUDA; }
    e = launch_kernel(page_merge_kernel, dim3(ctas, kBlockRows), dim3(128), 0, stream, a, (int)kBlockRows);
    count_launch();
    if (e != cudaSuccess) { set_cuda_error(e); return DAF_ERR_CUDA; }
    return check_launch();
}

}  // namespace daf
