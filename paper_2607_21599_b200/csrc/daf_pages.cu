// The paged 8-bit cache: argument checks of all daf_page_* calls, and the kernels that write rows into pages, read them back,
// and hand out, copy, take back and compact pages.  All of these move bytes: what bounds them is HBM where there are many and
// the length of the chain of dependent accesses (positions -> page -> scale -> bytes) where there are few.
#include <cuda_fp16.h>

#include "daf_common.cuh"

namespace daf {

constexpr int kMinScaleExp = -60;      // scales that the writer leaves are at least 2^-60

// ------------------------------------------------------------------------------------------------------------- 8-bit values
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ float4 unpack_e4m3x4(uint32_t w) {
    uint32_t lo, hi;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)(w & 0xFFFFu)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(w >> 16)));
    const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo)), b = __half22float2(*reinterpret_cast<__half2*>(&hi));
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }      // -126 <= e <= 127

// Largest magnitude (bf16 bits, which ascend with it) among the finite ones of eight bf16 values.
__device__ __forceinline__ uint32_t finite_max8(uint4 w) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t x = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w, b = (x >> (16 * (i & 1))) & 0x7FFFu;
        m = max(m, b < 0x7F80u ? b : 0u);
    }
    return m;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// Exponent of the least power of two s with magnitude <= 448 s (448 = 1.75 * 2^8), at least kMinScaleExp.
__device__ __forceinline__ int scale_exp(uint32_t bf16_bits) {
    const int e = (int)(bf16_bits >> 7) - 127 - 8 + ((bf16_bits & 0x7Fu) > 0x60u ? 1 : 0);
    return max(e, kMinScaleExp);
}

// ---------------------------------------------------------------------------------------------------------- rows into pages
struct WriteArgs {
    Pool p;
    int n, slots;               // `slots` CTAs share an entry's pages (for each head, K and V apart)
    const int32_t* seqs; const int32_t* lens; const int32_t* row_off; const int32_t* idx;
    const __nv_bfloat16* k; const __nv_bfloat16* v;
    const int32_t* table; const int32_t* refs;
    DeviceStatus* status;
};

// First of positions [a, b) of an ascending list whose value is at least `key`, found by all 128 threads of a CTA: 128 probes a
// round, so that 16k positions take two round trips to L2 instead of the fourteen of a bisection.
__device__ __forceinline__ int first_at_least(const int32_t* idx, int a, int b, int key) {
    while (a < b) {
        const int step = (b - a + 127) / 128, at = a + (int)threadIdx.x * step;
        const int below = __syncthreads_count(at < b && __ldg(idx + at) < key);
        if (step == 1) return a + below;
        if (below == 0) return a;
        b = min(b, a + below * step);
        a = a + (below - 1) * step + 1;
    }
    return a;
}

// One CTA of four warps takes one page, one head, K or V at a time.  Every new row of it is read once and held in registers
// (sixteen lanes a row, eight elements each) while the CTA finds their largest magnitude; the rows then leave scaled.  Kept bytes are
// touched only where the scale grows.  kGiven: positions come from a list, through a table in shared memory of which row a token
// gets; otherwise the rows are the newest tokens, whose addresses need nothing but the length, and are asked for ahead of the page.
//   Measured: a context of 16k tokens of 8 heads 21.7 us at 64 tokens a page (4.6 TB/s; a copy of as many bytes would take 15.4) and 26 at
// 16, where a CTA has 4 KB to fetch; a token of 64 sequences 3.4, a launch and the chain position -> page -> old scale -> bytes; every
// fifth of 14k tokens 10.7, that chain with two more trips for the list.
template <int kTokens, bool kGiven>
__global__ void __launch_bounds__(128) page_write_kernel(const WriteArgs a) {
    constexpr int T = kTokens, kPer = T / 8;      // tokens of a lane
    __shared__ int row_of[kGiven ? T : 1];        // new row of each token of the page, -1: none
    __shared__ uint32_t warp_max[4];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = threadIdx.x >> 4, piece = threadIdx.x & 15;
    const int b = blockIdx.x / a.slots, h = blockIdx.y, Hkv = a.p.Hkv;
    const bool reports = h == 0 && blockIdx.z == 0;       // (one of the CTAs that see the same fault)
    const int seq = a.seqs != nullptr ? __ldg(a.seqs + b) : b, len = __ldg(a.lens + b);
    const int r_lo = __ldg(a.row_off + b), r_hi = __ldg(a.row_off + b + 1);
    if (r_hi <= r_lo) return;
    if ((unsigned)seq >= (unsigned)a.p.n_seqs || len < 0 || (long long)len > (long long)a.p.max_pages * T || r_lo < 0 ||
        (!kGiven && r_hi - r_lo > len)) {
        if (reports && threadIdx.x == 0) report_status(a.status, DAF_ERR_BOUNDS, 200, b);
        return;
    }
    if (kGiven && reports && blockIdx.x % a.slots == 0 && threadIdx.x < 2) {      // the first and the last position: the others lie between
        const int at = __ldg(a.idx + (threadIdx.x == 0 ? r_lo : r_hi - 1));
        if (at < 0 || at >= len) report_status(a.status, DAF_ERR_BOUNDS, 203, at);
    }
    const int start = kGiven ? 0 : len - (r_hi - r_lo);       // first token that may be written
    const int kept_to = kGiven ? len : start;                 // tokens below this were there before
    const uint4* const src = reinterpret_cast<const uint4*>((blockIdx.z ? a.v : a.k) + (size_t)h * 128) + piece;
    uint8_t* const pool = blockIdx.z ? a.p.v8 : a.p.k8;
    float* const scales = blockIdx.z ? a.p.v_scale : a.p.k_scale;
    for (int j = start / T + (int)(blockIdx.x % a.slots); j * T < len; j += a.slots) {
        const int base = j * T;
        int ra = 0, rb = 1;
        if (kGiven) {
            ra = first_at_least(a.idx, r_lo, r_hi, base);
            rb = first_at_least(a.idx, ra, r_hi, base + T);
        }
        if (ra >= rb) continue;
        const int page = __ldg(a.table + (size_t)seq * a.p.max_pages + j);
        uint4 w[kPer];
        uint32_t news = 0;            // which of this lane's tokens get a new row
        auto take = [&](int i, int r) {
            news |= 1u << i;
            w[i] = __ldg(src + (size_t)r * Hkv * 16);
        };
        if (!kGiven) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int at = base + 8 * i + sub;
                w[i] = make_uint4(0u, 0u, 0u, 0u);
                if (at >= start && at < len) take(i, r_lo + at - start);
            }
        }
        const bool in_pool = (unsigned)page < (unsigned)a.p.n_pages;
        if (!in_pool || (a.refs != nullptr && __ldg(a.refs + page) != 1)) {
            if (reports && threadIdx.x == 0) report_status(a.status, DAF_ERR_BOUNDS, in_pool ? 202 : 201, page);
            continue;
        }
        float* const scale_at = scales + (size_t)page * Hkv + h;
        const float s_old = __ldcg(scale_at);
        if (kGiven) {
            for (int t = threadIdx.x; t < T; t += 128) row_of[t] = -1;
            __syncthreads();
            for (int r = ra + threadIdx.x; r < rb; r += 128) {
                const int at = __ldg(a.idx + r);
                if (at >= base && at < min(base + T, len)) atomicMax(&row_of[at - base], r);
                else if (reports) report_status(a.status, DAF_ERR_BOUNDS, 204, at);       // the list does not ascend
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = row_of[8 * i + sub];
                w[i] = make_uint4(0u, 0u, 0u, 0u);
                if (r >= 0) take(i, r);
            }
        }
        uint32_t m = 0;
        bool keeps = false;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            m = max(m, finite_max8(w[i]));
            keeps |= !((news >> i) & 1u) && base + 8 * i + sub < kept_to;
        }
        m = __reduce_max_sync(0xFFFFFFFFu, m);
        if (lane == 0) warp_max[warp] = m;
        keeps = __syncthreads_or(keeps);
        m = max(max(warp_max[0], warp_max[1]), max(warp_max[2], warp_max[3]));
        int e = scale_exp(m);
        if (keeps) {       // at least the old scale, rounded up to a power of two if it is none
            const int bits = __float_as_int(s_old);
            e = max(e, min((bits >> 23) - 127 + ((bits & 0x7FFFFF) != 0 ? 1 : 0), 120));
        }
        uint2* const dst = reinterpret_cast<uint2*>(pool + ((size_t)page * Hkv + h) * (T * 128)) + piece;
        const float inv = pow2f(-e), s_new = pow2f(e);
        const bool again = keeps && s_new != s_old;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int t = 8 * i + sub;
            if ((news >> i) & 1u) {
                dst[t * 16] = make_uint2(pack_e4m3x4(bf16_lo(w[i].x) * inv, bf16_hi(w[i].x) * inv, bf16_lo(w[i].y) * inv, bf16_hi(w[i].y) * inv),
                                         pack_e4m3x4(bf16_lo(w[i].z) * inv, bf16_hi(w[i].z) * inv, bf16_lo(w[i].w) * inv, bf16_hi(w[i].w) * inv));
            } else if (again && base + t < kept_to) {
                const float f = s_old * inv;
                const uint2 old = dst[t * 16];
                const float4 x = unpack_e4m3x4(old.x), y = unpack_e4m3x4(old.y);
                dst[t * 16] = make_uint2(pack_e4m3x4(x.x * f, x.y * f, x.z * f, x.w * f), pack_e4m3x4(y.x * f, y.y * f, y.z * f, y.w * f));
            }
        }
        if (threadIdx.x == 0) *scale_at = s_new;
        __syncthreads();       // row_of and warp_max are used again
    }
}

// ---------------------------------------------------------------------------------------------------------- pages into rows
struct ReadArgs {
    Pool p;
    int n, slots;
    const int32_t* seqs; const int32_t* first; const int32_t* row_off; const int32_t* table;
    __nv_bfloat16* k; __nv_bfloat16* v;
    DeviceStatus* status;
};

__device__ __forceinline__ uint4 widen8(uint32_t lo, uint32_t hi, float s) {
    const float4 x = unpack_e4m3x4(lo), y = unpack_e4m3x4(hi);
    auto two = [s](float a, float b) { return pack_bf16(mul_rn_keep_subnormals(a, s), mul_rn_keep_subnormals(b, s)); };
    return make_uint4(two(x.x, x.y), two(x.z, x.w), two(y.x, y.y), two(y.z, y.w));
}

// One CTA takes one page, one head, K or V at a time: T * 8 chunks of 16 bytes, all of a thread's requested ahead of the first
// use; a chunk becomes 32 bytes of its row.  32k tokens of 4 heads take 19.9 us (5.1 TB/s, 77 % of a copy's rate), 6k 6.1.
template <int kChunks>      // page_tokens * 8 / 128
__global__ void __launch_bounds__(128) page_read_kernel(const ReadArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int T = kChunks * 16;
    const int b = blockIdx.x / a.slots, h = blockIdx.y, Hkv = a.p.Hkv;
    const bool reports = h == 0 && blockIdx.z == 0 && threadIdx.x == 0;
    const int seq = a.seqs != nullptr ? __ldg(a.seqs + b) : b, first = a.first != nullptr ? __ldg(a.first + b) : 0;
    const int r_lo = __ldg(a.row_off + b), r_hi = __ldg(a.row_off + b + 1);
    if (r_hi <= r_lo) return;
    if ((unsigned)seq >= (unsigned)a.p.n_seqs || first < 0 || r_lo < 0 ||
        (long long)first + (r_hi - r_lo) > (long long)a.p.max_pages * T) {
        if (reports) report_status(a.status, DAF_ERR_BOUNDS, 210, b);
        return;
    }
    const int end = first + (r_hi - r_lo);
    const uint8_t* const pool = blockIdx.z ? a.p.v8 : a.p.k8;
    const float* const scales = blockIdx.z ? a.p.v_scale : a.p.k_scale;
    __nv_bfloat16* const out = blockIdx.z ? a.v : a.k;
    for (int j = first / T + (int)(blockIdx.x % a.slots); j * T < end; j += a.slots) {
        const int page = __ldg(a.table + (size_t)seq * a.p.max_pages + j);
        if ((unsigned)page >= (unsigned)a.p.n_pages) {
            if (reports) report_status(a.status, DAF_ERR_BOUNDS, 211, page);
            continue;
        }
        const float s = __ldg(scales + (size_t)page * Hkv + h);
        const uint4* const src = reinterpret_cast<const uint4*>(pool + ((size_t)page * Hkv + h) * (T * 128)) + threadIdx.x;
        uint4 w[kChunks];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int at = j * T + i * 16 + (int)(threadIdx.x >> 3);
            if (at >= first && at < end) w[i] = __ldcs(src + i * 128);
        }
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int at = j * T + i * 16 + (int)(threadIdx.x >> 3);
            if (at >= first && at < end) {
                uint4* const dst = reinterpret_cast<uint4*>(out + ((size_t)(r_lo + at - first) * Hkv + h) * 128) + 2 * (threadIdx.x & 7);
                dst[0] = widen8(w[i].x, w[i].y, s);
                dst[1] = widen8(w[i].z, w[i].w, s);
            }
        }
    }
}

// ----------------------------------------------------------------------------------------------------- which pages go where
// Both fork and compact run as two kernels: one CTA decides (who gets which page, which page is copied to which) from counts and
// prefix sums over items and over refs, then a grid does what was decided: table, refs and the bytes.  Copies of some 250 MB run at 5.4 to
// 5.8 TB/s (82 to 88 % of a copy's rate); of few pages the decision is what counts: some 5 us of dependent loads and
// scans in one CTA.  Its warps look at refs a word of 32 pages at a time, one ballot each, and share all pages evenly: eight answers over
// a context 12.5 us, compacting 700 pages 7.4; with 512 neighbouring pages a warp whatever their number 13.8 and 11.7.  Rows that grow by a
// token: 6.0 us for one or eight, 8.2 for 64, where none needs a page (7.1 and 9.5 where each does).
constexpr int kPlanThreads = 1024;
constexpr int kPlanRefs = 16;            // words of 32 pages that a warp looks at per round at most: 16k pages a round
constexpr int kPlanRound = kPlanThreads * kPlanRefs;
constexpr int kPlanRows = 1 << 16;       // up to as many rows of the table are marked in shared memory

struct PlanHead { int ok, n_new, n_copies, live; };
struct PlanArrays {       // in the workspace behind the status word
    PlanHead* head;
    int2* copies;         // [n_pages] (from, to)
    int32_t* fresh;       // [n_pages] pages handed out, ascending (compact: where a page goes, by its old number, or -1)
    int32_t* marks;       // [n_seqs]
    int2* items;          // [n + 1] running counts: new pages, copies
};

// Exclusive prefix sums of two counts packed in 64 bits over the 1024 threads of a CTA; *total gets the sums.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* total) {
    __shared__ unsigned long long sums[33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        unsigned long long s = sums[lane], t = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long y = __shfl_up_sync(0xFFFFFFFFu, t, o);
            if (lane >= o) t += y;
        }
        sums[lane] = t - s;
        if (lane == 31) sums[32] = t;
    }
    __syncthreads();
    const unsigned long long before = sums[warp] + x - v;
    *total = sums[32];
    __syncthreads();
    return before;
}
__device__ __forceinline__ unsigned long long pack2(int a, int b) { return ((unsigned long long)(unsigned)a << 32) | (unsigned)b; }

// Which of a round's pages from p0 on are free (or, kUsed, in use): word u of a warp holds 32 neighbouring pages from plan_page(p0, u,
// words) on, and no warp has more words than the round's pages, shared by all warps, need.
__device__ __forceinline__ int plan_words_of(int n_pages, int p0) { return min(kPlanRefs, (n_pages - p0 + kPlanThreads - 1) / kPlanThreads); }
__device__ __forceinline__ int plan_page(int p0, int u, int words) { return p0 + ((int)(threadIdx.x >> 5) * words + u) * 32; }
template <bool kUsed>
__device__ __forceinline__ void plan_words(const int32_t* refs, int n_pages, int p0, unsigned (&m)[kPlanRefs]) {
    const int words = plan_words_of(n_pages, p0);
    int r[kPlanRefs];
#pragma unroll
    for (int u = 0; u < kPlanRefs; ++u) {
        const int p = plan_page(p0, u, words) + (int)(threadIdx.x & 31);
        r[u] = u < words && p < n_pages ? refs[p] : (kUsed ? 0 : 1);
    }
#pragma unroll
    for (int u = 0; u < kPlanRefs; ++u) {
        m[u] = 0;
        if (u < words) m[u] = __ballot_sync(0xFFFFFFFFu, kUsed ? r[u] > 0 : r[u] == 0);
    }
}
// The sums of two counts of each warp over the warps in front of this one, and over all of them.
__device__ __forceinline__ int2 warps_before(int2 mine, int2* all) {
    __shared__ int2 of_warp[kPlanThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();
    if (lane == 0) of_warp[warp] = mine;
    __syncthreads();
    const int2 c = of_warp[lane];
    *all = make_int2(__reduce_add_sync(0xFFFFFFFFu, c.x), __reduce_add_sync(0xFFFFFFFFu, c.y));
    return make_int2(__reduce_add_sync(0xFFFFFFFFu, lane < warp ? c.x : 0), __reduce_add_sync(0xFFFFFFFFu, lane < warp ? c.y : 0));
}
__device__ __forceinline__ int words_sum(const unsigned (&m)[kPlanRefs]) {
    int n = 0;
#pragma unroll
    for (int u = 0; u < kPlanRefs; ++u) n += __popc(m[u]);
    return n;
}

struct ForkArgs {
    int n_pages, T, n_seqs, max_pages, n, share;
    const int32_t* src; const int32_t* dst; const int32_t* keep; const int32_t* want;
    int32_t* table; int32_t* refs;
    PlanArrays w;
    DeviceStatus* status;
};

// What one item asks for.  Its new pages, in order: `cow` or the copies of kept pages first, then empty ones.
struct ForkItem {
    int src, dst, first_new, n_new, n_copies;     // columns first_new .. first_new + n_new - 1 get new pages (a replaced one included)
};
__device__ __forceinline__ ForkItem fork_item(const ForkArgs& a, int4 given, bool* bad) {
    ForkItem f;
    f.src = given.x; f.dst = given.y;
    f.first_new = f.n_new = f.n_copies = 0;
    const int want = given.w, keep = f.src >= 0 ? given.z : 0;
    const long long room = (long long)a.max_pages * a.T;
    if ((unsigned)f.dst >= (unsigned)a.n_seqs || f.src >= a.n_seqs || want < 0 || want > room || keep < 0 || keep > room) {
        *bad = true;
        return f;
    }
    const int32_t* const row = a.table + (size_t)f.dst * a.max_pages;
    const int pages = (want + a.T - 1) / a.T, held = (keep + a.T - 1) / a.T, whole = keep / a.T;
    if (f.src == f.dst) {
        int lo = 0, hi = a.max_pages;             // entries in use come first
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (row[mid] >= 0) lo = mid + 1; else hi = mid;
        }
        if (held > lo) { *bad = true; return f; }
        f.first_new = lo;
        f.n_new = max(pages - lo, 0);
        // the page that the next token goes into, if the row holds it and others share it: replaced by a copy.  (It holds none of the
        // row's tokens where a row of more pages was set back to a border by its length alone.)
        if (whole < lo) {
            if ((unsigned)row[whole] >= (unsigned)a.n_pages) { *bad = true; return f; }
            if (a.refs[row[whole]] > 1) { f.n_copies = 1; f.n_new += 1; }
        }
    } else {
        if (row[0] >= 0) { *bad = true; return f; }       // (whether the source row holds all it should: source_has_holes)
        f.first_new = a.share ? whole : 0;
        f.n_copies = held - f.first_new;
        f.n_new = max(pages, held) - f.first_new;
    }
    return f;
}

// Whether a page that item i keeps of another row is none of the pool's, looked at by a warp; true in some lane.  Answers to one context
// often stand behind one another, and what the item before keeps of the same row has been looked at: 512 items of one row of 500 pages
// 22.8 us (20.5 without any of this), of rows of their own 55 (21); eight items 7.7 (7.7) and 7.8 (7.7) of 100 pages.
__device__ __forceinline__ bool source_has_holes(const ForkArgs& a, int i) {
    const int src = __ldg(a.src + i), dst = __ldg(a.dst + i), keep = __ldg(a.keep + i);
    if (src < 0 || src >= a.n_seqs || src == dst) return false;
    if (i > 0 && __ldg(a.src + i - 1) == src && __ldg(a.keep + i - 1) >= keep) return false;
    const int32_t* const row = a.table + (size_t)src * a.max_pages;
    const int held = min((int)(((long long)keep + a.T - 1) / a.T), a.max_pages);      // (fork_item refuses a longer one, or less than none)
    bool hole = false;
#pragma unroll 8
    for (int c = (int)(threadIdx.x & 31); c < held; c += 32) hole |= (unsigned)row[c] >= (unsigned)a.n_pages;
    return hole;
}

__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(const ForkArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31;
    __shared__ int any_bad;
    __shared__ unsigned named[kPlanRows / 32];
    // what the first round of everything needs is asked for at once
    unsigned free_words[kPlanRefs];
    plan_words<false>(a.refs, a.n_pages, 0, free_words);
    auto given = [&](int i) { return i < a.n ? make_int4(__ldg(a.src + i), __ldg(a.dst + i), __ldg(a.keep + i), __ldg(a.want + i)) : make_int4(-1, -1, 0, 0); };
    const int4 first = given(tid);
    if (tid == 0) any_bad = 0;
    const bool in_smem = a.n_seqs <= kPlanRows;
    if (in_smem) for (int i = tid; i < (a.n_seqs + 31) / 32; i += kPlanThreads) named[i] = 0;
    else for (int i = tid; i < a.n_seqs; i += kPlanThreads) a.w.marks[i] = 0;
    __syncthreads();
    // every row at most once as a target, and no target as another item's source
    for (int i = tid; i < a.n; i += kPlanThreads) {
        const int d = i == tid ? first.y : __ldg(a.dst + i);
        if ((unsigned)d >= (unsigned)a.n_seqs) continue;
        if (in_smem ? (atomicOr(&named[d >> 5], 1u << (d & 31)) >> (d & 31)) & 1u : (unsigned)(atomicAdd(&a.w.marks[d], 1) != 0)) any_bad = 1;
    }
    __syncthreads();
    // a warp per item, the last warps first: the first ones have the items' own chains of loads below
    for (int i = kPlanThreads / 32 - 1 - (tid >> 5); i < a.n; i += kPlanThreads / 32)
        if (source_has_holes(a, i)) any_bad = 1;
    auto is_named = [&](int d) { return in_smem ? ((named[d >> 5] >> (d & 31)) & 1u) != 0u : __ldcg(&a.w.marks[d]) != 0; };
    unsigned long long run = 0;
    for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        bool bad = false;
        ForkItem f = {};
        if (i < a.n) {
            f = fork_item(a, i == tid ? first : given(i), &bad);
            if (f.src >= 0 && f.src < a.n_seqs && f.src != f.dst && is_named(f.src)) bad = true;
            if (bad) any_bad = 1;
        }
        unsigned long long sum;
        const unsigned long long at = run + block_scan(pack2(f.n_new, f.n_copies), &sum);
        if (i < a.n) a.w.items[i] = make_int2((int)(at >> 32), (int)(at & 0xFFFFFFFFu));
        run += sum;
        if ((run >> 32) > (unsigned long long)a.n_pages) break;      // more than there are: the counts need not fit 32 bits
    }
    const long long n_new = (long long)(run >> 32);
    const int n_copies = (int)(run & 0xFFFFFFFFu);
    __syncthreads();
    if (any_bad || n_new > a.n_pages) {
        if (tid == 0) {
            report_status(a.status, any_bad ? DAF_ERR_BOUNDS : DAF_ERR_PAGES, 220, (int)n_new);
            *a.w.head = PlanHead{0, 0, 0, 0};
        }
        return;
    }
    // the n_new free pages of lowest number
    int found = 0;
    for (int p0 = 0; p0 < a.n_pages && found < n_new; p0 += kPlanRound) {
        if (p0 > 0) plan_words<false>(a.refs, a.n_pages, p0, free_words);
        int2 all;
        int at = found + warps_before(make_int2(words_sum(free_words), 0), &all).x;
        const int words = plan_words_of(a.n_pages, p0);
#pragma unroll
        for (int u = 0; u < kPlanRefs; ++u) {
            if (u >= words) break;
            const int rank = at + __popc(free_words[u] & ((1u << lane) - 1u));
            if (((free_words[u] >> lane) & 1u) && rank < n_new) a.w.fresh[rank] = plan_page(p0, u, words) + lane;
            at += __popc(free_words[u]);
        }
        found += all.x;
    }
    const bool ok = found >= n_new;
    if (tid == 0) {
        if (!ok) report_status(a.status, DAF_ERR_PAGES, 221, (int)n_new);
        *a.w.head = PlanHead{ok ? 1 : 0, (int)n_new, ok ? n_copies : 0, 0};
        a.w.items[a.n] = make_int2((int)n_new, n_copies);
    }
    __syncthreads();
    if (!ok) return;
    // the copies: a warp per item
    for (int i = tid >> 5; i < a.n; i += kPlanThreads / 32) {
        const int2 at = a.w.items[i];
        const int n_c = a.w.items[i + 1].y - at.y;
        const int src = __ldg(a.src + i), dst = __ldg(a.dst + i);
        const int first = (src == dst || a.share) ? __ldg(a.keep + i) / a.T : 0;      // (n_c > 0 only where src >= 0)
        for (int c = tid & 31; c < n_c; c += 32)
            a.w.copies[at.y + c] = make_int2(a.table[(size_t)src * a.max_pages + first + c], a.w.fresh[at.x + c]);
    }
}

struct MoveArgs {          // the bytes of pages, K and V with their scales, in all layers
    uint4* k8; uint4* v8; float* k_scale; float* v_scale;
    long long n_pages;
    int Hkv, n_layers, page_chunks;      // chunks of 16 bytes of one page of one layer, K or V
};
constexpr int kMoveThreads = 256, kMoveUnroll = 4;

// The pages of copies[0 .. n) by the whole grid: pieces of 16 KB, every thread's four chunks requested before the first is stored.
__device__ __forceinline__ void move_pages(const MoveArgs& m, const int2* copies, int n) {
    constexpr int kPiece = kMoveThreads * kMoveUnroll;
    const int pieces = (m.page_chunks + kPiece - 1) / kPiece;
    const long long units = (long long)n * m.n_layers * 2 * pieces;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int piece = (int)(u % pieces);
        const long long rest = u / pieces;
        const bool is_v = (rest & 1) != 0;
        const int layer = (int)((rest >> 1) % m.n_layers);
        const int2 c = __ldg(copies + (rest >> 1) / m.n_layers);
        const long long from = (long long)layer * m.n_pages + c.x, to = (long long)layer * m.n_pages + c.y;
        uint4* const pool = is_v ? m.v8 : m.k8;
        const uint4* const s = pool + from * m.page_chunks;
        uint4* const d = pool + to * m.page_chunks;
        const int i0 = piece * kPiece + (int)threadIdx.x;
        uint4 w[kMoveUnroll];
#pragma unroll
        for (int i = 0; i < kMoveUnroll; ++i)
            if (i0 + i * kMoveThreads < m.page_chunks) w[i] = __ldcs(s + i0 + i * kMoveThreads);
        float* const sc = is_v ? m.v_scale : m.k_scale;
        float x = 0.f;
        const bool scaled = piece == 0 && (int)threadIdx.x < m.Hkv;        // (256 heads at most)
        if (scaled) x = sc[from * m.Hkv + threadIdx.x];
#pragma unroll
        for (int i = 0; i < kMoveUnroll; ++i)
            if (i0 + i * kMoveThreads < m.page_chunks) __stcs(d + i0 + i * kMoveThreads, w[i]);
        if (scaled) sc[to * m.Hkv + threadIdx.x] = x;
    }
}

__global__ void __launch_bounds__(kMoveThreads) fork_apply_kernel(const ForkArgs a, const MoveArgs m) {
    pdl_wait();
    pdl_launch_dependents();
    const PlanHead head = *a.w.head;
    if (!head.ok) return;
    // table rows and counts: CTAs take columns of items
    const int parts = (a.max_pages + kMoveThreads - 1) / kMoveThreads;
    for (long long u = blockIdx.x; u < (long long)a.n * parts; u += gridDim.x) {
        const int i = (int)(u / parts), col = (int)(u % parts) * kMoveThreads + (int)threadIdx.x;
        if (col >= a.max_pages) continue;
        const int src = __ldg(a.src + i), dst = __ldg(a.dst + i);
        const int2 at = a.w.items[i], next = a.w.items[i + 1];
        const int n_new = next.x - at.x, n_copies = next.y - at.y;
        int32_t* const entry = a.table + (size_t)dst * a.max_pages + col;
        int first_new;          // first column of the new pages behind those held
        int fresh_at = at.x;
        if (src == dst) {
            const int held = (__ldg(a.want + i) + a.T - 1) / a.T - (n_new - n_copies);      // columns in use before, if it grows
            if (n_copies > 0) {
                fresh_at += 1;
                if (col == __ldg(a.keep + i) / a.T) {
                    const int old = *entry, page = a.w.fresh[at.x];
                    atomicSub(a.refs + old, 1);
                    a.refs[page] = 1;
                    *entry = page;
                    continue;
                }
            }
            if (n_new - n_copies <= 0) continue;
            first_new = held;
            const int j = col - first_new;
            if (j >= 0 && j < n_new - n_copies) {
                const int page = a.w.fresh[fresh_at + j];
                a.refs[page] = 1;
                *entry = page;
            }
            continue;
        }
        first_new = src >= 0 && a.share ? __ldg(a.keep + i) / a.T : 0;
        int page = -1;
        if (col < first_new) {
            page = a.table[(size_t)src * a.max_pages + col];
            atomicAdd(a.refs + page, 1);
        } else if (col - first_new < n_new) {
            page = a.w.fresh[fresh_at + col - first_new];
            a.refs[page] = 1;
        }
        *entry = page;
    }
    move_pages(m, a.w.copies, head.n_copies);
}

struct FreeArgs {
    int n_pages, T, n_seqs, max_pages, n;
    const int32_t* seqs; const int32_t* keep; int32_t* table; int32_t* refs;
    DeviceStatus* status;
};
__global__ void __launch_bounds__(256) page_free_kernel(const FreeArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const int i = blockIdx.x;
    const int seq = __ldg(a.seqs + i), keep = a.keep != nullptr ? __ldg(a.keep + i) : 0;
    if ((unsigned)seq >= (unsigned)a.n_seqs || keep < 0) {
        if (threadIdx.x == 0 && blockIdx.y == 0) report_status(a.status, DAF_ERR_BOUNDS, 230, seq);
        return;
    }
    const int held = (int)(((long long)keep + a.T - 1) / a.T);
    for (int col = held + (int)(blockIdx.y * 256 + threadIdx.x); col < a.max_pages; col += gridDim.y * 256) {
        int32_t* const entry = a.table + (size_t)seq * a.max_pages + col;
        if (*entry < 0) continue;
        const int page = atomicExch(entry, -1);          // a row named twice gives each page back once
        if (page < 0) continue;
        if (page >= a.n_pages) { report_status(a.status, DAF_ERR_BOUNDS, 231, page); continue; }
        if (atomicSub(a.refs + page, 1) <= 0) {          // the count did not cover this entry
            atomicAdd(a.refs + page, 1);
            report_status(a.status, DAF_ERR_BOUNDS, 232, page);
        }
    }
}

struct CompactArgs {
    int n_pages; long long entries;
    const int32_t* table; const int32_t* refs; int32_t* table_out; int32_t* refs_out; int32_t* live_out;
    PlanArrays w;
    DeviceStatus* status;
};
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(const CompactArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31;
    unsigned used[kPlanRefs];
    int2 all;
    int live = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += kPlanRound) {
        plan_words<true>(a.refs, a.n_pages, p0, used);
        warps_before(make_int2(words_sum(used), 0), &all);
        live += all.x;
    }
    // the r-th page in use at or above `live` goes to the r-th free one below it
    int holes = 0, movers = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += kPlanRound) {
        if (a.n_pages > kPlanRound) plan_words<true>(a.refs, a.n_pages, p0, used);
        const int words = plan_words_of(a.n_pages, p0);
        auto below = [&](int u) {            // pages of word u in front of `live`
            const int n = live - plan_page(p0, u, words);
            return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
        };
        int2 mine = make_int2(0, 0);
#pragma unroll
        for (int u = 0; u < kPlanRefs; ++u) {
            if (u >= words) break;
            mine.x += __popc(~used[u] & below(u));
            mine.y += __popc(used[u] & ~below(u));
        }
        const int2 before = warps_before(mine, &all);
        int h = holes + before.x, v = movers + before.y;
#pragma unroll
        for (int u = 0; u < kPlanRefs; ++u) {
            if (u >= words) break;
            const unsigned hole = ~used[u] & below(u), mover = used[u] & ~below(u), lower = (1u << lane) - 1u;
            const int p = plan_page(p0, u, words) + lane;
            if ((hole >> lane) & 1u) a.w.copies[h + __popc(hole & lower)].y = p;
            if ((mover >> lane) & 1u) a.w.copies[v + __popc(mover & lower)].x = p;
            else if (p >= live && p < a.n_pages) a.w.fresh[p] = -1;      // where no page goes to: an entry of the table must not name it
            h += __popc(hole);
            v += __popc(mover);
        }
        holes += all.x;
        movers += all.y;
    }
    __syncthreads();
    // The counts, here because refs_out may be refs: a moved page's goes to its new place before its old one is cleared, and nothing else
    // touches either.
    for (int r = tid; r < movers; r += kPlanThreads) {
        const int2 c = a.w.copies[r];
        const int count = a.refs[c.x];
        a.w.fresh[c.x] = c.y;
        a.refs_out[c.y] = count;
        a.refs_out[c.x] = 0;
    }
    if (a.refs_out != a.refs)
        for (int p = tid; p < live; p += kPlanThreads) {
            const int r = a.refs[p];
            if (r > 0) a.refs_out[p] = r;
        }
    for (int p = live + tid; p < a.n_pages; p += kPlanThreads)
        if (a.refs[p] <= 0) a.refs_out[p] = 0;
    if (tid == 0) {
        *a.w.head = PlanHead{1, 0, movers, live};
        if (a.live_out != nullptr) *a.live_out = live;
    }
}
__global__ void __launch_bounds__(kMoveThreads) compact_apply_kernel(const CompactArgs a, const MoveArgs m) {
    pdl_wait();
    pdl_launch_dependents();
    const PlanHead head = *a.w.head;
    for (long long i = (long long)blockIdx.x * kMoveThreads + threadIdx.x; i < a.entries; i += (long long)gridDim.x * kMoveThreads) {
        int page = a.table[i];
        if (page >= head.live) {
            const int to = page < a.n_pages ? a.w.fresh[page] : -1;
            if (to < 0) report_status(a.status, DAF_ERR_BOUNDS, 240, page);      // outside the pool, or of no count
            page = to;
        }
        a.table_out[i] = page < 0 ? -1 : page;
    }
    move_pages(m, a.w.copies, head.n_copies);
}

// ------------------------------------------------------------------------------------------------------------------ host side
constexpr int kPageMaxTokens = 1 << 22;

static int resolve_pages(const daf_page_params* p) {
    if (p == nullptr) return DAF_ERR_INVALID_ARG;
    if (p->n_pages <= 0 || p->n_kv_heads <= 0 || p->n_layers <= 0 || p->n_seqs <= 0 || p->max_pages <= 0) return DAF_ERR_INVALID_ARG;
    if (p->head_dim != 128 || p->n_kv_heads > 256) return DAF_ERR_UNSUPPORTED;
    if (p->page_tokens != 16 && p->page_tokens != 32 && p->page_tokens != 64 && p->page_tokens != 128) return DAF_ERR_UNSUPPORTED;
    if ((long long)p->max_pages * p->page_tokens > kPageMaxTokens) return DAF_ERR_UNSUPPORTED;
    // rows of one layer are numbered in 32 bits; tables, sequences and layers stay in the range of the kernels' products
    if ((long long)p->n_pages * p->n_kv_heads * p->page_tokens > 0x7FFFFFFFll) return DAF_ERR_UNSUPPORTED;
    if (p->n_seqs > (1 << 20) || p->n_layers > 4096) return DAF_ERR_UNSUPPORTED;
    return DAF_OK;
}
// daf_page_attn counts its steps of 32 keys in 32 bits.
static bool steps_fit(const daf_page_params* p, int n) {
    return (long long)n * p->n_kv_heads * p->max_pages * p->page_tokens <= 1ll << 35;
}
static size_t round256(size_t x) { return (x + 255) / 256 * 256; }
static size_t plan_bytes(const daf_page_params* p, int n) {
    return 256 + round256((size_t)p->n_pages * 8) + round256((size_t)p->n_pages * 4) + round256((size_t)p->n_seqs * 4) +
           round256(((size_t)n + 1) * 8);
}
static PlanArrays plan_arrays(const daf_page_params* p, void* workspace) {
    char* at = reinterpret_cast<char*>(workspace) + kStatusBytes;
    PlanArrays w;
    w.head = reinterpret_cast<PlanHead*>(at); at += 256;
    w.copies = reinterpret_cast<int2*>(at); at += round256((size_t)p->n_pages * 8);
    w.fresh = reinterpret_cast<int32_t*>(at); at += round256((size_t)p->n_pages * 4);
    w.marks = reinterpret_cast<int32_t*>(at); at += round256((size_t)p->n_seqs * 4);
    w.items = reinterpret_cast<int2*>(at);
    return w;
}
static Pool layer_of(const daf_page_params* p, int layer, const void* k8, const void* v8, const float* k_scale, const float* v_scale) {
    const size_t rows = (size_t)layer * p->n_pages * p->n_kv_heads;
    Pool q;
    q.n_pages = p->n_pages; q.T = p->page_tokens; q.Hkv = p->n_kv_heads; q.n_seqs = p->n_seqs; q.max_pages = p->max_pages;
    q.k8 = reinterpret_cast<uint8_t*>(const_cast<void*>(k8)) + rows * p->page_tokens * 128;
    q.v8 = reinterpret_cast<uint8_t*>(const_cast<void*>(v8)) + rows * p->page_tokens * 128;
    q.k_scale = const_cast<float*>(k_scale) + rows;
    q.v_scale = const_cast<float*>(v_scale) + rows;
    return q;
}
static MoveArgs move_args(const daf_page_params* p, void* k8, void* v8, float* k_scale, float* v_scale) {
    MoveArgs m;
    m.k8 = reinterpret_cast<uint4*>(k8); m.v8 = reinterpret_cast<uint4*>(v8); m.k_scale = k_scale; m.v_scale = v_scale;
    m.n_pages = p->n_pages; m.Hkv = p->n_kv_heads; m.n_layers = p->n_layers; m.page_chunks = p->n_kv_heads * p->page_tokens * 8;
    return m;
}
static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// The pool's four tensors, all needed; the bytes 16-byte, the scales 4-byte aligned.
static int check_pool(const void* k8, const void* v8, const float* k_scale, const float* v_scale) {
    if (!k8 || !v8 || !k_scale || !v_scale) return DAF_ERR_INVALID_ARG;
    if (!aligned16(k8) || !aligned16(v8) || !aligned4(k_scale) || !aligned4(v_scale)) return DAF_ERR_ALIGNMENT;
    return DAF_OK;
}
static int check_ints(const void* const* ptrs, int count) {
    for (int i = 0; i < count; ++i)
        if (!aligned4(ptrs[i])) return DAF_ERR_ALIGNMENT;
    return DAF_OK;
}
static int check_workspace(void* workspace, size_t have, size_t need) {
    if (workspace == nullptr || have < need) return DAF_ERR_WORKSPACE;
    return aligned16(workspace) ? DAF_OK : DAF_ERR_ALIGNMENT;
}
static int launched(cudaError_t e) {
    count_launch();
    if (e != cudaSuccess) { set_cuda_error(e); return DAF_ERR_CUDA; }
    return check_launch();
}
// Pages that `rows` newest (or any consecutive) tokens can touch.
static int touched_pages(const daf_page_params* p, int rows) {
    if (rows > kPageMaxTokens) rows = kPageMaxTokens;
    const int t = (rows + p->page_tokens - 2) / p->page_tokens + 1;
    return t < p->max_pages ? t : p->max_pages;
}
// CTAs for an entry's pages (for each head, K and V apart): one per page, but no more than `most` in the whole grid as long as each
// entry has one.  The grid's first dimension stays in its range either way.
static int page_slots(const daf_page_params* p, int n, int pages, long long most) {
    most /= 2ll * p->n_kv_heads * n;
    const long long room = 0x7FFFFFFFll / n;
    if (most > room) most = room;
    return (int)(pages < most ? pages : most < 1 ? 1 : most);
}
constexpr long long kAllPages = 1ll << 40;

}  // namespace daf

using namespace daf;

extern "C" {

size_t daf_page_workspace_bytes(const daf_page_params* p, int32_t n, int32_t L_q, int32_t n_q_heads) {
    if (resolve_pages(p) != DAF_OK || n < 0 || L_q < 0 || n_q_heads < 0) return 0;
    size_t need = plan_bytes(p, n);
    if (L_q > 0 && n_q_heads > 0) {
        if (n_q_heads % p->n_kv_heads != 0 || n_q_heads > 256 || L_q > kPageMaxTokens || n > kPageMaxSeqs || !steps_fit(p, n)) return 0;
        const size_t attn = page_attn_scratch_bytes(n, L_q, n_q_heads, p->n_kv_heads);
        if (attn > need) need = attn;
    }
    return kStatusBytes + need;
}

int daf_page_write(const daf_page_params* p, int32_t layer, int32_t n, const int32_t* seqs, const int32_t* lens,
                   const int32_t* row_off, const int32_t* idx, int32_t max_rows, const void* k, const void* v,
                   const int32_t* table, const int32_t* refs, void* k8, void* v8, float* k_scale, float* v_scale,
                   void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = resolve_pages(p)) return rc;
    if (int rc = check_workspace(workspace, workspace_bytes, kStatusBytes)) return rc;
    if (layer < 0 || layer >= p->n_layers || n < 0 || max_rows < 0) return DAF_ERR_INVALID_ARG;
    if (n == 0 || max_rows == 0) return DAF_OK;
    if (!lens || !row_off || !k || !v || !table) return DAF_ERR_INVALID_ARG;
    if (int rc = check_pool(k8, v8, k_scale, v_scale)) return rc;
    if (!aligned16(k) || !aligned16(v)) return DAF_ERR_ALIGNMENT;
    const void* ints[] = {seqs, lens, row_off, idx, table, refs};
    if (int rc = check_ints(ints, 6)) return rc;
    WriteArgs a;
    a.p = layer_of(p, layer, k8, v8, k_scale, v_scale);
    a.n = n;
    // (given positions may lie anywhere in a row of the table: CTAs for all of it, up to some rounds of the GPU)
    a.slots = idx == nullptr ? page_slots(p, n, touched_pages(p, max_rows), kAllPages) : page_slots(p, n, p->max_pages, 16384);
    a.seqs = seqs; a.lens = lens; a.row_off = row_off; a.idx = idx;
    a.k = reinterpret_cast<const __nv_bfloat16*>(k); a.v = reinterpret_cast<const __nv_bfloat16*>(v);
    a.table = table; a.refs = refs; a.status = reinterpret_cast<DeviceStatus*>(workspace);
    auto* kernel = p->page_tokens == 16 ? (idx ? page_write_kernel<16, true> : page_write_kernel<16, false>)
                 : p->page_tokens == 32 ? (idx ? page_write_kernel<32, true> : page_write_kernel<32, false>)
                 : p->page_tokens == 64 ? (idx ? page_write_kernel<64, true> : page_write_kernel<64, false>)
                                        : (idx ? page_write_kernel<128, true> : page_write_kernel<128, false>);
    return launched(launch_kernel(kernel, dim3((unsigned)n * a.slots, p->n_kv_heads, 2), dim3(128), 0, (cudaStream_t)stream, a));
}

int daf_page_read(const daf_page_params* p, int32_t layer, int32_t n, const int32_t* seqs, const int32_t* first,
                  const int32_t* row_off, int32_t max_rows, const int32_t* table, const void* k8, const void* v8,
                  const float* k_scale, const float* v_scale, void* k_rows, void* v_rows,
                  void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = resolve_pages(p)) return rc;
    if (int rc = check_workspace(workspace, workspace_bytes, kStatusBytes)) return rc;
    if (layer < 0 || layer >= p->n_layers || n < 0 || max_rows < 0) return DAF_ERR_INVALID_ARG;
    if (n == 0 || max_rows == 0) return DAF_OK;
    if (!row_off || !table || !k_rows || !v_rows) return DAF_ERR_INVALID_ARG;
    if (int rc = check_pool(k8, v8, k_scale, v_scale)) return rc;
    if (!aligned16(k_rows) || !aligned16(v_rows)) return DAF_ERR_ALIGNMENT;
    const void* ints[] = {seqs, first, row_off, table};
    if (int rc = check_ints(ints, 4)) return rc;
    ReadArgs a;
    a.p = layer_of(p, layer, k8, v8, k_scale, v_scale);
    a.n = n; a.slots = page_slots(p, n, touched_pages(p, max_rows), kAllPages);
    a.seqs = seqs; a.first = first; a.row_off = row_off; a.table = table;
    a.k = reinterpret_cast<__nv_bfloat16*>(k_rows); a.v = reinterpret_cast<__nv_bfloat16*>(v_rows);
    a.status = reinterpret_cast<DeviceStatus*>(workspace);
    auto* kernel = p->page_tokens == 16 ? page_read_kernel<1> : p->page_tokens == 32 ? page_read_kernel<2>
                 : p->page_tokens == 64 ? page_read_kernel<4> : page_read_kernel<8>;
    return launched(launch_kernel(kernel, dim3((unsigned)n * a.slots, p->n_kv_heads, 2), dim3(128), 0, (cudaStream_t)stream, a));
}

int daf_page_attn(const daf_page_params* p, int32_t layer, int32_t n, const int32_t* seqs, const int32_t* lens, int32_t L_q,
                  int32_t n_q_heads, float softmax_scale, const void* q, const int32_t* table, const void* k8, const void* v8,
                  const float* k_scale, const float* v_scale, void* out, float* lse,
                  void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = resolve_pages(p)) return rc;
    if (layer < 0 || layer >= p->n_layers || n < 0 || L_q < 0 || n_q_heads <= 0) return DAF_ERR_INVALID_ARG;
    if (n_q_heads % p->n_kv_heads != 0 || n_q_heads > 256 || n > kPageMaxSeqs) return DAF_ERR_UNSUPPORTED;
    if ((long long)n * L_q > kPageMaxTokens) return DAF_ERR_UNSUPPORTED;
    if (!steps_fit(p, n)) return DAF_ERR_UNSUPPORTED;
    if (int rc = check_workspace(workspace, workspace_bytes, kStatusBytes)) return rc;
    if (n == 0 || L_q == 0) return DAF_OK;
    if (int rc = check_workspace(workspace, workspace_bytes, kStatusBytes + page_attn_scratch_bytes(n, L_q, n_q_heads, p->n_kv_heads))) return rc;
    if (!lens || !q || !table || !out) return DAF_ERR_INVALID_ARG;
    if (int rc = check_pool(k8, v8, k_scale, v_scale)) return rc;
    if (!aligned16(q) || !aligned16(out)) return DAF_ERR_ALIGNMENT;
    const void* ints[] = {seqs, lens, table, lse};
    if (int rc = check_ints(ints, 4)) return rc;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.08838834764831845f;      // 1 / sqrt(128)
    return launch_page_attn(layer_of(p, layer, k8, v8, k_scale, v_scale), n, seqs, lens, L_q, n_q_heads, scale, q, table, out, lse,
                            reinterpret_cast<DeviceStatus*>(workspace), reinterpret_cast<char*>(workspace) + kStatusBytes,
                            (cudaStream_t)stream);
}

int daf_page_fork(const daf_page_params* p, int32_t n, const int32_t* src, const int32_t* dst, const int32_t* keep,
                  const int32_t* want, int32_t share, int32_t* table, int32_t* refs, void* k8, void* v8, float* k_scale,
                  float* v_scale, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = resolve_pages(p)) return rc;
    if (n < 0) return DAF_ERR_INVALID_ARG;
    if (n > p->n_seqs) return DAF_ERR_INVALID_ARG;         // some row would be named twice
    if (int rc = check_workspace(workspace, workspace_bytes, kStatusBytes + plan_bytes(p, n))) return rc;
    if (n == 0) return DAF_OK;
    if (!src || !dst || !keep || !want || !table || !refs) return DAF_ERR_INVALID_ARG;
    if (int rc = check_pool(k8, v8, k_scale, v_scale)) return rc;
    const void* ints[] = {src, dst, keep, want, table, refs};
    if (int rc = check_ints(ints, 6)) return rc;
    ForkArgs a;
    a.n_pages = p->n_pages; a.T = p->page_tokens; a.n_seqs = p->n_seqs; a.max_pages = p->max_pages; a.n = n; a.share = share != 0;
    a.src = src; a.dst = dst; a.keep = keep; a.want = want; a.table = table; a.refs = refs;
    a.w = plan_arrays(p, workspace); a.status = reinterpret_cast<DeviceStatus*>(workspace);
    cudaStream_t st = (cudaStream_t)stream;
    if (int rc = launched(launch_kernel(fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a))) return rc;
    return launched(launch_kernel(fork_apply_kernel, dim3((unsigned)num_sms() * 8), dim3(kMoveThreads), 0, st, a,
                                  move_args(p, k8, v8, k_scale, v_scale)));
}

int daf_page_free(const daf_page_params* p, int32_t n, const int32_t* seqs, const int32_t* keep, int32_t* table, int32_t* refs,
                  void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = resolve_pages(p)) return rc;
    if (n < 0) return DAF_ERR_INVALID_ARG;
    if (int rc = check_workspace(workspace, workspace_bytes, kStatusBytes)) return rc;
    if (n == 0) return DAF_OK;
    if (!seqs || !table || !refs) return DAF_ERR_INVALID_ARG;
    const void* ints[] = {seqs, keep, table, refs};
    if (int rc = check_ints(ints, 4)) return rc;
    FreeArgs a;
    a.n_pages = p->n_pages; a.T = p->page_tokens; a.n_seqs = p->n_seqs; a.max_pages = p->max_pages; a.n = n;
    a.seqs = seqs; a.keep = keep; a.table = table; a.refs = refs; a.status = reinterpret_cast<DeviceStatus*>(workspace);
    const unsigned parts = (unsigned)((p->max_pages + 255) / 256);
    return launched(launch_kernel(page_free_kernel, dim3(n, parts < 64 ? parts : 64), dim3(256), 0, (cudaStream_t)stream, a));
}

int daf_page_compact(const daf_page_params* p, const int32_t* table, const int32_t* refs, int32_t* table_out, int32_t* refs_out,
                     int32_t* live_out, void* k8, void* v8, float* k_scale, float* v_scale,
                     void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = resolve_pages(p)) return rc;
    if (int rc = check_workspace(workspace, workspace_bytes, kStatusBytes + plan_bytes(p, 0))) return rc;
    if (!table || !refs || !table_out || !refs_out) return DAF_ERR_INVALID_ARG;
    if (int rc = check_pool(k8, v8, k_scale, v_scale)) return rc;
    const void* ints[] = {table, refs, table_out, refs_out, live_out};
    if (int rc = check_ints(ints, 5)) return rc;
    CompactArgs a;
    a.n_pages = p->n_pages; a.entries = (long long)p->n_seqs * p->max_pages;
    a.table = table; a.refs = refs; a.table_out = table_out; a.refs_out = refs_out; a.live_out = live_out;
    a.w = plan_arrays(p, workspace); a.status = reinterpret_cast<DeviceStatus*>(workspace);
    cudaStream_t st = (cudaStream_t)stream;
    if (int rc = launched(launch_kernel(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a))) return rc;
    return launched(launch_kernel(compact_apply_kernel, dim3((unsigned)num_sms() * 8), dim3(kMoveThreads), 0, st, a,
                                  move_args(p, k8, v8, k_scale, v_scale)));
}

}  // extern "C"
