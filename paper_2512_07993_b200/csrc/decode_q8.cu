// skipkv_decode_attn_q8: GQA decode attention over a cache held in 8 bits, with the steering add in the same launch.
//
// out = sum_t softmax_t(q . (s_k c_k)[t] / sqrt(d)) (s_v c_v)[t].  A block's scale is one number for 16 tokens or more, so it never touches the
// codes: s_k multiplies 16 logits of a head at once, s_v the tile's share of the output sums.  Every live row is read once, 256 bytes
// per token and slab.
//  * Work = tiles of 128 tokens (a page) enumerated over all (sequence, head) slabs and cut into equal contiguous ranges, one per CTA, two CTAs
//    per SM (one: 312 us against 240 for 128 slabs of 32K to 64K: a tile is a chain of latencies); each (CTA, slab) intersection gives one partial
//    (maximum, sum, 128 sums per head); the last CTA that delivers one for a slab merges them.  A slab costs a few places beside its tiles in the
//    partition, because the end of a part costs time (80 slabs of 4.1K: 21.4 us with four, 24.2 with none).
//  * Four warps, each with its own 32 rows of every tile and its own ring of asynchronous copies (three stages of 8 KB): no barrier in the
//    stream, and nothing to wait for but a warp's own copies.  16 rows per warp and twice the warps, 304 us; tile copies by the bulk engine, issued by a
//    lane per warp or by a fifth warp for all, 242 and 246 against 240 (128 slabs of 32K to 64K), 53.4 and 51.5 against 50.2 (8.2K, paged).
//  * S = K Q^T on the tensor cores (a query row per head is far below a tcgen05 tile).  e4m3: the codes are operands as they lie in memory (mma.sync
//    m16n8k32), a query head is two e4m3 parts, which together have the 8 bits of a bf16.  int8: codes and queries as f16 (m16n8k16), exact for both.
//    O^T = V^T P^T in f16, of which every code is a value.  The order of channels in S and of tokens and channels in O is free, so a lane
//    takes 16 bytes of a row as they lie: 32 consecutive channels of a key row (two 16-byte loads), 16 consecutive channels of four value rows, of
//    which byte permutes make pairs of tokens.  Rows are 128 bytes; their 16-byte pieces lie permuted (piece c of row r at c ^ (r & 7)), so
//    neither load has bank conflicts.
//  * The probabilities go in as two f16 parts of 2^15 p, 22 bits of the fp32 value, absolute 2^-40 for small ones; a tile's products are added to the
//    sums over the tiles in fp32 with rounding (the tensor core's own accumulation truncates), times the scale and 2^-15: sums of
//    p |v| may reach 2^127.  Up to four heads per group the eight columns hold the high and low parts of a head side by side, so that a lane has one head to exponentiate.
//  * An arrival's answer is not waited for before the CTA's next part; the last CTA of a slab loads its partials 16 at a time.
// What it takes (back to back, some hundred calls, and what bounds it): one sequence of 2048 tokens 7.4 us, latency (wait 0.9, first rows 2.0, a tile 0.9, its warps
// merged 0.6, arrival 0.9, merge 1.3); 80 slabs of 4.1K 19.4 us, 0.66 of the copy rate: head and tail of a launch, between them 6.8 to 7.5 TB/s into the SMs; 128 slabs of
// 8.2K behind pages, int8, five heads 49.8 us, 0.82: conversions and latency; 128 slabs of 32K to 64K 241 to 250 us, 0.98 to 1.02.  In seconds of it the power limit
// takes the clock down: 55 and 285 us for the last two.
#include <type_traits>

#include "common.cuh"
#include "mma.cuh"
#include "q8.cuh"
#include "steer.cuh"

namespace skipkv {

constexpr int kQdWarps = 4;
constexpr int kQdThreads = kQdWarps * 32;
constexpr int kQdRows = 32;                                   // rows of a tile that one warp works on: two groups of 16
static_assert(kQdWarps * kQdRows == kQ8Tile, "a tile is a page");
constexpr int kQdStages = 3;
constexpr int kQdStageBytes = 2 * kQdRows * kQ8RowBytes;      // one warp's key rows, then its value rows
constexpr int kQdRingBytes = kQdWarps * kQdStages * kQdStageBytes;
constexpr int kQdMaxGrid = 512;
constexpr int kQdPartCost = 4;                                // what a slab costs beside its tiles, in tiles: the end of a part
constexpr int kQdPrefetch = 3;                                // tiles that a CTA starts towards L2 before it may read the cache
constexpr int kQdTableSlabs = 1024;                           // from so many slabs on their table has a launch of its own: 1024 of 300 rows 29.8 us
                                                              // with it and 31.7 without, 512 of 200 rows 15.9 and 15.3
constexpr float kQdLeast = -3.4028234663852886e38f;           // below no logit: the lowest finite number
constexpr float kQdUnit = 1.f / 32768.f;                      // what a probability of 2^15 stands for
constexpr int kQdSumStride = kHeadDim + 4;                    // (of a column's sums in shared memory)
static_assert(kQdStageBytes >= 8 * kQdSumStride * 4, "a warp's sums of a segment fit into a stage");
constexpr int kQdMergeParts = 16;                             // partials of a head that are merged at a time, half a warp
static_assert((1ull << 22) * kQdMaxGrid <= (1ull << 32), "places times CTAs in 32 bits");
static_assert(kQdThreads == kHeadDim, "a thread merges one channel");

// D[16 x 8] += A[16 x 16] B[16 x 8], f16 operands, fp32 accumulators; the first form has no sum to add to
__device__ __forceinline__ void mma16816h(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816h_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// D[16 x 8] (+)= A[16 x 32] B[32 x 8], e4m3 operands, fp32 accumulators
__device__ __forceinline__ void mma16832q(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16832q_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// two probabilities as two f16 parts each
__device__ __forceinline__ void split_f16(float2 x, uint32_t& hi, uint32_t& lo) {
    hi = pack_f16(x.x, x.y);
    const float2 r = __ffma2_rn(f16x2_to_f2(hi), make_float2(-1.f, -1.f), x);
    lo = pack_f16(r.x, r.y);
}
// Four f16 values to e4m3; 32 (y - h) of two f16 values
__device__ __forceinline__ uint32_t f16_to_e4m3(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f16x2 x, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 y, %2;\n\tmov.b32 %0, {x, y};\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t rest32(uint32_t y, uint32_t h) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(y), "r"(h));
    asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(d) : "r"(0x50005000u));
    return d;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr) : "memory");
    return r;
}
// 16 bytes global -> shared, asynchronously (rows are 128 bytes: no more than that is asked of L2); bytes = 0 writes zeros and reads nothing
__device__ __forceinline__ void cp_async_piece(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_piece(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// The lengths and the partition's prefix sum of many slabs (q8_table_kernel).
struct QdSlabs {
    struct Raw { int len, cap; };
    Q8View c;
    const int32_t *kv_len, *cap;
    int Hk;
    int* lens;
    __device__ __forceinline__ Raw load(int s) const { return {kv_len[s], cap[s / Hk]}; }
    __device__ __forceinline__ int count(int s, const Raw& r) const {
        const int len = min(max(r.len, 0), q8_room(c, r.cap));
        lens[s] = len;
        return len ? (len + kQ8Tile - 1) / kQ8Tile + kQdPartCost : 0;
    }
};

// kFew: up to four heads per group.  kTable: many slabs, whose table the launch ahead has made.
template <int kFmt, bool kFew, bool kTable>
__global__ void __launch_bounds__(kQdThreads, 2)
decode_q8_kernel(int batch, int Hq, int Hk, int n_slabs, const int64_t* slab_off, const int32_t* cap, const __nv_bfloat16* q, Q8View c,
                 const int32_t* kv_len, __nv_bfloat16* out, uint32_t* status, uint32_t* dec_cnt, float* dec_part, int d_model,
                 __nv_bfloat16* hidden, const __nv_bfloat16* steer_vec, const float* alpha, const uint8_t* flag, int* slab_table) {
    extern __shared__ __align__(128) uint8_t dsm[];
    const int n = Hq / Hk;                                                   // heads per group
    int* pref = kTable ? slab_table : reinterpret_cast<int*>(dsm + kQdRingBytes);      // [n_slabs + 1] tile prefix
    int* lens = pref + n_slabs + 1;                                          // [n_slabs]
    __shared__ __align__(16) float s_scale[kQdWarps][kQdStages][4];          // of each stage's key rows (two groups of 16), then of its value rows
    __shared__ float2 s_ml[kQdWarps][kMaxGroup];                             // a segment's maxima and sums
    __shared__ uint32_t s_wsum[kQdWarps];
    __shared__ int s_last;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = gridDim.x, cta = blockIdx.x;
    // ---- schedule: CTA k has the places [k T / Ge, (k + 1) T / Ge) of T, Ge = the CTAs that have work; a slab has kQdPartCost places and then one
    // for each tile.  The lengths may be written by
    // the launch ahead of this one, but the number of tiles they make is mostly older (a step adds one row).  So the schedule is derived from what
    // they are now, the CTA's first tiles are started towards L2 (the point of coherence, so a row that is still being written is not read too
    // early), and behind the wait the first copies go out under it at once; the lengths and the first row are read once more while those are on
    // their way, and only if the schedule is another one is it derived again.  (These reads bypass L1, which could keep the earlier value.)
    const int s_per = (n_slabs + kQdThreads - 1) / kQdThreads;
    const int s_lo = min(tid * s_per, n_slabs), s_hi = min(s_lo + s_per, n_slabs);
    auto length = [&](int s) { return min(max(__ldcg(kv_len + s), 0), q8_room(c, __ldcg(cap + s / Hk))); };
    auto slab_row = [&](int s) { return (long long)(__ldcg(reinterpret_cast<const long long*>(slab_off) + s / Hk) * Hk + (long long)(s % Hk) * __ldcg(cap + s / Hk)); };
    auto tiles = [](int rows) { return (rows + kQ8Tile - 1) / kQ8Tile; };
    if (kTable) {
        pdl_wait();
    } else {
#pragma unroll 1
        for (int s = s_lo; s < s_hi; ++s) lens[s] = length(s);
    }
    int T, Ge, t_begin, t_end, slab;
    auto derive = [&]() {
        if (!kTable) cta_prefix<kQdThreads>(n_slabs, [&](int s) { return lens[s] ? tiles(lens[s]) + kQdPartCost : 0; }, pref, s_wsum);
        T = pref[n_slabs];
        Ge = min(G, T);
        auto first_of = [&](int k) { return T < (1 << 22) ? int(uint32_t(k) * uint32_t(T) / uint32_t(Ge)) : int((long long)k * T / Ge); };
        t_begin = cta < Ge ? first_of(cta) : T;
        t_end = cta < Ge ? first_of(cta + 1) : T;
        slab = 0;                                         // slab holding place t_begin: the last one with pref <= t_begin
        if (kTable) {                                     // (two reads, not one for each halving)
            slab = max(__syncthreads_count(tid * s_per < n_slabs && pref[min(tid * s_per, n_slabs)] <= t_begin) - 1, 0) * s_per;
            slab += max(__syncthreads_count(tid < s_per && slab + tid < n_slabs && pref[min(slab + tid, n_slabs)] <= t_begin) - 1, 0);
        } else {
            int hi = n_slabs - 1;
            while (slab < hi) {
                const int mid = (slab + hi + 1) >> 1;
                if (pref[mid] <= t_begin) slab = mid; else hi = mid - 1;
            }
        }
        t_begin = max(t_begin, pref[slab] + kQdPartCost);
    };
    derive();
    // the slab that has place t, from one that ends at or before it on
    auto slab_at = [&](int s, int t) {
        if (!kTable) {
            while (pref[s + 1] <= t) ++s;
            return s;
        }
        if (pref[++s + 1] > t) return s;                  // (slabs without rows lie between)
        int step = 1;
        while (s + step < n_slabs && pref[s + step] <= t) { s += step; step *= 2; }
        for (; step; step >>= 1)
            if (s + step < n_slabs && pref[s + step] <= t) s += step;
        return s;
    };
    auto cta_of = [&](int place) {
        return T < (1 << 22) ? int((uint32_t(place + 1) * uint32_t(Ge) - 1u) / uint32_t(T)) : int(((long long)(place + 1) * Ge - 1) / T);
    };
    // first row of the first slab; paged: the page of the CTA's first tile
    auto first_row = [&]() {
        if (t_begin >= t_end) return 0ll;
        if (c.table) return (long long)__ldcg(c.table + size_t(slab) * c.max_pages + (t_begin - pref[slab] - kQdPartCost));
        return slab_row(slab);
    };
    long long row_first = first_row();
    if (!kTable && tid < 2 * kQdPrefetch && t_begin + (tid >> 1) < min(t_end, pref[slab + 1])) {
        const int t = t_begin + (tid >> 1), j = t - pref[slab] - kQdPartCost, rows = min(lens[slab] - j * kQ8Tile, kQ8Tile);
        const long long row = !c.table ? row_first + (long long)j * kQ8Tile
                                       : (t == t_begin ? row_first : (long long)__ldcg(c.table + size_t(slab) * c.max_pages + j)) * kQ8Tile;
        if (row >= 0 && row + rows <= c.rows) {
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(((tid & 1) ? c.V : c.K) + row * kQ8RowBytes), "r"(rows * kQ8RowBytes) : "memory");
            const size_t at = c.table ? size_t(row / kQ8Tile) * (kQ8Tile >> c.block_log2) : size_t(slab) * c.max_blocks + size_t(j) * (kQ8Tile >> c.block_log2);
            asm volatile("prefetch.global.L2 [%0];" ::"l"(((tid & 1) ? c.v_scale : c.k_scale) + at));
        }
    }
    // ---- copies: this warp's 32 rows of the CTA's k-th tile, and their scales, go to stage k % kQdStages.  The cursor walks the slab parts of
    // the range; divisions and the slab's tables are read once per part, a page's entry a tile ahead, and whole tiles take a short path.
    const uint32_t ring = smem_u32(dsm) + warp * kQdStages * kQdStageBytes;
    const int c_row = lane >> 3, c_col = lane & 7;
    const uint32_t dst0 = ring + c_row * kQ8RowBytes + ((c_col ^ c_row) << 4);        // row 4 i + c_row, i even; odd: ^ 64
    const float* const sp = (lane & 2) ? c.v_scale : c.k_scale;
    const uint32_t sp_dst = smem_u32(&s_scale[warp][0][lane & 3]);
    const int per_tile = kQ8Tile >> c.block_log2, sub = (warp * kQdRows + (lane & 1) * 16) >> c.block_log2;
    int p_t = t_begin, p_slab = slab, p_end = t_begin, p_stage = 0;
    int p_fast = 0;                                       // tiles ahead that are whole and, contiguous, inside the buffers
    int p_row0 = 0, p_page = 0;                           // contiguous: row of the slab's first token; paged: page of the next tile
    size_t p_off = 0;                                     // contiguous: where this lane's pieces of the next tile begin
    const float* p_sp = nullptr;                          // and the tile's scale
    const int32_t* p_table = c.table;
    const int pages = int(c.rows / kQ8Tile);
    const size_t lane_off = size_t(warp * kQdRows + c_row) * kQ8RowBytes + c_col * 16;
    const int all_scales = c.table ? 0x7fffffff : n_slabs * c.max_blocks;
    uint32_t inside = 0;                                  // a byte for each stage: how many of its rows the buffers have (0: nothing was copied)
    auto set_inside = [&](int rows) { inside = (inside & ~(0xffu << (8 * p_stage))) | (uint32_t(rows) << (8 * p_stage)); };
    bool far = false;                                     // rows were left out under the schedule from before the wait
    auto copy_rows = [&](size_t off, const float* scale) {
        const uint8_t *kp = c.K + off, *vp = c.V + off;
        const uint32_t to = dst0 + p_stage * kQdStageBytes;
#pragma unroll
        for (int i = 0; i < kQdRows / 4; ++i) {
            cp_async_piece((to ^ ((i & 1) << 6)) + i * 4 * kQ8RowBytes, kp + i * 4 * kQ8RowBytes);
            cp_async_piece((to ^ ((i & 1) << 6)) + (kQdRows + i * 4) * kQ8RowBytes, vp + i * 4 * kQ8RowBytes);
        }
        if (lane < 4) cp_async4(sp_dst + p_stage * 16, scale);
    };
    // the next slab part; false: there is none
    auto enter = [&]() {
        if (pref[p_slab + 1] <= p_t) p_slab = slab_at(p_slab, p_t);
        p_end = pref[p_slab + 1];
        p_t = max(p_t, pref[p_slab] + kQdPartCost);
        if (p_t >= t_end) { p_t = p_end = t_end; return false; }
        if (c.table) {
            p_table = c.table + size_t(p_slab) * c.max_pages + (p_t - pref[p_slab] - kQdPartCost);
            p_page = p_t == t_begin ? int(row_first) : __ldcg(p_table);
        } else {
            const long long row0 = p_t == t_begin ? row_first : slab_row(p_slab);
            p_row0 = int(row0 < 0 || row0 > c.rows ? c.rows : row0);
        }
        return true;
    };
    // the whole tiles from the slab's tile j = that at p_t on
    auto whole_tiles = [&](int j) {
        const int whole = lens[p_slab] / kQ8Tile;
        p_fast = !c.table && (long long)p_row0 + (long long)whole * kQ8Tile > c.rows ? 0 : min(min(p_end, t_end) - p_t, whole - j);
        if (!c.table) {
            p_off = size_t(uint32_t(p_row0)) * kQ8RowBytes + size_t(j) * (kQ8Tile * kQ8RowBytes) + lane_off;
            p_sp = sp + p_slab * c.max_blocks + j * per_tile + sub;
        }
    };
    // early: under the schedule from before the wait, with a length that may be old: all of the tile is copied
    auto issue_next = [&](bool early) {
        bool fast = p_fast > 0;
        if (c.table && uint32_t(p_page) >= uint32_t(pages)) fast = false;
        if (fast) {
            if (c.table) {
                copy_rows(size_t(p_page) * (kQ8Tile * kQ8RowBytes) + lane_off, sp + p_page * per_tile + sub);
                if (p_t + 1 < p_end) p_page = __ldcg(++p_table);
            } else {
                copy_rows(p_off, p_sp);
                p_off += kQ8Tile * kQ8RowBytes;
                p_sp += per_tile;
            }
            set_inside(kQdRows);
            --p_fast;
            ++p_t;
            if (++p_stage == kQdStages) p_stage = 0;
        } else if (p_t < t_end) {
            if (p_t == p_end && !enter()) { cp_async_commit(); return; }
            const int j = p_t - pref[p_slab] - kQdPartCost, left = lens[p_slab] - j * kQ8Tile, p_rows = left - warp * kQdRows;
            // (a page outside the pool: a row at which nothing lies; this warp's first row, at most the buffer's end)
            const int row = c.table ? (uint32_t(p_page) < uint32_t(pages) ? p_page * kQ8Tile + warp * kQdRows : int(c.rows))
                                    : int(min((long long)p_row0 + (long long)j * kQ8Tile + warp * kQdRows, c.rows));
            const int place = c.table ? (uint32_t(p_page) < uint32_t(pages) ? p_page * per_tile + sub : 0) : p_slab * c.max_blocks + j * per_tile + sub;
            if (c.table && p_t + 1 < p_end) p_page = __ldcg(++p_table);
            const int rows = early ? kQdRows : min(p_rows, kQdRows);
            const int have = rows > 0 ? min(int(c.rows) - row, kQdRows) : 0;
            const bool in = have >= min(p_rows, kQdRows);
            set_inside(have);
            if (have > 0) {
                // all 32 rows, also where the slab has fewer left: what follows them is not used (zeros behind the buffer)
                const size_t off = size_t(uint32_t(row + c_row)) * kQ8RowBytes + c_col * 16;
                const float* scale = sp + min(place, all_scales - 1);
                if (row + kQdRows <= int(c.rows)) {
                    copy_rows(off, scale);
                } else {
                    const uint32_t to = dst0 + p_stage * kQdStageBytes;
#pragma unroll 1
                    for (int i = 0; i < kQdRows / 4; ++i) {
                        const int bytes = row + c_row + 4 * i < int(c.rows) ? 16 : 0;
                        cp_async_piece((to ^ ((i & 1) << 6)) + i * 4 * kQ8RowBytes, bytes ? c.K + off + i * 4 * kQ8RowBytes : c.K, bytes);
                        cp_async_piece((to ^ ((i & 1) << 6)) + (kQdRows + i * 4) * kQ8RowBytes, bytes ? c.V + off + i * 4 * kQ8RowBytes : c.V, bytes);
                    }
                    if (lane < 4) cp_async4(sp_dst + p_stage * 16, scale);
                }
            }
            far = far || (early && !in);
            if (lane == 0 && !in && !early) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
            ++p_t;
            whole_tiles(j + 1);
            if (++p_stage == kQdStages) p_stage = 0;
        }
        cp_async_commit();                                // empty groups keep the count
    };
    const int g = lane >> 2, qd = lane & 3;               // mma fragments: rows (tokens, channels) g and g + 8, columns (heads) 2 qd and 2 qd + 1
    // Few heads: columns 2 h and 2 h + 1 belong to head h (high and low parts), so a lane has one head, qd; else column h to head h.
    const int hd = kFew ? g >> 1 : g;                     // head of this lane's column of the B operands
    uint32_t qa[16];                                      // bf16 pairs as they come; then the operand
    auto fetch_q = [&](int slab_) {                       // a slab's queries: channels 32 qd to 32 qd + 31 of head hd
        const uint4* qp = reinterpret_cast<const uint4*>(q + (size_t(slab_) * n + min(hd, n - 1)) * kHeadDim + qd * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = hd < n ? qp[i] : make_uint4(0u, 0u, 0u, 0u);
            qa[4 * i] = v.x; qa[4 * i + 1] = v.y; qa[4 * i + 2] = v.z; qa[4 * i + 3] = v.w;
        }
    };
    // The first copies' addresses are made ahead of the wait; what else comes from memory before the first tile is requested behind the first copies and
    // waited for behind the second ones.
    int q_slab = slab;
    if (t_begin < t_end && enter()) whole_tiles(p_t - pref[p_slab] - kQdPartCost);
    if (!kTable) pdl_wait();
    issue_next(!kTable);
    if (t_begin < t_end) fetch_q(slab);
    // the same for what the schedule was made of (as it comes: what is made of it waits for it)
    const bool mine = !kTable && s_lo < s_hi, work = !kTable && t_begin < t_end;
    const int len_again = mine ? __ldcg(kv_len + s_lo) : 0, room_again = mine ? __ldcg(cap + s_lo / Hk) : 0;
    const int page_again = work && c.table ? __ldcg(c.table + size_t(slab) * c.max_pages + (t_begin - pref[slab] - kQdPartCost)) : 0;
    const long long off_again = work && !c.table ? __ldcg(reinterpret_cast<const long long*>(slab_off) + slab / Hk) : 0;
    const int cap_again = work && !c.table ? __ldcg(cap + slab / Hk) : 0;
#pragma unroll 1
    for (int attempt = kTable ? 1 : 0;; ++attempt) {
#pragma unroll 1
        for (int k = kTable || attempt == 0; k < kQdStages - 1; ++k) issue_next(attempt == 0);
        if (attempt) break;
        int changed = far || (work && row_first != (c.table ? (long long)page_again : off_again * Hk + (long long)(slab % Hk) * cap_again));
#pragma unroll 1
        for (int s = s_lo; s < s_hi; ++s) {
            const int now = s == s_lo ? min(max(len_again, 0), q8_room(c, room_again)) : length(s);
            if (now == lens[s]) continue;
            // (a slab that now reaches beyond the buffer is left to the checks of the second attempt)
            if (tiles(now) != tiles(lens[s]) || (!c.table && (long long)slab_row0(slab_off, cap, Hk, s / Hk, s % Hk) + now > c.rows)) changed = 1;
            lens[s] = now;
        }
        if (!__syncthreads_or(changed)) break;
        // another schedule: what is on its way is waited for, and its place used anew
        cp_async_wait<0>();
        derive();
        row_first = first_row();
        p_t = p_end = t_begin; p_slab = slab; p_stage = p_fast = 0;
        q_slab = -1;
    }
    pdl_trigger();

    {
        const int side0 = (warp * G + cta) * 32 + lane, side_step = G * kQdThreads;
        const int vec_per_row = d_model / 8, steer_total = hidden != nullptr ? batch * vec_per_row : 0;
#pragma unroll 1
        for (int i = side0; i < steer_total; i += side_step)
            steer_store(i, vec_per_row, hidden, steer_load(i, vec_per_row, hidden, steer_vec, alpha, flag));
    }

    // The B operand of S = K Q^T, times 2^shift; unshift takes the heads of the accumulator's columns back.
    //  int8 (codes as f16): step i has channels 32 qd + 4 i + {0, 1} in qa[2 i] and {2, 3} in qa[2 i + 1], the largest magnitude in
    //  [2^14, 2^15), so the 8 bits are whole from 2^-17 on, 2^-31 of it, and smaller ones off by 2^-25; few heads: even columns only.
    //  e4m3 (codes as they are): the largest magnitude in [2^7, 2^8) and two e4m3 parts, high and 2^5 times the rest, together the 8 bits of
    //  every bf16 from 2^-7 on, 2^-14 of the head's largest at most.  (A smaller one goes to the next multiple of 2^-14, the last place of the low part:
    //  off by up to 2^-15, 2^-22 of the largest.  A third part would be a third product of every tile.)  Step i has channels 32 qd + 8 i + {0 to 3} in
    //  qa[2 i] and {4 to 7} in qa[2 i + 1]; low parts in odd columns (few heads) or in q_lo.
    float2 unshift = make_float2(1.f, 1.f);
    uint32_t q_lo[8];
    auto shift_q = [&]() {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = __vmaxu2(m, qa[i] & 0x7fff7fffu);
        m = max(m & 0xffffu, m >> 16);
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const int field = min(max((kFmt == SKIPKV_Q8_E4M3 ? 261 : 268) - int(m >> 7), 1), 253);       // exponent field of 2^shift
        const float up = __uint_as_float(uint32_t(field) << 23);
        if (kFmt == SKIPKV_Q8_E4M3) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // (as f16 the values have the bits that the two parts take)
                const float2 v0 = bf16x2_to_f2(qa[2 * i]), v1 = bf16x2_to_f2(qa[2 * i + 1]);
                const uint32_t y0 = pack_f16(v0.x * up, v0.y * up), y1 = pack_f16(v1.x * up, v1.y * up), hi = f16_to_e4m3(y0, y1);
                uint32_t h0, h1;
                q8_to_f16<SKIPKV_Q8_E4M3>(hi, h0, h1);
                const uint32_t lo = f16_to_e4m3(rest32(y0, h0), rest32(y1, h1));
                if (kFew) {
                    qa[i] = (g & 1) ? lo : hi;
                } else {
                    qa[i] = hi;                           // (qa[2 i] and qa[2 i + 1] have been read)
                    q_lo[i] = lo;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 v = bf16x2_to_f2(qa[i]);
                qa[i] = kFew && (g & 1) ? 0u : pack_f16(v.x * up, v.y * up);
            }
        }
        // (an infinity or a NaN in a head makes its logits NaN, as its products would)
        const float down = __uint_as_float(m < 0x7f80u ? uint32_t(254 - field) << 23 : 0x7fffffffu);
        unshift = make_float2(__shfl_sync(0xffffffffu, down, 8 * qd), __shfl_sync(0xffffffffu, down, 8 * qd + 4));
    };

    const float qscale = 1.4426950408889634f * rsqrtf(float(kHeadDim));
    // this lane's 16-byte pieces in a stage: pieces 2 qd and 2 qd + 1 (^ 16) of key rows g and g + 8; piece g of value rows 2 qd, 2 qd + 1 and 8 more
    const uint32_t k_at = ring + g * kQ8RowBytes + (((2 * qd) ^ g) << 4);
    const uint32_t v_at = ring + (kQdRows + 2 * qd) * kQ8RowBytes + ((g ^ (2 * qd)) << 4);
    const uint32_t v_at1 = (v_at ^ 16u) + kQ8RowBytes;

    int c_stage = 0;
    // a warp's sums of a segment lie in the stage of its last tile
    auto sums = [&](int w) { return reinterpret_cast<float*>(dsm + (size_t(w) * kQdStages + (c_stage == 0 ? kQdStages - 1 : c_stage - 1)) * kQdStageBytes); };
    int t = t_begin;
    // The slab whose part this CTA has delivered, and the answer to its arrival, which nothing waits for before the next part is worked on.
    int pend = -1, pend_parts = 0, pend_cta = 0;
    uint32_t pend_old = 0;
    while (true) {
        // -------------------------------------------------------------- one (CTA, slab) segment
        if (t < t_end && pref[slab + 1] <= t) slab = slab_at(slab, t);
        if (t < t_end) t = max(t, pref[slab] + kQdPartCost);
        const bool more = t < t_end;
        if (!more && pend < 0) break;
        int n_part = 0, first_cta = 0;
        if (more) {
        const int seg_end = min(t_end, pref[slab + 1]);
        first_cta = cta_of(pref[slab] + kQdPartCost);
        n_part = cta_of(pref[slab + 1] - 1) - first_cta + 1;
        if (slab != q_slab) { fetch_q(slab); q_slab = slab; }
        shift_q();
        q_slab = -1;
        if (kTable && seg_end < t_end && warp == 0 && lane < 2 * n && slab + 1 < n_slabs)      // the next slab's queries: 8192 slabs of 100 rows 129 -> 124 us
            asm volatile("prefetch.global.L1 [%0];" ::"l"(q + (size_t(slab + 1) * n * kHeadDim + lane * 64)));
        float2 acc[8][2];                                 // channels 16 g + 2 j and 16 g + 2 j + 1 of the lane's two columns
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j][0] = acc[j][1] = make_float2(0.f, 0.f);
        float2 m = make_float2(-INFINITY, -INFINITY), l = make_float2(0.f, 0.f);    // their running maximum, this lane's share of the sum
        int rows_left = lens[slab] - (t - pref[slab] - kQdPartCost) * kQ8Tile - warp * kQdRows;     // of this warp's part of the tile
#pragma unroll 1
        for (; t < seg_end; ++t, rows_left -= kQ8Tile) {
            cp_async_wait<kQdStages - 2>();
            __syncwarp();                                 // every lane's pieces have landed; the stage before is read out
            const int rows = min(rows_left, int((inside >> (8 * c_stage)) & 0xffu));       // that this warp has of the tile
            issue_next(false);
            if (rows > 0) {
                const uint32_t so = c_stage * kQdStageBytes;
                const float4 scales = *reinterpret_cast<const float4*>(s_scale[warp][c_stage]);
                const bool two = rows > 16;               // the second group has rows
                float s[2][2][4];                         // per group: two chains (int8), high and low parts (e4m3, many heads), one (few)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const uint32_t at = ((k_at + so) ^ (half << 4)) + u * 16 * kQ8RowBytes;
                        const uint4 k0 = lds128(at), k1 = lds128(at + 8 * kQ8RowBytes);
                        const uint32_t lo[4] = {k0.x, k0.y, k0.z, k0.w}, hi[4] = {k1.x, k1.y, k1.z, k1.w};
                        if (kFmt == SKIPKV_Q8_E4M3) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int k = 2 * half + i;
                                if (k == 0) mma16832q_first(s[u][0], lo[0], hi[0], lo[1], hi[1], qa[0], qa[1]);
                                else        mma16832q(s[u][0], lo[2 * i], hi[2 * i], lo[2 * i + 1], hi[2 * i + 1], qa[2 * k], qa[2 * k + 1]);
                                if (kFew) continue;
                                if (k == 0) mma16832q_first(s[u][1], lo[0], hi[0], lo[1], hi[1], q_lo[0], q_lo[1]);
                                else        mma16832q(s[u][1], lo[2 * i], hi[2 * i], lo[2 * i + 1], hi[2 * i + 1], q_lo[2 * k], q_lo[2 * k + 1]);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint32_t a0, a1, a2, a3;
                                q8_to_f16<kFmt>(lo[i], a0, a2);
                                q8_to_f16<kFmt>(hi[i], a1, a3);
                                const int k = 4 * half + i;
                                if (k < 2) mma16816h_first(s[u][i & 1], a0, a1, a2, a3, qa[2 * k], qa[2 * k + 1]);
                                else       mma16816h(s[u][i & 1], a0, a1, a2, a3, qa[2 * k], qa[2 * k + 1]);
                            }
                        }
                    }
                uint4 v[2][4];                            // value rows 2 qd, 2 qd + 1, 2 qd + 8, 2 qd + 9 of each group
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    v[u][0] = lds128(v_at + so + u * 16 * kQ8RowBytes); v[u][1] = lds128(v_at1 + so + u * 16 * kQ8RowBytes);
                    v[u][2] = lds128(v_at + so + (u * 16 + 8) * kQ8RowBytes); v[u][3] = lds128(v_at1 + so + (u * 16 + 8) * kQ8RowBytes);
                }
                uint32_t ph[2][2], pl[2][2];              // P^T as B operands: (few) high parts in even and low ones in odd columns, else apart
                if (kFew) {
                    // this lane's logits: tokens g and g + 8 of either group, head qd
                    float x[2][2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float f = qscale * (u ? scales.y : scales.x) * unshift.x;
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            x[u][r] = f * (kFmt == SKIPKV_Q8_E4M3 ? fmaf(s[u][0][2 * r + 1], 0.03125f, s[u][0][2 * r]) : s[u][0][2 * r] + s[u][1][2 * r]);
                    }
                    if (rows < kQdRows) {                 // the end of the slab: rows behind it hold anything, NaN too
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int r = 0; r < 2; ++r)
                                if (16 * u + 8 * r + g >= rows) x[u][r] = -INFINITY;
                    }
                    float top = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1]));
                    if (__any_sync(0xffffffffu, top > m.x)) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        top = fmaxf(top, m.x);
                        const float sc = ex2(m.x - top);  // first rows: 2^(-inf) = 0
                        l.x *= sc;
                        m.x = top;
                        const float2 sc2 = make_float2(sc, sc);
#pragma unroll
                        for (int j = 0; j < 8; ++j) { acc[j][0] = __fmul2_rn(acc[j][0], sc2); acc[j][1] = __fmul2_rn(acc[j][1], sc2); }
                    }
                    const float neg = 15.f - m.x;         // 2^15 p
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
#pragma unroll
                        for (int r = 0; r < 2; ++r) x[u][r] = ex2(x[u][r] + neg);
                        const float2 hi = f16x2_to_f2(pack_f16(x[u][0], x[u][1]));
                        ph[u][0] = movmatrix_trans(pack_f16(x[u][0], x[u][0] - hi.x));
                        ph[u][1] = movmatrix_trans(pack_f16(x[u][1], x[u][1] - hi.y));
                    }
                    l.x += (x[0][0] + x[0][1]) + (x[1][0] + x[1][1]);
                } else {
                    // the same for heads 2 qd and 2 qd + 1 (packed fp32 arithmetic: the two heads per instruction)
                    float2 x[2], y[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float f = qscale * (u ? scales.y : scales.x);
                        const float2 f2 = make_float2(f * unshift.x, f * unshift.y);
                        const float2 a = make_float2(s[u][0][0], s[u][0][1]), b = make_float2(s[u][0][2], s[u][0][3]);
                        const float2 a1 = make_float2(s[u][1][0], s[u][1][1]), b1 = make_float2(s[u][1][2], s[u][1][3]);
                        const float part = kFmt == SKIPKV_Q8_E4M3 ? 0.03125f : 1.f;
                        x[u] = __fmul2_rn(__ffma2_rn(a1, make_float2(part, part), a), f2);
                        y[u] = __fmul2_rn(__ffma2_rn(b1, make_float2(part, part), b), f2);
                    }
                    if (rows < kQdRows) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            if (16 * u + g >= rows) x[u] = make_float2(-INFINITY, -INFINITY);
                            if (16 * u + 8 + g >= rows) y[u] = make_float2(-INFINITY, -INFINITY);
                        }
                    }
                    float2 top = make_float2(fmaxf(fmaxf(x[0].x, y[0].x), fmaxf(x[1].x, y[1].x)), fmaxf(fmaxf(x[0].y, y[0].y), fmaxf(x[1].y, y[1].y)));
                    if (__any_sync(0xffffffffu, top.x > m.x || top.y > m.y)) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) {
                            top.x = fmaxf(top.x, __shfl_xor_sync(0xffffffffu, top.x, d));
                            top.y = fmaxf(top.y, __shfl_xor_sync(0xffffffffu, top.y, d));
                        }
                        top = make_float2(fmaxf(top.x, m.x), fmaxf(top.y, m.y));
                        const float2 sc = make_float2(ex2(m.x - top.x), ex2(m.y - top.y));
                        l = __fmul2_rn(l, sc);
#pragma unroll
                        for (int j = 0; j < 8; ++j) { acc[j][0] = __fmul2_rn(acc[j][0], sc); acc[j][1] = __fmul2_rn(acc[j][1], sc); }
                        m = top;
                    }
                    const float2 neg = make_float2(15.f - m.x, 15.f - m.y);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        x[u] = __fadd2_rn(x[u], neg); y[u] = __fadd2_rn(y[u], neg);
                        x[u] = make_float2(ex2(x[u].x), ex2(x[u].y)); y[u] = make_float2(ex2(y[u].x), ex2(y[u].y));
                        uint32_t hx, lx, hy, ly;
                        split_f16(x[u], hx, lx);
                        split_f16(y[u], hy, ly);
                        ph[u][0] = movmatrix_trans(hx); ph[u][1] = movmatrix_trans(hy);
                        pl[u][0] = movmatrix_trans(lx); pl[u][1] = movmatrix_trans(ly);
                    }
                    l = __fadd2_rn(l, __fadd2_rn(__fadd2_rn(x[0], y[0]), __fadd2_rn(x[1], y[1])));
                }
                if (rows < kQdRows) {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (16 * u + 2 * qd + (k & 1) + (k >> 1) * 8 >= rows) v[u][k] = make_uint4(0u, 0u, 0u, 0u);
                }
                // (the 2^15 of the probabilities comes off here, before the sums, whose range is that of 32 bits then)
                const float vs0 = scales.z * kQdUnit, vs1 = two ? scales.w * kQdUnit : 0.f;
                const float2 vs2[2] = {make_float2(vs0, vs0), make_float2(vs1, vs1)};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    auto word = [&](int u, int k) { return w == 0 ? v[u][k].x : w == 1 ? v[u][k].y : w == 2 ? v[u][k].z : v[u][k].w; };
#pragma unroll
                    for (int half = 0; half < 2; ++half) {     // channels 16 g + 4 w + 2 half and the next; tokens 2 qd, 2 qd + 1 and 8 more
                        const uint32_t pick = half ? 0x7362u : 0x5140u;
                        const int j = 2 * w + half;
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            uint32_t a0, a1, a2, a3;
                            q8_to_f16<kFmt>(__byte_perm(word(u, 0), word(u, 1), pick), a0, a1);
                            q8_to_f16<kFmt>(__byte_perm(word(u, 2), word(u, 3), pick), a2, a3);
                            float d[4];
                            mma16816h_first(d, a0, a1, a2, a3, ph[u][0], ph[u][1]);
                            if (!kFew) mma16816h(d, a0, a1, a2, a3, pl[u][0], pl[u][1]);
                            acc[j][0] = __ffma2_rn(make_float2(d[0], d[1]), vs2[u], acc[j][0]);
                            acc[j][1] = __ffma2_rn(make_float2(d[2], d[3]), vs2[u], acc[j][1]);
                        }
                    }
                }
            }
            if (++c_stage == kQdStages) c_stage = 0;
        }

        // -------------------------------------------------------------- the end of a segment
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l.x += __shfl_xor_sync(0xffffffffu, l.x, d);
            l.y += __shfl_xor_sync(0xffffffffu, l.y, d);
        }
        l.x *= kQdUnit; l.y *= kQdUnit;
        // The heads' sums go to the stage of the tile that was worked on last: its rows are read out, and the next copy into it is issued behind
        // the barriers below.
        if (kFew) {
            float4* wp = reinterpret_cast<float4*>(sums(warp) + size_t(qd) * kQdSumStride + 16 * g);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                wp[j] = make_float4(acc[2 * j][0].x + acc[2 * j][0].y, acc[2 * j][1].x + acc[2 * j][1].y, acc[2 * j + 1][0].x + acc[2 * j + 1][0].y,
                                    acc[2 * j + 1][1].x + acc[2 * j + 1][1].y);
            if (g == 0) s_ml[warp][qd] = make_float2(m.x, l.x);
        } else {
            float* wp = sums(warp) + size_t(2 * qd) * kQdSumStride + 16 * g;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                reinterpret_cast<float4*>(wp)[j] = make_float4(acc[2 * j][0].x, acc[2 * j][1].x, acc[2 * j + 1][0].x, acc[2 * j + 1][1].x);
                reinterpret_cast<float4*>(wp + kQdSumStride)[j] = make_float4(acc[2 * j][0].y, acc[2 * j][1].y, acc[2 * j + 1][0].y, acc[2 * j + 1][1].y);
            }
            if (g == 0) { s_ml[warp][2 * qd] = make_float2(m.x, l.x); s_ml[warp][2 * qd + 1] = make_float2(m.y, l.y); }
        }
        }
        if (pend >= 0 && tid == 0) {
            const int last = pend_old == uint32_t(pend_parts - 1) ? 1 : 0;
            if (last) dec_cnt[pend] = 0u;                 // self-resetting for the next launch
            s_last = last;
        }
        __syncthreads();
        const bool last = pend >= 0 && s_last;
        const int done = pend, done_parts = pend_parts, done_cta = pend_cta;
        pend = -1;
        if (more) {
            // merge the warps; thread -> channel
            __nv_bfloat16* o = out + size_t(slab) * n * kHeadDim;
            float* rec = dec_part + size_t(cta + slab) * n * kDecPartStride;
#pragma unroll
            for (int hl = 0; hl < (kFew ? 4 : kMaxGroup); ++hl) {
                if (hl >= n) break;
                float M = kQdLeast, L = 0.f, A = 0.f;     // (finite: a warp without rows has -inf)
#pragma unroll
                for (int w = 0; w < kQdWarps; ++w) M = fmaxf(M, s_ml[w][hl].x);
#pragma unroll
                for (int w = 0; w < kQdWarps; ++w) {
                    const float2 ml = s_ml[w][hl];
                    const float e = ex2(ml.x - M);
                    L = fmaf(ml.y, e, L);
                    A = fmaf(sums(w)[hl * kQdSumStride + tid], e, A);
                }
                if (n_part == 1) {
                    o[hl * kHeadDim + tid] = __float2bfloat16_rn(L == 0.f ? 0.f : A / L);
                } else {
                    rec[hl * kDecPartStride + tid] = A;
                    if (tid == 0) *reinterpret_cast<float2*>(rec + hl * kDecPartStride + kHeadDim) = make_float2(M, L);
                }
            }
            __syncthreads();                              // every thread's record stores are ordered before the arrival; the sums are read
            if (n_part > 1) {
                pend = slab;
                pend_parts = n_part;
                pend_cta = first_cta;
                if (tid == 0) pend_old = arrive_acq_rel(dec_cnt + slab);
            }
        }
        if (last) {
            // This CTA was the last to deliver a part of slab `done`: a warp takes a head, a lane a partial for the weights (maximum, sum) and four
            // channels for the sums; the loads of 16 partials are on their way at once (into registers; by way of shared memory: 7.9 us for one sequence of
            // 2K against 7.4).
            const float* r0 = dec_part + size_t(done_cta + done) * n * kDecPartStride;
            const size_t stride = size_t(n) * kDecPartStride;
#pragma unroll 1
            for (int hl = warp; hl < n; hl += kQdWarps) {
                const float* rh = r0 + hl * kDecPartStride;
                float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
                float M = kQdLeast, L = 0.f;
#pragma unroll 1
                for (int p0 = 0; p0 < done_parts; p0 += kQdMergeParts) {
                    const int cnt = min(kQdMergeParts, done_parts - p0);
                    const bool on = lane < cnt;
                    const float2 ml = __ldcg(reinterpret_cast<const float2*>(rh + size_t(p0 + min(lane, cnt - 1)) * stride + kHeadDim));
                    float4 part[kQdMergeParts];
#pragma unroll
                    for (int k = 0; k < kQdMergeParts; ++k)
                        part[k] = k < cnt ? __ldcg(reinterpret_cast<const float4*>(rh + size_t(p0 + k) * stride) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
                    float mx = on ? ml.x : -INFINITY;
#pragma unroll
                    for (int d = kQdMergeParts / 2; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    mx = __shfl_sync(0xffffffffu, mx, 0);
                    const float Mn = fmaxf(M, mx), keep = ex2(M - Mn);
                    const float w = on ? ex2(ml.x - Mn) : 0.f;
                    float ls = on ? ml.y * w : 0.f;
#pragma unroll
                    for (int d = kQdMergeParts / 2; d; d >>= 1) ls += __shfl_xor_sync(0xffffffffu, ls, d);
                    L = fmaf(L, keep, __shfl_sync(0xffffffffu, ls, 0));
                    M = Mn;
                    A.x *= keep; A.y *= keep; A.z *= keep; A.w *= keep;
#pragma unroll
                    for (int k = 0; k < kQdMergeParts; ++k) {
                        const float wk = __shfl_sync(0xffffffffu, w, k);
                        A.x = fmaf(part[k].x, wk, A.x); A.y = fmaf(part[k].y, wk, A.y);
                        A.z = fmaf(part[k].z, wk, A.z); A.w = fmaf(part[k].w, wk, A.w);
                    }
                }
                const float inv = L == 0.f ? 0.f : 1.f / L;
                __nv_bfloat162* oi = reinterpret_cast<__nv_bfloat162*>(out + (size_t(done) * n + hl) * kHeadDim + lane * 4);
                oi[0] = __floats2bfloat162_rn(A.x * inv, A.y * inv);
                oi[1] = __floats2bfloat162_rn(A.z * inv, A.w * inv);
            }
        }
    }
    cp_async_wait<0>();
    // slabs with no row to attend to: zeros (owned round-robin)
#pragma unroll 1
    for (int k = 0; cta + G * k < n_slabs; k += 32) {
        const int mine = cta + G * (k + lane);
        uint32_t empty = __ballot_sync(0xffffffffu, mine < n_slabs && lens[min(mine, n_slabs - 1)] == 0);
#pragma unroll 1
        for (; empty; empty &= empty - 1) {
            __nv_bfloat16* o = out + size_t(cta + G * (k + __ffs(int(empty)) - 1)) * n * kHeadDim;
#pragma unroll 1
            for (int i = tid; i < n * kHeadDim; i += kQdThreads) o[i] = __float2bfloat16_rn(0.f);
        }
    }
}

}  // namespace skipkv

using namespace skipkv;

extern "C" int skipkv_decode_attn_q8(const skipkv_shape* shape, const skipkv_q8_cache* cache, const void* q, const int32_t* kv_len,
                                     void* out, void* hidden, const void* steer_vec, const float* alpha, const uint8_t* flag, void* ws,
                                     void* stream) {
    if (int rc = check_shape(shape)) return rc;
    if (int rc = check_q8(shape, cache)) return rc;
    if (!q || !kv_len || !out) return SKIPKV_ERR_INVALID_ARG;
    if (hidden && (!steer_vec || !alpha || !flag || shape->d_model <= 0)) return SKIPKV_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return SKIPKV_ERR_WORKSPACE;
    if ((reinterpret_cast<uintptr_t>(q) & 15) || (reinterpret_cast<uintptr_t>(out) & 3)) return SKIPKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(hidden) | reinterpret_cast<uintptr_t>(steer_vec)) & 15) return SKIPKV_ERR_INVALID_ARG;
    const WsLayout L = make_layout(*shape);
    uint8_t* w = static_cast<uint8_t*>(ws);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool table = L.slabs >= kQdTableSlabs;
    int* slab_table = reinterpret_cast<int*>(w + L.slab_table);
    if (table) {
        const QdSlabs slabs{q8_view(*cache), kv_len, shape->cap, int(shape->n_kv_heads), slab_table + L.slabs + 1};
        SKIPKV_CUDA(launch_dependent(q8_table_kernel<QdSlabs>, dim3(1), dim3(kQ8TableThreads), 0, st, int(L.slabs), slabs, slab_table));
    }
    const size_t smem = size_t(kQdRingBytes) + (table ? 0 : size_t(2 * L.slabs + 1) * 4);
    const int grid = 2 * num_sms() < kQdMaxGrid ? 2 * num_sms() : kQdMaxGrid;
    auto run = [&](auto kernel) {
        return launch_dependent(kernel, dim3(grid), dim3(kQdThreads), smem, st, int(shape->batch), int(shape->n_q_heads), int(shape->n_kv_heads),
                                int(L.slabs), shape->slab_off, shape->cap, static_cast<const __nv_bfloat16*>(q), q8_view(*cache), kv_len,
                                static_cast<__nv_bfloat16*>(out), &reinterpret_cast<Header*>(w + L.header)->status,
                                reinterpret_cast<uint32_t*>(w + L.dec_cnt), reinterpret_cast<float*>(w + L.dec_part), int(shape->d_model),
                                static_cast<__nv_bfloat16*>(hidden), static_cast<const __nv_bfloat16*>(steer_vec), alpha, flag, slab_table);
    };
    auto pick = [&](auto fmt) {
        constexpr int kFmt = decltype(fmt)::value;
        if (L.group <= 4) return table ? run(decode_q8_kernel<kFmt, true, true>) : run(decode_q8_kernel<kFmt, true, false>);
        return table ? run(decode_q8_kernel<kFmt, false, true>) : run(decode_q8_kernel<kFmt, false, false>);
    };
    SKIPKV_CUDA(cache->format == SKIPKV_Q8_E4M3 ? pick(std::integral_constant<int, SKIPKV_Q8_E4M3>()) : pick(std::integral_constant<int, SKIPKV_Q8_INT8>()));
    return SKIPKV_OK;
}
