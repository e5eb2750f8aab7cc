// Storing bf16 rows in 8 bits (skipkv_pack_q8, skipkv_append_q8, skipkv_append_step_q8) and getting them back (skipkv_unpack_q8).
//
// A block of block_rows tokens of a (sequence, head) slab shares the scale s = 2^e, e the least with amax <= top * 2^e (top 448 or
// 127): with a = f * 2^x, 1 <= f < 2, that is e = x - 8 for f <= 1.75 and x - 7 above (e4m3: 448 = 1.75 * 2^8), x - 6 for
// f <= 127/64 and x - 5 above (int8).  Both follow from the bits of the largest bf16 magnitude alone; x / s is exact in fp32, so a code is
// rounded once.  Powers of two, although int8 gives away half a bit of its range on average: codes that are rounded again under a
// larger scale (a block that grows, a cache that is packed again after a compaction) then stay what one rounding gives but for ties
// and what falls below the new spacing, and e4m3 loses nothing by them.
//
// The calls are bound by DRAM: 256 bytes read and 128 written per row and tensor (the other way round for loading).  Work = tiles of 128
// tokens of one slab and tensor, aligned to 128 tokens of the slab, so a block is never shared by two CTAs; all slabs' tiles are
// enumerated from the lengths on the GPU (ragged lengths cost nothing), K and V in turn.  A warp takes 16 rows, 16 lanes to a row (16 bytes of bf16,
// 8 bytes of codes each), all its loads in flight together; maxima meet in shared memory where a block has more than 16 rows.
#include <type_traits>

#include "common.cuh"
#include "q8.cuh"

namespace skipkv {

constexpr int kQsThreads = 256;
constexpr int kQsWarps = kQsThreads / 32;
static_assert(kQsWarps * 16 == kQ8Tile, "a warp takes 16 rows of a tile");
constexpr int kQsTableSlabs = 2048;           // from so many slabs on their table has a launch of its own: storing 1024 slabs of 300 rows 45.2 us with it and
                                              // 42.9 without, 2048 of 1000 rows 256.5 and 256.9

// Where the rows come from, and what else a decode step writes.
struct StoreArgs {
    const uint4* k_src;          // pack: slabs of bf16 rows; append: [n_new][Hk][16]
    const uint4* v_src;
    long long src_rows;          // pack: rows of the bf16 buffers
    const int32_t* new_off;      // append of several rows: [batch + 1]
    int n_new;
    const int32_t* len_in;       // pack: rows to store; append: rows already there
    int32_t* len_out;            // append
    // the decode step (n_sent == nullptr: none of it)
    int32_t* sent_off;
    int32_t* sent_id;
    int32_t* n_sent;
    const uint8_t* new_sent;
    const int32_t* gen_id;
    uint4* q_win;
    const uint4* q;
    int Hq, window, slot, max_sent;
};

// The slab that holds tile t: the last one with pref <= t; not before slab lo.
__device__ __forceinline__ int slab_of(const int* pref, int n_slabs, int t, int lo) {
    if (pref[lo + 1] > t) return lo;
    int hi = n_slabs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (pref[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// A CTA's tiles of T: every G-th, so that neighbouring CTAs work on neighbouring rows, or, where there are few, the CTA's own contiguous share,
// which has fewer slabs to find.  80 slabs of 16K to 32K: storing 240 us against 248 with contiguous shares, loading 260 against 266; loading the keys
// of 80 slabs of 2.1K: 16.2 with contiguous shares against 17.0.
struct Share {
    int first, end, step;
    __device__ __forceinline__ Share(int T, int cta, int G) {
        const bool few = T < 4 * G;
        first = few ? int((long long)T * cta / G) : cta;
        end = few ? int((long long)T * (cta + 1) / G) : T;
        step = few ? 1 : G;
    }
};

// Eight bf16 values times inv (a power of two) to codes.
template <int kFmt>
__device__ __forceinline__ uint2 codes8(const uint4& x, float inv) {
    const float2 k = make_float2(inv, inv), v0 = bf16x2_to_f2(x.x), v1 = bf16x2_to_f2(x.y), v2 = bf16x2_to_f2(x.z), v3 = bf16x2_to_f2(x.w);
    if (kFmt == SKIPKV_Q8_INT8) return make_uint2(q8_round_scaled(v0, v1, k), q8_round_scaled(v2, v3, k));
    const float2 y0 = __fmul2_rn(v0, k), y1 = __fmul2_rn(v1, k), y2 = __fmul2_rn(v2, k), y3 = __fmul2_rn(v3, k);
    return make_uint2(q8_round<kFmt>(y0.x, y0.y, y1.x, y1.y), q8_round<kFmt>(y2.x, y2.y, y3.x, y3.y));
}

// Exponent of the scale that the magnitude with these (finite) bf16 bits needs.
template <int kFmt>
__device__ __forceinline__ int scale_exp(uint32_t bits) {
    const int x = int(bits >> 7) - 127, f = int(bits & 127u);
    const int e = kFmt == SKIPKV_Q8_E4M3 ? x - 8 + (f > 96) : x - 6 + (f > 126);
    return max(e, kQ8LeastExp);
}

// Two bf16 values with 0 in the place of a NaN; fin: the largest magnitude of the finite ones.
__device__ __forceinline__ uint32_t without_nan(uint32_t w, uint32_t& fin) {
    uint32_t h[2] = {w & 0xffffu, w >> 16};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if ((h[u] & 0x7fffu) > 0x7f80u) h[u] = 0u;
        if ((h[u] & 0x7fffu) < 0x7f80u) fin = max(fin, h[u] & 0x7fffu);
    }
    return h[0] | (h[1] << 16);
}
// int8: four values, infinities among them, times inv to codes: an infinity to the largest code of its sign (e4m3 saturates by itself).  It is held to
// that behind the scaling, not before it: 127 times the largest scale, 2^122, is no number of 32 bits.
__device__ __forceinline__ uint32_t codes4_wild(const uint2& x, float inv) {
    auto held = [&](float v) { return fminf(fmaxf(v * inv, -127.f), 127.f); };
    const float2 v0 = bf16x2_to_f2(x.x), v1 = bf16x2_to_f2(x.y);
    return q8_round<SKIPKV_Q8_INT8>(held(v0.x), held(v0.y), held(v1.x), held(v1.y));
}
// Exponent of a scale that a block has: one that is no power of two goes to the next.
__device__ __forceinline__ int held_exp(float s) {
    const uint32_t bits = __float_as_uint(fminf(fmaxf(s, pow2f(kQ8LeastExp)), pow2f(122)));
    return int(bits >> 23) - 127 + ((bits & 0x7fffffu) != 0u);
}

// What a slab is to get: old rows that it has, now rows afterwards, row0 its first row in a contiguous layout.
struct Span { int old, now, row0; bool bad; };
template <bool kAppend>
struct StoreSlabs {
    struct Raw { int lo, hi, len, cap; int64_t off; };
    Q8View c;
    const int64_t* slab_off;
    const int32_t *cap, *new_off, *len_in;
    int32_t* len_out;
    uint32_t* status;
    int n_new, Hk;
    __device__ __forceinline__ Raw load(int s) const {
        const int b = s / Hk;
        return {kAppend ? new_off[b] : 0, kAppend ? new_off[b + 1] : 0, len_in[s], cap[b], slab_off[b]};
    }
    __device__ __forceinline__ Span span(int s, const Raw& r) const {
        Span x;
        x.row0 = q8_row0(r.off, r.cap, Hk, s);
        if (kAppend) {
            x.old = r.len;
            x.bad = r.len < 0 || r.lo < 0 || r.hi < r.lo || r.hi > n_new || (long long)r.len + (r.hi - r.lo) > q8_room_inside(c, r.cap, x.row0);
            x.now = x.bad ? r.len : r.len + (r.hi - r.lo);
        } else {
            x.old = 0;
            x.bad = r.len < 0 || r.len > r.cap || r.len > q8_room_inside(c, r.cap, x.row0);
            x.now = x.bad ? 0 : r.len;
        }
        return x;
    }
    static __device__ __forceinline__ int tiles(int old, int now) { return now > old ? (now - 1) / kQ8Tile - old / kQ8Tile + 1 : 0; }
    __device__ __forceinline__ int count(int s, const Raw& r) const {                  // (q8_table_kernel)
        const Span x = span(s, r);
        if (x.bad) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
        if (kAppend) len_out[s] = x.now;
        return tiles(x.old, x.now);
    }
};

// kTable: many slabs, whose tile prefix the launch ahead has made.
template <int kFmt, bool kAppend, bool kTable>
__global__ void __launch_bounds__(kQsThreads, 4)
q8_store_kernel(int n_slabs, StoreSlabs<kAppend> slabs, StoreArgs a, const int* slab_table) {
    extern __shared__ __align__(16) uint8_t qsm[];
    int* pref = reinterpret_cast<int*>(qsm);                  // [n_slabs + 1] tile prefix
    int2* span = reinterpret_cast<int2*>(qsm + ((size_t(n_slabs) + 2) / 2) * 8);     // (not kTable) [n_slabs] rows already there, rows afterwards
    int* row0 = reinterpret_cast<int*>(span + n_slabs);       // (not kTable) [n_slabs] first rows in a contiguous layout
    const Q8View& c = slabs.c;
    const int Hk = slabs.Hk;
    uint32_t* const status = slabs.status;
    __shared__ uint32_t s_wsum[kQsWarps];
    __shared__ uint32_t s_amax[2][kQsWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = gridDim.x, cta = blockIdx.x;
    pdl_trigger();
    pdl_wait();

    // ---- which tiles there are
    if (kTable) {
#pragma unroll 4
        for (int s = tid; s <= n_slabs; s += kQsThreads) pref[s] = slab_table[s];
        __syncthreads();
    } else {
#pragma unroll 1
        for (int s = tid; s < n_slabs; s += kQsThreads) {
            const Span x = slabs.span(s, slabs.load(s));
            if (x.bad && cta == 0) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
            row0[s] = x.row0;
            span[s] = make_int2(x.old, x.now);
        }
        __syncthreads();
        cta_prefix<kQsThreads>(n_slabs, [&](int s) { return slabs.tiles(span[s].x, span[s].y); }, pref, s_wsum);
    }
    const Share share(2 * pref[n_slabs], cta, G);             // K and V of a tile one after the other

    const int c16 = lane & 15, half = lane >> 4;
    const int group = 1 << (c.block_log2 - 4);                // warps to a block
    int flip = 0, s = 0;
    for (int t2 = share.first; t2 < share.end; t2 += share.step) {
        const int t = t2 >> 1;
        s = slab_of(pref, n_slabs, t, s);
        const Span x_s = kTable ? slabs.span(s, slabs.load(s)) : Span{span[s].x, span[s].y, row0[s], false};
        const int old = x_s.old, now = x_s.now;
        const int j = old / kQ8Tile + (t - pref[s]);
        const int t0 = j * kQ8Tile;                           // the tile's first token
        const Q8Tile at = q8_tile(c, s, j, min(now - t0, kQ8Tile), x_s.row0);
        const uint4* src = (t2 & 1) ? a.v_src : a.k_src;
        uint8_t* dst = ((t2 & 1) ? c.V : c.K) + at.row * kQ8RowBytes;
        float* scale = ((t2 & 1) ? c.v_scale : c.k_scale) + at.scale;
        bool ok = at.row >= 0;
        // row of token tok in units of 16 bytes: src0 + tok * step
        long long src0, step;
        if (kAppend) {
            const int b = s / Hk;
            src0 = ((long long)a.new_off[b] - old) * Hk + s % Hk;
            step = Hk;
        } else {
            src0 = x_s.row0;
            step = 1;
            ok = ok && src0 >= 0 && src0 + now <= a.src_rows;
        }
        if (!ok) {                                            // (uniform over the CTA)
            if (tid == 0) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
            continue;
        }

        // ---- the new rows among this warp's 16 (whole: all of them are), and their largest magnitude
        const int r0 = warp * 16 + half;
        const bool whole = t0 + warp * 16 >= old && t0 + warp * 16 + 16 <= now;
        const uint4* from = src + (src0 + (long long)(t0 + r0) * step) * 16 + c16;
        const size_t inc = size_t(step) * 32;                 // two rows
        uint4 x[8];
        if (whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __ldcs(from + i * inc);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int tok = t0 + r0 + 2 * i;
                x[i] = make_uint4(0u, 0u, 0u, 0u);
                if (tok >= old && tok < now) x[i] = __ldcs(from + i * inc);
            }
        }
        const int blk = (warp * 16) >> c.block_log2;          // this warp's block in the tile
        const int b0 = t0 + (blk << c.block_log2);
        const bool held = b0 < old;                           // the block has rows under a scale of its own
        const float s_old = held ? scale[blk] : 0.f;
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m = __vimax3_u16x2(m, x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu);
            m = __vimax3_u16x2(m, x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu);
        }
        m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
        const bool wild = m >= 0x7f80u;
        if (wild) {                                           // infinities and NaN do not count for the scale; a NaN becomes zero
            if (lane == 0) atomicOr(status, SKIPKV_STATUS_NOT_FINITE);
            uint32_t fin = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = make_uint4(without_nan(x[i].x, fin), without_nan(x[i].y, fin), without_nan(x[i].z, fin), without_nan(x[i].w, fin));
            m = __reduce_max_sync(0xffffffffu, fin);
        }
        if (group > 1) {                                      // (two sets of places in turn: one barrier per tile)
            if (lane == 0) s_amax[flip][warp] = m;
            __syncthreads();
            for (int w = warp & ~(group - 1), k = 0; k < group; ++k) m = max(m, s_amax[flip][w + k]);
            flip ^= 1;
        }
        if (b0 >= now || b0 + (1 << c.block_log2) <= old) continue;      // no new row in the block (no barrier below)
        int e = scale_exp<kFmt>(m);
        if (held) e = max(e, held_exp(s_old));                // a scale only grows
        const float s_new = pow2f(e);
        if (lane == 0 && (warp & (group - 1)) == 0) scale[blk] = s_new;
        const float inv = pow2f(-e);

        // ---- codes
        uint2* const to = reinterpret_cast<uint2*>(dst + size_t(r0) * kQ8RowBytes) + c16;
        if (whole && !wild) {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i * 2 * (kQ8RowBytes / 8)] = codes8<kFmt>(x[i], inv);
            continue;
        }
        const float again = held ? s_old * inv : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int tok = t0 + r0 + 2 * i;
            if (tok >= now) continue;
            uint2* p = to + i * 2 * (kQ8RowBytes / 8);
            if (tok >= old) {
                if (kFmt == SKIPKV_Q8_INT8 && wild) {
                    *p = make_uint2(codes4_wild(make_uint2(x[i].x, x[i].y), inv), codes4_wild(make_uint2(x[i].z, x[i].w), inv));
                } else {
                    *p = codes8<kFmt>(x[i], inv);
                }
            } else if (held && s_new != s_old) {              // a row of the block as it was
                const uint2 cd = *p;
                uint32_t f[4];
                q8_to_f16<kFmt>(cd.x, f[0], f[1]);
                q8_to_f16<kFmt>(cd.y, f[2], f[3]);
                float2 y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    y[k] = f16x2_to_f2(f[k]);
                    y[k].x *= again; y[k].y *= again;
                }
                *p = make_uint2(q8_round<kFmt>(y[0].x, y[0].y, y[1].x, y[1].y), q8_round<kFmt>(y[2].x, y[2].y, y[3].x, y[3].y));
            }
        }
    }

    if constexpr (kAppend && !kTable) {
        for (int i = cta * kQsThreads + tid; i < n_slabs; i += G * kQsThreads) a.len_out[i] = span[i].y;
    }
}

// A row to each slab, or a few: kParts warps to a slab and tensor, four channels to a lane, a warp with every kParts-th block.  Nothing but latency:
// lengths and offsets are requested together, the rows and the scale behind them (paged: behind the page's entry); the codes that a block has are
// touched only where its scale grows.  A call takes it with up to four rows per sequence: the general kernel enumerates tiles first and has one step
// of the work (a tile) go through each CTA after the other.  Eight heads, us here / there: 16 sequences with a row each 2.0 / 5.7, four each 2.2 / 5.7;
// 256 sequences 3.0 / 33 and 6.6 / 33.  Where one sequence has all the rows (of 16 to 64, or 256 sequences) it is 3.0 / 4.5, 7.2 / 4.6 and, with
// 1024 rows, 31 / 8: the offsets are on the GPU, and that is the rarer case.  Four parts cost more than they give where there is a row to a
// sequence: 256 sequences 6.3 against 3.4.
constexpr int kQoThreads = 128;
constexpr int kQoMost = 4;                                     // rows per sequence, on average
constexpr int kQoParts = 4;                                    // with more rows than sequences
constexpr int kQoRows = 8;                                     // rows of new tokens on their way at a time
constexpr int kQoHeld = 16;                                    // and of rows that a block had

// kStep: a decode step, one row to each sequence.
template <int kFmt, int kParts, bool kStep>
__global__ void __launch_bounds__(kQoThreads)
q8_append_few_kernel(int batch, int Hk, int n_slabs, const int64_t* slab_off, const int32_t* cap, Q8View c, StoreArgs a, uint32_t* status) {
    const int lane = threadIdx.x & 31, w = (blockIdx.x * kQoThreads + threadIdx.x) >> 5;
    pdl_trigger();
    pdl_wait();
    if (w >= 2 * kParts * n_slabs) {                          // the step's queries into their slot of the window
        const int i = (w - 2 * kParts * n_slabs) * 32 + lane;
        if (kStep && a.q_win != nullptr && i < batch * a.Hq * 16) a.q_win[(size_t(i >> 4) * a.window + a.slot) * 16 + (i & 15)] = a.q[i];
        return;
    }
    const int s = w / (2 * kParts), part = (w >> 1) & (kParts - 1), b = s / Hk, block = 1 << c.block_log2;
    const int lo = a.new_off ? a.new_off[b] : b, hi = a.new_off ? a.new_off[b + 1] : b + 1;
    const int row0 = c.table ? 0 : q8_row0(slab_off, cap, Hk, s);        // (read beside the length)
    const int old = a.len_in[s], room = q8_room(c, cap, Hk, s);
    // (read beside the length too.  The slab's other warp may have added the sentence that this token opens: the count is a good one all the same)
    const int S0 = kStep ? a.n_sent[s] : 0;
    const long long end = (long long)old + (hi - lo);
    const bool inside = c.table != nullptr || (row0 >= 0 && end <= c.rows - row0);       // (not by q8_room_inside, a longer chain: 2.20 us against 1.93)
    const bool fits = old >= 0 && lo >= 0 && hi >= lo && hi <= a.n_new && end <= room && inside && (!kStep || (S0 >= 0 && S0 <= a.max_sent));
    const int count = fits ? hi - lo : 0;
    if (!fits && lane == 0) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
    const uint2* const src = reinterpret_cast<const uint2*>((w & 1) ? a.v_src : a.k_src) + (size_t(fits ? lo : 0) * Hk + s % Hk) * 32 + lane;
    const size_t next = size_t(Hk) * 32;                      // from one new row to the next
    for (int done = 0; done < count;) {
        const int tok = old + done, j = tok / kQ8Tile, r = tok % kQ8Tile;
        const int held = r & (block - 1), take = min(count - done, block - held);        // rows that the block has, and that it gets
        if (kParts > 1 && ((tok >> c.block_log2) & (kParts - 1)) != part) { done += take; continue; }
        const uint2* const x = src + done * next;
        uint2 y[kQoRows];
        auto load = [&](int k0) {
#pragma unroll
            for (int i = 0; i < kQoRows; ++i) y[i] = k0 + i < take ? x[(k0 + i) * next] : make_uint2(0u, 0u);
        };
        load(0);
        done += take;
        const Q8Tile at = q8_tile(c, s, j, r + take, row0);
        if (at.row < 0) {
            if (lane == 0) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
            continue;
        }
        float* const scale = ((w & 1) ? c.v_scale : c.k_scale) + at.scale + (r >> c.block_log2);
        uint32_t* const row = reinterpret_cast<uint32_t*>(((w & 1) ? c.V : c.K) + (at.row + r) * kQ8RowBytes) + lane;
        const float s_old = held ? *scale : 0.f;
        uint32_t m = 0;
#pragma unroll 1
        for (int k0 = 0; k0 < take; k0 += kQoRows) {
            if (k0) load(k0);
#pragma unroll
            for (int i = 0; i < kQoRows; ++i) m = __vimax3_u16x2(m, y[i].x & 0x7fff7fffu, y[i].y & 0x7fff7fffu);
        }
        m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
        const bool wild = m >= 0x7f80u;
        if (wild) {                                           // infinities and NaN do not count for the scale
            if (lane == 0) atomicOr(status, SKIPKV_STATUS_NOT_FINITE);
            uint32_t fin = 0;
            for (int k = 0; k < take; ++k) { (void)without_nan(x[k * next].x, fin); (void)without_nan(x[k * next].y, fin); }
            m = __reduce_max_sync(0xffffffffu, fin);
        }
        int e = scale_exp<kFmt>(m);
        if (held) e = max(e, held_exp(s_old));                // a scale only grows
        const float s_new = pow2f(e), inv = pow2f(-e);
#pragma unroll 1
        for (int k0 = 0; k0 < take; k0 += kQoRows) {
            if (take > kQoRows) load(k0);
#pragma unroll
            for (int i = 0; i < kQoRows; ++i) {
                if (k0 + i >= take) break;
                if (wild) { uint32_t fin = 0; y[i].x = without_nan(y[i].x, fin); y[i].y = without_nan(y[i].y, fin); }
                const float2 v0 = bf16x2_to_f2(y[i].x), v1 = bf16x2_to_f2(y[i].y);
                row[(k0 + i) * (kQ8RowBytes / 4)] = kFmt != SKIPKV_Q8_INT8 ? q8_round<kFmt>(v0.x * inv, v0.y * inv, v1.x * inv, v1.y * inv)
                                                    : wild ? codes4_wild(y[i], inv) : q8_round_scaled(v0, v1, make_float2(inv, inv));
            }
        }
        if (s_new == s_old) continue;
        __syncwarp();                                         // (every lane has read the scale)
        if (lane == 0) *scale = s_new;
        const float again = s_old * inv;                      // the rows that the block had, under the new scale
#pragma unroll 1
        for (int k0 = 1; k0 <= held; k0 += kQoHeld) {
            uint32_t* const p = row - k0 * (kQ8RowBytes / 4);
            uint32_t cd[kQoHeld];
#pragma unroll
            for (int i = 0; i < kQoHeld; ++i) cd[i] = k0 + i <= held ? p[-i * (kQ8RowBytes / 4)] : 0u;
#pragma unroll
            for (int i = 0; i < kQoHeld; ++i) {
                uint32_t f0, f1;
                q8_to_f16<kFmt>(cd[i], f0, f1);
                const float2 y0 = f16x2_to_f2(f0), y1 = f16x2_to_f2(f1);
                if (k0 + i <= held) p[-i * (kQ8RowBytes / 4)] = q8_round<kFmt>(y0.x * again, y0.y * again, y1.x * again, y1.y * again);
            }
        }
    }
    if (w & (2 * kParts - 1)) return;
    // ---- the length, and the rest of a decode step
    const int now = old + count;
    if (lane == 0) a.len_out[s] = now;
    if (!kStep || !fits) return;                              // (no room, or a list that makes no sense: reported above, tables as they were)
    const bool opens = S0 == 0 || a.new_sent[b];
    int32_t* so = a.sent_off + size_t(s) * (a.max_sent + 1);
    const int S = opens && S0 < a.max_sent ? S0 + 1 : S0;     // (a full list: the token joins the last sentence)
    __syncwarp();
    if (lane == 0 && opens && S == S0) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
    if (lane == 0 && S != S0) {
        if (S0 == 0) so[0] = 0;
        a.sent_id[size_t(s) * a.max_sent + S0] = a.gen_id[b];
        a.n_sent[s] = S;
    }
    for (int i = S + lane; i <= a.max_sent; i += 32) so[i] = now;
}

// Eight codes times their scale (32 bits), rounded once to bf16.
template <int kFmt>
__device__ __forceinline__ uint4 values8(const uint2& x, float sc) {
    uint32_t o[4];
    float2 y[4];
    if (kFmt == SKIPKV_Q8_INT8) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            // the byte u = c + 128 below 0x4b0000 is the float 2^23 + u
            const uint32_t u = (k ? x.y : x.x) ^ 0x80808080u;
            const float2 off = make_float2(-8388736.f, -8388736.f);
            y[2 * k] = __fadd2_rn(make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7541))), off);
            y[2 * k + 1] = __fadd2_rn(make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7542)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7543))), off);
        }
    } else {
        uint32_t f[4];
        q8_to_f16<kFmt>(x.x, f[0], f[1]);
        q8_to_f16<kFmt>(x.y, f[2], f[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = f16x2_to_f2(f[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 v = __fmul2_rn(y[k], make_float2(sc, sc));
        const __nv_bfloat162 r = __floats2bfloat162_rn(v.x, v.y);
        o[k] = *reinterpret_cast<const uint32_t*>(&r);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// Codes back to bf16: K and V of a tile in turn (one of them where the other has no destination).
struct LoadSlabs {
    struct Raw { int len, cap; int64_t off; };
    Q8View c;
    const int64_t* slab_off;
    const int32_t *cap, *kv_len;
    uint32_t* status;
    int Hk;
    int dst_rows;                                             // of the bf16 buffers
    __device__ __forceinline__ Raw load(int s) const { return {kv_len[s], cap[s / Hk], slab_off[s / Hk]}; }
    __device__ __forceinline__ Span span(int s, const Raw& r) const {
        const int row0 = q8_row0(r.off, r.cap, Hk, s);
        const int room = rows_inside(q8_room_inside(c, r.cap, row0), row0, dst_rows);
        return {0, min(max(r.len, 0), room), row0, r.len < 0 || r.len > room};
    }
    __device__ __forceinline__ int count(int s, const Raw& r) const {
        const Span x = span(s, r);
        if (x.bad) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
        return (x.now + kQ8Tile - 1) / kQ8Tile;
    }
};

template <int kFmt, bool kTable>
__global__ void __launch_bounds__(kQsThreads, 6)
q8_load_kernel(int n_slabs, LoadSlabs slabs, uint4* K, uint4* V, const int* slab_table) {
    extern __shared__ __align__(16) uint8_t qsm[];
    int* pref = reinterpret_cast<int*>(qsm);
    int* lens = pref + n_slabs + 1;                           // (not kTable)
    int* row0 = lens + n_slabs;                               // (not kTable) first rows in a contiguous layout
    const Q8View& c = slabs.c;
    uint32_t* const status = slabs.status;
    __shared__ uint32_t s_wsum[kQsWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = gridDim.x, cta = blockIdx.x;
    pdl_trigger();
    pdl_wait();
    if (kTable) {
#pragma unroll 4
        for (int s = tid; s <= n_slabs; s += kQsThreads) pref[s] = slab_table[s];
        __syncthreads();
    } else {
        for (int s = tid; s < n_slabs; s += kQsThreads) {
            const Span x = slabs.span(s, slabs.load(s));
            if (x.bad && cta == 0) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
            row0[s] = x.row0;
            lens[s] = x.now;
        }
        __syncthreads();
        cta_prefix<kQsThreads>(n_slabs, [&](int s) { return (lens[s] + kQ8Tile - 1) / kQ8Tile; }, pref, s_wsum);
    }
    const int per = (K ? 1 : 0) + (V ? 1 : 0);
    const Share share(pref[n_slabs] * per, cta, G);
    const int c16 = lane & 15, r0 = warp * 16 + (lane >> 4);
    int s = 0;
    for (int t2 = share.first; t2 < share.end; t2 += share.step) {
        const int t = per == 2 ? t2 >> 1 : t2;
        const bool is_v = per == 2 ? (t2 & 1) != 0 : V != nullptr;
        s = slab_of(pref, n_slabs, t, s);
        const Span x_s = kTable ? slabs.span(s, slabs.load(s)) : Span{0, lens[s], row0[s], false};
        const int j = t - pref[s], rows = min(x_s.now - j * kQ8Tile, kQ8Tile);
        const Q8Tile at = q8_tile(c, s, j, rows, x_s.row0);
        const long long to = (long long)x_s.row0 + (long long)j * kQ8Tile;
        if (at.row < 0) {
            if (tid == 0) atomicOr(status, SKIPKV_STATUS_BAD_TABLE);
            continue;
        }
        if (warp * 16 >= rows) continue;
        const uint2* src = reinterpret_cast<const uint2*>((is_v ? c.V : c.K) + (at.row + r0) * kQ8RowBytes) + c16;
        uint4* dst = (is_v ? V : K) + (to + r0) * 16 + c16;
        const bool whole = warp * 16 + 16 <= rows;
        const float sc = ((is_v ? c.v_scale : c.k_scale) + at.scale)[(warp * 16) >> c.block_log2];
        uint2 x[8];
        if (whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __ldcs(src + i * 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[i * 32] = values8<kFmt>(x[i], sc);
        } else {
#pragma unroll 1
            for (int i = 0; i < 8; ++i)
                if (r0 + 2 * i < rows) dst[i * 32] = values8<kFmt>(__ldcs(src + i * 32), sc);
        }
    }
}

int check_q8(const skipkv_shape* s, const skipkv_q8_cache* c) {
    if (!c || !c->K || !c->V || !c->k_scale || !c->v_scale || c->rows <= 0) return SKIPKV_ERR_INVALID_ARG;
    if (c->format != SKIPKV_Q8_E4M3 && c->format != SKIPKV_Q8_INT8) return SKIPKV_ERR_UNSUPPORTED;
    if (c->block_rows != 16 && c->block_rows != 32 && c->block_rows != 64 && c->block_rows != 128) return SKIPKV_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(c->K) | reinterpret_cast<uintptr_t>(c->V)) & 15) return SKIPKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & 3) return SKIPKV_ERR_INVALID_ARG;
    if ((c->batch || c->n_kv_heads) && (c->batch < s->batch || c->n_kv_heads != s->n_kv_heads)) {
        set_error_text("the 8-bit cache is laid out for fewer sequences, or for other KV heads");
        return SKIPKV_ERR_INVALID_ARG;
    }
    if (c->block_table ? c->max_pages <= 0 || c->rows % kQ8Tile != 0 : c->max_blocks <= 0) return SKIPKV_ERR_INVALID_ARG;
    if (c->rows > int64_t(0x7fffffff) - 256) return SKIPKV_ERR_UNSUPPORTED;
    const int64_t slabs = int64_t(s->batch) * s->n_kv_heads;
    if (slabs > kQ8MaxSlabs) {
        set_error_text("8-bit cache: batch * n_kv_heads above 8192");
        return SKIPKV_ERR_UNSUPPORTED;
    }
    // places of scales, and tiles of K and V of all slabs with a grid's step more, in 32 bits
    if (slabs * (c->block_table ? c->max_pages : c->max_blocks) >= (1 << 30) - 4096) return SKIPKV_ERR_UNSUPPORTED;
    if (c->device >= 0) {
        int dev = 0;
        SKIPKV_CUDA(cudaGetDevice(&dev));
        if (dev != c->device) {
            set_error_text("the 8-bit cache is on another device than the current one");
            return SKIPKV_ERR_INVALID_ARG;
        }
    }
    return SKIPKV_OK;
}

}  // namespace skipkv

using namespace skipkv;

// CTAs of a launch over at most `tiles` tiles: four (six) to an SM.
static int store_grid(long long tiles, int per_sm) {
    const long long most = (long long)num_sms() * per_sm;
    return int(tiles < 1 ? 1 : tiles < most ? tiles : most);
}

template <bool kAppend>
static int store(const skipkv_shape* shape, const skipkv_q8_cache* cache, const StoreArgs& a, long long tiles, void* ws, void* stream) {
    const int n_slabs = shape->batch * shape->n_kv_heads;
    const bool table = n_slabs >= kQsTableSlabs;
    uint8_t* w = static_cast<uint8_t*>(ws);
    int* slab_table = reinterpret_cast<int*>(w + make_layout(*shape).slab_table);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const StoreSlabs<kAppend> slabs{q8_view(*cache), shape->slab_off, shape->cap, a.new_off, a.len_in, a.len_out, &static_cast<Header*>(ws)->status,
                                    a.n_new, int(shape->n_kv_heads)};
    if (table) SKIPKV_CUDA(launch_dependent(q8_table_kernel<StoreSlabs<kAppend>>, dim3(1), dim3(kQ8TableThreads), 0, st, n_slabs, slabs, slab_table));
    const size_t prefix = (size_t(n_slabs) + 2) / 2 * 8, smem = table ? prefix : prefix + size_t(n_slabs) * 12;
    auto run = [&](auto kernel) {
        return launch_dependent(kernel, dim3(store_grid(2 * tiles, 4)), dim3(kQsThreads), smem, st, n_slabs, slabs, a,
                                static_cast<const int*>(slab_table));
    };
    auto pick = [&](auto fmt) {
        constexpr int kFmt = decltype(fmt)::value;
        return table ? run(q8_store_kernel<kFmt, kAppend, true>) : run(q8_store_kernel<kFmt, kAppend, false>);
    };
    SKIPKV_CUDA(cache->format == SKIPKV_Q8_E4M3 ? pick(std::integral_constant<int, SKIPKV_Q8_E4M3>()) : pick(std::integral_constant<int, SKIPKV_Q8_INT8>()));
    return SKIPKV_OK;
}

static int append(const skipkv_shape* shape, const skipkv_q8_cache* cache, const void* k_new, const void* v_new, const int32_t* new_off,
                  int32_t n_new, const int32_t* kv_len_in, int32_t* kv_len_out, StoreArgs a, void* ws, void* stream) {
    if (n_new < 0 || (n_new > 0 && (!k_new || !v_new)) || !kv_len_in || !kv_len_out || kv_len_in == kv_len_out) return SKIPKV_ERR_INVALID_ARG;
    if (!new_off && n_new != shape->batch) return SKIPKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new)) & 15) return SKIPKV_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return SKIPKV_ERR_WORKSPACE;
    a.k_src = static_cast<const uint4*>(k_new); a.v_src = static_cast<const uint4*>(v_new);
    a.new_off = new_off; a.n_new = n_new; a.len_in = kv_len_in; a.len_out = kv_len_out;
    const int slabs = shape->batch * shape->n_kv_heads;
    if (new_off && (long long)n_new > (long long)kQoMost * shape->batch) {
        // a slab's new rows lie in one tile more than they fill, at most
        return store<true>(shape, cache, a, (long long)n_new * shape->n_kv_heads / kQ8Tile + 2ll * slabs, ws, stream);
    }
    const bool parts = n_new > shape->batch;
    const long long warps = (parts ? 2ll * kQoParts : 2ll) * slabs + (a.q_win ? ((long long)shape->batch * shape->n_q_heads * 16 + 31) / 32 : 0);
    auto run = [&](auto kernel) {
        return launch_dependent(kernel, dim3(unsigned((warps * 32 + kQoThreads - 1) / kQoThreads)), dim3(kQoThreads), 0, static_cast<cudaStream_t>(stream),
                                int(shape->batch), int(shape->n_kv_heads), slabs, shape->slab_off, shape->cap, q8_view(*cache), a,
                                &static_cast<Header*>(ws)->status);
    };
    auto pick = [&](auto fmt) {
        constexpr int kFmt = decltype(fmt)::value;
        if (a.n_sent) return run(q8_append_few_kernel<kFmt, 1, true>);
        return parts ? run(q8_append_few_kernel<kFmt, kQoParts, false>) : run(q8_append_few_kernel<kFmt, 1, false>);
    };
    SKIPKV_CUDA(cache->format == SKIPKV_Q8_E4M3 ? pick(std::integral_constant<int, SKIPKV_Q8_E4M3>()) : pick(std::integral_constant<int, SKIPKV_Q8_INT8>()));
    return SKIPKV_OK;
}

extern "C" int skipkv_pack_q8(const skipkv_shape* shape, const skipkv_q8_cache* cache, const void* K, const void* V,
                              const int32_t* kv_len, void* ws, void* stream) {
    if (int rc = check_shape(shape)) return rc;
    if (int rc = check_q8(shape, cache)) return rc;
    if (!K || !V || !kv_len) return SKIPKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15) return SKIPKV_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return SKIPKV_ERR_WORKSPACE;
    StoreArgs a{};
    a.k_src = static_cast<const uint4*>(K); a.v_src = static_cast<const uint4*>(V);
    a.src_rows = shape->total_rows; a.len_in = kv_len;
    const long long tiles = (long long)shape->batch * shape->n_kv_heads * ((shape->max_cap + kQ8Tile - 1) / kQ8Tile);
    return store<false>(shape, cache, a, tiles, ws, stream);
}

extern "C" int skipkv_append_q8(const skipkv_shape* shape, const skipkv_q8_cache* cache, const void* k_new, const void* v_new,
                                const int32_t* new_off, int32_t n_new, const int32_t* kv_len_in, int32_t* kv_len_out, void* ws,
                                void* stream) {
    if (int rc = check_shape(shape)) return rc;
    if (int rc = check_q8(shape, cache)) return rc;
    return append(shape, cache, k_new, v_new, new_off, n_new, kv_len_in, kv_len_out, StoreArgs{}, ws, stream);
}

extern "C" int skipkv_append_step_q8(const skipkv_shape* shape, const skipkv_q8_cache* cache, const void* k_new, const void* v_new,
                                     const int32_t* kv_len_in, int32_t* kv_len_out, int32_t* sent_off, int32_t* sent_id,
                                     int32_t* n_sent, const uint8_t* new_sent, const int32_t* gen_id, void* q_win, const void* q,
                                     int32_t slot, void* ws, void* stream) {
    if (int rc = check_shape(shape)) return rc;
    if (int rc = check_q8(shape, cache)) return rc;
    if (!sent_off || !sent_id || !n_sent || !new_sent || !gen_id || shape->max_sent <= 0) return SKIPKV_ERR_INVALID_ARG;
    if ((q_win != nullptr) != (q != nullptr)) return SKIPKV_ERR_INVALID_ARG;
    if (q_win && (slot < 0 || slot >= shape->window)) return SKIPKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(q_win) | reinterpret_cast<uintptr_t>(q)) & 15) return SKIPKV_ERR_INVALID_ARG;
    StoreArgs a{};
    a.sent_off = sent_off; a.sent_id = sent_id; a.n_sent = n_sent; a.new_sent = new_sent; a.gen_id = gen_id;
    a.q_win = static_cast<uint4*>(q_win); a.q = static_cast<const uint4*>(q);
    a.Hq = shape->n_q_heads; a.window = shape->window; a.slot = slot; a.max_sent = shape->max_sent;
    return append(shape, cache, k_new, v_new, nullptr, shape->batch, kv_len_in, kv_len_out, a, ws, stream);
}

extern "C" int skipkv_unpack_q8(const skipkv_shape* shape, const skipkv_q8_cache* cache, const int32_t* kv_len, void* K, void* V,
                                void* ws, void* stream) {
    if (int rc = check_shape(shape)) return rc;
    if (int rc = check_q8(shape, cache)) return rc;
    if (!kv_len || (!K && !V)) return SKIPKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15) return SKIPKV_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return SKIPKV_ERR_WORKSPACE;
    const int n_slabs = shape->batch * shape->n_kv_heads;
    const long long tiles = (long long)n_slabs * ((shape->max_cap + kQ8Tile - 1) / kQ8Tile) * ((K ? 1 : 0) + (V ? 1 : 0));
    const bool table = n_slabs >= kQsTableSlabs;
    int* slab_table = reinterpret_cast<int*>(static_cast<uint8_t*>(ws) + make_layout(*shape).slab_table);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const LoadSlabs slabs{q8_view(*cache), shape->slab_off, shape->cap, kv_len, &static_cast<Header*>(ws)->status, int(shape->n_kv_heads),
                          int(shape->total_rows)};
    if (table) SKIPKV_CUDA(launch_dependent(q8_table_kernel<LoadSlabs>, dim3(1), dim3(kQ8TableThreads), 0, st, n_slabs, slabs, slab_table));
    auto run = [&](auto kernel) {
        return launch_dependent(kernel, dim3(store_grid(tiles, 6)), dim3(kQsThreads), size_t(table ? n_slabs + 1 : 3 * n_slabs + 1) * 4, st, n_slabs,
                                slabs, static_cast<uint4*>(K), static_cast<uint4*>(V), static_cast<const int*>(slab_table));
    };
    auto pick = [&](auto fmt) {
        constexpr int kFmt = decltype(fmt)::value;
        return table ? run(q8_load_kernel<kFmt, true>) : run(q8_load_kernel<kFmt, false>);
    };
    SKIPKV_CUDA(cache->format == SKIPKV_Q8_E4M3 ? pick(std::integral_constant<int, SKIPKV_Q8_E4M3>()) : pick(std::integral_constant<int, SKIPKV_Q8_INT8>()));
    return SKIPKV_OK;
}
