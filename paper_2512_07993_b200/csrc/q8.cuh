// The cache in 8 bits (skipkv_q8_cache): addresses, scales and codes, shared by the calls that store, load and attend to it.
#pragma once
#include "common.cuh"

namespace skipkv {

constexpr int kQ8RowBytes = kHeadDim;         // one row of codes
constexpr int kQ8Tile = SKIPKV_PAGE_ROWS;     // rows that a CTA works on at a time: a page, a whole number of blocks
constexpr int kQ8MaxSlabs = 8192;             // tables of slabs in shared memory
constexpr int kQ8LeastExp = -100;             // of a scale: what lies 2^-109 below is rounded to zero, long before subnormals

// The cache as the kernels see it.
struct Q8View {
    uint8_t* K;
    uint8_t* V;
    float* k_scale;
    float* v_scale;
    const int32_t* table;                     // nullptr: contiguous slabs
    long long rows;
    int end;                                  // the same: fewer than 2^31
    int block_log2, max_blocks, max_pages;
};

inline Q8View q8_view(const skipkv_q8_cache& c) {
    Q8View v{};
    v.K = static_cast<uint8_t*>(c.K); v.V = static_cast<uint8_t*>(c.V);
    v.k_scale = c.k_scale; v.v_scale = c.v_scale; v.table = c.block_table; v.rows = c.rows;
    v.end = int(c.rows);
    v.block_log2 = c.block_rows == 16 ? 4 : c.block_rows == 32 ? 5 : c.block_rows == 64 ? 6 : 7;
    v.max_blocks = c.max_blocks; v.max_pages = c.max_pages;
    return v;
}
int check_q8(const skipkv_shape* s, const skipkv_q8_cache* c);      // SKIPKV_OK or an error code

#ifdef __CUDACC__

// Rows that a slab of `cap` rows has room for: in any case so few that a tile's rows more are a number of 32 bits.
__host__ __device__ __forceinline__ int q8_room(const Q8View& v, int cap) {
    const long long lim = v.table ? (long long)v.max_pages * kQ8Tile : (long long)v.max_blocks << v.block_log2;
    return min(max(cap, 0), int(min(lim, 0x7fffff00ll)));
}
__host__ __device__ __forceinline__ int q8_room(const Q8View& v, const int32_t* cap, int Hk, int s) { return q8_room(v, cap[s / Hk]); }
__host__ __device__ __forceinline__ int q8_row0(int64_t off, int cap, int Hk, int s) {
    const long long row = (long long)(size_t(off) * Hk + size_t(s % Hk) * cap);
    return row < 0 || row > 0x7fffff00ll ? -1 : int(row);
}
// First row of slab s in a contiguous layout; -1 where it lies nowhere near the buffers (fewer than 2^31 rows).
__host__ __device__ __forceinline__ int q8_row0(const int64_t* slab_off, const int32_t* cap, int Hk, int s) {
    return q8_row0(slab_off[s / Hk], cap[s / Hk], Hk, s);
}
// Of `room` rows those that lie between row0 (as q8_row0 gives it) and the end of a buffer.
__host__ __device__ __forceinline__ int rows_inside(int room, int row0, int end) { return row0 < 0 || row0 > end ? 0 : min(room, end - row0); }
// Rows that a slab has room for, in the buffers too.
__host__ __device__ __forceinline__ int q8_room_inside(const Q8View& v, int cap, int row0) {
    return v.table ? q8_room(v, cap) : rows_inside(q8_room(v, cap), row0, v.end);
}
// Where tile j (tokens [128 j, 128 j + 128)) of slab s lies: its first row, and the place of its first block's scale.  Of its first
// `rows` rows none may lie outside the buffers, else row = -1.  row0: as q8_row0 gives it (not used for a paged cache).
struct Q8Tile { long long row; size_t scale; };
__host__ __device__ __forceinline__ Q8Tile q8_tile(const Q8View& v, int s, int j, int rows, int row0) {
    Q8Tile t;
    if (v.table) {
        const int page = v.table[size_t(s) * v.max_pages + j];
        t.row = (long long)page * kQ8Tile;
        t.scale = size_t(page > 0 ? page : 0) << (7 - v.block_log2);
        if (page < 0 || t.row + kQ8Tile > v.rows) t.row = -1;
    } else {
        t.row = (long long)row0 + (long long)j * kQ8Tile;
        t.scale = size_t(s) * v.max_blocks + (size_t(j) << (7 - v.block_log2));
        if (row0 < 0 || t.row + rows > v.rows) t.row = -1;
    }
    return t;
}

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }      // -126 <= e <= 127

// Four codes as two pairs of f16, exactly: codes 0 and 1, codes 2 and 3.
template <int kFmt>
__device__ __forceinline__ void q8_to_f16(uint32_t c, uint32_t& lo, uint32_t& hi) {
    if (kFmt == SKIPKV_Q8_E4M3) {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(c));
    } else {
        // 0x64 in front of an unsigned byte u is the f16 1024 + u; with u = c + 128 it takes 1152 off
        const uint32_t u = c ^ 0x80808080u;
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
    }
}
__device__ __forceinline__ float2 f16x2_to_f2(uint32_t x) {
    float2 r;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(r.x), "=f"(r.y) : "r"(x));
    return r;
}
// Four values (|y| <= 448 or 127, or infinite) to codes, each rounded once to nearest even.
template <int kFmt>
__device__ __forceinline__ uint32_t q8_round(float y0, float y1, float y2, float y3) {
    uint32_t r;
    if (kFmt == SKIPKV_Q8_E4M3) {
        asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\tmov.b32 %0, {a, b};\n\t}"
            : "=r"(r) : "f"(y0), "f"(y1), "f"(y2), "f"(y3));
    } else {
        // 1.5 * 2^23 + y has the whole number nearest to y in its low bits
        const float big = 12582912.f;
        const uint32_t a = __float_as_uint(__fadd_rn(y0, big)), b = __float_as_uint(__fadd_rn(y1, big));
        const uint32_t c = __float_as_uint(__fadd_rn(y2, big)), d = __float_as_uint(__fadd_rn(y3, big));
        r = __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
    }
    return r;
}

// int8: four values times a power of two to codes, in one rounding: 1.5 * 2^23 + the (exact) product has the nearest whole number in its low bits.
__device__ __forceinline__ uint32_t q8_round_scaled(float2 a, float2 b, float2 k) {
    const float2 big = make_float2(12582912.f, 12582912.f);
    a = __ffma2_rn(a, k, big);
    b = __ffma2_rn(b, k, big);
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}

// Many slabs: one CTA, in a launch of its own, makes the prefix sum over the slabs' tiles that the CTAs of the launch behind it else make each for
// itself, which takes the longer the more slabs there are, and shared memory that costs resident CTAs.  8192 slabs of 500 rows: attention 217 us
// with it against 460, storing 531 against 1050, loading 581 against 694.
constexpr int kQ8TableThreads = 1024;
constexpr int kQ8TableEach = kQ8MaxSlabs / kQ8TableThreads;

// Slabs::load(s) reads what the GPU memory says of slab s, Slabs::count(s, ...) makes its number of it.  pref: [n_slabs + 1].
template <typename Slabs>
__global__ void __launch_bounds__(kQ8TableThreads)
q8_table_kernel(int n_slabs, Slabs slabs, int* pref) {
    __shared__ int s_wsum[kQ8TableThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_trigger();                                            // (behind the wait: the CTAs of the launch behind wait on the SMs as it is)
    const int per = (n_slabs + kQ8TableThreads - 1) / kQ8TableThreads, s0 = tid * per;
    typename Slabs::Raw raw[kQ8TableEach];
#pragma unroll
    for (int i = 0; i < kQ8TableEach; ++i)
        if (i < per && s0 + i < n_slabs) raw[i] = slabs.load(s0 + i);
    int cnt[kQ8TableEach], local = 0;
#pragma unroll
    for (int i = 0; i < kQ8TableEach; ++i) {
        cnt[i] = i < per && s0 + i < n_slabs ? slabs.count(s0 + i, raw[i]) : 0;
        local += cnt[i];
    }
    int inc = local;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += x;
    }
    if (lane == 31) s_wsum[warp] = inc;
    __syncthreads();
    int run = lane < warp ? s_wsum[lane] : 0;
#pragma unroll
    for (int d = 16; d; d >>= 1) run += __shfl_xor_sync(0xffffffffu, run, d);
    run += inc - local;
#pragma unroll
    for (int i = 0; i < kQ8TableEach; ++i) {
        if (i < per && s0 + i < n_slabs) pref[s0 + i] = run;
        run += cnt[i];
    }
    if (tid == kQ8TableThreads - 1) pref[n_slabs] = run;
}

#endif  // __CUDACC__

}  // namespace skipkv
