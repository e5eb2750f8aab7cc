// The page server of a paged cache: which slab holds which pages (skipkv_page_tables) and the pool row of every new token
// (skipkv_slot_map).
//
// Tables: per slab the pages it holds and the pages that its tokens need; two prefix sums over the slabs, of the pages taken and of
// the pages given back, say from which place of the ring each slab takes and to which it gives.  Every CTA works them out for itself from
// the call's inputs, which the call does not change (counts and the ring's state go to other buffers), so no CTA waits for another.
// The free pages are a ring, not a stack: pages are taken at its head and given back behind its tail, and with f free pages of P at most
// P - f come back, so what is written is never what is read.  The order is that of the slabs, whatever the CTAs' order.
// Latency: a prologue over the slabs and one chain ring -> table per page: 3.2 us for 128 slabs, whether sixteen of them enter their next page or
// all take 256 to 512 pages.
//
// Slots: 8 bytes written per token and head.  50 MB (sixteen prompts of 32K to 64K, eight heads) take 10.1 us, 0.76 of the copy rate with the launch;
// a decode step's 128 take 2.4.
#include "common.cuh"

namespace skipkv {

constexpr int kPtThreads = 256;
constexpr int kPtWarps = kPtThreads / 32;
constexpr int kPtMaxSlabs = 8192;
constexpr int kPtAhead = 4;                                   // pages that a lane has on their way from the ring
constexpr int kPtPageRows = SKIPKV_PAGE_ROWS;
constexpr int kPtOffsets = 1024;

__global__ void __launch_bounds__(kPtThreads)
page_tables_kernel(int n_slabs, int max_pages, int pool, const int32_t* need, const int32_t* have_in, int32_t* have_out, int32_t* table,
                   int32_t* ring, const int32_t* ring_in, int32_t* ring_out, uint32_t* status) {
    extern __shared__ __align__(16) int ptsm[];
    int* take = ptsm;                                         // [n_slabs + 1] pages taken by the slabs before
    int* give = take + n_slabs + 1;                           // [n_slabs + 1] pages given back by them
    int* delta = give + n_slabs + 1;                          // [n_slabs] pages wanted beyond those held
    __shared__ uint32_t s_wsum[kPtWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
    pdl_wait();
    pdl_trigger();                                            // (see the slots)
    uint32_t bad = 0;
    const int head = ring_in[0], free0 = ring_in[1];
    const bool ring_ok = head >= 0 && head < pool && free0 >= 0 && free0 <= pool;
    for (int s = tid; s < n_slabs; s += kPtThreads) {
        const int have = have_in[s], rows = need[s];
        const int want = int(((long long)rows + kPtPageRows - 1) / kPtPageRows);
        const bool ok = ring_ok && rows >= 0 && want <= max_pages && have >= 0 && have <= max_pages;
        if (!ok) bad = SKIPKV_STATUS_BAD_TABLE;
        delta[s] = ok ? want - have : 0;
    }
    __syncthreads();
    cta_prefix<kPtThreads>(n_slabs, [&](int s) { return max(delta[s], 0); }, take, s_wsum);
    cta_prefix<kPtThreads>(n_slabs, [&](int s) { return max(-delta[s], 0); }, give, s_wsum);
    auto at = [&](int place) { return place >= pool ? place - pool : place; };       // of the ring; place < 2 * pool
    // a slab's pages are shared out over `per` warps, 32 at a time
    const int warps = gridDim.x * kPtWarps, wid = cta * kPtWarps + warp;
    const int per = max(1, warps / n_slabs);
    for (int w = wid; w < n_slabs * per; w += warps) {
        const int s = w % n_slabs, part = w / n_slabs;
        const int d = delta[s], have = have_in[s];
        int32_t* row = table + size_t(s) * max_pages;
        const bool served = take[s + 1] <= free0;
        if (part == 0 && lane == 0) {
            have_out[s] = d > 0 && !served ? have : have + d;
            if (d > 0 && !served) bad |= SKIPKV_STATUS_NO_PAGES;
        }
        if (d > 0 && served) {
            for (int j = part * 32 + lane; j < d; j += per * 32 * kPtAhead) {
                int page[kPtAhead];
#pragma unroll
                for (int k = 0; k < kPtAhead; ++k) {
                    const int jk = j + k * per * 32;
                    page[k] = jk < d ? ring[at(head + take[s] + jk)] : 0;
                }
#pragma unroll
                for (int k = 0; k < kPtAhead; ++k) {
                    const int jk = j + k * per * 32;
                    const bool ok = page[k] >= 0 && page[k] < pool;
                    if (!ok) bad |= SKIPKV_STATUS_BAD_TABLE;
                    if (jk < d) row[have + jk] = ok ? page[k] : -1;
                }
            }
        } else if (d < 0) {
            for (int j = part * 32 + lane; j < -d; j += per * 32) {
                if (free0 + give[s] + j >= pool) { bad |= SKIPKV_STATUS_BAD_TABLE; continue; }       // more pages than there are
                ring[at(head + free0 + give[s] + j)] = row[have + d + j];
            }
        }
    }
    if (cta == 0 && tid == 0) {
        // what was taken: the requests up to the last that fitted
        int lo = 0, hi = n_slabs;                             // the largest s with take[s] <= free0
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (take[mid] <= free0) lo = mid; else hi = mid - 1;
        }
        const int taken = ring_ok ? take[lo] : 0, back = ring_ok ? min(give[n_slabs], pool - free0) : 0;
        ring_out[0] = ring_ok ? at(head + taken) : head;
        ring_out[1] = free0 - taken + back;
    }
    if (bad && status) atomicOr(status, bad);
}

// kHeads: KV heads of a token that a thread does (a 16-byte store where there are two).  A warp takes a range of tokens, a lane the same heads of
// every few of them: it goes from one sequence to the next only now and then, and looks up a page every 128 tokens.  (A CTA's range with its
// threads side by side looks up a page every other token: 12.3 us against 10.1 for sixteen prompts of 32K to 64K, eight heads.)
template <int kHeads>
__global__ void __launch_bounds__(kPtThreads)
slot_map_kernel(int batch, int Hk, int max_pages, const int32_t* table, const int32_t* n_pages, const int32_t* start, const int32_t* new_off,
                int n_new, int64_t* slots) {
    __shared__ int s_off[kPtOffsets];
    const int lane = threadIdx.x & 31;
    const int hw = Hk / kHeads;
    const int tokens = hw < 32 ? 32 / hw : 1;                 // of one pass of the warp
    const int first = hw < 32 ? lane / hw : 0;
    const uint32_t warps = gridDim.x * kPtWarps, w = blockIdx.x * kPtWarps + (threadIdx.x >> 5);
    const uint32_t share = (uint32_t(n_new) + warps - 1) / warps;
    const int i0 = int(min(share * w, uint32_t(n_new))), i1 = int(min(share * w + share, uint32_t(n_new)));
    pdl_wait();
    // Triggered behind the wait, here and in the tables: at most one call behind this one has CTAs on the SMs while it runs.  With two of them there
    // the CTAs of slots crowd on the SMs that were free first: 26 us for tables and slots of those prompts in turn, against 14.1.
    pdl_trigger();
    // the offsets are searched in shared memory where they fit: a search is a chain of reads
    if (new_off != nullptr && batch < kPtOffsets) {
        for (int k = threadIdx.x; k <= batch; k += kPtThreads) s_off[k] = new_off[k];
        new_off = s_off;
        __syncthreads();
    }
    if (first >= tokens) return;
    for (int hp = hw < 32 ? lane % hw : lane; hp < hw; hp += 32) {
        int i = i0 + first, b = 0;
        int64_t* p = slots + (long long)i * Hk + hp * kHeads;
        const size_t next = size_t(tokens) * Hk;
        while (i < i1) {
            int lo = i, hi = i + 1;                           // the tokens of sequence b
            if (new_off == nullptr) {
                b = i;
            } else {
                int r = batch;                                // the first sequence that ends behind token i
                while (b < r) {
                    const int mid = (b + r) >> 1;
                    if (new_off[mid + 1] > i) r = mid; else b = mid + 1;
                }
                if (b == batch) break;                        // tokens of no sequence
                lo = new_off[b]; hi = new_off[b + 1];
            }
            if (i < lo) { i += tokens; p += next; continue; }
            uint32_t t[kHeads], end[kHeads], page_end[kHeads];     // per head: the token (below 2^32), the end of the slab's pages and of the last one looked up
            long long page_row[kHeads];                       // that one's first row
            const int32_t* row[kHeads];
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
                const int s = b * Hk + hp * kHeads + k, at = start[s];
                t[k] = uint32_t(at) + uint32_t(i - lo);
                end[k] = at < 0 ? 0u : uint32_t(min(max(n_pages[s], 0), min(max_pages, 1 << 24))) * kPtPageRows;
                row[k] = table + size_t(s) * max_pages;
                page_end[k] = 0u;
                page_row[k] = -1;
            }
            for (const int stop = min(hi, i1); i < stop; i += tokens, p += next) {
                long long v[kHeads];
#pragma unroll
                for (int k = 0; k < kHeads; ++k) {
                    if (t[k] >= page_end[k]) {
                        const int page = t[k] < end[k] ? row[k][t[k] / kPtPageRows] : -1;
                        page_row[k] = page < 0 ? -1ll : (long long)page * kPtPageRows;
                        page_end[k] = t[k] < end[k] ? (t[k] | (kPtPageRows - 1u)) + 1u : 0xffffffffu;
                    }
                    v[k] = page_row[k] | (long long)(t[k] & (kPtPageRows - 1u));       // (-1 stays -1)
                    t[k] += uint32_t(tokens);
                }
                if (kHeads == 2) __stcs(reinterpret_cast<longlong2*>(p), make_longlong2(v[0], v[kHeads - 1]));
                else __stcs(reinterpret_cast<long long*>(p), v[0]);
            }
        }
    }
}

}  // namespace skipkv

using namespace skipkv;

extern "C" int skipkv_page_tables(int32_t batch, int32_t n_kv_heads, int32_t max_pages, int32_t pool_pages, const int32_t* need,
                                  const int32_t* n_pages_in, int32_t* n_pages_out, int32_t* block_table, int32_t* free_ring,
                                  const int32_t* ring_in, int32_t* ring_out, uint32_t* status, void* stream) {
    if (batch <= 0 || n_kv_heads <= 0 || max_pages <= 0 || pool_pages <= 0) return SKIPKV_ERR_INVALID_ARG;
    if (!need || !n_pages_in || !n_pages_out || !block_table || !free_ring || !ring_in || !ring_out) return SKIPKV_ERR_INVALID_ARG;
    if (n_pages_in == n_pages_out || need == n_pages_out || ring_in == ring_out) return SKIPKV_ERR_INVALID_ARG;
    const int64_t slabs = int64_t(batch) * n_kv_heads;
    if (slabs > kPtMaxSlabs) {
        set_error_text("skipkv_page_tables: batch * n_kv_heads above 8192");
        return SKIPKV_ERR_UNSUPPORTED;
    }
    // rows of the pool, sums over the slabs, and places of the ring (free pages, then those that n_pages_in says are given back) in 32 bits
    if (int64_t(pool_pages) * SKIPKV_PAGE_ROWS > 0x7fffffff || slabs * max_pages + pool_pages > 0x7fffffff) return SKIPKV_ERR_UNSUPPORTED;
    const size_t smem = size_t(3 * slabs + 2) * 4;
    const int64_t want = (slabs * 16 + kPtWarps - 1) / kPtWarps;       // 16 warps to a slab, as far as the SMs go
    const int grid = int(want < num_sms() ? want : num_sms());
    SKIPKV_CUDA(launch_dependent(page_tables_kernel, dim3(grid), dim3(kPtThreads), smem, static_cast<cudaStream_t>(stream), int(slabs),
                                 int(max_pages), int(pool_pages), need, n_pages_in, n_pages_out, block_table, free_ring, ring_in, ring_out, status));
    return SKIPKV_OK;
}

extern "C" int skipkv_slot_map(int32_t batch, int32_t n_kv_heads, int32_t max_pages, const int32_t* block_table, const int32_t* n_pages,
                               const int32_t* start, const int32_t* new_off, int32_t n_new, int64_t* slots, void* stream) {
    if (batch <= 0 || n_kv_heads <= 0 || max_pages <= 0 || n_new < 0) return SKIPKV_ERR_INVALID_ARG;
    if (!block_table || !n_pages || !start || (!slots && n_new > 0)) return SKIPKV_ERR_INVALID_ARG;
    if (!new_off && n_new > batch) return SKIPKV_ERR_INVALID_ARG;
    if (int64_t(batch) * n_kv_heads > 0x7fffffff || int64_t(n_new) * n_kv_heads > 0x7fffff00) return SKIPKV_ERR_UNSUPPORTED;
    if (n_new == 0) return SKIPKV_OK;
    const bool two = n_kv_heads % 2 == 0 && (reinterpret_cast<uintptr_t>(slots) & 15) == 0;
    const int64_t work = int64_t(n_new) * n_kv_heads / (two ? 2 : 1);
    const int64_t want = (work + kPtThreads - 1) / kPtThreads, most = int64_t(num_sms()) * 2;
    const int grid = int(want < most ? want : most);
    SKIPKV_CUDA(launch_dependent(two ? slot_map_kernel<2> : slot_map_kernel<1>, dim3(grid), dim3(kPtThreads), 0, static_cast<cudaStream_t>(stream),
                                 int(batch), int(n_kv_heads), int(max_pages), block_table, n_pages, start, new_off, int(n_new), slots));
    return SKIPKV_OK;
}
