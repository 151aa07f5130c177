// Pages of the cache in other hands: keys and values moved between slots, rows of the table forked, pages given back.
#include "osc_internal.h"
#include "lds_dma.h"
#include "wave_util.h"

namespace osc {

// ---- keys and values from slot to slot -----------------------------------------------------------------------------------
// A wavefront has a group of pairs, one head of one layer, and its keys or its values.  It holds 64 pairs a round, those that move anything put
// together, and takes 32 (heads of 64: 64) of them at a time: a lane moves 16 bytes of a row, all loads of a batch before its stores, batches
// and rounds in order, so a slot may be read by a pair and written by a later one.  Bound by HBM where much is moved, by
// latency otherwise: the pairs' read, the rows' read, the store.  Stores go past the caches: plain ones stay there until the kernel's end, and are
// all written then.  150 (1000) groups of 32 pairs, 4 heads of 128 in 4 layers, 79 (524) MB read and written: 12 (103) us, with plain stores
// 30 (155), with loads past the caches too 16 (102).
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
struct MoveArgs {
    uint8_t *K, *V;
    int64_t layer;  // bytes from layer to layer
    int Hkv, lg, slots;
    const int32_t *src, *dst, *offsets;
    int64_t T;
    int N, per;  // without offsets: pairs of a group
};
template <int D>
__global__ __launch_bounds__(256) void cache_move_kernel(const MoveArgs p) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES, BATCH = 8;  // lanes a row, rows a load, loads in a batch
    const int lane = threadIdx.x & 63;
    const unsigned unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = unit / (unsigned)p.Hkv, h = unit - g * p.Hkv;
    if (g >= p.N) return;
    int64_t from = (int64_t)g * p.per, to = from + p.per;
    if (p.offsets) {
        from = p.offsets[g], to = p.offsets[g + 1];
        if (from < 0 || to > p.T) return;
    }
    uint8_t* C = (blockIdx.y & 1 ? p.V : p.K) + (blockIdx.y >> 1) * p.layer;
    auto row = [&](int slot) { return ((((int64_t)(slot >> p.lg) * p.Hkv + h) << p.lg) + (slot & ((1 << p.lg) - 1))) * (D * 2) + lane % LANES * 16; };
    for (int64_t t = from; t < to; t += 64) {
        int a = -1, b = -1;
        if (t + lane < to) a = p.src[t + lane], b = p.dst[t + lane];
        const bool moves = a != b && (uint32_t)a < (uint32_t)p.slots && (uint32_t)b < (uint32_t)p.slots;
        const uint64_t who = __ballot(moves);
        const int m = __popcll(who);
        // the k-th pair that moves to lane k; the others behind them
        const int below = __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0)), at = moves ? below : m + lane - below;
        a = __builtin_amdgcn_ds_permute(at * 4, a), b = __builtin_amdgcn_ds_permute(at * 4, b);
        for (int k = 0; k < m; k += ROWS * BATCH) {
            uint4v v[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int j = k + i * ROWS + lane / LANES, slot = __shfl(a, j & 63);
                if (j < m) v[i] = *reinterpret_cast<const uint4v*>(C + row(slot));
            }
            wait_vmcnt<0>();  // what a store overwrites has been read
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int j = k + i * ROWS + lane / LANES, slot = __shfl(b, j & 63);
                if (j < m) __builtin_nontemporal_store(v[i], reinterpret_cast<uint4v*>(C + row(slot)));
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

int launch_cache_move(void* K, void* V, int32_t n_layers, int64_t layer_stride, int64_t n_pages, int32_t Hkv, int lg, int32_t D, const int32_t* src, const int32_t* dst,
                      const int32_t* offsets, int32_t N, int64_t T, hipStream_t st) {
    MoveArgs p;
    p.K = static_cast<uint8_t*>(K), p.V = static_cast<uint8_t*>(V), p.layer = layer_stride * 2, p.Hkv = Hkv, p.lg = lg, p.slots = (int)(n_pages << lg);
    p.src = src, p.dst = dst, p.offsets = offsets, p.T = T, p.N = N, p.per = offsets ? 0 : (int)(T / N);
    const dim3 grid((unsigned)(((int64_t)N * Hkv + 3) / 4), (unsigned)n_layers * 2);
    if (D == 64) cache_move_kernel<64><<<grid, 256, 0, st>>>(p);
    else cache_move_kernel<128><<<grid, 256, 0, st>>>(p);
    return check_launch("osc_cache_move");
}

// Sums over the lanes below and this one of a workgroup of NT; `part`: a number a wavefront, in LDS.  All threads take part.
template <int NT>
__device__ __forceinline__ int block_scan(int v, int* part, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = wave_scan(v, [](int a, int b) { return a + b; });
    __syncthreads();  // `part` may still be read for a scan before
    if (lane == 63) part[wave] = v;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) v += part[w];
        total += part[w];
    }
    return v;
}

// ---- rows of the table forked -------------------------------------------------------------------------------------------------
// Every workgroup decides all forks for itself, in LDS (which rows are forked from, the first fork into every row, running sum of the
// pages), then its wavefronts carry out their share: no word is passed between workgroups, and what they read (lengths and
// rows that are forked from) no fork writes.  Bound by latency, as osc_page_slots: forks, lengths, rows.  So what depends on no decision is asked
// for first: the list's end, lengths and the first pages of the rows (150 forks of 512 requests 6.6 us, asked for in order 7.5).  None of these is
// written meanwhile: a row that is forked from is no fork's to write.
template <int NT>
__global__ __launch_bounds__(NT) void page_fork_kernel(const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int N, int B, int lg, int32_t* kv_lens, int32_t* table,
                                                       int64_t ldt, int32_t* refs, int64_t n_pages, const int32_t* __restrict__ free_pages, int64_t n_pool,
                                                       const int32_t* __restrict__ n_free_ptr, int32_t* __restrict__ src_slots, int32_t* __restrict__ dst_slots,
                                                       int32_t* __restrict__ info) {
    extern __shared__ int32_t lds[];
    // first fork into a row, -1 for a row that is forked from; a fork's page: its place from the list's end, -1 none, -2 refused; the list's end
    int32_t *first = lds, *page_at = first + B, *fresh = page_at + N;
    __shared__ int part[NT / 64];
    __shared__ int sums[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ps1 = (1 << lg) - 1;
    const int n_free = (int)max((int64_t)0, min((int64_t)*n_free_ptr, n_pool));
    if (tid < 3) sums[tid] = 0;
    for (int b = tid; b < B; b += NT) first[b] = 0x7fffffff;
    auto length = [&](int a) { return (int)min((int64_t)max(kv_lens[a], 0), min(ldt << lg, (int64_t)0x7fffffff)); };
    const int per = (N + NT - 1) / NT, f0 = min(N, tid * per), f1 = min(N, f0 + per);
    const int w0 = blockIdx.x * (NT / 64) + wave;
    // of this thread's first fork, and of its wavefront's first one
    int a0 = -1, to0 = -1, len0 = 0, row0 = -1, into0 = -1, L0 = 0, page0 = -1, last0 = -1;
    int fresh0 = 0;
    if (N > 0) {
        const int fa = min(f0, N - 1), fw = min(w0, N - 1);
        a0 = src[fa], to0 = dst[fa], row0 = src[fw], into0 = dst[fw];
        if (tid < min(N, n_free)) fresh0 = free_pages[n_free - 1 - tid];
        if (B > 0) {  // loads without conditions, which the compiler would wait for one by one
            len0 = kv_lens[min((uint32_t)a0, (uint32_t)B - 1)];
            L0 = length(min((uint32_t)row0, (uint32_t)B - 1));
            const int32_t* rows = ldt ? table + min((uint32_t)row0, (uint32_t)B - 1) * ldt : kv_lens;
            page0 = rows[min((int64_t)lane, max(ldt - 1, (int64_t)0))], last0 = rows[min((int64_t)(L0 >> lg), max(ldt - 1, (int64_t)0))];
        }
    }
    __syncthreads();
    for (int f = tid; f < N; f += NT) {
        const int a = per == 1 ? a0 : src[f], b = per == 1 ? to0 : dst[f];
        if ((uint32_t)b < (uint32_t)B) atomicMin(&first[b], f);
        if ((uint32_t)a < (uint32_t)B) atomicMin(&first[a], -1);
    }
    for (int f = tid; f < min(N, n_free); f += NT) fresh[f] = f == tid ? fresh0 : free_pages[n_free - 1 - f];
    __syncthreads();
    auto valid = [&](int f, int& L) {
        const int a = f == f0 ? a0 : src[f], b = f == f0 ? to0 : dst[f];
        if ((uint32_t)a >= (uint32_t)B || (uint32_t)b >= (uint32_t)B || first[b] != f) return false;
        L = max(f == f0 ? len0 : kv_lens[a], 0);
        return L <= ldt << lg;
    };
    int mine = 0, L;
    for (int f = f0; f < f1; ++f) mine += valid(f, L) && (L & ps1);
    int total;
    int at = block_scan<NT>(mine, part, total) - mine;
    int taken = 0, refused = 0, shared = 0;
    for (int f = f0; f < f1; ++f) {
        const bool ok = valid(f, L);
        const int need = ok && (L & ps1) ? 1 : 0;
        page_at[f] = !ok || (need && at >= n_free) ? -2 : need ? at : -1;
        at += need;
        if (page_at[f] == -2) ++refused;
        else taken += need, shared += L >> lg;
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        if (taken) atomicAdd(&sums[0], taken);
        if (refused) atomicAdd(&sums[1], refused);
        if (shared) atomicAdd(&sums[2], shared);
        __syncthreads();
        if (tid == 0) info[0] = n_free - sums[0], info[1] = sums[0], info[2] = sums[1], info[3] = sums[2];
    }
    for (int f = w0; f < N; f += gridDim.x * (NT / 64)) {
        const int place = __builtin_amdgcn_readfirstlane(page_at[f]);
        int32_t *s = src_slots + ((int64_t)f << lg), *d = dst_slots + ((int64_t)f << lg);
        int used = 0, from = -1, to = -1;
        if (place != -2) {
            const int from_row = f == w0 ? row0 : src[f], to_row = f == w0 ? into0 : dst[f], L = f == w0 ? L0 : length(from_row), full = L >> lg;
            const int32_t* rows = table + from_row * ldt;
            int32_t* mine_row = table + to_row * ldt;
            for (int j = lane; j < full; j += 64) {
                const int page = f == w0 && j == lane ? page0 : rows[j];
                mine_row[j] = page;
                if ((uint64_t)(int64_t)page < (uint64_t)n_pages) atomicAdd(&refs[page], 1);
            }
            if (place >= 0) {
                used = L & ps1, from = f == w0 ? last0 : rows[full], to = fresh[place];
                if (lane == 0) mine_row[full] = to;
                if ((uint64_t)(int64_t)from >= (uint64_t)n_pages || (uint64_t)(int64_t)to >= (uint64_t)n_pages) used = 0;  // nothing that a cache has
            }
            if (lane == 0) kv_lens[to_row] = L;
        }
        for (int j = lane; j <= ps1; j += 64) {
            s[j] = j < used ? (from << lg) + j : -1;
            d[j] = j < used ? (to << lg) + j : -1;
        }
    }
}

int launch_page_fork(const int32_t* src, const int32_t* dst, int32_t N, int32_t B, int lg, int32_t* kv_lens, int32_t* table, int64_t ldt, int32_t* refs, int64_t n_pages,
                     const int32_t* free_pages, int64_t n_pool, const int32_t* n_free, int32_t* src_slots, int32_t* dst_slots, int32_t* info, hipStream_t st) {
    const size_t lds = ((size_t)B + 2 * N) * 4;
    const int64_t most = cu_count();
    if (most <= 0) return fail(OSC_ERR_HIP, "osc_page_fork: cannot read the device");
    auto go = [&](auto kernel, int nt, LdsReserved& r) {
        if (lds > 48 * 1024) {
            const int rc = reserve_lds((const void*)kernel, lds, r);
            if (rc) return rc;
        }
        int64_t wgs = ((int64_t)N + nt / 64 - 1) / (nt / 64);
        wgs = wgs < 1 ? 1 : wgs > most ? most : wgs;
        kernel<<<dim3((unsigned)wgs), nt, lds, st>>>(src, dst, N, B, lg, kv_lens, table, ldt, refs, n_pages, free_pages, n_pool, n_free, src_slots, dst_slots, info);
        return check_launch("osc_page_fork");
    };
    static LdsReserved r256, r1024;
    if (N <= 256) return go(page_fork_kernel<256>, 256, r256);
    return go(page_fork_kernel<1024>, 1024, r1024);
}

// ---- pages given back ---------------------------------------------------------------------------------------------------------
// One workgroup: running sums of the requests' pages that go, one page a thread after that; a page that has lost its last holder
// is a bit in LDS, and the bits' order is the list's, so the list is the same in every run and a page enters it once.  Caches of
// more pages than bits are done range by range.  Bound by latency: lengths, sum, table, holders, bits, list.
// Where no request lets more than FEW_PAGES go, a thread has its requests' pages itself, all of one on their way at once, and nothing is summed or
// searched: 150 of 512 requests of up to 5 pages 6.6 us, summed and searched 7.5 (a launch alone is 2 to 3); 16 requests of up to 19 pages 4.6.  Many
// pages are many turns of one workgroup: 150 requests of 250, 500 and 1500 pages 124, 259 and 755 us.
constexpr int FREE_NT = 1024, FREE_WORDS = 16384;  // 2^19 pages a range, 64 KB
constexpr int FEW_PAGES = 8;
__global__ __launch_bounds__(FREE_NT, 1) void page_free_kernel(const int32_t* __restrict__ kv_lens, const int32_t* __restrict__ new_lens, int B, int lg, const int32_t* __restrict__ table,
                                                            int64_t ldt, int32_t* refs, int64_t n_pages, int32_t* free_pages, int64_t n_pool, const int32_t* __restrict__ n_free_ptr,
                                                            int32_t* __restrict__ info) {
    extern __shared__ uint32_t bits[];  // [words of a range], then the requests' running sums
    __shared__ int part[FREE_NT / 64];
    __shared__ int sums[2];  // releases that left a page to others; that were of no page, or of one that was free already
    const int tid = threadIdx.x, ps1 = (1 << lg) - 1;
    const int range_words = (int)min((n_pages + 31) / 32, (int64_t)FREE_WORDS);
    int32_t* before = reinterpret_cast<int32_t*>(bits + range_words);
    const int n_free = (int)max((int64_t)0, min((int64_t)*n_free_ptr, n_pool));
    if (tid < 2) sums[tid] = 0;
    const int per = (B + FREE_NT - 1) / FREE_NT, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int32_t* news = new_lens ? new_lens : kv_lens;  // always read, so that no branch parts the two loads
    auto span = [&](int b, int& from) {  // pages of request b that go
        const int had = kv_lens[b], left = news[b];
        const int64_t have = min(((int64_t)max(had, 0) + ps1) >> lg, ldt), keep = new_lens ? ((int64_t)max(left, 0) + ps1) >> lg : 0;
        from = (int)keep;
        return (int)max(have - keep, (int64_t)0);
    };
    int mine = 0, most = 0, from = 0, total = 0;
    for (int b = b0; b < b1; ++b) {
        const int n = span(b, from);
        mine += n, most = max(most, n);
    }
    const bool many = __syncthreads_or(most > FEW_PAGES) || n_pages == 0;
    if (many) {
        int at = block_scan<FREE_NT>(mine, part, total) - mine;
        for (int b = b0; b < b1; ++b) {
            before[b] = at;
            at += span(b, from);
        }
    }
    int entered = 0, lost = 0;  // pages on the list by now, pages that it had no room for
    for (int64_t base = 0; base < n_pages; base += (int64_t)range_words * 32) {  // no pages: range_words is 0, and so are the rounds
        for (int w = tid; w < range_words; w += FREE_NT) bits[w] = 0;
        __syncthreads();
        int kept = 0, extra = 0;
        const uint32_t pages = (uint32_t)n_pages, from_page = (uint32_t)base, here = (uint32_t)min(n_pages - base, (int64_t)range_words * 32);
        const int once = base == 0;  // entries of no page are counted then
        auto marked = [&](uint32_t page) -> int {  // it was already
            const uint32_t i = page - from_page;
            return atomicOr(&bits[i >> 5], 1u << (i & 31)) >> (i & 31) & 1;
        };
        for (int b = b0; b < b1 && !many; ++b) {
            const int n = per == 1 ? mine : span(b, from);  // one request a thread: `from` is still its own
            if (n == 0) continue;
            uint32_t page[FEW_PAGES];
            int others[FEW_PAGES];
#pragma unroll
            for (int j = 0; j < FEW_PAGES; ++j) page[j] = table[b * ldt + from + min(j, n - 1)];
            __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0), here once: behind conditions the compiler would wait before each
#pragma unroll
            for (int j = 0; j < FEW_PAGES; ++j) {
                if (j < n && page[j] >= pages) extra += once;
                if (j >= n) page[j] = 0xffffffffu;
            }
#pragma unroll
            for (int j = 0; j < FEW_PAGES; ++j) {
                others[j] = 0;
                if (refs && page[j] - from_page < here) others[j] = atomicAdd(&refs[page[j]], -1);
            }
#pragma unroll
            for (int j = 0; j < FEW_PAGES; ++j)
                if (page[j] - from_page < here) {
                    if (others[j] > 0) ++kept;
                    else extra += marked(page[j]);
                }
        }
        for (int e = tid; e < total; e += FREE_NT) {
            int lo = 0, hi = B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (before[mid] <= e) lo = mid;
                else hi = mid;
            }
            span(lo, from);
            const uint32_t page = table[lo * ldt + from + (e - before[lo])];
            if (page >= pages) extra += once;
            if (page - from_page < here) {
                if (refs && atomicAdd(&refs[page], -1) > 0) ++kept;
                else extra += marked(page);
            }
        }
        if (kept) atomicAdd(&sums[0], kept);
        if (extra) atomicAdd(&sums[1], extra);
        __syncthreads();
        const int wper = (range_words + FREE_NT - 1) / FREE_NT, w0 = min(range_words, tid * wper), w1 = min(range_words, w0 + wper);
        int n = 0;
        for (int w = w0; w < w1; ++w) n += __popc(bits[w]);
        int found;
        int place = block_scan<FREE_NT>(n, part, found) - n + entered;
        for (int w = w0; w < w1; ++w)
            for (uint32_t left = bits[w]; left; left &= left - 1) {
                const int64_t page = base + w * 32 + __ffs((int)left) - 1;
                if (refs) refs[page] = 0;
                if (n_free + (int64_t)place < n_pool) free_pages[n_free + place] = (int32_t)page;
                ++place;
            }
        entered += found;
        __syncthreads();
    }
    if (n_pages == 0 && tid == 0) sums[1] = total;
    lost = (int)max((int64_t)n_free + entered - n_pool, (int64_t)0);
    if (tid == 0) info[0] = n_free + entered - lost, info[1] = entered - lost, info[2] = sums[0], info[3] = sums[1] + lost;
}

int launch_page_free(const int32_t* kv_lens, const int32_t* new_lens, int32_t B, int lg, const int32_t* table, int64_t ldt, int32_t* refs, int64_t n_pages, int32_t* free_pages,
                     int64_t n_pool, const int32_t* n_free, int32_t* info, hipStream_t st) {
    const size_t lds = (size_t)((n_pages + 31) / 32 < FREE_WORDS ? (n_pages + 31) / 32 : FREE_WORDS) * 4 + (size_t)B * 4;
    static LdsReserved r;
    if (lds > 48 * 1024) {
        const int rc = reserve_lds((const void*)page_free_kernel, lds, r);
        if (rc) return rc;
    }
    page_free_kernel<<<dim3(1), FREE_NT, lds, st>>>(kv_lens, new_lens, B, lg, table, ldt, refs, n_pages, free_pages, n_pool, n_free, info);
    return check_launch("osc_page_free");
}

}  // namespace osc
