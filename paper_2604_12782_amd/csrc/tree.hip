// Trees of drafted tokens: which of them a row sees and where it stands, and the path that the model agrees with.
//
// A request's new tokens are rows q_offsets[b] .. of a step; row i continues row parents[i] < i of the same request, or nothing but
// what is cached (any other number).  A wavefront has a request; lanes past the last request's rows fill the padding.  Both
// kernels are bound by latency: offsets, the rows' numbers, a few steps between lanes, the stores.  Masks of one tree of 8 tokens 1.8 us, of 48 of 32 tokens
// 4.0, of 6 of 97 tokens with two words 4.6; paths of 4 trees of 8 tokens 2.8 us, of 200 of 24 4.0; a launch alone is 2 to 3.
#include "osc_internal.h"

namespace osc {

struct Rows {
    int q0, n;
};
// rows and length of request b, no rows if its offsets fall or leave [0, T]
__device__ __forceinline__ Rows rows_of(const int32_t* q_offsets, const int32_t* kv_lens, int b, int64_t T, int& L) {
    Rows r{q_offsets[b], 0};
    const int end = q_offsets[b + 1];
    L = kv_lens[b];
    asm volatile("" : : "s"(r.q0), "s"(end), "s"(L));  // asked for together: the compiler would read each at the branch that needs it
    if (r.q0 >= 0 && end >= r.q0 && end <= T) r.n = end - r.q0;
    return r;
}
// rows that no request has: before the first offset and from the last on; f(row) for each
template <class F>
__device__ __forceinline__ void padding(const int32_t* q_offsets, int B, int64_t T, int64_t at, int64_t step, F f) {
    int from = 0, to = 0;
    if (B) {
        from = q_offsets[0], to = q_offsets[B];
        asm volatile("" : : "s"(from), "s"(to));
    }
    const int64_t first = min(max((int64_t)from, (int64_t)0), T), last = min(max((int64_t)to, first), T);
    for (int64_t i = at; i < first + T - last; i += step) f(i < first ? i : i - first + last);
}
constexpr int PAD_WGS = 8;

// ---- bits and positions -----------------------------------------------------------------------------------------------
// 64 rows at a time: by doubling, a lane gathers the bits of its ancestors among the 64 and the first one outside them, whose words
// are there already.
__global__ __launch_bounds__(64) void tree_mask_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ q_offsets, const int32_t* __restrict__ kv_lens, int B,
                                                       int64_t T, int pos_base, int words, uint64_t* __restrict__ mask, int64_t ldm, int32_t* __restrict__ positions) {
    extern __shared__ uint64_t seen[];  // [rows before the last 64][words], where words > 1
    const int lane = threadIdx.x;
    if ((int)blockIdx.x >= B) {
        padding(q_offsets, B, T, (blockIdx.x - B) * 64 + lane, PAD_WGS * 64, [&](int64_t t) {
            for (int w = 0; w < words; ++w) mask[t * ldm + w] = 0;
            positions[t] = -1;
        });
        return;
    }
    const int b = blockIdx.x;
    asm volatile("" : : "s"(parents));  // the argument too
    int L;
    const Rows r = rows_of(q_offsets, kv_lens, b, T, L);
    const int64_t start = (int64_t)pos_base + max(L, 0) - r.n;
    auto place = [&](int i, int64_t depth) { positions[r.q0 + i] = (int)max(min(start + depth, (int64_t)0x7fffffff), (int64_t)-1); };
    if (r.n > 64 * words) {  // no tree
        for (int i = lane; i < r.n; i += 64) {
            for (int w = 0; w < words; ++w) mask[(int64_t)(r.q0 + i) * ldm + w] = 0;
            place(i, i);
        }
        return;
    }
    for (int c = 0; c * 64 < r.n; ++c) {
        const int i = c * 64 + lane;
        int up = i < r.n ? parents[r.q0 + i] : -1;
        if (up < 0 || up >= i) up = -1;
        uint64_t mine = 1ull << lane;
        const int base = c * 64;
#pragma unroll
        for (int d = 0; d < 6; ++d) {
            const bool inside = up >= base;
            const int from = inside ? up - base : lane;
            const uint32_t lo = __shfl((uint32_t)mine, from), hi = __shfl((uint32_t)(mine >> 32), from);
            const int next = __shfl(up, from);
            if (inside) mine |= (uint64_t)hi << 32 | lo, up = next;
        }
        int depth = __popcll(mine) - 1;
        uint64_t* out = mask + (int64_t)(r.q0 + min(i, r.n - 1)) * ldm;
        for (int w = 0; w < words; ++w) {
            const uint64_t one = w == c ? mine : w < c && up >= 0 ? seen[up * words + w] : 0;
            if (w < c) depth += __popcll(one);
            if (i < r.n) {
                out[w] = one;
                if (words > 1 && base + 64 < r.n) seen[i * words + w] = one;
            }
        }
        if (i < r.n) place(i, depth);
        __syncthreads();  // the next rows read `seen`
    }
}

int launch_tree_mask(const int32_t* parents, const int32_t* q_offsets, const int32_t* kv_lens, int32_t B, int64_t T, int32_t pos_base, int32_t words, uint64_t* mask,
                     int64_t ldm, int32_t* positions, hipStream_t st) {
    const size_t lds = words > 1 ? (size_t)(words - 1) * 64 * words * 8 : 0;  // 28 KB at most
    tree_mask_kernel<<<dim3((unsigned)(B + PAD_WGS)), 64, lds, st>>>(parents, q_offsets, kv_lens, B, T, pos_base, words, mask, ldm, positions);
    return check_launch("osc_tree_mask");
}

// ---- the accepted path ---------------------------------------------------------------------------------------------------
// From row `at` the path goes on at the lowest row that continues it with the token chosen there (or with a given one, number below
// 0).  Rows that continue the row before them so are marked for 64 rows at once: a run of marks behind `at` is the path as far as
// it goes, since no row is lower; otherwise the rows are searched.  So a chain is a step, a branch another.
__global__ __launch_bounds__(64) void tree_accept_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ tokens, const int32_t* __restrict__ choices, int64_t ldc,
                                                         const int32_t* __restrict__ q_offsets, const int32_t* kv_lens, const int32_t* __restrict__ slots, int B, int64_t T,
                                                         int32_t* __restrict__ path, int32_t* __restrict__ n_accepted, int32_t* __restrict__ next_tokens,
                                                         int32_t* kv_lens_out, int32_t* __restrict__ src_slots) {
    const int lane = threadIdx.x;
    if ((int)blockIdx.x >= B) {
        padding(q_offsets, B, T, (blockIdx.x - B) * 64 + lane, PAD_WGS * 64, [&](int64_t t) { path[t] = src_slots[t] = -1; });
        return;
    }
    const int b = blockIdx.x;
    int L;
    const Rows r = rows_of(q_offsets, kv_lens, b, T, L);
    const int32_t *par = parents + r.q0, *tok = tokens + r.q0, *chosen = choices + r.q0 * ldc;
    int count = 0, next = -1, L_out = L;
    int chunk = -1, up = -1, token = 0, choice = 0, slot = -1;  // of the 64 rows that the lanes hold, all read at once
    uint64_t runs = 0;
    auto hold = [&](int c) {
        if (c == chunk) return;
        chunk = c;
        const int i = c * 64 + lane, row = min(i, r.n - 1);
        const bool there = i < r.n;
        up = par[row], token = tok[row], choice = chosen[(int64_t)row * ldc], slot = slots[r.q0 + row];
        const int before = c ? chosen[(int64_t)(i - lane - 1) * ldc] : 0, below = __shfl_up(choice, 1);
        if (!there) up = -1;
        runs = __ballot(there && i > 0 && up == i - 1 && (token < 0 || token == (lane ? below : before)));
    };
    if (r.n > 0) hold(0);
    if (r.n > 0 && __builtin_amdgcn_readlane(slot, 0) >= 0) {  // otherwise the request got no pages: its tokens are not cached
        auto put = [&](int k, int i, int from) {
            path[r.q0 + k] = i;
            src_slots[r.q0 + k] = from;
        };
        int at = 0;
        count = 1;
        if (lane == 0) put(0, 0, slot);
        next = __builtin_amdgcn_readlane(choice, 0);
        while (at + 1 < r.n) {
            hold((at + 1) >> 6);
            const int bit = (at + 1) & 63;
            const uint64_t ahead = runs >> bit;
            int run = ~ahead ? __ffsll((unsigned long long)~ahead) - 1 : 64;
            run = min(run, 64 - bit);
            if (run > 0) {
                if (lane >= bit && lane < bit + run) put(count + lane - bit, chunk * 64 + lane, slot);
                count += run, at += run;
            } else {
                int found = -1;
                for (int c = (at + 1) >> 6; c * 64 < r.n && found < 0; ++c) {
                    hold(c);
                    const int i = c * 64 + lane;
                    const uint64_t who = __ballot(i > at && i < r.n && up == at && (token < 0 || token == next));
                    if (who) found = c * 64 + __ffsll((unsigned long long)who) - 1;
                }
                if (found < 0) break;
                at = found;
                const int from = __builtin_amdgcn_readlane(slot, at & 63);
                if (lane == 0) put(count, at, from);
                ++count;
            }
            next = __builtin_amdgcn_readlane(choice, at & 63);
        }
        L_out = L - r.n + count;
    }
    for (int i = count + lane; i < r.n; i += 64) path[r.q0 + i] = src_slots[r.q0 + i] = -1;
    if (lane == 0) n_accepted[b] = count, next_tokens[b] = next, kv_lens_out[b] = L_out;
}

int launch_tree_accept(const int32_t* parents, const int32_t* tokens, const int32_t* choices, int64_t ldc, const int32_t* q_offsets, const int32_t* kv_lens, const int32_t* slots,
                       int32_t B, int64_t T, int32_t* path, int32_t* n_accepted, int32_t* next_tokens, int32_t* kv_lens_out, int32_t* src_slots, hipStream_t st) {
    tree_accept_kernel<<<dim3((unsigned)(B + PAD_WGS)), 64, 0, st>>>(parents, tokens, choices, ldc, q_offsets, kv_lens, slots, B, T, path, n_accepted, next_tokens,
                                                                     kv_lens_out, src_slots);
    return check_launch("osc_tree_accept");
}

}  // namespace osc
