// Log probabilities of given tokens, entropy and top alternatives of rows of logits.
//
//   p_j = exp(scale x_j) / sum,  lse = log sum_j exp(scale x_j),  entropy = -sum_j p_j log p_j = lse - sum_j p_j scale x_j
//
// One pass over the logits.  A lane keeps, for what it has seen: a base b (a logit), S = sum of w_j = 2^(c x_j - B) and U = sum of
// w_j (c x_j - B), c = scale log2 e, B = c b rounded: one fused operation gives the power, and what B was rounded by is known at the end.
// The base is the lane's first chunk's largest logit and follows only when a chunk's weights reach 2^8, so sums are rarely scaled; a change of
// base by d = B - B' turns (S, U) into 2^d (S, U + S d), which is also how lanes, wavefronts and parts of a row are joined.  Then log p_j
// = scale (x_j - b) - log S and the entropy is log S - ln 2 U / S; logits enter by their distance from the base alone, so large
// ones lose nothing.  Everything is single precision.  B is rounded by up to half its last place, and the base's own weight is 2 to that:
// 2^-5 at 2^20, but 64 at 1e9 and infinite or 0 beyond 1e10.  So from LP_FAR on (fills for tokens that may not come, rows of large logits) powers are
// made of c (x_j - b), relative to c b itself, and the usual path is left.
//
// The top k.  A logit's key is its value in the order of unsigned numbers, then its index, lower ones first: 64 bits, no two alike.  In
// the pass a lane keeps its largest logit, and a bit for every chunk whose largest one k lanes of the wavefront had not passed yet.  After the
// pass 256 groups of lanes have a largest logit each, and no logit below the k-th of them is among the top k: the few lanes whose largest one
// reaches that read their marked chunks again (from L2; one chunk, where no other of the lane's reaches the bound: 100 rows 15.8 -> 14.9 us), and a wavefront counts the ranks of what they find.  Should that be more than LDS
// has room for (many equal logits, a row with fewer than k tokens that can come), wavefronts walk their chunks once more and rank as they go
// (2048 rows of 131072 where thousands are equal to the largest: 317 us, not 95).
//
// Bounds.  2048 rows of 131072 bf16 logits, top 5: 95 us, 5.6 TB/s; 78 would be a reading pass.  Without the top 86; 4 bytes a logit 6.5 TB/s: a bf16 logit takes ten
// operations, one of them a power.  Reads past the caches are 8 % faster (103 with plain ones): nothing here is read twice but the marked
// chunks.  511 rows of 32000 10.1 us: 33 MB in about 4, the start and the end of a workgroup.  100 rows of 50001, four bytes each, top 20, 15.2: one
// workgroup a CU on 100 of them, 25 GB/s each; the top's three steps (largest logits, bound, marked chunks) are 4 of it.  One row of 131072: 8.5 and 3.1 us for the
// two kernels.  Ranking candidates on the way instead of marking them: 100 rows 30 us, 2048 126.
// Masked logits.  Finite fills cost nothing (half or nine tenths of the 2048 rows' logits -1e4, -1e10 or -1e30: 90 to 101 us).  A chunk with -infinity leaves
// the usual path and makes its powers twice, since 0 times -infinity is NaN: with half of the logits -infinity here and there 145 us, nine tenths 142, all behind the
// first half 114, behind the first tenth 134.
#include <type_traits>

#include "osc_internal.h"

namespace osc {

struct LogpArgs {
    const uint8_t* X;
    int64_t T, V, ldl;  // ldl in elements
    float scale, c;
    const int32_t* tokens;
    int n_tok, k;
    float* lp;
    int32_t* ids;
    float *top, *lse, *entropy;
    int splits;  // parts of a row
    float4* stats;   // workspace: of a part of a row, base, S, U
    uint64_t* keys;  // and its k best, best first
};

constexpr int LP_BUF = 128, LP_MAX_SPLITS = 64, LP_FOUND = 512;
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
constexpr float LP_FAR = 0x1p20f, LN2 = 0.69314718055994531f;

struct Weights {
    float b, S, U;
};
__device__ __forceinline__ bool is_far(float B) { return !(fabsf(B) < LP_FAR); }
// turned to base nb >= b; nothing seen is b = -infinity, S = U = 0.  Weights are relative to 2^B, of a far base to 2^(c b): d is the difference of the
// two as they are, in one rounding each.
__device__ __forceinline__ void rebase(Weights& w, float nb, float c) {
#pragma clang fp contract(off)  // products are rounded before their difference, as B is
    if (w.b == -INFINITY) {
        w.S *= nb == INFINITY ? NAN : 0.0f, w.U = 0.0f;  // 0 stays 0, NaN stays NaN
    } else {
        const float from = w.b * c, to = nb * c;
        const float d = fmaxf(is_far(from) ? is_far(to) ? (w.b - nb) * c : fmaf(w.b, c, -to) : is_far(to) ? fmaf(-nb, c, from) : from - to, -1e4f);
        const float f = __builtin_amdgcn_exp2f(d);
        w.U = (w.U + w.S * d) * f;
        w.S *= f;
    }
    w.b = nb;
}
// over the wavefront, on the vector ALU: four steps inside rows of 16 lanes, then the rows' last lanes; every lane gets the last one's
template <class T, class Op>
__device__ __forceinline__ T wave_reduce(T v, T none, Op op) {
    auto from = [&](auto ctrl, auto rows) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
    };
    using std::integral_constant;
    v = op(v, from(integral_constant<int, 0x111>(), integral_constant<int, 0xF>()));
    v = op(v, from(integral_constant<int, 0x112>(), integral_constant<int, 0xF>()));
    v = op(v, from(integral_constant<int, 0x114>(), integral_constant<int, 0xF>()));
    v = op(v, from(integral_constant<int, 0x118>(), integral_constant<int, 0xF>()));
    v = op(v, from(integral_constant<int, 0x142>(), integral_constant<int, 0xA>()));
    v = op(v, from(integral_constant<int, 0x143>(), integral_constant<int, 0xC>()));
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ uint32_t wave_top(uint32_t v) { return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }); }
__device__ __forceinline__ Weights wave_joined(Weights w, float c) {
    rebase(w, wave_max(w.b), c);
    return Weights{w.b, wave_sum(w.S), wave_sum(w.U)};
}

// Values in the order of unsigned numbers: NaN aside, -infinity is 0x007fffff; 0 is below all.  Zeros are alike.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __builtin_bit_cast(float, o & 0x80000000u ? o ^ 0x80000000u : ~o); }

__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// a barrier for LDS alone: it does not wait for what is on its way from memory
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
// how many of keys[0 .. n) are above `key`
__device__ __forceinline__ int above(const uint64_t* keys, int n, uint64_t key) {
    int r = 0, j = 0;
    for (; j + 8 <= n; j += 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) r += keys[j + i] > key;
    for (; j < n; ++j) r += keys[j] > key;
    return r;
}

// A wavefront's candidates, in LDS of its own.
struct Best {
    uint64_t* buf;  // [LP_BUF]
    int count, k;
    uint64_t least;  // the k-th best of those that were ranked, 0 before there are k
};
// the best k in order, from the first place on
__device__ __forceinline__ void rank(Best& s, int lane) {
    wave_lds_order();
    const uint64_t a = lane < s.count ? s.buf[lane] : 0, b = 64 + lane < s.count ? s.buf[64 + lane] : 0;
    const int ra = above(s.buf, s.count, a), rb = s.count > 64 ? above(s.buf, s.count, b) : 0;
    wave_lds_order();
    if (a && ra < s.k) s.buf[ra] = a;
    if (b && rb < s.k) s.buf[rb] = b;
    wave_lds_order();
    s.count = min(s.count, s.k);
    if (s.count == s.k) s.least = s.buf[s.k - 1];
}
// at most 64 before, at most 128 after
__device__ __forceinline__ void append(Best& s, uint64_t key, uint64_t who, bool take) {
    if (take) s.buf[s.count + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key;
    s.count += __popcll(who);
}
// A number that k of the lanes' N numbers or more reach, and hardly more than k: bisection between the smallest and the largest.
template <int N>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&top)[N], int k) {
    uint32_t lo = top[0], hi = top[0];
#pragma unroll
    for (int i = 1; i < N; ++i) lo = min(lo, top[i]), hi = max(hi, top[i]);
    lo = ~wave_top(~lo), hi = wave_top(hi);
    for (int step = 0; step < 16 && lo < hi; ++step) {
        const uint32_t at = hi - (hi - lo) / 2;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot(top[i] >= at));
        if (n < k) hi = at - 1;
        else lo = at;
        if (n >= k && n <= k + k / 4 + 4) break;
    }
    return lo;
}
// one of N, by number
__device__ __forceinline__ float either(bool second, float a, float b) { return second ? b : a; }
template <int N>
__device__ __forceinline__ float pick(const float (&v)[N], int e) {
    if constexpr (N == 2) {
        return either(e & 1, v[0], v[1]);
    } else {
        float half[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) half[i] = either(e & 1, v[2 * i], v[2 * i + 1]);
        return pick(half, e >> 1);
    }
}

template <bool F32>
__device__ __forceinline__ float logit(const uint8_t* x, int64_t i) {
    return F32 ? reinterpret_cast<const float*>(x)[i] : __builtin_bit_cast(float, (uint32_t)reinterpret_cast<const uint16_t*>(x)[i] << 16);
}
// The i-th token given to a row (-1: none), and its logit.
__device__ __forceinline__ int32_t given(const LogpArgs& p, int64_t row, int i) { return i < p.n_tok ? p.tokens[row * p.n_tok + i] : -1; }
template <bool F32>
__device__ __forceinline__ float given_logit(const LogpArgs& p, const uint8_t* x, int32_t t) { return (uint32_t)t < (uint64_t)p.V ? logit<F32>(x, t) : 0.0f; }
// One row's results, from all of it, by one wavefront; `sorted`: its k best; the token given to this lane and its logit.
template <bool F32>
__device__ __forceinline__ void finish(const LogpArgs& p, int64_t row, const Weights& w, const uint64_t* sorted, int lane, const uint8_t* x, int32_t token, float its) {
    const bool bad = !(w.S < INFINITY) || w.b == INFINITY;  // NaN or infinity among the logits
    const float B = w.b * p.c, off = is_far(B) ? 0.0f : fmaf(w.b, p.c, -B);
    const float logS = logf(w.S), logZ = logS - off * LN2;  // of the powers of c (x - b)
    auto log_p = [&](float v) {
        const float far = v - w.b, d = far == -INFINITY && v > -INFINITY ? fmaf(p.scale, v, -(p.scale * w.b)) : p.scale * far;  // a distance past the type's range, times scale perhaps inside it
        return bad ? NAN : w.S > 0.0f ? d - logZ : -INFINITY;
    };
    if (lane == 0) {
        if (p.lse) p.lse[row] = bad ? NAN : w.S > 0.0f ? fmaf(p.scale, w.b, logZ) : -INFINITY;
        if (p.entropy) p.entropy[row] = bad ? NAN : w.S > 0.0f ? logS - w.U / w.S * LN2 : 0.0f;
    }
    for (int i = lane; i < p.n_tok; i += 64) {
        if (i >= 64) token = given(p, row, i), its = given_logit<F32>(p, x, token);
        p.lp[row * p.n_tok + i] = (uint32_t)token < (uint64_t)p.V ? log_p(its) : 0.0f;
    }
    if (lane < p.k) {
        const uint64_t key = sorted[lane];
        p.ids[row * p.k + lane] = bad ? -1 : (int32_t)~(uint32_t)key;
        p.top[row * p.k + lane] = log_p(value_of((uint32_t)(key >> 32)));
    }
}

// A workgroup takes a part of a row (all of it where there are many rows), its wavefronts chunks in turn.  A chunk is NV times 16 bytes a
// lane, from the row's first 16-byte boundary on; logits before the first and after the last whole 16
// bytes are the first wavefront's, after its chunks, as one more, one logit a lane.
template <bool F32, int NV>
struct Part {
    static constexpr int E = F32 ? 4 : 8, PER = NV * E;  // logits of 16 bytes, of a lane's chunk
    const uint8_t* x;
    const uint4v* body;
    int V, head, vecs, tail, chunks;
    // STREAMED: not to stay in the caches
    template <bool STREAMED>
    __device__ __forceinline__ void load(int ch, int lane, uint4v (&r)[NV]) const {
        const uint4v* q = body + (int64_t)ch * (64 * NV);
        const int last = vecs - 1 - ch * (64 * NV);
#pragma unroll
        for (int i = 0; i < NV; ++i) r[i] = STREAMED ? __builtin_nontemporal_load(q + min(i * 64 + lane, last)) : q[min(i * 64 + lane, last)];
    }
    // a lane's logits of a chunk, -infinity where there is none (`there`: bits)
    __device__ __forceinline__ void unpack(int ch, int lane, const uint4v (&r)[NV], float (&v)[PER], uint32_t& there) const {
        there = ~0u >> (32 - PER);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
            for (int e = 0; e < E; ++e) v[i * E + e] = __builtin_bit_cast(float, F32 ? q[e & 3] : e & 1 ? q[e >> 1 & 3] & 0xffff0000u : q[e >> 1 & 3] << 16);
        }
        if ((ch + 1) * (64 * NV) > vecs) {
            const int left = vecs - ch * (64 * NV) - lane;
            there = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i * 64 < left) there |= ((1u << E) - 1) << i * E;
#pragma unroll
                for (int e = 0; e < E; ++e) v[i * E + e] = i * 64 < left ? v[i * E + e] : -INFINITY;
            }
        }
    }
    __device__ __forceinline__ void singles(int lane, float (&v)[PER], uint32_t& there) const {
        there = lane < head || (lane >= 32 && lane - 32 < tail);
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = -INFINITY;
        if (there) v[0] = logit<F32>(x, index(chunks, lane, 0));
    }
    __device__ __forceinline__ int index(int ch, int lane, int e) const {
        if (ch < chunks) return head + (ch * (64 * NV) + lane) * E + e / E * (64 * E) + e % E;
        return lane < head ? lane : V - tail + lane - 32;
    }
    __device__ __forceinline__ uint64_t key(float v, int ch, int lane, int e) const { return (uint64_t)ordered(v) << 32 | (uint32_t)~(uint32_t)index(ch, lane, e); }
};

template <bool F32, bool TOP, int WAVES, int NV>
__global__ __launch_bounds__(64 * WAVES, NV == 2 ? 8 : 4) void token_logprobs_kernel(const LogpArgs p) {
    constexpr bool STREAMED = WAVES < 16;
    constexpr int E = Part<F32, NV>::E, PER = Part<F32, NV>::PER, GROUP = WAVES / 4;  // lanes of a group
    constexpr int LIST = WAVES * 64 > LP_FOUND ? WAVES * 64 : LP_FOUND;
    __shared__ uint64_t bufs[TOP ? WAVES : 1][LP_BUF], list[TOP ? LIST : 1], sorted[64];
    __shared__ uint32_t tops[256];
    __shared__ float parts[WAVES][3];
    __shared__ int counts[WAVES], found;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = p.splits == 1 ? blockIdx.x : blockIdx.y;
    const int split = p.splits == 1 ? 0 : blockIdx.x;
    Part<F32, NV> t;
    t.x = p.X + row * p.ldl * (F32 ? 4 : 2), t.V = (int)p.V;
    t.head = (int)min((int64_t)((16 - ((uintptr_t)t.x & 15)) & 15) / (F32 ? 4 : 2), p.V);
    t.vecs = (t.V - t.head) / E, t.tail = t.V - t.head - t.vecs * E;
    t.body = reinterpret_cast<const uint4v*>(t.x + t.head * (F32 ? 4 : 2));
    t.chunks = (t.vecs + 64 * NV - 1) / (64 * NV);
    const int part = split * WAVES + wave, step = p.splits * WAVES;
    // rounds: chunks part, part + step, ..; the first wavefront's last one are the single logits
    const int own = part < t.chunks ? (t.chunks - part - 1) / step + 1 : 0, rounds = own + (part == 0 && t.head + t.tail > 0);
    auto chunk_of = [&](int it) { return it < own ? part + it * step : t.chunks; };
    uint4v now[NV], next[NV];
    if (own) t.template load<STREAMED>(part, lane, now);
    const bool finishes = wave == 0 && p.splits == 1;
    const int32_t token = finishes ? given(p, row, lane) : -1;

    Weights w{-INFINITY, 0.0f, 0.0f};
    const float c = p.c;
    const int shift = rounds > 64 ? 26 - __builtin_clz(rounds - 1) : 0;  // 2^shift rounds a bit
    bool usual = false;  // every lane has a base, and none a far one
    float B = 0.0f, mine = -INFINITY, second = -INFINITY, passed = -INFINITY;  // chunks' largest logits, the best two; passed: k lanes of the wavefront have reached it
    int best_it = 0;
    uint64_t marks = 0;
    for (int it = 0; it < rounds; ++it) {
        const int ch = chunk_of(it);
        float v[PER];
        uint32_t there;
        if (it < own) {
            if (it + 1 < own) t.template load<STREAMED>(ch + step, lane, next);
            t.unpack(ch, lane, now, v, there);
#pragma unroll
            for (int i = 0; i < NV; ++i) now[i] = next[i];
        } else t.singles(lane, v, there);
        if (TOP) {
            float largest = v[0];
#pragma unroll
            for (int e = 1; e < PER; ++e) largest = fmaxf(largest, v[e]);
            if (it && (it & (it - 1)) == 0) {
                passed = value_of(reached_by<1>({ordered(mine)}, p.k));
                if (mine < passed) marks = 0;
            }
            if (largest >= passed) marks |= 1ull << (it >> shift);
            second = __builtin_amdgcn_fmed3f(second, mine, largest);
            best_it = largest > mine ? it : best_it;
            mine = fmaxf(mine, largest);
        }
        float s = 0.0f, u = 0.0f;
        if (usual) {
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const float y = fmaf(v[e], c, -B), g = __builtin_amdgcn_exp2f(y);
                s += g;
                u = fmaf(g, y, u);
            }
        }
        if (!usual || __ballot(!(s < 256.0f) || u != u)) {  // -infinity leaves u NaN
            float largest = v[0];
#pragma unroll
            for (int e = 1; e < PER; ++e) largest = fmaxf(largest, v[e]);
            const float nb = fmaxf(w.b, largest);
            if (nb > w.b) rebase(w, nb, c);
            const float b = w.b == -INFINITY ? 0.0f : w.b;
            B = __fmul_rn(b, c);
            const bool far = is_far(B);
            usual = __ballot(w.b == -INFINITY || far) == 0;
            s = u = 0.0f;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const float y = far ? (v[e] - b) * c : fmaf(v[e], c, -B), g = __builtin_amdgcn_exp2f(y);
                s += g;
                u = fmaf(g, fmaxf(y, -1e3f), u);  // 0 times -infinity counts as 0
            }
        }
        w.S += s, w.U += u;
    }

    const float its = finishes ? given_logit<F32>(p, t.x, token) : 0.0f;
    w = wave_joined(w, c);
    if (lane == 0) parts[wave][0] = w.b, parts[wave][1] = w.S, parts[wave][2] = w.U;
    if (TOP) {
        const uint32_t top = ordered(mine);
        uint32_t most = top;
#pragma unroll
        for (int d = 1; d < GROUP; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
        if (lane % GROUP == 0) tops[(wave * 64 + lane) / GROUP] = most;
        if (threadIdx.x == 0) found = 0;
        if (wave == 0) sorted[lane] = 0;
        lds_barrier();
        const uint32_t bound = reached_by<4>({tops[lane], tops[lane + 64], tops[lane + 128], tops[lane + 192]}, p.k);
        if (top >= bound) {
            const float from = value_of(bound);
            const bool one = ordered(second) < bound;  // one chunk has all that the lane can give
            for (uint64_t left = one ? 1 : marks; left; left &= left - 1) {
                const int it0 = one ? best_it : __builtin_ctzll(left) << shift, it1 = one ? it0 + 1 : min(rounds, it0 + (1 << shift));
                for (int it = it0; it < it1; ++it) {
                    const int ch = chunk_of(it);
                    float v[PER];
                    uint32_t there;
                    if (ch < t.chunks) {
                        uint4v r[NV];
                        t.template load<false>(ch, lane, r);
                        t.unpack(ch, lane, r, v, there);
                    } else t.singles(lane, v, there);
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (v[e] >= from && there >> e & 1) {
                            const int at = atomicAdd(&found, 1);  // any order: ranks are counted
                            if (at < LP_FOUND) list[at] = t.key(v[e], ch, lane, e);
                        }
                }
            }
        }
        lds_barrier();
        int n = found;
        if (n > LP_FOUND) {  // the same for all
            Best best{bufs[wave], 0, p.k, 0};
            for (int it = 0; it < rounds; ++it) {
                const int ch = chunk_of(it);
                float v[PER];
                uint32_t there;
                if (ch < t.chunks) {
                    uint4v r[NV];
                    t.template load<false>(ch, lane, r);
                    t.unpack(ch, lane, r, v, there);
                } else t.singles(lane, v, there);
                float largest = v[0];
#pragma unroll
                for (int e = 1; e < PER; ++e) largest = fmaxf(largest, v[e]);
                // chunks come in order: a later one has nothing that equals the k-th best and is before it
                if (__ballot(ordered(largest) >= (uint32_t)(best.least >> 32) + (ch < t.chunks)) == 0) continue;
                const float from = value_of(best.least ? (uint32_t)(best.least >> 32) : reached_by<1>({ordered(largest)}, p.k));
                uint32_t wanted = 0;
#pragma unroll
                for (int e = 0; e < PER; ++e) wanted |= v[e] >= from ? 1u << e : 0;
                wanted &= there;
                while (__ballot(wanted != 0)) {
                    const int e = wanted ? __builtin_ctz(wanted) : 0;
                    const uint64_t key = t.key(pick(v, e), ch, lane, e);
                    const bool take = wanted != 0 && key > best.least;
                    wanted &= wanted - 1;
                    const uint64_t who = __ballot(take);
                    if (who == 0) continue;
                    append(best, key, who, take);
                    if (best.count > 64) rank(best, lane);
                }
                if (best.least == 0 && best.count >= p.k) rank(best, lane);
            }
            if (lane == 0) counts[wave] = best.count;
            lds_barrier();
            int before = 0;
            n = 0;
            for (int k = 0; k < WAVES; ++k) before += k < wave ? counts[k] : 0, n += counts[k];
            if (lane < best.count) list[before + lane] = best.buf[lane];
            lds_barrier();
        }
        if (wave == 0)
            for (int i = lane; i - lane < n; i += 64) {
                const uint64_t key = i < n ? list[i] : 0;
                const int r = above(list, n, key);
                if (key && r < p.k) sorted[r] = key;
            }
    } else lds_barrier();
    if (wave) return;
    wave_lds_order();
    const int k = min(lane, WAVES - 1);
    w = Weights{parts[k][0], lane < WAVES ? parts[k][1] : 0.0f, lane < WAVES ? parts[k][2] : 0.0f};
    w = wave_joined(w, c);
    if (p.splits == 1) {
        finish<F32>(p, row, w, sorted, lane, t.x, token, its);
    } else {
        const int64_t at = row * p.splits + split;
        if (lane == 0) p.stats[at] = make_float4(w.b, w.S, w.U, 0.0f);
        if (TOP && lane < p.k) p.keys[at * p.k + lane] = sorted[lane];
    }
}

// The parts of a row, one a lane; then their keys, all parts' best ones first, until none is wanted.
template <bool F32, bool TOP>
__global__ __launch_bounds__(64) void token_logprobs_join_kernel(const LogpArgs p) {
    __shared__ uint64_t buf[LP_BUF];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const uint8_t* x = p.X + row * p.ldl * (F32 ? 4 : 2);
    Weights w{-INFINITY, 0.0f, 0.0f};
    if (lane < p.splits) {
        const float4 s = p.stats[row * p.splits + lane];
        w = Weights{s.x, s.y, s.z};
    }
    const int32_t token = given(p, row, lane);
    Best best{buf, 0, p.k, 0};
    if (TOP) {
        const uint64_t* keys = p.keys + row * p.splits * p.k;
        const int n = p.splits * p.k;
        for (int i = lane; i - lane < n; i += 64) {
            const int j = i / p.splits;
            const uint64_t key = i < n ? keys[(i - j * p.splits) * p.k + j] : 0;
            const bool take = key > best.least;
            const uint64_t who = __ballot(take);
            if (who == 0) break;  // nor are those behind them
            append(best, key, who, take);
            rank(best, lane);
        }
    }
    const float its = given_logit<F32>(p, x, token);
    w = wave_joined(w, p.c);
    finish<F32>(p, row, w, buf, lane, x, token, its);
}

// Workgroups: all rows' wavefronts at once on the card where there are enough rows; parts of rows where that gives four workgroups or more a
// row (or the row is very long) and no more than the CUs.  us, bf16, top 5: parts of 1, 2, 4, 8, 16 of one row of 131072 logits 19.3, 16.2, 13.4, 10.9, 10.7, of
// 64 rows 20.7, 18.5, 15.0, 14.4, 20.3, of 64 rows of 50001 13.9, 14.2, 11.5, 14.0, 20.5, of 32000 11.0, 12.0, 11.5, 14.3, 22.0.  Wavefronts a row 4, 8, 16, rows of 131072, no
// top: 256 rows 30.9, 20.7, 17.1, 600 38.3, 33.2, 35.5, 1000 45.8, 46.2, 48.9, 2048 86.6, 85.3, 91.4, 4096 165, 160, 176; of 32000, top 5: 512 rows 18.3, 16.5, 15.8, 1000
// 23.7, 24.5, 26.8, 4096 58.9, 69.7, 86.8.  Rows of floats, of twice the bytes, go by the same rule, which was not measured for them.
struct LogpShape {
    int waves, splits;
};
static LogpShape logprob_shape(int64_t T, int64_t V) {
    if (T > 512) return LogpShape{T > 1024 ? 4 : 8, 1};
    const int64_t most = V / 8192, want = T > 0 ? 256 / T : 1, n = want < most ? want : most;
    return LogpShape{16, (int)(n < 2 || (n < 4 && V < 100000) ? 1 : n > LP_MAX_SPLITS ? LP_MAX_SPLITS : n)};
}

size_t token_logprobs_workspace(int64_t T, int64_t V, int32_t k) {
    const int n = logprob_shape(T, V).splits;
    return n == 1 ? 0 : align_up((size_t)T * n * (16 + 8 * (size_t)k), 256);
}

int launch_token_logprobs(const void* X, bool f32, int64_t T, int64_t V, int64_t ldl, float scale, const int32_t* tokens, int32_t n_tok, int32_t k, float* lp,
                          int32_t* ids, float* top, float* lse, float* entropy, uint8_t* workspace, hipStream_t st) {
    LogpArgs p;
    p.V = V, p.ldl = ldl, p.scale = scale, p.c = scale * 1.44269504088896341f, p.n_tok = n_tok, p.k = k;
    const LogpShape shape = logprob_shape(T, V);  // of the whole call, as its workspace
    p.splits = shape.splits;
    p.stats = reinterpret_cast<float4*>(workspace), p.keys = reinterpret_cast<uint64_t*>(workspace + (size_t)T * p.splits * 16);
    auto go = [&](auto f, auto t) {
        constexpr bool F32 = decltype(f)::value, TOP = decltype(t)::value;
        const dim3 grid = p.splits == 1 ? dim3((unsigned)p.T) : dim3((unsigned)p.splits, (unsigned)p.T);
        if (shape.waves == 4) token_logprobs_kernel<F32, TOP, 4, 2><<<grid, 256, 0, st>>>(p);
        else if (shape.waves == 8) token_logprobs_kernel<F32, TOP, 8, 2><<<grid, 512, 0, st>>>(p);
        else if (T > 256 || p.splits > 1) token_logprobs_kernel<F32, TOP, 16, 2><<<grid, 1024, 0, st>>>(p);
        else token_logprobs_kernel<F32, TOP, 16, 4><<<grid, 1024, 0, st>>>(p);
        if (p.splits > 1) token_logprobs_join_kernel<F32, TOP><<<dim3((unsigned)p.T), 64, 0, st>>>(p);
    };
    auto by_top = [&](auto f) { k ? go(f, std::true_type()) : go(f, std::false_type()); };
    constexpr int64_t MOST = 1 << 23;  // rows of a launch, which has less than 2^32 threads along an axis; calls of as many are not split
    for (int64_t r = 0; r < T; r += MOST) {
        p.X = static_cast<const uint8_t*>(X) + r * ldl * (f32 ? 4 : 2), p.T = T - r < MOST ? T - r : MOST;
        p.tokens = tokens + (tokens ? r * n_tok : 0), p.lp = lp + (lp ? r * n_tok : 0), p.ids = ids + (ids ? r * k : 0), p.top = top + (top ? r * k : 0);
        p.lse = lse + (lse ? r : 0), p.entropy = entropy + (entropy ? r : 0);
        f32 ? by_top(std::true_type()) : by_top(std::false_type());
        const int rc = check_launch("osc_token_logprobs");
        if (rc) return rc;
    }
    return OSC_OK;
}

}  // namespace osc
