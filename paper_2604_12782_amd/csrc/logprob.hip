// Log probabilities of given tokens, entropy and top alternatives of rows of logits.
//
//   p_j = exp(scale x_j) / sum,  lse = log sum_j exp(scale x_j),  entropy = -sum_j p_j log p_j = lse - sum_j p_j scale x_j
//
// One pass over the logits.  A lane keeps, for what it has seen: a base b (a logit), S = sum of w_j = 2^(c (x_j - b)) and U = sum of
// w_j c (x_j - b), c = scale log2 e.  The base follows the largest logit only when that is 2^8 above it in weight, so sums are
// rarely scaled; a change of base by d = c (b - b') turns (S, U) into 2^d (S, U + S d), which is also how lanes, wavefronts
// and parts of a row are joined.  Then log p_j = scale (x_j - b) - log S and the entropy is log S - ln 2 U / S; logits enter by their
// distance from the base alone, so large ones lose nothing.  Everything is single precision.
//
// The top k.  A logit's key is its value in the order of unsigned numbers, then its index, lower ones first: 64 bits, no two alike.  A
// wavefront walks its part of a row in order and keeps keys that may be among the top k in LDS; when more than 64 are there
// their ranks are counted and the first k stay.  A chunk of 1024 logits is looked into only if its largest one is above the k-th of them.  In
// the first chunks that would be all: there no logit below the k-th largest of the lanes' largest ones is taken.
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
    int splits;
    float4* stats;   // workspace: of a part of a row, base, S, U
    uint64_t* keys;  // and its k best, best first
};

constexpr int LP_WG = 256, LP_WAVES = LP_WG / 64, LP_PER = 16, LP_CHUNK = 64 * LP_PER, LP_BUF = 128, LP_MAX_SPLITS = 64;

struct Weights {
    float b, S, U;
};
// turned to base nb >= b; nothing seen is b = -infinity, S = U = 0
__device__ __forceinline__ void rebase(Weights& w, float nb, float c) {
    if (w.b == -INFINITY) {
        w.S *= nb == INFINITY ? NAN : 0.0f, w.U = 0.0f;  // 0 stays 0, NaN stays NaN
    } else {
        const float d = fmaxf((w.b - nb) * c, -1e4f), f = __builtin_amdgcn_exp2f(d);
        w.U = (w.U + w.S * d) * f;
        w.S *= f;
    }
    w.b = nb;
}
__device__ __forceinline__ Weights joined(Weights v, Weights w, float c) {
    const float nb = fmaxf(v.b, w.b);
    rebase(v, nb, c);
    rebase(w, nb, c);
    v.S += w.S, v.U += w.U;
    return v;
}
__device__ __forceinline__ Weights wave_joined(Weights w, float c) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const Weights o{__shfl_xor(w.b, d), __shfl_xor(w.S, d), __shfl_xor(w.U, d)};
        w = joined(w, o, c);
    }
    return w;
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
    int ra = 0, rb = 0;
    if (s.count <= 64) {
        for (int j = 0; j < s.count; ++j) ra += s.buf[j] > a;
    } else {
#pragma unroll 4
        for (int j = 0; j < s.count; ++j) {
            const uint64_t o = s.buf[j];
            ra += o > a, rb += o > b;
        }
    }
    wave_lds_order();
    if (a && ra < s.k) s.buf[ra] = a;
    if (b && rb < s.k) s.buf[rb] = b;
    wave_lds_order();
    s.count = min(s.count, s.k);
    if (s.count == s.k) s.least = s.buf[s.k - 1];
}
__device__ __forceinline__ void offer(Best& s, uint64_t key, bool take, int lane) {
    const uint64_t who = __ballot(take);
    if (who == 0) return;
    if (take) s.buf[s.count + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key;
    s.count += __popcll(who);
    if (s.count > 64) rank(s, lane);
}
// A number that k lanes' `top` or more reach: the k-th largest's upper 16 bits.
__device__ __forceinline__ uint32_t reached_by(uint32_t top, int k) {
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t more = t | 1u << bit;
        if (__popcll(__ballot(top >= more)) >= k) t = more;
    }
    return t;
}

// one row's results, from all of it; `best` in order
__device__ __forceinline__ void finish(const LogpArgs& p, int64_t row, const Weights& w, const Best& best, int lane, const uint8_t* x, bool f32) {
    const bool bad = !(w.S < INFINITY) || w.b == INFINITY;  // NaN or infinity among the logits
    const float logS = w.S > 0.0f ? logf(w.S) : -INFINITY;
    auto log_p = [&](float v) { return bad ? NAN : w.S > 0.0f ? p.scale * (v - w.b) - logS : -INFINITY; };
    if (lane == 0) {
        if (p.lse) p.lse[row] = bad ? NAN : w.S > 0.0f ? p.scale * w.b + logS : -INFINITY;
        if (p.entropy) p.entropy[row] = bad ? NAN : w.S > 0.0f ? logS - w.U / w.S * 0.69314718055994531f : 0.0f;
    }
    for (int i = lane; i < p.n_tok; i += 64) {
        const int32_t t = p.tokens[row * p.n_tok + i];
        float r = 0.0f;
        if ((uint32_t)t < (uint64_t)p.V) {
            const float v = f32 ? reinterpret_cast<const float*>(x)[t] : __builtin_bit_cast(float, (uint32_t)reinterpret_cast<const uint16_t*>(x)[t] << 16);
            r = log_p(v);
        }
        p.lp[row * p.n_tok + i] = r;
    }
    if (lane < p.k) {
        const uint64_t key = best.buf[lane];
        p.ids[row * p.k + lane] = bad ? -1 : (int32_t)~(uint32_t)key;
        p.top[row * p.k + lane] = log_p(value_of((uint32_t)(key >> 32)));
    }
}

// A workgroup takes a part of a row (all of it where there are many rows), its wavefronts a run of chunks each.  A chunk is 16 logits a
// lane, read 16 bytes at a time from the row's first 16-byte boundary on; logits before the first and after the last whole 16
// bytes are the first and the last wavefront's.
template <bool F32, bool TOP>
__global__ __launch_bounds__(LP_WG) void token_logprobs_kernel(const LogpArgs p) {
    constexpr int E = F32 ? 4 : 8, NV = LP_PER / E;  // logits of 16 bytes, vectors of a lane's chunk
    __shared__ uint64_t bufs[TOP ? LP_WAVES : 1][LP_BUF];
    __shared__ float parts[LP_WAVES][3];
    __shared__ int counts[LP_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x / p.splits;
    const int split = (int)(blockIdx.x - row * p.splits);
    const uint8_t* x = p.X + row * p.ldl * (F32 ? 4 : 2);
    const int head = (int)min((int64_t)((16 - ((uintptr_t)x & 15)) & 15) / (F32 ? 4 : 2), p.V);
    const int64_t vecs = (p.V - head) / E;
    const int tail = (int)(p.V - head - vecs * E);
    const uint4* body = reinterpret_cast<const uint4*>(x + head * (F32 ? 4 : 2));
    const int64_t chunks = (vecs + 64 * NV - 1) / (64 * NV), per = (chunks + p.splits * LP_WAVES - 1) / (p.splits * LP_WAVES);
    const int part = split * LP_WAVES + wave;
    const int64_t c0 = min(chunks, part * per), c1 = min(chunks, c0 + per);

    Weights w{-INFINITY, 0.0f, 0.0f};
    Best best{bufs[TOP ? wave : 0], 0, p.k, 0};
    const float c = p.c, far = 8.0f / c;

    auto take_in = [&](const float (&v)[LP_PER], int n, float largest, int64_t first, auto index, auto there) {
        if (__ballot(largest > w.b + far || (w.b == -INFINITY && largest > -INFINITY))) {
            const float nb = fmaxf(w.b, largest);
            if (nb > w.b) rebase(w, nb, c);
        }
        const float b = w.b == -INFINITY ? 0.0f : w.b;
        float s = 0.0f, u = 0.0f;
#pragma unroll
        for (int e = 0; e < LP_PER; ++e) {
            if (e >= n) break;
            const float y = (v[e] - b) * c, g = __builtin_amdgcn_exp2f(y);
            s += g;
            u = fmaf(g, fmaxf(y, -200.0f), u);  // 0 times -infinity counts as 0
        }
        w.S += s, w.U += u;
        if (TOP) {
            const uint32_t top = ordered(largest);
            const uint64_t above = __ballot(top > (uint32_t)(best.least >> 32));
            if (above) {
                const uint32_t floor = __popcll(above) > 16 ? reached_by(top, best.k) : 0;
#pragma unroll
                for (int e = 0; e < LP_PER; ++e) {
                    if (e >= n) break;
                    const uint32_t o = ordered(v[e]);
                    const uint64_t key = (uint64_t)o << 32 | (uint32_t)~(uint32_t)(first + index(e));
                    offer(best, key, there(e) && o >= floor && key > best.least, lane);
                }
            }
        }
    };
    auto single = [&](int64_t first, int n) {  // n < 16 logits from `first` on, one a lane
        float v[LP_PER];
        v[0] = -INFINITY;
        if (lane < n)
            v[0] = F32 ? reinterpret_cast<const float*>(x)[first + lane] : __builtin_bit_cast(float, (uint32_t)reinterpret_cast<const uint16_t*>(x)[first + lane] << 16);
        take_in(v, 1, v[0], first, [&](int) { return lane; }, [&](int) { return lane < n; });
    };
    if (part == 0 && head) single(0, head);
    auto load = [&](int64_t ch, uint4 (&r)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t at = ch * (64 * NV) + i * 64 + lane;
            r[i] = body[min(at, vecs - 1)];
        }
    };
    uint4 now[NV], next[NV];
    if (c0 < c1) load(c0, now);
    for (int64_t ch = c0; ch < c1; ++ch) {
        if (ch + 1 < c1) load(ch + 1, next);
        float v[LP_PER];
        const int64_t left = vecs - ch * (64 * NV) - lane;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t q[4] = {now[i].x, now[i].y, now[i].z, now[i].w};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float f = __builtin_bit_cast(float, F32 ? q[e & 3] : e & 1 ? q[e >> 1 & 3] & 0xffff0000u : q[e >> 1 & 3] << 16);
                v[i * E + e] = i * 64 < left ? f : -INFINITY;
            }
        }
        float largest = v[0];
#pragma unroll
        for (int e = 1; e < LP_PER; ++e) largest = fmaxf(largest, v[e]);
        take_in(v, LP_PER, largest, head + ch * (64 * NV * E), [&](int e) { return ((e / E) * 64 + lane) * E + e % E; }, [&](int e) { return (e / E) * 64 < left; });
#pragma unroll
        for (int i = 0; i < NV; ++i) now[i] = next[i];
    }
    if (part == p.splits * LP_WAVES - 1 && tail) single(p.V - tail, tail);

    w = wave_joined(w, c);
    if (TOP) rank(best, lane);
    if (lane == 0) parts[wave][0] = w.b, parts[wave][1] = w.S, parts[wave][2] = w.U, counts[wave] = best.count;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int k = 1; k < LP_WAVES; ++k) w = joined(w, Weights{parts[k][0], parts[k][1], parts[k][2]}, c);
    if (TOP)
        for (int k = 1; k < LP_WAVES; ++k) {  // at most 64 of another's are offered to at most 64 of this one's
            const bool has = lane < counts[k];
            const uint64_t key = has ? bufs[k][lane] : 0;
            offer(best, key, has && key > best.least, lane);
            rank(best, lane);
        }
    if (p.splits == 1) {
        finish(p, row, w, best, lane, x, F32);
    } else {
        const int64_t at = row * p.splits + split;
        if (lane == 0) p.stats[at] = make_float4(w.b, w.S, w.U, 0.0f);
        if (TOP && lane < p.k) p.keys[at * p.k + lane] = lane < best.count ? best.buf[lane] : 0;
    }
}

// The parts of a row, one a lane; their keys are in order, so a lane whose key is not wanted has none that is.
template <bool F32, bool TOP>
__global__ __launch_bounds__(64) void token_logprobs_join_kernel(const LogpArgs p) {
    __shared__ uint64_t buf[LP_BUF];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    Weights w{-INFINITY, 0.0f, 0.0f};
    if (lane < p.splits) {
        const float4 s = p.stats[row * p.splits + lane];
        w = Weights{s.x, s.y, s.z};
    }
    Best best{buf, 0, p.k, 0};
    if (TOP) {
        const uint64_t* keys = p.keys + (row * p.splits + min(lane, p.splits - 1)) * p.k;
        uint32_t floor = 0;
        for (int j = 0; j < p.k; ++j) {
            const uint64_t key = lane < p.splits ? keys[j] : 0;
            if (j == 0) floor = reached_by((uint32_t)(key >> 32), p.k);
            const bool take = key > best.least && (uint32_t)(key >> 32) >= floor;
            if (__ballot(take) == 0) break;
            offer(best, key, take, lane);
        }
        rank(best, lane);
    }
    w = wave_joined(w, p.c);
    finish(p, row, w, best, lane, p.X + row * p.ldl * (F32 ? 4 : 2), F32);
}

// Parts of a row: as many as give every CU four workgroups, none with less than a chunk a wavefront.
static int logprob_splits(int64_t T, int64_t V) {
    const int64_t most = (V / LP_CHUNK + LP_WAVES - 1) / LP_WAVES, want = T > 0 ? 1024 / T : 1;
    const int64_t n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > LP_MAX_SPLITS ? LP_MAX_SPLITS : n);
}

size_t token_logprobs_workspace(int64_t T, int64_t V, int32_t k) {
    const int n = logprob_splits(T, V);
    return n == 1 ? 0 : align_up((size_t)T * n * (16 + 8 * (size_t)k), 256);
}

int launch_token_logprobs(const void* X, bool f32, int64_t T, int64_t V, int64_t ldl, float scale, const int32_t* tokens, int32_t n_tok, int32_t k, float* lp,
                          int32_t* ids, float* top, float* lse, float* entropy, uint8_t* workspace, hipStream_t st) {
    LogpArgs p;
    p.X = static_cast<const uint8_t*>(X), p.T = T, p.V = V, p.ldl = ldl, p.scale = scale, p.c = scale * 1.44269504088896341f;
    p.tokens = tokens, p.n_tok = n_tok, p.k = k, p.lp = lp, p.ids = ids, p.top = top, p.lse = lse, p.entropy = entropy;
    p.splits = logprob_splits(T, V);
    p.stats = reinterpret_cast<float4*>(workspace), p.keys = reinterpret_cast<uint64_t*>(workspace + (size_t)T * p.splits * 16);
    const dim3 grid((unsigned)(T * p.splits));
    if (f32) {
        if (k) token_logprobs_kernel<true, true><<<grid, LP_WG, 0, st>>>(p);
        else token_logprobs_kernel<true, false><<<grid, LP_WG, 0, st>>>(p);
    } else {
        if (k) token_logprobs_kernel<false, true><<<grid, LP_WG, 0, st>>>(p);
        else token_logprobs_kernel<false, false><<<grid, LP_WG, 0, st>>>(p);
    }
    if (p.splits > 1) {
        const dim3 rows((unsigned)T);
        if (f32) {
            if (k) token_logprobs_join_kernel<true, true><<<rows, 64, 0, st>>>(p);
            else token_logprobs_join_kernel<true, false><<<rows, 64, 0, st>>>(p);
        } else {
            if (k) token_logprobs_join_kernel<false, true><<<rows, 64, 0, st>>>(p);
            else token_logprobs_join_kernel<false, false><<<rows, 64, 0, st>>>(p);
        }
    }
    return check_launch("osc_token_logprobs");
}

}  // namespace osc
