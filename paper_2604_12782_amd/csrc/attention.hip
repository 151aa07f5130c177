// Attention of a step's rows over a shared prefix and each request's own cached tokens.
#include <algorithm>

#include "osc_internal.h"
#include "lds_dma.h"

namespace osc {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t* lds_ptr;

struct AttnArgs {
    const uint16_t* Q;
    int64_t T, ldq;
    int Hq, Hkv, G;
    const uint8_t *K, *V;
    uint32_t n_pages;
    int lg;
    const int32_t* prefix_pages;
    int P;
    const int32_t* table;
    int64_t ldt;
    int max_kv;  // tokens that a row of the table can name
    const int32_t *kv_lens, *q_offsets;
    int B;
    float c;  // scale * log2(e): scores leave the matrix core unscaled, and powers are of two
    uint16_t* O;
    int64_t ldo;
    float* lse;
};

// ---- a tile of 32 cached tokens in LDS ------------------------------------------------------------------------------
// Rows of D bf16 in pieces of 16 bytes; piece c of row r sits at c ^ spread(r), so that both readers find all banks: keys by
// 32 rows of one piece, values by 8 rows of four neighbouring pieces.
template <int D>
__device__ __forceinline__ int spread(int r) {
    return D == 128 ? (r & 3) << 2 | ((r >> 2) & 3) : ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
}

struct Span {  // 32 tokens of one key/value head: its pages hold 16-token runs in one piece
    const uint8_t *half0, *half1;  // bytes from the cache's start are the same for keys and values: held for keys
    int last;                      // the last token there is, 0..31
};

template <int D>
__device__ __forceinline__ Span locate(const AttnArgs& p, const int32_t* pages, int h, int j0, int end) {
    auto at = [&](int j) {
        uint32_t page = (uint32_t)pages[j >> p.lg];
        if (page >= p.n_pages) page = 0;  // nothing outside the cache is read, whatever a table holds
        return p.K + ((((int64_t)page * p.Hkv + h) << p.lg) + ((j & ((1 << p.lg) - 1)) & ~15)) * (D * 2);
    };
    Span s;
    s.last = min(31, end - 1 - j0);
    s.half0 = at(j0);
    s.half1 = at(min(j0 + 16, end - 1));
    return s;
}

// Asks for the tile: rows past the last token repeat it, so that whatever a page holds there is never multiplied.
template <int D>
__device__ __forceinline__ void fetch(const Span& s, int64_t shift, uint8_t* dst, int lane) {
    constexpr int CH = D / 8, RPI = 64 / CH, NI = 32 / RPI;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int r = i * RPI + lane / CH, piece = (lane % CH) ^ spread<D>(r), src = min(r, s.last);
        const uint8_t* base = (src < 16 ? s.half0 : s.half1) + shift;
        load_to_lds16(base + (src & 15) * (D * 2) + piece * 16, dst + i * 1024);
    }
}

// Softmax state of 32 rows, transposed: lane l holds row l % 32; its upper and lower half hold different tokens of a tile and
// different channels of the sums.  `sum` is the lane's own share.
template <int D>
struct State {
    v16f o[D / 32];
    float top, sum;
};

__device__ __forceinline__ float other_half_max(float v) {
    const int x = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return fmaxf(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1]));
}
__device__ __forceinline__ float other_half_sum(float v) {
    const int x = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
}

// One tile: S^T = K Q^T leaves a lane 16 tokens of its row, the weights go to bf16 and are the second operand of O^T += V^T P^T as
// they lie, because the order of the tokens inside a product is free as long as both operands have the same.
// `seen`: tokens below it count for the lane's row.
template <int D, bool MASK>
__device__ __forceinline__ void attend(State<D>& st, const v8bf (&q)[D / 16], const uint8_t* kt, const uint8_t* vt, int lane, float c, int seen) {
    const int r = lane & 31, hi = lane >> 5;
    v16f s = {};
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        const v8bf kf = *reinterpret_cast<const v8bf*>(kt + r * (D * 2) + (((2 * k + hi) ^ spread<D>(r)) << 4));
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[k], s, 0, 0, 0);
    }
    if (MASK) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if ((e & 3) + 8 * (e >> 2) + 4 * hi >= seen) s[e] = -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
    top = fmaxf(other_half_max(top), st.top);
    const float base = top == -INFINITY ? 0.0f : top * c;  // a row that has seen nothing yet keeps sums of zero
    const float fade = __builtin_amdgcn_exp2f(st.top * c - base);
    st.top = top;
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -base));
        sum += s[e];
    }
    st.sum = st.sum * fade + sum;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) st.o[d][e] *= fade;
    const int i = lane & 15;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        v8bf w;  // rounded to 8 bits for the matrix core: half an ulp each, and of either sign; their sum is taken before
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (__bf16)s[8 * k + e];
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
            union {
                v4s part[2];
                v8bf all;
            } vf;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int row = 16 * k + 8 * x + 4 * hi + (i >> 2), piece = 4 * d + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
                vf.part[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) v4s*)(lds_ptr)(vt + row * (D * 2) + ((piece ^ spread<D>(row)) << 4) + (i & 1) * 8));
            }
            st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.all, w, st.o[d], 0, 0, 0);
        }
    }
}

template <int D>
__global__ __launch_bounds__(256) void prefix_attention_kernel(const AttnArgs p) {
    constexpr int TILE = 32 * D * 2;
    extern __shared__ uint8_t lds[];
    int32_t* first = reinterpret_cast<int32_t*>(lds + 8 * TILE + 1024);  // row tiles before request b
    __shared__ int64_t wsum[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int T = (int)p.T;
    auto rows_of = [&](int b, int& q0, int& n) {
        q0 = min(max(p.q_offsets[b], 0), T);
        n = max(min(p.q_offsets[b + 1], T) - q0, 0);
    };
    {
        const int per = (p.B + 255) / 256, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
        int64_t mine = 0;  // offsets that do not rise can name more rows than there are: 64 bits, and the stored sums stay in range
        for (int b = b0; b < b1; ++b) {
            int q0, n;
            rows_of(b, q0, n);
            mine += (n * p.G + 31) >> 5;
        }
        int64_t s = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t u = __shfl_up(s, d);
            if (lane >= d) s += u;
        }
        if (lane == 63) wsum[wave] = s;
        __syncthreads();
        s -= mine;
        for (int w = 0; w < wave; ++w) s += wsum[w];
        for (int b = b0; b < b1; ++b) {
            int q0, n;
            rows_of(b, q0, n);
            first[b] = (int)min(s, (int64_t)0x7fffffff);
            s += (n * p.G + 31) >> 5;
        }
        if (tid == 255) first[p.B] = (int)min(s, (int64_t)0x7fffffff);
        __syncthreads();
    }
    const int64_t units = (int64_t)first[p.B] * p.Hkv;
    uint8_t* mine = lds + wave * 2 * TILE;
    const int64_t to_v = p.V - p.K;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int tile = (int)(u / p.Hkv), h = (int)(u - (int64_t)tile * p.Hkv);
        int b = 0, hi = p.B;
        while (hi - b > 1) {
            const int mid = (b + hi) >> 1;
            if (first[mid] <= tile) b = mid;
            else hi = mid;
        }
        b = __builtin_amdgcn_readfirstlane(b);
        int q0, n;
        rows_of(b, q0, n);
        const int L = min(max(p.kv_lens[b], 0), p.max_kv);
        const int r0 = (tile - first[b]) * 32, r = r0 + (lane & 31), rows = n * p.G;
        const int rc = min(r, rows - 1), ti = rc / p.G, g = rc - ti * p.G;
        v8bf q[D / 16];
        const uint16_t* qp = p.Q + (int64_t)(q0 + ti) * p.ldq + (h * p.G + g) * D + (lane >> 5) * 8;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = *reinterpret_cast<const v8bf*>(qp + k * 16);
        const int seen = L - n + ti + 1;  // own tokens that the lane's row may see
        const int own = max(0, L - n + min(r0 + 31, rows - 1) / p.G + 1);
        const int clear = L - n + r0 / p.G + 1;  // ... that all rows may see
        const int np = (p.P + 31) >> 5, nt = np + ((own + 31) >> 5);

        State<D> st;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) st.o[d] = v16f{};
        st.top = -INFINITY, st.sum = 0.0f;
        for (int k = wave; k < nt; k += 4) {
            const bool pre = k < np;
            const int j0 = (pre ? k : k - np) * 32, end = pre ? p.P : own;
            const Span sp = locate<D>(p, pre ? p.prefix_pages : p.table + (int64_t)b * p.ldt, h, j0, end);
            fetch<D>(sp, 0, mine, lane);
            fetch<D>(sp, to_v, mine + TILE, lane);
            wait_vmcnt<0>();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (j0 + 32 > (pre ? p.P : clear)) attend<D, true>(st, q, mine, mine + TILE, lane, p.c, (pre ? p.P : seen) - j0);
            else attend<D, false>(st, q, mine, mine + TILE, lane, p.c, 0);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        // the four wavefronts' parts: each leaves its sums in its own LDS, [row][channel], pieces of 16 bytes spread by row
        st.sum = other_half_sum(st.sum);
        float* parts = reinterpret_cast<float*>(lds);
        float* stats = reinterpret_cast<float*>(lds + 8 * TILE);  // [wave][row] top, then sum
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = lane & 31, piece = 8 * d + 2 * e + (lane >> 5);
                *reinterpret_cast<float4*>(parts + wave * 32 * D + row * D + ((piece ^ (row & 7)) << 2)) =
                    make_float4(st.o[d][4 * e], st.o[d][4 * e + 1], st.o[d][4 * e + 2], st.o[d][4 * e + 3]);
            }
        if (lane < 32) stats[wave * 32 + lane] = st.top, stats[128 + wave * 32 + lane] = st.sum;
        __syncthreads();
        const int row = tid >> 3, part = tid & 7;
        if (r0 + row < rows) {
            float top = -INFINITY, w[4], sum = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) top = fmaxf(top, stats[k * 32 + row]);
            const float base = top == -INFINITY ? 0.0f : top * p.c;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[k] = __builtin_amdgcn_exp2f(stats[k * 32 + row] * p.c - base);
                sum += w[k] * stats[128 + k * 32 + row];
            }
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            const int to = (r0 + row) / p.G, tg = r0 + row - to * p.G;
            const int64_t t = q0 + to;
            uint16_t* out = p.O + t * p.ldo + (h * p.G + tg) * D;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const int piece = k * 8 + part;
                float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float4 y = *reinterpret_cast<const float4*>(parts + v * 32 * D + row * D + ((piece ^ (row & 7)) << 2));
                    x[0] = fmaf(w[v], y.x, x[0]), x[1] = fmaf(w[v], y.y, x[1]), x[2] = fmaf(w[v], y.z, x[2]), x[3] = fmaf(w[v], y.w, x[3]);
                }
                ushort4 y;
                y.x = f32_to_bf16_rne(x[0] * inv), y.y = f32_to_bf16_rne(x[1] * inv), y.z = f32_to_bf16_rne(x[2] * inv), y.w = f32_to_bf16_rne(x[3] * inv);
                *reinterpret_cast<ushort4*>(out + piece * 4) = y;
            }
            if (p.lse && part == 0)
                p.lse[t * p.Hq + h * p.G + tg] = sum > 0.0f ? (base + __log2f(sum)) * 0.69314718055994531f : -INFINITY;
        }
        __syncthreads();
    }
}

size_t prefix_attention_workspace(int64_t, int32_t, int32_t, int32_t, int32_t, int64_t) { return 256; }

int launch_prefix_attention(const AttnCall& a, hipStream_t st) {
    AttnArgs p;
    p.Q = static_cast<const uint16_t*>(a.Q), p.T = a.T, p.ldq = a.ldq, p.Hq = a.Hq, p.Hkv = a.Hkv, p.G = a.Hq / a.Hkv;
    p.K = static_cast<const uint8_t*>(a.K), p.V = static_cast<const uint8_t*>(a.V), p.n_pages = (uint32_t)a.n_pages, p.lg = a.lg;
    p.prefix_pages = a.prefix_pages, p.P = (int)a.prefix_len, p.table = a.table, p.ldt = a.ldt;
    p.max_kv = (int)std::min<int64_t>(a.ldt << a.lg, 0x7fffffff);
    p.kv_lens = a.kv_lens, p.q_offsets = a.q_offsets, p.B = a.B, p.c = a.scale * 1.44269504088896341f;
    p.O = static_cast<uint16_t*>(a.O), p.ldo = a.ldo, p.lse = a.lse;
    const int cus = cu_count();
    if (cus <= 0) return fail(OSC_ERR_HIP, "osc_prefix_attention: cannot read the device");
    auto go = [&](auto kernel, LdsReserved& r, size_t lds) {
        const int rc = reserve_lds((const void*)kernel, lds, r);
        if (rc) return rc;
        const int64_t most = ((int64_t)a.B + a.T * p.G / 32) * a.Hkv;
        kernel<<<dim3((unsigned)std::min<int64_t>(most, 2 * cus)), 256, lds, st>>>(p);
        return check_launch("osc_prefix_attention");
    };
    static LdsReserved r64, r128;
    const size_t extra = 1024 + ((size_t)a.B + 1) * 4;
    if (a.D == 64) return go(prefix_attention_kernel<64>, r64, 8 * 32 * 64 * 2 + extra);
    return go(prefix_attention_kernel<128>, r128, 8 * 32 * 128 * 2 + extra);
}

}  // namespace osc
