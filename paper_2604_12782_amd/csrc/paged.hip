// What an attention step needs before its scores: cache pages and slots of the new tokens, the table of rotation
// angles, and the per-head norms with the rotation and the write into the paged cache.
#include <type_traits>

#include "osc_internal.h"
#include "wave_util.h"

namespace osc {

// ---- block tables and slots from lengths -------------------------------------------------------------------
// Two running sums over the requests place everything: q_off[b] = sum of the new tokens before b, need_off[b] = sum of the new
// pages before b.  A workgroup computes both for all requests in LDS (a request costs it 8 bytes from L2) and then serves its
// share of the tokens: a binary search in q_off finds the request, need_off the page.  So the step is one launch with
// no word passed between workgroups; the first token of a new page writes that page's table entry, and where T leaves that token
// without a row, the first workgroup's lane of the request does.  Sums stop at 2^32 - 1,
// which keeps them in order: what lies past 2^31 - 1 tokens or past the free pages needs no exact number.
// Bound by latency: the lengths' read, the two sums, the table's read and the store depend on one another.
template <int NT, int PER>
__global__ __launch_bounds__(NT) void page_slots_kernel(const int32_t* __restrict__ kv_lens, const int32_t* __restrict__ q_lens, int B, int lg,
                                                        const int32_t* __restrict__ free_pages, int64_t n_pool,
                                                        const int32_t* __restrict__ n_free_ptr, int32_t* table, int64_t ldt, int pos_base,
                                                        int64_t T, int32_t* __restrict__ kv_out, int32_t* __restrict__ q_offsets,
                                                        int32_t* __restrict__ positions, int32_t* __restrict__ slots, int32_t* __restrict__ info) {
    extern __shared__ int32_t lds[];
    int32_t *q_off = lds, *need_off = lds + B, *kv_at = lds + 2 * B;  // need_off: -1 for a refused request
    __shared__ uint32_t part[NT / 64][2];
    __shared__ int32_t sums[2];  // pages taken, requests refused
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t ps1 = (1u << lg) - 1;
    const uint32_t n_free = (uint32_t)max(0, (int)min((int64_t)*n_free_ptr, n_pool));
    if (tid < 2) sums[tid] = 0;

    const int b0 = tid * PER;
    uint32_t kv[PER], q[PER], need[PER], my_q = 0, my_need = 0;
    bool fits[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const bool there = b0 + k < B;
        kv[k] = there ? max(kv_lens[b0 + k], 0) : 0;
        q[k] = there ? max(q_lens[b0 + k], 0) : 0;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const uint32_t all = kv[k] + q[k], pages = (uint32_t)(((uint64_t)all + ps1) >> lg);  // below 2^32
        fits[k] = all <= 0x7fffffffu && pages <= (uint64_t)ldt;
        need[k] = fits[k] ? pages - ((kv[k] + ps1) >> lg) : 0;
        my_q = __builtin_elementwise_add_sat(my_q, q[k]);
        my_need = __builtin_elementwise_add_sat(my_need, need[k]);
    }
    uint32_t sq = my_q, sn = my_need;  // over the lanes below and this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t uq = __shfl_up(sq, d), un = __shfl_up(sn, d);
        if (lane >= d) sq = __builtin_elementwise_add_sat(sq, uq), sn = __builtin_elementwise_add_sat(sn, un);
    }
    if (lane == 63) part[wave][0] = sq, part[wave][1] = sn;
    sq = __shfl_up(sq, 1), sn = __shfl_up(sn, 1);
    if (lane == 0) sq = sn = 0;
    __syncthreads();
    uint32_t total = 0, before_q = 0, before_n = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const uint32_t pq = part[w][0], pn = part[w][1];
        if (w < wave) before_q = __builtin_elementwise_add_sat(before_q, pq), before_n = __builtin_elementwise_add_sat(before_n, pn);
        total = __builtin_elementwise_add_sat(total, pq);
    }
    sq = __builtin_elementwise_add_sat(before_q, sq), sn = __builtin_elementwise_add_sat(before_n, sn);
    int taken = 0, refused = 0;
    const bool first = blockIdx.x == 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = b0 + k;
        const uint32_t to = __builtin_elementwise_add_sat(sn, need[k]);
        if (b < B) {
            const bool ok = fits[k] && (need[k] == 0 || to <= n_free);
            q_off[b] = (int32_t)min(sq, 0x7fffffffu);
            need_off[b] = ok ? (int32_t)min(sn, 0x7fffffffu) : -1;
            kv_at[b] = (int32_t)kv[k];
            if (first) {
                q_offsets[b] = q_off[b];
                kv_out[b] = (int32_t)(ok ? kv[k] + q[k] : kv[k]);
                if (ok) taken += (int)need[k];
                else ++refused;
                if (ok && need[k] && (int64_t)sq + q[k] > T) {  // pages whose first token has no row are entered all the same: they are the request's
                    const int64_t have = ((int64_t)kv[k] + ps1) >> lg, from = ((int64_t)kv[k] + max(T - (int64_t)sq, (int64_t)0) + ps1) >> lg;
                    for (int64_t i = max(have, from); i < have + need[k]; ++i) table[(int64_t)b * ldt + i] = free_pages[n_free - 1 - (sn + (i - have))];
                }
            }
        }
        sq = __builtin_elementwise_add_sat(sq, q[k]);
        sn = to;
    }
    if (first) {
        if (taken) atomicAdd(&sums[0], taken);  // integers in LDS: no order shows
        if (refused) atomicAdd(&sums[1], refused);
    }
    __syncthreads();
    const int tokens = (int)min(total, 0x7fffffffu);
    if (first && tid == 0) {
        q_offsets[B] = tokens;
        info[0] = (int)n_free - sums[0];
        info[1] = sums[0];
        info[2] = sums[1];
        info[3] = tokens;
    }
    for (int64_t t = (int64_t)blockIdx.x * NT + tid; t < T; t += (int64_t)gridDim.x * NT) {
        int slot = -1, pos = -1;
        if (t < tokens) {
            int lo = 0, hi = B;  // the last request that starts at or before t is the one that holds it
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (q_off[mid] <= t) lo = mid;
                else hi = mid;
            }
            const int64_t have_kv = kv_at[lo], p = have_kv + (t - q_off[lo]);
            pos = (int)min((int64_t)pos_base + p, (int64_t)0x7fffffff);
            if (need_off[lo] >= 0) {
                const int64_t i = p >> lg, have = (have_kv + ps1) >> lg;
                int32_t* entry = table + (int64_t)lo * ldt + i;
                int page;
                if (i < have) page = *entry;
                else {
                    page = free_pages[n_free - 1 - (need_off[lo] + (i - have))];
                    if ((p & ps1) == 0) *entry = page;
                }
                if ((uint32_t)page <= 0x7fffffffu >> lg) slot = (int)(((int64_t)page << lg) + (p & ps1));  // otherwise no cache has it, and 32 bits would name another
            }
        }
        positions[t] = pos;
        slots[t] = slot;
    }
}

int launch_page_slots(const int32_t* kv_lens, const int32_t* q_lens, int32_t B, int lg, const int32_t* free_pages, int64_t n_pool,
                      const int32_t* n_free, int32_t* table, int64_t ldt, int32_t pos_base, int64_t T, int32_t* kv_out, int32_t* q_offsets,
                      int32_t* positions, int32_t* slots, int32_t* info, hipStream_t st) {
    const size_t lds = (size_t)B * 12;
    const int64_t most = 4 * (int64_t)cu_count();
    if (most <= 0) return fail(OSC_ERR_HIP, "osc_page_slots: cannot read the device");
    auto go = [&](auto kernel, int nt, LdsReserved& r) {
        if (lds > 48 * 1024) {
            const int rc = reserve_lds((const void*)kernel, lds, r);
            if (rc) return rc;
        }
        int64_t wgs = (T + nt - 1) / nt;
        wgs = wgs < 1 ? 1 : wgs > most ? most : wgs;
        kernel<<<dim3((unsigned)wgs), nt, lds, st>>>(kv_lens, q_lens, B, lg, free_pages, n_pool, n_free, table, ldt, pos_base, T, kv_out, q_offsets,
                                                     positions, slots, info);
        return check_launch("osc_page_slots");
    };
    static LdsReserved r256, r1, r2, r8;
    if (B <= 256) return go(page_slots_kernel<256, 1>, 256, r256);
    if (B <= 1024) return go(page_slots_kernel<1024, 1>, 1024, r1);
    if (B <= 2048) return go(page_slots_kernel<1024, 2>, 1024, r2);
    return go(page_slots_kernel<1024, 8>, 1024, r8);
}

// ---- rotation angles -------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void rope_table_kernel(double base, int half, int64_t n_pos, float* __restrict__ out) {
    const int64_t n = n_pos * half;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n; k += (int64_t)gridDim.x * 256) {
        const int64_t pos = k / half;
        const int i = (int)(k - pos * half);
        // doubles: a position of 2^20 times a frequency rounded to 24 bits would be off by 2^-5 of a radian
        const double a = (double)pos * pow(base, -(double)i / half);
        out[pos * 2 * half + i] = (float)cos(a);
        out[pos * 2 * half + half + i] = (float)sin(a);
    }
}

int launch_rope_table(double base, int32_t rot, int64_t n_pos, float* out, hipStream_t st) {
    const int64_t wgs = (n_pos * (rot / 2) + 255) / 256;
    rope_table_kernel<<<dim3((unsigned)(wgs > 16384 ? 16384 : wgs)), 256, 0, st>>>(base, rot / 2, n_pos, out);
    return check_launch("osc_rope_table");
}

// ---- per-head norms, rotation, cache -----------------------------------------------------------------------------
// A lane holds eight elements of a head, a head is D/8 lanes, a wavefront iteration 512/D heads.  The eight are two runs of four, a
// and b, chosen so that a pair's partner is in the same lane: rotated halves take elements 4l.. and 4l + rot/2.., everything
// else (neighbouring pairs, elements past `rot`, values) the eight from 8l.  The norm's sum crosses the head's lanes on the
// vector ALU; norm and rotation are single precision, rounded once to bf16 at the end.
// Bound by HBM: every element is read and written once.
struct RopeArgs {
    const uint16_t* X;
    int64_t T, ldx;
    int Hq, Hkv, heads;  // heads: Hq + 2 Hkv, or Hq where nothing is cached
    const uint16_t *gq, *gk;
    float eps;
    const float* cos_sin;
    int64_t n_pos;
    int rot, n_axes;
    const int32_t* pos;
    int64_t ldpos;
    int s0, s1;  // pairs below s0 turn by axis 0, below s1 by axis 1, others by axis 2
    int quads;   // both are multiples of four: a lane's pairs turn by one axis
    const int32_t* slots;
    uint16_t* Y;
    int64_t ldy;
    uint16_t *K, *V;
    int64_t n_pages;
    int lg;
    int units;  // wavefronts a token
};

__device__ __forceinline__ void unpack4(uint2 w, float (&f)[4]) {
    f[0] = __builtin_bit_cast(float, w.x << 16);
    f[1] = __builtin_bit_cast(float, w.x & 0xffff0000u);
    f[2] = __builtin_bit_cast(float, w.y << 16);
    f[3] = __builtin_bit_cast(float, w.y & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){a, b}, v2bf));  // nearest even
}
__device__ __forceinline__ uint2 pack4(const float (&f)[4]) { return make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3])); }
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
    v = dpp_add<0x141>(dpp_add<0x4E>(dpp_add<0xB1>(v)));  // lane ^ 1, lane ^ 2, 7 - lane
    return LANES == 16 ? dpp_add<0x140>(v) : v;           // 15 - lane
}

template <int D, bool PAIRS, bool AXES, int U>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const RopeArgs p) {
    constexpr int LPH = D / 8, HPI = 64 / LPH;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int lane = threadIdx.x & 63, l = lane % LPH, sub = lane / LPH;
    const int64_t t = unit / p.units;
    if (t >= p.T) return;
    const int h0 = (int)(unit - t * p.units) * (U * HPI) + sub;
    const int half = p.rot >> 1, i0 = 4 * l;
    const bool turned = i0 < half;
    const int ea = turned && !PAIRS ? i0 : 8 * l, eb = turned && !PAIRS ? i0 + half : 8 * l + 4;  // of a query or key head

    const uint16_t* row = p.X + t * p.ldx;
    uint2 a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * HPI;
        if (h < p.heads) {
            a[u] = *reinterpret_cast<const uint2*>(row + h * D + ea);
            b[u] = *reinterpret_cast<const uint2*>(row + h * D + eb);
        }
    }
    float c[4], s[4];
    bool real;
    {
        int64_t at[3];
        at[0] = p.pos[t];
        real = (uint64_t)at[0] < (uint64_t)p.n_pos;
        if constexpr (AXES) {
            at[1] = p.pos[p.ldpos + t];
            at[2] = p.n_axes > 2 ? p.pos[2 * p.ldpos + t] : at[1];
            real = real && (uint64_t)at[1] < (uint64_t)p.n_pos && (uint64_t)at[2] < (uint64_t)p.n_pos;
        }
        if (real && turned) {
            if (AXES && !p.quads) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + k;
                    const float* w = p.cos_sin + (i < p.s0 ? at[0] : i < p.s1 ? at[1] : at[2]) * p.rot + i;
                    c[k] = w[0];
                    s[k] = w[half];
                }
            } else {
                const float* w = p.cos_sin + (!AXES || i0 < p.s0 ? at[0] : i0 < p.s1 ? at[1] : at[2]) * p.rot + i0;
                const float4 cv = *reinterpret_cast<const float4*>(w), sv = *reinterpret_cast<const float4*>(w + half);
                c[0] = cv.x, c[1] = cv.y, c[2] = cv.z, c[3] = cv.w;
                s[0] = sv.x, s[1] = sv.y, s[2] = sv.z, s[3] = sv.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) c[k] = 1.0f, s[k] = 0.0f;
        }
    }
    const int slot = p.heads > p.Hq ? p.slots[t] : -1;
    const int64_t page = slot >> p.lg;
    const bool cached = real && slot >= 0 && page < p.n_pages;
    const int in_page = slot & ((1 << p.lg) - 1);

#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * HPI;
        if (h >= p.heads) continue;
        const bool query = h < p.Hq, key = !query && h < p.Hq + p.Hkv;
        uint16_t* out;
        if (query) out = p.Y + t * p.ldy + h * D;
        else {
            if (!cached) continue;
            const int hk = key ? h - p.Hq : h - p.Hq - p.Hkv;
            out = (key ? p.K : p.V) + (((page * p.Hkv + hk) << p.lg) + in_page) * (int64_t)D;
        }
        if (query || key) {
            float fa[4], fb[4];
            unpack4(a[u], fa);
            unpack4(b[u], fb);
            const uint16_t* gamma = query ? p.gq : p.gk;
            if (gamma) {
                float q = 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) q = fmaf(fa[k], fa[k], fmaf(fb[k], fb[k], q));
                q = head_sum<LPH>(q);  // the lanes of a head take the same way here
                const float r = 1.0f / sqrtf(q * (1.0f / D) + p.eps);
                float ga[4], gb[4];
                unpack4(*reinterpret_cast<const uint2*>(gamma + ea), ga);
                unpack4(*reinterpret_cast<const uint2*>(gamma + eb), gb);
#pragma unroll
                for (int k = 0; k < 4; ++k) fa[k] = fa[k] * r * ga[k], fb[k] = fb[k] * r * gb[k];
            }
            float ya[4], yb[4];
            if (!turned) {
#pragma unroll
                for (int k = 0; k < 4; ++k) ya[k] = fa[k], yb[k] = fb[k];
            } else if (PAIRS) {
                ya[0] = fa[0] * c[0] - fa[1] * s[0], ya[1] = fa[1] * c[0] + fa[0] * s[0];
                ya[2] = fa[2] * c[1] - fa[3] * s[1], ya[3] = fa[3] * c[1] + fa[2] * s[1];
                yb[0] = fb[0] * c[2] - fb[1] * s[2], yb[1] = fb[1] * c[2] + fb[0] * s[2];
                yb[2] = fb[2] * c[3] - fb[3] * s[3], yb[3] = fb[3] * c[3] + fb[2] * s[3];
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) ya[k] = fa[k] * c[k] - fb[k] * s[k], yb[k] = fb[k] * c[k] + fa[k] * s[k];
            }
            a[u] = real ? pack4(ya) : make_uint2(0, 0);
            b[u] = real ? pack4(yb) : make_uint2(0, 0);
        }
        *reinterpret_cast<uint2*>(out + ea) = a[u];  // a value head is copied: the same elements, whichever they are
        *reinterpret_cast<uint2*>(out + eb) = b[u];
    }
}

int launch_qk_norm_rope(const void* X, int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int64_t ldx, const void* gq, const void* gk, float eps,
                        const float* cos_sin, int64_t n_pos, int32_t rot, bool pairs, const int32_t* pos, int64_t ldpos, int32_t n_axes,
                        const int32_t* sections, const int32_t* slots, void* Y, int64_t ldy, void* K, void* V, int64_t n_pages, int lg,
                        hipStream_t st) {
    RopeArgs p;
    p.X = static_cast<const uint16_t*>(X), p.T = T, p.ldx = ldx, p.Hq = Hq, p.Hkv = Hkv, p.heads = K ? Hq + 2 * Hkv : Hq;
    p.gq = static_cast<const uint16_t*>(gq), p.gk = static_cast<const uint16_t*>(gk), p.eps = eps, p.cos_sin = cos_sin, p.n_pos = n_pos;
    p.rot = rot, p.n_axes = n_axes, p.pos = pos, p.ldpos = ldpos, p.slots = slots, p.Y = static_cast<uint16_t*>(Y), p.ldy = ldy;
    p.s0 = n_axes > 1 ? sections[0] : rot / 2, p.s1 = n_axes > 2 ? p.s0 + sections[1] : rot / 2;
    p.quads = (p.s0 | p.s1) % 4 == 0;
    p.K = static_cast<uint16_t*>(K), p.V = static_cast<uint16_t*>(V), p.n_pages = n_pages, p.lg = lg;
    const int groups = (p.heads * D + 511) / 512;
    auto go = [&](auto kernel, int u) {
        p.units = (groups + u - 1) / u;
        const int64_t wgs = (T * p.units + 3) / 4;
        if (wgs > 0x7fffffff) return fail(OSC_ERR_UNSUPPORTED, "osc_qk_norm_rope: %lld rows are too many for one call", (long long)T);
        kernel<<<dim3((unsigned)wgs), 256, 0, st>>>(p);
        return check_launch("osc_qk_norm_rope");
    };
    // Four groups of heads a wavefront where there are wavefronts enough: the row's positions and angles are read once for all and 16 loads of a
    // lane are on their way; one group otherwise.  us: 8192 rows of 48 heads of 128 35.7 / 38.0, 2501 of 40 of 64 on three axes 7.4 / 8.9.
    auto pick = [&](auto d, auto turn, auto axes) {
        constexpr int W = decltype(d)::value;
        constexpr bool PR = decltype(turn)::value, AX = decltype(axes)::value;
        return T * groups >= 8192 ? go(qk_norm_rope_kernel<W, PR, AX, 4>, 4) : go(qk_norm_rope_kernel<W, PR, AX, 1>, 1);
    };
    auto with_axes = [&](auto d, auto turn) { return n_axes > 1 ? pick(d, turn, std::true_type{}) : pick(d, turn, std::false_type{}); };
    auto with_turn = [&](auto d) { return pairs ? with_axes(d, std::true_type{}) : with_axes(d, std::false_type{}); };
    return D == 128 ? with_turn(std::integral_constant<int, 128>{}) : with_turn(std::integral_constant<int, 64>{});
}

}  // namespace osc
