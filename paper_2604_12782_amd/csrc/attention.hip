// Attention of a step's rows over a shared prefix and each request's own cached tokens.
//
// Rows.  Query heads that share a key/value head are rows of one problem: row r = i * G + g is token i of its request, head g of
// the G = Hq / Hkv.  Requests are served in two ways:
//   long   their own tiles of 128 rows walk the prefix and then their own tokens (`joint`)
//   short  tiles of 32 rows walk the own tokens only; the short requests' rows, one behind the other, form tiles of 128 that
//          walk the prefix, which is therefore read once for all of them (`packed`; 32 rows or fewer: one tile of 32).  A prefix so short
//          that every request may walk it as well is the start of their own items instead (`pre_tiles`), and nothing is joined
// With a prefix, long means 256 rows or more (a last tile that is not full costs at most a third); without one, more than 32.
//
// Work.  Tiles of 128 rows and tiles of 32 rows are two lists.  An item is a tile with the tokens that it walks; the items of
// a list lie behind each other on a line that measures work, and every workgroup takes its piece of both lines, so
// all end together whatever the lengths are, no length is read back to the host, and an item is cut at most where a
// piece ends (pieces of the line of 32-row tiles may be a wavefront's, and rounded up to items: see the modes below).  What is computed of
// an item in one piece is a segment: unnormalised sums, their weight and their base.  Rows whose tokens are all in one segment are written
// as they are; all others go to the workspace and a second kernel joins them, in the order of the line: the same bits in every run.
// The two lists are bound by different things (matrix cores and power; HBM), so half of the workgroups take them in the other
// order.
//
// Bounds.  256 requests behind 32700 tokens take 233 to 238 us (86 for the products at the rate of bare matrix loops, 98 for the bytes at that of a
// reading pass), 40 prompts and decoding requests behind 4096 238 to 244 (109, products): matrix cores 30 to 40 % busy, the weights'
// exponentials and LDS reads take turns with them, and power brings the clock from 2.4 to 1.9 GHz meanwhile; no one part left out makes
// up the difference.  12 long requests without a prefix 66 us (42, bytes): 5.3 TB/s in the first kernel, then the second.  Small
// batches are bound by latency: the plan's reads, a few tiles that depend on one another, the second kernel's reads.
#include <algorithm>

#include "osc_internal.h"
#include "lds_dma.h"

namespace osc {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr int WG = 256, WROWS = 128, GROUPS = 256;
// Workgroups: two on a CU (LDS for their tiles), three where heads are small.
template <int D>
constexpr int attn_wgs() { return D == 128 ? 512 : 768; }
// How the narrow line is dealt out.  By workgroups, whose wavefronts take every fourth tile and merge their sums in LDS:
//   SOLO  an item a workgroup, nothing joined: no wide work, no more items than workgroups, and no request that sees more than SOLO_FEW
//         tokens, or SOLO_MANY where a quarter of the workgroups or more have an item
//   TEAM  few items: rounded up to pieces of TEAM tiles, as many as workgroups at most
//   CUT   long lines, cut where the workgroups' pieces end
// By wavefronts, each its own: items rounded up to pieces of 3, 6 or 12 tiles, the shortest that the wavefronts can take at once; not where
// items would come to more than FEW_PIECES of the longest each, whose joining costs more than the merges in LDS do.
// Here and below: us, 32 heads on 8, heads of 128 and in brackets of 64; "of up to n tokens" is n/B, 2n/B .. n, up to 100 of their own where
// nothing is said.  This rule / without the variant:  SOLO 32 requests behind 390 tokens 17.0 / 21.4 (14.1 / 17.4), and with four times the limits
// 16 of up to 2000 tokens 32.2 instead of 26.2 (25.4, 20.1);  TEAM 4 of up to 1000 tokens 16.5 / 17.6 (14.4 / 15.0);  wavefronts' pieces 100 of up to
// 100 tokens 16.7 / 26.1, 20.3 without the rule for pieces of 6 (13.3 / 21.9, 17.2), 200 behind 200 25.8 / 35.8 (22.2 / 27.0), 100 behind 3000
// 35.3 / 43.1 (25.8 / 29.1);  FEW_PIECES 16 of up to 8000 tokens 65.2 / 69.6 (39.5 / 40.8), one behind 30000 38.8 / 50.9 (26.0 / 35.6), 8 behind
// 12000 with up to 2000 of their own 33.2 / 42.7 (23.9 / 27.9).
enum { CUT = 0, SOLO = -1, TEAM = 5, PIECE1 = 3, PIECE2 = 6, PIECE3 = 12 };
constexpr int SOLO_FEW = 512, SOLO_MANY = 1024, FEW_PIECES = 4;
// Short requests walk the prefix themselves, tile after tile of their own items, where that is no more than this many tiles a wavefront
// (with 0, 4, 8: 32 requests behind 300 tokens 23.4, 15.6, 16.0 (18.9, 12.7, 12.5); behind 1000 22.4, 22.3, 25.7 (17.9, 20.8, 21.2: heads of 64 would
// do with less); behind 1500 22.5, 22.7, 32.7 (17.9, 18.0, 24.2)).
constexpr int INLINE_TILES = 4;
// The line of 32-row tiles is measured in tiles of 32 tokens, that of 128-row tiles in tokens.  Starting and ending a segment costs
// about as much as the EDGEs; no piece is smaller than the MINs.  MIN_WIDE: pieces of packed rows where workgroups have no more than 16 narrow tiles
// each (with 256 / 512: 32 requests behind 1000 tokens 22.3 / 26.8 (packed with heads of 128 alone), 20 behind 9000 26.4 / 29.4 (20.5 / 23.3)), and of
// prompts where nothing is packed (66 new tokens behind 1000 of the request's own 24.3 / 28.5, with 192 25.6 (18.9 / 22.4, 19.7)); twice that otherwise (with 512 / 256: 100
// behind 2000 with up to 2000 of their own 101 / 109 (60.4 / 62.2), 256 behind 1500 with up to 1000 135 / 145 (73.6 / 81.7); 30 decoding requests and 8
// prompts of 20 to 107 behind 1112 with up to 600 69.2 / 69.5 (38.8 / 44.0)).
constexpr int CUT_EDGE = 4, PIECE_EDGE = 1, MIN_NARROW = 8, WIDE_EDGE = 128, MIN_WIDE = 256;
// Wide tiles are dealt out whole, as many to every workgroup, and not joined, where the longest ones take no more than cut pieces and their joining:
// JOIN_COST tokens, and one for 2^JOIN_ROWS rows.  Whole / cut, the rule takes the whole ones: a prompt of 512 tokens 21.9 / 31.2 (16.9 / 24.2), of 2048
// 67 / 80 (48.8 / 57.0), 16 of 500 97 / 129 (61.5 / 91.7);  it cuts: a prompt of 8192 657 / 655 (381 / 380), 66 new tokens behind 4000 of the request's own 89 / 33
// (63 / 24), 300 behind 6000 132 / 61 (94 / 42), 12 of 20 behind 4000 each 92 / 65 (65 / 42), 30 of 40 behind 2000 87 / 83 (56 / 52), 12 of up to 20 behind 830 32 / 25 (25 / 21).
// It still cuts where whole tiles would do better: 12 of 20 behind 830 each 29.8 / 32.2 (23.1 / 24.1), 6 of 80 behind 900 32.3 / 40.1 (24.4 / 30.4).
constexpr int JOIN_COST = 512, JOIN_ROWS = 6;
constexpr int SUPER = 4096, MAX_SUPER = 16;
// Rows of a long request, with a prefix and without (with 128, 256, 512, 24 prompts behind 4000 tokens: of 40 tokens 123, 98, 104 (80, 65, 71), of 80 180, 179,
// 174 (114, 112, 113), of 120 244, 244, 274 (131, 130, 158)).
constexpr int LONG_PREFIX = 256, LONG = 33;

struct AttnArgs {
    const uint16_t* Q;
    int64_t T, ldq;
    int Hq, Hkv, G, tpt;  // tpt: tokens of a 128-row tile
    const uint8_t *K, *V;
    uint32_t n_pages;
    int lg;
    const int32_t* prefix_pages;
    int P;
    const int32_t* table;
    int64_t ldt;
    int max_kv;  // tokens that a row of the table can name
    const int32_t *kv_lens, *q_offsets;
    int B, per;  // per: requests of a group
    int pre_tiles;  // tiles of the prefix that short requests' items start with, or 0: their rows are packed
    int ns, ws;  // a step on the line of 32-row (128-row) tiles is 2^ns (2^ws) of its units: 0 unless the lines could pass 2^30
    float c;     // scale * log2(e): scores leave the matrix core unscaled, and powers are of two
    uint16_t* O;
    int64_t ldo;
    float* lse;
    // workspace: the plan, one record a request, segments in blocks of 32 rows: of long requests (two places a workgroup), of packed
    // tiles, of short requests
    struct Plan* plan;
    int* records;
    uint8_t* blocks;
    int64_t joint_blocks, packed_blocks, narrow_blocks;
};
template <int D>
constexpr int block_bytes() { return 32 * (D + 2) * 4; }  // [32][D] sums, [32] base and weight

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

// ---- where things are on the two lines -----------------------------------------------------------------------------------
struct Request {
    int q0, n, L;
};
struct Extent {  // of one request, or of all before one
    int narrow, items, rows, wide;
};
__device__ __forceinline__ Request request(const AttnArgs& p, int b) {
    Request r;
    r.q0 = p.q_offsets[b];  // checked before anything is looked up
    r.n = p.q_offsets[b + 1] - r.q0;
    r.L = min(max(p.kv_lens[b], 0), p.max_kv);
    return r;
}
__device__ __forceinline__ bool is_long(const AttnArgs& p, int n) { return n * p.G >= (p.P ? LONG_PREFIX : LONG); }
__device__ __forceinline__ int narrow_tiles(const AttnArgs& p, int n) { return (n * p.G + 31) >> 5; }
// `piece`: CUT or the length that items are rounded up to
__device__ __forceinline__ int narrow_edge(int piece) { return piece == CUT ? CUT_EDGE : PIECE_EDGE; }
__device__ __forceinline__ int narrow_units(const AttnArgs& p, int L, int piece) { return (((L + 31) >> 5) + narrow_edge(piece) + (1 << p.ns) - 1) >> p.ns; }
__device__ __forceinline__ int rounded(int n, int piece) { return piece ? (n + piece - 1) / piece * piece : n; }
__device__ __forceinline__ int narrow_length(const AttnArgs& p, int L, int piece) { return piece == SOLO ? 1 : rounded(narrow_units(p, L, piece) + p.pre_tiles, piece); }
__device__ __forceinline__ int narrow_tile(const AttnArgs& p, int y, int piece) { return max(0, (y << p.ns) - narrow_edge(piece)); }  // the first tile at place y of an item
// Tiles of a long request on their line: each sees `step` more tokens than the one before it, the first `seen` and that; dealt out whole
// (SOLO), each is 1 long.
__device__ __forceinline__ int wide_step(const AttnArgs& p, int piece) { return piece == SOLO ? 0 : p.tpt >> p.ws; }
__device__ __forceinline__ int wide_seen(const AttnArgs& p, const Request& r, int piece) { return piece == SOLO ? 1 : ((WIDE_EDGE + p.P + max(r.L - r.n, 0)) >> p.ws) + 1; }
__device__ __forceinline__ int wide_sum(int step, int seen, int k) { return k * seen + step * (k * (k + 1) / 2); }  // the first k
__device__ __forceinline__ int wide_length(int step, int seen, int tile) { return seen + (tile + 1) * step; }
__device__ __forceinline__ int wide_tiles(const AttnArgs& p, int n) { return (n + p.tpt - 1) / p.tpt; }
__device__ __forceinline__ int packed_length(const AttnArgs& p, int blocks) { return ((blocks * 64 + WIDE_EDGE) >> p.ws) + 1; }
__device__ __forceinline__ Extent extent(const AttnArgs& p, const Request& r, int piece) {
    Extent e{0, 0, 0, 0};
    if (r.n == 0) return e;
    if (is_long(p, r.n)) {
        e.wide = p.Hkv * wide_sum(wide_step(p, piece), wide_seen(p, r, piece), wide_tiles(p, r.n));
    } else {
        e.items = narrow_tiles(p, r.n) * p.Hkv;
        e.narrow = e.items * narrow_length(p, r.L, piece);
        if (p.P && !p.pre_tiles) e.rows = r.n * p.G;
    }
    return e;
}

// What follows from the totals: the prefix's items, which come first on their line, and the pieces.
// Wide pieces are equal, in tokens or whole tiles; the first `with_wide` workgroups have one.  A narrow piece is a wavefront's: those of these workgroups take
// pieces of length `a`, the others, which come first on the line, of length `b`, so that all have the same to do: a wide block of 64 tokens takes about a third
// of the time of a narrow tile (2 us where a CU has two workgroups at it; 16 KB, 6 us where all wavefronts share 5.5 TB/s).  Where there are
// wavefronts enough for pieces of 3, 6 or 12 tiles, items are rounded up to whole ones: a wavefront has parts of one item, and most
// items are in one piece.  Where pieces are workgroups', the same with four times the tiles.
// (Tests read it at the workspace's start, by the places of its members.)
struct Plan {
    int narrow, wide;      // lengths of the lines
    int narrow0, items0;   // of which the prefix's narrow items are the first
    int wide0, head;       // of which the packed tiles are the first, `head` for every key/value head
    int wide_per, wide_piece, a, b, cut;
    int with_wide, others, piece, team;
    int rows, tiles, supers, super, nbp;  // packed rows, their wide tiles; pieces of the prefix, blocks of 64 tokens in one, in the prefix
    int valid;  // offsets are in order
    int joins;  // anything to join
};
// Many packed tiles walk the prefix in pieces that stay in an XCD's L2 meanwhile.
__device__ __host__ inline int super_count(int64_t P, int64_t tiles) {
    const int64_t n = (P + SUPER - 1) / SUPER;
    return tiles > 1 ? (int)(n < 1 ? 1 : n > MAX_SUPER ? MAX_SUPER : n) : 1;
}
template <int D>
__device__ __forceinline__ Plan make_plan(const AttnArgs& p, int narrow, int teams, int pieces1, int pieces2, int pieces3, int items, int rows, int wide, int wide_items, int longest, int small) {
    constexpr int N = attn_wgs<D>(), WAVES = 4 * N;
    Plan a;
    a.valid = 1;
    a.rows = rows;
    a.nbp = (p.P + 63) >> 6;
    a.narrow0 = a.items0 = a.wide0 = a.head = 0;
    a.tiles = a.supers = a.super = 0;
    if (rows > 0 && rows <= 32) {
        const int n = narrow_units(p, p.P, TEAM);
        a.items0 = p.Hkv;
        narrow += p.Hkv * narrow_units(p, p.P, CUT);
        teams += p.Hkv * ((n + TEAM - 1) / TEAM);
        pieces1 += p.Hkv * ((n + PIECE1 - 1) / PIECE1), pieces2 += p.Hkv * ((n + PIECE2 - 1) / PIECE2), pieces3 += p.Hkv * ((n + PIECE3 - 1) / PIECE3);
    }
    // all in one piece of the second length, and nothing else: nothing to join, which takes longer than three tiles
    const bool alone = rows == 0 && wide == 0 && pieces2 == items && items <= WAVES;
    const bool solo = rows == 0 && wide == 0 && items <= N && (items < N / 4 ? small & 1 : small >> 1);
    a.piece = solo ? SOLO : alone ? PIECE2 : teams <= N ? TEAM : pieces3 > FEW_PIECES * items ? CUT : pieces1 <= WAVES ? PIECE1 : pieces2 <= WAVES ? PIECE2 : pieces3 <= WAVES ? PIECE3 : CUT;
    a.team = a.piece == SOLO || a.piece == TEAM || a.piece == CUT;
    if (solo) narrow = items;
    else if (a.piece) narrow = a.piece * (a.piece == TEAM ? teams : a.piece == PIECE1 ? pieces1 : a.piece == PIECE2 ? pieces2 : pieces3);
    if (a.items0) a.narrow0 = p.Hkv * rounded(narrow_units(p, p.P, a.piece), a.piece);
    a.wide_per = 0;
    if (rows > 32) {
        a.tiles = (rows + WROWS - 1) / WROWS;
        const int th = p.Hkv * a.tiles;
        const bool whole = wide == 0 && th <= N;  // nothing else on the line: an item a piece, in one round
        const int load = (narrow + (int)min((int64_t)th * a.nbp * 5 / 4, (int64_t)1 << 29)) / N;
        a.supers = whole ? max(1, min(N / th, a.nbp * 64 / (load < 16 ? MIN_WIDE : 2 * MIN_WIDE))) : super_count(p.P, a.tiles);
        a.super = (a.nbp + a.supers - 1) / a.supers;
        a.supers = (a.nbp + a.super - 1) / a.super;
        a.head = a.tiles * a.supers * packed_length(p, a.super);
        a.wide0 = p.Hkv * a.head;
        if (whole) a.wide_per = packed_length(p, a.super);
    }
    a.narrow = narrow;
    a.wide = a.wide0 + wide;
    a.wide_piece = CUT;
    int busy = a.wide_per;  // what a workgroup has of the wide line
    if (!busy) {
        busy = a.wide_per = max((a.wide + N - 1) / N, max((a.wide0 ? 2 * MIN_WIDE : MIN_WIDE) >> p.ws, 1));
        if (wide_items > 0 && rows <= 32) {
            const int each = (wide_items + N - 1) / N;
            if ((int64_t)each * longest <= busy + ((JOIN_COST + (p.T * p.Hq >> JOIN_ROWS)) >> p.ws))
                a.wide_piece = SOLO, a.wide = wide_items, a.wide_per = each, busy = each * (wide / wide_items);
        }
    }
    a.with_wide = ((a.wide + a.wide_per - 1) / a.wide_per + 7) / 8 * 8;  // as many on every XCD
    const int all = a.team ? N : WAVES, with = all / N * a.with_wide, others = all - with;
    const int cost = (int)min((((int64_t)busy << p.ws) * 5 / (64 * 4) * N / all) >> p.ns, (int64_t)1 << 18);
    a.b = (narrow + all - 1) / all + (with * cost + all - 1) / all;
    a.a = a.b - cost;
    if (a.piece == SOLO) a.a = a.b = 1;
    else if (a.piece) a.a = a.b = a.piece;
    else if (others == 0) a.a = max((narrow + all - 1) / all, MIN_NARROW);
    else if (a.a < MIN_NARROW) a.a = MIN_NARROW, a.b = max((narrow + others - 1) / others, MIN_NARROW);
    a.others = others;
    a.cut = a.b * others;
    a.joins = (a.wide > 0 && a.wide_piece != SOLO) || a.items0 > 0 || (a.piece != SOLO && (!a.piece || narrow > items * a.piece));
    return a;
}
// the workgroup or wavefront, in the order of the pieces, that has place x of the narrow line: those without a wide piece come first
__device__ __forceinline__ int narrow_piece_of(const Plan& a, int x) { return x < a.cut ? x / a.b : a.others + (x - a.cut) / a.a; }

// Running sums over groups of `per` requests, in LDS: what a place on a line or a packed row is searched in.
struct Sums {
    int narrow[GROUPS], items[GROUPS], rows[GROUPS], wide[GROUPS];
};
// the last group whose sum does not exceed x (x below the total)
__device__ __forceinline__ int find_group(const int (&sums)[GROUPS], int x, int lane) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < GROUPS / 64; ++k) n += __popcll(__ballot(sums[k * 64 + lane] <= x));
    return n - 1;
}
// The request that holds place x of a line: its number and what is before it.  All lanes of a wavefront take part.
template <bool WIDE>
__device__ __forceinline__ int find_request(const AttnArgs& p, const Sums& s, int piece, int x, int lane, Extent& before) {
    const int g = uni(find_group(WIDE ? s.wide : s.narrow, x, lane));
    before = Extent{uni(s.narrow[g]), uni(s.items[g]), uni(s.rows[g]), uni(s.wide[g])};
    int b = g * p.per;
    if (p.per > 1) {  // at most 32 requests of a group: one a lane
        Extent e{0, 0, 0, 0};
        if (lane < p.per && b + lane < p.B) e = extent(p, request(p, b + lane), piece);
        Extent sum = e;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int n = __shfl_up(sum.narrow, d), i = __shfl_up(sum.items, d), r = __shfl_up(sum.rows, d), w = __shfl_up(sum.wide, d);
            if (lane >= d) sum.narrow += n, sum.items += i, sum.rows += r, sum.wide += w;
        }
        const int end = WIDE ? before.wide + sum.wide : before.narrow + sum.narrow;
        const int k = uni(__ffsll((unsigned long long)__ballot(end > x)) - 1);  // lanes past the group repeat its end, which is above x
        before.narrow += uni(__shfl(sum.narrow - e.narrow, k));
        before.items += uni(__shfl(sum.items - e.items, k));
        before.rows += uni(__shfl(sum.rows - e.rows, k));
        before.wide += uni(__shfl(sum.wide - e.wide, k));
        b += k;
    }
    return uni(b);
}
// The token and head of packed row r (below the total), each lane its own.
__device__ __forceinline__ void packed_row(const AttnArgs& p, const Sums& s, int r, int& t, int& g) {
    int lo = 0, hi = GROUPS;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.rows[mid] <= r) lo = mid;
        else hi = mid;
    }
    int at = s.rows[lo];
    int b = lo * p.per;
    Request q = request(p, b);
    for (int last = min(p.B, b + p.per) - 1; b < last; q = request(p, ++b)) {
        const int n = extent(p, q, CUT).rows;
        if (at + n > r) break;
        at += n;
    }
    const int i = (r - at) / p.G;
    t = q.q0 + i;
    g = r - at - i * p.G;
}

__device__ __forceinline__ uint32_t lds_at(const uint8_t* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p; }

// ---- tiles of cached tokens in LDS ---------------------------------------------------------------------------------------------
// Rows of D bf16 in pieces of 16 bytes; piece c of row r sits at c ^ spread(r), so that both readers find all banks: keys by
// 32 rows of one piece, values by 8 rows of four neighbouring pieces.
template <int D>
__device__ __forceinline__ int spread(int r) {
    return D == 128 ? (r & 3) << 2 | ((r >> 2) & 3) : ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
}
// Start of the 16-token run that token j lies in (a page holds whole runs), for keys; values lie V - K further.
template <int D>
__device__ __forceinline__ const uint8_t* run_of(const AttnArgs& p, int page_number, int h, int j) {
    uint32_t page = (uint32_t)uni(page_number);
    if (page >= p.n_pages) page = 0;  // nothing outside the cache is read, whatever a table holds
    return p.K + ((((int64_t)page * p.Hkv + h) << p.lg) + ((j & ((1 << p.lg) - 1)) & ~15)) * (D * 2);
}
// 16 bytes a lane from memory to LDS, at `to` + 16 lane.  (The request's own instruction, not the compiler's builtin: that
// makes every later LDS read wait for all requests on their way, also those for other tiles.  It has no result in
// registers; the waits are counted by hand below.)
__device__ __forceinline__ void request16(const uint8_t* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(to) : "memory");  // m0 is not the compiler's to keep: it sets it before any use
}
// Asks for 16 rows, tile rows 16 * half .., of which `last` + 1 exist from the run's start: rows past the last token repeat it, so that
// whatever a page holds there is never multiplied.
template <int D>
__device__ __forceinline__ void fetch16(const uint8_t* run, int half, int last, uint32_t to, int lane) {
    constexpr int CH = D / 8, RPI = 64 / CH, NI = 16 / RPI;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int r = i * RPI + lane / CH, piece = (lane % CH) ^ spread<D>(r);  // spread() repeats after 16 rows
        const uint32_t whole = r * (D * 2) + piece * 16, cut = min(r, last) * (D * 2) + piece * 16;
        request16(run, last == 15 ? whole : cut, to + half * (16 * D * 2) + i * 1024);
    }
}

// Softmax state of 32 rows, transposed: lane l holds row l % 32; its upper and lower half hold different tokens of a tile and
// different channels of the sums.  `sum` is the lane's own share.  Weights are 2^(score * c - base); the base follows the
// maximum only when that is 2^8 above it, so sums are rarely scaled.
template <int D>
struct State {
    v16f o[D / 32];
    float base, sum;
};
template <int D>
__device__ __forceinline__ void clear(State<D>& st) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) st.o[d] = v16f{};
    st.base = -INFINITY, st.sum = 0.0f;
}
__device__ __forceinline__ float half_max(float v) {
    const int x = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return fmaxf(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const int x = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
}

// N tiles of 32 tokens: S^T = K Q^T leaves a lane 16 tokens of its row a tile, the weights go to bf16 and are the second operand of
// O^T += V^T P^T as they lie, because the order of the tokens inside a product is free as long as both operands have the same.
// LDS addresses are numbers, the lane's part made once: a tile starts at a multiple of 256 bytes, so a piece's place is an exclusive or.
template <int D>
__device__ __forceinline__ uint32_t key_lane(int lane) {
    const int r = lane & 31;
    return r * (D * 2) + (((lane >> 5) ^ spread<D>(r)) << 4);
}
template <int D>
__device__ __forceinline__ uint32_t value_lane(int lane) {
    const int i = lane & 15, row = 4 * (lane >> 5) + (i >> 2);
    return row * (D * 2) + (((((lane >> 4) & 1) * 2 + ((i & 3) >> 1)) ^ spread<D>(row)) << 4) + (i & 1) * 8;
}
__device__ __forceinline__ v16f mfma(v8bf a, v8bf b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v8bf read16(uint32_t at) { return *(const __attribute__((address_space(3))) v8bf*)(uintptr_t)at; }
__device__ __forceinline__ v4s read_turned(uint32_t at) {  // four rows of one channel, of 16 channels over 16 lanes
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)at);
}
// Reads run a batch ahead of the products: the barriers keep the compiler from drawing each read to its use.
template <int D, int N>
__device__ __forceinline__ void scores(v16f (&s)[N], const v8bf (&q)[D / 16], uint32_t kt) {
    constexpr int BATCH = 4 / N, STEPS = D / 16 / BATCH;  // pieces of a batch: four reads
    v8bf f[2][BATCH][N];
    auto read = [&](int j) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
#pragma unroll
            for (int u = 0; u < N; ++u) f[j & 1][i][u] = read16((kt ^ ((j * BATCH + i) << 5)) + u * (32 * D * 2));
    };
#pragma unroll
    for (int u = 0; u < N; ++u) s[u] = v16f{};
    read(0);
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        if (j + 1 < STEPS) read(j + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
#pragma unroll
            for (int u = 0; u < N; ++u) s[u] = mfma(f[j & 1][i][u], q[j * BATCH + i], s[u]);
        __builtin_amdgcn_sched_barrier(0);
    }
}
// `seen`: tokens below it count for the lane's row
template <int N>
__device__ __forceinline__ void mask(v16f (&s)[N], int lane, int seen) {
    const int left = seen - 4 * (lane >> 5);
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[u][e] = 32 * u + (e & 3) + 8 * (e >> 2) < left ? s[u][e] : -INFINITY;
}
template <int D, int N>
__device__ __forceinline__ void weigh(State<D>& st, v16f (&s)[N], float c) {
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
    top = half_max(top) * c;
    if (__ballot(top > st.base + 8.0f)) {
        const float base = fmaxf(st.base, top);
        const float fade = base == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(st.base - base);
        st.base = base;
        st.sum *= fade;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) st.o[d][e] *= fade;
    }
    const float base = st.base == -INFINITY ? 0.0f : st.base;  // a row that has seen nothing yet keeps sums of zero
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][e], c, -base));
            sum += s[u][e];
        }
    st.sum += sum;
}
template <int D>
union Values {  // 16 tokens of all channels
    v4s part[D / 16];
    v8bf all[D / 32];
};
template <int D>
__device__ __forceinline__ void read_values(Values<D>& f, uint32_t vt, int t) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        f.part[2 * d] = read_turned((vt ^ (d << 6)) + 16 * t * (D * 2));
        f.part[2 * d + 1] = read_turned((vt ^ (d << 6) ^ 32) + (16 * t + 8) * (D * 2));  // eight tokens on, the spread differs in one bit
    }
}
// `f`: the first 16 tokens' values
template <int D, int N>
__device__ __forceinline__ void gather(State<D>& st, const v16f (&s)[N], const Values<D>& first, uint32_t vt) {
    Values<D> f[2];
    f[0] = first;
#pragma unroll
    for (int t = 0; t < 2 * N; ++t) {
        if (t + 1 < 2 * N) read_values<D>(f[(t + 1) & 1], vt, t + 1);
        v8bf w;  // rounded to 8 bits for the matrix core: half an ulp each, and of either sign; their sum is taken before
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (__bf16)s[t >> 1][8 * (t & 1) + e];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) st.o[d] = mfma(f[t & 1].all[d], w, st.o[d]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){a, b}, v2bf));  // nearest even
}
// A row without weight has seen nothing: zeros, and -infinity.  A weight that is NaN (queries that are not finite) is not taken for
// none: it makes the row NaN, whichever way its sums are finished.
__device__ __forceinline__ float inverse(float sum) { return sum == 0.0f ? 0.0f : 1.0f / sum; }
__device__ __forceinline__ float lse_of(float base, float sum) {
    return sum == 0.0f ? -INFINITY : (base + __log2f(sum)) * 0.69314718055994531f;
}
__device__ __forceinline__ void lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_sched_barrier(0);
}

// a barrier for LDS alone: it does not wait for stores to memory
__device__ __forceinline__ void lds_barrier() {
    lds_order();
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    lds_order();
}

// A row's sums: normalised, as its result, or as they are, to the workspace.
template <int D>
__device__ __forceinline__ void leave(const AttnArgs& p, const State<D>& st, bool direct, int64_t t, int head, uint8_t* blk, int row, int hi) {
    if (direct) {
        const float inv = inverse(st.sum);
        uint16_t* out = p.O + t * p.ldo + head * D + 4 * hi;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<uint2*>(out + 32 * d + 8 * e) =
                    make_uint2(pack2(st.o[d][4 * e] * inv, st.o[d][4 * e + 1] * inv), pack2(st.o[d][4 * e + 2] * inv, st.o[d][4 * e + 3] * inv));
        if (p.lse && hi == 0) p.lse[t * p.Hq + head] = lse_of(st.base, st.sum);
    } else {
        float* out = reinterpret_cast<float*>(blk) + row * D + 4 * hi;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<float4*>(out + 32 * d + 8 * e) = make_float4(st.o[d][4 * e], st.o[d][4 * e + 1], st.o[d][4 * e + 2], st.o[d][4 * e + 3]);
        if (hi == 0) *reinterpret_cast<float2*>(blk + (32 * D + row * 2) * 4) = make_float2(st.base, st.sum);
    }
}

// The four wavefronts' parts of the same rows, each in its own LDS as [row][channel], pieces of 16 bytes spread by row; then eight lanes a row.
template <int D>
__device__ __forceinline__ void merge(const AttnArgs& p, const State<D>& st, uint8_t* lds, float* stats, int tid, int wave, int lane, int rows, bool direct, int64_t t, int head,
                                      uint8_t* blk) {
    float* parts = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = lane & 31, piece = 8 * d + 2 * e + (lane >> 5);
            *reinterpret_cast<float4*>(parts + wave * 32 * D + row * D + ((piece ^ (row & 7)) << 2)) =
                make_float4(st.o[d][4 * e], st.o[d][4 * e + 1], st.o[d][4 * e + 2], st.o[d][4 * e + 3]);
        }
    if (lane < 32) stats[wave * 32 + lane] = st.base, stats[128 + wave * 32 + lane] = st.sum;
    lds_barrier();
    const int row = tid >> 3, part = tid & 7;
    if (row < rows) {
        float base = -INFINITY, f[4], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) base = fmaxf(base, stats[k * 32 + row]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[k] = base == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(stats[k * 32 + row] - base);
            sum += f[k] * stats[128 + k * 32 + row];
        }
        const float inv = inverse(sum);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const int piece = k * 8 + part;
            float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float4 z = *reinterpret_cast<const float4*>(parts + v * 32 * D + row * D + ((piece ^ (row & 7)) << 2));
                y[0] = fmaf(f[v], z.x, y[0]), y[1] = fmaf(f[v], z.y, y[1]), y[2] = fmaf(f[v], z.z, y[2]), y[3] = fmaf(f[v], z.w, y[3]);
            }
            if (direct) *reinterpret_cast<uint2*>(p.O + t * p.ldo + head * D + piece * 4) = make_uint2(pack2(y[0] * inv, y[1] * inv), pack2(y[2] * inv, y[3] * inv));
            else *reinterpret_cast<float4*>(blk + (row * D + piece * 4) * 4) = make_float4(y[0], y[1], y[2], y[3]);
        }
        if (part == 0) {
            if (!direct) *reinterpret_cast<float2*>(blk + (32 * D + row * 2) * 4) = make_float2(base, sum);
            else if (p.lse) p.lse[t * p.Hq + head] = lse_of(base, sum);
        }
    }
    lds_barrier();  // the next item's tiles land where these parts are
}

// ---- a piece of the line of 32-row tiles ----------------------------------------------------------------------------------------
// A wavefront's tiles of 32 tokens are in LDS that no other wavefront uses.  Keys of the next tile are asked for once this tile's
// scores are there, values once they are summed, so half a tile or more is on its way at any time, and no wavefront
// waits for another before a team's sums are merged.
template <int D>
__device__ __forceinline__ void narrow_piece(const AttnArgs& p, const Plan& plan, const Sums& sums, uint8_t* lds, float* stats) {
    constexpr int TILE = 32 * D * 2, NI = D / 16;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // what follows from it is made here, not kept in registers from the kernel's start
    const int lane = tid & 63, wave = uni(tid >> 6);
    const int64_t to_v = p.V - p.K;
    const uint32_t kt = lds_at(lds) + wave * 2 * TILE, vt = kt + TILE, kl = kt + key_lane<D>(lane), vl = vt + value_lane<D>(lane);
    const bool team = plan.team;
    const int wg = blockIdx.x, order = wg < plan.with_wide ? attn_wgs<D>() - plan.with_wide + wg : wg - plan.with_wide, w = team ? order : order * 4 + wave;
    int x = w < plan.others ? w * plan.b : plan.cut + (w - plan.others) * plan.a;
    const int end = min(x + (w < plan.others ? plan.b : plan.a), plan.narrow);
    while (x < end) {
        // the item at x: its start and length on the line, its rows, its tokens
        int start, item, length, h, r0, rows, n_prefix, tokens = 0, seen = 0, clear_to = 0, b = -1;  // tiles of the prefix, then own tokens
        Request rq{0, 0, 0};
        if (x < plan.narrow0) {
            length = rounded(narrow_units(p, p.P, plan.piece), plan.piece);
            h = x / length;
            start = h * length, item = h;
            r0 = 0, rows = plan.rows, n_prefix = (p.P + 31) >> 5;
        } else {
            Extent before;
            b = find_request<false>(p, sums, plan.piece, x - plan.narrow0, lane, before);
            rq = request(p, b);
            length = narrow_length(p, rq.L, plan.piece);
            const int nt = narrow_tiles(p, rq.n), k = (x - plan.narrow0 - before.narrow) / length;
            start = plan.narrow0 + before.narrow + k * length, item = plan.items0 + before.items + k;
            h = k / nt;
            r0 = (k - h * nt) * 32, rows = rq.n * p.G;
            tokens = max(0, rq.L - rq.n + min(r0 + 31, rows - 1) / p.G + 1), clear_to = rq.L - rq.n + r0 / p.G + 1;
            n_prefix = p.pre_tiles;
        }
        const int stop = min(end, start + length);
        const int step = team ? 4 : 1, t0 = narrow_tile(p, x - start, plan.piece) + (team ? wave : 0), t1 = min(stop == start + length ? 0x7fffffff : narrow_tile(p, stop - start, plan.piece), n_prefix + ((tokens + 31) >> 5));
        const bool whole = x == start && stop == start + length;
        x = stop;

        const int rc = min(r0 + (lane & 31), rows - 1);
        int ti = rc / p.G, g = rc - ti * p.G;
        if (b < 0) {
            packed_row(p, sums, rc, ti, g);
        } else {
            seen = rq.L - rq.n + ti + 1;
            ti += rq.q0;
        }
        v8bf q[D / 16];
        const uint16_t* qp = p.Q + (int64_t)ti * p.ldq + (h * p.G + g) * D + (lane >> 5) * 8;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = *reinterpret_cast<const v8bf*>(qp + k * 16);

        State<D> st;
        clear(st);
        auto runs = [&](int tile, const uint8_t*& a, const uint8_t*& c) {
            const bool pre = tile < n_prefix;
            const int32_t* pages = pre ? p.prefix_pages : p.table + (int64_t)b * p.ldt;
            const int j = (pre ? tile : tile - n_prefix) * 32, j2 = min(j + 16, (pre ? p.P : tokens) - 1), one = pages[j >> p.lg], two = pages[j2 >> p.lg];
            a = run_of<D>(p, one, h, j);
            c = run_of<D>(p, two, h, j2);
        };
        auto fetch = [&](int tile, const uint8_t* a, const uint8_t* c, int64_t shift, uint32_t dst) {
            const bool pre = tile < n_prefix;
            const int last = (pre ? p.P : tokens) - 1, left = last - (pre ? tile : tile - n_prefix) * 32;
            fetch16<D>(a + shift, 0, min(left, 15), dst, lane);
            fetch16<D>(c + shift, 1, left >= 16 ? min(left - 16, 15) : last & 15, dst, lane);
        };
        int tile = t0;
        const uint8_t *ra = nullptr, *rb = nullptr, *na = nullptr, *nb = nullptr;
        if (tile < t1) {
            runs(tile, ra, rb);
            fetch(tile, ra, rb, 0, kt);
            lds_order();  // the waits below count: keys first
            fetch(tile, ra, rb, to_v, vt);
        }
        for (; tile < t1; tile += step) {
            const bool more = tile + step < t1;
            if (more) runs(tile + step, na, nb);
            wait_vmcnt<NI>();  // the keys are there; the values may not be
            lds_order();
            v16f s[1];
            scores<D, 1>(s, q, kl);
            lds_order();
            __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the keys are read
            if (more) fetch(tile + step, na, nb, 0, kt);
            const bool pre = tile < n_prefix;
            const int j0 = (pre ? tile : tile - n_prefix) * 32;
            if (j0 + 32 > (pre ? p.P : clear_to)) mask<1>(s, lane, (pre ? p.P : seen) - j0);
            weigh<D, 1>(st, s, p.c);
            if (more) wait_vmcnt<NI>();
            else wait_vmcnt<0>();
            lds_order();
            Values<D> f;
            read_values<D>(f, vl, 0);
            gather<D, 1>(st, s, f, vl);
            lds_order();
            __builtin_amdgcn_s_waitcnt(0xC07F);
            if (more) fetch(tile + step, na, nb, to_v, vt);
        }
        st.sum = half_sum(st.sum);
        const bool direct = whole && (p.P == 0 || p.pre_tiles);
        const int slot = item + w;
        uint8_t* blk = p.blocks + (p.joint_blocks + p.packed_blocks + slot) * block_bytes<D>();
        if (team) {
            const int row = r0 + (tid >> 3);
            merge<D>(p, st, lds, stats, tid, wave, lane, direct || slot < p.narrow_blocks ? rows - r0 : 0, direct, rq.q0 + row / p.G, h * p.G + row % p.G, blk);
        } else if (r0 + (lane & 31) < rows && (direct || slot < p.narrow_blocks)) {
            leave<D>(p, st, direct, (int64_t)ti, h * p.G + g, blk, lane & 31, lane >> 5);
        }
    }
}

// ---- a piece of the line of 128-row tiles -----------------------------------------------------------------------------------------
// Every wavefront has 32 rows; all read the same 64 tokens from LDS, of which each has asked for 16, a block ahead.
template <int D>
__device__ __forceinline__ void wide_piece(const AttnArgs& p, const Plan& plan, const Sums& sums, uint8_t* lds, int w) {
    constexpr int TILE = 64 * D * 2;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // what follows from it is made here, not kept in registers from the kernel's start
    const int lane = tid & 63, wave = uni(tid >> 6);
    const int64_t to_v = p.V - p.K;
    const uint32_t kl = key_lane<D>(lane), vl = value_lane<D>(lane);
    // Segments are taken from the piece's end: the start of a tile first, the rest of the tile before it after that.  So all
    // workgroups walk the tokens that they share side by side, whatever their pieces' places, and an XCD's L2 reads them once.
    const int begin = w * plan.wide_per;
    int stop = min(begin + plan.wide_per, plan.wide);
    while (stop > begin) {
        int x = stop - 1;
        int64_t slot;
        int start, length, h, rows, n_prefix, n_own, b = -1, first_block = 0, own = 0, r0 = 0, t_base = 0;
        Request rq{0, 0, 0};
        if (x < plan.wide0) {
            // head, then piece of the prefix, then tile
            length = packed_length(p, plan.super);
            h = x / plan.head;
            const int y = x - h * plan.head, item = y / length, s = item / plan.tiles, tile = item - s * plan.tiles;
            const int blocks = min(plan.super, plan.nbp - s * plan.super);
            start = h * plan.head + item * length;
            r0 = tile * WROWS, rows = plan.rows - r0;
            first_block = s * plan.super, n_prefix = blocks, n_own = 0;
            slot = p.joint_blocks + ((int64_t)(h * plan.supers + s) * plan.tiles + tile + w) * 4;
        } else {
            Extent before;
            b = find_request<true>(p, sums, plan.wide_piece, x - plan.wide0, lane, before);
            rq = request(p, b);
            const int nt = wide_tiles(p, rq.n);
            const int step = wide_step(p, plan.wide_piece), seen = wide_seen(p, rq, plan.wide_piece), head = wide_sum(step, seen, nt), y = x - plan.wide0 - before.wide;
            h = y / head;
            int lo = 0, hi = nt;  // the last tile that starts at or before y
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (wide_sum(step, seen, mid) <= y - h * head) lo = mid;
                else hi = mid;
            }
            start = plan.wide0 + before.wide + h * head + wide_sum(step, seen, lo);
            length = wide_length(step, seen, lo);
            t_base = lo * p.tpt;
            const int tokens = min(p.tpt, rq.n - t_base);
            rows = tokens * p.G;
            own = max(0, rq.L - rq.n + t_base + tokens);
            n_prefix = plan.nbp, n_own = (own + 63) >> 6;
            slot = 0;
        }
        x = max(begin, start);
        const int blocks = n_prefix + n_own;
        constexpr int EDGE = WIDE_EDGE;
        auto block_at = [&](int y) {  // the same for both workgroups at a cut, and not falling: all that is asked of it
            const int edge = EDGE >> p.ws;
            return y >= length ? blocks : min(blocks, (int)((float)max(y - edge, 0) * (float)blocks / (float)(length - edge)));
        };
        const int k0 = block_at(x - start), k1 = block_at(stop - start);
        const bool whole = x == start && stop == start + length;
        if (b >= 0) slot = (2 * (int64_t)w + (x == start)) * 4;

        const int r = wave * 32 + (lane & 31), rc = min(r, rows - 1);
        int ti = rc / p.G, g = rc - ti * p.G, seen = 0;
        if (b < 0) packed_row(p, sums, r0 + rc, ti, g);
        else {
            seen = rq.L - rq.n + t_base + ti + 1;
            ti += rq.q0 + t_base;
        }
        const int clear_to = rq.L - rq.n + t_base + (wave * 32) / p.G + 1;  // own tokens that all of the wavefront's rows see
        v8bf q[D / 16];
        const uint16_t* qp = p.Q + (int64_t)ti * p.ldq + (h * p.G + g) * D + (lane >> 5) * 8;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = *reinterpret_cast<const v8bf*>(qp + k * 16);

        State<D> st;
        clear(st);
        // the wavefront's 16 tokens of block k: their page's number is read a block before it is needed
        auto token = [&](int k, int& last) {
            const bool pre = k < n_prefix;
            const int n = pre ? p.P : own, j = ((pre ? k + first_block : k - n_prefix) * 64) + wave * 16;
            const int jc = min(j, n - 1);
            last = j < n ? min(15, n - 1 - j) : (n - 1) & 15;
            return jc;
        };
        auto page_of = [&](int k) {
            int last;
            const int j = token(k, last) >> p.lg;
            return k < n_prefix ? p.prefix_pages[j] : p.table[(int64_t)b * p.ldt + j];
        };
        auto fetch = [&](int k, int page) {
            int last;
            const int j = token(k, last);
            const uint8_t* run = run_of<D>(p, page, h, j);
            const uint32_t dst = lds_at(lds) + (k & 1) * 2 * TILE;
            fetch16<D>(run, wave, last, dst, lane);
            fetch16<D>(run + to_v, wave, last, dst + TILE, lane);
        };
        int page = 0;
        if (k0 < k1) {
            fetch(k0, page_of(k0));
            if (k0 + 1 < k1) page = page_of(k0 + 1);
        }
        auto next = [&](int k) {
            wait_vmcnt<0>();
            __syncthreads();  // everyone's part of block k is there, and everyone is done with block k - 1
            if (k + 1 < k1) {
                fetch(k + 1, page);
                if (k + 2 < k1) page = page_of(k + 2);
            }
        };
        // A CU's older wavefronts go first when both want the same unit, and its older workgroup would end long before the
        // younger: they take turns block by block.
        const int turn = blockIdx.x >= attn_wgs<D>() / 2;
        if (wave * 32 < rows) {
            for (int k = k0; k < k1; ++k) {
                next(k);
                if ((k ^ turn) & 1) __builtin_amdgcn_s_setprio(1);
                else __builtin_amdgcn_s_setprio(0);
                const uint32_t buffer = lds_at(lds) + (k & 1) * 2 * TILE;
                const bool pre = k < n_prefix;
                const int j0 = (pre ? k + first_block : k - n_prefix) * 64;
                v16f s[2];
                scores<D, 2>(s, q, buffer + kl);
                Values<D> f;  // on their way while the weights are made
                read_values<D>(f, buffer + TILE + vl, 0);
                if (j0 + 64 > (pre ? p.P : clear_to)) mask<2>(s, lane, (pre ? p.P : seen) - j0);
                weigh<D, 2>(st, s, p.c);
                gather<D, 2>(st, s, f, buffer + TILE + vl);
            }
            __builtin_amdgcn_s_setprio(0);
        } else {
            for (int k = k0; k < k1; ++k) next(k);
        }
        st.sum = half_sum(st.sum);
        const bool direct = whole && b >= 0;
        if (r < rows && (direct || slot + 4 <= p.joint_blocks + (b < 0 ? p.packed_blocks : 0)))
            leave<D>(p, st, direct, (int64_t)ti, h * p.G + g, p.blocks + (slot + wave) * block_bytes<D>(), lane & 31, lane >> 5);
        lds_barrier();  // the next item's first block lands where others may still be reading this one's last
        stop = x;
    }
}

struct AttnShared {
    Sums sums;
    int part[4][11];
    float stats[256];
};

// of the lanes below and this one, on the vector ALU: four steps inside rows of 16 lanes, then the rows' last lanes; op(x, 0) is x
template <class Op>
__device__ __forceinline__ int wave_scan(int v, Op op) {
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true));   // from one lane below
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true));   // two
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true));   // four
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true));   // eight
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));  // lane 15 of a row to the next, in rows 1 and 3
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));  // lane 31 to rows 2 and 3
    return v;
}

template <int D>
__global__ __launch_bounds__(WG, D == 128 ? 2 : 3) void prefix_attention_kernel(const AttnArgs p) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    AttnShared& sh = *reinterpret_cast<AttnShared*>(lds + 8 * 32 * D * 2);  // behind the tiles, which start at 0
    Sums& sums = sh.sums;
    auto& part = sh.part;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int T = (int)p.T;
    constexpr int NV = 9;  // narrow, pieces of the three lengths, items, rows, wide, teams' pieces, wide tiles
    int mine[NV] = {0, 0, 0, 0, 0, 0, 0, 0, 0}, v[NV], total[NV];
    bool wrong = false, few = true, many = true;  // no more than SOLO_FEW, SOLO_MANY tokens
    int longest = 0;  // the wide tile that sees most
    const int b0 = min(p.B, tid * p.per), b1 = min(p.B, b0 + p.per);
    for (int b = b0; b < b1; ++b) {
        const Request r = request(p, b);
        wrong |= r.q0 < 0 || r.n < 0 || r.q0 > T - r.n;
        if (wrong) break;
        const Extent e = extent(p, r, CUT);
        few &= p.P + r.L <= SOLO_FEW, many &= p.P + r.L <= SOLO_MANY;
        const int n = narrow_units(p, r.L, TEAM) + p.pre_tiles;
        if (e.wide > 0) {
            const int nt = wide_tiles(p, r.n);
            mine[8] += p.Hkv * nt, longest = max(longest, wide_length(wide_step(p, CUT), wide_seen(p, r, CUT), nt - 1));
        }
        mine[0] += e.narrow, mine[4] += e.items, mine[5] += e.rows, mine[6] += e.wide, mine[7] += e.items * ((n + TEAM - 1) / TEAM);
        mine[1] += e.items * ((n + PIECE1 - 1) / PIECE1), mine[2] += e.items * ((n + PIECE2 - 1) / PIECE2), mine[3] += e.items * ((n + PIECE3 - 1) / PIECE3);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = mine[k];
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = wave_scan(v[k], [](int a, int b) { return a + b; });
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < NV; ++k) part[wave][k] = v[k];
    const int small = (__ballot(!few) == 0) + 2 * (__ballot(!many) == 0);
    longest = wave_scan(longest, [](int a, int b) { return max(a, b); });
    if (lane == 63) part[wave][NV] = small, part[wave][NV + 1] = longest;
    if (__syncthreads_or(wrong)) {  // offsets that fall or name rows that are not there: nothing is read or written
        if (blockIdx.x == 0 && tid == 0) p.plan->valid = 0;
        return;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        v[k] -= mine[k];
        total[k] = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u < wave) v[k] += part[u][k];
            total[k] += part[u][k];
        }
    }
    const Plan plan = make_plan<D>(p, uni(total[0]), uni(total[7]), uni(total[1]), uni(total[2]), uni(total[3]), uni(total[4]), uni(total[5]), uni(total[6]), uni(total[8]),
                                   uni(max(max(part[0][NV + 1], part[1][NV + 1]), max(part[2][NV + 1], part[3][NV + 1]))),
                                   uni(part[0][NV] & part[1][NV] & part[2][NV] & part[3][NV]));
    if (plan.piece == SOLO) v[0] = v[4];
    else if (plan.piece) v[0] = plan.piece * (plan.piece == TEAM ? v[7] : plan.piece == PIECE1 ? v[1] : plan.piece == PIECE2 ? v[2] : v[3]);
    if (plan.wide_piece == SOLO) v[6] = v[8];
    sums.narrow[tid] = v[0], sums.items[tid] = v[4], sums.rows[tid] = v[5], sums.wide[tid] = v[6];
    if (blockIdx.x == 0) {  // what the second kernel looks its segments up with
        if (tid == 0) *p.plan = plan;
        for (int b = b0; b < b1; ++b) {
            const Extent e = extent(p, request(p, b), plan.piece);
            int* r = p.records + (int64_t)b * 4;
            r[0] = v[0], r[1] = v[4], r[2] = v[5], r[3] = v[6];
            v[0] += e.narrow, v[4] += e.items, v[5] += e.rows, v[6] += plan.wide_piece == plan.piece ? e.wide : extent(p, request(p, b), plan.wide_piece).wide;
        }
    }
    __syncthreads();

    // Workgroups are dealt to the XCDs in turn: each XCD takes a run of wide pieces, whose items are neighbours and share keys and
    // values; narrow ones share nothing.
    // Those that a CU gets second take their narrow piece first: the two lists are bound by different things.
    constexpr int N = attn_wgs<D>();
    const int xcd = blockIdx.x & 7, i = blockIdx.x >> 3, run = plan.with_wide >> 3;
    const bool with_wide = i < run, swap = blockIdx.x >= N / 2;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
        if ((turn == 0) == swap) {
            narrow_piece<D>(p, plan, sums, lds, sh.stats);
            if (turn == 0 && with_wide) lds_barrier();  // the tiles of both are in the same place
        } else if (with_wide) wide_piece<D>(p, plan, sums, lds, xcd * run + i);
    }
}

// ---- the segments of a row, joined ------------------------------------------------------------------------------------------------
// A wavefront joins H = 1 or 4 rows (heads) of a token.  First 64 / H lanes a row find one segment each and read its base and
// weight; then D/4 lanes hold four channels each of a row's sums: all groups of lanes share one row's segments (H = 1: few
// rows, of many segments), or have rows of their own (H = 4: more rows than the card holds wavefronts).
template <int D, int H>
__global__ __launch_bounds__(256) void prefix_attention_join_kernel(const AttnArgs p) {
    constexpr int LANES = D / 4, GRP = 64 / LANES, S = 64 / H, ROWS = H == 1 ? 1 : H / GRP, STEP = H == 1 ? GRP : 1;
    const int lane = threadIdx.x & 63, sub = lane / LANES, l = lane % LANES, jl = lane % S;
    const int per_token = (p.Hq + H - 1) / H;
    const int64_t unit = (int64_t)blockIdx.x * 4 + uni((int)(threadIdx.x >> 6));
    const int t = (int)(unit / per_token);
    if (t >= p.T) return;
    const int head0 = (int)(unit - (int64_t)t * per_token) * H;
    // Reads that depend on one another are what this kernel's time is, so they are as few as can be: the last request that starts at or
    // before t is searched until 64 are left, whose lengths and records are read with their offsets, and beside the plan.
    const Plan plan = *p.plan;
    int lo = 0, hi = p.B + 1;
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const int n = __popcll(__ballot(at < hi && p.q_offsets[min(at, p.B)] <= t));
        if (n == 0) return;
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    const int at_b = min(lo + lane, p.B - 1), start = p.q_offsets[min(lo + lane, p.B)], after = p.q_offsets[at_b + 1], len = p.kv_lens[at_b];
    const int4 all = *reinterpret_cast<const int4*>(p.records + (int64_t)at_b * 4);
    if (!plan.valid || !plan.joins) return;
    const int found = uni(__popcll(__ballot(lo + lane < hi && start <= t))) - 1;
    if (found < 0 || lo + found >= p.B) return;
    const Request rq{__builtin_amdgcn_readlane(start, found), __builtin_amdgcn_readlane(after, found) - __builtin_amdgcn_readlane(start, found),
                     min(max(__builtin_amdgcn_readlane(len, found), 0), p.max_kv)};
    const int rec[4] = {__builtin_amdgcn_readlane(all.x, found), __builtin_amdgcn_readlane(all.y, found), __builtin_amdgcn_readlane(all.z, found),
                        __builtin_amdgcn_readlane(all.w, found)};
    const int i = t - rq.q0;
    if (i < 0 || i >= rq.n) return;
    const bool joint = is_long(p, rq.n);
    const int cp = rounded(narrow_units(p, p.P, plan.piece), plan.piece), packed_item = packed_length(p, plan.super);
    const int pre_pieces = packed_item == plan.wide_per ? 1 : plan.tiles ? (packed_item - 1) / plan.wide_per + 2 : 0;  // of a piece of the prefix, at most

    // this lane's row: `own` segments of its request's tile, the first at `first`; then up to `more` of the prefix
    const int head = min(head0 + lane / S, p.Hq - 1), h = head / p.G, r = i * p.G + head - h * p.G;
    const int packed = rec[2] + r;
    int own, more = 0, row, first;
    if (joint) {
        const int step = wide_step(p, plan.wide_piece), seen = wide_seen(p, rq, plan.wide_piece), tile = i / p.tpt;
        const int s0 = plan.wide0 + rec[3] + h * wide_sum(step, seen, wide_tiles(p, rq.n)) + wide_sum(step, seen, tile);
        first = s0 / plan.wide_per;
        own = (s0 + wide_length(step, seen, tile) - 1) / plan.wide_per - first + 1;
        row = r - tile * p.tpt * p.G;
    } else {
        const int length = narrow_length(p, rq.L, plan.piece);
        const int k = h * narrow_tiles(p, rq.n) + r / 32, s0 = plan.narrow0 + rec[0] + k * length;
        first = narrow_piece_of(plan, s0);
        own = narrow_piece_of(plan, s0 + length - 1) - first + 1;
        row = r & 31;
        first += plan.items0 + rec[1] + k;  // its block in the narrow part
        if (p.P && !p.pre_tiles) more = plan.tiles ? plan.supers * pre_pieces : narrow_piece_of(plan, (h + 1) * cp - 1) - narrow_piece_of(plan, h * cp) + 1;
    }
    const bool done = own == 1 && more == 0 && (joint || p.P == 0 || p.pre_tiles);  // written by the first kernel
    const int count = done ? 0 : own + more;
    int most = count;
#pragma unroll
    for (int d = S; d < 64; d <<= 1) most = max(most, __shfl_xor(most, d));
    most = uni(most);
    // segment j's place, or -1 where there is none
    auto place = [&](int j, int& at_row) -> int64_t {
        at_row = row & 31;
        if (j >= count) return -1;
        if (j < own) {
            if (joint) return (2 * (int64_t)(first + j) + (j == 0)) * 4 + (row >> 5);
            return first + j < p.narrow_blocks ? p.joint_blocks + p.packed_blocks + first + j : -1;
        }
        j -= own;
        at_row = packed & 31;
        if (!plan.tiles) {
            const int blk = h + narrow_piece_of(plan, h * cp) + j;
            return blk < p.narrow_blocks ? p.joint_blocks + p.packed_blocks + blk : -1;
        }
        const int s = j / pre_pieces, item = s * plan.tiles + packed / WROWS, a = h * plan.head + item * packed_item;
        const int w = a / plan.wide_per + j - s * pre_pieces;
        if (w > (a + packed_item - 1) / plan.wide_per) return -1;
        const int64_t blk = ((int64_t)h * plan.supers * plan.tiles + item + w) * 4;
        return blk + 4 <= p.packed_blocks ? p.joint_blocks + blk + ((packed % WROWS) >> 5) : -1;
    };
    float base = -INFINITY, sum = 0.0f;
    float4 acc[ROWS];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) acc[q] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int j0 = 0; j0 < most; j0 += S) {
        int at_row = 0;
        const int64_t blk = place(j0 + jl, at_row), at = blk < 0 ? 0 : blk * block_bytes<D>();
        const float2 z = *reinterpret_cast<const float2*>(p.blocks + at + (32 * D + at_row * 2) * 4);
        const int64_t off = at + at_row * D * 4;
        const int m = min(S, most - j0);
        // four loads of a lane for a row of sums, segments j ..; the first ones are asked for before the weights are there
        auto first_lane = [&](int q) { return H == 1 ? 0 : (sub * ROWS + q) * S; };
        auto load = [&](int q, int j, float4 (&y)[4]) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                y[k] = *reinterpret_cast<const float4*>(p.blocks + __shfl(off, first_lane(q) + min(j + k * STEP + (H == 1 ? sub : 0), S - 1)) + l * 16);
        };
        float4 y[ROWS][4];
#pragma unroll
        for (int q = 0; q < ROWS; ++q) load(q, 0, y[q]);
        const float bs = blk < 0 ? -INFINITY : z.x, wt = blk < 0 ? 0.0f : z.y;
        float top = bs;
#pragma unroll
        for (int d = 1; d < S; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        const float next = fmaxf(base, top), fade = next == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(base - next);
        const float f = wt == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(bs - next);
        base = next;
        sum = fmaf(f, wt, sum * fade);
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            const float fd = __shfl(fade, first_lane(q));
            acc[q].x *= fd, acc[q].y *= fd, acc[q].z *= fd, acc[q].w *= fd;
            for (int j = 0; j < m; j += 4 * STEP) {
                if (j) load(q, j, y[q]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {  // a segment without weight may not have left sums
                    const int at_j = j + k * STEP + (H == 1 ? sub : 0);
                    const float g = __shfl(f, first_lane(q) + min(at_j, S - 1)), fy = at_j < m ? g : 0.0f;
                    const float4 v = y[q][k];
                    const bool has = fy > 0.0f;
                    acc[q].x = has ? fmaf(fy, v.x, acc[q].x) : acc[q].x, acc[q].y = has ? fmaf(fy, v.y, acc[q].y) : acc[q].y;
                    acc[q].z = has ? fmaf(fy, v.z, acc[q].z) : acc[q].z, acc[q].w = has ? fmaf(fy, v.w, acc[q].w) : acc[q].w;
                }
            }
        }
    }
#pragma unroll
    for (int d = 1; d < S; d <<= 1) sum += __shfl_xor(sum, d);
    if (H == 1) {
#pragma unroll
        for (int d = LANES; d < 64; d <<= 1)
            acc[0].x += __shfl_xor(acc[0].x, d), acc[0].y += __shfl_xor(acc[0].y, d), acc[0].z += __shfl_xor(acc[0].z, d), acc[0].w += __shfl_xor(acc[0].w, d);
    }
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        const int u = H == 1 ? 0 : sub * ROWS + q;
        const float total = __shfl(sum, u * S);
        const bool write = __shfl((int)done, u * S) == 0 && head0 + u < p.Hq && (H != 1 || sub == 0);
        const float inv = inverse(total);
        if (write)
            *reinterpret_cast<uint2*>(p.O + (int64_t)t * p.ldo + (head0 + u) * D + l * 4) =
                make_uint2(pack2(acc[q].x * inv, acc[q].y * inv), pack2(acc[q].z * inv, acc[q].w * inv));
    }
    if (p.lse && jl == 0 && !done && head0 + lane / S < p.Hq) p.lse[(int64_t)t * p.Hq + head] = lse_of(base, sum);
}

// ---- host ---------------------------------------------------------------------------------------------------------------------------
// Tiles of the prefix that short requests' items start with: all of them, or none where that would be too many.
static int inline_tiles(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int64_t P) {
    const int64_t items = Hkv * (T * (Hq / Hkv) / 32 + std::min<int64_t>(B, T)), waves = 4 * (D == 128 ? attn_wgs<128>() : attn_wgs<64>());
    return P && items * ((P + 31) / 32) <= INLINE_TILES * waves ? (int)((P + 31) / 32) : 0;
}
struct AttnSpace {
    int64_t joint, packed, narrow;  // blocks
    size_t records, blocks, total;  // offsets
};
static AttnSpace attn_space(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int64_t P) {
    const int64_t G = Hq / Hkv, rows = T * G, wgs = D == 128 ? attn_wgs<128>() : attn_wgs<64>(), some = std::min<int64_t>(B, T);
    const int64_t is_short = P && !inline_tiles(T, B, Hq, Hkv, D, P) ? std::min<int64_t>(rows, (LONG_PREFIX - 1) * (int64_t)B) : 0;  // rows that walk the prefix packed, at most
    AttnSpace a;
    a.joint = rows >= (P ? LONG_PREFIX : LONG) ? 2 * wgs * 4 : 0;
    const int64_t tiles = (is_short + WROWS - 1) / WROWS;
    a.packed = is_short > 32 ? (std::max(Hkv * tiles * super_count(P, tiles), wgs) + wgs) * 4 : 0;
    a.narrow = Hkv * (1 + (P ? std::min<int64_t>(rows, (LONG_PREFIX - 1) * (int64_t)B) / 32 + some : some)) + 4 * wgs;
    a.records = 256;
    a.blocks = align_up(a.records + (size_t)B * 16, 256);
    a.total = a.blocks + (size_t)(a.joint + a.packed + a.narrow) * (32 * (D + 2) * 4);
    return a;
}

size_t prefix_attention_workspace(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int64_t prefix_len) {
    return attn_space(T, B, Hq, Hkv, D, prefix_len).total;
}

template <int D>
static int launch(const AttnArgs& p, hipStream_t st) {
    static LdsReserved r;
    constexpr size_t lds = 8 * 32 * D * 2 + sizeof(AttnShared);
    const int rc = reserve_lds((const void*)prefix_attention_kernel<D>, lds, r);
    if (rc) return rc;
    prefix_attention_kernel<D><<<dim3(attn_wgs<D>()), WG, lds, st>>>(p);
    // a wavefront a row while the card holds them at once, four rows beyond that
    const bool few = p.T * p.Hq <= 4096;
    const int64_t wgs = (p.T * (few ? p.Hq : (p.Hq + 3) / 4) + 3) / 4;
    if (few) prefix_attention_join_kernel<D, 1><<<dim3((unsigned)wgs), 256, 0, st>>>(p);
    else prefix_attention_join_kernel<D, 4><<<dim3((unsigned)wgs), 256, 0, st>>>(p);
    return check_launch("osc_prefix_attention");
}

int launch_prefix_attention(const AttnCall& a, hipStream_t st) {
    AttnArgs p;
    p.Q = static_cast<const uint16_t*>(a.Q), p.T = a.T, p.ldq = a.ldq, p.Hq = a.Hq, p.Hkv = a.Hkv, p.G = a.Hq / a.Hkv;
    p.tpt = WROWS / p.G;
    p.K = static_cast<const uint8_t*>(a.K), p.V = static_cast<const uint8_t*>(a.V), p.n_pages = (uint32_t)a.n_pages, p.lg = a.lg;
    p.prefix_pages = a.prefix_pages, p.P = (int)a.prefix_len, p.table = a.table, p.ldt = a.ldt;
    p.max_kv = (int)std::min<int64_t>(a.ldt << a.lg, ATTN_MAX_TOKENS);
    p.kv_lens = a.kv_lens, p.q_offsets = a.q_offsets, p.B = a.B, p.per = (a.B + GROUPS - 1) / GROUPS, p.c = a.scale * 1.44269504088896341f;
    p.O = static_cast<uint16_t*>(a.O), p.ldo = a.ldo, p.lse = a.lse;
    p.pre_tiles = inline_tiles(a.T, a.B, a.Hq, a.Hkv, a.D, a.prefix_len);
    const AttnSpace s = attn_space(a.T, a.B, a.Hq, a.Hkv, a.D, a.prefix_len);
    p.plan = reinterpret_cast<Plan*>(a.workspace), p.records = reinterpret_cast<int*>(a.workspace + s.records);
    p.blocks = a.workspace + s.blocks;
    p.joint_blocks = s.joint, p.packed_blocks = s.packed, p.narrow_blocks = s.narrow;
    // the longest that the lines can be
    const int64_t rows = a.T * p.G, is_long = rows / (p.P ? LONG_PREFIX : LONG), tiles = rows / WROWS + 1, some = std::min<int64_t>(a.B, a.T);
    const int64_t wide = (int64_t)p.Hkv * (a.T / p.tpt + is_long) * (WIDE_EDGE + p.P + (int64_t)p.max_kv + a.T + WROWS) +
                         (int64_t)p.Hkv * tiles * 2 * (p.P + (WIDE_EDGE + 64) * MAX_SUPER);
    const int64_t narrow = (int64_t)p.Hkv * (rows / 32 + some + 1) * (std::max<int64_t>(p.P, p.max_kv) / 32 + p.pre_tiles + CUT_EDGE + PIECE3 + 1);
    for (p.ws = 0; wide >> p.ws > 1 << 30;) ++p.ws;
    for (p.ns = 0; narrow >> p.ns > 1 << 30;) ++p.ns;
    return a.D == 64 ? launch<64>(p, st) : launch<128>(p, st);
}

}  // namespace osc
