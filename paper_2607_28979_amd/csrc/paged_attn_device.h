// What the kernels of the paged attention share: the positions that a tile of query
// rows sees, the pages they lie in, buffers over them, V^T operands from LDS.
//
// The G = H_q / H_kv query heads of a KV head and the new tokens of a sequence
// are the rows of one product: row r = token r / G, head r % G.  A workgroup
// takes a tile of rows of one (sequence, KV head) and a range of positions and
// keeps, per row, the running maximum and sum of the softmax and the
// accumulators of O^T[d][row]:
//     S^T[position][row] = K . Q^T,   P = 2^(S scale log2(e) - max),
//     O^T += V^T . P^T
// Positions go through LDS in groups of 16 of one page (pages hold 16 or more,
// a power of two), loaded straight from the pages (buffer loads into LDS).
// Rows of a group past the sequence's end, and groups in holes, read as zeros.
//
// A value that is not finite multiplies the probability 0 of rows that do not
// see it: a tile whose result is not finite is computed again token by token,
// the positions the token does not see read as zeros.
#pragma once

#include <type_traits>

#include "attn_device.h"
#include "cache_internal.h"

namespace mot {

// The rows of a tile and the positions that they see.
struct Tile {
    int n_rows;        // rows of the sequence and KV head
    int r0;            // first row
    int t0, t1;        // first and last token
    int u0;            // position of the sequence's first new token (may be negative)
    int lo, hi;        // positions [lo, hi) seen by some row; none: [0, 0)
};
__device__ __forceinline__ Tile tile_of(const AttendProblem& p, const NewTokens& nt, int tile, int rows) {
    Tile t;
    const int G = p.H_q / p.c.H_kv;
    t.n_rows = nt.n * G;
    t.r0 = tile * rows;
    t.t0 = t.r0 / G;
    t.t1 = max(min(t.r0 + rows, t.n_rows) - 1, 0) / G;
    t.u0 = nt.kv - nt.count;
    t.hi = max(t.u0 + t.t1 + 1, 0);
    t.lo = p.window > 0 ? max(t.u0 + t.t0 - p.window + 1, 0) : 0;
    if (t.hi <= t.lo) t.lo = t.hi = 0;
    return t;
}

// First position that the token at position u sees.
__device__ __forceinline__ int low_of(const AttendProblem& p, int u) { return p.window > 0 ? max(u - p.window + 1, 0) : 0; }

// The pages of up to 64 groups of 16 positions, one per lane, from group `base` on:
// a bit per group that lies in no hole, and the page numbers.
struct Groups {
    int base, page;
    unsigned long long ok;
    __device__ __forceinline__ void fetch(const AttendProblem& p, int b, int g) {
        const int at = ((g + (threadIdx.x & 63)) << 4) >> p.c.page_shift;
        base = g;
        page = at < p.c.max_pages ? p.c.table[(int64_t)b * p.c.max_pages + at] : -1;
    }
    __device__ __forceinline__ void ready(const AttendProblem& p) {
        ok = __builtin_amdgcn_ballot_w64(page >= 0 && page < p.c.n_pages);
    }
    __device__ __forceinline__ void load(const AttendProblem& p, int b, int g) {
        fetch(p, b, g);
        ready(p);
    }
    __device__ __forceinline__ int page_of(int g) const { return __builtin_amdgcn_readlane(page, g - base); }
};

// Group g's rows of KV head h that lie before position `end`: offset into the pools
// and bytes.
struct GroupRows {
    int64_t at;
    uint32_t bytes;
};
template <typename T, int D>
__device__ __forceinline__ GroupRows group_rows(const AttendProblem& p, const Groups& gr, int g, int h, int end) {
    const int rows = min(16, end - (g << 4));
    GroupRows r;
    r.at = gr.page_of(g) * p.c.page_elems + (uint32_t)(((g << 4) & ((1 << p.c.page_shift) - 1)) * p.c.ts + h * p.c.hs);
    r.bytes = rows > 0 && ((gr.ok >> (g - gr.base)) & 1ull) ? (uint32_t)((rows - 1) * p.c.ts + D) * (uint32_t)sizeof(T) : 0u;
    return r;
}
template <typename T>
__device__ __forceinline__ rsrc_t group_rsrc(const void* pool, const GroupRows& r) {
    return make_rsrc(reinterpret_cast<const T*>(pool) + r.at, r.bytes);
}

// LDS swizzle of a V row of D bf16 (chunk c at c ^ v_swizzle(row)): the 4 rows x 64 bytes
// that 32 lanes of a transposing read take, and the 8 x 32 that two groups of 16 lanes
// of either half take, lie in different banks.
template <int D>
__device__ __forceinline__ int v_swizzle(int r) {
    return D == 128 ? (4 * (r & 3)) ^ (2 * ((r >> 2) & 1)) : (4 * ((r >> 1) & 1)) ^ (2 * ((r >> 2) & 1));
}

// V^T operands of one step of 16 positions: 32 elements d from 32 db on in v[2 db],
// v[2 db + 1].  at[db]: LDS address of this lane's 8 bytes of the step's first
// eight positions.  In assembly, since before the builtin the compiler waits for every load
// into LDS that is under way; the block ends with its own wait.
template <int D, int OFF>
__device__ __forceinline__ void read_vt(const uint32_t (&at)[D / 32], u32x2 (&v)[D / 16]) {
    constexpr int NEXT = 8 * D * 2;   // bytes of eight rows
    if constexpr (D == 128)
        asm volatile(
            "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
            "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
            "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
            "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
            : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(OFF), "n"(OFF + NEXT)
            : "memory");
    else
        asm volatile(
            "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
            "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
            : "v"(at[0]), "v"(at[1]), "n"(OFF), "n"(OFF + NEXT)
            : "memory");
}
// The same for the two steps from OFF on: v[0 .. D / 16) and v[D / 16 .. D / 8).
template <int D, int OFF>
__device__ __forceinline__ void read_vt2(const uint32_t (&at)[D / 32], u32x2 (&v)[D / 8]) {
    constexpr int NEXT = 8 * D * 2;
    if constexpr (D == 128)
        asm volatile(
            "ds_read_b64_tr_b16 %0, %16 offset:%20\n\tds_read_b64_tr_b16 %1, %16 offset:%21\n\t"
            "ds_read_b64_tr_b16 %2, %17 offset:%20\n\tds_read_b64_tr_b16 %3, %17 offset:%21\n\t"
            "ds_read_b64_tr_b16 %4, %18 offset:%20\n\tds_read_b64_tr_b16 %5, %18 offset:%21\n\t"
            "ds_read_b64_tr_b16 %6, %19 offset:%20\n\tds_read_b64_tr_b16 %7, %19 offset:%21\n\t"
            "ds_read_b64_tr_b16 %8, %16 offset:%22\n\tds_read_b64_tr_b16 %9, %16 offset:%23\n\t"
            "ds_read_b64_tr_b16 %10, %17 offset:%22\n\tds_read_b64_tr_b16 %11, %17 offset:%23\n\t"
            "ds_read_b64_tr_b16 %12, %18 offset:%22\n\tds_read_b64_tr_b16 %13, %18 offset:%23\n\t"
            "ds_read_b64_tr_b16 %14, %19 offset:%22\n\tds_read_b64_tr_b16 %15, %19 offset:%23\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7]),
              "=&v"(v[8]), "=&v"(v[9]), "=&v"(v[10]), "=&v"(v[11]), "=&v"(v[12]), "=&v"(v[13]), "=&v"(v[14]), "=&v"(v[15])
            : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(OFF), "n"(OFF + NEXT), "n"(OFF + 2 * NEXT), "n"(OFF + 3 * NEXT)
            : "memory");
    else
        asm volatile(
            "ds_read_b64_tr_b16 %0, %8 offset:%10\n\tds_read_b64_tr_b16 %1, %8 offset:%11\n\t"
            "ds_read_b64_tr_b16 %2, %9 offset:%10\n\tds_read_b64_tr_b16 %3, %9 offset:%11\n\t"
            "ds_read_b64_tr_b16 %4, %8 offset:%12\n\tds_read_b64_tr_b16 %5, %8 offset:%13\n\t"
            "ds_read_b64_tr_b16 %6, %9 offset:%12\n\tds_read_b64_tr_b16 %7, %9 offset:%13\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
            : "v"(at[0]), "v"(at[1]), "n"(OFF), "n"(OFF + NEXT), "n"(OFF + 2 * NEXT), "n"(OFF + 3 * NEXT)
            : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_void*)p; }

template <int S>
using Step = std::integral_constant<int, S>;

constexpr uint32_t kPastEnd = 0x80000000u;   // byte offset that every group's buffer reads as zero

// The exponents' base of a row moves only when a row's largest exponent passes it by
// more than this (base 2): probabilities up to 2^8 are as exact, relative to their sum, as
// those up to 1, and the accumulators are rarely rescaled.
constexpr float kSlack = 8.f;

// l + both bf16 of w: a row's sum takes the probabilities as they go into the product with V,
// rounded, two in one instruction.
__device__ __forceinline__ float add_bf16x2(uint32_t w, float l) {
    typedef __bf16 two __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(two, w), __builtin_bit_cast(two, 0x3f803f80u), l, false);
}

// Two probabilities as two bf16 terms each, x: cut to 8 bits from just below, y: the rounded
// rest, off by 2^-15 of them at most.  Neither term of a probability above 0 is 0 or
// negative, so that an infinite value times it stays what it is.
__device__ __forceinline__ u32x2 split_bf16x2(float a, float b) {
    const uint32_t x = __builtin_elementwise_sub_sat(__float_as_uint(a), 1u) & 0xffff0000u;
    const uint32_t y = __builtin_elementwise_sub_sat(__float_as_uint(b), 1u) & 0xffff0000u;
    return {x >> 16 | y, pack_bf16x2(a - __uint_as_float(x), b - __uint_as_float(y))};
}

// Running softmax of a row: `mo` is the largest exponent so far (base 2), -inf
// before the first visible position; `base` replaces it where it is -inf.
__device__ __forceinline__ float base_of(float mo) { return mo == -INFINITY ? 0.f : mo; }

// The base of a row that sees positions, all with the score -inf (infinite keys): any other's is above
// it, so it adds nothing to what other waves or parts of the row have seen.
constexpr float kLowest = -3.4028234663852886e38f;
// The base of this lane's row (token at position u of sequence b) once a wave's positions are done: blocks
// of 32 of [lo, hi), the w-th and every nw-th after it (nw = 1: all).  By a whole wave; the pages are
// looked at again only where no score of a row that lies behind one of them was above -inf.
__device__ __forceinline__ float settled(const AttendProblem& p, int b, float mo, int u, int lo, int hi, int w, int nw) {
    if (!__builtin_amdgcn_ballot_w64(mo == -INFINITY)) return mo;   // uniform
    const int a = max(low_of(p, u), lo), e = min(u + 1, hi);        // seen, as far as no hole covers it
    // the wave's first block that holds a or lies behind it
    const int j = a >> 5, first = 32 * (j + ((w - j + (lo >> 5)) & (nw - 1)));
    const bool none = mo == -INFINITY && a < e && first < e;
    if (!__builtin_amdgcn_ballot_w64(none)) return mo;
    bool seen = false;
    for (int g = lo >> 4; (g << 4) < hi; g += 64) {
        Groups gr;
        gr.load(p, b, g);
        const int from = max((a >> 4) - g, 0), to = min(((e + 15) >> 4) - g, 64);
        if (from < to) seen |= (gr.ok >> from & ~0ull >> (64 - (to - from))) != 0;
    }
    return none && seen ? kLowest : mo;
}

// What a row's accumulators are divided by: nothing seen gives zeros, a softmax of -inf alone
// is no number.
__device__ __forceinline__ float inverse_of(float mo, float l) { return l != 0.f ? 1.0f / l : mo == -INFINITY ? 0.f : NAN; }

// ---- sharing the work --------------------------------------------------------
//
// Lengths differ within a batch, and only the device knows them.  With few tiles and
// long contexts the positions of a (sequence, KV head) are cut into parts, each of them
// for all its tiles.  Every workgroup adds up the blocks (of `step` positions) of all
// sequences by itself, each of its waves in registers, and finds its own (sequence, KV
// head, part, tile): n blocks are cut into ceil(n / share) equal parts, where share is
// the even share of all tiles' blocks of p.n_split workgroups.  The parts of a cut one
// leave partial sums, which k_paged_join adds in their order.

constexpr int kSeqPerLane = 8, kMostSeq = 64 * kSeqPerLane;   // sequences of a call whose work is shared

__host__ __device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }

// First block of positions that the rows of a sequence see, and how many (1 where there are
// rows but no positions).
__device__ __forceinline__ int blocks_of(const AttendProblem& p, const NewTokens& nt, int step, int* from) {
    const int u0 = nt.kv - nt.count, hi = max(u0 + nt.n, 0), lo = min(low_of(p, u0), hi) & -step;
    *from = lo;
    return nt.n > 0 ? max(div_up(hi - lo, step), 1) : 0;
}

__device__ __forceinline__ int wave_scan(int x) {   // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d, 64);
        if (lane >= d) x += y;
    }
    return x;
}

// What a workgroup does: a tile of a (sequence, KV head), over part `part` of `parts` of its
// positions: [lo, hi).  cut: number of its first partial tile among those of the call.
struct Work {
    int b, kvh, tile, tiles, part, parts, cut;
    int lo, hi;
    NewTokens nt;
};
__device__ __forceinline__ void span_of(const AttendProblem& p, Work& w, int step) {
    int from;
    const int n = blocks_of(p, w.nt, step, &from);
    w.lo = from + step * (int)((int64_t)n * w.part / w.parts);
    w.hi = from + step * (int)((int64_t)n * (w.part + 1) / w.parts);
}

// Tile i in an order that alternates the last (which see most) with the first ones, so
// that any run of them is about the same work.
__device__ __forceinline__ int mixed_tile(int i, int n) { return i & 1 ? i >> 1 : n - 1 - (i >> 1); }

// The share of a call, and the workgroups (`cuts`: those of cut sequences) of this lane's
// sequences.  I: 32 bits, or 64 where sums of a call's sizes may pass that (p.wide; 64 bits
// throughout cost a decoding step 0.3 us).  False: more workgroups than a launch holds, which
// only starts that do not ascend ask for (their rows are unspecified).
template <typename I, int N>
__device__ __forceinline__ bool shares_of(const AttendProblem& p, const int (&blocks)[N], const int (&tiles)[N], int& share, int& mine,
                                          int& cuts) {
    share = p.least;
    if (p.part) {
        I sum = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) sum += (I)blocks[i] * tiles[i];
        if constexpr (sizeof(I) == 4) {
            share = max(div_up(__builtin_amdgcn_readlane(wave_scan(sum), 63) * p.c.H_kv, p.n_split), share);
        } else {
            // multiples of 2^20 and the rest; from 2^44 blocks on the share is longer than any sequence
            const int high = (int)min(sum >> 20, (I)1 << 24), low = (int)(sum & ((1 << 20) - 1));
            const I total = ((I)__builtin_amdgcn_readlane(wave_scan(high), 63) << 20) + __builtin_amdgcn_readlane(wave_scan(low), 63);
            share = max((int)min((total * p.c.H_kv + p.n_split - 1) / p.n_split, (I)1 << 30), share);
        }
    }
    I all = 0, cut = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int parts = div_up(blocks[i], share);
        const I n = (I)parts * tiles[i] * p.c.H_kv;
        all += n;
        cut += parts > 1 ? n : 0;
    }
    mine = (int)all;
    cuts = (int)cut;
    return sizeof(I) == 4 || !__builtin_amdgcn_ballot_w64(all > 1 << 24);
}

// N sequences per lane (lane i: N i .. N i + N - 1).  False: none for this workgroup.  Where
// sequences have several tiles the workgroups of an XCD (every eighth) take neighbouring
// ones, so that the tiles of one (sequence, KV head, part) meet its K and V in one L2.
template <int N>
__device__ __forceinline__ bool shared_work(const AttendProblem& p, int rows, int step, bool by_xcd, Work& w) {
    const int lane = threadIdx.x & 63, H = p.c.H_kv, G = p.H_q / H;
    NewTokens nt[N];
    int blocks[N], tiles[N], share, mine, cuts;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int s = lane * N + i;
        int from;
        nt[i] = new_tokens(p.c, min(s, p.c.B - 1));
        blocks[i] = s < p.c.B ? blocks_of(p, nt[i], step, &from) : 0;
        tiles[i] = div_up(nt[i].n * G, rows);
    }
    if (!(__builtin_expect(p.wide, 0) ? shares_of<int64_t>(p, blocks, tiles, share, mine, cuts) : shares_of<int>(p, blocks, tiles, share, mine, cuts)))
        return false;
    const int upto = wave_scan(mine), cutto = wave_scan(cuts);
    int id = blockIdx.x;
    if (by_xcd) {
        const int per = div_up(__builtin_amdgcn_readlane(upto, 63), 8);
        if ((id >> 3) >= per) return false;
        id = (id & 7) * per + (id >> 3);
    }
    const unsigned long long after = __builtin_amdgcn_ballot_w64(upto > id);
    if (!after) return false;
    const int who = __builtin_ctzll(after);   // the lane whose sequences hold it
    int at = __builtin_amdgcn_readlane(upto - mine, who), cut = __builtin_amdgcn_readlane(cutto - cuts, who);
    bool found = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int parts = div_up(__builtin_amdgcn_readlane(blocks[i], who), share);
        const int t = __builtin_amdgcn_readlane(tiles[i], who), n = parts * t * H;
        if (!found && id < at + n) {
            found = true;
            const int x = id - at;
            w.b = who * N + i;
            w.parts = parts;
            w.tiles = t;
            w.kvh = x / (parts * t);
            w.part = (x - w.kvh * parts * t) / t;
            w.tile = mixed_tile(x % t, t);
            w.cut = cut + w.kvh * parts * t;
            w.nt.row = __builtin_amdgcn_readlane(nt[i].row, who);
            w.nt.count = __builtin_amdgcn_readlane(nt[i].count, who);
            w.nt.n = __builtin_amdgcn_readlane(nt[i].n, who);
            w.nt.kv = __builtin_amdgcn_readlane(nt[i].kv, who);
        }
        at += n;
        cut += parts > 1 ? n : 0;
    }
    span_of(p, w, step);
    return true;
}

// Nothing shared: a workgroup per (sequence, KV head, tile), neighbouring ones on one XCD;
// `tiles` of a sequence at most.  grid xcd_grid(B * H_kv * tiles)
__device__ __forceinline__ bool own_work(const AttendProblem& p, int rows, int step, int tiles, Work& w) {
    const int n = p.c.B * p.c.H_kv * tiles, id = tiles > 1 ? xcd_item(blockIdx.x, n) : blockIdx.x, group = id / tiles;
    if (id >= n) return false;
    w.b = group / p.c.H_kv;
    w.kvh = group - w.b * p.c.H_kv;
    w.nt = new_tokens(p.c, w.b);
    w.tiles = div_up(w.nt.n * (p.H_q / p.c.H_kv), rows);
    w.tile = mixed_tile(id - group * tiles, tiles);
    w.part = w.cut = 0;
    w.parts = 1;
    if (w.tile >= w.tiles) return false;
    span_of(p, w, step);
    return true;
}

// Partial tiles, and where those of each (sequence, KV head) are.  The parts of a cut one
// have half a share of blocks at least, so there are under 2 n_split of them.
struct Partial {
    float* rows;     // [2 n_split][R][D]
    float2* ml;      // [2 n_split][R] (base, sum)
    int2* span;      // [B * H_kv] first partial tile, parts
    int R;
};
__host__ __device__ inline Partial partial_of(const AttendProblem& p, int rows) {
    Partial o;
    const int64_t most = (int64_t)p.c.max_new * (p.H_q / p.c.H_kv);
    o.R = most < rows ? (int)most : rows;
    const int64_t n = (int64_t)2 * p.n_split * o.R;
    o.rows = p.part;
    o.ml = reinterpret_cast<float2*>(p.part + n * p.c.D);
    o.span = reinterpret_cast<int2*>(o.ml + n);
    return o;
}
// First partial row of this workgroup's tile.
__device__ __forceinline__ int64_t partial_row(const Partial& o, const Work& w) {
    return (int64_t)(w.cut + w.part * w.tiles + w.tile) * o.R;
}
__device__ __forceinline__ void leave_span(const AttendProblem& p, const Partial& o, const Work& w) {
    if (p.part && threadIdx.x == 0 && w.part == 0 && w.tile == 0) o.span[w.b * p.c.H_kv + w.kvh] = make_int2(w.cut, w.parts);
}

// Workgroups of a shared call at most: the even shares, and one more per tile for the last
// part's remainder.
inline int64_t most_workgroups(const AttendProblem& p, int rows) {
    const int64_t G = p.H_q / p.c.H_kv, each = ((int64_t)p.c.max_new * G + rows - 1) / rows;
    const int64_t packed = (int64_t)p.c.n_new * G / rows + p.c.B, tiles = each * p.c.B < packed ? each * p.c.B : packed;
    return p.n_split + tiles * p.c.H_kv;
}

// The problem for kernels that find their work by shared_work(): without a workspace every
// (sequence, KV head) is one part.
inline AttendProblem shared_out(AttendProblem p) {
    if (!p.part) {
        p.n_split = 1;
        p.least = 1 << 30;
    }
    return p;
}

// Tiles that own_work() has for a sequence.
inline int64_t own_tiles(const AttendProblem& p, int rows) {
    return ((int64_t)p.c.max_new * (p.H_q / p.c.H_kv) + rows - 1) / rows * p.c.H_kv;
}

// Whether the workgroups of a call of tiles of `rows` rows find their work (shared_work()):
// where it is cut; where decoding has several tiles to a sequence; and where packed tokens of
// which one sequence might have most, but has not, would make most of own_work()'s grid leave
// at once.  47 single tokens and 512 of one sequence, contexts of 1000, 28 heads on 4 of 128:
// 96 and 35 us; 200 and 1500 on 1500: 316 and 172; fp32, 47 and 100 on 1000: 81 and 33.
inline bool finds_work(const AttendProblem& p, int rows) {
    const int64_t tiles = own_tiles(p, rows);
    if (p.part || rows == 32) return p.part || tiles > p.c.H_kv;
    AttendProblem s = shared_out(p);
    s.c.B = p.c.B < kMostSeq ? p.c.B : kMostSeq;
    return s.c.B * tiles > 4 * most_workgroups(s, rows);
}

}  // namespace mot
