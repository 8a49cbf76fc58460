// Attention of new tokens over the paged cache (one layer).
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
// * k_paged_decode: tiles of 32 rows (few new tokens); the four waves take
//   positions in turn, each with its own tiles, and are joined at the end.
// * k_paged_chunk: tiles of 128 rows, 32 per wave, over shared chunks of 64
//   positions.
// * k_paged_f32: fp32, tiles of 64 rows, 16 per wave, chunks of 32 positions,
//   on v_mfma_f32_16x16x4_f32.
// * k_paged_join: joins the ranges of a tile whose positions were cut.
//
// A value that is not finite multiplies the probability 0 of rows that do not
// see it: a tile whose result is not finite is computed again token by token,
// the positions the token does not see read as zeros.
#include <type_traits>

#include "attn_device.h"
#include "cache_internal.h"

namespace mot {

namespace {

// The rows of a tile and the positions that they see.
struct Tile {
    int n_rows;        // rows of the sequence and KV head
    int r0;            // first row
    int t0, t1;        // first and last token
    int u0;            // position of the sequence's first new token (may be negative)
    int lo, hi;        // positions [lo, hi) seen by some row; none: [0, 0)
    int s0, s1;        // first and last range that they lie in
};
__device__ __forceinline__ Tile tile_of(const AttendProblem& p, const NewTokens& nt, int tile, int rows) {
    Tile t;
    const int G = p.H_q / p.c.H_kv;
    t.n_rows = nt.n * G;
    t.r0 = tile * rows;
    t.t0 = t.r0 / G;
    t.t1 = min(t.r0 + rows, t.n_rows) - 1;
    t.t1 = t.t1 < 0 ? 0 : t.t1 / G;
    t.u0 = nt.kv - nt.count;
    t.hi = max(t.u0 + t.t1 + 1, 0);
    t.lo = p.window > 0 ? max(t.u0 + t.t0 - p.window + 1, 0) : 0;
    if (t.hi <= t.lo) t.lo = t.hi = 0;
    t.s0 = t.lo / p.split_len;
    t.s1 = t.hi > 0 ? (t.hi - 1) / p.split_len : 0;
    return t;
}

// First position that the token at position u sees.
__device__ __forceinline__ int low_of(const AttendProblem& p, int u) { return p.window > 0 ? max(u - p.window + 1, 0) : 0; }

// The pages of up to 64 groups of 16 positions, one per lane, from group `base` on:
// a bit per group that lies in no hole, and the page numbers.
struct Groups {
    int base, page;
    unsigned long long ok;
    __device__ __forceinline__ void load(const AttendProblem& p, int b, int g) {
        const int lane = threadIdx.x & 63;
        base = g;
        const int at = ((g + lane) << 4) >> p.c.page_shift;
        page = at < p.c.max_pages ? p.c.table[(int64_t)b * p.c.max_pages + at] : -1;
        ok = __builtin_amdgcn_ballot_w64(page >= 0 && page < p.c.n_pages);
    }
    __device__ __forceinline__ int page_of(int g) const { return __builtin_amdgcn_readlane(page, g - base); }
};

// Buffer over group g's rows of KV head h that lie before position `end`.
template <typename T, int D>
__device__ __forceinline__ rsrc_t group_rsrc(const AttendProblem& p, const void* pool, const Groups& gr, int g, int h, int end) {
    const int page = gr.page_of(g), at = (g << 4) & ((1 << p.c.page_shift) - 1);
    const int rows = min(16, end - (g << 4));
    const T* base = reinterpret_cast<const T*>(pool) + page * p.c.page_elems + (int64_t)at * p.c.ts + (int64_t)h * p.c.hs;
    const uint32_t bytes = ((rows - 1) * p.c.ts + D) * sizeof(T);
    return make_rsrc(base, rows > 0 && ((gr.ok >> (g - gr.base)) & 1ull) ? bytes : 0u);
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
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_void*)p; }

template <int S>
using Step = std::integral_constant<int, S>;

constexpr uint32_t kPastEnd = 0x80000000u;   // byte offset that every group's buffer reads as zero

// Running softmax of a row: `mo` is the largest exponent so far (base 2), -inf
// before the first visible position; `base` replaces it where it is -inf.
__device__ __forceinline__ float base_of(float mo) { return mo == -INFINITY ? 0.f : mo; }

// Row r's offset in the partial buffer's rows, of `row_of_head` order: (row of the
// packed axis, or batch row and token) x head.
__device__ __forceinline__ int64_t part_row(const AttendProblem& p, const NewTokens& nt, int b, int t, int h) {
    const int64_t row = p.c.start ? nt.row + t : (int64_t)b * p.c.max_new + t;
    return row * p.H_q + h;
}
__device__ __forceinline__ int64_t part_rows(const AttendProblem& p) { return (int64_t)p.c.n_new * p.H_q; }

// ---- few rows --------------------------------------------------------------

// grid (B * H_kv, n_split), 256 threads
template <int D>
__global__ __launch_bounds__(256, 2) void k_paged_decode(AttendProblem p) {
    constexpr int DC = D / 8, TILE = 32 * DC;      // 16-byte chunks of a row, of 32 rows
    constexpr int RPL = 64 / DC, NL = 32 / RPL;    // rows per wave load, loads per tile
    __shared__ u32x4 s_lds[4 * 2 * TILE + 4 * 32 / 2 + 1];   // K and V tiles per wave, (maximum, sum) per wave and row
    float2* s_ml = reinterpret_cast<float2*>(s_lds + 4 * 2 * TILE);   // [4][32]
    int* s_bad = reinterpret_cast<int*>(s_lds + 4 * 2 * TILE + 64);
    const int b = blockIdx.x / p.c.H_kv, kvh = blockIdx.x % p.c.H_kv, split = blockIdx.y;
    const NewTokens nt = new_tokens(p.c, b);
    if (nt.n <= 0) return;
    const Tile tl = tile_of(p, nt, 0, 32);
    if (split < tl.s0 || split > tl.s1) return;    // uniform over the workgroup
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5, G = p.H_q / p.c.H_kv;
    const int lrow = lane / DC, lch = lane % DC;
    const int l16 = lane & 15, vrow = 4 * g + (l16 >> 2), vch = 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1);
    auto vswz = [](int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); };
    u32x4* Kt = s_lds + w * 2 * TILE;   // row r: chunk c at c ^ causal_kswz(r)
    u32x4* Vt = Kt + TILE;              // row r: chunk c at c ^ vswz(r)

    // this lane's query row
    const bool row_ok = l32 < tl.n_rows;
    const int tok = min(l32, tl.n_rows - 1) / G, head = kvh * G + min(l32, tl.n_rows - 1) % G;
    u32x4 qop[D / 16];
    {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        const uint16_t* row = reinterpret_cast<const uint16_t*>(p.q) + row_offset(p.c, p.qs, nt, b, tok) + head * p.qs.head + 8 * g;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qop[ks] = row_ok ? *reinterpret_cast<const u32x4*>(row + 16 * ks) : zero;
    }
    const int u = tl.u0 + tok, ulo = low_of(p, u);
    const bool cut = tl.s0 != tl.s1;
    const int s_lo = split * p.split_len, s_hi = s_lo + p.split_len;
    const bool one = tl.t0 == tl.t1;
    uint32_t koff[NL], voff[NL];   // byte offsets within a group's buffer
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int r = i * RPL + lrow;
        koff[i] = ((uint32_t)(r & 15) * p.c.ts + 8 * (lch ^ causal_kswz<D>(r))) * 2;
        voff[i] = ((uint32_t)(r & 15) * p.c.ts + 8 * (lch ^ vswz(r))) * 2;
    }

    uint32_t vat[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) vat[db] = lds_address(Vt + vrow * DC + ((4 * db + vch) ^ vswz(vrow))) + 8 * (l16 & 1);

    // pass 0: all tokens; later passes, where that was not finite: one token each
    for (int pass = one ? 1 : 0; pass <= tl.t1 + 1; ++pass) {
        const int only = one ? 0 : pass - 1;      // token of this pass, -1: all
        const bool exact = only >= 0;             // positions below `lo` read as zeros
        const int lo = max(exact ? low_of(p, tl.u0 + only) : tl.lo, s_lo);
        const int hi = min(exact ? max(tl.u0 + only + 1, 0) : tl.hi, s_hi);
        f32x16 acc[D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;
        float mo = -INFINITY, l = 0.f;
        Groups gr;
        gr.base = 0; gr.page = -1; gr.ok = 0;
        auto load = [&](int kb, const void* pool, const uint32_t (&off)[NL], u32x4* tile) {
            const int gk = kb >> 4;
            const rsrc_t r0 = group_rsrc<uint16_t, D>(p, pool, gr, gk, kvh, hi), r1 = group_rsrc<uint16_t, D>(p, pool, gr, gk + 1, kvh, hi);
#pragma unroll
            for (int i = 0; i < NL; ++i)
                load_lds16(i * RPL < 16 ? r0 : r1, exact && kb + i * RPL + lrow < lo ? kPastEnd : off[i], tile + i * 64);
        };
        auto load_k = [&](int kb) { load(kb, p.k, koff, Kt); };
        auto load_v = [&](int kb) { load(kb, p.v, voff, Vt); };
        int kb = (lo & ~31) + 32 * w;
        __builtin_amdgcn_s_waitcnt(0x70);   // vmcnt(0) lgkmcnt(0): the waits below count loads into LDS only
        uint32_t okb = 0, oknext = 0;   // groups of the block in no hole
        if (kb < hi) {
            gr.load(p, b, kb >> 4);
            oknext = (uint32_t)gr.ok & 3u;
            load_k(kb);
            load_v(kb);
        }
        for (; kb < hi; kb += 128) {
            okb = oknext;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");   // K of this block
            f32x16 sc;
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                sc = mfma_32x32x16(Kt[l32 * DC + ((2 * ks + g) ^ causal_kswz<D>(l32))], qop[ks], sc);
            const int nx = kb + 128;
            const bool more = nx < hi;   // uniform
            wave_lds_sync();             // the operands are read: the next K may land
            if (more) {
                if ((nx >> 4) - gr.base > 62) {
                    // V of this block is in flight; its pages are not looked at again
                    gr.load(p, b, nx >> 4);
                }
                oknext = (uint32_t)(gr.ok >> ((nx >> 4) - gr.base)) & 3u;
                load_k(nx);
            }
            // rows that see every position of the block need no mask
            if (kb < lo || kb + 31 > tl.u0 + (exact ? only : 0) || okb != 3u || p.window > 0) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int v = kb + 8 * (e >> 2) + 4 * g + (e & 3);
                    sc[e] = v <= u && v >= ulo && v >= lo && v < hi && ((okb >> (e >> 3)) & 1u) ? sc[e] : -INFINITY;
                }
            }
            float cm = sc[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) cm = fmaxf(cm, sc[e]);
            cm = fmaxf(cm, __shfl_xor(cm, 32, 64));
            const float mon = fmaxf(mo, cm * p.scale_log2), off = base_of(mon);
            const float alpha = __builtin_amdgcn_exp2f(mo - off);
            float rs = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sc[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], p.scale_log2, -off));
                rs += sc[e];
            }
            rs += __shfl_xor(rs, 32, 64);
            l = l * alpha + rs;
            if (__builtin_amdgcn_ballot_w64(mon != mo)) {
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[db][e] *= alpha;
            }
            mo = mon;
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");   // V of this block
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            auto step = [&](auto s_) {
                constexpr int s = decltype(s_)::value;
                u32x2 va[D / 16];
                read_vt<D, s * 16 * D * 2>(vat, va);
                const u32x4 pf = {pack_bf16x2(sc[8 * s], sc[8 * s + 1]), pack_bf16x2(sc[8 * s + 2], sc[8 * s + 3]),
                                  pack_bf16x2(sc[8 * s + 4], sc[8 * s + 5]), pack_bf16x2(sc[8 * s + 6], sc[8 * s + 7])};
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
                    acc[db] = mfma_32x32x16(u32x4{va[2 * db].x, va[2 * db].y, va[2 * db + 1].x, va[2 * db + 1].y}, pf, acc[db]);
            };
            step(Step<0>{});
            step(Step<1>{});
            if (more) load_v(nx);   // the V operands are read
        }
        // the waves' rows, joined through their tiles: row, chunk c of four floats at c ^ (row % (D / 4))
        f32x4* mine = reinterpret_cast<f32x4*>(Kt);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                mine[l32 * (D / 4) + ((8 * db + 2 * i + g) ^ (l32 & (D / 4 - 1)))] =
                    f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]};
        if (g == 0) s_ml[w * 32 + l32] = make_float2(mo, l);
        if (tid == 0) *s_bad = 0;
        __syncthreads();
        const int r = tid >> 3;   // eight threads per row, D / 8 elements each
        float M = -INFINITY, sum = 0.f, wt[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) M = fmaxf(M, s_ml[i * 32 + r].x);
        const float off = base_of(M);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 ml = s_ml[i * 32 + r];
            wt[i] = __builtin_amdgcn_exp2f(ml.x - off);
            sum += ml.y * wt[i];
        }
        f32x4 x[D / 32];
        float t = 0.f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            const int at = r * (D / 4) + (((tid & 7) * (D / 32) + c) ^ (r & (D / 4 - 1)));
            x[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 y = reinterpret_cast<const f32x4*>(s_lds + i * 2 * TILE)[at];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[c][j] += wt[i] * y[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) t = fmaf(x[c][j], 0.f, t);
        }
        const int rt = r / G;
        const bool store = r < tl.n_rows && (!exact || rt == only);
        if (!exact) {
            if (store && t != t) *s_bad = 1;
            __syncthreads();
            const int bad = *s_bad;
            __syncthreads();   // the tiles and the flag may be written again
            if (bad) continue;
        }
        if (store) {
            const int hh = kvh * G + r - rt * G;
            if (cut) {
                const int64_t row = split * part_rows(p) + part_row(p, nt, b, rt, hh);
                f32x4* o = reinterpret_cast<f32x4*>(p.part + row * D) + (tid & 7) * (D / 32);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) o[c] = x[c];
                if ((tid & 7) == 0)
                    reinterpret_cast<float2*>(p.part + p.n_split * part_rows(p) * D)[row] = make_float2(M, sum);
            } else {
                const float inv = sum != 0.f ? 1.0f / sum : 0.f;
                uint16_t* o = reinterpret_cast<uint16_t*>(p.o) + row_offset(p.c, p.os, nt, b, rt) + hh * p.os.head + (tid & 7) * (D / 8);
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
                    reinterpret_cast<u32x2*>(o)[c] = u32x2{pack_bf16x2(x[c][0] * inv, x[c][1] * inv), pack_bf16x2(x[c][2] * inv, x[c][3] * inv)};
            }
        }
        if (!exact || one) break;
        __syncthreads();   // the tiles are read: the next token's may land
    }
}

// ---- many rows -------------------------------------------------------------

// Work items (sequence, KV head, range) x tile: the tiles of one go to one XCD, so that
// its K and V are read into one L2, the longest tile first.  grid 8 * ceil(groups / 8)
// * n_tile, 256 threads
template <int D>
__global__ __launch_bounds__(256, 2) void k_paged_chunk(AttendProblem p, int n_tile) {
    constexpr int DC = D / 8, KS = 64 * DC;        // 16-byte slots of a K or V chunk
    constexpr int RPL = 64 / DC, NQ = 16 / RPL;    // rows per wave load, loads per wave and chunk
    // two stages of K rows (chunk c at c ^ causal_kswz(row)) and V rows (c ^ vswz(row)), one flag
    __shared__ u32x4 lds[4 * KS + 1];
    int* s_bad = reinterpret_cast<int*>(lds + 4 * KS);
    const int slot = blockIdx.x >> 3, group = slot / n_tile * 8 + (blockIdx.x & 7);
    const int tile = n_tile - 1 - slot % n_tile;
    if (group >= p.c.B * p.c.H_kv * p.n_split) return;
    const int split = group % p.n_split, kvh = group / p.n_split % p.c.H_kv, b = group / p.n_split / p.c.H_kv;
    const NewTokens nt = new_tokens(p.c, b);
    const int G = p.H_q / p.c.H_kv;
    if (tile * 128 >= nt.n * G) return;            // uniform over the workgroup
    const Tile tl = tile_of(p, nt, tile, 128);
    if (split < tl.s0 || split > tl.s1) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5, lrow = lane / DC, lch = lane % DC;
    const int l16 = lane & 15, vrow = 4 * g + (l16 >> 2), vch = 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1);
    auto vswz = [](int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); };

    const int r = tl.r0 + 32 * w + l32, rr = min(r, tl.n_rows - 1);
    const bool row_ok = r < tl.n_rows;
    const int tok = rr / G, head = kvh * G + rr - tok * G;
    const bool wave_ok = tl.r0 + 32 * w < tl.n_rows;
    u32x4 qop[D / 16];
    {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        const uint16_t* row = reinterpret_cast<const uint16_t*>(p.q) + row_offset(p.c, p.qs, nt, b, tok) + head * p.qs.head + 8 * g;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qop[ks] = row_ok ? *reinterpret_cast<const u32x4*>(row + 16 * ks) : zero;
    }
    const int u = tl.u0 + tok, ulo = low_of(p, u);
    // first and last position of this wave's tokens
    const int wu0 = tl.u0 + min(tl.r0 + 32 * w, tl.n_rows - 1) / G, wu1 = tl.u0 + min(tl.r0 + 32 * w + 31, tl.n_rows - 1) / G;
    const int wlo = low_of(p, wu0), wlo1 = low_of(p, wu1);
    const bool cut = tl.s0 != tl.s1;
    const int s_lo = split * p.split_len, s_hi = s_lo + p.split_len;
    uint32_t koff[NQ], voff[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int row = 16 * w + q * RPL + lrow;
        koff[q] = ((uint32_t)(row & 15) * p.c.ts + 8 * (lch ^ causal_kswz<D>(row))) * 2;
        voff[q] = ((uint32_t)(row & 15) * p.c.ts + 8 * (lch ^ vswz(row))) * 2;
    }
    auto barrier = [&]() {
        __builtin_amdgcn_s_waitcnt(0x70);   // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    uint32_t vat[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) vat[db] = lds_address(lds + KS + vrow * DC + ((4 * db + vch) ^ vswz(vrow))) + 8 * (l16 & 1);
    const int tokens = tl.t1 - tl.t0 + 1;
    if (tid == 0) *s_bad = 0;
    // pass 0: all tokens; later passes, where that was not finite: one token each
    for (int pass = tokens > 1 ? 0 : 1; pass <= tokens; ++pass) {
        const int only = pass - 1 + tl.t0;
        const bool exact = pass > 0;
        const int lo = max(exact ? low_of(p, tl.u0 + only) : tl.lo, s_lo);
        const int hi = min(exact ? max(tl.u0 + only + 1, 0) : tl.hi, s_hi);
        f32x16 acc[D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;
        float mo = -INFINITY, l = 0.f;
        Groups gr;
        gr.base = 0; gr.page = -1; gr.ok = 0;
        auto issue = [&](int kc, int st) {
            u32x4* kd = lds + st * 2 * KS + w * NQ * 64;
            const int gw = (kc >> 4) + w;
            const rsrc_t kr = group_rsrc<uint16_t, D>(p, p.k, gr, gw, kvh, hi), vr = group_rsrc<uint16_t, D>(p, p.v, gr, gw, kvh, hi);
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const bool low = exact && kc + 16 * w + q * RPL + lrow < lo;
                load_lds16(kr, low ? kPastEnd : koff[q], kd + q * 64);
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const bool low = exact && kc + 16 * w + q * RPL + lrow < lo;
                load_lds16(vr, low ? kPastEnd : voff[q], kd + KS + q * 64);
            }
        };
        const int k0 = lo & ~63;
        uint32_t ok = 0, oknext = 0;
        barrier();   // the last pass's chunks are consumed
        if (k0 < hi) {
            gr.load(p, b, k0 >> 4);
            oknext = (uint32_t)gr.ok & 15u;
            issue(k0, 0);
        }
        barrier();
        for (int kc = k0, st = 0; kc < hi; kc += 64, st ^= 1) {
            ok = oknext;
            if (kc + 64 < hi) {
                if (((kc + 64) >> 4) - gr.base > 60) gr.load(p, b, (kc + 64) >> 4);
                oknext = (uint32_t)(gr.ok >> (((kc + 64) >> 4) - gr.base)) & 15u;
                issue(kc + 64, st ^ 1);
            }
            const u32x4* Kl = lds + st * 2 * KS;
            // a chunk that no row of this wave sees adds nothing (uniform)
            if (wave_ok && kc <= wu1 && kc + 63 >= wlo) {
                const bool masked = kc + 63 > wu0 || kc < wlo1 || kc < lo || kc + 64 > hi || ok != 15u;
                f32x16 sc[2];
                float cm = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[kb][e] = 0.f;
                    const int kr = kb * 32 + l32;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)
                        sc[kb] = mfma_32x32x16(Kl[kr * DC + ((2 * ks + g) ^ causal_kswz<D>(kr))], qop[ks], sc[kb]);
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int v = kc + kb * 32 + 8 * (e >> 2) + 4 * g + (e & 3);
                            sc[kb][e] = v <= u && v >= ulo && v >= lo && v < hi && ((ok >> (2 * kb + (e >> 3))) & 1u) ? sc[kb][e] : -INFINITY;
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) cm = fmaxf(cm, sc[kb][e]);
                }
                cm = fmaxf(cm, __shfl_xor(cm, 32, 64));
                const float mon = fmaxf(mo, cm * p.scale_log2), off = base_of(mon);
                const float alpha = __builtin_amdgcn_exp2f(mo - off);
                float rs = 0.f;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float ex = __builtin_amdgcn_exp2f(fmaf(sc[kb][e], p.scale_log2, -off));
                        sc[kb][e] = ex;
                        rs += ex;
                    }
                rs += __shfl_xor(rs, 32, 64);
                l = l * alpha + rs;
                if (__builtin_amdgcn_ballot_w64(mon != mo)) {
#pragma unroll
                    for (int db = 0; db < D / 32; ++db)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[db][e] *= alpha;
                }
                mo = mon;
                uint32_t at[D / 32];
#pragma unroll
                for (int db = 0; db < D / 32; ++db) at[db] = vat[db] + (uint32_t)st * (2 * KS * 16);
                auto step = [&](auto s_) {
                    constexpr int s = decltype(s_)::value, kb = s >> 1, e0 = 8 * (s & 1);
                    u32x2 va[D / 16];
                    read_vt<D, s * 16 * D * 2>(at, va);
                    const u32x4 pf = {pack_bf16x2(sc[kb][e0], sc[kb][e0 + 1]), pack_bf16x2(sc[kb][e0 + 2], sc[kb][e0 + 3]),
                                      pack_bf16x2(sc[kb][e0 + 4], sc[kb][e0 + 5]), pack_bf16x2(sc[kb][e0 + 6], sc[kb][e0 + 7])};
#pragma unroll
                    for (int db = 0; db < D / 32; ++db)
                        acc[db] = mfma_32x32x16(u32x4{va[2 * db].x, va[2 * db].y, va[2 * db + 1].x, va[2 * db + 1].y}, pf, acc[db]);
                };
                step(Step<0>{});
                step(Step<1>{});
                step(Step<2>{});
                step(Step<3>{});
            }
            barrier();   // the next chunk has landed; every wave is done with this one
        }
        if (!exact) {
            float t = 0.f;   // NaN where an accumulator is not finite
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int e = 0; e < 16; ++e) t = fmaf(acc[db][e], 0.f, t);
            if (row_ok && t != t) *s_bad = 1;
            __syncthreads();
            if (*s_bad) continue;    // uniform: not written again
        }
        // lane holds d = 32 db + 8 i + 4 g + {0..3} of its row
        if (row_ok && (!exact || tok == only)) {
            if (cut) {
                const int64_t row = split * part_rows(p) + part_row(p, nt, b, tok, head);
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(p.part + row * D + 32 * db + 8 * i + 4 * g) =
                            f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]};
                if (g == 0) reinterpret_cast<float2*>(p.part + p.n_split * part_rows(p) * D)[row] = make_float2(mo, l);
            } else {
                const float inv = l != 0.f ? 1.0f / l : 0.f;
                uint16_t* o = reinterpret_cast<uint16_t*>(p.o) + row_offset(p.c, p.os, nt, b, tok) + head * p.os.head;
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<u32x2*>(o + 32 * db + 8 * i + 4 * g) =
                            u32x2{pack_bf16x2(acc[db][4 * i] * inv, acc[db][4 * i + 1] * inv),
                                  pack_bf16x2(acc[db][4 * i + 2] * inv, acc[db][4 * i + 3] * inv)};
            }
        }
        if (!exact) break;
    }
}

// ---- fp32 ------------------------------------------------------------------

// D(16x16) += A(16x4) * B(4x16), fp32: lane l holds A row (l % 16), k = l / 16; B
// column (l % 16), the same k; D column (l % 16), rows 4 * (l / 16) + j at element j.
__device__ __forceinline__ f32x4 mfma_16x16x4(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// The order of the contraction is free as long as both operands keep it: step (s, j)
// of K . Q^T takes d = 16 s + 4 k + j, so that a lane's four steps are one 16-byte
// read; step j of V^T . P^T takes position 4 k + j, where the scores already lie.
// grid as k_paged_chunk, tiles of 64 rows
template <int D>
__global__ __launch_bounds__(256, 2) void k_paged_f32(AttendProblem p, int n_tile) {
    constexpr int DC = D / 4, KS = 32 * DC;        // 16-byte slots of a K or V chunk of 32 positions
    constexpr int RPL = 64 / DC, NQ = 8 / RPL;     // rows per wave load, loads per wave and chunk
    __shared__ f32x4 lds[4 * KS + 1];
    int* s_bad = reinterpret_cast<int*>(lds + 4 * KS);
    const int slot = blockIdx.x >> 3, group = slot / n_tile * 8 + (blockIdx.x & 7);
    const int tile = n_tile - 1 - slot % n_tile;
    if (group >= p.c.B * p.c.H_kv * p.n_split) return;
    const int split = group % p.n_split, kvh = group / p.n_split % p.c.H_kv, b = group / p.n_split / p.c.H_kv;
    const NewTokens nt = new_tokens(p.c, b);
    const int G = p.H_q / p.c.H_kv;
    if (tile * 64 >= nt.n * G) return;             // uniform over the workgroup
    const Tile tl = tile_of(p, nt, tile, 64);
    if (split < tl.s0 || split > tl.s1) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g4 = lane >> 4, lrow = lane / DC, lch = lane % DC;
    auto kswz = [](int row) { return row & 15; };
    auto vswz = [](int row) { return 4 * ((row >> 2) & 3); };

    const int r = tl.r0 + 16 * w + l16, rr = min(r, tl.n_rows - 1);
    const bool row_ok = r < tl.n_rows, wave_ok = tl.r0 + 16 * w < tl.n_rows;
    const int tok = rr / G, head = kvh * G + rr - tok * G;
    f32x4 qop[D / 16];
    {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const float* row = reinterpret_cast<const float*>(p.q) + row_offset(p.c, p.qs, nt, b, tok) + head * p.qs.head + 4 * g4;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qop[s] = row_ok ? *reinterpret_cast<const f32x4*>(row + 16 * s) : zero;
    }
    const int u = tl.u0 + tok, ulo = low_of(p, u);
    const bool cut = tl.s0 != tl.s1;
    const int s_lo = split * p.split_len, s_hi = s_lo + p.split_len;
    uint32_t koff[NQ], voff[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int row = 8 * w + q * RPL + lrow;
        koff[q] = ((uint32_t)(row & 15) * p.c.ts + 4 * (lch ^ kswz(row))) * 4;
        voff[q] = ((uint32_t)(row & 15) * p.c.ts + 4 * (lch ^ vswz(row))) * 4;
    }
    auto barrier = [&]() {
        __builtin_amdgcn_s_waitcnt(0x70);   // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    const int tokens = tl.t1 - tl.t0 + 1;
    if (tid == 0) *s_bad = 0;
    // pass 0: all tokens; later passes, where that was not finite: one token each
    for (int pass = tokens > 1 ? 0 : 1; pass <= tokens; ++pass) {
        const int only = pass - 1 + tl.t0;
        const bool exact = pass > 0;
        const int lo = max(exact ? low_of(p, tl.u0 + only) : tl.lo, s_lo);
        const int hi = min(exact ? max(tl.u0 + only + 1, 0) : tl.hi, s_hi);
        f32x4 acc[D / 16];
#pragma unroll
        for (int db = 0; db < D / 16; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
        float mo = -INFINITY, l = 0.f;
        Groups gr;
        gr.base = 0; gr.page = -1; gr.ok = 0;
        auto issue = [&](int kc, int st) {
            u32x4* kd = reinterpret_cast<u32x4*>(lds) + st * 2 * KS + w * NQ * 64;
            const int gw = (kc >> 4) + (w >> 1);
            const rsrc_t kr = group_rsrc<float, D>(p, p.k, gr, gw, kvh, hi), vr = group_rsrc<float, D>(p, p.v, gr, gw, kvh, hi);
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const bool low = exact && kc + 8 * w + q * RPL + lrow < lo;
                load_lds16(kr, low ? kPastEnd : koff[q], kd + q * 64);
                load_lds16(vr, low ? kPastEnd : voff[q], kd + KS + q * 64);
            }
        };
        const int k0 = lo & ~31;
        uint32_t ok = 0, oknext = 0;
        barrier();   // the last pass's chunks are consumed
        if (k0 < hi) {
            gr.load(p, b, k0 >> 4);
            oknext = (uint32_t)gr.ok & 3u;
            issue(k0, 0);
        }
        barrier();
        for (int kc = k0, st = 0; kc < hi; kc += 32, st ^= 1) {
            ok = oknext;
            if (kc + 32 < hi) {
                if (((kc + 32) >> 4) - gr.base > 62) gr.load(p, b, (kc + 32) >> 4);
                oknext = (uint32_t)(gr.ok >> (((kc + 32) >> 4) - gr.base)) & 3u;
                issue(kc + 32, st ^ 1);
            }
            const f32x4* Kl = lds + st * 2 * KS;
            const float* Vl = reinterpret_cast<const float*>(Kl + KS);
            if (wave_ok) {
                f32x4 sc[2];
                float cm = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    sc[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
                    const int kr = 16 * kb + l16;
#pragma unroll
                    for (int s = 0; s < D / 16; ++s) {
                        const f32x4 a = Kl[kr * DC + ((4 * s + g4) ^ kswz(kr))];
#pragma unroll
                        for (int j = 0; j < 4; ++j) sc[kb] = mfma_16x16x4(a[j], qop[s][j], sc[kb]);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int v = kc + 16 * kb + 4 * g4 + j;
                        sc[kb][j] = v <= u && v >= ulo && v >= lo && v < hi && ((ok >> kb) & 1u) ? sc[kb][j] : -INFINITY;
                        cm = fmaxf(cm, sc[kb][j]);
                    }
                }
                cm = fmaxf(cm, __shfl_xor(cm, 16, 64));
                cm = fmaxf(cm, __shfl_xor(cm, 32, 64));
                const float mon = fmaxf(mo, cm * p.scale_log2), off = base_of(mon);
                const float alpha = __builtin_amdgcn_exp2f(mo - off);
                float rs = 0.f;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sc[kb][j] = __builtin_amdgcn_exp2f(fmaf(sc[kb][j], p.scale_log2, -off));
                        rs += sc[kb][j];
                    }
                rs += __shfl_xor(rs, 16, 64);
                rs += __shfl_xor(rs, 32, 64);
                l = l * alpha + rs;
                if (__builtin_amdgcn_ballot_w64(mon != mo)) {
#pragma unroll
                    for (int db = 0; db < D / 16; ++db)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[db][j] *= alpha;
                }
                mo = mon;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int db = 0; db < D / 16; ++db)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int row = 16 * kb + 4 * g4 + j;
                            acc[db] = mfma_16x16x4(Vl[row * D + (((4 * db + (l16 >> 2)) ^ vswz(row)) << 2) + (l16 & 3)], sc[kb][j], acc[db]);
                        }
            }
            barrier();   // the next chunk has landed; every wave is done with this one
        }
        if (!exact) {
            float t = 0.f;
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
#pragma unroll
                for (int j = 0; j < 4; ++j) t = fmaf(acc[db][j], 0.f, t);
            if (row_ok && t != t) *s_bad = 1;
            __syncthreads();
            if (*s_bad) continue;    // uniform: not written again
        }
        // lane holds d = 16 db + 4 g4 + {0..3} of its row
        if (row_ok && (!exact || tok == only)) {
            float* o;
            float inv = 1.f;
            if (cut) {
                const int64_t row = split * part_rows(p) + part_row(p, nt, b, tok, head);
                o = p.part + row * D;
                if (g4 == 0) reinterpret_cast<float2*>(p.part + p.n_split * part_rows(p) * D)[row] = make_float2(mo, l);
            } else {
                o = reinterpret_cast<float*>(p.o) + row_offset(p.c, p.os, nt, b, tok) + head * p.os.head;
                inv = l != 0.f ? 1.0f / l : 0.f;
            }
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                f32x4 x = acc[db];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] *= inv;
                *reinterpret_cast<f32x4*>(o + 16 * db + 4 * g4) = x;
            }
        }
        if (!exact) break;
    }
}

// ---- cut rows ----------------------------------------------------------------

// Rows of tiles of `rows` rows whose positions were cut: the ranges' sums brought to
// one maximum and added in their order.  Four elements per thread.
// grid (ceil(max_new * H_q * D / 4 / 256), B)
template <typename T, int D>
__global__ __launch_bounds__(256) void k_paged_join(AttendProblem p, int rows) {
    const int b = blockIdx.y, x = blockIdx.x * 256 + threadIdx.x, c = x % (D / 4), th = x / (D / 4);
    const int t = th / p.H_q, h = th - t * p.H_q, G = p.H_q / p.c.H_kv;
    const NewTokens nt = new_tokens(p.c, b);
    if (t >= nt.n) return;
    const Tile tl = tile_of(p, nt, (t * G + h % G) / rows, rows);
    if (tl.s0 == tl.s1) return;
    const int64_t row = part_row(p, nt, b, t, h), step = part_rows(p);
    const float2* ml = reinterpret_cast<const float2*>(p.part + p.n_split * step * D) + row;
    const f32x4* part = reinterpret_cast<const f32x4*>(p.part + row * D) + c;
    float M = -INFINITY, sum = 0.f;
    for (int s = tl.s0; s <= tl.s1; ++s) M = fmaxf(M, ml[s * step].x);
    const float off = base_of(M);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s = tl.s0; s <= tl.s1; ++s) {
        const float2 y = ml[s * step];
        const float wt = __builtin_amdgcn_exp2f(y.x - off);
        const f32x4 z = part[s * step * (D / 4)];
        sum += y.y * wt;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += wt * z[j];
    }
    const float inv = sum != 0.f ? 1.0f / sum : 0.f;
    T* o = reinterpret_cast<T*>(p.o) + row_offset(p.c, p.os, nt, b, t) + h * p.os.head + 4 * c;
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x2*>(o) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
    else
        *reinterpret_cast<f32x4*>(o) = f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
}

// Rows of a tile: 32 where all of a sequence's fit, else 128; fp32 64.
int tile_rows(const AttendProblem& p, bool bf16) {
    return !bf16 ? 64 : (int64_t)p.c.max_new * (p.H_q / p.c.H_kv) <= 32 ? 32 : 128;
}
int tile_count(const AttendProblem& p, int rows) {
    return (int)(((int64_t)p.c.max_new * (p.H_q / p.c.H_kv) + rows - 1) / rows);
}

template <int D>
hipError_t launch_d(const AttendProblem& p, bool bf16, hipStream_t stream) {
    const int rows = tile_rows(p, bf16), tiles = tile_count(p, rows);
    const int64_t groups = (int64_t)p.c.B * p.c.H_kv * p.n_split;
    const int64_t grid = 8 * ((groups + 7) / 8) * tiles;
    if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
    if (rows == 32) k_paged_decode<D><<<dim3(p.c.B * p.c.H_kv, p.n_split), 256, 0, stream>>>(p);
    else if (bf16) k_paged_chunk<D><<<(unsigned)grid, 256, 0, stream>>>(p, tiles);
    else k_paged_f32<D><<<(unsigned)grid, 256, 0, stream>>>(p, tiles);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.n_split == 1) return e;
    const dim3 join((unsigned)(((int64_t)p.c.max_new * p.H_q * (D / 4) + 255) / 256), p.c.B);
    if (bf16) k_paged_join<uint16_t, D><<<join, 256, 0, stream>>>(p, rows);
    else k_paged_join<float, D><<<join, 256, 0, stream>>>(p, rows);
    return hipGetLastError();
}

}  // namespace

void attend_cuts(AttendProblem& p, bool bf16) {
    const int rows = tile_rows(p, bf16);
    const int64_t most = (int64_t)p.c.max_pages << p.c.page_shift;
    const int64_t work = (int64_t)p.c.B * p.c.H_kv * tile_count(p, rows);
    // ranges until there are several workgroups for every CU
    int64_t n = (1024 + work - 1) / work, len = (p.max_kv + n - 1) / n;
    const int64_t least = rows == 32 ? 256 : 512;
    if (n == 1 || (int64_t)p.c.max_new * p.H_q * p.c.D > (int64_t)1 << 31) len = most;
    len = ((len < least ? least : len) + 127) / 128 * 128;
    n = (most + len - 1) / len;
    if (n > 65535) {
        n = 65535;
        len = ((most + n - 1) / n + 127) / 128 * 128;
        n = (most + len - 1) / len;
    }
    p.n_split = (int32_t)n;
    p.split_len = (int32_t)len;
}

size_t attend_part_bytes(const AttendProblem& p) {
    if (p.n_split == 1) return 0;
    return (size_t)p.n_split * p.c.n_new * p.H_q * (p.c.D + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const AttendProblem& p, bool bf16, hipStream_t stream) {
    return p.c.D == 128 ? launch_d<128>(p, bf16, stream) : launch_d<64>(p, bf16, stream);
}

}  // namespace mot
