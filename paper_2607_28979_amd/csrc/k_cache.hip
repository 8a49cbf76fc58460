// The paged cache: new tokens into their pages (norms and rotation on the
// way), reordering of the table's rows, compaction of the pool.
#include "cache_internal.h"
#include "mot_device.h"

namespace mot {

namespace {

// 8 elements of a row as floats, and back
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x4 w = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = w[j];
    }
}
// PAST: past the caches
template <bool PAST, typename V>
__device__ __forceinline__ void store16(V* p, V v) {
    if constexpr (PAST) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool PAST>
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    store16<PAST>(reinterpret_cast<u32x4*>(p),
            u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])});
}
template <bool PAST>
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
        store16<PAST>(reinterpret_cast<f32x4*>(p) + i, f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]});
}

constexpr int kMostTokens = 4;   // tokens of a workgroup (4 kMostWorkgroups of a call)

// The sequence whose new tokens packed row `row` is among (-1: none), and its number among
// them, by a wave: the last sequence that starts at `row` or before, 64 starts at a time.
__device__ __forceinline__ int sequence_of(const PageTable& c, int row, int* i) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = c.B;   // it is one of lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 63) / 64, at = lo + lane * step;
        const unsigned long long before = __builtin_amdgcn_ballot_w64(lane * step < n && c.start[min(at, c.B - 1)] <= row);
        const int k = before ? 63 - __builtin_clzll(before) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    const NewTokens t = new_tokens(c, lo);
    *i = row - t.row;
    return *i >= 0 && *i < t.n ? lo : -1;
}

// Norms, rotation and stores of `tpb` new tokens of one sequence and layer: rows are
// the token's query, key and value heads, LPR lanes each, two 16-byte chunks of
// 8 elements (bf16) per lane: c and c + rot / 16 of the rotated part, so that
// both elements of a half-split pair are in one lane.  Angles are shared by a
// token's heads: computed once per workgroup, into LDS; position * inv_freq in
// fp64, since fp32 leaves an error of 2e-3 turns at position 32768.
// Bound: bytes for long prompts (4096 tokens of 28 + 2 x 4 heads of 128, 75 MB: 17 us of
// which 3.5 are the launch; 28 layers of 1501 tokens, 172 MB: 28 to 32 us), the launch
// and one chain of loads for single tokens (32 sequences: 5 us).  Rows two at a time, for
// more loads under way, took 108 registers and 10 to 25 % longer.
//
// grid (ceil(max_new / tpb), B, L), or FIND: (ceil(n_new / tpb), 1, L) over packed rows, whose
// sequences it finds among the starts; 256 threads
template <typename T, int LPR, bool PAST, bool FIND>
__global__ __launch_bounds__(256) void k_cache_append(AppendProblem p, int tpb) {
    __shared__ float2 s_turn[kMostTokens][128];
    __shared__ int64_t s_slot[kMostTokens];   // element offset of the token's place, -1: not stored
    __shared__ int s_pos[kMostTokens], s_b[kMostTokens];   // its position, its sequence (FIND; -1: none)
    const int l = blockIdx.z, tid = threadIdx.x, D = p.c.D, i0 = blockIdx.x * tpb;
    const int b = FIND ? 0 : blockIdx.y;
    NewTokens nt = {};
    int m;
    if constexpr (FIND) {
        m = min(tpb, p.c.n_new - i0);
        const int w = tid >> 6;
        if (w < m) {
            int i;
            const int at = sequence_of(p.c, i0 + w, &i);
            if ((tid & 63) == 0) {
                s_b[w] = at;
                const NewTokens n = new_tokens(p.c, max(at, 0));
                s_pos[w] = n.kv - n.count + i;
            }
        }
        __syncthreads();
    } else {
        nt = new_tokens(p.c, b);
        m = min(tpb, nt.n - i0);
        if (m <= 0) return;   // uniform over the workgroup
    }
    const int pos0 = nt.kv - nt.count + i0;
    auto position = [&](int t) { return FIND ? s_pos[t] : pos0 + t; };
    auto offset = [&](const RowStrides& st, int t) {
        return FIND ? (int64_t)(i0 + t) * st.token : row_offset(p.c, st, nt, b, i0 + t);
    };
    if (tid < m) {
        const int pos = position(tid), row = FIND ? s_b[tid] : b;
        int64_t at = -1;
        if (pos >= 0 && row >= 0) {
            const int page = p.c.table[(int64_t)row * p.c.max_pages + (pos >> p.c.page_shift)];
            if (page >= 0 && page < p.c.n_pages)
                at = ((int64_t)l * p.c.n_pages + page) * p.c.page_elems +
                     (int64_t)(pos & ((1 << p.c.page_shift) - 1)) * p.c.ts;
        }
        s_slot[tid] = at;
    }
    const int half = p.rot >> 1;
    if (p.inv_freq)
        for (int x = tid; x < m * half; x += 256) {
            const int t = x / half, r = x - t * half;
            const int pos = p.positions ? p.positions[p.c.start ? nt.row + i0 + t : b * p.c.max_new + i0 + t] : position(t);
            double turns = (double)pos * (double)p.inv_freq[r] * 0.15915494309189533577;
            turns -= rint(turns);
            float sn, cs;
            sincospif(2.0f * (float)turns, &sn, &cs);
            s_turn[t][r] = make_float2(cs, sn);
        }
    __syncthreads();
    const int nq = p.q ? p.H_q : 0, nk = p.k ? p.c.H_kv : 0, heads = nq + 2 * nk;
    const int c = tid % LPR, rc = p.rot >> 4, lanes = D >> 4;
    const bool live = c < lanes, turned = c < rc;
    const int lo = turned ? c : rc + c, hi = turned ? c + rc : lo + lanes - rc;   // chunks of 8
    for (int r = tid / LPR; r < m * heads; r += 256 / LPR) {
        const int t = r / heads, h = r - t * heads;
        if (FIND && s_b[t] < 0) continue;   // a row of no sequence
        const int kind = h < nq ? 0 : h < nq + nk ? 1 : 2, hh = kind == 0 ? h : kind == 1 ? h - nq : h - nq - nk;
        const RowStrides& st = kind == 0 ? p.qs : kind == 1 ? p.ks : p.vs;
        const T* src = reinterpret_cast<const T*>(kind == 0 ? p.q : kind == 1 ? p.k : p.v) + l * st.layer +
                       offset(st, t) + hh * st.head;
        T* dst;
        if (kind == 0) {
            dst = reinterpret_cast<T*>(p.q_out) + l * p.qos.layer + offset(p.qos, t) + hh * p.qos.head;
        } else {
            const int64_t at = s_slot[t];
            if (at < 0) continue;   // uniform over the row's lanes
            dst = reinterpret_cast<T*>(kind == 1 ? p.k_pages : p.v_pages) + at + (int64_t)hh * p.c.hs;
        }
        float x[8], y[8];
        if (live) {
            load8(src + 8 * lo, x);
            load8(src + 8 * hi, y);
        }
        const T* gain = reinterpret_cast<const T*>(kind == 0 ? p.q_gain : kind == 1 ? p.k_gain : nullptr);
        if (gain) {
            float ss = 0.f;
            if (live) {
#pragma unroll
                for (int j = 0; j < 8; ++j) ss += x[j] * x[j] + y[j] * y[j];
            }
#pragma unroll
            for (int w = 1; w < LPR; w <<= 1) ss += __shfl_xor(ss, w, 64);
            const float inv = 1.0f / sqrtf(ss / (float)D + p.eps);
            if (live) {
                float gx[8], gy[8];
                load8(gain + (int64_t)l * D + 8 * lo, gx);
                load8(gain + (int64_t)l * D + 8 * hi, gy);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] *= inv * gx[j];
                    y[j] *= inv * gy[j];
                }
            }
        }
        if (p.inv_freq && kind != 2 && turned) {
            if (p.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 u = s_turn[t][4 * lo + j], v = s_turn[t][4 * hi + j];
                    const float x0 = x[2 * j], y0 = y[2 * j];
                    x[2 * j] = x0 * u.x - x[2 * j + 1] * u.y;
                    x[2 * j + 1] = x[2 * j + 1] * u.x + x0 * u.y;
                    y[2 * j] = y0 * v.x - y[2 * j + 1] * v.y;
                    y[2 * j + 1] = y[2 * j + 1] * v.x + y0 * v.y;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 u = s_turn[t][8 * lo + j];
                    const float x0 = x[j];
                    x[j] = x0 * u.x - y[j] * u.y;
                    y[j] = y[j] * u.x + x0 * u.y;
                }
            }
        }
        if (live) {
            store8<PAST>(dst + 8 * lo, x);
            store8<PAST>(dst + 8 * hi, y);
        }
    }
}

template <typename T, bool PAST, bool FIND>
void append_by(const AppendProblem& p, int lpr, int tpb, dim3 grid, hipStream_t stream) {
    if (lpr == 2) k_cache_append<T, 2, PAST, FIND><<<grid, 256, 0, stream>>>(p, tpb);
    else if (lpr == 4) k_cache_append<T, 4, PAST, FIND><<<grid, 256, 0, stream>>>(p, tpb);
    else if (lpr == 8) k_cache_append<T, 8, PAST, FIND><<<grid, 256, 0, stream>>>(p, tpb);
    else k_cache_append<T, 16, PAST, FIND><<<grid, 256, 0, stream>>>(p, tpb);
}

template <typename T>
hipError_t append_as(const AppendProblem& p, hipStream_t stream) {
    // Tokens of a workgroup: one until there are several for every CU, then four where four
    // tokens' heads are one turn of its threads, else two.  Measured (us with 1, 2, 4 tokens,
    // heads of 128): 36 heads, 512 tokens 5.4, 6.2, 7.8; 2048: 11.8, 11.1, 12.2; 8192: 38,
    // 37, 42; 8 heads, 1800 tokens 4.6, 4.2, 4.1; 42000: 51, 42, 37 (8 tokens: 39), all with
    // ordinary stores.
    const int64_t tokens = (int64_t)p.c.n_new * p.L;
    const int lanes = p.c.D >> 4, lpr = lanes <= 2 ? 2 : lanes <= 4 ? 4 : lanes <= 8 ? 8 : 16;
    const int heads = (p.q ? p.H_q : 0) + (p.k ? 2 * p.c.H_kv : 0);
    // Packed rows one by one where most of the places that max_new admits are none: 200 single
    // tokens and 1500 of one sequence, 36 heads of 128, 49 -> 9.5 us, 47 and 512 11.8 -> 5.7,
    // 256 single ones with no bound 27 -> 5.2 (4.6 with it: finding the sequence).
    const bool find = p.c.start && (int64_t)p.c.max_new * p.c.B > 2 * (int64_t)p.c.n_new;
    const int rows = find ? p.c.n_new : p.c.max_new;
    // calls of more than 2^25 rows take four for the launch to hold them
    const int tpb = tokens < 1792 ? 1 : kMostTokens * heads * lpr <= 256 || rows > 2 * kMostWorkgroups ? kMostTokens : 2;
    const dim3 grid((rows + tpb - 1) / tpb, find ? 1 : p.c.B, p.L);
    // Stores past the caches where what is written is more than attention finds there again:
    // 28 layers of 1501 tokens, 86 MB written, 36.6 -> 28.4 us, 8192 tokens of 36 heads, 75 MB,
    // 36.7 -> 26.7.  Below, the call itself gains little (38 MB 17.5 -> 16.8) and attention
    // after it loses more (4096 tokens, both calls 202 -> 205).
    const bool past = (int64_t)p.c.n_new * p.L * heads * p.c.D * (int64_t)sizeof(T) > 64 << 20;
    if (past && find) append_by<T, true, true>(p, lpr, tpb, grid, stream);
    else if (past) append_by<T, true, false>(p, lpr, tpb, grid, stream);
    else if (find) append_by<T, false, true>(p, lpr, tpb, grid, stream);
    else append_by<T, false, false>(p, lpr, tpb, grid, stream);
    return hipGetLastError();
}

// ---- pages ----------------------------------------------------------------

constexpr int kThreads = 1024;   // of the one workgroup that gives out pages

// Workspace of reordering and compaction (int32 words), W = words of a bit per
// page.
struct PagesWs {
    uint32_t* held;    // [W] pages that new rows (or the table) name
    uint32_t* whole;   // [W] reorder: pages that a new row keeps whole
    int32_t* first;    // [n_pages] reorder: lowest row that keeps the page in part
    int32_t* list;     // [n_pages] reorder: free pages to give out; compact: targets of moves
    int32_t* from;     // [n_pages] compact: pages to move
    int32_t* rank;     // [W + 1] compact: held pages before each word
    int32_t* base;     // [n_rows] reorder: pages given out before each row
    int4* pair;        // [n_rows] reorder: (source page, new page, positions) of each copy
    int32_t* n_pair;   // [1] copies or moves
};
size_t r64(size_t n) { return (n + 63) & ~size_t(63); }
size_t ws_words(int64_t n_pages, int64_t n_rows, const void* at, PagesWs* out) {
    const size_t W = r64((size_t)(n_pages + 31) / 32 + 1), P = r64((size_t)n_pages), R = r64((size_t)n_rows);
    int32_t* c = reinterpret_cast<int32_t*>(const_cast<void*>(at));
    size_t n = 0;
    auto take = [&](size_t k) { int32_t* r = c + n; n += k; return r; };
    PagesWs w;
    w.pair = reinterpret_cast<int4*>(take(4 * R));
    w.held = reinterpret_cast<uint32_t*>(take(W));
    w.whole = reinterpret_cast<uint32_t*>(take(n_rows ? W : 0));
    w.first = take(n_rows ? P : 0);
    w.list = take(P);
    w.from = take(n_rows ? 0 : P);
    w.rank = take(n_rows ? 0 : W);
    w.base = take(R);
    w.n_pair = take(64);
    if (out) *out = w;
    return n;
}

// kept, whole and wanted pages of new row b
struct RowPlan {
    int32_t src, full, kept, need, rest;   // rest: positions of the last page, in part
};
__device__ __forceinline__ RowPlan row_plan(const PagesProblem& p, int b) {
    RowPlan r;
    const int sh = p.c.page_shift, most = p.c.max_pages << sh;
    r.src = p.source[b];
    const bool ok = r.src >= 0 && r.src < p.c.B;
    const int keep = ok ? min(max(p.keep[b], 0), most) : 0, want = max(min(p.want[b], most), keep);
    if (!ok) r.src = 0;
    r.full = keep >> sh;
    r.rest = keep - (r.full << sh);
    r.kept = r.full + (r.rest > 0);
    r.need = (want + (1 << sh) - 1) >> sh;
    return r;
}

__device__ __forceinline__ bool bit_of(const uint32_t* w, int page) { return (w[page >> 5] >> (page & 31)) & 1u; }

__global__ __launch_bounds__(256) void k_pages_clear(PagesProblem p, PagesWs w) {
    const int W = (p.c.n_pages + 31) / 32, i = blockIdx.x * 256 + threadIdx.x;
    if (i < W) {
        w.held[i] = 0;
        if (p.n_rows) w.whole[i] = 0;
    }
    if (p.n_rows && i < p.c.n_pages) w.first[i] = INT32_MAX;
}

// grid (ceil(max_pages / 256), rows)
__global__ __launch_bounds__(256) void k_pages_mark(PagesProblem p, PagesWs w) {
    const int b = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
    if (p.n_rows) {
        const RowPlan r = row_plan(p, b);
        if (j >= r.kept) return;
        const int page = p.c.table[(int64_t)r.src * p.c.max_pages + j];
        if (page < 0 || page >= p.c.n_pages) return;
        atomicOr(w.held + (page >> 5), 1u << (page & 31));
        if (j < r.full) atomicOr(w.whole + (page >> 5), 1u << (page & 31));
        else atomicMin(w.first + page, b);
    } else {
        if (j >= p.c.max_pages) return;
        const int page = p.c.table[(int64_t)b * p.c.max_pages + j];
        if (page >= 0 && page < p.c.n_pages) atomicOr(w.held + (page >> 5), 1u << (page & 31));
    }
}

// Exclusive sum over the workgroup's threads; *all: the total.
__device__ __forceinline__ int block_scan(int x, int* s_wave, int* all) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int y = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int z = __shfl_up(y, d, 64);
        if (lane >= d) y += z;
    }
    __syncthreads();   // the last call's sums are read
    if (lane == 63) s_wave[wv] = y;
    __syncthreads();
    int before = 0, sum = 0;
    for (int i = 0; i < kThreads / 64; ++i) {
        const int n = s_wave[i];
        before += i < wv ? n : 0;
        sum += n;
    }
    *all = sum;
    return before + y - x;
}

// One workgroup: what each row needs, the free pages in order, the copies.
__global__ __launch_bounds__(kThreads) void k_pages_give(PagesProblem p, PagesWs w) {
    __shared__ int s_wave[kThreads / 64];
    const int tid = threadIdx.x, W = (p.c.n_pages + 31) / 32;
    int asked = 0, copies = 0, all;
    for (int b0 = 0; b0 < p.n_rows; b0 += kThreads) {
        const int b = b0 + tid;
        int need = 0, copy = 0, page = -1, rest = 0;
        if (b < p.n_rows) {
            const RowPlan r = row_plan(p, b);
            if (r.rest) {
                page = p.c.table[(int64_t)r.src * p.c.max_pages + r.full];
                copy = page >= 0 && page < p.c.n_pages && (bit_of(w.whole, page) || w.first[page] != b);
                rest = r.rest;
            }
            need = copy + max(r.need - r.kept, 0);
        }
        const int at = asked + block_scan(need, s_wave, &all);
        asked += all;
        const int c = copies + block_scan(copy, s_wave, &all);
        copies += all;
        if (b < p.n_rows) w.base[b] = at;
        if (copy) w.pair[c] = make_int4(page, at, rest, 0);   // the page's place in the list, for now
    }
    int n_free = 0;
    for (int i0 = 0; i0 < W; i0 += kThreads) {
        const int i = i0 + tid;
        uint32_t f = i < W ? ~w.held[i] : 0u;
        if (i == W - 1 && (p.c.n_pages & 31)) f &= (1u << (p.c.n_pages & 31)) - 1u;
        int at = n_free + block_scan(__popc(f), s_wave, &all);
        n_free += all;
        for (; f && at < asked; f &= f - 1, ++at) w.list[at] = 32 * i + __ffs(f) - 1;
        if (n_free >= asked) break;   // uniform
    }
    __syncthreads();
    for (int c = tid; c < copies; c += kThreads) {
        const int at = w.pair[c].y;
        w.pair[c].y = at < n_free ? w.list[at] : -1;
    }
    if (tid == 0) {
        *w.n_pair = copies;
        *p.count = max(asked - n_free, 0);
    }
    // how many of the list exist, for the rows' tables
    if (tid == 0) w.n_pair[1] = min(asked, n_free);
}

// One workgroup: held pages before every word, the moves.
__global__ __launch_bounds__(kThreads) void k_pages_squeeze(PagesProblem p, PagesWs w) {
    __shared__ int s_wave[kThreads / 64];
    const int tid = threadIdx.x, W = (p.c.n_pages + 31) / 32;
    int used = 0, all;
    for (int i0 = 0; i0 < W; i0 += kThreads) {
        const int i = i0 + tid, at = block_scan(i < W ? __popc(w.held[i]) : 0, s_wave, &all);
        if (i < W) w.rank[i] = used + at;
        used += all;
    }
    __syncthreads();
    // held pages before page `used`: those that stay
    const int uw = used >> 5, stay = used == 0 ? 0
        : uw < W ? w.rank[uw] + __popc(w.held[uw] & ((1u << (used & 31)) - 1u)) : used;
    for (int i = tid; i < W; i += kThreads) {
        const uint32_t h = w.held[i];
        int before = w.rank[i];
        for (int k = 0; k < 32 && 32 * i + k < p.c.n_pages; ++k) {
            const int page = 32 * i + k;
            if ((h >> k) & 1u) {
                if (page >= used) w.from[before - stay] = page;
                ++before;
            } else if (page < used) {
                w.list[page - before] = page;
            }
        }
    }
    if (tid == 0) {
        *w.n_pair = used - stay;
        w.n_pair[1] = stay;
        *p.count = used;
    }
}

constexpr int kCopyChunks = 1024;   // 16-byte chunks of one copying work item at most

// Work item `it` of the copies of a call, by THREADS threads of which this is `tid`: a piece of
// a page of a layer's keys or values.  pair(c): pages from and to, and the positions to
// copy (0: all).  Four chunks per thread are under way at a time.
template <int THREADS, class Pair>
__device__ __forceinline__ void copy_item(const PagesProblem& p, int64_t it, int pieces, int tid, Pair pair) {
    // in 32 bits: the pools of 2^31 pages or pieces would not fit in the device's memory
    const uint32_t i0 = __builtin_amdgcn_readfirstlane((uint32_t)it), i1 = i0 / (uint32_t)pieces, i2 = i1 / (2u * p.L);
    const int piece = (int)(i0 - i1 * pieces), side = (int)(i1 - i2 * 2u * p.L);
    const int4 pr = pair((int)i2);
    if (pr.y < 0) return;
    const int64_t page_bytes = p.c.page_elems * p.elem_bytes, row_bytes = (int64_t)p.c.D * p.elem_bytes;
    // contiguous bytes: of each head where the heads come first
    int64_t run = page_bytes, pitch = 0;
    int runs = 1;
    if (pr.z && p.heads_first) {
        run = pr.z * row_bytes;
        runs = p.c.H_kv;
        pitch = row_bytes << p.c.page_shift;
    } else if (pr.z) {
        run = pr.z * row_bytes * p.c.H_kv;
    }
    char* pool = reinterpret_cast<char*>(side & 1 ? p.v_pages : p.k_pages) + (int64_t)(side >> 1) * p.c.n_pages * page_bytes;
    const char* from = pool + pr.x * page_bytes;
    char* to = pool + pr.y * page_bytes;
    const int chunks = (int)(run / 16), end = min((piece + 1) * kCopyChunks, chunks * runs);
    for (int x0 = piece * kCopyChunks + tid; x0 < end; x0 += 4 * THREADS) {
        u32x4 v[4];
        int64_t off[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = x0 + i * THREADS, y = runs > 1 ? x / chunks : 0;
            off[i] = y * pitch + (int64_t)(x - y * chunks) * 16;
            if (x < end) v[i] = *reinterpret_cast<const u32x4*>(from + off[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            // past the caches: 23 MB of last pages 11.9 -> 10.7 us, 455 MB of pages 192 -> 189
            if (x0 + i * THREADS < end) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(to + off[i]));
    }
}
__host__ __device__ inline int copy_pieces(const PagesProblem& p) {
    return (int)((p.c.page_elems * p.elem_bytes / 16 + kCopyChunks - 1) / kCopyChunks);
}

// The new table (the first `tables` workgroups), and the copies.
__global__ __launch_bounds__(256) void k_pages_apply(PagesProblem p, PagesWs w, int tables) {
    const int tid = threadIdx.x, M = p.c.max_pages;
    if ((int)blockIdx.x < tables) {
        const int rows = p.n_rows ? p.n_rows : p.c.B;
        const int64_t at = (int64_t)blockIdx.x * 256 + tid;
        if (at >= (int64_t)rows * M) return;
        const int b = (int)(at / M), j = (int)(at - (int64_t)b * M);
        int page = -1;
        if (p.n_rows) {
            const RowPlan r = row_plan(p, b);
            const int given = w.n_pair[1];
            int ask = -1;   // place in the list
            if (j < r.kept) {
                page = p.c.table[(int64_t)r.src * M + j];
                if (page < 0 || page >= p.c.n_pages) page = -1;
            }
            // a copied last page takes the row's first place in the list, added pages the next
            int copied = 0;
            if (r.rest && j >= r.full) {
                const int last = p.c.table[(int64_t)r.src * M + r.full];
                copied = last >= 0 && last < p.c.n_pages && (bit_of(w.whole, last) || w.first[last] != b);
            }
            if (j == r.full && r.rest && copied) ask = w.base[b];
            else if (j >= r.kept && j < r.need) ask = w.base[b] + copied + j - r.kept;
            if (ask >= 0) page = ask < given ? w.list[ask] : -1;
        } else {
            page = p.c.table[at];
            if (page < 0 || page >= p.c.n_pages) page = -1;
            else if (page >= *p.count)
                page = w.list[w.rank[page >> 5] + __popc(w.held[page >> 5] & ((1u << (page & 31)) - 1u)) - w.n_pair[1]];
        }
        p.new_table[at] = page;
        return;
    }
    const int pieces = copy_pieces(p);
    const int64_t items = (int64_t)*w.n_pair * 2 * p.L * pieces;
    for (int64_t it = blockIdx.x - tables; it < items; it += gridDim.x - tables)
        copy_item<256>(p, it, pieces, tid, [&](int c) { return p.n_rows ? w.pair[c] : make_int4(w.from[c], w.list[c], 0, 0); });
}

// ---- small pools and tables: one launch -----------------------------------------
//
// Every workgroup works out the whole plan in its own LDS, from the table and the rows
// (L2 holds them), and then does its share of the new table and of the copies: no
// workspace, no order between workgroups. All 16 waves of a CU run the plan, so an
// instruction more in its loops is felt (16 cycles per 1024 threads): a wave walks rows,
// not entries, and what a row says stays in scalars (entry by entry the reorder of 200 rows
// took 22 us). Against the launches above, replayed from a graph: 200 rows of 123 entries,
// 9015 pages, few copies 12.3 and 16.7 us; 64 rows of 39, 23 MB moved 10.7 and 18.6; a pool
// of 101 pages squeezed 7.8 and 14.7, one of 2096 pages x 14 layers (909 MB moved) 189
// (4.8 TB/s) and 201. At the limits, 16384 pages and 512 rows of 128: reorder 16.0 and 14.1,
// compaction 18.8 and 21.5 (4 rows of 16384: 26.5 and 14.3, 29.9 and 21.3), but issuing from
// the host 7 and 16 us.

constexpr int kOncePages = 16384, kOnceRows = 512, kOnceEntries = 65536;
constexpr int kOnceGrid = 256;   // a workgroup per CU
constexpr int kWaves = kThreads / 64;

// f(page, row, j) for the entries j < count(b) of rows b of a table of `rows` rows of M
// (row b reads row source(b)); a page out of range is skipped. A wave takes rows w, w + 16,
// ..., 8 rows x 128 entries of loads under way together; with fewer than 16 rows the waves
// share a row's entries.
template <class Source, class Count, class Use>
__device__ __forceinline__ void each_page(const int32_t* table, int N, int rows, int M, int wave, Source source, Count count,
                                          Use use) {
    constexpr int kRows = 8, kCuts = 2;
    const int lane = threadIdx.x & 63;
    const int share = rows >= kWaves ? 0 : 4 - (31 - __clz(rows));   // 2^share waves to a row
    const int step = kWaves >> share, b0 = wave >> share, cut0 = wave & ((1 << share) - 1);
    for (int bb = b0; bb < rows; bb += kRows * step) {
        for (int j0 = 64 * kCuts * cut0; j0 < M; j0 += 64 * kCuts << share) {
            int v[kRows * kCuts];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int32_t* t = table + (int64_t)source(min(bb + r * step, rows - 1)) * M;
#pragma unroll
                for (int k = 0; k < kCuts; ++k) v[r * kCuts + k] = t[min(j0 + 64 * k + lane, M - 1)];
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int b = bb + r * step;
                if (b >= rows) break;
                const int n = count(b);
#pragma unroll
                for (int k = 0; k < kCuts; ++k) {
                    const int j = j0 + 64 * k + lane, page = v[r * kCuts + k];
                    if (j < n && (uint32_t)page < (uint32_t)N) use(page, b, j);
                }
            }
        }
    }
}

struct OnceRow {
    int src, full, kept, need, rest, base, copied, spare;
};

// Bits of the words of mark[N] that are not 0, 32 to a word, by all threads. words: at
// least 2 * ceil(N / 64).
__device__ __forceinline__ void bits_of(const uint32_t* mark, int N, uint32_t* words, int wave) {
    const int lane = threadIdx.x & 63;
    for (int g = wave; 64 * g < N; g += kWaves) {
        const int i = 64 * g + lane;
        const uint64_t m = __ballot(i < N && mark[min(i, N - 1)] != 0);
        if (lane < 2) words[2 * g + lane] = (uint32_t)(m >> (32 * lane));
    }
}

__global__ __launch_bounds__(kThreads) void k_pages_reorder(PagesProblem p) {
    // a word per page: 0 free, ~0 kept whole by a row, else kept in part and the lowest
    // such row b as kOnceRows - b; once this is read, the free pages in order
    __shared__ __attribute__((aligned(16))) uint32_t mark[kOncePages];
    __shared__ OnceRow row[kOnceRows];
    __shared__ int4 pair[kOnceRows];
    __shared__ int last[kOnceRows];   // the page kept in part, -1: none
    __shared__ uint32_t held[kOncePages / 32 + 2];
    __shared__ int s_wave[kWaves];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int M = p.c.max_pages, N = p.c.n_pages, W = (N + 31) / 32, R = p.n_rows;
    for (int i = tid; i < (N + 3) / 4; i += kThreads) reinterpret_cast<u32x4*>(mark)[i] = u32x4{};
    if (tid < R) {
        const RowPlan r = row_plan(p, tid);
        row[tid] = OnceRow{r.src, r.full, r.kept, r.need, r.rest, 0, 0, 0};
        last[tid] = -1;
    }
    __syncthreads();
    if (p.c.B > 0) each_page(   // a table without rows is not read
        p.c.table, N, R, M, wave, [&](int b) { return __builtin_amdgcn_readfirstlane(row[b].src); },
        [&](int b) { return __builtin_amdgcn_readfirstlane(row[b].kept); },
        [&](int page, int b, int j) {
            // ~0 is the largest word, so a plain store and the maximum agree in any order
            if (j < row[b].full) {
                mark[page] = ~0u;
            } else {
                atomicMax(mark + page, (uint32_t)(kOnceRows - b));
                last[b] = page;
            }
        });
    __syncthreads();
    bits_of(mark, N, held, wave);
    // a row copies its last page if another keeps it whole, or a lower row in part
    int copied = 0, need = 0, sums;
    if (tid < R) {
        const int mine = last[tid];
        copied = mine >= 0 && mark[mine] != (uint32_t)(kOnceRows - tid);
        need = copied + max(row[tid].need - row[tid].kept, 0);
    }
    // both sums in one scan: at most kOnceEntries + kOnceRows pages, kOnceRows copies
    static_assert(kOnceEntries + kOnceRows < 1 << 20 && kOnceRows < 1 << 11, "");
    const int before = block_scan(copied << 20 | need, s_wave, &sums);
    const int at = before & ((1 << 20) - 1), c = before >> 20, asked = sums & ((1 << 20) - 1), copies = sums >> 20;
    if (tid < R) {
        row[tid].base = at;
        row[tid].copied = copied;
        if (copied) pair[c] = make_int4(last[tid], at, row[tid].rest, 0);   // its place in the list, for now
    }
    int* list = reinterpret_cast<int*>(mark);
    int n_free;
    {
        uint32_t f = tid < W ? ~held[tid] : 0u;   // W <= kThreads
        if (tid == W - 1 && (N & 31)) f &= (1u << (N & 31)) - 1u;
        int to = block_scan(__popc(f), s_wave, &n_free);
        for (; f && to < asked; f &= f - 1, ++to) list[to] = 32 * tid + __ffs(f) - 1;
    }
    __syncthreads();
    const int given = min(asked, n_free);
    if (blockIdx.x == 0 && tid == 0) *p.count = asked - given;
    for (int e = blockIdx.x + gridDim.x * tid; e < R * M; e += gridDim.x * kThreads) {
        const int b = e / M, j = e - b * M;
        const OnceRow r = row[b];
        int page = j < r.kept ? p.c.table[(int64_t)r.src * M + j] : -1, ask = -1;
        if ((uint32_t)page >= (uint32_t)N) page = -1;
        if (r.copied && j == r.full) ask = r.base;
        else if (j >= r.kept && j < r.need) ask = r.base + r.copied + j - r.kept;
        p.new_table[e] = ask < 0 ? page : ask < given ? list[ask] : -1;
    }
    const int pieces = copy_pieces(p);
    const int64_t items = (int64_t)copies * 2 * p.L * pieces;
    for (int64_t it = blockIdx.x + gridDim.x * (tid >> 8); it < items; it += gridDim.x * (kThreads >> 8))
        copy_item<256>(p, it, pieces, tid & 255, [&](int i) {
            const int4 x = pair[i];
            return make_int4(x.x, x.y < given ? list[x.y] : -1, x.z, 0);
        });
}

__global__ __launch_bounds__(kThreads) void k_pages_compact(PagesProblem p) {
    // a word per page, not 0: held; once this is read, pages to move and their places
    __shared__ __attribute__((aligned(16))) uint32_t mark[kOncePages + 4];
    // held as bits, and the held pages before each of its words
    __shared__ uint32_t held[kOncePages / 32 + 2];
    __shared__ int rank[kOncePages / 32 + 1];
    __shared__ int s_wave[kWaves];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int M = p.c.max_pages, N = p.c.n_pages, W = (N + 31) / 32;
    int* from = reinterpret_cast<int*>(mark);
    int* list = from + N / 2 + 1;
    for (int i = tid; i < (N + 3) / 4; i += kThreads) reinterpret_cast<u32x4*>(mark)[i] = u32x4{};
    __syncthreads();
    each_page(p.c.table, N, p.c.B, M, wave, [](int b) { return b; }, [&](int) { return M; },
              [&](int page, int, int) { mark[page] = 1; });
    __syncthreads();
    bits_of(mark, N, held, wave);
    __syncthreads();
    int used;
    const uint32_t h = tid < W ? held[tid] : 0u;
    const int before = block_scan(__popc(h), s_wave, &used);
    for (int i = tid; i <= W; i += kThreads) rank[i] = i < W ? before : used;   // W <= kThreads
    if (tid == 0) held[W] = 0;
    __syncthreads();
    // held pages before page `used`: those that stay (word W, past the last, holds none)
    const int stay = rank[used >> 5] + __popc(held[used >> 5] & ((1u << (used & 31)) - 1u));
    if (tid < W) {
        const int first = 32 * tid;
        // holes below `used` and held pages from there on: a word has few of either
        const uint32_t all = first + 32 <= N ? ~0u : (1u << (N - first)) - 1u;
        const uint32_t low = first + 32 <= used ? ~0u : first >= used ? 0u : (1u << (used - first)) - 1u;
        for (uint32_t m = ~h & all & low; m; m &= m - 1) {
            const int k = __ffs(m) - 1;
            list[first + k - before - __popc(h & ((1u << k) - 1u))] = first + k;
        }
        int n = before + __popc(h & low) - stay;
        for (uint32_t m = h & ~low; m; m &= m - 1) from[n++] = first + __ffs(m) - 1;
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) *p.count = used;
    for (int e = blockIdx.x + gridDim.x * tid; e < p.c.B * M; e += gridDim.x * kThreads) {
        int page = p.c.table[e];
        if ((uint32_t)page >= (uint32_t)N) page = -1;
        else if (page >= used) page = list[rank[page >> 5] + __popc(held[page >> 5] & ((1u << (page & 31)) - 1u)) - stay];
        p.new_table[e] = page;
    }
    const int pieces = copy_pieces(p);
    const int64_t items = (int64_t)(used - stay) * 2 * p.L * pieces;
    for (int64_t it = blockIdx.x + gridDim.x * (tid >> 8); it < items; it += gridDim.x * (kThreads >> 8))
        copy_item<256>(p, it, pieces, tid & 255, [&](int i) { return make_int4(from[i], list[i], 0, 0); });
}

bool once(int64_t n_pages, int64_t n_rows, int64_t rows, int64_t max_pages) {
    return n_pages <= kOncePages && n_rows <= kOnceRows && rows * max_pages <= kOnceEntries;
}

hipError_t launch_once(const PagesProblem& p, hipStream_t stream) {
    if (p.n_rows) k_pages_reorder<<<kOnceGrid, kThreads, 0, stream>>>(p);
    else k_pages_compact<<<kOnceGrid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t pages_apply(const PagesProblem& p, const PagesWs& w, hipStream_t stream) {
    const int64_t entries = (int64_t)(p.n_rows ? p.n_rows : p.c.B) * p.c.max_pages;
    const int tables = (int)((entries + 255) / 256);
    k_pages_apply<<<tables + 2048, 256, 0, stream>>>(p, w, tables);
    return hipGetLastError();
}

hipError_t pages_mark(const PagesProblem& p, const PagesWs& w, hipStream_t stream) {
    const int W = (p.c.n_pages + 31) / 32, clear = p.n_rows ? p.c.n_pages : W;
    k_pages_clear<<<(clear + 255) / 256, 256, 0, stream>>>(p, w);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_pages_mark<<<dim3((p.c.max_pages + 255) / 256, p.n_rows ? p.n_rows : p.c.B), 256, 0, stream>>>(p, w);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const AppendProblem& p, bool bf16, hipStream_t stream) {
    return bf16 ? append_as<uint16_t>(p, stream) : append_as<float>(p, stream);
}

size_t pages_workspace_bytes(int64_t n_pages, int64_t n_rows, int64_t rows, int64_t max_pages) {
    return once(n_pages, n_rows, rows, max_pages) ? 0 : 4 * ws_words(n_pages, n_rows, nullptr, nullptr);
}

hipError_t launch_cache_reorder(const PagesProblem& p, hipStream_t stream) {
    if (once(p.c.n_pages, p.n_rows, p.n_rows ? p.n_rows : p.c.B, p.c.max_pages)) return launch_once(p, stream);
    PagesWs w;
    ws_words(p.c.n_pages, p.n_rows, p.ws, &w);
    hipError_t e = pages_mark(p, w, stream);
    if (e != hipSuccess) return e;
    k_pages_give<<<1, kThreads, 0, stream>>>(p, w);
    e = hipGetLastError();
    return e != hipSuccess ? e : pages_apply(p, w, stream);
}

hipError_t launch_cache_compact(const PagesProblem& p, hipStream_t stream) {
    if (once(p.c.n_pages, p.n_rows, p.n_rows ? p.n_rows : p.c.B, p.c.max_pages)) return launch_once(p, stream);
    PagesWs w;
    ws_words(p.c.n_pages, 0, p.ws, &w);
    hipError_t e = pages_mark(p, w, stream);
    if (e != hipSuccess) return e;
    k_pages_squeeze<<<1, kThreads, 0, stream>>>(p, w);
    e = hipGetLastError();
    return e != hipSuccess ? e : pages_apply(p, w, stream);
}

}  // namespace mot
