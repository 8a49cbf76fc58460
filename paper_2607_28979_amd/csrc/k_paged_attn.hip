// Attention of new tokens over the paged cache: which kernel, how the work is cut, and
// the joining of what was cut.
#include "paged_attn_device.h"

namespace mot {

namespace {

// The partial sums of a cut (sequence, KV head), brought to one base and added, in the order
// of the parts within each of the groups of D / 4 threads, then of the groups: query head h
// of new token t of sequence b, by a workgroup.  Four parts' loads of every group are under
// way together: it is all latency (48 tokens of 28 heads over up to 8192 positions: 4.8 us;
// one token: 3.4).  rows: of a tile
template <typename T, int D>
__device__ __forceinline__ void join_row(const AttendProblem& p, int rows, int b, int t, int h, f32x4* s_acc, float2* s_ml) {
    constexpr int TH = D / 4, NG = 256 / TH;   // threads of a group, groups
    const int G = p.H_q / p.c.H_kv, kvh = h / G;
    const int c = threadIdx.x % TH, grp = threadIdx.x / TH;
    const Partial pt = partial_of(p, rows);
    const int2 span = pt.span[b * p.c.H_kv + kvh];
    const NewTokens nt = new_tokens(p.c, b);
    if (t >= nt.n) return;   // uniform over the workgroup
    const int r = t * G + h - kvh * G, tile = r / rows, tiles = div_up(nt.n * G, rows);
    // whole ones are done (uniform); starts that do not ascend may make more tiles than there are workgroups, and spans that
    // no one has left: nothing outside the partial tiles is read
    if (span.x < 0 || span.y < 2 || span.x + (int64_t)span.y * tiles > 2 * p.n_split) return;
    const int64_t at = (int64_t)(span.x + tile) * pt.R + r - tile * rows, step = (int64_t)tiles * pt.R;
    float M = -INFINITY, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int w0 = grp; w0 < span.y; w0 += 4 * NG) {
        float2 y[4];
        f32x4 z[4];
        float m = M;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = w0 + i * NG;
            y[i] = make_float2(-INFINITY, 0.f);
            z[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (w < span.y) {
                y[i] = pt.ml[at + w * step];
                z[i] = reinterpret_cast<const f32x4*>(pt.rows + (at + w * step) * D)[c];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, y[i].x);
        const float off = base_of(m), a = __builtin_amdgcn_exp2f(M - off);
        M = m;
        l *= a;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] *= a;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float wt = __builtin_amdgcn_exp2f(y[i].x - off);
            l += wt * y[i].y;
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] += wt * z[i][j];
        }
    }
    s_acc[threadIdx.x] = acc;
    if (c == 0) s_ml[grp] = make_float2(M, l);
    __syncthreads();
    if (grp) return;
    M = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) M = fmaxf(M, s_ml[i].x);
    const float off = base_of(M);
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        const float2 y = s_ml[i];
        const float wt = __builtin_amdgcn_exp2f(y.x - off);
        const f32x4 z = s_acc[i * TH + c];
        l += wt * y.y;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += wt * z[j];
    }
    const float inv = inverse_of(M, l);
    T* o = reinterpret_cast<T*>(p.o) + row_offset(p.c, p.os, nt, b, t) + h * p.os.head + 4 * c;
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x2*>(o) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
    else
        *reinterpret_cast<f32x4*>(o) = f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
}

// grid (max_new * H_q, B), or by_row (some rows * H_q) of packed tokens: the rows between the
// slice's first start and its last, whose sequences every wave finds among the starts.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_paged_join(AttendProblem p, int rows, bool by_row) {
    __shared__ f32x4 s_acc[256];
    __shared__ float2 s_ml[1024 / D];
    const int h = blockIdx.x % p.H_q, t = blockIdx.x / p.H_q;
    if (!by_row) {
        join_row<T, D>(p, rows, blockIdx.y, t, h, s_acc, s_ml);
        return;
    }
    const int lane = threadIdx.x & 63, end = min(p.c.start[p.c.B], p.c.n_new), step = gridDim.x / p.H_q;
    for (int row = max(p.c.start[0], 0) + t; row < end; row += step) {
        for (int b0 = 0; b0 < p.c.B; b0 += 64) {
            const NewTokens nt = new_tokens(p.c, min(b0 + lane, p.c.B - 1));
            const unsigned long long here = __builtin_amdgcn_ballot_w64(b0 + lane < p.c.B && row >= nt.row && row < nt.row + nt.n);
            if (!here) continue;   // uniform over the workgroup
            const int who = __builtin_ctzll(here);
            join_row<T, D>(p, rows, b0 + who, row - __builtin_amdgcn_readlane(nt.row, who), h, s_acc, s_ml);
            break;
        }
        __syncthreads();   // the sums are read: the next row's may be written
    }
}

// Rows of a tile: 32 where all of a sequence's fit, or an average one's do (packed tokens
// with a loose max_new), else 128; fp32 16.  With no max_new, 128 and 32 rows: 48 single
// tokens on 4000 114 and 89 us, 256 on 300 41 and 38, 32 x 4 on 2000 40 and 39, 47 and 100 of
// one sequence on 4000 101 and 106.
int tile_rows(const AttendProblem& p, bool bf16) {
    const int64_t G = p.H_q / p.c.H_kv;
    return !bf16 ? 16 : p.c.max_new * G <= 32 || p.c.n_new * G <= 32 * (int64_t)p.c.B ? 32 : 128;
}

}  // namespace

// When positions are cut, and over how many workgroups.  Cutting costs a second launch and
// 4 us or so of finding the parts and joining them, more with many rows; it saves
// the time that a long context takes a few workgroups.  28 heads on 4 of 128 unless said.
// Few rows, calls back to back, whole against cut: one sequence of 500 positions 8.7 /
// 13.0 us, 800 10.2 / 12.7, 1100 12.3 / 12.9, 1500 15.8 / 12.6; 32 of 1000 15.9 / 20.4; 48
// of up to 8192 69 / 53.  Tiles of 128 rows (replayed): 37 new tokens on 8000 171 / 29 us,
// 200 on 1000 29.7 / 28.5, 2 x 300 on 700 24 / 49, 2 x 500 alone 20 / 60, 16 x 20 on up to
// 6000 130 / 42, 1000 on 4000 93 / 120, 2 x 300 on 3000 with 16 heads of 64 53 / 42.  fp32: 12
// heads of 64, one token on 1000 19 / 11.2, 3 x 64 on 333 10.6 / 15.4, 40 ragged ones on up to
// 2000 46 / 44; 12 heads on 2 of 128, 500 tokens on 2000 105 / 97.
// Shares: 448, 7/8 of the workgroups that the chip holds at two per CU, since remainders add
// some: 30 ragged contexts on 2 heads 18.6 us with 448, 22.1 with 512 to 704.  bf16 at D = 64,
// three per CU: 704 of 768 (48 ragged contexts 20.3 us with 672 or 704, 20.0 with 448).  fp32 at
// D = 128 holds one per CU (131 KB of LDS) and still takes 448, since parts of several tiles
// do better in two rounds: 500 tokens on 2000 99 us and 3 x 64 on 2000 55, with 224 111 and 65; 40
// single ones on up to 2000 24.6 and 20.1.
size_t attend_plan(AttendProblem& p, bool bf16) {
    const int rows = tile_rows(p, bf16), step = rows == 128 ? 64 : 32, B = min(p.c.B, kMostSeq);
    p.n_split = 1;
    p.least = 4;   // blocks: one per wave, or four chunks
    // all tiles' blocks, whatever the lengths and starts hold
    const int64_t blocks = (((int64_t)p.c.max_pages << p.c.page_shift) + step - 1) / step + 1;
    const int64_t tiles = ((int64_t)p.c.max_new * (p.H_q / p.c.H_kv) + rows - 1) / rows;
    p.wide = (double)B * p.c.H_kv * tiles * blocks > 1 << 30;
    const int64_t whole = most_workgroups(p, rows) - 1;   // workgroups of the call uncut
    if (rows == 32 ? p.max_kv <= 1024 : rows == 128 ? whole >= 192 || p.max_kv <= 512 + 8 * whole
                                                    : whole >= 512 || p.max_kv <= 512) return 0;
    // nor are calls whose rows are too many for the joining launch
    const bool by_row = (int64_t)p.c.max_new * B > 2 * (int64_t)p.c.n_new;
    if ((int64_t)(by_row ? max(p.c.n_new, p.c.max_new) : p.c.max_new) * p.H_q > kMostWorkgroups) return 0;
    p.n_split = !bf16 || p.c.D == 128 ? 448 : 704;
    const size_t R = (size_t)partial_of(p, rows).R;
    return 2 * p.n_split * R * (p.c.D + 2) * sizeof(float) + (size_t)B * p.c.H_kv * sizeof(int2);
}

namespace {

// slices: of the call
hipError_t launch_slice(const AttendProblem& p, bool bf16, int rows, bool finds, int slices, hipStream_t stream) {
    hipError_t e = rows == 32 ? launch_paged_decode(p, finds, stream)
                   : bf16     ? launch_paged_chunk(p, finds, stream)
                              : launch_paged_f32(p, finds, stream);
    if (e != hipSuccess || !p.part) return e;
    const bool by_row = p.c.start && (int64_t)p.c.max_new * p.c.B > 2 * (int64_t)p.c.n_new;
    // packed rows: a slice's share of the call's, and its workgroups walk further where it has more
    // (4096 single tokens without a bound, one on 9000 positions: 803 us; every slice with a
    // workgroup for every row of the call 1680)
    const dim3 join((by_row ? div_up(p.c.n_new, slices) : p.c.max_new) * p.H_q, by_row ? 1 : p.c.B);
    if (bf16 && p.c.D == 128) k_paged_join<uint16_t, 128><<<join, 256, 0, stream>>>(p, rows, by_row);
    else if (bf16) k_paged_join<uint16_t, 64><<<join, 256, 0, stream>>>(p, rows, by_row);
    else if (p.c.D == 128) k_paged_join<float, 128><<<join, 256, 0, stream>>>(p, rows, by_row);
    else k_paged_join<float, 64><<<join, 256, 0, stream>>>(p, rows, by_row);
    return hipGetLastError();
}

}  // namespace

bool attend_fits(const AttendProblem& p, bool bf16) {
    const int rows = tile_rows(p, bf16);
    if (!finds_work(p, rows)) return own_tiles(p, rows) <= kMostWorkgroups;
    AttendProblem s = shared_out(p);
    s.c.B = min(p.c.B, kMostSeq);
    return most_workgroups(s, rows) <= kMostWorkgroups;
}

// Workgroups that find their work add up as many sequences at a time as fit in a wave's
// lanes; the slices share the workspace, one after the other.  599 single tokens on 300
// positions and one on 30000: 396 us whole, 136 so.  Where each has a tile of its own, all
// sequences are one launch: 4096 single tokens on 100 positions 224 us, in slices 251.
hipError_t launch_paged_attention(const AttendProblem& p, bool bf16, hipStream_t stream) {
    const int rows = tile_rows(p, bf16);
    const bool finds = finds_work(p, rows);
    const int most = finds ? kMostSeq : min(p.c.B, (int)(kMostWorkgroups / own_tiles(p, rows)));
    for (int b0 = 0; b0 < p.c.B; b0 += most) {
        AttendProblem s = p;
        s.c.B = min(p.c.B - b0, most);
        s.c.table += (int64_t)b0 * p.c.max_pages;
        s.c.kv_len += b0;
        if (p.c.start) {
            s.c.start += b0;
        } else {
            const int64_t bytes = b0 * (bf16 ? 2 : 4);
            s.q = reinterpret_cast<const char*>(p.q) + bytes * p.qs.batch;
            s.o = reinterpret_cast<char*>(p.o) + bytes * p.os.batch;
            s.c.n_new = s.c.B * p.c.max_new;
        }
        const hipError_t e = launch_slice(s, bf16, rows, finds, div_up(p.c.B, most), stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace mot
