// fp32 attention of new tokens over the paged cache (paged_attn_device.h says what a
// workgroup computes): tiles of 16 query rows; the four waves take blocks of 32
// positions in turn, each with its own tiles and no barrier, and are joined through LDS at
// the end.  On v_mfma_f32_16x16x4_f32: exact fp32 products, at a sixteenth of the rate of the
// bf16 ones (as many cycles for a sixteenth of the work).
//
// Bound: latency for short contexts (3 x 64 tokens of 12 heads of 64 over 333 positions:
// 9.5 us; tiles of 32 rows gave it too few workgroups, 24.7 us).  Long ones reach 40 to 55 %
// of a large product's rate (500 tokens of 12 heads of 128 over 2000: 98 us, 55 TFLOP/s; 1024
// over 4096 301 us, 75): at D = 128 the 131 KB of LDS leave one workgroup to a CU and one wave to a
// SIMD, whose products, softmax and masks follow one another, and K and V come again for
// every 16 rows.
#include "paged_attn_device.h"

namespace mot {

namespace {

// D(16x16) += A(16x4) * B(4x16), fp32: lane l holds A row (l % 16), k = l / 16; B
// column (l % 16), the same k; D column (l % 16), rows 4 * (l / 16) + j at element j.
__device__ __forceinline__ f32x4 mfma_16x16x4(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// The order of the contraction is free as long as both operands keep it: step (s, j)
// of K . Q^T takes d = 16 s + 4 k + j, so that a lane's four steps are one 16-byte
// read; step j of V^T . P^T takes position 4 k + j, where the scores already lie.
// grid as k_paged_chunk
template <int D, int N>
__global__ __launch_bounds__(256, 2) void k_paged_f32(AttendProblem p, int tiles) {
    constexpr int NW = 4, DC = D / 4, TILE = 32 * DC;   // 16-byte chunks of a row, of 32 rows
    constexpr int RPL = 64 / DC, NL = 32 / RPL;         // rows per wave load, loads per tile
    constexpr int CPT = DC / 16;                        // chunks of four floats per thread of the join
    // K and V tiles per wave, (base, sum) per wave and row, a flag
    __shared__ f32x4 s_lds[NW * (2 * TILE + 8) + 1];
    float2* s_ml = reinterpret_cast<float2*>(s_lds + NW * 2 * TILE);   // [NW][16]
    int* s_bad = reinterpret_cast<int*>(s_lds + NW * (2 * TILE + 8));
    Work wk;
    if constexpr (N > 0) {
        if (!shared_work<N>(p, 16, 32, tiles > 1, wk)) return;   // uniform over the workgroup
    } else {
        if (!own_work(p, 16, 32, tiles, wk)) return;
    }
    const int b = wk.b, kvh = wk.kvh, G = p.H_q / p.c.H_kv;
    const NewTokens nt = wk.nt;
    const Tile tl = tile_of(p, nt, wk.tile, 16);
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g4 = lane >> 4, lrow = lane / DC, lch = lane % DC;
    auto kswz = [](int row) { return row & 15; };
    auto vswz = [](int row) { return 4 * ((row >> 2) & 3); };
    f32x4* Kt = s_lds + w * 2 * TILE;   // row r: chunk c at c ^ kswz(r)
    f32x4* Vt = Kt + TILE;              // row r: chunk c at c ^ vswz(r)
    uint32_t koff[NL], voff[NL];        // byte offsets within a group's buffer
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int r = i * RPL + lrow;
        koff[i] = ((uint32_t)(r & 15) * p.c.ts + 4 * (lch ^ kswz(r))) * 4;
        voff[i] = ((uint32_t)(r & 15) * p.c.ts + 4 * (lch ^ vswz(r))) * 4;
    }
    // this lane's query row
    const int row0 = tl.r0 + l16, rq = min(row0, tl.n_rows - 1), tok = rq / G, head = kvh * G + rq - tok * G;
    f32x4 qop[D / 16];
    {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const float* row = reinterpret_cast<const float*>(p.q) + row_offset(p.c, p.qs, nt, b, tok) + head * p.qs.head + 4 * g4;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qop[s] = row0 < tl.n_rows ? *reinterpret_cast<const f32x4*>(row + 16 * s) : zero;
    }
    const int u = tl.u0 + tok, ulo = low_of(p, u), tokens = tl.t1 - tl.t0 + 1;
    const bool cut = wk.parts > 1;

    // pass 0: all tokens; later passes, where that was not finite: one token each
    for (int pass = tokens > 1 ? 0 : 1; pass <= tokens; ++pass) {
        const int only = pass - 1 + tl.t0;
        const bool exact = pass > 0;   // positions below `lo` read as zeros
        const int lo = max(exact ? low_of(p, tl.u0 + only) : tl.lo, wk.lo);
        const int hi = min(exact ? max(tl.u0 + only + 1, 0) : tl.hi, wk.hi);
        f32x4 acc[D / 16];
#pragma unroll
        for (int db = 0; db < D / 16; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
        float mo = -INFINITY, l = 0.f;
        Groups gr;
        gr.base = 0; gr.page = -1; gr.ok = 0;
        GroupRows rows[2];   // of the block loaded last
        auto load = [&](int kb, const void* pool, const uint32_t (&off)[NL], f32x4* tile) {
            const rsrc_t r0 = group_rsrc<float>(pool, rows[0]), r1 = group_rsrc<float>(pool, rows[1]);
            u32x4* to = reinterpret_cast<u32x4*>(tile);
            if (exact && kb < lo) {   // uniform
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    load_lds16(i * RPL < 16 ? r0 : r1, kb + i * RPL + lrow < lo ? kPastEnd : off[i], to + i * 64);
            } else {
#pragma unroll
                for (int i = 0; i < NL; ++i) load_lds16(i * RPL < 16 ? r0 : r1, off[i], to + i * 64);
            }
        };
        auto load_k = [&](int kb) {
            rows[0] = group_rows<float, D>(p, gr, kb >> 4, kvh, hi);
            rows[1] = group_rows<float, D>(p, gr, (kb >> 4) + 1, kvh, hi);
            load(kb, p.k, koff, Kt);
        };
        int kb = (lo & ~31) + 32 * w;
        __builtin_amdgcn_s_waitcnt(0x70);   // vmcnt(0) lgkmcnt(0): the waits below count loads into LDS only
        uint32_t ok = 0, oknext = 0;        // groups of the block in no hole
        if (kb < hi) {
            gr.load(p, b, kb >> 4);
            oknext = (uint32_t)gr.ok & 3u;
            load_k(kb);
            load(kb, p.v, voff, Vt);
        }
        for (; kb < hi; kb += 32 * NW) {
            ok = oknext;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");   // K of this block
            f32x4 sc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                f32x4 a[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) a[h] = Kt[(16 * h + l16) * DC + ((4 * s + g4) ^ kswz(l16))];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) sc[h] = mfma_16x16x4(a[h][j], qop[s][j], sc[h]);
            }
            const int nx = kb + 32 * NW;
            const bool more = nx < hi;   // uniform
            wave_lds_sync();             // the operands are read: the next K may land
            if (more) {
                if ((nx >> 4) - gr.base > 62) gr.load(p, b, nx >> 4);
                oknext = (uint32_t)(gr.ok >> ((nx >> 4) - gr.base)) & 3u;
                load_k(nx);
            }
            float cm = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int v = kb + 16 * h + 4 * g4 + j;
                    sc[h][j] = v <= u && v >= ulo && v >= lo && v < hi && ((ok >> h) & 1u) ? sc[h][j] : -INFINITY;
                    cm = fmaxf(cm, sc[h][j]);
                }
            cm = fmaxf(cm, __shfl_xor(cm, 16, 64));
            cm = fmaxf(cm, __shfl_xor(cm, 32, 64));
            const float top = cm * p.scale_log2;
            if (__builtin_amdgcn_ballot_w64(top > mo + kSlack)) {
                const float mon = fmaxf(mo, top), alpha = __builtin_amdgcn_exp2f(mo - base_of(mon));
                l *= alpha;
#pragma unroll
                for (int db = 0; db < D / 16; ++db)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[db][j] *= alpha;
                mo = mon;
            }
            const float off = base_of(mo);
            float rs = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sc[h][j] = __builtin_amdgcn_exp2f(fmaf(sc[h][j], p.scale_log2, -off));
                    rs += sc[h][j];
                }
            rs += __shfl_xor(rs, 16, 64);
            rs += __shfl_xor(rs, 32, 64);
            l += rs;
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");   // V of this block
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const float* Vf = reinterpret_cast<const float*>(Vt);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int db = 0; db < D / 16; ++db)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int row = 16 * h + 4 * g4 + j;
                        acc[db] = mfma_16x16x4(Vf[row * D + (((4 * db + (l16 >> 2)) ^ vswz(row)) << 2) + (l16 & 3)], sc[h][j], acc[db]);
                    }
            wave_lds_sync();   // the V operands are read: the next V may land
            if (more) load(nx, p.v, voff, Vt);
        }
        mo = settled(p, b, mo, u, lo, hi, w, NW);
        // the waves' rows, joined through their tiles: row, chunk c of four floats at c ^ row
#pragma unroll
        for (int db = 0; db < D / 16; ++db) Kt[l16 * DC + ((4 * db + g4) ^ l16)] = acc[db];
        if (g4 == 0) s_ml[w * 16 + l16] = make_float2(mo, l);
        if (tid == 0) *s_bad = 0;
        __syncthreads();
        const int r = tid >> 4, c0 = (tid & 15) * CPT;   // sixteen threads per row
        float M = -INFINITY, sum = 0.f, wt[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) M = fmaxf(M, s_ml[i * 16 + r].x);
        const float off = base_of(M);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float2 ml = s_ml[i * 16 + r];
            wt[i] = __builtin_amdgcn_exp2f(ml.x - off);
            sum += ml.y * wt[i];
        }
        f32x4 o4[CPT];
        float t = 0.f;
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            o4[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const f32x4 y = s_lds[i * 2 * TILE + r * DC + ((c0 + c) ^ r)];
#pragma unroll
                for (int j = 0; j < 4; ++j) o4[c][j] += wt[i] * y[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) t = fmaf(o4[c][j], 0.f, t);
        }
        const int rg = tl.r0 + r, rt = rg / G;
        const bool store = rg < tl.n_rows && (!exact || rt == only);
        if (!exact) {
            if (store && t != t) *s_bad = 1;
            __syncthreads();
            const int bad = *s_bad;
            __syncthreads();   // the tiles and the flag may be written again
            if (bad) continue;
        }
        if (store) {
            float* o;
            float inv = 1.f;
            if (cut) {
                const Partial pt = partial_of(p, 16);
                const int64_t row = partial_row(pt, wk) + r;
                o = pt.rows + row * D;
                if (c0 == 0) pt.ml[row] = make_float2(M, sum);
            } else {
                o = reinterpret_cast<float*>(p.o) + row_offset(p.c, p.os, nt, b, rt) + (kvh * G + rg - rt * G) * p.os.head;
                inv = inverse_of(M, sum);
            }
#pragma unroll
            for (int c = 0; c < CPT; ++c) {
                f32x4 x = o4[c];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] *= inv;
                *reinterpret_cast<f32x4*>(o + 4 * (c0 + c)) = x;
            }
        }
        if (!exact || tokens == 1) break;
        __syncthreads();   // the tiles are read: the next token's may land
    }
    if constexpr (N > 0) leave_span(p, partial_of(p, 16), wk);
}

template <int D>
hipError_t launch_d(const AttendProblem& p, bool finds, hipStream_t stream) {
    const int tiles = div_up(p.c.max_new * (p.H_q / p.c.H_kv), 16);
    const AttendProblem s = shared_out(p);
    const int64_t grid = ((finds ? most_workgroups(s, 16) : (int64_t)p.c.B * p.c.H_kv * tiles) + 7) / 8 * 8;
    if (!finds) k_paged_f32<D, 0><<<(unsigned)grid, 256, 0, stream>>>(p, tiles);
    else if (p.c.B <= 64) k_paged_f32<D, 1><<<(unsigned)grid, 256, 0, stream>>>(s, tiles);
    else k_paged_f32<D, kSeqPerLane><<<(unsigned)grid, 256, 0, stream>>>(s, tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_f32(const AttendProblem& p, bool finds, hipStream_t stream) {
    return p.c.D == 128 ? launch_d<128>(p, finds, stream) : launch_d<64>(p, finds, stream);
}

}  // namespace mot
