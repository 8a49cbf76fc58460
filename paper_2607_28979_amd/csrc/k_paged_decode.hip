// Attention of few new tokens (decoding) over the paged cache: tiles of 32 rows, which
// hold all rows of one KV head of most sequences (paged_attn_device.h says what a workgroup
// computes).
//
// The waves of a workgroup take blocks of 32 positions in turn, each with its own
// tiles and no barrier, and are joined through LDS at the end: K of the next block lands
// during this one's softmax, V after its second product.
//
// Bound: memory where contexts are long (48 sequences of 205 to 8192 positions, 4 KV heads
// of 128, 207 MB: 47 us, 4.4 TB/s where a copy reaches 5.2), latency where they are short
// (one of 1100: 8 us, and 3 of joining its parts).  The work is shared out (cut) rather
// than a workgroup given to each sequence and KV head, since the longest sequence would
// hold the call up: 104 us for the 48.  V read through the transposing LDS read with its own
// wait: 63 -> 52 us (with the join).  Eight waves where there is a CU for every workgroup and nothing to
// cut, four else: eight leave room for one workgroup per CU only.
//
// The probabilities go into the second product as two bf16 terms, a product each: the matrix
// unit is 7 % busy, and the error against 64 bits falls from 2.25e-3 to 1.66e-3 of the result,
// which is the rounding of the result alone (the 48 sequences: 51.2 -> 52.2 us with the join,
// one of 1100 10.4 -> 10.6; 48 of 2 heads of 64 19.7 -> 20.0).
#include "paged_attn_device.h"

namespace mot {

namespace {

// NW waves.  N: sequences per lane of the shared work (grid most_workgroups), 0: nothing
// shared, and a tile to a sequence (grid B * H_kv)
template <int D, int NW, int N>
__global__ __launch_bounds__(64 * NW, 2) void k_paged_decode(AttendProblem p) {
    constexpr int DC = D / 8, TILE = 32 * DC;        // 16-byte chunks of a row, of 32 rows
    constexpr int RPL = 64 / DC, NL = 32 / RPL;      // rows per wave load, loads per tile
    constexpr int TPR = 2 * NW, CPT = D / 4 / TPR;   // threads per row of the join, chunks of four floats per thread
    // K and V tiles per wave, (maximum, sum) per wave and row, a flag
    __shared__ u32x4 s_lds[NW * (2 * TILE + 16) + 1];
    float2* s_ml = reinterpret_cast<float2*>(s_lds + NW * 2 * TILE);   // [NW][32]
    int* s_bad = reinterpret_cast<int*>(s_lds + NW * (2 * TILE + 16));
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = p.H_q / p.c.H_kv;
    Work wk;
    Groups gr;
    gr.base = -1;
    if constexpr (N > 0) {
        if (!shared_work<N>(p, 32, 32, false, wk)) return;   // uniform over the workgroup
    } else {
        const int group = blockIdx.x;
        gr.fetch(p, group / p.c.H_kv, 2 * w);   // beside the lengths: with no window it is where this wave starts
        if (!own_work(p, 32, 32, 1, wk)) return;
        gr.ready(p);
    }
    const int b = wk.b, kvh = wk.kvh;
    const NewTokens nt = wk.nt;

    const int l32 = lane & 31, g = lane >> 5, lrow = lane / DC, lch = lane % DC;
    const int l16 = lane & 15, vrow = 4 * g + (l16 >> 2), vch = 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1);
    auto vswz = [](int r) { return v_swizzle<D>(r); };
    u32x4* Kt = s_lds + w * 2 * TILE;   // row r: chunk c at c ^ causal_kswz(r)
    u32x4* Vt = Kt + TILE;              // row r: chunk c at c ^ vswz(r)
    uint32_t koff[NL], voff[NL];        // byte offsets within a group's buffer
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int r = i * RPL + lrow;
        koff[i] = ((uint32_t)(r & 15) * p.c.ts + 8 * (lch ^ causal_kswz<D>(r))) * 2;
        voff[i] = ((uint32_t)(r & 15) * p.c.ts + 8 * (lch ^ vswz(r))) * 2;
    }
    uint32_t vat[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) vat[db] = lds_address(Vt + vrow * DC + ((4 * db + vch) ^ vswz(vrow))) + 8 * (l16 & 1);

    const Tile tl = tile_of(p, nt, N > 0 ? wk.tile : 0, 32);
    const bool cut = wk.parts > 1;
    // this lane's query row
    const bool row_ok = tl.r0 + l32 < tl.n_rows;
    const int rq = min(tl.r0 + l32, tl.n_rows - 1), tok = rq / G, head = kvh * G + rq - tok * G;
    u32x4 qop[D / 16];
    {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        const uint16_t* row = reinterpret_cast<const uint16_t*>(p.q) + row_offset(p.c, p.qs, nt, b, tok) + head * p.qs.head + 8 * g;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qop[ks] = row_ok ? *reinterpret_cast<const u32x4*>(row + 16 * ks) : zero;
    }
    const int u = tl.u0 + tok, ulo = low_of(p, u);
    const int tokens = tl.t1 - tl.t0 + 1;
    const bool one = tokens == 1;

    // pass 0: all tokens; later passes, where that was not finite: one token each
    for (int pass = one ? 1 : 0; pass <= tokens; ++pass) {
        const int only = tl.t0 + pass - 1;        // token of an exact pass
        const bool exact = pass > 0;              // positions below `lo` read as zeros
        const int lo = max(exact ? low_of(p, tl.u0 + only) : tl.lo, wk.lo);
        const int hi = min(exact ? max(tl.u0 + only + 1, 0) : tl.hi, wk.hi);
        f32x16 acc[D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;
        float mo = -INFINITY, l = 0.f;
        GroupRows rows[2];   // of the block loaded last
        auto load = [&](int kb, const void* pool, const uint32_t (&off)[NL], u32x4* tile) {
            const rsrc_t r0 = group_rsrc<uint16_t>(pool, rows[0]), r1 = group_rsrc<uint16_t>(pool, rows[1]);
            if (exact && kb < lo) {   // uniform
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    load_lds16(i * RPL < 16 ? r0 : r1, kb + i * RPL + lrow < lo ? kPastEnd : off[i], tile + i * 64);
            } else {
#pragma unroll
                for (int i = 0; i < NL; ++i) load_lds16(i * RPL < 16 ? r0 : r1, off[i], tile + i * 64);
            }
        };
        auto load_k = [&](int kb) {
            rows[0] = group_rows<uint16_t, D>(p, gr, kb >> 4, kvh, hi);
            rows[1] = group_rows<uint16_t, D>(p, gr, (kb >> 4) + 1, kvh, hi);
            load(kb, p.k, koff, Kt);
        };
        auto load_v = [&](int kb) { load(kb, p.v, voff, Vt); };
        int kb = (lo & ~31) + 32 * w;
        __builtin_amdgcn_s_waitcnt(0x70);   // vmcnt(0) lgkmcnt(0): the waits below count loads into LDS only
        uint32_t okb = 0, oknext = 0;   // groups of the block in no hole
        if (kb < hi) {
            if (pass > 1 || gr.base != kb >> 4) gr.load(p, b, kb >> 4);
            oknext = (uint32_t)gr.ok & 3u;
            load_k(kb);
            load_v(kb);
        }
        for (; kb < hi; kb += 32 * NW) {
            okb = oknext;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");   // K of this block
            f32x16 sc;
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                sc = mfma_32x32x16(Kt[l32 * DC + ((2 * ks + g) ^ causal_kswz<D>(l32))], qop[ks], sc);
            const int nx = kb + 32 * NW;
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
            if (kb < lo || kb + 31 > tl.u0 + (exact ? only : tl.t0) || okb != 3u || p.window > 0) {
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
            const float top = cm * p.scale_log2;
            if (__builtin_amdgcn_ballot_w64(top > mo + kSlack)) {
                const float mon = fmaxf(mo, top), alpha = __builtin_amdgcn_exp2f(mo - base_of(mon));
                l *= alpha;
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[db][e] *= alpha;
                mo = mon;
            }
            const float off = base_of(mo);
            float rs = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sc[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], p.scale_log2, -off));
                rs += sc[e];
            }
            rs += __shfl_xor(rs, 32, 64);
            l += rs;
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");   // V of this block
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            auto step = [&](auto s_) {
                constexpr int s = decltype(s_)::value;
                u32x2 va[D / 16];
                read_vt<D, s * 16 * D * 2>(vat, va);
                u32x4 hi, lo;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x2 t = split_bf16x2(sc[8 * s + 2 * i], sc[8 * s + 2 * i + 1]);
                    hi[i] = t.x;
                    lo[i] = t.y;
                }
#pragma unroll
                for (int db = 0; db < D / 32; ++db) {
                    const u32x4 vt = {va[2 * db].x, va[2 * db].y, va[2 * db + 1].x, va[2 * db + 1].y};
                    acc[db] = mfma_32x32x16(vt, lo, acc[db]);
                    acc[db] = mfma_32x32x16(vt, hi, acc[db]);
                }
            };
            step(Step<0>{});
            step(Step<1>{});
            if (more) load_v(nx);   // the V operands are read
        }
        mo = settled(p, b, mo, u, lo, hi, w, NW);
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
        const int r = tid / TPR, c0 = tid % TPR * CPT;
        float M = -INFINITY, sum = 0.f, wt[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) M = fmaxf(M, s_ml[i * 32 + r].x);
        const float off = base_of(M);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float2 ml = s_ml[i * 32 + r];
            wt[i] = __builtin_amdgcn_exp2f(ml.x - off);
            sum += ml.y * wt[i];
        }
        f32x4 o4[CPT];
        float t = 0.f;
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            const int at = r * (D / 4) + ((c0 + c) ^ (r & (D / 4 - 1)));
            o4[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const f32x4 y = reinterpret_cast<const f32x4*>(s_lds + i * 2 * TILE)[at];
#pragma unroll
                for (int j = 0; j < 4; ++j) o4[c][j] += wt[i] * y[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) t = fmaf(o4[c][j], 0.f, t);
        }
        const int rr = tl.r0 + r, rt = rr / G;
        const bool store = rr < tl.n_rows && (!exact || rt == only);
        if (!exact) {
            if (store && t != t) *s_bad = 1;
            __syncthreads();
            const int bad = *s_bad;
            __syncthreads();   // the tiles and the flag may be written again
            if (bad) continue;
        }
        if (store) {
            const int hh = kvh * G + rr - rt * G;
            if (cut) {
                const Partial pt = partial_of(p, 32);
                const int64_t row = partial_row(pt, wk) + r;
                f32x4* o = reinterpret_cast<f32x4*>(pt.rows + row * D) + c0;
#pragma unroll
                for (int c = 0; c < CPT; ++c) o[c] = o4[c];
                if (c0 == 0) pt.ml[row] = make_float2(M, sum);
            } else {
                const float inv = inverse_of(M, sum);
                uint16_t* o = reinterpret_cast<uint16_t*>(p.o) + row_offset(p.c, p.os, nt, b, rt) + hh * p.os.head + 4 * c0;
#pragma unroll
                for (int c = 0; c < CPT; ++c)
                    reinterpret_cast<u32x2*>(o)[c] = u32x2{pack_bf16x2(o4[c][0] * inv, o4[c][1] * inv), pack_bf16x2(o4[c][2] * inv, o4[c][3] * inv)};
            }
        }
        if (!exact || one) break;
        __syncthreads();   // the tiles are read: the next token's may land
    }
    if constexpr (N > 0) leave_span(p, partial_of(p, 32), wk);
}

template <int D>
hipError_t launch_d(const AttendProblem& p, bool finds, hipStream_t stream) {
    const int whole = p.c.B * p.c.H_kv;
    if (finds) {
        const AttendProblem s = shared_out(p);
        const int64_t grid = most_workgroups(s, 32);
        if (p.c.B <= 64 && !p.part && grid <= 256) k_paged_decode<D, 8, 1><<<(unsigned)grid, 512, 0, stream>>>(s);
        else if (p.c.B <= 64) k_paged_decode<D, 4, 1><<<(unsigned)grid, 256, 0, stream>>>(s);
        else k_paged_decode<D, 4, kSeqPerLane><<<(unsigned)grid, 256, 0, stream>>>(s);
    } else if (whole <= 256) {   // a CU for each: more waves
        k_paged_decode<D, 8, 0><<<whole, 512, 0, stream>>>(p);
    } else {
        k_paged_decode<D, 4, 0><<<whole, 256, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_decode(const AttendProblem& p, bool finds, hipStream_t stream) {
    return p.c.D == 128 ? launch_d<128>(p, finds, stream) : launch_d<64>(p, finds, stream);
}

}  // namespace mot
