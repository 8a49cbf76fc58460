// Attention of many new tokens over the paged cache (paged_attn_device.h says what a
// workgroup computes): tiles of 128 query rows, 32 per wave, over shared chunks of 64
// positions, the next chunk landing in LDS while this one is used.
//
// Bound: issue. A wave's chunk is 32 matrix products (1024 cycles of its SIMD's matrix unit)
// and about 850 cycles of softmax on the vector unit, of which 512 are the exponentials;
// two workgroups share a CU, and what overlaps is one's products with the other's softmax.
// 2 x 2048 tokens of 28 heads, head size 128, over contexts of 8192: 403 to 436 us by the card, 0.97
// to 1.04 PFLOP/s (a plain 8192^3 bf16 product reaches 1.21). What led there from 562: operands of both
// products read ahead (541), a base that rarely moves (509), V rows swizzled for the
// transposed reads (501), neighbouring tiles on one XCD (469; 490 on the card of the next figures), wave
// priority to the products (475), no lane waiting for its row's other lane (443), row sums
// by two-element dot products (436), V of a whole chunk read at once (429).
// Not kept: the next chunk's scores beside this one's softmax within a wave (it spills at
// two waves per SIMD, 1061; with one wave 628), in halves (559), priority by workgroup (447).
//
// The probabilities are rounded to bf16 for the second product, and a row's sum takes them as
// rounded, so that the weights add up to 1.  The error against 64 bits is 2.35e-3 of the result,
// 1.66e-3 of which is the result's own rounding.  As two bf16 terms, a product each, they would
// leave that alone, at 607 us instead of 413 (560 instead of 405 with every step's exponentials
// beside the products of the step before; 1000 tokens on 4000 positions 114 and 91, 6 x 37 on
// 4096 20.9 and 19.5): the products are what bounds this kernel.
#include "paged_attn_device.h"

namespace mot {

namespace {

// grid most_workgroups rounded up to 8, or own_work's (N = 0), 256 threads; `tiles` of a
// sequence at most
template <int D, int N>
__global__ __launch_bounds__(256, 2) void k_paged_chunk(AttendProblem p, int tiles) {
    constexpr int DC = D / 8, KS = 64 * DC;        // 16-byte slots of a K or V chunk
    constexpr int RPL = 64 / DC, NQ = 16 / RPL;    // rows per wave load, loads per wave and chunk
    // two stages of K rows (chunk c at c ^ causal_kswz(row)) and V rows (c ^ vswz(row)), one flag
    __shared__ u32x4 lds[4 * KS + 1];
    int* s_bad = reinterpret_cast<int*>(lds + 4 * KS);
    Work wk;
    if constexpr (N > 0) {
        if (!shared_work<N>(p, 128, 64, tiles > 1, wk)) return;   // uniform over the workgroup
    } else {
        if (!own_work(p, 128, 64, tiles, wk)) return;
    }
    const int b = wk.b, kvh = wk.kvh, G = p.H_q / p.c.H_kv;
    const NewTokens nt = wk.nt;
    const Tile tl = tile_of(p, nt, wk.tile, 128);
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5, lrow = lane / DC, lch = lane % DC;
    const int l16 = lane & 15, vrow = 4 * g + (l16 >> 2), vch = 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1);
    auto vswz = [](int r) { return v_swizzle<D>(r); };

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
    const bool cut = wk.parts > 1;
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
        const int lo = max(exact ? low_of(p, tl.u0 + only) : tl.lo, wk.lo);
        const int hi = min(exact ? max(tl.u0 + only + 1, 0) : tl.hi, wk.hi);
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
            const GroupRows rows = group_rows<uint16_t, D>(p, gr, gw, kvh, hi);
            const rsrc_t kr = group_rsrc<uint16_t>(p.k, rows), vr = group_rsrc<uint16_t>(p.v, rows);
            if (exact && kc < lo) {   // uniform
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const bool low = kc + 16 * w + q * RPL + lrow < lo;
                    load_lds16(kr, low ? kPastEnd : koff[q], kd + q * 64);
                    load_lds16(vr, low ? kPastEnd : voff[q], kd + KS + q * 64);
                }
            } else {
#pragma unroll
                for (int q = 0; q < NQ; ++q) load_lds16(kr, koff[q], kd + q * 64);
#pragma unroll
                for (int q = 0; q < NQ; ++q) load_lds16(vr, voff[q], kd + KS + q * 64);
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
                __builtin_amdgcn_s_setprio(1);   // products first: the other workgroup's waves do softmax meanwhile
                f32x16 sc[2];
                u32x4 ka[2][D / 16];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)
                        ka[kb][ks] = Kl[(kb * 32 + l32) * DC + ((2 * ks + g) ^ causal_kswz<D>(l32))];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[kb][e] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) sc[kb] = mfma_32x32x16(ka[kb][ks], qop[ks], sc[kb]);
                }
                // the first block's operands, then a read of the second's behind every product
                __builtin_amdgcn_sched_group_barrier(0x100, D / 16, 0);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, D / 16, 0);
                uint32_t at[D / 32];
#pragma unroll
                for (int db = 0; db < D / 32; ++db) at[db] = vat[db] + (uint32_t)st * (2 * KS * 16);
                u32x2 va[D / 8], vb[D / 8];
                read_vt2<D, 0>(at, va);   // while the products run
                read_vt2<D, 2 * 16 * D * 2>(at, vb);
                __builtin_amdgcn_s_setprio(0);
                if (masked) {
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int v = kc + kb * 32 + 8 * (e >> 2) + 4 * g + (e & 3);
                            sc[kb][e] = v <= u && v >= ulo && v >= lo && v < hi && ((ok >> (2 * kb + (e >> 3))) & 1u) ? sc[kb][e] : -INFINITY;
                        }
                }
                float cm = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) cm = fmaxf(cm, sc[kb][e]);
                // no lane waits for its row's other lane (base and row sum): they meet where the
                // base moves, and at the end
                if (__builtin_amdgcn_ballot_w64(cm * p.scale_log2 > mo + kSlack)) {
                    const float top = fmaxf(cm, __shfl_xor(cm, 32, 64)) * p.scale_log2;
                    const float mon = fmaxf(mo, top), alpha = __builtin_amdgcn_exp2f(mo - base_of(mon));
                    l *= alpha;
#pragma unroll
                    for (int db = 0; db < D / 32; ++db)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[db][e] *= alpha;
                    mo = mon;
                }
                const float off = base_of(mo);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[kb][e] = __builtin_amdgcn_exp2f(fmaf(sc[kb][e], p.scale_log2, -off));
                auto step = [&](int s, const u32x2* v) {
                    const int kb = s >> 1, e0 = 8 * (s & 1);
                    const u32x4 pf = {pack_bf16x2(sc[kb][e0], sc[kb][e0 + 1]), pack_bf16x2(sc[kb][e0 + 2], sc[kb][e0 + 3]),
                                      pack_bf16x2(sc[kb][e0 + 4], sc[kb][e0 + 5]), pack_bf16x2(sc[kb][e0 + 6], sc[kb][e0 + 7])};
#pragma unroll
                    for (int i = 0; i < 4; ++i) l = add_bf16x2(pf[i], l);
#pragma unroll
                    for (int db = 0; db < D / 32; ++db)
                        acc[db] = mfma_32x32x16(u32x4{v[2 * db].x, v[2 * db].y, v[2 * db + 1].x, v[2 * db + 1].y}, pf, acc[db]);
                };
                __builtin_amdgcn_s_setprio(1);
                step(0, va);
                step(1, va + D / 16);
                step(2, vb);
                step(3, vb + D / 16);
                __builtin_amdgcn_s_setprio(0);
            }
            barrier();   // the next chunk has landed; every wave is done with this one
        }
        l += __shfl_xor(l, 32, 64);
        if (wave_ok) mo = settled(p, b, mo, u, lo, hi, 0, 1);
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
            // opaque, so that addresses are not held through the loop above, which has every register
            int at = tok, h = head, x = r;
            asm volatile("" : "+v"(at), "+v"(h), "+v"(x));
            if (cut) {
                const Partial pt = partial_of(p, 128);
                const int64_t row = partial_row(pt, wk) + x - tl.r0;
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(pt.rows + row * D + 32 * db + 8 * i + 4 * g) =
                            f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]};
                if (g == 0) pt.ml[row] = make_float2(mo, l);
            } else {
                const float inv = inverse_of(mo, l);
                uint16_t* o = reinterpret_cast<uint16_t*>(p.o) + row_offset(p.c, p.os, nt, b, at) + h * p.os.head;
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
    if constexpr (N > 0) leave_span(p, partial_of(p, 128), wk);
}

template <int D>
hipError_t launch_d(const AttendProblem& p, bool finds, hipStream_t stream) {
    const int tiles = div_up(p.c.max_new * (p.H_q / p.c.H_kv), 128);
    const AttendProblem s = shared_out(p);
    const int64_t grid = ((finds ? most_workgroups(s, 128) : (int64_t)p.c.B * p.c.H_kv * tiles) + 7) / 8 * 8;
    if (!finds) k_paged_chunk<D, 0><<<(unsigned)grid, 256, 0, stream>>>(p, tiles);
    else if (p.c.B <= 64) k_paged_chunk<D, 1><<<(unsigned)grid, 256, 0, stream>>>(s, tiles);
    else k_paged_chunk<D, kSeqPerLane><<<(unsigned)grid, 256, 0, stream>>>(s, tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_chunk(const AttendProblem& p, bool finds, hipStream_t stream) {
    return p.c.D == 128 ? launch_d<128>(p, finds, stream) : launch_d<64>(p, finds, stream);
}

}  // namespace mot
