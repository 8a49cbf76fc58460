// Attention of new tokens over the paged cache.
#include "attn_device.h"
#include "cache_internal.h"

namespace mot {

namespace {

__device__ __forceinline__ float as_float(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }

// One wave per (token, query head): a key at a time, its D products summed over
// the lanes, running maximum and sum.  grid (ceil(max_new * H_q / 4), B), 256 threads
template <typename T, int D>
__global__ __launch_bounds__(256) void k_paged_rows(AttendProblem p) {
    constexpr int N = D / 64;
    const int b = blockIdx.y, lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    const NewTokens nt = new_tokens(p.c, b);
    const int i = r / p.H_q, h = r - i * p.H_q;
    if (i >= nt.n) return;
    const int u = nt.kv - nt.count + i, kvh = h / (p.H_q / p.c.H_kv);
    const T* q = reinterpret_cast<const T*>(p.q) + row_offset(p.c, p.qs, nt, b, i) + h * p.qs.head;
    float x[N], acc[N], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        x[j] = as_float(q[lane + 64 * j]);
        acc[j] = 0.f;
    }
    for (int v = p.window > 0 ? max(0, u - p.window + 1) : 0; v <= u; ++v) {
        const int page = p.c.table[(int64_t)b * p.c.max_pages + (v >> p.c.page_shift)];
        if (page < 0 || page >= p.c.n_pages) continue;
        const int64_t at = page * p.c.page_elems + (int64_t)(v & ((1 << p.c.page_shift) - 1)) * p.c.ts + (int64_t)kvh * p.c.hs;
        const T* k = reinterpret_cast<const T*>(p.k) + at;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) s += x[j] * as_float(k[lane + 64 * j]);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
        s *= p.scale_log2;
        const float mn = fmaxf(m, s), a = exp2f(m - mn), e = exp2f(s - mn);
        m = mn;
        l = l * a + e;
        const T* val = reinterpret_cast<const T*>(p.v) + at;
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] = acc[j] * a + e * as_float(val[lane + 64 * j]);
    }
    T* o = reinterpret_cast<T*>(p.o) + row_offset(p.c, p.os, nt, b, i) + h * p.os.head;
#pragma unroll
    for (int j = 0; j < N; ++j) put(o + lane + 64 * j, l != 0.f ? acc[j] / l : 0.f);
}

}  // namespace

void attend_cuts(AttendProblem& p, bool bf16) {
    p.n_split = 1;
    p.split_len = p.max_kv;
}

size_t attend_part_bytes(const AttendProblem& p) { return 0; }

hipError_t launch_paged_attention(const AttendProblem& p, bool bf16, hipStream_t stream) {
    const dim3 grid((unsigned)(((int64_t)p.c.max_new * p.H_q + 3) / 4), p.c.B);
    if (bf16) {
        if (p.c.D == 128) k_paged_rows<uint16_t, 128><<<grid, 256, 0, stream>>>(p);
        else k_paged_rows<uint16_t, 64><<<grid, 256, 0, stream>>>(p);
    } else {
        if (p.c.D == 128) k_paged_rows<float, 128><<<grid, 256, 0, stream>>>(p);
        else k_paged_rows<float, 64><<<grid, 256, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace mot
