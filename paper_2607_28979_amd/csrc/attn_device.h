// Device helpers of the attention kernels: buffer loads into LDS, LDS
// swizzles, transposing reads, work order over the XCDs.
#pragma once

#include "mot_device.h"

namespace mot {

constexpr float kLog2e = 1.4426950408889634f;

typedef __attribute__((address_space(3))) void lds_void;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

// Raw buffer over `bytes` bytes at `base` (reads past the end return 0).
__device__ __forceinline__ rsrc_t make_rsrc(const void* base, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0,
                                             (int)(bytes < 0xFFFFFFFFu ? bytes : 0xFFFFFFFFu), 0x00020000);
}

// 16 bytes per lane from the buffer straight into this wave's 1 KB of LDS
__device__ __forceinline__ void load_lds16(rsrc_t r, uint32_t off, u32x4* lds_dst_wave_base) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)lds_dst_wave_base, 16, off, 0, 0, 0);
}

// Workgroups are dispatched round-robin over the 8 XCDs, each with its own
// L2.  A grid of 8 * ceil(n / 8) workgroups is remapped so that XCD k walks
// the contiguous range [k * per, (k + 1) * per) of the n work items: items
// that share K/V rows (neighbouring positions, the heads of one KV group)
// meet in one L2.  Items >= n return at once.
__device__ __forceinline__ int xcd_item(int id, int n) { return (id & 7) * ((n + 7) >> 3) + (id >> 3); }
inline int xcd_grid(int n) { return 8 * ((n + 7) / 8); }

__device__ __forceinline__ void wave_lds_sync() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// LDS swizzle of a row of D bf16 (K rows: chunk c at c ^ causal_kswz(row))
template <int D>
__device__ __forceinline__ int causal_kswz(int r) {   // K rows: D/8 chunks
    return D == 128 ? (r & 15) : ((r >> 1) & 7);
}

// four bf16 of 16-byte chunk `at` (half 0 or 1) per lane, transposed within 16
// lanes: lane i's 8 bytes are row i / 4, columns 4 (i % 4) .. +3 of a 4 x 16
// block, and it gets column i of the four rows
__device__ __forceinline__ u32x2 read_tr16(const u32x4* at, int half) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const u32x2* q = reinterpret_cast<const u32x2*>(at) + half;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q));
}

}  // namespace mot
