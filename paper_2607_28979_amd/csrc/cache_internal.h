// Launch descriptors of the paged cache's operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mot {

constexpr int kMostWorkgroups = (1 << 24) - 8;   // of 256 threads: a launch takes under 2^32 work items

// Pools and page table of one call (element = 2 or 4 bytes).
struct PageTable {
    const int32_t* table;    // [B][max_pages]
    const int32_t* kv_len;   // [B]
    const int32_t* start;    // [B + 1] or NULL
    int32_t B, max_pages, n_pages, page_shift;
    int32_t n_new, max_new;
    int32_t H_kv, D;
    int64_t page_elems;      // elements of a page
    int32_t ts, hs;          // elements between positions and between heads of a page
};

struct RowStrides {
    int64_t layer, batch, token, head;
};

// The new tokens of a sequence: rows at `row` (of the packed axis) or batch
// row b, `count` of them, `n` computed; the first is at position kv - count.
struct NewTokens {
    int32_t row, count, n, kv;
};
__device__ __forceinline__ NewTokens new_tokens(const PageTable& c, int b) {
    NewTokens t;
    const int64_t most = (int64_t)c.max_pages << c.page_shift;
    const int kv = c.kv_len[b];
    t.kv = kv < 0 ? 0 : kv > most ? (int)most : kv;
    if (c.start) {
        const int s = min(max(c.start[b], 0), c.n_new), e = min(max(c.start[b + 1], s), c.n_new);
        t.row = s;
        t.count = e - s;
    } else {
        t.row = 0;
        t.count = c.max_new;
    }
    t.n = min(t.count, c.max_new);
    return t;
}
__device__ __forceinline__ int64_t row_offset(const PageTable& c, const RowStrides& s, const NewTokens& t, int b, int i) {
    return c.start ? (int64_t)(t.row + i) * s.token : b * s.batch + i * s.token;
}

struct AttendProblem {
    PageTable c;
    const void *q, *k, *v;
    void* o;
    float* part;             // partial sums, NULL: nothing is cut
    int32_t H_q, window;
    int32_t n_split, least;  // workgroups that share the work (1: they do not), blocks of a share at least
    int32_t max_kv;          // bound on kv_len that the cuts go by
    int32_t wide;            // sums over the sequences may pass 32 bits
    float scale_log2;        // scale * log2(e)
    RowStrides qs, os;
};

struct AppendProblem {
    PageTable c;
    const void *q, *k, *v;
    void *q_out, *k_pages, *v_pages;
    const void *q_gain, *k_gain;
    const float* inv_freq;
    const int32_t* positions;
    int32_t L, H_q, rot, interleaved;
    float eps;
    RowStrides qs, qos, ks, vs;
};

// Reordering (n_rows > 0) or compaction (n_rows = 0).
struct PagesProblem {
    PageTable c;
    void *k_pages, *v_pages;
    const int32_t *source, *keep, *want;
    int32_t* new_table;
    int32_t* count;          // missing, or used
    int32_t L, n_rows, elem_bytes;
    bool heads_first;        // page layout [H_kv][page_size][D]
    void* ws;
};

// Sets p.n_split, p.least and p.wide; the bytes of `part` that they need (0: nothing is cut).
size_t attend_plan(AttendProblem& p, bool bf16);
// Whether every launch of the call is one that a device takes.
bool attend_fits(const AttendProblem& p, bool bf16);
hipError_t launch_paged_attention(const AttendProblem& p, bool bf16, hipStream_t stream);
// bf16 calls on tiles of 32 query rows (k_paged_decode.hip), of 128 (k_paged_chunk.hip), and fp32
// ones, of 16 (k_paged_f32.hip).  finds: the workgroups find their work, of 512 sequences at most
hipError_t launch_paged_decode(const AttendProblem& p, bool finds, hipStream_t stream);
hipError_t launch_paged_chunk(const AttendProblem& p, bool finds, hipStream_t stream);
hipError_t launch_paged_f32(const AttendProblem& p, bool finds, hipStream_t stream);
hipError_t launch_cache_append(const AppendProblem& p, bool bf16, hipStream_t stream);
// n_rows: of a reordering, 0: compaction; rows x max_pages: entries of the new table (0 bytes:
// the plan fits a workgroup's LDS)
size_t pages_workspace_bytes(int64_t n_pages, int64_t n_rows, int64_t rows, int64_t max_pages);
hipError_t launch_cache_reorder(const PagesProblem& p, hipStream_t stream);
hipError_t launch_cache_compact(const PagesProblem& p, hipStream_t stream);

}  // namespace mot
