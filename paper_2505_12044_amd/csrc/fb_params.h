// Host/device-shared parameter blocks for the attention kernels (plain data only).
#ifndef FB_PARAMS_H_
#define FB_PARAMS_H_

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

struct FwdParams {
    const void* q;        // [B,H,N,C]
    const void* k;
    const void* v;
    const void* phi_q;    // [Bp,H,N,R] or null
    const void* phi_k;
    const float* slopes;  // [H] per-head ALiBi slopes (in-kernel factor generation only)
    const void* bias;     // [Bb,H,N,N] or null (dense-bias mode)
    void* out;            // [B,H,N,C]
    float* lse;           // [B,H,N]
    int B, H, N, R;       // N = number of queries
    int M;                // number of keys (= N except for cross-attention: fp32, four-wave and few-query kernels)
    int causal;
    int phi_f32;          // factors stored as float (else bf16)
    long long phi_bstride;   // elements between batch items of phi_q (0 when shared over batch)
    long long phik_bstride;  // ... of phi_k
    long long bias_bstride;  // elements between batch items of bias (0 when shared)
    float scale;
    float inv_scale;      // 1 / scale, formed on the host (the backward forms the same value there)
    int causal_up;        // causal pairs: the first tile walks its off-diagonal blocks upwards from key 0
    int n_qtiles;         // query tiles per (b,h)
    int n_units;          // work units (workgroups) per (b,h): tiles, or tile pairs when causal
    int total_tiles;      // B*H*n_units
    int tiles_per_xcd;    // ceil(total_tiles / 8)
};

struct BwdParams {
    const void* q; const void* k; const void* v;
    const void* phi_q; const void* phi_k;
    const void* out; const float* lse; const void* dout;
    void* dq; void* dk; void* dv; void* dphi_q; void* dphi_k;
    const float* slopes;  // [H] ALiBi slopes: factors phi_q(i) = [-m i, m], phi_k(j) = [1, j] are generated in the
                          // pre-pass instead of read (phi_q, phi_k, dphi_q, dphi_k NULL, R = 2, phi_f32 = 1); else NULL
    float* dslope;        // [B,H,N] or NULL (with slopes only): per-row gradient of the head's slope, sum_j dS_ij (j - i)
    const void* bias;     // [Bb,H,N,M] dense-bias backward only
    void* dbias;          // [B,H,N,M]
    long long bias_bstride;  // elements between batch items of bias (0 when shared)
    void* workspace;      // device scratch: -lse2 and -D of every query row, and the operand columns that are not read in place
    size_t workspace_bytes;  // its size (what it holds beyond the rest takes dS)
    int B, H, N, R;       // N = number of queries
    int M;                // number of keys (= N except for cross-attention)
    int Cg;               // channels per head in caller memory (16 runs on the C = 32 kernels), else C
    int causal;
    int phi_f32;
    int grad_f32;         // dq, dk, dphi_q, dphi_k are written as float (multiplicative bias: the fold kernel
                          // sums them, so they must not be rounded to bf16 first); dv stays bf16
    long long phi_bstride;   // elements between batch items of phi_q (0 when shared over batch)
    long long phik_bstride;  // ... of phi_k
    float scale;
    int n_tiles;          // tiles per (b,h) along the kernel's outer dimension
    int total_tiles;
    int tiles_per_xcd;
};

// Rotary positions: one tensor of rows [B, heads, N, C], read with strides (elements), written contiguously.
struct RotaryTensor {
    const void* x;
    void* y;
    long long sb, sh, sn;
};

struct RotaryParams {
    RotaryTensor t0, t1;     // H1 = 0: the first only
    const void* positions;   // [axes, B or 1, N] int or float
    const float* freqs;      // [pairs]
    int B, N, C, H0, H1;
    int pairs;               // turned pairs of a row
    int end0, end1, end2;    // pairs of the first axis, of the first two, of the first three
    int pos_f32, pos_shared, interleaved;
    int inverse;             // turn back (the backward)
    int heads_per_group;     // set by the launch
    long long block0;        // workgroups of the launches before this one
};

// Pages of a key-value cache.  Requests b = 0..B-1 own ceil(len / page) pages each, table[b][0..).
struct PagedPlanParams {
    const int* lens;         // [B] tokens held
    const int* new_lens;     // [B] tokens wanted
    int* table;              // [B, max_blocks]
    int* ring;               // [n_pages] free pages, count of them from head on
    const int* state;        // head, count
    int* lens_out;           // [B]
    int* state_out;
    int* slots;              // [B, N]
    int* positions;          // [B, N] or null
    int B, N, page_shift, n_pages, max_blocks;
};

struct PagedAppendParams {
    const void* k;           // [B, Hkv, N, C] with strides
    const void* v;
    long long k_sb, k_sh, k_sn, v_sb, v_sh, v_sn;
    const void* phi_k;       // [Bp, Hkv, N, R] or null
    long long phik_bstride;  // 0 when shared over the batch
    const int* slots;        // [B, N]
    void* k_pages;           // [n_pages, Hkv, page, C]
    void* v_pages;
    void* phi_pages;         // [n_pages, Hkv, page, R]
    int B, Hkv, N, C, R, page_shift, n_pages;
    int heads_per_group;     // set by the launch
    long long block0;        // workgroups of the launches before this one
};

struct PagedAttnParams {
    const void* q;           // [B, H, N, C]
    const void* k_pages;     // [n_pages, Hkv, page, C]
    const void* v_pages;
    const void* phi_q;       // [Bp, H, N, R] or null
    const void* phi_pages;   // [n_pages, Hkv, page, R]
    const float* slopes;     // [H] or null
    const int* table;        // [B, max_blocks]
    const int* lens;         // [B]
    const int* starts;       // [B] position of a request's first query, or null: lens - N
    void* out;               // [B, H, N, C]
    float* lse;              // [B, H, N]
    long long phiq_bstride;
    int B, H, Hkv, N, R, page_shift, n_pages, max_blocks, causal, phi_f32;
    float scale;
    int tile_rows, row_tiles;    // query rows of a key head (H / Hkv * N of them, below 2^24) in tiles of 16 or 32
    int G, capacity;         // set by the launch: H / Hkv; keys that a table row has room for
    float inv_n;             // 1 / N
    int workers;             // waves the keys are split over; 0: a workgroup per key head and row tile, no split
    int waves;               // of such a workgroup, set by the launch
    unsigned block0;         // such workgroups of the launches before this one
    int joins_by_group;      // joins has an entry per (request, key head, row tile), else one per worker
    float* part_o;           // scratch: two parts per worker, [workers, 2, rows, C], rows = min(tile_rows, H / Hkv * N)
    float* part_m;           // [workers, 2, rows] maxima
    float* part_l;           // [workers, 2, rows] sums
    int4* joins;             // workers behind the first that have parts (0: no join), the first, the group, its rows
};

#endif
