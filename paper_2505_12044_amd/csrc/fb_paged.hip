// Pages of a key-value cache: which request owns which page, and the new tokens' rows stored into them.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "fb_device.h"
#include "fb_launch.h"
#include "fb_params.h"

namespace {

// ---- tables and slots ------------------------------------------------------------------------
// Request b goes from o = lens[b] to w = new_lens[b] tokens.  Shrinking ones give their last pages back, to the end of
// the ring of free pages, in the order (b, page); growing ones then take theirs from the ring's head in the order of b:
// b gets its pages if the needs of 0..b add up to no more than there are.  Token i of the call is o + i.
//
// Bound by latency: a few reads per request and one written int or two per token.  One launch: every workgroup sums
// the whole batch's needs by itself (a scan of at most 4096 lengths from L2), so nothing is handed over between
// workgroups, and then owns kPlanItems tokens of [B, N].  The thread of a page's first token enters the page in the
// table.  A page taken in the same call in which it was given back is looked up where it comes from (a shrinking
// request's table row, which no one writes), not in the ring, which another workgroup may not have written yet.
// us for B 64 N 1; B 256 N 4096; B 1024 N 1; B 4096 N 1: with 512 threads and tokens 6.2, 9.8, 9.9, 14.0; 256 each 6.0, 9.6,
// 10.4, 17.7; 1024 each 6.8, 13.8, 11.2, 13.9.  For a prompt's many tokens the scan of the batch, repeated by each of 2048
// workgroups for one token a thread, is most of the time (B 256 N 4096: 10.3 us for 8.4 MB written).
constexpr int kPlanThreads = 512;
constexpr int kPlanItems = 512;

struct Request {
    int used, goal;      // pages before and after (as wanted)
    int len, want;
};

FB_DEV Request request_of(const PagedPlanParams& p, int b) {
    Request r;
    const int cap = (int)min((long long)p.max_blocks << p.page_shift, (long long)0x7fffffff);
    r.len = min(max(p.lens[b], 0), cap);
    r.want = max(p.new_lens[b], 0);
    if (r.want > cap || r.want - r.len > p.N) r.want = r.len;          // refused: no room in the table or in the slots
    const int up = (1 << p.page_shift) - 1;
    r.used = (int)(((unsigned)r.len + up) >> p.page_shift);
    r.goal = (int)(((unsigned)r.want + up) >> p.page_shift);
    return r;
}

// inclusive sums over the workgroup; total in every thread
FB_DEV long long block_scan(long long x, long long* sm, long long& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const long long y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) sm[wave] = x;
    __syncthreads();
    long long before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; w++) {
        if (w < wave) before += sm[w];
        total += sm[w];
    }
    __syncthreads();
    return x + before;
}

__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(PagedPlanParams p) {
    extern __shared__ int sm_ends[];                   // [B] pages given back up to b, [B] pages needed up to b
    int* give_end = sm_ends;
    int* need_end = sm_ends + p.B;
    __shared__ long long sm[kPlanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    const int n = p.n_pages, state_head = p.state[0], state_count = p.state[1];
    // the sums stay below 2^31: B * max_blocks does (checked on the host)
    long long gives = 0, needs = 0;
    for (int b0 = 0; b0 < p.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        int give = 0, need = 0;
        if (b < p.B) {
            const Request r = request_of(p, b);
            give = max(r.used - r.goal, 0);
            need = max(r.goal - r.used, 0);
        }
        // both sums at once: 32 bits each
        long long total;
        const long long end = block_scan(((long long)give << 32) | need, sm, total);
        if (b < p.B) {
            give_end[b] = (int)((end >> 32) + gives);
            need_end[b] = (int)((end & 0xffffffffLL) + needs);
        }
        gives += total >> 32;
        needs += total & 0xffffffffLL;
    }
    __syncthreads();
    int head = state_head % n;
    if (head < 0) head += n;
    const int count = min(max(state_count, 0), n);
    const long long avail = count + gives;
    auto granted = [&](int b, const Request& r) { return r.goal <= r.used || need_end[b] <= avail; };
    auto ring_at = [&](long long k) { return (int)((unsigned)(head + k) % (unsigned)n); };      // head + k < 2^32: see the host's checks

    const unsigned items = (unsigned)p.B * p.N, N = p.N;               // below 2^31
    const unsigned i0 = blockIdx.x * kPlanItems, i1 = min(i0 + kPlanItems, items);
    for (unsigned it = i0 + tid; it < i1; it += kPlanThreads) {
        const int b = (int)(it / N), i = (int)(it - b * N);
        const Request r = request_of(p, b);
        const int len = granted(b, r) ? r.want : r.len;
        int slot = -1, pos = 0;
        if (i < len - r.len) {
            pos = r.len + i;
            const int j = pos >> p.page_shift;
            int* entry = p.table + (long long)b * p.max_blocks + j;
            int page;
            if (j < r.used) {
                page = *entry;
            } else {
                const int k = need_end[b] - (r.goal - r.used) + j - r.used;      // the k-th page taken
                if (k < count) {
                    page = p.ring[ring_at(k)];
                } else {
                    const int g = k - count;                                      // the g-th page given back
                    int lo = 0, hi = p.B - 1;
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (give_end[mid] > g) hi = mid;
                        else lo = mid + 1;
                    }
                    const Request from = request_of(p, lo);
                    page = p.table[(long long)lo * p.max_blocks + from.goal + g - (give_end[lo] - (from.used - from.goal))];
                }
                if ((pos & ((1 << p.page_shift) - 1)) == 0) *entry = page;
            }
            if (page >= 0 && page < n) slot = (page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
        }
        p.slots[it] = slot;
        if (p.positions) p.positions[it] = pos;
        if (i == 0) p.lens_out[b] = len;
    }

    // pages given back by the requests whose first token is here, a wave each
    const int b_begin = (int)((i0 + N - 1) / N), b_end = (int)((i1 + N - 1) / N);
    for (int b0 = b_begin + wave * 64; b0 < b_end; b0 += kPlanThreads) {
        const int bl = b0 + lane;
        const bool gives_back = bl < b_end && give_end[bl] > (bl > 0 ? give_end[bl - 1] : 0);
        for (unsigned long long m = __ballot(gives_back); m != 0; m &= m - 1) {
            const int b = b0 + __builtin_ctzll(m);
            const Request r = request_of(p, b);
            const long long at = count + give_end[b] - (r.used - r.goal);
            for (int j = lane; j < r.used - r.goal; j += 64)
                p.ring[ring_at(at + j)] = p.table[(long long)b * p.max_blocks + r.goal + j];
        }
    }

    if (blockIdx.x == 0) {       // pages taken: the needs of the last request that got its pages
        int taken = 0;
        for (int b = tid; b < p.B; b += kPlanThreads)
            if (need_end[b] <= avail) taken = max(taken, need_end[b]);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) taken = max(taken, __shfl_xor(taken, d));
        if (lane == 0) sm[wave] = taken;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kPlanThreads / 64; w++) taken = max(taken, (int)sm[w]);
            p.state_out[0] = ring_at(taken);
            p.state_out[1] = (int)min(avail - taken, (long long)n);
        }
    }
}

// ---- new rows into their pages ---------------------------------------------------------------
// Bound by memory: every row is read once and written once.  A thread owns one vector of one token's rows (its slot is
// read once) and walks a group of heads, kAppHeads keys and values in flight.  B 8, N 4000 (ragged), 16 heads, C 128 from a
// fused projection: 89 us, 4.8 TB/s read and written (a copy kernel reaches 5.6, 6.1 with non-temporal loads and stores); with
// 2048 workgroups and more 95 us.  Factors go element by element, head after head: with rank 2 100 us, rank 16 108 us.
constexpr int kAppThreads = 256;
constexpr int kAppHeads = 4;

template <typename PT>
FB_DEV void append_factors(const PagedAppendParams& p, int b, int n, int h, long long row, int u, int units) {
    const PT* src = (const PT*)p.phi_k + (long long)b * p.phik_bstride + ((long long)h * p.N + n) * p.R;
    PT* dst = (PT*)p.phi_pages + row * p.R;
    for (int r = u; r < p.R; r += units) dst[r] = src[r];
}

// V: the vector copied at once
template <typename V, int SIZE>
__global__ __launch_bounds__(kAppThreads) void paged_append_kernel(PagedAppendParams p, int phi_size) {
    constexpr int VEC = sizeof(V) / SIZE;               // elements of a vector
    const int units = p.C / VEC;
    const long long id = (p.block0 + blockIdx.x) * kAppThreads + threadIdx.x;
    const long long token = id / units;
    const int u = (int)(id - token * units);
    if (token >= (long long)p.B * p.N) return;
    const int slot = p.slots[token];
    const int page = slot >> p.page_shift;
    if (slot < 0 || page >= p.n_pages) return;
    const int b = (int)(token / p.N), n = (int)(token - (long long)b * p.N);
    const long long row0 = (((long long)page * p.Hkv) << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
    const char* kx = (const char*)p.k + (b * p.k_sb + n * p.k_sn + u * VEC) * SIZE;
    const char* vx = (const char*)p.v + (b * p.v_sb + n * p.v_sn + u * VEC) * SIZE;
    const int h_begin = blockIdx.y * p.heads_per_group, h_end = min(h_begin + p.heads_per_group, p.Hkv);
    for (int h0 = h_begin; h0 < h_end; h0 += kAppHeads) {
        V kr[kAppHeads], vr[kAppHeads];
#pragma unroll
        for (int i = 0; i < kAppHeads; i++) {
            const int h = h0 + i;
            if (h >= h_end) break;
            kr[i] = *(const V*)(kx + h * p.k_sh * SIZE);
            vr[i] = *(const V*)(vx + h * p.v_sh * SIZE);
        }
#pragma unroll
        for (int i = 0; i < kAppHeads; i++) {
            const int h = h0 + i;
            if (h >= h_end) break;
            const long long row = row0 + ((long long)h << p.page_shift);
            ((V*)p.k_pages)[row * units + u] = kr[i];
            ((V*)p.v_pages)[row * units + u] = vr[i];
        }
    }
    if (p.R > 0)
        for (int h = h_begin; h < h_end; h++) {
            const long long row = row0 + ((long long)h << p.page_shift);
            if (phi_size == 4) append_factors<unsigned>(p, b, n, h, row, u, units);
            else append_factors<unsigned short>(p, b, n, h, row, u, units);
        }
}

template <typename V, int SIZE>
int launch_append(PagedAppendParams& p, int phi_size, hipStream_t stream) {
    const long long threads = (long long)p.B * p.N * (p.C / (int)(sizeof(V) / SIZE));
    const long long blocks = (threads + kAppThreads - 1) / kAppThreads;
    long long groups = (512 + blocks - 1) / blocks;     // heads per thread: as many as leave 512 workgroups
    if (groups > p.Hkv) groups = p.Hkv;
    p.heads_per_group = (int)((p.Hkv + groups - 1) / groups);
    groups = (p.Hkv + p.heads_per_group - 1) / p.heads_per_group;
    for (p.block0 = 0; p.block0 < blocks; p.block0 += kFbLaunchBlocks)
        hipLaunchKernelGGL((paged_append_kernel<V, SIZE>), dim3((unsigned)std::min(blocks - p.block0, kFbLaunchBlocks), (unsigned)groups),
                           dim3(kAppThreads), 0, stream, p, phi_size);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace

int fb_launch_paged_plan(const PagedPlanParams& p, hipStream_t stream) {
    const long long blocks = ((long long)p.B * p.N + kPlanItems - 1) / kPlanItems;
    hipLaunchKernelGGL(paged_plan_kernel, dim3((unsigned)blocks), dim3(kPlanThreads), (size_t)p.B * 2 * sizeof(int), stream, p);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

// The widest vector, up to 16 bytes, that every row start allows (pages are 16-byte aligned, rows at least 32 bytes long).
int fb_launch_paged_append(PagedAppendParams p, bool f32, bool phi_f32, hipStream_t stream) {
    const int size = f32 ? 4 : 2, phi_size = phi_f32 ? 4 : 2;
    long long bits = 16 | (long long)reinterpret_cast<uintptr_t>(p.k) | (long long)reinterpret_cast<uintptr_t>(p.v);
    if (p.B > 1) bits |= (p.k_sb | p.v_sb) * size;      // strides of axes of one element do not count
    if (p.Hkv > 1) bits |= (p.k_sh | p.v_sh) * size;
    if (p.N > 1) bits |= (p.k_sn | p.v_sn) * size;
    const int bytes = (int)(bits & -bits);
    if (f32) {
        if (bytes == 16) return launch_append<u32x4, 4>(p, phi_size, stream);
        if (bytes == 8) return launch_append<u32x2, 4>(p, phi_size, stream);
        return launch_append<unsigned, 4>(p, phi_size, stream);
    }
    if (bytes == 16) return launch_append<u32x4, 2>(p, phi_size, stream);
    if (bytes == 8) return launch_append<u32x2, 2>(p, phi_size, stream);
    if (bytes == 4) return launch_append<unsigned, 2>(p, phi_size, stream);
    return launch_append<unsigned short, 2>(p, phi_size, stream);
}
