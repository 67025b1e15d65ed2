// Attention of a few new tokens per request over a paged key-value cache, gfx950.
//
//     out = softmax(q k^T scale + b) v  over the request's own keys, causal for the new tokens among themselves;
// b: none, low-rank factors phi_q phi_k^T (phi_k in pages beside the keys), or ALiBi -m_h (i - j).  G = H / Hkv query
// heads share a key head, so the G N rows that meet the same keys form one tile of 16 rows (several where there are more).
//
// Bound by memory: every key and value row is read once per row tile, 4 C flops per row and key against 4 C bytes per
// key (bf16).  The matrix pipe has twenty times the rate that needs, so the 16-row tile runs whatever G N is (and where there
// are more rows a wave takes two tiles at once, RT: B 32, H 32 / 8, N 5, 500 to 16384 keys 239 -> 153 us, N 16 454 -> 272):
//   scores   S^T = K Q^T      keys are the rows of the A operand, read from their page straight into its layout
//   values   O^T += V^T P^T   P^T comes from the S^T registers as they are; a lane loads NV = C / 16 adjacent channels of
//                             its eight keys (whole rows per 16 lanes) and turns 8 x NV into operands by byte permutes
// so nothing passes through LDS and no wave waits for another inside the loop.  P enters as two bf16 limbs (its
// rounding to one would be as large as that of the result); scores, maxima and sums are fp32, in natural units (a bias
// of the type's lowest value keeps its differences).  fp32 tensors and all factors take the fp32 matrix instruction.
//
// The keys of all (request, key head, row tile) groups are laid end to end in steps of KW keys, and each of `workers`
// waves takes an equal share, found from the lengths on the device: one long request among short ones, or a table with
// room for far more than it holds, costs no balance, and no wave waits for another.  A share may end inside a group: the
// parts go to scratch, two per worker at most, and a second launch joins them in a fixed order.  Without scratch, and
// where no request can be long, a workgroup's waves share one group and join through LDS.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "fb_device.h"
#include "fb_launch.h"
#include "fb_params.h"

namespace {

constexpr int kPaWaves = 4;
constexpr int kPaThreads = kPaWaves * 64;
constexpr size_t group_lds(int waves, int rows, int c) { return (size_t)waves * rows * (c + 6) * sizeof(float); }
constexpr int pa_threads(int w) { return w == 1 ? kPaThreads : w * 64; }
// Costs of a worker's share at least, and the steps that a group's beginning and end count for in the shares.  us at 1, 2, 3 of
// the first: B 4, H 8 / 4, fp32 drafts 21.2, 17.9, 17.2; B 8, H 16, 100 to 1024 keys 13.5, 13.5, 14.9; of the second: encoder
// states (B 48, 1 to 1500 keys, 12 heads) 25.2, 25.0 and, not counted, 27.9; B 8, 100 to 1024 keys 13.7, 13.5, 15.1.
constexpr int kPaLeast = 2;
constexpr int kPaLead = 2;

typedef float f32x8 __attribute__((ext_vector_type(8)));

// Both values of the rows of 16 lanes 2 n, 2 n + 1 in both rows (half_pair of fb_device.h, one level down).
FB_DEV HalfPair row_pair(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    unsigned w = u;
    asm volatile("" : "+v"(w));
    auto r = __builtin_amdgcn_permlane16_swap(u, w, false, false);
    return {__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])};
}
// over the four lanes of a column
FB_DEV float column_max(float x) {
    const HalfPair p = row_pair(x);
    return half_max(fmaxf(p.lo, p.hi));
}
FB_DEV float column_sum(float x) {
    const HalfPair p = row_pair(x);
    return half_sum(p.lo + p.hi);
}

// exp(a - m) for a <= m; 0 where a is -inf, whatever m is
FB_DEV float weight(float a, float m) { return a == -INFINITY ? 0.f : fast_exp2((a - m) * kLog2e); }

// ---- one step of a wave: KW keys against 16 rows -----------------------------------------------
// Values are read past the caches (each row once, by whole lines): B 32 H 32 / 8 C 128 152 -> 139 us, C 64 128 -> 108 us at
// 604 MB.  Keys are not: half a line per load instruction, and the same figures within 3 % either way.
// KW: 32 keys in bf16, 16 in fp32, twice that below 64 channels, where a row is little.  A wave has one step in flight and a
// step takes a memory latency, but fewer keys a step reach more waves: C 64, 576 groups of 500 keys, 32 / 64 keys a step 16.8 /
// 19.3 us, C 128 drafts and long batches 5 % apart; C 32, 1024 groups of 8192 keys 222 / 186 us.
// Lane l: g = l / 16, i = l % 16.  S^T group s (16 keys): column i (the query row), keys 4 g + r.
template <typename T, int C, int GROUPS>
struct Step;
constexpr int step_groups(int c, bool f32) { return (c <= 32 ? 4 : 2) / (f32 ? 2 : 1); }
// Waves a SIMD has where each has its own share, and the launch counts on.  us at 2, 3, 4: B 48 encoder states to 8000 keys, C 64
// 86, 82, 84; B 64 to 8192 keys, C 16 75, 62, 63, C 32 103, 107, 107; C 128 has no registers for three.
constexpr int waves_per_simd(int c, int tiles) { return tiles > 1 ? 2 : (c == 16 ? 4 : (c == 64 ? 3 : 2)); }
constexpr bool two_tiles(int c, bool f32) { return c >= 64 && !f32; }    // whether a step may serve 32 rows

template <int C, int GROUPS>
struct Step<bf16_t, C, GROUPS> {
    static constexpr int KW = 16 * GROUPS, NV = C / 16;
    static constexpr int NU = C >= 32 ? C / 32 : 1;
    using KVec = std::conditional_t<C == 16, u32x2, u32x4>;
    using VVec = std::conditional_t<NV == 8, u32x4, std::conditional_t<NV == 4, u32x2, std::conditional_t<NV == 2, unsigned, unsigned short>>>;
    struct Query { KVec x[NU]; };
    struct Keys { KVec x[GROUPS][NU]; };
    struct Values { VVec x[GROUPS][4]; };

    static FB_DEV KVec row_chunk(const bf16_t* row, int g, int u) {
        return *(const KVec*)(row + (C == 16 ? 4 * g : 32 * u + 8 * g));
    }
    static FB_DEV void load_keys(Keys& k, int s, const bf16_t* rows, int g, int i) {
#pragma unroll
        for (int u = 0; u < NU; u++) k.x[s][u] = row_chunk(rows + i * C, g, u);
    }
    static FB_DEV void load_values(Values& v, int s, const bf16_t* rows, int g, int i) {
#pragma unroll
        for (int r = 0; r < 4; r++) v.x[s][r] = __builtin_nontemporal_load((const VVec*)(rows + (4 * g + r) * C + i * NV));
    }
    static FB_DEV f32x4 scores(const Keys& k, int s, const Query& q) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < NU; u++) {
            if constexpr (C == 16)
                acc = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, k.x[s][u]), __builtin_bit_cast(s16x4, q.x[u]), acc,
                                                                0, 0, 0);
            else
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k.x[s][u]), __builtin_bit_cast(bf16x8, q.x[u]), acc,
                                                              0, 0, 0);
        }
        return acc;
    }
    struct Probs { bf16x8 hi[GROUPS / 2], lo[GROUPS / 2]; };       // two key groups an operand
    static FB_DEV Probs probs(const f32x4 (&p)[GROUPS]) {
        Probs w;
#pragma unroll
        for (int e = 0; e < 4 * GROUPS; e++) {
            const float x = p[e / 4][e % 4];
            const bf16_t hi = (bf16_t)x;
            w.hi[e / 8][e % 8] = hi;
            w.lo[e / 8][e % 8] = (bf16_t)(x - (float)hi);
        }
        return w;
    }
    // 32-bit word of channels 2 w, 2 w + 1 (of the lane's NV) of key e
    static FB_DEV unsigned word(const Values& v, int e, int w) {
        const VVec x = v.x[e / 4][e % 4];
        if constexpr (NV <= 2) return x;
        else return x[w];
    }
    // o + channel t's values times the probabilities
    static FB_DEV f32x4 product(const Values& v, int t, const Probs& p, f32x4 o) {
#pragma unroll
        for (int s = 0; s < GROUPS / 2; s++) {
            u32x4 a;
#pragma unroll
            for (int j = 0; j < 4; j++)
                a[j] = __builtin_amdgcn_perm(word(v, 8 * s + 2 * j + 1, t / 2), word(v, 8 * s + 2 * j, t / 2), t % 2 ? 0x07060302u : 0x05040100u);
            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), p.hi[s], o, 0, 0, 0);
            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), p.lo[s], o, 0, 0, 0);
        }
        return o;
    }
};

template <int C, int GROUPS>
struct Step<float, C, GROUPS> {
    static constexpr int KW = 16 * GROUPS, NV = C / 16;
    static constexpr int NU = C / 16;
    using VVec = std::conditional_t<NV == 8, f32x8, std::conditional_t<NV == 4, f32x4, std::conditional_t<NV == 2, f32x2, float>>>;
    struct Query { f32x4 x[NU]; };
    struct Keys { f32x4 x[GROUPS][NU]; };
    struct Values { VVec x[GROUPS][4]; };

    static FB_DEV f32x4 row_chunk(const float* row, int g, int u) { return *(const f32x4*)(row + 16 * u + 4 * g); }
    static FB_DEV void load_keys(Keys& k, int s, const float* rows, int g, int i) {
#pragma unroll
        for (int u = 0; u < NU; u++) k.x[s][u] = row_chunk(rows + i * C, g, u);
    }
    static FB_DEV void load_values(Values& v, int s, const float* rows, int g, int i) {
#pragma unroll
        for (int r = 0; r < 4; r++) v.x[s][r] = __builtin_nontemporal_load((const VVec*)(rows + (4 * g + r) * C + i * NV));
    }
    static FB_DEV f32x4 scores(const Keys& k, int s, const Query& q) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < NU; u++)
#pragma unroll
            for (int e = 0; e < 4; e++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[s][u][e], q.x[u][e], acc, 0, 0, 0);
        return acc;
    }
    struct Probs { f32x4 x[GROUPS]; };
    static FB_DEV Probs probs(const f32x4 (&p)[GROUPS]) {
        Probs w;
#pragma unroll
        for (int s = 0; s < GROUPS; s++) w.x[s] = p[s];
        return w;
    }
    static FB_DEV f32x4 product(const Values& v, int t, const Probs& p, f32x4 o) {
#pragma unroll
        for (int s = 0; s < GROUPS; s++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                float a;
                if constexpr (NV == 1) a = v.x[s][r];
                else a = v.x[s][r][t];
                o = __builtin_amdgcn_mfma_f32_16x16x4f32(a, p.x[s][r], o, 0, 0, 0);
            }
        return o;
    }
};

// factors: up to four; up to 16, a multiple of four; any number
enum { kBiasNone = 0, kBiasAlibi = 1, kBiasFactors4 = 2, kBiasFactors16 = 3, kBiasFactors = 4 };

// Arrays that are not written while the kernel runs, read at wave-uniform places: scalar loads, which do not queue behind
// the rows in flight.
typedef const __attribute__((address_space(4))) int* ConstInts;
FB_DEV ConstInts const_ints(const int* x) { return (ConstInts)(uintptr_t)x; }

// Keys of a request: its length within the table (capacity: 31 bits).
FB_DEV int held_keys(const PagedAttnParams& p, int len) { return max(min(len, p.capacity), 0); }

// Whether k + stride lies below end; their sum may pass 31 bits.
constexpr bool goes_on(int k, int stride, int end) { return k < end - stride; }
static_assert(goes_on(64, 512, 577) && !goes_on(64, 512, 576) && !goes_on(0, 512, 0) && !goes_on(0x7ffffe80, 512, 0x7fffff00), "");

// Steps of a request per group; one that holds nothing has one too (its rows are written).
template <int KW>
FB_DEV int steps_of(int len) { return len > KW ? (int)((unsigned)(len + KW - 1) / KW) : 1; }

// Sums up to the lane's.
FB_DEV int wave_scan(int x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// The costs of all requests' groups (their steps, and kPaLead that lie before them) laid end to end and cut in shares of
// `base` or, the first `longer` of them, base + 1: this wave's is [u, u_end), u lies in request b, rem behind its beginning.
// All below 2^31 (the launch sees to it).
struct Share {
    int u, u_end, b, rem;
    int len, start;          // of request b, as stored
    int base, longer, workers;
    FB_DEV void cut(int total, int most, int worker) {
        workers = min(most, (total + kPaLeast - 1) / kPaLeast);
        base = total / workers;
        longer = total - base * workers;
        u = worker * base + min(worker, longer);
        u_end = worker < workers ? u + base + (worker < longer ? 1 : 0) : u;
    }
    FB_DEV int worker_of(int x) const {
        const int edge = longer * (base + 1);
        return x < edge ? x / (base + 1) : longer + (x - edge) / base;
    }
};

template <int KW>
FB_DEV Share share_of(const PagedAttnParams& p, int groups, int worker) {
    __shared__ int sm_sum[kPaWaves], sm_b[kPaWaves], sm_rem[kPaWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Share s{};
    const auto cost = [&](int b, int len) { return b < p.B ? (steps_of<KW>(held_keys(p, len)) + kPaLead) * groups : 0; };
    if (p.B <= 64) {                                     // every wave by itself
        const int at = min(lane, p.B - 1), len = p.lens[at], start = p.starts ? p.starts[at] : 0;
        const int own = cost(lane, len), end = wave_scan(own);
        s.cut(__builtin_amdgcn_readlane(end, 63), p.workers, worker);
        if (s.u < s.u_end) {
            s.b = __builtin_ctzll(__ballot(end > s.u));
            s.rem = s.u - __builtin_amdgcn_readlane(end - own, s.b);
            s.len = __builtin_amdgcn_readlane(len, s.b);
            s.start = __builtin_amdgcn_readlane(start, s.b);
        }
        return s;
    }
    // the workgroup's four shares together, 256 requests at a time: the total first
    const auto tile = [&](int b0, int& own, int& sum) {
        own = cost(b0 + tid, p.lens[min(b0 + tid, p.B - 1)]);
        const int in_wave = wave_scan(own);
        __syncthreads();
        if (lane == 63) sm_sum[wave] = in_wave;
        __syncthreads();
        int before = 0;
        sum = 0;
#pragma unroll
        for (int w = 0; w < kPaWaves; w++) {
            if (w < wave) before += sm_sum[w];
            sum += sm_sum[w];
        }
        return before + in_wave;
    };
    int own, sum, total = 0, before = 0;
    for (int b0 = 0; b0 < p.B; b0 += kPaThreads) {
        tile(b0, own, sum);
        total += sum;
    }
    s.cut(total, p.workers, worker);
    for (int b0 = 0; b0 < p.B; b0 += kPaThreads) {
        const int end = before + tile(b0, own, sum);
        for (int w = 0; w < kPaWaves; w++) {
            const int k = worker - wave + w, u = k * s.base + min(k, s.longer);
            if (end - own <= u && u < end) {
                sm_b[w] = b0 + tid;
                sm_rem[w] = u - (end - own);
            }
        }
        before += sum;
    }
    __syncthreads();
    if (s.u < s.u_end) {
        s.b = __builtin_amdgcn_readfirstlane(sm_b[wave]);
        s.rem = sm_rem[wave];
        s.len = const_ints(p.lens)[s.b];
        s.start = p.starts ? const_ints(p.starts)[s.b] : 0;
    }
    return s;
}

// Four channels of a result row from its sums.
template <typename T, int C>
FB_DEV void write_row(const PagedAttnParams& p, long long row, int c4, const f32x4& o, float l, float m) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    struct alignas(4 * sizeof(T)) Four { T x[4]; } v;
#pragma unroll
    for (int e = 0; e < 4; e++) v.x[e] = (T)(l == 0.f ? 0.f : o[e] * inv);
    *(Four*)((T*)p.out + row * C + c4 * 4) = v;
    if (c4 == 0) p.lse[row] = l == 0.f ? -INFINITY : m + __log2f(l) * kLn2;
}

// One wave's (SPLIT) or workgroup's part of a group: steps t0..t1 of n_steps.
struct Segment {
    int b, len, start, n_steps, grp, t0, t1;
};

// BIAS, PF32: kind of bias and whether the factors are float
// W: waves that share a group, one workgroup (4 or 8), or 1: each wave has its own share of all groups
// RT: tiles of 16 query rows that a step serves
template <typename T, int C, int BIAS, bool PF32, int W, int RT>
__global__ __launch_bounds__(pa_threads(W), W == 1 ? waves_per_simd(C, RT) : 2) void paged_attn_kernel(PagedAttnParams p) {
    constexpr bool SPLIT = W == 1;
    constexpr int ROWS = 16 * RT;
    constexpr int GROUPS = step_groups(C, std::is_same_v<T, float>);
    using S = Step<T, C, GROUPS>;
    constexpr int KW = S::KW, NV = S::NV;
    constexpr int STRIDE = W * KW;                        // keys from one step of a wave to its next
    constexpr int NF = BIAS == kBiasFactors4 ? 1 : (BIAS >= kBiasFactors16 ? 4 : 0);
    using PT = std::conditional_t<PF32, float, bf16_t>;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, i = lane & 15;
    const int groups = p.Hkv * p.row_tiles;               // of a request
    const int rows_all = p.G * p.N;
    const int page_mask = (1 << p.page_shift) - 1;

    auto enter = [&](Segment& s, int len, int start) __attribute__((always_inline)) {      // request s.b, its len and start as stored
        s.len = held_keys(p, len);
        s.n_steps = steps_of<KW>(s.len);
        s.start = p.starts ? min(max(start, -(1 << 30)), 1 << 30) : s.len - p.N;
    };
    auto enter_next = [&](Segment& s) __attribute__((always_inline)) {
        enter(s, const_ints(p.lens)[s.b], p.starts ? const_ints(p.starts)[s.b] : 0);
    };
    Segment f;                                            // of the step to load next, at key fk
    Share share{};
    const int worker = blockIdx.x * kPaWaves + wave;
    int left = 0;                                         // of this worker's share behind that segment
    if constexpr (SPLIT) {
        share = share_of<KW>(p, groups, worker);
        f.b = __builtin_amdgcn_readfirstlane(share.b);
        left = __builtin_amdgcn_readfirstlane(share.u_end - share.u);
        f.t0 = f.t1 = 0;
        if (left > 0) {
            enter(f, __builtin_amdgcn_readfirstlane(share.len), __builtin_amdgcn_readfirstlane(share.start));
            const int rem = __builtin_amdgcn_readfirstlane(share.rem), cost = f.n_steps + kPaLead;
            f.grp = __builtin_amdgcn_readfirstlane((int)((unsigned)rem / (unsigned)cost));
            const int at = rem - f.grp * cost;            // the share's beginning in the group's costs
            f.t0 = max(at - kPaLead, 0);
            f.t1 = max(min(f.n_steps, at - kPaLead + left), 0);
            left -= f.t1 + kPaLead - at;
        }
        if (f.t1 <= f.t0) {                               // no share, or all of it before a group's first step
            if (!p.joins_by_group && worker < p.workers && lane == 0) p.joins[worker] = make_int4(0, 0, 0, 0);
            return;
        }
    } else {
        const unsigned block = p.block0 + blockIdx.x;
        f.b = __builtin_amdgcn_readfirstlane(block / (unsigned)groups);
        f.grp = block - f.b * groups;
        enter_next(f);
        f.t0 = 0;
        f.t1 = f.n_steps;
    }

    // ---- what a step reads ----
    // Pages of the 16-key groups, -1 behind the segment and for an entry that is no page: such a group is not visible, and the
    // first rows of page 0 stand in for it.
    auto pages_at = [&](int (&page)[GROUPS], const Segment& s, int k) __attribute__((always_inline)) {
        const ConstInts table = const_ints(p.table) + (long long)s.b * p.max_blocks;
        const int end = min(s.len, s.t1 * KW);
#pragma unroll
        for (int x = 0; x < GROUPS; x++) {
            const int held = table[max(min(k + 16 * x, end - 1), 0) >> p.page_shift];
            page[x] = k + 16 * x < end && (unsigned)held < (unsigned)p.n_pages ? held : -1;
        }
    };
    auto row_at = [&](int page, int h, int k) __attribute__((always_inline)) {      // row of key k, the first of a group
        return page < 0 ? 0LL : (((long long)page * p.Hkv + h) << p.page_shift) + (k & page_mask);
    };
    typename S::Keys kr;
    typename S::Values vr;
    unsigned fr[GROUPS][NF > 0 ? NF : 1];                 // factors as loaded (unpacking them would wait for the load)
    // Factors of one row, the lane's share: factor g of up to four; 4 g .. 4 g + 3 of the first 16.
    auto load_factors = [&](unsigned (&f)[NF > 0 ? NF : 1], const PT* pk) __attribute__((always_inline)) {
        using Bits = std::conditional_t<PF32, unsigned, unsigned short>;
        if constexpr (BIAS == kBiasFactors16) {
            using Four = std::conditional_t<PF32, u32x4, u32x2>;
            Four v = {};
            if (4 * g < p.R) v = *(const Four*)(pk + 4 * g);
#pragma unroll
            for (int y = 0; y < (PF32 ? 4 : 2); y++) f[y] = v[y];
        } else {
#pragma unroll
            for (int y = 0; y < NF; y++) {
                f[y] = 0u;
                if (NF * g + y < p.R) f[y] = ((const Bits*)pk)[NF * g + y];
            }
        }
    };
    auto factor = [&](const unsigned (&f)[NF > 0 ? NF : 1], int y) __attribute__((always_inline)) {
        if constexpr (PF32) return __builtin_bit_cast(float, f[y]);
        else if constexpr (BIAS == kBiasFactors16) return __builtin_bit_cast(float, y & 1 ? f[y / 2] & 0xffff0000u : f[y / 2] << 16);
        else return __builtin_bit_cast(float, f[y] << 16);
    };

    // One loop over the steps of all segments, one step ahead: the next step's keys are loaded when the scores have used this
    // one's, its values after this one's product, its pages before that.  With SPLIT the first turn only loads (every CU walks
    // through the code cold, and many waves start at once: a second copy of the loads costs more than it saves).
    Segment s = f;
    int fk = f.t0 * KW + (SPLIT ? 0 : wave * KW), k0 = 0;
    int f_page[GROUPS], page[GROUPS];
    pages_at(f_page, f, fk);
    bool have = false, more = true;                       // a step is loaded; one is to be loaded

    // of the segment: the lane's query row in each tile, its sums
    struct Row {
        bool has;
        int pos, limit;                                   // limit: keys the row sees
        typename S::Query q;
        float phi_q[NF > 0 ? NF : 1], slope, m, l;
        const PT* pq;
        f32x4 o[NV];
    } row[RT];
    int all_see = 0, rows = 0, h = 0;
    long long row_base = 0;

    // ---- a segment (s) begins ----
    auto begin = [&]() __attribute__((always_inline)) {
        h = p.row_tiles == 1 ? s.grp : s.grp / p.row_tiles;
        const int r0 = (s.grp - h * p.row_tiles) * ROWS;
        rows = min(ROWS, rows_all - r0);
        row_base = (long long)s.b * p.H * p.N + (long long)h * rows_all + r0;       // of q, out, lse
        all_see = p.causal ? max(min(s.start + 1, s.len), 0) : s.len;                // keys every row sees
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            Row& w = row[rt];
            const int at = 16 * rt + i;
            w.has = at < rows;
            // (r0 + at) / N and the rest, rows below 2^24
            int head = (int)((float)(r0 + at) * p.inv_n);
            int n = r0 + at - head * p.N;
            if (n < 0) head--, n += p.N;
            else if (n >= p.N) head++, n -= p.N;
            w.pos = s.start + n;
            w.limit = !w.has ? 0 : (p.causal ? (w.pos >= s.len || w.pos < 0 ? 0 : w.pos + 1) : s.len);
#pragma unroll
            for (int x = 0; x < S::NU; x++) {
                w.q.x[x] = {};
                if (w.has) w.q.x[x] = S::row_chunk((const T*)p.q + (row_base + at) * C, g, x);
            }
            if constexpr (NF > 0) {
                w.pq = (const PT*)p.phi_q + (long long)s.b * p.phiq_bstride + ((long long)h * rows_all + r0 + at) * p.R;
#pragma unroll
                for (int x = 0; x < NF; x++) {
                    w.phi_q[x] = 0.f;
                    if (w.has && NF * g + x < p.R) w.phi_q[x] = (float)w.pq[NF * g + x];
                }
            }
            w.slope = 0.f;
            if constexpr (BIAS == kBiasAlibi)
                if (w.has) w.slope = p.slopes[h * p.G + head];
            w.m = -INFINITY;
            w.l = 0.f;
#pragma unroll
            for (int t = 0; t < NV; t++) w.o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    auto load_keys = [&]() __attribute__((always_inline)) {              // of step f, fk
        const int fh = p.row_tiles == 1 ? f.grp : f.grp / p.row_tiles;
#pragma unroll
        for (int x = 0; x < GROUPS; x++) {
            const long long at = row_at(f_page[x], fh, fk + 16 * x);
            S::load_keys(kr, x, (const T*)p.k_pages + at * C, g, i);
            if constexpr (NF > 0) load_factors(fr[x], (const PT*)p.phi_pages + (at + i) * p.R);
        }
    };
    auto load_values = [&]() __attribute__((always_inline)) {
        const int fh = p.row_tiles == 1 ? f.grp : f.grp / p.row_tiles;
#pragma unroll
        for (int x = 0; x < GROUPS; x++) S::load_values(vr, x, (const T*)p.v_pages + row_at(f_page[x], fh, fk + 16 * x) * C, g, i);
    };
    auto advance = [&]() __attribute__((always_inline)) {               // on to the step that was just loaded, and the one behind it
        s = f;
        k0 = fk;
#pragma unroll
        for (int x = 0; x < GROUPS; x++) page[x] = f_page[x];
        have = true;
        if (goes_on(fk, STRIDE, min(f.len, f.t1 * KW))) {
            fk += STRIDE;
        } else if (SPLIT && left > kPaLead) {
            if (++f.grp == groups) {
                f.grp = 0;
                f.b++;
                enter_next(f);
            }
            f.t0 = 0;
            f.t1 = min(f.n_steps, left - kPaLead);
            left -= f.t1 + kPaLead;
            fk = 0;
        } else {
            more = false;
        }
        if (more) pages_at(f_page, f, fk);
    };
    if constexpr (!SPLIT) {       // one segment: its query rows are the first to be read
        begin();
        load_keys();
        load_values();
        advance();
    }

    for (;;) {
        f32x4 sc[RT][GROUPS];
        int held = 0;
        bool whole = false;
        if (have) {
            if constexpr (SPLIT)
                if (k0 == s.t0 * KW) begin();
#pragma unroll
            for (int x = 0; x < GROUPS; x++) held |= page[x] >= 0 ? 1 << x : 0;
            whole = k0 + KW <= all_see && held == (1 << GROUPS) - 1;
#pragma unroll
            for (int x = 0; x < GROUPS; x++) {
                const int key0 = k0 + 16 * x + 4 * g;
                f32x4 bias[RT];
                if constexpr (NF > 0) {
#pragma unroll
                    for (int rt = 0; rt < RT; rt++) {
                        bias[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int y = 0; y < NF; y++)
                            bias[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(factor(fr[x], y), row[rt].phi_q[y], bias[rt], 0, 0, 0);
                    }
                    if constexpr (BIAS == kBiasFactors) {
                        const PT* pk = (const PT*)p.phi_pages + (row_at(page[x], h, k0 + 16 * x) + i) * p.R;
                        for (int y = 4; 4 * y < p.R; y++) {
                            const bool in = 4 * y + g < p.R;
                            const float a = in ? (float)pk[4 * y + g] : 0.f;
#pragma unroll
                            for (int rt = 0; rt < RT; rt++) {
                                const float f = in && row[rt].has ? (float)row[rt].pq[4 * y + g] : 0.f;
                                bias[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, f, bias[rt], 0, 0, 0);
                            }
                        }
                    }
                }
#pragma unroll
                for (int rt = 0; rt < RT; rt++) {
                    f32x4 z = S::scores(kr, x, row[rt].q);
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        if constexpr (NF > 0) z[r] = fmaf(z[r], p.scale, bias[rt][r]);
                        else z[r] *= p.scale;
                        if constexpr (BIAS == kBiasAlibi) z[r] = fmaf(row[rt].slope, (float)(key0 + r - row[rt].pos), z[r]);
                    }
                    if (!whole) {
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (key0 + r >= row[rt].limit || !(held >> x & 1)) z[r] = -INFINITY;
                    }
                    sc[rt][x] = z;
                }
            }
        }
        if (more) load_keys();
        if (have) {
            // ---- softmax of the rows ----
            typename S::Probs pr[RT];
#pragma unroll
            for (int rt = 0; rt < RT; rt++) {
                Row& w = row[rt];
                float mx = w.m;
#pragma unroll
                for (int x = 0; x < GROUPS; x++)
#pragma unroll
                    for (int r = 0; r < 4; r++) mx = fmaxf(mx, sc[rt][x][r]);
                mx = column_max(mx);
                if (__any(mx > w.m)) {
                    const float alpha = weight(w.m, mx);
                    w.l *= alpha;
#pragma unroll
                    for (int t = 0; t < NV; t++)
#pragma unroll
                        for (int r = 0; r < 4; r++) w.o[t][r] *= alpha;
                    w.m = mx;
                }
                const float ref = w.m == -INFINITY ? 0.f : w.m;
#pragma unroll
                for (int x = 0; x < GROUPS; x++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        sc[rt][x][r] = fast_exp2((sc[rt][x][r] - ref) * kLog2e);
                        w.l += sc[rt][x][r];
                    }
                pr[rt] = S::probs(sc[rt]);
            }
            // ---- values ----
            // Values a row does not see may be anything (0 * inf is NaN), so around the last keys rows of different limits are
            // done one limit after the other, the largest first, with the values behind it cleared.
            unsigned long long todo[RT], any = 0;
            bool mine[RT];
#pragma unroll
            for (int rt = 0; rt < RT; rt++) {
                todo[rt] = whole ? ~0ull : __ballot(row[rt].limit > k0);
                mine[rt] = true;
                any |= todo[rt];
            }
            while (any != 0) {
                any = 0;
                if (!whole) {
                    int cut = 0;
#pragma unroll
                    for (int rt = 0; rt < RT; rt++) cut = max(cut, todo[rt] >> lane & 1 ? min(row[rt].limit, k0 + KW) : 0);
#pragma unroll
                    for (int d = 1; d < 16; d *= 2) cut = max(cut, __shfl_xor(cut, d));
#pragma unroll
                    for (int rt = 0; rt < RT; rt++) {
                        mine[rt] = min(row[rt].limit, k0 + KW) == cut;
                        todo[rt] &= ~__ballot(mine[rt]);
                        any |= todo[rt];
                    }
#pragma unroll
                    for (int x = 0; x < GROUPS; x++)
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (k0 + 16 * x + 4 * g + r >= cut || !(held >> x & 1)) vr.x[x][r] = {};
                }
#pragma unroll
                for (int t = 0; t < NV; t++)
#pragma unroll
                    for (int rt = 0; rt < RT; rt++) {
                        const f32x4 d = S::product(vr, t, pr[rt], row[rt].o[t]);
#pragma unroll
                        for (int r = 0; r < 4; r++) row[rt].o[t][r] = mine[rt] ? d[r] : row[rt].o[t][r];
                    }
            }
        }
        if (more) load_values();
        if (have && !goes_on(k0, STRIDE, min(s.len, s.t1 * KW))) {
            // ---- a segment ends ----
#pragma unroll
            for (int rt = 0; rt < RT; rt++) {
                row[rt].l = column_sum(row[rt].l);
                if (row[rt].limit <= 0) {                 // a row that sees nothing went along with the others
                    row[rt].m = -INFINITY;
                    row[rt].l = 0.f;
                }
            }
            if constexpr (SPLIT) {
                // The lane's channels of its row: 4 NV adjacent ones from 4 g NV on.
                const bool all = s.t0 == 0 && s.t1 == s.n_steps;
#pragma unroll
                for (int rt = 0; rt < RT; rt++) {
                    const Row& w = row[rt];
                    if (all && w.has) {
                        const float inv = w.l == 0.f ? 0.f : 1.f / w.l;
                        struct alignas(4 * NV * sizeof(T) < 16 ? 4 * NV * sizeof(T) : 16) Mine { T x[4 * NV]; } v;
#pragma unroll
                        for (int r = 0; r < 4; r++)
#pragma unroll
                            for (int t = 0; t < NV; t++) v.x[r * NV + t] = (T)(w.l == 0.f ? 0.f : w.o[t][r] * inv);
                        const long long at = row_base + 16 * rt + i;
                        *(Mine*)((T*)p.out + at * C + 4 * g * NV) = v;
                        if (g == 0) p.lse[at] = w.l == 0.f ? -INFINITY : w.m + __log2f(w.l) * kLn2;
                    }
                    if (!all && w.has) {
                        const long long at = ((long long)worker * 2 + (s.t0 > 0 ? 0 : 1)) * min(ROWS, rows_all) + 16 * rt + i;
                        struct alignas(16) Mine { float x[4 * NV]; } v;
#pragma unroll
                        for (int r = 0; r < 4; r++)
#pragma unroll
                            for (int t = 0; t < NV; t++) v.x[r * NV + t] = w.o[t][r];
                        *(Mine*)(p.part_o + at * C + 4 * g * NV) = v;
                        if (g == 0) {
                            p.part_m[at] = w.m;
                            p.part_l[at] = w.l;
                        }
                    }
                }
                // The group's first worker says who has the rest; a share that ends inside a group ends with its step t1.
                if (lane == 0) {
                    int rest = 0;
                    if (s.t0 == 0 && s.t1 < s.n_steps) rest = share.worker_of(share.u_end - 1 + s.n_steps - s.t1) - worker;
                    const int4 join = make_int4(rest, worker, s.b * groups + s.grp, rows);
                    if (p.joins_by_group) {
                        if (s.t0 == 0) p.joins[join.z] = join;
                    } else if (!more) {
                        p.joins[worker] = join;
                    }
                }
            } else {
                // ---- the waves of the workgroup ----
                extern __shared__ __align__(16) float sm_parts[];
                constexpr int PITCH = C + 4;                              // rows start in different banks
                const int part_rows = min(ROWS, rows_all);
                float* sm_m = sm_parts + W * part_rows * PITCH;
                float* sm_l = sm_m + W * part_rows;
#pragma unroll
                for (int rt = 0; rt < RT; rt++)
                    if (row[rt].has) {
                        const int at = wave * part_rows + 16 * rt + i;
#pragma unroll
                        for (int r = 0; r < 4; r++)
#pragma unroll
                            for (int t = 0; t < NV; t++) sm_parts[at * PITCH + (4 * g + r) * NV + t] = row[rt].o[t][r];
                        if (g == 0) {
                            sm_m[at] = row[rt].m;
                            sm_l[at] = row[rt].l;
                        }
                    }
                __syncthreads();
                for (int x = tid; x < rows * (C / 4); x += pa_threads(W)) {
                    const int r = x / (C / 4), c4 = x % (C / 4);
                    float mx = sm_m[r];
#pragma unroll
                    for (int w = 1; w < W; w++) mx = fmaxf(mx, sm_m[w * part_rows + r]);
                    float lt = 0.f;
                    f32x4 ot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < W; w++) {
                        const float a = weight(sm_m[w * part_rows + r], mx);
                        const f32x4 y = *(const f32x4*)&sm_parts[(w * part_rows + r) * PITCH + c4 * 4];
                        lt = fmaf(a, sm_l[w * part_rows + r], lt);
#pragma unroll
                        for (int e = 0; e < 4; e++) ot[e] = fmaf(a, y[e], ot[e]);
                    }
                    write_row<T, C>(p, row_base + r, c4, ot, lt, mx);
                }
            }
        }
        if (!more) return;
        advance();
    }
}

// Joins the parts of a group's rows: part 1 of the worker where the group begins and part 0 of the `more` workers behind
// it.  A workgroup takes `8 / lanes` rows of one group, `lanes` parts at a time.
template <typename T, int C>
__global__ __launch_bounds__(2 * C) void paged_join_kernel(PagedAttnParams p, int lanes) {
    constexpr int LN = C / 4, SL = 8;                     // threads of a row, (row, part) slots
    __shared__ __align__(16) float sm_o[SL][C];
    __shared__ float sm_l[SL];
    const int4 join = p.joins[blockIdx.x];
    const int more = join.x, first = join.y;
    const int tid = threadIdx.x, c4 = tid % LN, slot = tid / LN, lane = slot % lanes;
    const int r = blockIdx.y * (SL / lanes) + slot / lanes;
    if (more == 0) return;                                // (uniform)
    const bool has_row = r < join.w;
    const int part_rows = min(p.tile_rows, p.G * p.N);
    auto part = [&](int k) { return ((long long)(first + k) * 2 + (k == 0 ? 1 : 0)) * part_rows + (has_row ? r : 0); };

    // the slot's parts, and then the slots', each by the running maximum
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = lane; k0 <= more; k0 += 4 * lanes) {
        float pm[4], pl[4];
        f32x4 po[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {                     // behind the last: the last again, weighing nothing
            const long long at = part(min(k0 + j * lanes, more));
            pm[j] = k0 + j * lanes <= more ? p.part_m[at] : -INFINITY;
            pl[j] = p.part_l[at];
            po[j] = *(const f32x4*)(p.part_o + at * C + c4 * 4);
        }
        const float mx = fmaxf(fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])), m);
        const float a = weight(m, mx);
        l *= a;
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] *= a;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float w = weight(pm[j], mx);
            if (k0 + j * lanes <= more) {
                l = fmaf(w, pl[j], l);
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] = fmaf(w, po[j][e], o[e]);
            }
        }
        m = mx;
    }
    __shared__ float sm_m[SL];
    *(f32x4*)&sm_o[slot][c4 * 4] = o;
    if (c4 == 0) {
        sm_l[slot] = l;
        sm_m[slot] = m;
    }
    __syncthreads();
    if (lane != 0 || !has_row) return;
    float mx = m;
    for (int k = 1; k < lanes; k++) mx = fmaxf(mx, sm_m[slot + k]);
    float lt = 0.f;
    f32x4 ot = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < lanes; k++) {
        const float w = weight(sm_m[slot + k], mx);
        const f32x4 x = *(const f32x4*)&sm_o[slot + k][c4 * 4];
        lt = fmaf(w, sm_l[slot + k], lt);
#pragma unroll
        for (int e = 0; e < 4; e++) ot[e] = fmaf(w, x[e], ot[e]);
    }
    const int b = join.z / (p.Hkv * p.row_tiles), grp = join.z - b * p.Hkv * p.row_tiles;
    const int h = grp / p.row_tiles, r0 = (grp - h * p.row_tiles) * p.tile_rows;
    write_row<T, C>(p, (long long)b * p.H * p.N + (long long)h * (p.G * p.N) + r0 + r, c4, ot, lt, mx);
}

template <typename T, int C, int BIAS, bool PF32, int W, int RT>
int launch_groups(PagedAttnParams p, hipStream_t stream) {
    const long long blocks = (long long)p.B * p.Hkv * p.row_tiles;       // at most B H N, below 2^31
    const int rows = p.G * p.N < 16 * RT ? p.G * p.N : 16 * RT;
    if constexpr (group_lds(W, 16 * RT, C) > 65536) {
        static FbLdsOnce once;
        if (!fb_raise_lds_limit((const void*)paged_attn_kernel<T, C, BIAS, PF32, W, RT>, group_lds(W, 16 * RT, C), once)) return 1;
    }
    const size_t lds = group_lds(W, rows, C);
    for (long long block0 = 0; block0 < blocks; block0 += kFbLaunchBlocks) {
        p.block0 = (unsigned)block0;
        hipLaunchKernelGGL((paged_attn_kernel<T, C, BIAS, PF32, W, RT>), dim3((unsigned)std::min(blocks - block0, kFbLaunchBlocks)),
                           dim3(pa_threads(W)), lds, stream, p);
    }
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

template <typename T, int C, int BIAS, bool PF32>
int launch_attn(const PagedAttnParams& p, hipStream_t stream) {
    if (p.workers == 0) {
        if constexpr (two_tiles(C, std::is_same_v<T, float>)) {
            if (p.tile_rows == 32) return launch_groups<T, C, BIAS, PF32, 4, 2>(p, stream);
        }
        return p.waves == 8 ? launch_groups<T, C, BIAS, PF32, 8, 1>(p, stream) : launch_groups<T, C, BIAS, PF32, 4, 1>(p, stream);
    }
    const dim3 blocks((unsigned)((p.workers + kPaWaves - 1) / kPaWaves));
    if constexpr (two_tiles(C, std::is_same_v<T, float>)) {
        if (p.tile_rows == 32) hipLaunchKernelGGL((paged_attn_kernel<T, C, BIAS, PF32, 1, 2>), blocks, dim3(kPaThreads), 0, stream, p);
    }
    if (p.tile_rows == 16) hipLaunchKernelGGL((paged_attn_kernel<T, C, BIAS, PF32, 1, 1>), blocks, dim3(kPaThreads), 0, stream, p);
    if (hipGetLastError() != hipSuccess) return 1;
    const long long groups = (long long)p.B * p.Hkv * p.row_tiles;
    const int rows = p.G * p.N < p.tile_rows ? p.G * p.N : p.tile_rows;
    // slots: as many parts at a time as a group has on average, the rest are rows
    const long long parts = p.workers / groups;
    const int lanes = parts >= 6 ? 8 : (parts >= 3 ? 4 : 2);
    const dim3 grid((unsigned)(p.joins_by_group ? groups : p.workers), (unsigned)((rows * lanes + 7) / 8));
    hipLaunchKernelGGL((paged_join_kernel<T, C>), grid, dim3(2 * C), 0, stream, p, lanes);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

template <typename T, int C, bool PF32>
int attn_factors(const PagedAttnParams& p, hipStream_t stream) {
    if (p.R <= 4) return launch_attn<T, C, kBiasFactors4, PF32>(p, stream);
    if (p.R <= 16 && p.R % 4 == 0) return launch_attn<T, C, kBiasFactors16, PF32>(p, stream);
    return launch_attn<T, C, kBiasFactors, PF32>(p, stream);
}

template <typename T, int C>
int attn_bias(const PagedAttnParams& p, hipStream_t stream) {
    if (p.slopes) return launch_attn<T, C, kBiasAlibi, true>(p, stream);
    if (p.R == 0) return launch_attn<T, C, kBiasNone, true>(p, stream);
    if constexpr (!std::is_same_v<T, float>) {
        if (!p.phi_f32) return attn_factors<T, C, false>(p, stream);
    }
    return attn_factors<T, C, true>(p, stream);
}

template <typename T>
int attn_channels(const PagedAttnParams& p, int C, hipStream_t stream) {
    switch (C) {
        case 16: return attn_bias<T, 16>(p, stream);
        case 32: return attn_bias<T, 32>(p, stream);
        case 64: return attn_bias<T, 64>(p, stream);
        case 128: return attn_bias<T, 128>(p, stream);
        default: return -1;
    }
}

}  // namespace

// rows: query rows of a key head
static size_t parts_of(int workers, long long rows, int tile_rows) {
    return (size_t)workers * 2 * (rows < tile_rows ? rows : tile_rows);
}

// Waves that share the keys: all that are resident.  Short requests (by the table's width) are not split: a turn of a workgroup's
// waves takes a memory latency, 1.2 us at C = 64 and 1.7 at 128, the split's bookkeeping, its join and the launch of
// that 5 us on either side of the queue.  us without / with the split, on the GPU; as calls one after the other:
//   bf16 C 64, 16 groups 1024 keys 10.6 / 11.0; 11.6 / 16.5, 1536 keys 16.5 / 11.2; 15.7 / 16.2; 1024 groups 1024 keys 46 / 50; 44 / 50
//   bf16 C 128, 16 groups 640 keys 11.6 / 13.0; 11.4 / 16.2, 1024 keys 16.8 / 13.2; 16.2 / 16.2
//   fp32 C 64, 16 groups 512 keys 11.2 / 11.2; 11.7 / 16.3, 768 keys 16.0 / 11.4; 15.4 / 16.5; C 128 320 keys 12.6 / 14.3; 11.7 / 16.1
//
// Two tiles of 16 rows read a key once, for a longer step and twice the parts.  That pays where the loads bound the call: in bf16 at
// 64 and 128 channels (fp32 is bound by its matrix products, 16 and 32 channels by the softmax: N 20, B 8, H 16, C 16 31.2 / 35.4 us
// with 16 / 32 rows, C 32 38.4 / 38.8; B 32, H 8 / 4, fp32 C 64 83 / 96), and from 12 steps a wave on or, without a split, three groups
// per CU of more than two turns.  us with 16 / 32 rows, N 20, H = Hkv = 16:
//   up to 8200 keys, C 128: B 1 36 / 42, 2 39 / 43, 3 50 / 49, 4 58 / 53, 8 99 / 73, with 64 rows 173 / 128; C 64: B 2 27 / 31, 4 37 / 36,
//   6 44 / 41, 8 54 / 47
//   no split, C 128, 300 keys: B 8 16 / 23, 16 23 / 24, 24 33 / 28, 128 132 / 108; C 64, 1024 keys: B 16 30 / 29, 32 49 / 37; 112 keys: B 64
//   28 / 31
PagedAttnSplit fb_paged_attn_split(int B, int Hkv, long long rows, long long capacity, int C, bool f32) {
    PagedAttnSplit s;
    const int step = 16 * step_groups(C, f32);
    const long long steps = (capacity + step - 1) / step;
    int cus = fb_cu_count();
    if (cus <= 0) cus = 256;
    long long groups = (long long)B * Hkv * ((rows + 15) / 16);
    // (costs are counted in 32 bits)
    const bool split = capacity > (C == 128 ? 640 : 1024) / (f32 ? 2 : 1) && steps + kPaLead < (1LL << 31) / groups;
    const bool large = split ? steps * groups >= 12LL * 4 * waves_per_simd(C, 1) * cus : groups >= 3LL * cus && capacity > 2 * 4 * step;
    s.tile_rows = rows > 16 && two_tiles(C, f32) && large ? 32 : 16;
    s.row_tiles = (int)((rows + s.tile_rows - 1) / s.tile_rows);
    groups = (long long)B * Hkv * s.row_tiles;
    const long long most = groups * ((steps + kPaLeast - 1) / kPaLeast), all = 4LL * waves_per_simd(C, s.tile_rows / 16) * cus;
    s.workers = !split ? 0 : (int)(most < all ? most : all);
    s.bytes = 0;
    if (split) {
        const size_t joins = (size_t)(groups < s.workers ? groups : s.workers);
        s.bytes = parts_of(s.workers, rows, s.tile_rows) * (C + 2) * sizeof(float) + joins * sizeof(int4);
    }
    return s;
}

int fb_launch_paged_attn(PagedAttnParams p, int C, bool f32, void* ws, hipStream_t stream) {
    p.G = p.H / p.Hkv;
    p.inv_n = 1.0f / (float)p.N;
    const long long capacity = (long long)p.max_blocks << p.page_shift;
    p.capacity = capacity < 0x7fffff00 ? (int)capacity : 0x7fffff00;
    if (p.workers) {
        const long long groups = (long long)p.B * p.Hkv * p.row_tiles;
        const size_t parts = parts_of(p.workers, (long long)p.G * p.N, p.tile_rows);
        p.joins_by_group = groups <= p.workers;
        p.joins = (int4*)ws;
        p.part_o = (float*)(p.joins + (p.joins_by_group ? groups : p.workers));
        p.part_m = p.part_o + parts * C;
        p.part_l = p.part_m + parts;
    }
    // Eight waves a group where every group has a CU of its own and four would take more than two turns.  us with four / eight,
    // C 64: 16 groups 128 keys 4.5 / 5.3, 512 keys 7.3 / 6.6, 1024 keys 10.9 / 9.2; 128 groups 512 keys 8.9 / 7.3, 1024 keys 15.1 /
    // 11.4; 576 groups 17.0 / 19.6, 28.5 / 31.5.  C 128, 128 groups, 512 keys 11.8 / 11.5; fp32 C 64 15.9 / 12.8.
    p.waves = (long long)p.B * p.Hkv * p.row_tiles <= fb_cu_count() && capacity > 2 * 4 * 16 * step_groups(C, f32) ? 8 : 4;
    return f32 ? attn_channels<float>(p, C, stream) : attn_channels<bf16_t>(p, C, stream);
}
