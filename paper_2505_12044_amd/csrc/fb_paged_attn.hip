// Attention of a few new tokens per request over a paged key-value cache, gfx950.
//
//     out = softmax(q k^T scale + b) v  over the request's own keys, causal for the new tokens among themselves;
// b: none, low-rank factors phi_q phi_k^T (phi_k in pages beside the keys), or ALiBi -m_h (i - j).  G = H / Hkv query
// heads share a key head, so the G N rows that meet the same keys form one tile of 16 rows (several where there are more).
//
// Bound by memory: every key and value row is read once per row tile, 4 C flops per row and key against 4 C bytes per
// key (bf16).  The matrix pipe has twenty times the rate that needs, so the 16-row tile runs whatever G N is:
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
// where no request can be long, a workgroup's four waves share one group and join through LDS.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fb_device.h"
#include "fb_launch.h"
#include "fb_params.h"

namespace {

constexpr int kPaWaves = 4;
constexpr int kPaThreads = kPaWaves * 64;
constexpr int kPaRows = 16;
constexpr int kPaLeast = 4;       // steps of a worker's share at least (the join of smaller shares costs more than they save)

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
// Lane l: g = l / 16, i = l % 16.  S^T group s (16 keys): column i (the query row), keys 4 g + r.
template <typename T, int C>
struct Step;

template <int C>
struct Step<bf16_t, C> {
    static constexpr int KW = 32, GROUPS = 2, NV = C / 16;
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
        for (int r = 0; r < 4; r++) v.x[s][r] = *(const VVec*)(rows + (4 * g + r) * C + i * NV);
    }
    static FB_DEV f32x4 scores(const Keys& k, int s, const Query& q) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < NU; u++) {
            if constexpr (C == 16)
                acc = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, k.x[s][u]), __builtin_bit_cast(s16x4, q.x[u]), acc, 0, 0, 0);
            else
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k.x[s][u]), __builtin_bit_cast(bf16x8, q.x[u]), acc, 0, 0, 0);
        }
        return acc;
    }
    struct Probs { bf16x8 hi, lo; };
    static FB_DEV Probs probs(const f32x4 (&p)[GROUPS]) {
        Probs w;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float x = p[e / 4][e % 4];
            w.hi[e] = (bf16_t)x;
            w.lo[e] = (bf16_t)(x - (float)w.hi[e]);
        }
        return w;
    }
    // 32-bit word of channels 2 w, 2 w + 1 (of the lane's NV) of key e
    static FB_DEV unsigned word(const Values& v, int e, int w) {
        const VVec x = v.x[e / 4][e % 4];
        if constexpr (NV <= 2) return x;
        else return x[w];
    }
    // o[t] += channel t's values times the probabilities
    static FB_DEV f32x4 product(const Values& v, int t, const Probs& p, f32x4 o) {
        u32x4 a;
#pragma unroll
        for (int j = 0; j < 4; j++)
            a[j] = __builtin_amdgcn_perm(word(v, 2 * j + 1, t / 2), word(v, 2 * j, t / 2), t % 2 ? 0x07060302u : 0x05040100u);
        o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), p.hi, o, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), p.lo, o, 0, 0, 0);
    }
};

template <int C>
struct Step<float, C> {
    static constexpr int KW = 16, GROUPS = 1, NV = C / 16;
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
        for (int r = 0; r < 4; r++) v.x[s][r] = *(const VVec*)(rows + (4 * g + r) * C + i * NV);
    }
    static FB_DEV f32x4 scores(const Keys& k, int s, const Query& q) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < NU; u++)
#pragma unroll
            for (int e = 0; e < 4; e++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[s][u][e], q.x[u][e], acc, 0, 0, 0);
        return acc;
    }
    struct Probs { f32x4 x; };
    static FB_DEV Probs probs(const f32x4 (&p)[GROUPS]) { return Probs{p[0]}; }
    static FB_DEV f32x4 product(const Values& v, int t, const Probs& p, f32x4 o) {
#pragma unroll
        for (int r = 0; r < 4; r++) {
            float a;
            if constexpr (NV == 1) a = v.x[0][r];
            else a = v.x[0][r][t];
            o = __builtin_amdgcn_mfma_f32_16x16x4f32(a, p.x[r], o, 0, 0, 0);
        }
        return o;
    }
};

enum { kBiasNone = 0, kBiasAlibi = 1, kBiasFactors4 = 2, kBiasFactors = 3 };    // factors: up to 4, any number

// Arrays that are not written while the kernel runs, read at wave-uniform places: scalar loads, which do not queue behind
// the rows in flight.
typedef const __attribute__((address_space(4))) int* ConstInts;
FB_DEV ConstInts const_ints(const int* x) { return (ConstInts)(uintptr_t)x; }

FB_DEV int held_keys(const PagedAttnParams& p, int b) {
    return max((int)min((long long)const_ints(p.lens)[b], (long long)p.max_blocks << p.page_shift), 0);
}

// Steps of a request per group; one that holds nothing has one too (its rows are written).
template <int KW>
FB_DEV int steps_of(int len) { return len > KW ? (len + KW - 1) / KW : 1; }

// Inclusive sums over the wave.
FB_DEV long long wave_scan(long long x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const long long y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// The steps of all requests laid end to end, cut in equal shares: where this wave's begins and ends.  `total`, `workers`
// (those that have a share), `u`, `u_end`: steps; b, rem: the request that step u lies in and its place there.
struct Share {
    long long total, u, u_end, rem;
    int workers, b;
};

template <int KW>
FB_DEV Share share_of(const PagedAttnParams& p, int groups, int worker) {
    __shared__ long long sm_sum[kPaWaves];
    __shared__ long long sm_rem[kPaWaves];
    __shared__ int sm_b[kPaWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Share s{};
    const auto cut = [&]() {
        s.workers = (int)min((long long)p.workers, (s.total + kPaLeast - 1) / kPaLeast);
        s.u = worker * s.total / s.workers;
        s.u_end = worker < s.workers ? (worker + 1) * s.total / s.workers : s.u;
    };
    if (p.B <= 64) {                                     // every wave by itself
        const long long own = lane < p.B ? (long long)steps_of<KW>(max((int)min((long long)p.lens[lane], (long long)p.max_blocks << p.page_shift), 0)) * groups : 0;
        const long long end = wave_scan(own);
        s.total = __shfl(end, 63);
        cut();
        if (s.u < s.u_end) {
            s.b = __builtin_ctzll(__ballot(end > s.u));
            s.rem = s.u - __shfl(end - own, s.b);
        }
        return s;
    }
    // the workgroup's four shares together, 256 requests at a time: the total first
    const auto tile = [&](int b0, long long& own, long long& sum) {
        const int b = b0 + tid;
        own = b < p.B ? (long long)steps_of<KW>(max((int)min((long long)p.lens[b], (long long)p.max_blocks << p.page_shift), 0)) * groups : 0;
        const long long in_wave = wave_scan(own);
        __syncthreads();
        if (lane == 63) sm_sum[wave] = in_wave;
        __syncthreads();
        long long before = 0;
        sum = 0;
#pragma unroll
        for (int w = 0; w < kPaWaves; w++) {
            if (w < wave) before += sm_sum[w];
            sum += sm_sum[w];
        }
        return before + in_wave;
    };
    long long own, sum;
    for (int b0 = 0; b0 < p.B; b0 += kPaThreads) {
        tile(b0, own, sum);
        s.total += sum;
    }
    cut();
    long long before = 0;
    for (int b0 = 0; b0 < p.B; b0 += kPaThreads) {
        const long long end = before + tile(b0, own, sum);
        for (int w = 0; w < kPaWaves; w++) {
            const int k = worker - wave + w;
            const long long u = k * s.total / s.workers;
            if (end - own <= u && u < end) {
                sm_b[w] = b0 + tid;
                sm_rem[w] = u - (end - own);
            }
        }
        before += sum;
    }
    __syncthreads();
    s.b = sm_b[wave];                                    // (waves without a share do not read on)
    s.rem = sm_rem[wave];
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
    int b, len, n_steps, grp, t0, t1;
};

// BIAS, PF32: kind of bias and whether the factors are float
template <typename T, int C, int BIAS, bool PF32, bool SPLIT>
__global__ __launch_bounds__(kPaThreads, 2) void paged_attn_kernel(PagedAttnParams p) {
    using S = Step<T, C>;
    constexpr int KW = S::KW, NV = S::NV, GROUPS = S::GROUPS;
    constexpr int STRIDE = SPLIT ? KW : kPaWaves * KW;    // keys from one step of a wave to its next
    constexpr int NF = BIAS == kBiasFactors4 ? 1 : (BIAS == kBiasFactors ? 4 : 0);
    using PT = std::conditional_t<PF32, float, bf16_t>;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, i = lane & 15;
    const int groups = p.Hkv * p.row_tiles;               // of a request
    const int rows_all = p.H / p.Hkv * p.N;
    const int part_rows = min(kPaRows, rows_all);
    const int page_mask = (1 << p.page_shift) - 1;

    Segment seg;
    Share share{};
    const int worker = blockIdx.x * kPaWaves + wave;
    long long left = 0;                                   // steps of this worker behind the segment
    if constexpr (SPLIT) {
        share = share_of<KW>(p, groups, worker);
        if (share.u >= share.u_end) {
            if (!p.joins_by_group && worker < p.workers && lane == 0) p.joins[worker] = make_int4(0, 0, 0, 0);
            return;
        }
        seg.b = __builtin_amdgcn_readfirstlane(share.b);
        seg.len = held_keys(p, seg.b);
        seg.n_steps = steps_of<KW>(seg.len);
        const unsigned rem = __builtin_amdgcn_readfirstlane((int)share.rem);      // < groups * steps of one request < 2^31
        seg.grp = (int)(rem / (unsigned)seg.n_steps);
        seg.t0 = (int)rem - seg.grp * seg.n_steps;
        left = share.u_end - share.u;
        left = ((long long)__builtin_amdgcn_readfirstlane((int)(left >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)left);
        seg.t1 = (int)min((long long)seg.n_steps, seg.t0 + left);
        left -= seg.t1 - seg.t0;
    } else {
        seg.b = blockIdx.x / groups;
        seg.grp = blockIdx.x - seg.b * groups;
        seg.len = held_keys(p, seg.b);
        seg.t0 = 0;
        seg.t1 = seg.n_steps = steps_of<KW>(seg.len);
    }
    int4 join = make_int4(0, 0, 0, 0);

    // ---- what a step reads ----
    // pages of the 16-key groups from key k on (-1 behind `end`), and the first row of each in its page; a group whose page is
    // none is not visible, and the first rows of page 0 stand in for it
    auto pages_at = [&](int (&page)[GROUPS], const Segment& s, int k, int end) __attribute__((always_inline)) {
        const ConstInts table = const_ints(p.table) + (long long)s.b * p.max_blocks;
#pragma unroll
        for (int x = 0; x < GROUPS; x++) page[x] = k + 16 * x < end ? table[(k + 16 * x) >> p.page_shift] : -1;
    };
    auto rows_of = [&](long long (&row)[GROUPS], const int (&page)[GROUPS], int h, int k) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < GROUPS; x++)
            row[x] = (unsigned)page[x] < (unsigned)p.n_pages
                         ? (((long long)page[x] * p.Hkv + h) << p.page_shift) + ((k + 16 * x) & page_mask) : -1;
    };
    typename S::Keys kr;
    typename S::Values vr;
    PT fr[GROUPS][NF > 0 ? NF : 1];
    // Factors of one row, the lane's share: factor g (up to four), or 4 g .. 4 g + 3 of the first 16, at once where rows allow.
    const bool factors_x4 = NF == 4 && p.R % 4 == 0;
    auto load_factors = [&](PT (&f)[NF > 0 ? NF : 1], const PT* pk) __attribute__((always_inline)) {
        if (factors_x4) {
            struct alignas(4 * sizeof(PT)) Four { PT x[4]; } v = {};
            if (4 * g < p.R) v = *(const Four*)(pk + 4 * g);
#pragma unroll
            for (int y = 0; y < NF; y++) f[y] = v.x[y];
        } else {
#pragma unroll
            for (int y = 0; y < NF; y++) f[y] = NF * g + y < p.R ? pk[NF * g + y] : (PT)0.f;
        }
    };
    auto load_keys = [&](const long long (&row)[GROUPS]) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < GROUPS; x++) {
            const long long at = row[x] >= 0 ? row[x] : 0;
            S::load_keys(kr, x, (const T*)p.k_pages + at * C, g, i);
            if constexpr (NF > 0) {
                load_factors(fr[x], (const PT*)p.phi_pages + (at + i) * p.R);
            }
        }
    };
    auto load_values = [&](const long long (&row)[GROUPS]) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < GROUPS; x++) S::load_values(vr, x, (const T*)p.v_pages + (row[x] >= 0 ? row[x] : 0) * C, g, i);
    };
    auto first_key = [&](const Segment& s) { return s.t0 * KW + (SPLIT ? 0 : wave * KW); };
    auto key_end = [&](const Segment& s) { return min(s.len, s.t1 * KW); };

    // One step ahead: the next keys are loaded when the scores have used this step's, the next values after this step's
    // product; the next segment's first step counts as the last step's next.  Pages are read a step before that.
    long long row[GROUPS], next[GROUPS];
    int page[GROUPS];
    pages_at(page, seg, first_key(seg), key_end(seg));
    rows_of(row, page, seg.grp / p.row_tiles, first_key(seg));
    if (first_key(seg) < key_end(seg)) {
        load_keys(row);
        load_values(row);
    }

    for (;;) {
        const int h = seg.grp / p.row_tiles, r0 = (seg.grp - h * p.row_tiles) * kPaRows;
        const int rows = min(kPaRows, rows_all - r0), len = seg.len;
        const int start = p.starts ? min(max(const_ints(p.starts)[seg.b], -(1 << 30)), 1 << 30) : len - p.N;
        const long long row_base = (long long)seg.b * p.H * p.N + (long long)h * rows_all + r0;      // of q, out, lse

        // the lane's query row
        const bool has_row = i < rows;
        const int pos = start + (r0 + i) % p.N;
        const int limit = !has_row ? 0 : (p.causal ? (pos >= len || pos < 0 ? 0 : pos + 1) : len);      // keys the row sees
        const int all_see = p.causal ? max(min(start + 1, len), 0) : len;                               // keys every row sees
        typename S::Query q;
#pragma unroll
        for (int x = 0; x < S::NU; x++) {
            q.x[x] = {};
            if (has_row) q.x[x] = S::row_chunk((const T*)p.q + (row_base + i) * C, g, x);
        }
        float phi_q[4] = {0.f, 0.f, 0.f, 0.f};
        const PT* pq_row = nullptr;
        if constexpr (NF > 0) {
            pq_row = (const PT*)p.phi_q + (long long)seg.b * p.phiq_bstride + ((long long)h * rows_all + r0 + i) * p.R;
#pragma unroll
            for (int x = 0; x < NF; x++)
                if (has_row && NF * g + x < p.R) phi_q[x] = (float)pq_row[NF * g + x];
        }
        float slope = 0.f;
        if constexpr (BIAS == kBiasAlibi)
            if (has_row) slope = p.slopes[h * (p.H / p.Hkv) + (r0 + i) / p.N];

        Segment after = seg;                              // the worker's next segment
        const bool has_after = SPLIT && left > 0;
        if constexpr (SPLIT) {
            if (has_after) {
                after.grp++;
                if (after.grp == groups) {
                    after.grp = 0;
                    after.b++;
                    after.len = held_keys(p, after.b);
                    after.n_steps = steps_of<KW>(after.len);
                }
                after.t0 = 0;
                after.t1 = (int)min((long long)after.n_steps, left);
                left -= after.t1;
            }
        }

        float m = -INFINITY, l = 0.f;
        f32x4 o[NV];
#pragma unroll
        for (int t = 0; t < NV; t++) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

        const int k_end = key_end(seg);
        int k0 = first_key(seg);                          // wave-uniform
        const auto next_pages = [&](int k) __attribute__((always_inline)) {       // of the step behind the one at k - STRIDE
            if (k < k_end) pages_at(page, seg, k, k_end);
            else if (has_after) pages_at(page, after, first_key(after), key_end(after));
        };
        const bool idle = k0 >= k_end;                    // no keys at all: the next segment's first step is still to be loaded
        next_pages(k0 + STRIDE);
        if (idle && has_after) {
            rows_of(row, page, after.grp / p.row_tiles, 0);
            if (key_end(after) > 0) {
                load_keys(row);
                load_values(row);
            }
        }
        for (; k0 < k_end; k0 += STRIDE) {
            const bool more = k0 + STRIDE < k_end, load = more || (has_after && key_end(after) > 0);
            if (more) rows_of(next, page, h, k0 + STRIDE);
            else rows_of(next, page, after.grp / p.row_tiles, first_key(after));
            if (more) next_pages(k0 + 2 * STRIDE);
            bool whole = k0 + KW <= all_see;
#pragma unroll
            for (int s = 0; s < GROUPS; s++) whole = whole && row[s] >= 0;
            f32x4 sc[GROUPS];
#pragma unroll
            for (int s = 0; s < GROUPS; s++) {
                sc[s] = S::scores(kr, s, q);
                const int key0 = k0 + 16 * s + 4 * g;
                if constexpr (NF > 0) {
                    f32x4 f = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int x = 0; x < NF; x++) f = __builtin_amdgcn_mfma_f32_16x16x4f32((float)fr[s][x], phi_q[x], f, 0, 0, 0);
                    if constexpr (BIAS == kBiasFactors) {
                        const PT* pk = (const PT*)p.phi_pages + ((row[s] >= 0 ? row[s] : 0) + i) * p.R;
                        for (int x = 4; 4 * x < p.R; x++) {
                            const bool in = 4 * x + g < p.R;
                            const float a = in ? (float)pk[4 * x + g] : 0.f, c = in && has_row ? (float)pq_row[4 * x + g] : 0.f;
                            f = __builtin_amdgcn_mfma_f32_16x16x4f32(a, c, f, 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 4; r++) sc[s][r] = fmaf(sc[s][r], p.scale, f[r]);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        sc[s][r] *= p.scale;
                        if constexpr (BIAS == kBiasAlibi) sc[s][r] = fmaf(slope, (float)(key0 + r - pos), sc[s][r]);
                    }
                }
                if (!whole) {
#pragma unroll
                    for (int r = 0; r < 4; r++)
                        if (key0 + r >= limit || row[s] < 0) sc[s][r] = -INFINITY;
                }
            }
            if (load) load_keys(next);
            // ---- softmax of the rows ----
            float mx = m;
#pragma unroll
            for (int s = 0; s < GROUPS; s++)
#pragma unroll
                for (int r = 0; r < 4; r++) mx = fmaxf(mx, sc[s][r]);
            mx = column_max(mx);
            if (__any(mx > m)) {
                const float alpha = weight(m, mx);
                l *= alpha;
#pragma unroll
                for (int t = 0; t < NV; t++)
#pragma unroll
                    for (int r = 0; r < 4; r++) o[t][r] *= alpha;
                m = mx;
            }
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int s = 0; s < GROUPS; s++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    sc[s][r] = fast_exp2((sc[s][r] - ref) * kLog2e);
                    l += sc[s][r];
                }
            const typename S::Probs pr = S::probs(sc);
            // ---- values ----
            if (whole) {
#pragma unroll
                for (int t = 0; t < NV; t++) o[t] = S::product(vr, t, pr, o[t]);
            } else {
                // Values a row does not see may be anything (0 * inf is NaN), so rows of different limits are done one
                // after the other with the values behind their limit cleared; at most N of them, only around the last keys.
                unsigned long long todo = __ballot(limit > k0);
                while (todo != 0) {
                    const int cut = min(__builtin_amdgcn_readlane(limit, __builtin_ctzll(todo)), k0 + KW);
                    const bool mine = min(limit, k0 + KW) == cut;
                    typename S::Values vm = vr;
#pragma unroll
                    for (int s = 0; s < GROUPS; s++)
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (k0 + 16 * s + 4 * g + r >= cut || row[s] < 0) vm.x[s][r] = {};
#pragma unroll
                    for (int t = 0; t < NV; t++) {
                        const f32x4 d = S::product(vm, t, pr, o[t]);
#pragma unroll
                        for (int r = 0; r < 4; r++) o[t][r] = mine ? d[r] : o[t][r];
                    }
                    todo &= ~__ballot(mine);
                }
            }
            if (load) load_values(next);
#pragma unroll
            for (int s = 0; s < GROUPS; s++) row[s] = next[s];
        }

        l = column_sum(l);
        if (limit <= 0) {                                 // a row that sees nothing went along with the others
            m = -INFINITY;
            l = 0.f;
        }
        if constexpr (SPLIT) {
            // The lane's channels of row i: 4 NV adjacent ones from 4 g NV on.
            if (seg.t0 == 0 && seg.t1 == seg.n_steps) {
                if (has_row) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    struct alignas(4 * NV * sizeof(T) < 16 ? 4 * NV * sizeof(T) : 16) Mine { T x[4 * NV]; } v;
#pragma unroll
                    for (int r = 0; r < 4; r++)
#pragma unroll
                        for (int t = 0; t < NV; t++) v.x[r * NV + t] = (T)(l == 0.f ? 0.f : o[t][r] * inv);
                    *(Mine*)((T*)p.out + (row_base + i) * C + 4 * g * NV) = v;
                    if (g == 0) p.lse[row_base + i] = l == 0.f ? -INFINITY : m + __log2f(l) * kLn2;
                }
            } else if (has_row) {
                const long long at = ((long long)worker * 2 + (seg.t0 > 0 ? 0 : 1)) * part_rows + i;
                struct alignas(16) Mine { float x[4 * NV]; } v;
#pragma unroll
                for (int r = 0; r < 4; r++)
#pragma unroll
                    for (int t = 0; t < NV; t++) v.x[r * NV + t] = o[t][r];
                *(Mine*)(p.part_o + at * C + 4 * g * NV) = v;
                if (g == 0) {
                    p.part_m[at] = m;
                    p.part_l[at] = l;
                }
            }
            if (seg.t0 == 0) {                            // the group's first worker says who has the rest
                int more = 0;
                if (seg.t1 < seg.n_steps) {
                    // the group's last step is share.u_end - 1 + (n_steps - t1): here the share ends inside the group
                    const long long last = share.u_end - 1 + (seg.n_steps - seg.t1);
                    more = (int)(((last + 1) * share.workers - 1) / share.total) - worker;
                }
                const int4 mine = make_int4(more, worker, (int)((long long)seg.b * groups + seg.grp), rows);
                if (p.joins_by_group) {
                    if (lane == 0) p.joins[mine.z] = mine;
                } else if (more > 0) {
                    join = mine;
                }
            }
            if (!has_after) break;
            seg = after;
        } else {
            // ---- the waves of the workgroup ----
            __shared__ __align__(16) float sm_o[kPaWaves][kPaRows][C + 4];      // + 4: rows start in different banks
            __shared__ float sm_m[kPaWaves][kPaRows], sm_l[kPaWaves][kPaRows];
            if (has_row) {
#pragma unroll
                for (int r = 0; r < 4; r++)
#pragma unroll
                    for (int t = 0; t < NV; t++) sm_o[wave][i][(4 * g + r) * NV + t] = o[t][r];
                if (g == 0) {
                    sm_m[wave][i] = m;
                    sm_l[wave][i] = l;
                }
            }
            __syncthreads();
            for (int x = tid; x < rows * (C / 4); x += kPaThreads) {
                const int r = x / (C / 4), c4 = x % (C / 4);
                float mx = sm_m[0][r];
#pragma unroll
                for (int w = 1; w < kPaWaves; w++) mx = fmaxf(mx, sm_m[w][r]);
                float lt = 0.f;
                f32x4 ot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kPaWaves; w++) {
                    const float a = weight(sm_m[w][r], mx);
                    const f32x4 y = *(const f32x4*)&sm_o[w][r][c4 * 4];
                    lt = fmaf(a, sm_l[w][r], lt);
#pragma unroll
                    for (int e = 0; e < 4; e++) ot[e] = fmaf(a, y[e], ot[e]);
                }
                write_row<T, C>(p, row_base + r, c4, ot, lt, mx);
            }
            break;
        }
    }
    if constexpr (SPLIT)
        if (!p.joins_by_group && lane == 0) p.joins[worker] = join;
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
    const int part_rows = min(kPaRows, p.H / p.Hkv * p.N);
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
    const int h = grp / p.row_tiles, r0 = (grp - h * p.row_tiles) * kPaRows;
    write_row<T, C>(p, (long long)b * p.H * p.N + (long long)h * (p.H / p.Hkv * p.N) + r0 + r, c4, ot, lt, mx);
}

template <typename T, int C, int BIAS, bool PF32>
int launch_attn(const PagedAttnParams& p, hipStream_t stream) {
    if (p.workers == 0) {
        const long long blocks = (long long)p.B * p.Hkv * p.row_tiles;
        if (blocks >= (1LL << 31)) return -1;
        hipLaunchKernelGGL((paged_attn_kernel<T, C, BIAS, PF32, false>), dim3((unsigned)blocks), dim3(kPaThreads), 0, stream, p);
        return hipGetLastError() == hipSuccess ? 0 : 1;
    }
    hipLaunchKernelGGL((paged_attn_kernel<T, C, BIAS, PF32, true>), dim3((unsigned)((p.workers + kPaWaves - 1) / kPaWaves)), dim3(kPaThreads), 0,
                       stream, p);
    if (hipGetLastError() != hipSuccess) return 1;
    const long long groups = (long long)p.B * p.Hkv * p.row_tiles;
    const int rows = p.H / p.Hkv * p.N < kPaRows ? p.H / p.Hkv * p.N : kPaRows;
    // slots: as many parts at a time as a group has on average, the rest are rows
    const long long parts = p.workers / groups;
    const int lanes = parts >= 6 ? 8 : (parts >= 3 ? 4 : 2);
    hipLaunchKernelGGL((paged_join_kernel<T, C>), dim3((unsigned)(p.joins_by_group ? groups : p.workers), (unsigned)((rows * lanes + 7) / 8)), dim3(2 * C),
                       0, stream, p, lanes);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

template <typename T, int C>
int attn_bias(const PagedAttnParams& p, hipStream_t stream) {
    if (p.slopes) return launch_attn<T, C, kBiasAlibi, true>(p, stream);
    if (p.R == 0) return launch_attn<T, C, kBiasNone, true>(p, stream);
    if constexpr (!std::is_same_v<T, float>) {
        if (!p.phi_f32) return p.R <= 4 ? launch_attn<T, C, kBiasFactors4, false>(p, stream) : launch_attn<T, C, kBiasFactors, false>(p, stream);
    }
    return p.R <= 4 ? launch_attn<T, C, kBiasFactors4, true>(p, stream) : launch_attn<T, C, kBiasFactors, true>(p, stream);
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

// Waves that share the keys: all that are resident, two per SIMD.  Requests of at most 16 steps are not split.
int fb_paged_attn_workers(int B, int Hkv, int row_tiles, long long capacity, int C, bool f32) {
    const int step = f32 ? 16 : 32;
    const long long steps = (capacity + step - 1) / step;
    if (steps <= 16) return 0;
    int cus = fb_cu_count();
    if (cus <= 0) cus = 256;
    const long long groups = (long long)B * Hkv * row_tiles;
    if (steps * Hkv * row_tiles >= (1LL << 31)) return 0;            // a request's steps are counted in 32 bits
    const long long most = groups * ((steps + kPaLeast - 1) / kPaLeast), all = 8LL * cus;
    return (int)(most < all ? most : all);
}

// rows: query rows of a key head
static size_t parts_of(int workers, long long rows) { return (size_t)workers * 2 * (rows < kPaRows ? rows : kPaRows); }

size_t fb_paged_attn_workspace_bytes(int workers, long long groups, long long rows, int C) {
    return parts_of(workers, rows) * (C + 2) * sizeof(float) + (size_t)(groups < workers ? groups : workers) * sizeof(int4);
}

int fb_launch_paged_attn(PagedAttnParams p, int C, bool f32, void* ws, hipStream_t stream) {
    if (p.workers) {
        const long long groups = (long long)p.B * p.Hkv * p.row_tiles;
        const size_t parts = parts_of(p.workers, (long long)(p.H / p.Hkv) * p.N);
        p.joins_by_group = groups <= p.workers;
        p.joins = (int4*)ws;
        p.part_o = (float*)(p.joins + (p.joins_by_group ? groups : p.workers));
        p.part_m = p.part_o + parts * C;
        p.part_l = p.part_m + parts;
    }
    return f32 ? attn_channels<float>(p, C, stream) : attn_channels<bf16_t>(p, C, stream);
}
