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
// The keys of all requests are laid end to end in steps of 4 KW keys, and each of `workers` workgroups takes an equal
// share, found from the lengths on the device: one long request among short ones, or a table with room for far more
// than it holds, costs no balance.  A share ends inside a (request, key head): the parts go to scratch, two per
// worker at most, and a second launch joins them in a fixed order.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fb_device.h"
#include "fb_launch.h"
#include "fb_params.h"

namespace {

constexpr int kPaWaves = 4;
constexpr int kPaThreads = kPaWaves * 64;
constexpr int kPaRows = 16;
constexpr int kPaLeast = 2;       // steps of a worker's share at least (the join of smaller shares costs more than they save)

typedef float f32x8 __attribute__((ext_vector_type(8)));

FB_DEV float lane_xor_max(float x) {      // over the four lanes of a column
    x = fmaxf(x, __shfl_xor(x, 16));
    return half_max(x);
}
FB_DEV float lane_xor_sum(float x) {
    x += __shfl_xor(x, 16);
    return half_sum(x);
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

// Sums over the workgroup; every thread gets the total and its own inclusive sum.
FB_DEV long long pa_scan(long long x, long long* sm, long long& total) {
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
    for (int w = 0; w < kPaWaves; w++) {
        if (w < wave) before += sm[w];
        total += sm[w];
    }
    __syncthreads();
    return x + before;
}

FB_DEV int held_keys(const PagedAttnParams& p, int b) {
    return max((int)min((long long)p.lens[b], (long long)p.max_blocks << p.page_shift), 0);
}

// BIAS, PF32: kind of bias and whether the factors are float
template <typename T, int C, int BIAS, bool PF32>
__global__ __launch_bounds__(kPaThreads, 2) void paged_attn_kernel(PagedAttnParams p) {
    using S = Step<T, C>;
    constexpr int KW = S::KW, TK = kPaWaves * KW, NV = S::NV, GROUPS = S::GROUPS;
    constexpr int OP = C + 4;                             // LDS row pitch: 16 rows of a wave's O start in different banks
    using PT = std::conditional_t<PF32, float, bf16_t>;
    __shared__ __align__(16) float sm_o[kPaWaves][kPaRows][OP];
    __shared__ float sm_m[kPaWaves][kPaRows], sm_l[kPaWaves][kPaRows];
    __shared__ long long sm_scan[kPaWaves];
    __shared__ long long sm_at[2];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, i = lane & 15;
    const int groups = p.Hkv * p.row_tiles;               // (key head, row tile) pairs of a request
    const int rows_all = p.H / p.Hkv * p.N;
    const int page_mask = (1 << p.page_shift) - 1;

    auto steps_of = [&](int len) { return len > TK ? (len + TK - 1) / TK : 1; };      // a request without keys has one step too

    // ---- this worker's share: steps [u, u_end) of all, the first of them in request b, `rem` steps into it ----
    int b;
    long long u, u_end, rem, total = 0, n_workers = 0;
    if (p.workers == 0) {
        b = blockIdx.x / groups;
        const int len = held_keys(p, b);
        rem = (long long)(blockIdx.x - b * groups) * steps_of(len);
        u = 0;
        u_end = steps_of(len);
    } else {
        for (int b0 = 0; b0 < p.B; b0 += kPaThreads) {
            const int bb = b0 + tid;
            long long sum;
            pa_scan(bb < p.B ? (long long)steps_of(held_keys(p, bb)) * groups : 0, sm_scan, sum);
            total += sum;
        }
        n_workers = min((long long)p.workers, (total + kPaLeast - 1) / kPaLeast);
        const int w = blockIdx.x;
        if (w >= n_workers) {
            if (tid == 0) p.joins[w] = make_int4(0, 0, 0, 0);
            return;
        }
        u = w * total / n_workers;
        u_end = (w + 1) * total / n_workers;
        long long before = 0;
        for (int b0 = 0; b0 < p.B; b0 += kPaThreads) {
            const int bb = b0 + tid;
            const long long own = bb < p.B ? (long long)steps_of(held_keys(p, bb)) * groups : 0;
            long long sum;
            const long long end = before + pa_scan(own, sm_scan, sum);
            if (end - own <= u && u < end) {
                sm_at[0] = bb;
                sm_at[1] = u - (end - own);
            }
            before += sum;
            if (before > u) break;                        // (uniform)
        }
        __syncthreads();
        b = (int)sm_at[0];
        rem = sm_at[1];
    }
    b = __builtin_amdgcn_readfirstlane(b);
    int4 join = make_int4(0, 0, 0, 0);

    while (u < u_end) {
        const int len = __builtin_amdgcn_readfirstlane(held_keys(p, b));
        const int n_steps = steps_of(len);
        const int grp = __builtin_amdgcn_readfirstlane((int)(rem / n_steps));
        const int t0 = __builtin_amdgcn_readfirstlane((int)(rem - (long long)grp * n_steps));
        const int t1 = __builtin_amdgcn_readfirstlane((int)min((long long)n_steps, t0 + (u_end - u)));
        const int h = grp / p.row_tiles, r0 = (grp - h * p.row_tiles) * kPaRows;
        const int rows = min(kPaRows, rows_all - r0);
        const int start = __builtin_amdgcn_readfirstlane(p.starts ? min(max(p.starts[b], -(1 << 30)), 1 << 30) : len - p.N);
        const long long row_base = (long long)b * p.H * p.N + (long long)h * rows_all + r0;      // of q, out, lse

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
        float phi_q[4] = {0.f, 0.f, 0.f, 0.f};            // BIAS 2: [0] only; lane: factor 4 x + g
        const PT* pq_row = nullptr;
        if constexpr (BIAS >= kBiasFactors4) {
            pq_row = (const PT*)p.phi_q + (long long)b * p.phiq_bstride + ((long long)h * rows_all + r0 + i) * p.R;
            constexpr int NF = BIAS == kBiasFactors4 ? 1 : 4;
#pragma unroll
            for (int x = 0; x < NF; x++)
                if (has_row && 4 * x + g < p.R) phi_q[x] = (float)pq_row[4 * x + g];
        }
        float slope = 0.f;
        if constexpr (BIAS == kBiasAlibi)
            if (has_row) slope = p.slopes[h * (p.H / p.Hkv) + (r0 + i) / p.N];

        const int* table = p.table + (long long)b * p.max_blocks;
        float m = -INFINITY, l = 0.f;
        f32x4 o[NV];
#pragma unroll
        for (int t = 0; t < NV; t++) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

        // first row of the 16 keys from k on in their page, -1: no such page (its keys are not visible)
        auto group_row = [&](int k) -> long long {
            if (k >= len) return -1;
            const int page = __builtin_amdgcn_readfirstlane(table[k >> p.page_shift]);
            if ((unsigned)page >= (unsigned)p.n_pages) return -1;
            return (((long long)page * p.Hkv + h) << p.page_shift) + (k & page_mask);
        };

        for (int t = t0; t < t1; t++) {
            const int k0 = t * TK + wave * KW;            // wave-uniform
            if (k0 >= len) break;
            typename S::Keys kr;
            typename S::Values vr;
            long long row[GROUPS];
            bool whole = k0 + KW <= all_see;
#pragma unroll
            for (int s = 0; s < GROUPS; s++) {
                row[s] = group_row(k0 + 16 * s);
                whole = whole && row[s] >= 0;
            }
#pragma unroll
            for (int s = 0; s < GROUPS; s++) {
                const long long at = row[s] >= 0 ? row[s] : 0;       // page 0 stands in
                S::load_keys(kr, s, (const T*)p.k_pages + at * C, g, i);
                S::load_values(vr, s, (const T*)p.v_pages + at * C, g, i);
            }
            f32x4 sc[GROUPS];
#pragma unroll
            for (int s = 0; s < GROUPS; s++) {
                sc[s] = S::scores(kr, s, q);
                const int key0 = k0 + 16 * s + 4 * g;
                if constexpr (BIAS >= kBiasFactors4) {
                    const PT* pk = (const PT*)p.phi_pages + ((row[s] >= 0 ? row[s] : 0) + i) * p.R;
                    f32x4 f = {0.f, 0.f, 0.f, 0.f};
                    constexpr int NF = BIAS == kBiasFactors4 ? 1 : 4;
#pragma unroll
                    for (int x = 0; x < NF; x++) {
                        const float a = 4 * x + g < p.R ? (float)pk[4 * x + g] : 0.f;
                        f = __builtin_amdgcn_mfma_f32_16x16x4f32(a, phi_q[x], f, 0, 0, 0);
                    }
                    if constexpr (BIAS == kBiasFactors)
                        for (int x = 4; 4 * x < p.R; x++) {
                            const bool in = 4 * x + g < p.R;
                            const float a = in ? (float)pk[4 * x + g] : 0.f, c = in && has_row ? (float)pq_row[4 * x + g] : 0.f;
                            f = __builtin_amdgcn_mfma_f32_16x16x4f32(a, c, f, 0, 0, 0);
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
            // ---- softmax of the rows ----
            float mx = m;
#pragma unroll
            for (int s = 0; s < GROUPS; s++)
#pragma unroll
                for (int r = 0; r < 4; r++) mx = fmaxf(mx, sc[s][r]);
            mx = lane_xor_max(mx);
            if (__any(mx > m)) {
                const float alpha = weight(m, mx);
                l *= alpha;
#pragma unroll
                for (int t2 = 0; t2 < NV; t2++)
#pragma unroll
                    for (int r = 0; r < 4; r++) o[t2][r] *= alpha;
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
                for (int t2 = 0; t2 < NV; t2++) o[t2] = S::product(vr, t2, pr, o[t2]);
            } else {
                // Values a row does not see may be anything (0 * inf is NaN), so rows of different limits are done one
                // after the other with the values behind their limit cleared; at most N of them, only around the last keys.
                auto masked = [&](int seen, bool mine) __attribute__((always_inline)) {
                    typename S::Values vm = vr;
#pragma unroll
                    for (int s = 0; s < GROUPS; s++)
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (k0 + 16 * s + 4 * g + r >= seen || row[s] < 0) vm.x[s][r] = {};
#pragma unroll
                    for (int t2 = 0; t2 < NV; t2++) {
                        const f32x4 d = S::product(vm, t2, pr, o[t2]);
#pragma unroll
                        for (int r = 0; r < 4; r++) o[t2][r] = mine ? d[r] : o[t2][r];
                    }
                };
                unsigned long long todo = __ballot(limit > k0);
                while (todo != 0) {
                    const int seen = __builtin_amdgcn_readlane(limit, __builtin_ctzll(todo));
                    const int cut = min(seen, k0 + KW);
                    const bool mine = min(limit, k0 + KW) == cut;
                    masked(cut, mine);
                    todo &= ~__ballot(mine);
                }
            }
        }

        // ---- the waves of the workgroup ----
        l = lane_xor_sum(l);
        __syncthreads();                                  // the last segment's sums have been read
        if (has_row) {
#pragma unroll
            for (int r = 0; r < 4; r++)
#pragma unroll
                for (int t = 0; t < NV; t++) sm_o[wave][i][(4 * g + r) * NV + t] = o[t][r];
            if (g == 0) {
                sm_m[wave][i] = limit > 0 ? m : -INFINITY;       // a row that sees nothing went along with the others
                sm_l[wave][i] = limit > 0 ? l : 0.f;
            }
        }
        __syncthreads();
        const bool split = t0 > 0 || t1 < n_steps;
        const int slot = blockIdx.x * 2 + (t0 > 0 ? 0 : 1);
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
            if (!split) {
                const float inv = lt == 0.f ? 0.f : 1.f / lt;
                T* out = (T*)p.out + (row_base + r) * C + c4 * 4;
                struct alignas(4 * sizeof(T)) Four { T x[4]; } v;
#pragma unroll
                for (int e = 0; e < 4; e++) v.x[e] = (T)(lt == 0.f ? 0.f : ot[e] * inv);
                *(Four*)out = v;
                if (c4 == 0) p.lse[row_base + r] = lt == 0.f ? -INFINITY : mx + __log2f(lt) * kLn2;
            } else {
                const long long at = (long long)slot * kPaRows + r;
                *(f32x4*)(p.part_o + at * C + c4 * 4) = ot;
                if (c4 == 0) {
                    p.part_m[at] = mx;
                    p.part_l[at] = lt;
                }
            }
        }
        if (t0 == 0 && t1 < n_steps) {                    // the first of several workers
            const long long last = u + n_steps - 1;       // the group's last step, and who has it
            const long long lw = ((last + 1) * n_workers - 1) / total;
            join = make_int4((int)(lw - blockIdx.x), (int)(row_base & 0xffffffff), (int)(row_base >> 32), rows);
        }
        u += t1 - t0;
        rem += t1 - t0;
        if (rem == (long long)groups * n_steps) {
            b++;
            rem = 0;
        }
    }
    if (p.workers != 0 && tid == 0) p.joins[blockIdx.x] = join;
}

// Joins the parts of one row: part 1 of the worker where the group begins and part 0 of the `more` workers behind it.
template <typename T, int C>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnParams p) {
    constexpr int LN = C / 4, PL = 256 / LN;              // lanes of a row, parts at a time
    __shared__ __align__(16) float sm_o[PL][C];
    __shared__ float sm_l[PL], sm_m[4];
    const int4 join = p.joins[blockIdx.x];
    const int more = join.x, r = blockIdx.y;
    if (more == 0 || r >= join.w) return;
    const long long row = (((long long)join.z << 32) | (unsigned)join.y) + r;
    const int tid = threadIdx.x, c4 = tid % LN, pl = tid / LN;
    auto part = [&](int k) { return ((long long)(blockIdx.x + k) * 2 + (k == 0 ? 1 : 0)) * kPaRows + r; };

    float mx = -INFINITY;
    for (int k = tid; k <= more; k += 256) mx = fmaxf(mx, p.part_m[part(k)]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) mx = fmaxf(mx, __shfl_xor(mx, d));
    if ((tid & 63) == 0) sm_m[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
    float lt = 0.f;
    f32x4 ot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = pl; k <= more; k += PL) {
        const float a = weight(p.part_m[part(k)], mx);
        const f32x4 x = *(const f32x4*)(p.part_o + part(k) * C + c4 * 4);
        lt = fmaf(a, p.part_l[part(k)], lt);
#pragma unroll
        for (int e = 0; e < 4; e++) ot[e] = fmaf(a, x[e], ot[e]);
    }
    *(f32x4*)&sm_o[pl][c4 * 4] = ot;
    if (c4 == 0) sm_l[pl] = lt;
    __syncthreads();
    if (tid >= LN) return;
#pragma unroll
    for (int k = 1; k < PL; k++) {
        const f32x4 x = *(const f32x4*)&sm_o[k][c4 * 4];
        lt += sm_l[k];
#pragma unroll
        for (int e = 0; e < 4; e++) ot[e] += x[e];
    }
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    struct alignas(4 * sizeof(T)) Four { T x[4]; } v;
#pragma unroll
    for (int e = 0; e < 4; e++) v.x[e] = (T)(lt == 0.f ? 0.f : ot[e] * inv);
    *(Four*)((T*)p.out + row * C + c4 * 4) = v;
    if (c4 == 0) p.lse[row] = lt == 0.f ? -INFINITY : mx + __log2f(lt) * kLn2;
}

template <typename T, int C, int BIAS, bool PF32>
int launch_attn(const PagedAttnParams& p, hipStream_t stream) {
    const long long blocks = p.workers ? p.workers : (long long)p.B * p.Hkv * p.row_tiles;
    if (blocks >= (1LL << 31)) return -1;
    hipLaunchKernelGGL((paged_attn_kernel<T, C, BIAS, PF32>), dim3((unsigned)blocks), dim3(kPaThreads), 0, stream, p);
    if (hipGetLastError() != hipSuccess) return 1;
    if (p.workers) {
        const int rows = p.H / p.Hkv * p.N;
        hipLaunchKernelGGL((paged_join_kernel<T, C>), dim3((unsigned)p.workers, (unsigned)(rows < kPaRows ? rows : kPaRows)), dim3(256), 0, stream, p);
        if (hipGetLastError() != hipSuccess) return 1;
    }
    return 0;
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

// Two workgroups a CU are resident.  Requests of at most four steps are not split.
int fb_paged_attn_workers(int B, int Hkv, int row_tiles, long long capacity, int C, bool f32) {
    const int step = kPaWaves * (f32 ? 16 : 32);
    const long long steps = (capacity + step - 1) / step;
    if (steps <= 4) return 0;
    int cus = fb_cu_count();
    if (cus <= 0) cus = 256;
    const long long most = (long long)B * Hkv * row_tiles * ((steps + kPaLeast - 1) / kPaLeast);
    return (int)(most < 2LL * cus ? most : 2LL * cus);
}

size_t fb_paged_attn_workspace_bytes(int workers, int C) {
    return (size_t)workers * (2 * kPaRows * (C + 2) * sizeof(float) + sizeof(int4));
}

int fb_launch_paged_attn(PagedAttnParams p, int C, bool f32, void* ws, hipStream_t stream) {
    if (p.workers) {
        p.part_o = (float*)ws;
        p.joins = (int4*)(p.part_o + (size_t)p.workers * 2 * kPaRows * C);
        p.part_m = (float*)(p.joins + p.workers);
        p.part_l = p.part_m + (size_t)p.workers * 2 * kPaRows;
    }
    return f32 ? attn_channels<float>(p, C, stream) : attn_channels<bf16_t>(p, C, stream);
}
