// Rotary positions with several axes, forward and backward.
//
// Pair p of a row, (x1, x2), is turned by theta = pos[axis(p)] * freq[p]:
//     y1 = x1 cos(theta) - x2 sin(theta),   y2 = x2 cos(theta) + x1 sin(theta);
// the backward turns by -theta (the map is orthogonal and nothing else has to be kept).  Channels behind the
// pairs are copied.
//
// Bound by memory: two numbers in and two out per pair against six multiply-adds.  What could cost more is the angle:
// positions reach 1e5 and more, where an fp32 product has lost the angle's low digits, so theta is the exact product
// of two fp32 values in fp64, reduced to an eighth of a turn there, and the rest is fp32 (Taylor polynomials on
// |theta| <= pi/4, cut off below 2e-9 and evaluated in fp32: 6e-8 a rounding).  The angle belongs to the token and not to the head: a thread owns VEC pairs of
// one token, keeps their sines in registers and walks a group of heads, so each angle is formed once per group.
// B 4, N 16384, 20 heads, C 128 from a fused projection, three axes: 133 us, 5.1 TB/s read and written (a copy kernel
// reaches 5.6, 6.1 with non-temporal loads and stores); B 8, N 1024, 24 heads, C 64: 12.2 us, 4.1 TB/s; B 8, N 1: 4.3 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "fb_device.h"
#include "fb_launch.h"
#include "fb_params.h"

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotHeads = 4;      // rows a thread has in flight

template <typename T, int VEC>
struct alignas(VEC * sizeof(T)) Chunk { T x[VEC]; };

// cos and sin of pos * freq
FB_DEV void turn(double pos, double freq, float& c, float& s) {
    const double quarter = pos * freq * 0.63661977236758134308;        // 2 / pi: in quarter turns
    const double whole = __builtin_rint(quarter);
    const float a = (float)(quarter - whole) * 1.57079632679489661923f;
    const int k = (int)(whole - 4.0 * __builtin_floor(whole * 0.25));  // which quarter, 0..3 (0 for what is not finite)
    const float z = a * a;
    const float sn = a + a * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
    const float cs = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
    const float c0 = (k & 1) ? sn : cs, s0 = (k & 1) ? cs : sn;
    c = (k == 1 || k == 2) ? -c0 : c0;
    s = k >= 2 ? -s0 : s0;
}

template <typename T, int VEC, bool INTER>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryParams p) {
    const int units = p.C / (2 * VEC);
    const long long id = (p.block0 + blockIdx.x) * kRotThreads + threadIdx.x;
    const long long token = id / units;
    const int u = (int)(id - token * units);
    if (token >= (long long)p.B * p.N) return;
    const int b = (int)(token / p.N), n = (int)(token - (long long)b * p.N);
    const bool turned = u * VEC < p.pairs;
    int c0, c1;
    if (turned) {
        c0 = INTER ? 2 * u * VEC : u * VEC;
        c1 = INTER ? c0 + VEC : p.pairs + u * VEC;
    } else {
        c0 = 2 * u * VEC;
        c1 = c0 + VEC;
    }
    float cs[VEC], sn[VEC];
#pragma unroll
    for (int e = 0; e < VEC; e++) {
        cs[e] = 1.f;
        sn[e] = 0.f;
    }
    if (turned) {
        const long long at = (long long)(p.pos_shared ? 0 : b) * p.N + n, plane = (long long)(p.pos_shared ? 1 : p.B) * p.N;
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            const int pair = u * VEC + e;
            const int axis = (pair >= p.end0) + (pair >= p.end1) + (pair >= p.end2);
            const double pos = p.pos_f32 ? (double)((const float*)p.positions)[axis * plane + at]
                                         : (double)((const int*)p.positions)[axis * plane + at];
            turn(pos, (double)p.freqs[pair], cs[e], sn[e]);
            if (p.inverse) sn[e] = -sn[e];
        }
    }
    // kRotHeads rows are read before the first of them is written (y may be x, so the compiler may not move loads itself).
    const int h_begin = blockIdx.y * p.heads_per_group, h_end = min(h_begin + p.heads_per_group, p.H0 + p.H1);
    for (int h0 = h_begin; h0 < h_end; h0 += kRotHeads) {
        Chunk<T, VEC> ra[kRotHeads], rd[kRotHeads];
        T* y[kRotHeads];
#pragma unroll
        for (int i = 0; i < kRotHeads; i++) {
            const int h = h0 + i;
            if (h >= h_end) break;
            const bool first = h < p.H0;
            const int hh = first ? h : h - p.H0;
            const RotaryTensor& t = first ? p.t0 : p.t1;
            const T* x = (const T*)t.x + (b * t.sb + hh * t.sh + n * t.sn);
            y[i] = (T*)t.y + (((long long)b * (first ? p.H0 : p.H1) + hh) * p.N + n) * p.C;
            ra[i] = *(const Chunk<T, VEC>*)(x + c0);
            rd[i] = *(const Chunk<T, VEC>*)(x + c1);
        }
#pragma unroll
        for (int i = 0; i < kRotHeads; i++) {
            if (h0 + i >= h_end) break;
            if (turned) {
                float x[2 * VEC], z[2 * VEC];           // both chunks: channels c0.., c1..
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    x[e] = (float)ra[i].x[e];
                    x[VEC + e] = (float)rd[i].x[e];
                }
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    constexpr int step = INTER ? 2 : 1, mate = INTER ? 1 : VEC;
                    const float x1 = x[step * e], x2 = x[step * e + mate];
                    z[step * e] = x1 * cs[e] - x2 * sn[e];
                    z[step * e + mate] = x2 * cs[e] + x1 * sn[e];
                }
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    ra[i].x[e] = (T)z[e];
                    rd[i].x[e] = (T)z[VEC + e];
                }
            }
            *(Chunk<T, VEC>*)(y[i] + c0) = ra[i];
            *(Chunk<T, VEC>*)(y[i] + c1) = rd[i];
        }
    }
}

template <typename T, int VEC>
void launch_rotary(RotaryParams& p, long long blocks, unsigned groups, hipStream_t stream) {
    for (p.block0 = 0; p.block0 < blocks; p.block0 += kFbLaunchBlocks) {
        const dim3 grid((unsigned)std::min(blocks - p.block0, kFbLaunchBlocks), groups);
        if (p.interleaved) hipLaunchKernelGGL((rotary_kernel<T, VEC, true>), grid, dim3(kRotThreads), 0, stream, p);
        else hipLaunchKernelGGL((rotary_kernel<T, VEC, false>), grid, dim3(kRotThreads), 0, stream, p);
    }
}

}  // namespace

// The widest vector that every row start, the pairs' split and 16 bytes allow.
int fb_launch_rotary(RotaryParams p, bool f32, hipStream_t stream) {
    const int size = f32 ? 4 : 2;
    long long bits = p.pairs | (16 / size);
    const auto starts = [&](const RotaryTensor& t, int heads) {          // strides of axes of one element do not count
        if (heads > 0)
            bits |= (long long)(reinterpret_cast<uintptr_t>(t.x) / size) | (p.B > 1 ? t.sb : 0) | (heads > 1 ? t.sh : 0) | (p.N > 1 ? t.sn : 0);
    };
    starts(p.t0, p.H0);
    starts(p.t1, p.H1);
    const int vec = (int)(bits & -bits);
    const long long threads = (long long)p.B * p.N * (p.C / (2 * vec));
    const long long blocks = (threads + kRotThreads - 1) / kRotThreads;
    // Heads per thread: as many as leave 512 workgroups.  Fewer heads form the angles more often, fewer workgroups leave CUs
    // idle: B 8, N 1024, 24 heads, C 64 on 256, 512, 1024, 2048, 4096 workgroups: 13.5, 12.3, 12.7, 14.6, 18.7 us.
    const int heads = p.H0 + p.H1;
    long long groups = (512 + blocks - 1) / blocks;
    if (groups > heads) groups = heads;
    p.heads_per_group = (int)((heads + groups - 1) / groups);
    groups = (heads + p.heads_per_group - 1) / p.heads_per_group;
    if (f32) {
        if (vec == 4) launch_rotary<float, 4>(p, blocks, (unsigned)groups, stream);
        else if (vec == 2) launch_rotary<float, 2>(p, blocks, (unsigned)groups, stream);
        else launch_rotary<float, 1>(p, blocks, (unsigned)groups, stream);
    } else {
        if (vec == 8) launch_rotary<bf16_t, 8>(p, blocks, (unsigned)groups, stream);
        else if (vec == 4) launch_rotary<bf16_t, 4>(p, blocks, (unsigned)groups, stream);
        else if (vec == 2) launch_rotary<bf16_t, 2>(p, blocks, (unsigned)groups, stream);
        else launch_rotary<bf16_t, 1>(p, blocks, (unsigned)groups, stream);
    }
    return hipGetLastError() == hipSuccess ? 0 : 1;
}
