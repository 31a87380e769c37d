// Root-mean-square norm of every query and key head and the rotation by position, in one pass:
//   y = x * rsqrt(mean(x^2) + eps) * w          (fp32; left out without the norm)
//   (y_a, y_b) -> (y_a cos t - y_b sin t, y_a sin t + y_b cos t),  t = position * inv_freq[pair]
// and one rounding to 16 bits.  A pair is (i, i + rot/2), or (2i, 2i + 1) with `interleaved`; what is behind rot passes.
//
// Bound by memory: every element is read and written once.  8192 tokens of 32 + 8 heads of 128 in bf16 (168 MB) take 33.5 us,
// 5.0 TB/s, what a copy of that size reaches; one token of 64 heads 3.2 us: a launch, position and frequencies, then the rows.
#include "bwta_heads.h"

namespace bwta {
namespace {

constexpr int kWaves = 4;

// A wavefront has one token and some of its heads.  LPH lanes hold a head, 16 elements each, as the two runs of 8 whose
// elements pair with each other, so the rotation needs no exchange (and all accesses are 16 bytes wide).  The angle is formed
// in fp64 and reduced to a part of a turn there: in fp32 it would be 0.06 off at position 10^6.  Each pair's cosine and sine are
// computed once per wavefront, a pair a lane, and shared through LDS: each lane its own eight would be 8 times the work.
template <typename T, int LPH, bool INTERLEAVED>
__global__ __launch_bounds__(kWaves * 64) void k_head_norm_rope(HeadRopeArgs a, int chunks, int heads_per_wave)
{
    __shared__ float2 cs[kWaves][128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t item = (int64_t)blockIdx.x * kWaves + wave;
    const int64_t m = item / chunks;
    const int chunk = (int)(item - m * chunks);
    const int half = a.rot / 2;
    if (m < a.M && half > 0) {  // without a rotation there need be no positions
        const double pos = (double)a.positions[m];
        for (int p = lane; p < half; p += 64) {
            const double turns = pos * (double)a.inv_freq[p] * 0.15915494309189533577, part = turns - rint(turns);
            const float r = 2.0f * (float)part, rest = (float)((part - 0.5 * (double)r) * 6.28318530717958647693);
            const float c = cospif(r), s = sinpif(r);  // of the angle as fp32 has it; the rest, up to 9.4e-8, turns them the last bit
            cs[wave][p] = make_float2(fmaf(-rest, s, c), fmaf(rest, c, s));
        }
    }
    __syncthreads();
    if (m >= a.M) return;
    const int part = lane & (LPH - 1), p0 = 8 * part;
    const bool has = 16 * part < a.dim, rotated = p0 < half;
    const int o0 = INTERLEAVED || !rotated ? 2 * p0 : p0, o1 = INTERLEAVED || !rotated ? 2 * p0 + 8 : p0 + half;
    float c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 v = rotated ? cs[wave][p0 + j] : make_float2(1.0f, 0.0f);
        c[j] = v.x, s[j] = v.y;
    }
    const int total = a.heads[0] + a.heads[1], end = min(total, (chunk + 1) * heads_per_wave);
    for (int h = chunk * heads_per_wave + lane / LPH; h < end; h += 64 / LPH) {
        const int which = h >= a.heads[0], hh = which ? h - a.heads[0] : h;
        const T *x = (const T *)a.x[which] + m * a.ldx[which] + (int64_t)hh * a.dim;
        uint4 in[2] = {};
        if (has) in[0] = load_once(x + o0), in[1] = load_once(x + o1);
        float f[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = i < 4 ? (&in[0].x)[i] : (&in[1].x)[i - 4];
            f[2 * i] = Half<T>::to_float(w & 0xffff), f[2 * i + 1] = Half<T>::to_float(w >> 16);
        }
        if (a.norm) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(f[i], f[i], sum);
#pragma unroll
            for (int d = 1; d < LPH; d *= 2) sum += __shfl_xor(sum, d);  // lanes behind the head's end hold zeros
            const float r = 1.0f / sqrtf(sum / (float)a.dim + a.eps);
            const T *wt = (const T *)a.w[which];
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] *= r;
            if (wt && has) {
                const uint4 ww[2] = {*(const uint4 *)(wt + o0), *(const uint4 *)(wt + o1)};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t w = i < 4 ? (&ww[0].x)[i] : (&ww[1].x)[i - 4];
                    f[2 * i] *= Half<T>::to_float(w & 0xffff), f[2 * i + 1] *= Half<T>::to_float(w >> 16);
                }
            }
        }
        if (rotated) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int u = INTERLEAVED ? 2 * j : j, v = INTERLEAVED ? 2 * j + 1 : j + 8;
                const float x0 = f[u], x1 = f[v];
                f[u] = x0 * c[j] - x1 * s[j], f[v] = x0 * s[j] + x1 * c[j];
            }
        }
        if (!has) continue;
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = Half<T>::pack(f[2 * i], f[2 * i + 1]);
        T *y = (T *)a.out[which] + m * a.ldo[which] + (int64_t)hh * a.dim;
        *(uint4 *)(y + o0) = make_uint4(o[0], o[1], o[2], o[3]);
        *(uint4 *)(y + o1) = make_uint4(o[4], o[5], o[6], o[7]);
    }
}

template <typename T, int LPH>
void launch(const HeadRopeArgs &a, int chunks, int per_wave, hipStream_t st)
{
    const int64_t groups = ((int64_t)a.M * chunks + kWaves - 1) / kWaves;
    if (a.interleaved)
        hipLaunchKernelGGL((k_head_norm_rope<T, LPH, true>), dim3((unsigned)groups), dim3(kWaves * 64), 0, st, a, chunks, per_wave);
    else
        hipLaunchKernelGGL((k_head_norm_rope<T, LPH, false>), dim3((unsigned)groups), dim3(kWaves * 64), 0, st, a, chunks, per_wave);
}

template <typename T>
void launch_type(const HeadRopeArgs &a, hipStream_t st)
{
    const int lph = a.dim <= 16 ? 1 : a.dim <= 32 ? 2 : a.dim <= 64 ? 4 : a.dim <= 128 ? 8 : 16;
    const int step = 64 / lph, total = a.heads[0] + a.heads[1], steps = (total + step - 1) / step;
    // A wavefront takes all heads of a token, which pays for its angles once, unless there are fewer than four wavefronts for
    // every SIMD; then heads are spread.
    int chunks = 1;
    while (chunks < steps && (int64_t)a.M * chunks < 4096) chunks *= 2;
    if (chunks > steps) chunks = steps;
    const int per_wave = (steps + chunks - 1) / chunks * step;
    chunks = (total + per_wave - 1) / per_wave;
    switch (lph) {
    case 1: return launch<T, 1>(a, chunks, per_wave, st);
    case 2: return launch<T, 2>(a, chunks, per_wave, st);
    case 4: return launch<T, 4>(a, chunks, per_wave, st);
    case 8: return launch<T, 8>(a, chunks, per_wave, st);
    default: return launch<T, 16>(a, chunks, per_wave, st);
    }
}

}  // namespace

hipError_t launch_head_norm_rope(const HeadRopeArgs &a, hipStream_t st)
{
    if (a.bf16)
        launch_type<__bf16>(a, st);
    else
        launch_type<_Float16>(a, st);
    return hipGetLastError();
}

}  // namespace bwta
