// Attention of 16-bit queries over the 8-bit cache, in one pass over the keys:
//   out = sum_j p_j v_j / sum_j p_j,   p_j = exp(alpha q . k_j - m),   m a running maximum
// with sums, maximum and scores in fp32.
//
// Codes are exact in both 16-bit types, so q . k is the matrix cores' sum of exact products; a block's key scale joins
// alpha.  Weights are rounded to fp16 for the second product whatever the queries' type: they lie in [0, 2^12], where
// fp16 has 11 bits to bf16's 8.  Value codes enter without their scale; sums are kept in units of 2^eref, the scale of
// some block, and the few bits between that and the block at hand go into the weights' exponent.
//
// Everything stays in registers.  The first product is computed transposed, keys by queries: its result has a query per
// lane and, with the key rows taken in the right order (row 4 i + r of the b-th 16 is token 16 i + 4 b + r), 16 tokens in
// a row per lane, which is what the second product (values transposed by queries) wants as its operand.  Keys are loaded
// as 16 codes of a token, values as 16 tokens of a channel, both 16 bytes in a row in the cache's layout.
#include "bwta_heads.h"

namespace bwta {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

template <typename T> struct Mma;
template <> struct Mma<_Float16> {
    typedef half8 Frag;
    static __device__ __forceinline__ half2v two(uint32_t codes, bool hi)
    {
        return hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.0f, false);
    }
    static __device__ __forceinline__ float4v mma(half8 a, half8 b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float16v mma(half8 a, half8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<__bf16> {
    typedef bf8 Frag;
    static __device__ __forceinline__ bf2v two(uint32_t codes, bool hi)
    {
        return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, false);
    }
    static __device__ __forceinline__ float4v mma(bf8 a, bf8 b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float16v mma(bf8 a, bf8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// eight codes as a matrix-core operand's eight values
template <typename T>
__device__ __forceinline__ typename Mma<T>::Frag widen(uint32_t lo, uint32_t hi)
{
    const auto a = Mma<T>::two(lo, false), b = Mma<T>::two(lo, true), c = Mma<T>::two(hi, false), d = Mma<T>::two(hi, true);
    return typename Mma<T>::Frag{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kSlack = 8.0f;  // weights may reach 2^kSlack before the maximum is moved
constexpr int kDrift = 4;       // bits a block's value scale may differ from eref

// The larger one; a NaN if either is one (which saves making a quiet one of it first).
__device__ __forceinline__ float most(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// the same value for all four lanes that share a query (lane, lane ^ 16, lane ^ 32, lane ^ 48)
__device__ __forceinline__ float max_of_query(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_of_query(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Four channels of a row, and once per row its maximum (as a power of two) and sum: the result, or this split's part of it.
template <typename T, int D>
__device__ __forceinline__ void give(const CacheAttentionArgs &a, const Seq &s, int head, int group, int split, int64_t row, int channel, float4v x, float m, float l, bool once)
{
    const int64_t token = s.row + row / group, at = token * a.heads + head * group + row % group;
    if (a.splits > 1) {
        const int64_t all_rows = (int64_t)a.seq.M * a.heads;
        *(float4v *)(a.partial + (split * all_rows + at) * D + channel) = x;
        if (once) ((float2 *)(a.partial + a.splits * all_rows * D))[split * all_rows + at] = make_float2(m, l);
        return;
    }
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    *(uint2 *)((T *)a.out + token * a.ldo + (head * group + row % group) * D + channel) = make_uint2(Half<T>::pack(x[0] * f, x[1] * f), Half<T>::pack(x[2] * f, x[3] * f));
    if (once && a.lse) a.lse[at] = kLn2 * (m + log2f(l));
}

// Rows of one sequence and key head: row r is query head r % group of the r / group-th new token.  Here a workgroup has
// NB * 16 of them, and its wavefronts take turns at the steps of 64 keys.
template <typename T, int D, int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, (NB == 1 && D <= 128) ? 2 : 1) void k_cache_attention(CacheAttentionArgs a, int row_tiles)
{
    constexpr int R = 16 * NB, KL = D / 64, NV = D / 16;
    typedef typename Mma<T>::Frag Frag;
    __shared__ float4 merged[WAVES * R * (D / 4)];
    __shared__ float2 merged_ml[WAVES * R];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q16 = lane & 15, g = lane >> 4;
    const int H = a.cache.heads, group = a.heads / H;

    unsigned i = blockIdx.x;
    const int split = i % a.splits;
    i /= a.splits;
    const int bh = i % (a.seq.batch * H), head = bh % H, b = bh / H;
    const int tile_of_rows = row_tiles - 1 - (int)(i / (a.seq.batch * H));  // causal rows at the end see most: first
    const Seq s = sequence(a.seq, b);
    const int64_t total = (int64_t)s.n * group;
    const int64_t first = (int64_t)tile_of_rows * R;
    if (first >= total) return;
    const int64_t last = min(first + R, total) - 1;

    // keys that some row sees, and those that every row sees
    const int t_first = (int)(first / group), t_last = (int)(last / group);
    const int key_end = a.causal ? max(0, min(s.len, s.start + t_last + 1)) : s.len;
    const int key_begin = a.window ? max(0, s.start + t_first - a.window + 1) : 0;
    const int all_end = a.causal ? min(s.len, s.start + t_first + 1) : s.len, all_begin = a.window ? s.start + t_last - a.window + 1 : 0;
    const int step0 = key_begin / kCacheTile, steps = max(0, (key_end + kCacheTile - 1) / kCacheTile - step0);
    const int from = step0 + (int)((int64_t)steps * split / a.splits), to = step0 + (int)((int64_t)steps * (split + 1) / a.splits);

    // this lane's query of each 16
    int see_lo[NB], see_hi[NB];
    Frag q[NB][2 * KL];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int64_t row = first + nb * 16 + q16;
        const bool has = row < total;
        const int t = has ? (int)(row / group) : 0, h = head * group + (has ? (int)(row % group) : 0);
        see_hi[nb] = !has ? -1 : a.causal ? min(s.len - 1, s.start + t) : s.len - 1;
        see_lo[nb] = a.window ? s.start + t - a.window + 1 : 0;
        const T *x = (const T *)a.q + (s.row + t) * a.ldq + (int64_t)h * D;
#pragma unroll
        for (int j = 0; j < KL; ++j)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                if (has) q[nb][2 * j + hf] = *(const Frag *)(x + 64 * j + 16 * g + 8 * hf);
                else q[nb][2 * j + hf] = Frag{};
            }
    }

    float4v o[NB][NV] = {};
    float m[NB], l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) m[nb] = -INFINITY, l[nb] = 0.0f;
    int eref = 0;
    bool begun = false;
    const int block_shift = a.cache.block >> 7;  // 64, 128, 256 tokens: 1, 2, 4 steps
    const int key_row = 16 * (q16 >> 2) + (q16 & 3);  // + 4 b

    // Loads run ahead of what waits for them: a step's codes and scales are asked for one turn before, its block two turns
    // before (the address depends on it).
    uint4 kc[4][KL], vc[NV], kn[4][KL], vn[NV];
    float ks_next = 0.0f, vs_next = 0.0f;
    bool ok_next = false;
    int page_next = -1;
    auto page_of = [&](int step) { return a.seq.table[b * a.seq.ldt + (min(step, to - 1) >> block_shift)]; };
    auto fetch = [&](int step) {
        const int sub = step & ((1 << block_shift) - 1);
        int page = __builtin_amdgcn_readfirstlane(page_next);
        ok_next = page >= 0 && page < a.cache.blocks;
        if (!ok_next) page = 0;
        const int64_t unit = (int64_t)page * H + head;
        const uint8_t *kp = a.cache.k + (unit * a.cache.block + sub * kCacheTile) * D;
        const uint8_t *vp = a.cache.v + unit * D * a.cache.block + sub * kCacheTile;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int j = 0; j < KL; ++j) kn[kb][j] = *(const uint4 *)(kp + (key_row + 4 * kb) * D + 64 * j + 16 * g);
        ks_next = a.cache.k_scale[unit];
        vs_next = a.cache.v_scale[unit];
#pragma unroll
        for (int n = 0; n < NV; ++n) vn[n] = *(const uint4 *)(vp + (16 * n + q16) * a.cache.block + 16 * g);
        page_next = page_of(step + WAVES);
    };
    if (from + wave < to) {
        page_next = page_of(from + wave);
        fetch(from + wave);
    }
    for (int step = from + wave; step < to; step += WAVES) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int j = 0; j < KL; ++j) kc[kb][j] = kn[kb][j];
#pragma unroll
        for (int n = 0; n < NV; ++n) vc[n] = vn[n];
        const float ks = ks_next, vs = vs_next;
        const bool page_ok = ok_next;
        if (step + WAVES < to) fetch(step + WAVES);

        float4v sc[NB][4] = {};
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int j = 0; j < KL; ++j) {
                const Frag k0 = widen<T>(kc[kb][j].x, kc[kb][j].y), k1 = widen<T>(kc[kb][j].z, kc[kb][j].w);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    sc[nb][kb] = Mma<T>::mma(k0, q[nb][2 * j], sc[nb][kb]);
                    sc[nb][kb] = Mma<T>::mma(k1, q[nb][2 * j + 1], sc[nb][kb]);
                }
            }

        const int key0 = step * kCacheTile + 16 * g;  // this lane's first key
        if (!page_ok || (step + 1) * kCacheTile > all_end || step * kCacheTile < all_begin) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int hi = page_ok ? see_hi[nb] : -1, lo = see_lo[nb];
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = key0 + 4 * kb + r;
                        sc[nb][kb][r] = ((key > hi) | (key < lo)) ? -INFINITY : sc[nb][kb][r];
                    }
            }
        }
        // a slot behind the sequence holds anything, a NaN too: its weight 0 does not hide that
        if (!page_ok || (step + 1) * kCacheTile > s.len) {
            const int valid = page_ok ? s.len - key0 : 0;
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int bytes = min(max(valid - 4 * w, 0), 4);
                    (&vc[n].x)[w] &= bytes == 4 ? 0xffffffffu : (1u << (8 * bytes)) - 1;
                }
        }

        const float c = fmaxf(a.alpha * kLog2e * ks, 1.17549435e-38f);
        const int ev = __builtin_amdgcn_readfirstlane(exponent_of(vs));
        if (!begun) eref = ev, begun = true;
        if (ev - eref > kDrift || eref - ev > kDrift) {
            const float f = pow2(eref - ev);
            eref = ev;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int n = 0; n < NV; ++n) o[nb][n] *= f;
        }
        const float drift = (float)(ev - eref), undrift = pow2(eref - ev);
        half8 p[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float top = most(most(sc[nb][0][0], sc[nb][0][1]), most(sc[nb][0][2], sc[nb][0][3]));
#pragma unroll
            for (int kb = 1; kb < 4; ++kb) top = most(most(top, most(sc[nb][kb][0], sc[nb][kb][1])), most(sc[nb][kb][2], sc[nb][kb][3]));
            top *= c;
            if (__any(top > m[nb] + kSlack)) {
                const float now = fmaxf(m[nb], max_of_query(top));
                const float f = m[nb] == -INFINITY ? 0.0f : exp2f(m[nb] - now);
                m[nb] = now;
                l[nb] *= f;
#pragma unroll
                for (int n = 0; n < NV; ++n) o[nb][n] *= f;
            }
            const float base = (m[nb] == -INFINITY ? 0.0f : m[nb]) - drift;
            float sum = 0.0f, w[16];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    w[4 * kb + r] = __builtin_amdgcn_exp2f(fmaf(sc[nb][kb][r], c, -base));
                    sum += w[4 * kb + r];
                }
            l[nb] = fmaf(sum, undrift, l[nb]);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                p[nb][hf] = half8{(_Float16)w[8 * hf], (_Float16)w[8 * hf + 1], (_Float16)w[8 * hf + 2], (_Float16)w[8 * hf + 3],
                                  (_Float16)w[8 * hf + 4], (_Float16)w[8 * hf + 5], (_Float16)w[8 * hf + 6], (_Float16)w[8 * hf + 7]};
        }
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const half8 v0 = widen<_Float16>(vc[n].x, vc[n].y), v1 = widen<_Float16>(vc[n].z, vc[n].w);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                o[nb][n] = Mma<_Float16>::mma(v0, p[nb][0], o[nb][n]);
                o[nb][n] = Mma<_Float16>::mma(v1, p[nb][1], o[nb][n]);
            }
        }
    }

    // o[nb][n][r]: query q16 of the nb-th 16, channel 16 n + 4 g + r, in units of 2^eref
    const float unit = pow2(eref);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l[nb] = sum_of_query(l[nb]);
#pragma unroll
        for (int n = 0; n < NV; ++n) o[nb][n] *= unit;
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int at = wave * R + nb * 16 + q16;
        if (g == 0) merged_ml[at] = make_float2(m[nb], l[nb]);
#pragma unroll
        for (int n = 0; n < NV; ++n) merged[at * (D / 4) + 4 * n + g] = make_float4(o[nb][n][0], o[nb][n][1], o[nb][n][2], o[nb][n][3]);
    }
    __syncthreads();
    for (int at = threadIdx.x; at < R * (D / 4); at += WAVES * 64) {
        const int r = at / (D / 4);
        if (first + r >= total) continue;
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, merged_ml[w * R + r].x);
        float4v x = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 ml = merged_ml[w * R + r];
            const float f = ml.x == -INFINITY && ml.y == 0.0f ? 0.0f : exp2f(ml.x - top);  // a NaN among the scores stays one
            const float4 y = merged[w * R * (D / 4) + at];
            x += float4v{y.x, y.y, y.z, y.w} * f;
            sum = fmaf(ml.y, f, sum);
        }
        give<T, D>(a, s, head, group, split, first + r, at % (D / 4) * 4, x, top, sum, at % (D / 4) == 0);
    }
}

// Many rows: each wavefront has NB * 32 of its own, and a workgroup's wavefronts share the keys and values of a step, which
// reach LDS as 16-bit numbers (each code is widened once for the workgroup, not once for each wavefront), two steps' worth:
// one is computed with while the next arrives.  Products of 32 x 32: key row 8 i + 4 j + r of a block of 32 is token
// 16 j + 4 i + r, so a lane again has 16 tokens in a row.  16-byte chunks of a row are swapped by bits of the row's number,
// which spreads the rows that are read at a time over the banks.
// (Rows of 16 chunks or more by the row's last four bits, rows of 8 by the three above the last.)
template <int D>
__device__ __forceinline__ int key_swap(int row) { return D >= 128 ? row & 15 : row >> 1 & 7; }

template <typename T, int D, int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, (NB == 1 && D <= 128) ? 2 : 1) void k_cache_attention_rows(CacheAttentionArgs a, int row_tiles)
{
    constexpr int R = 32 * NB, kRows = R * WAVES, NT = WAVES * 64, KK = D / 16, DN = D / 32, kUnits = 4 * D / NT;
    typedef typename Mma<T>::Frag Frag;
    __shared__ uint4 keys[2][kCacheTile * D / 8], values[2][kCacheTile * D / 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q32 = lane & 31, h2 = lane >> 5;
    const int H = a.cache.heads, group = a.heads / H;

    unsigned i = blockIdx.x;
    const int split = i % a.splits;
    i /= a.splits;
    const int bh = i % (a.seq.batch * H), head = bh % H, b = bh / H;
    const int tile_of_rows = row_tiles - 1 - (int)(i / (a.seq.batch * H));  // causal rows at the end see most: first
    const Seq s = sequence(a.seq, b);
    const int64_t total = (int64_t)s.n * group;
    const int64_t first = (int64_t)tile_of_rows * kRows;
    if (first >= total) return;

    // keys that some row of rows [lo, lo + count) sees, and those that every one sees
    struct Span {
        int begin, end, all_begin, all_end;
    };
    auto span = [&](int64_t lo, int count) {
        const int64_t hi = min(lo + count, total) - 1;
        const int t0 = (int)(lo / group), t1 = (int)(hi / group);
        Span r;
        r.end = hi < lo ? 0 : a.causal ? max(0, min(s.len, s.start + t1 + 1)) : s.len;
        r.begin = a.window ? max(0, s.start + t0 - a.window + 1) : 0;
        r.all_end = a.causal ? min(s.len, s.start + t0 + 1) : s.len;
        r.all_begin = a.window ? s.start + t1 - a.window + 1 : 0;
        return r;
    };
    const Span whole = span(first, kRows), mine = span(first + wave * R, R);
    const int step0 = whole.begin / kCacheTile, steps = max(0, (whole.end + kCacheTile - 1) / kCacheTile - step0);
    const int from = step0 + (int)((int64_t)steps * split / a.splits), to = step0 + (int)((int64_t)steps * (split + 1) / a.splits);

    int see_lo[NB], see_hi[NB];
    Frag q[NB][KK];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int64_t row = first + wave * R + nb * 32 + q32;
        const bool has = row < total;
        const int t = has ? (int)(row / group) : 0, h = head * group + (has ? (int)(row % group) : 0);
        see_hi[nb] = !has ? -1 : a.causal ? min(s.len - 1, s.start + t) : s.len - 1;
        see_lo[nb] = a.window ? s.start + t - a.window + 1 : 0;
        const T *x = (const T *)a.q + (s.row + t) * a.ldq + (int64_t)h * D;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (has) q[nb][kk] = *(const Frag *)(x + 16 * kk + 8 * h2);
            else q[nb][kk] = Frag{};
        }
    }

    float16v o[NB][DN] = {};
    float m[NB], l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) m[nb] = -INFINITY, l[nb] = 0.0f;
    int eref = 0;
    bool begun = false;
    const int block_shift = a.cache.block >> 7;  // 64, 128, 256 tokens: 1, 2, 4 steps

    // Loads run ahead of what waits for them: a step's codes and scales are asked for one step before, its block two steps
    // before (the address depends on it).
    uint4 kc[kUnits], vc[kUnits];
    float ks_next = 0.0f, vs_next = 0.0f;
    bool ok_next = false;
    int page_next;
    auto page_of = [&](int step) { return a.seq.table[b * a.seq.ldt + (min(step, to - 1) >> block_shift)]; };
    auto fetch = [&](int step) {
        const int sub = step & ((1 << block_shift) - 1);
        int page = __builtin_amdgcn_readfirstlane(page_next);
        ok_next = page >= 0 && page < a.cache.blocks;
        if (!ok_next) page = 0;
        const int64_t unit = (int64_t)page * H + head;
        const uint8_t *kp = a.cache.k + (unit * a.cache.block + sub * kCacheTile) * D;
        const uint8_t *vp = a.cache.v + unit * D * a.cache.block + sub * kCacheTile;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = tid + u * NT;
            kc[u] = *(const uint4 *)(kp + 16 * at);
            vc[u] = *(const uint4 *)(vp + (at >> 2) * a.cache.block + 16 * (at & 3));
        }
        ks_next = a.cache.k_scale[unit];
        vs_next = a.cache.v_scale[unit];
        page_next = page_of(step + 1);
    };
    auto stage = [&](int step, int buffer) {
        // a slot behind the sequence holds anything, a NaN too: its weight 0 does not hide that
        const bool tail = !ok_next || (step + 1) * kCacheTile > s.len;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = tid + u * NT, token = at / KK, c = 2 * (at % KK);
            const int row = (token & 32) + 8 * (token >> 2 & 3) + 4 * (token >> 4 & 1) + (token & 3), k0 = row * (D / 8), swap = key_swap<D>(row);
            union {
                Frag f;
                uint4 w;
            } x, y;
            x.f = widen<T>(kc[u].x, kc[u].y), y.f = widen<T>(kc[u].z, kc[u].w);
            keys[buffer][k0 + (c ^ swap)] = x.w;
            keys[buffer][k0 + ((c + 1) ^ swap)] = y.w;
            const int d = at >> 2, cv = 2 * (at & 3);
            uint4 codes = vc[u];
            if (tail) {
                const int valid = ok_next ? s.len - step * kCacheTile - 16 * (at & 3) : 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int bytes = min(max(valid - 4 * w, 0), 4);
                    (&codes.x)[w] &= bytes == 4 ? 0xffffffffu : (1u << (8 * bytes)) - 1;
                }
            }
            union {
                half8 f;
                uint4 w;
            } v, z;
            v.f = widen<_Float16>(codes.x, codes.y), z.f = widen<_Float16>(codes.z, codes.w);
            values[buffer][d * 8 + (cv ^ (d >> 1 & 7))] = v.w;
            values[buffer][d * 8 + ((cv + 1) ^ (d >> 1 & 7))] = z.w;
        }
    };

    if (from < to) {
        page_next = page_of(from);
        fetch(from);
        stage(from, 0);
    }
    for (int step = from; step < to; ++step) {
        const int buffer = (step - from) & 1;
        const float ks = ks_next, vs = vs_next;
        const bool ok = ok_next;
        __syncthreads();
        if (step + 1 < to) fetch(step + 1);
        if (ok && step * kCacheTile < mine.end && (step + 1) * kCacheTile > mine.begin) {  // else no row of this wavefront sees any of these keys
            float16v sc[NB][2] = {};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    const int row = 32 * kb + q32;
                    const Frag f = *(const Frag *)&keys[buffer][row * (D / 8) + ((2 * kk + h2) ^ key_swap<D>(row))];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) sc[nb][kb] = Mma<T>::mma(f, q[nb][kk], sc[nb][kb]);
                }
            if ((step + 1) * kCacheTile > mine.all_end || step * kCacheTile < mine.all_begin) {
                const int key0 = step * kCacheTile + 16 * h2;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int key = key0 + 32 * kb + r;
                            sc[nb][kb][r] = ((key > see_hi[nb]) | (key < see_lo[nb])) ? -INFINITY : sc[nb][kb][r];
                        }
            }
            const float c = fmaxf(a.alpha * kLog2e * ks, 1.17549435e-38f);
            const int ev = __builtin_amdgcn_readfirstlane(exponent_of(vs));
            if (!begun) eref = ev, begun = true;
            if (ev - eref > kDrift || eref - ev > kDrift) {
                const float f = pow2(eref - ev);
                eref = ev;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int n = 0; n < DN; ++n) o[nb][n] *= f;
            }
            const float drift = (float)(ev - eref), undrift = pow2(eref - ev);
            half8 p[NB][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float top = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; r += 2) top = most(top, most(sc[nb][kb][r], sc[nb][kb][r + 1]));
                top *= c;
                if (__any(top > m[nb] + kSlack)) {
                    const float now = fmaxf(m[nb], fmaxf(top, __shfl_xor(top, 32)));
                    const float f = m[nb] == -INFINITY ? 0.0f : exp2f(m[nb] - now);
                    m[nb] = now;
                    l[nb] *= f;
#pragma unroll
                    for (int n = 0; n < DN; ++n) o[nb][n] *= f;
                }
                const float base = (m[nb] == -INFINITY ? 0.0f : m[nb]) - drift;
                float sum[4] = {};
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        float w[8];
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            w[r] = __builtin_amdgcn_exp2f(fmaf(sc[nb][kb][8 * hf + r], c, -base));
                            sum[r & 3] += w[r];
                        }
                        p[nb][2 * kb + hf] = half8{(_Float16)w[0], (_Float16)w[1], (_Float16)w[2], (_Float16)w[3], (_Float16)w[4], (_Float16)w[5], (_Float16)w[6], (_Float16)w[7]};
                    }
                l[nb] = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), undrift, l[nb]);
            }
#pragma unroll
            for (int n = 0; n < DN; ++n)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int d = 32 * n + q32;
                    const half8 f = *(const half8 *)&values[buffer][d * 8 + ((4 * (t >> 1) + 2 * h2 + (t & 1)) ^ (d >> 1 & 7))];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) o[nb][n] = Mma<_Float16>::mma(f, p[nb][t], o[nb][n]);
                }
        }
        if (step + 1 < to) stage(step + 1, buffer ^ 1);
    }

    // o[nb][n][r]: query q32 of the nb-th 32, channel 32 n + 8 (r / 4) + 4 h2 + r % 4, in units of 2^eref
    const float unit = pow2(eref);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const float sum = l[nb] + __shfl_xor(l[nb], 32);
        const int64_t row = first + wave * R + nb * 32 + q32;
        if (row >= total) continue;
#pragma unroll
        for (int n = 0; n < DN; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                give<T, D>(a, s, head, group, split, row, 32 * n + 8 * r + 4 * h2, float4v{o[nb][n][4 * r], o[nb][n][4 * r + 1], o[nb][n][4 * r + 2], o[nb][n][4 * r + 3]} * unit,
                           m[nb], sum, n == 0 && r == 0 && h2 == 0);
    }
}

// The parts of one row: a workgroup per row, some threads for each four channels.
constexpr int kMostSplits = 128;
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cache_attention_join(CacheAttentionArgs a)
{
    constexpr int C = D / 4, kSide = 256 / C;  // parts side by side
    __shared__ float weight[kMostSplits], total[2];
    __shared__ float4v side[kSide][C];
    const int tid = threadIdx.x, h = (int)(blockIdx.x % a.heads);
    const unsigned bt = blockIdx.x / a.heads;
    const int b = (int)(bt / a.seq.max_new), t = (int)(bt % a.seq.max_new);
    const Seq s = sequence(a.seq, b);
    if (t >= s.n) return;
    const int64_t all_rows = (int64_t)a.seq.M * a.heads, row = (int64_t)(s.row + t) * a.heads + h;
    if (tid < 64) {
        const float2 *ml = (const float2 *)(a.partial + a.splits * all_rows * D) + row;
        float2 p[kMostSplits / 64];
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kMostSplits / 64; ++j) {
            p[j] = tid + 64 * j < a.splits ? ml[(tid + 64 * j) * all_rows] : make_float2(-INFINITY, 0.0f);
            top = fmaxf(top, p[j].x);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
#pragma unroll
        for (int j = 0; j < kMostSplits / 64; ++j) {
            const float f = p[j].x == -INFINITY && p[j].y == 0.0f ? 0.0f : exp2f(p[j].x - top);
            weight[tid + 64 * j] = f;
            sum = fmaf(f, p[j].y, sum);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        if (tid == 0) total[0] = top, total[1] = sum;
    }
    __syncthreads();
    const int c = tid % C, first = tid / C;
    const float *o = a.partial + row * D + 4 * c;
    float4v x = {};
#pragma unroll 4
    for (int k = first; k < a.splits; k += kSide) x += *(const float4v *)(o + k * all_rows * D) * weight[k];
    side[first][c] = x;
    __syncthreads();
    if (first) return;
#pragma unroll
    for (int k = 1; k < kSide; ++k) x += side[k][c];
    const float sum = total[1], f = sum == 0.0f ? 0.0f : 1.0f / sum;
    *(uint2 *)((T *)a.out + (s.row + t) * a.ldo + (int64_t)h * D + 4 * c) = make_uint2(Half<T>::pack(x[0] * f, x[1] * f), Half<T>::pack(x[2] * f, x[3] * f));
    if (c == 0 && a.lse) a.lse[row] = kLn2 * (total[0] + log2f(sum));
}

// Rows a workgroup takes: up to 16 or 32 shared by four wavefronts, else 32 for each of four.
struct Shape {
    int rows;
    bool shared;
};
Shape shape_of(int64_t rows, int dim)
{
    if (rows <= 16) return {16, true};
    if (rows <= 32 && dim < 256) return {32, true};
    return {128, false};
}
constexpr int kAttWaves = 4;

template <typename T, int D>
void launch(const CacheAttentionArgs &a, const Shape &shape, int row_tiles, int64_t groups, hipStream_t st)
{
    constexpr int NB = D < 256 ? 2 : 1;
    const dim3 grid((unsigned)groups), block(kAttWaves * 64);
    if (!shape.shared)
        hipLaunchKernelGGL((k_cache_attention_rows<T, D, 1, kAttWaves>), grid, block, 0, st, a, row_tiles);
    else if (shape.rows == 16)
        hipLaunchKernelGGL((k_cache_attention<T, D, 1, kAttWaves>), grid, block, 0, st, a, row_tiles);
    else
        hipLaunchKernelGGL((k_cache_attention<T, D, NB, kAttWaves>), grid, block, 0, st, a, row_tiles);
    if (a.splits > 1) {
        const int64_t rows = (int64_t)a.seq.batch * a.seq.max_new * a.heads;
        hipLaunchKernelGGL((k_cache_attention_join<T, D>), dim3((unsigned)rows), block, 0, st, a);
    }
}

template <typename T>
void launch_type(const CacheAttentionArgs &a, const Shape &shape, int row_tiles, int64_t groups, hipStream_t st)
{
    if (a.cache.dim == 64) launch<T, 64>(a, shape, row_tiles, groups, st);
    else if (a.cache.dim == 128) launch<T, 128>(a, shape, row_tiles, groups, st);
    else launch<T, 256>(a, shape, row_tiles, groups, st);
}

}  // namespace

double cache_attention_groups(int batch, int heads, int kv_heads, int dim, int max_new, int splits)
{
    const int64_t rows = (int64_t)max_new * (heads / kv_heads);
    const Shape shape = shape_of(rows, dim);
    return (double)((rows + shape.rows - 1) / shape.rows) * batch * kv_heads * splits;
}

int cache_attention_splits(int batch, int heads, int kv_heads, int dim, int max_new, int max_len)
{
    const int64_t rows = (int64_t)max_new * (heads / kv_heads);
    const Shape shape = shape_of(rows, dim);
    const double groups = cache_attention_groups(batch, heads, kv_heads, dim, max_new, 1);
    const int64_t steps = ((int64_t)max_len + kCacheTile - 1) / kCacheTile;
    // four workgroups for every compute unit, as long as each of their wavefronts still has a few steps
    if (!shape.shared && groups >= 256) return 1;
    const int64_t want = groups >= 1024 ? 1 : (int64_t)((1024 + groups - 1) / groups), most = steps / (shape.shared ? kAttWaves : 4);
    const int64_t s = want < most ? want : most;
    return (int)(s < 1 ? 1 : s > kMostSplits ? kMostSplits : s);
}

hipError_t launch_cache_attention(const CacheAttentionArgs &a, hipStream_t st)
{
    const int64_t rows = (int64_t)a.seq.max_new * (a.heads / a.cache.heads);
    const Shape shape = shape_of(rows, a.cache.dim);
    const int row_tiles = (int)((rows + shape.rows - 1) / shape.rows);
    const int64_t groups = (int64_t)row_tiles * a.seq.batch * a.cache.heads * a.splits;
    if (a.bf16)
        launch_type<__bf16>(a, shape, row_tiles, groups, st);
    else
        launch_type<_Float16>(a, shape, row_tiles, groups, st);
    return hipGetLastError();
}

}  // namespace bwta
