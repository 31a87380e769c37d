// Attention of 16-bit queries over the 8-bit cache, in one pass over the keys:
//   out = sum_j p_j v_j / sum_j p_j,   p_j = 2^(s_j - m),   s_j = alpha log2(e) q . k_j,   m near a running maximum
// with sums and scores in fp32.
//
// Codes are exact in both 16-bit types, so q . k is the matrix cores' sum of exact products; a block's key scale joins
// alpha.  Value codes enter without their scale 2^e, which joins the weights: s_j + e - m is the exponent of what the second
// product takes, rounded to fp16 whatever the queries' type (11 bits to bf16's 8).  m is moved when an exponent exceeds 15, so
// that it becomes 11: the upper end of fp16's range.  A weight times scale is then off by at most 2^-11 of itself, or 2^-25 where
// the row's largest is 2^11 or more, 2^-36 of that, which is less than sums in fp32 lose.  What m was moved for last is
// exactly 2^11, so a row that one key rules does not feel the rounding; and the log-sum-exp sums the weights in fp32.
//
// The first product is computed transposed, keys by queries: its result has a query per
// lane and, with the key rows taken in the right order (row 4 i + r of the b-th 16 is token 16 i + 4 b + r), 16 tokens in
// a row per lane, which is what the second product (values transposed by queries) wants as its operand.  Keys are loaded
// as 16 codes of a token, values as 16 tokens of a channel, both 16 bytes in a row in the cache's layout.
#include "bwta_heads.h"
#include <type_traits>

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

constexpr float kHighest = 15.0f, kPlace = 11.0f;  // exponents of weights: where m has to move, and what the moved one leaves
constexpr float kNothing = -3e38f;                  // m before any key has been seen
// m for keys of which the largest has exponent e.  (As it was for a NaN, and for the -Inf of keys that are not seen.)  On a grid of
// 2^-16, so that what is added to it below, whole numbers, is exact; that largest one's weight is 2^kPlace but for 2^-17 of it.
__device__ __forceinline__ float moved(float e, float m)
{
    if (!(e > m + kHighest)) return m;
    const float x = e - kPlace;
    return fabsf(x) < 128.0f ? rintf(x * 65536.0f) * (1.0f / 65536.0f) : x;
}
// The natural logarithm of l 2^m, rounded once: m and l's exponent join first.
__device__ __forceinline__ float log_of(float m, float l)
{
    return fmaf(m + (float)__builtin_amdgcn_frexp_expf(l), kLn2, kLn2 * log2f(__builtin_amdgcn_frexp_mantf(l)));
}

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

// Rows of one sequence and key head: row r is query head r % group of the r / group-th new token.  What all of them see,
// taken together: steps of 64 keys from step0 on, of which keys all_begin to all_end - 1 are seen by each.
struct Reach {
    int rows, step0, steps, units, all_begin, all_end;  // units: steps, at least one where there are rows
};
__device__ __forceinline__ Reach reach(const CacheAttentionArgs &a, const Seq &s)
{
    const int group = a.heads / a.cache.heads, n = min(s.n, a.seq.max_new);
    Reach r;
    r.rows = n * group;
    const int end = a.causal ? max(0, min(s.len, s.start + n)) : s.len, begin = a.window ? max(0, s.start - a.window + 1) : 0;
    r.step0 = begin / kCacheTile;
    r.steps = max(0, (end + kCacheTile - 1) / kCacheTile - r.step0);
    r.units = n > 0 ? max(r.steps, 1) : 0;
    r.all_end = a.causal ? min(s.len, s.start + 1) : s.len;
    r.all_begin = a.window ? s.start + n - a.window : 0;
    return r;
}

// Four channels of a result.  Averages of finite values stay finite: a code may stand for more than fp16 has (65504 is held as
// 256 * 2^8, infinities as 448 * 2^e), and what is beyond the type's range is its largest, as in reading.
template <typename T>
__device__ __forceinline__ uint2 result(float4v x, float f)
{
    auto fit = [&](float y) { return y * f != y * f ? y * f : fminf(fmaxf(y * f, -Half<T>::kMax), Half<T>::kMax); };  // (a NaN stays one)
    return make_uint2(Half<T>::pack(fit(x[0]), fit(x[1])), Half<T>::pack(fit(x[2]), fit(x[3])));
}

// Four channels of a row, and once per row its m and sum: the result, or the part of it that
// `part` says is kept for the join.
template <typename T, int D>
__device__ __forceinline__ void give(const CacheAttentionArgs &a, const Seq &s, int head, int group, int64_t part, int row, int channel, float4v x, float m, float l, bool once)
{
    if (part >= 0) {
        *(float4v *)(a.partial + part * D + channel) = x;
        if (once) ((float2 *)(a.partial + a.part_rows * D))[part] = make_float2(m, l);
        return;
    }
    const int t = (unsigned)row / (unsigned)group, h = head * group + (row - t * group);
    const int64_t token = s.row + t;
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    *(uint2 *)((T *)a.out + token * a.ldo + (int64_t)h * D + channel) = result<T>(x, f);
    if (once && a.lse) a.lse[token * a.heads + h] = log_of(m, l);
}

// Workgroups that share `total` steps, as a power of two: not more than there are, so that everybody has one; and where the
// w-th one's begin.
__device__ __forceinline__ int shares_log2(const CacheAttentionArgs &a, int total) { return total > 0 ? min(a.share_log2, 31 - __builtin_clz(total)) : 0; }
__device__ __forceinline__ int share_begin(unsigned w, int total, int log2) { return (int)((uint64_t)w * (unsigned)total >> log2); }

// units of all sequences before each, behind the parts
__device__ __forceinline__ int *shares_of(const CacheAttentionArgs &a) { return (int *)(a.partial + a.part_rows * (a.cache.dim + 2)); }

// Few rows (decoding): a workgroup has all NB * 16, and its wavefronts take turns at the steps of 64 keys, each with what it
// needs in registers and nothing in LDS until their sums are joined; 16 rows is what the matrix cores take anyway, so heads that
// share their keys cost nothing.  Bound by the cache's bytes: 64 sequences of 2048 to 8192 tokens, 32 heads on 8 of 128 (680 MB)
// take 119 us, 5.7 TB/s, equal ones of 8192 6.4 TB/s; one token over 131072 keys (268 MB) 48.8 us with the join, over 2048 keys
// of 32 heads (17 MB) 9.5 us, most of it the latency of lengths, table and codes one after the other, and of a second launch.
// 17 to 32 rows of heads of 128 take all the registers of a SIMD for one wavefront, or in workgroups of eight, which need two on
// a SIMD, leave some in scratch, which they read outside the steps.
template <typename T, int D, int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, (NB == 1 && D <= 128) ? 2 : 1) void k_cache_attention(CacheAttentionArgs a)
{
    constexpr int R = 16 * NB, KL = D / 64, NV = D / 16;
    typedef typename Mma<T>::Frag Frag;
    __shared__ float4 merged[WAVES * R * (D / 4)];
    __shared__ float2 merged_ml[WAVES * R];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q16 = lane & 15, g = lane >> 4;
    const int H = a.cache.heads, group = a.heads / H;

    // This workgroup's part: one of a sequence's and head's `splits`, or its share of all steps of all sequences and heads in a
    // row (lengths may differ, and only the device knows them).
    int b, head, off = 0, left;
    int64_t part = -1;
    Seq s;
    Reach see;
    auto look_at = [&](int sequence_) { s = sequence(a.seq, sequence_), see = reach(a, s); };
    if (a.share_log2 < 0) {
        const int bh = blockIdx.x / a.splits, split = blockIdx.x - bh * a.splits;
        b = bh / H, head = bh - b * H;
        look_at(b);
        off = (unsigned)(see.units * split) / (unsigned)a.splits;
        left = (unsigned)(see.units * (split + 1)) / (unsigned)a.splits - off;
        if (a.splits > 1) part = blockIdx.x;
        if (left == 0) {  // fewer steps than splits: nothing to add
            for (int at = threadIdx.x; at < see.rows * (D / 4); at += WAVES * 64)
                give<T, D>(a, s, 0, 1, part * R + at / (D / 4), 0, at % (D / 4) * 4, float4v{}, kNothing, 0.0f, at % (D / 4) == 0);
            return;
        }
    } else {
        // every wavefront for itself: a lane has some of the sequences, in a row
        const int each = (a.seq.batch + 63) / 64, b0 = min(lane * each, a.seq.batch), b1 = min(b0 + each, a.seq.batch);
        int mine = 0;
        for (int s = b0; s < b1; ++s) mine += reach(a, sequence(a.seq, s)).units;
        int upto = mine;
        if (each * 2 <= a.seq.batch) {  // more than one lane has any
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
        }
        const int before = upto - mine, all = __builtin_amdgcn_readlane(upto, min(63, (a.seq.batch - 1) / each));
        const int total = all * H, share_log2 = shares_log2(a, total);  // below 2^31: the host's bound
        const int u0 = share_begin(blockIdx.x, total, share_log2), u1 = share_begin(blockIdx.x + 1, total, share_log2);
        if (blockIdx.x == 0 && wave == 0) {  // for those who join the parts
            int *const table = shares_of(a);
            for (int s = b0, at = before; s < b1; ++s) {
                table[s] = at;
                at += reach(a, sequence(a.seq, s)).units;
            }
            if (lane == 0) table[a.seq.batch] = all;
        }
        if (blockIdx.x >> share_log2 || total == 0) return;
        const int owner = __builtin_ctzll(__ballot(u0 < upto * H));  // the first lane whose sequences reach so far
        int at = __builtin_amdgcn_readlane(before, owner);
        for (b = owner * each;; ++b, at += see.units) {
            if (b >= a.seq.batch) return;  // only if the lengths change meanwhile
            look_at(b);
            if (u0 < (at + see.units) * H) break;
        }
        off = u0 - at * H;
        head = off / see.units, off -= head * see.units;
        left = u1 - u0;
    }

    for (;;) {
        const int take = min(see.units - off, left);
        if (a.share_log2 >= 0) part = take == see.units ? -1 : 2 * (int64_t)blockIdx.x + (off == 0);  // what began in another workgroup, or ends in one
        const int total = see.rows, from = see.step0 + off, to = min(from + take, see.step0 + see.steps);

        const int block_shift = a.cache.block >> 7;  // 64, 128, 256 tokens: 1, 2, 4 steps
        const int key_row = 16 * (q16 >> 2) + (q16 & 3);  // + 4 b

        // A turn's loads all leave at once, and its block (the address depends on it) is asked for one turn before.  Keeping the
        // next turn's codes in registers as well took longer (64 sequences of up to 8192 keys 119 us, 123 with them).
        struct Turn {
            uint4 k[4][KL], v[NV];
            float ks, vs;
            int page;
            bool ok;
        };
        auto page_of = [&](int step) { return a.seq.table[b * a.seq.ldt + (min(step, to - 1) >> block_shift)]; };
        // (each code is read by one wavefront once: a batch of 32 sequences of 4096 tokens, 32 key heads, 5.1 TB/s through the
        // caches' order, 6.2 past it)
        auto fetch = [&](Turn &x, int step) {
            const int sub = step & ((1 << block_shift) - 1);
            int page = __builtin_amdgcn_readfirstlane(x.page);
            x.page = page_of(step + WAVES);
            x.ok = page >= 0 && page < a.cache.blocks;
            if (!x.ok) page = 0;
            const int64_t unit = (int64_t)page * H + head;
            const uint8_t *kp = a.cache.k + (unit * a.cache.block + sub * kCacheTile) * D;
            const uint8_t *vp = a.cache.v + unit * D * a.cache.block + sub * kCacheTile;
            x.ks = a.cache.k_scale[unit];
            x.vs = a.cache.v_scale[unit];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int j = 0; j < KL; ++j) x.k[kb][j] = load_once(kp + (key_row + 4 * kb) * D + 64 * j + 16 * g);
#pragma unroll
            for (int n = 0; n < NV; ++n) x.v[n] = load_once(vp + (16 * n + q16) * a.cache.block + 16 * g);
        };
        Turn turn;
        turn.page = from + wave < to ? page_of(from + wave) : -1;

        // this lane's query of each 16
        int see_lo[NB], see_hi[NB];
        Frag q[NB][2 * KL];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int row = nb * 16 + q16;
            const bool has = row < total;
            const int t = has ? (unsigned)row / (unsigned)group : 0, h = head * group + (has ? row - t * group : 0);
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
        for (int nb = 0; nb < NB; ++nb) m[nb] = kNothing, l[nb] = 0.0f;
        auto compute = [&](Turn &x, int step) {
            float4v sc[NB][4] = {};
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int j = 0; j < KL; ++j) {
                    const Frag k0 = widen<T>(x.k[kb][j].x, x.k[kb][j].y), k1 = widen<T>(x.k[kb][j].z, x.k[kb][j].w);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        sc[nb][kb] = Mma<T>::mma(k0, q[nb][2 * j], sc[nb][kb]);
                        sc[nb][kb] = Mma<T>::mma(k1, q[nb][2 * j + 1], sc[nb][kb]);
                    }
                }

            const int key0 = step * kCacheTile + 16 * g;  // this lane's first key
            if (!x.ok || (step + 1) * kCacheTile > see.all_end || step * kCacheTile < see.all_begin) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const int hi = x.ok ? see_hi[nb] : -1, lo = see_lo[nb];
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
            if (!x.ok || (step + 1) * kCacheTile > s.len) {
                const int valid = x.ok ? s.len - key0 : 0;
#pragma unroll
                for (int n = 0; n < NV; ++n)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int bytes = min(max(valid - 4 * w, 0), 4);
                        (&x.v[n].x)[w] &= bytes == 4 ? 0xffffffffu : (1u << (8 * bytes)) - 1;
                    }
            }

            const float c = fmaxf(a.alpha * kLog2e * x.ks, 1.17549435e-38f);
            // (a block that is not there has no scale: what memory holds in its place decides nothing)
            const int ev = x.ok ? __builtin_amdgcn_readfirstlane(exponent_of(x.vs)) : 0;
            half8 p[NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float top = most(most(sc[nb][0][0], sc[nb][0][1]), most(sc[nb][0][2], sc[nb][0][3]));
#pragma unroll
                for (int kb = 1; kb < 4; ++kb) top = most(most(top, most(sc[nb][kb][0], sc[nb][kb][1])), most(sc[nb][kb][2], sc[nb][kb][3]));
                top = fmaf(top, c, (float)ev);
                if (__any(top > m[nb] + kHighest)) {
                    const float to = moved(max_of_query(top), m[nb]);
                    const float f = exp2f(m[nb] - to);
                    m[nb] = to;
                    l[nb] *= f;
#pragma unroll
                    for (int n = 0; n < NV; ++n) o[nb][n] *= f;
                }
                const float base = m[nb] - (float)ev;
                float sum = 0.0f, w[16];
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        w[4 * kb + r] = __builtin_amdgcn_exp2f(fmaf(sc[nb][kb][r], c, -base));
                        sum += w[4 * kb + r];
                    }
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    p[nb][hf] = half8{(_Float16)w[8 * hf], (_Float16)w[8 * hf + 1], (_Float16)w[8 * hf + 2], (_Float16)w[8 * hf + 3],
                                      (_Float16)w[8 * hf + 4], (_Float16)w[8 * hf + 5], (_Float16)w[8 * hf + 6], (_Float16)w[8 * hf + 7]};
                l[nb] = fmaf(sum, pow2(-ev), l[nb]);  // the sum of weights alone knows no value's scale
            }
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const half8 v0 = widen<_Float16>(x.v[n].x, x.v[n].y), v1 = widen<_Float16>(x.v[n].z, x.v[n].w);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    o[nb][n] = Mma<_Float16>::mma(v0, p[nb][0], o[nb][n]);
                    o[nb][n] = Mma<_Float16>::mma(v1, p[nb][1], o[nb][n]);
                }
            }
        };
        for (int step = from + wave; step < to; step += WAVES) {
            fetch(turn, step);
            compute(turn, step);
        }

        // o[nb][n][r]: query q16 of the nb-th 16, channel 16 n + 4 g + r
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) l[nb] = sum_of_query(l[nb]);
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
            if (r >= total) continue;
            float top = kNothing, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, merged_ml[w * R + r].x);
            float4v x = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float2 ml = merged_ml[w * R + r];
                const float f = exp2f(ml.x - top);
                const float4 y = merged[w * R * (D / 4) + at];
                x += float4v{y.x, y.y, y.z, y.w} * f;
                sum = fmaf(ml.y, f, sum);
            }
            give<T, D>(a, s, head, group, part < 0 ? -1 : part * R + r, r, at % (D / 4) * 4, x, top, sum, at % (D / 4) == 0);
        }

        left -= take, off += take;
        if (left == 0) break;
        off = 0;  // another workgroup's share ends inside a head's steps, this one's goes on with the next
        if (++head == H) {
            head = 0;
            do {
                if (++b >= a.seq.batch) return;  // as above
                look_at(b);
            } while (see.units == 0);
        }
        __syncthreads();  // before the next part's sums
    }
}

// Where a row's sixteen-byte chunk lies in LDS: rows are one chunk longer than they need be, so that the sixteen rows that are
// read at a time cover all banks once, and a lane's chunks are constant offsets from one address.
template <int CHUNKS>
__device__ __forceinline__ constexpr int padded(int row, int chunk) { return row * (CHUNKS + 1) + chunk; }

// What one tile of 128 rows of a sequence and key head sees.
struct RowsReach {
    int step0, steps, units;  // as Reach's
};
constexpr int kTileRows = 128, kMostShared = 1024;  // tiles that are shared at most (sequences, too: a workgroup counts each one's steps)
__device__ __forceinline__ RowsReach rows_reach(const CacheAttentionArgs &a, const Seq &s, int group, int total, int tile)
{
    const int first = tile * kTileRows, last = min(first + kTileRows, total) - 1;
    const int t_first = (unsigned)first / (unsigned)group, t_last = (unsigned)last / (unsigned)group;
    const int end = a.causal ? max(0, min(s.len, s.start + t_last + 1)) : s.len, begin = a.window ? max(0, s.start + t_first - a.window + 1) : 0;
    RowsReach r;
    r.step0 = begin / kCacheTile;
    r.steps = max(0, (end + kCacheTile - 1) / kCacheTile - r.step0);
    r.units = max(r.steps, 1);
    return r;
}
// where each sharing workgroup begins, behind the parts: sequence (-1: nowhere), head, tile, steps of the tile before it
__device__ __forceinline__ int4 *begins_of(const CacheAttentionArgs &a) { return (int4 *)(a.partial + a.part_rows * (a.cache.dim + 2)); }

// Many rows: each wavefront has 32 of its own, and four wavefronts share the keys and values of a step, which reach LDS as
// 16-bit numbers (each code is widened once for the four).  Products of 32 x 32: key row 8 i + 4 j + r of a block of 32 is
// token 16 j + 4 i + r, so a lane again has 16 tokens in a row.
// A turn computes the scores of the next step beside the weights and the sums of this one: matrix cores and vector ALU have
// work that does not wait for each other's.  Keys are therefore fetched one step before values.
// With GROUPS = 2 a workgroup has the rows twice: one four take the even steps, the other the odd ones, and their sums are
// joined through LDS.
// With SHARES workgroups share all steps equally: those of a sequence's first head's first 128 rows, second 128 and so on, next
// head, next sequence.  What begins or ends inside somebody else's share becomes a part, and each leaves where it begins for
// the join.
// A step of 32 rows of heads of 128 is 1024 cycles of matrix cores and some 1100 of vector ALU (32 weights a lane with a fused
// multiply-add, a power, an addition and half a conversion each, and the widening), and 32 KB from LDS a wavefront.  Counted in
// chunks of long prompts, a SIMD takes 2400 cycles a step: matrix cores are busy 43 % of them, the vector ALU 50 %, seldom both.
// Its two wavefronts wait for their turn to issue 28 % of their time, and 26 % for memory, LDS and each other.  8192 keys for each
// of 2048 rows, 32 heads of 128: 980 TFLOP/s with one group, and 800 with two (16 heads, 1024 rows), where a large fp16 product
// reaches 1322; 64 rows a wavefront need more registers than the vector ALU can address and copy sums between the two files at
// every step (half as fast), codes widened by each wavefront cost it 128 conversions a step for 32 (5 % slower).  Heads of 128
// need 7 to 13 registers more than there are: 32 to 56 bytes a lane lie in scratch and are read at a tile's ends, outside the steps.
template <typename T, int D, int GROUPS, bool SHARES>
__global__ __launch_bounds__(GROUPS * 256, D <= 128 ? 2 : 1) void k_cache_attention_rows(CacheAttentionArgs a, int row_tiles)
{
    constexpr int WAVES = 4, R = 32, kRows = kTileRows, NT = WAVES * 64, KK = D / 16, DN = D / 32, kUnits = 4 * D / NT;
    typedef typename Mma<T>::Frag Frag;
    struct Tile {
        uint4 keys[kCacheTile * (D / 8 + 1)], values[D * (kCacheTile / 8 + 1)];
    };
    __shared__ Tile tiles[GROUPS][2];
    const int side = __builtin_amdgcn_readfirstlane(threadIdx.x / NT), tid = threadIdx.x % NT;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q32 = lane & 31, h2 = lane >> 5;
    const int H = a.cache.heads, group = a.heads / H;

    int b, head, tile_of_rows, off = 0, left = 0;
    unsigned share = 0;
    Seq s;
    if constexpr (!SHARES) {
        // Causal rows at the end see most: first.  Workgroups go around the eight XCDs, and inside one around its four shader
        // engines, in order: consecutive ones have the heads of a sequence, and sequences change places from one round of all of
        // them to the next, or a long one would always fall to the same engines (half of the time of a ragged batch of four).
        const unsigned i = blockIdx.x / a.splits;
        const int round = (int)(i / (a.seq.batch * H)), bh = i % (a.seq.batch * H);
        head = bh % H, b = (bh / H + round) % a.seq.batch;
        tile_of_rows = row_tiles - 1 - round;
        s = sequence_of_all(a.seq, b);
        if (tile_of_rows * kRows >= min(s.n, a.seq.max_new) * group) return;
    } else {
        // steps of each sequence, for one head
        int *const steps_of = (int *)&tiles[0][0];
        static_assert(sizeof(tiles) >= kMostShared * sizeof(int), "the counts go where keys and values will be");
        for (int i = threadIdx.x; i < a.seq.batch; i += GROUPS * NT) steps_of[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < a.seq.batch * row_tiles; i += GROUPS * NT) {
            const int c = i / row_tiles, tile = i - c * row_tiles;
            const Seq x = sequence(a.seq, c);
            const int total = min(x.n, a.seq.max_new) * group;
            if (tile * kRows < total) atomicAdd(&steps_of[c], rows_reach(a, x, group, total, tile).units);
        }
        __syncthreads();
        const int each = (a.seq.batch + 63) / 64, b0 = min(lane * each, a.seq.batch), b1 = min(b0 + each, a.seq.batch);
        int mine = 0;
        for (int c = b0; c < b1; ++c) mine += steps_of[c];
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(upto, d);
            if (lane >= d) upto += x;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63) * H, share_log2 = shares_log2(a, all);  // below 2^31: the host's bound
        // an XCD's workgroups (every eighth) have shares in a row, of few heads: their keys and values stay in its L2
        const unsigned low = blockIdx.x & ((1u << share_log2) - 1);
        share = share_log2 < 3 ? blockIdx.x : (blockIdx.x - low) | (low & 7) << (share_log2 - 3) | low >> 3;
        if (share >> share_log2 || all == 0) {
            if (threadIdx.x == 0) begins_of(a)[share] = make_int4(-1, 0, 0, 0);
            return;
        }
        const int u0 = share_begin(share, all, share_log2);
        left = share_begin(share + 1, all, share_log2) - u0;
        const int owner = __builtin_ctzll(__ballot(u0 < upto * H));  // the first lane whose sequences reach so far
        int at = __builtin_amdgcn_readlane(upto - mine, owner);
        for (b = owner * each;; ++b) {
            const int of = __builtin_amdgcn_readfirstlane(steps_of[b]);
            if (u0 < (at + of) * H) {
                off = u0 - at * H;
                head = off / of, off -= head * of;
                break;
            }
            at += of;
        }
        s = sequence_of_all(a.seq, b);
        const int total = min(s.n, a.seq.max_new) * group, last_tile = (total - 1) / kRows;
        for (tile_of_rows = 0;; tile_of_rows += 64) {
            const int tile = tile_of_rows + lane, units = tile <= last_tile ? rows_reach(a, s, group, total, tile).units : 0;
            int to = units;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int x = __shfl_up(to, d);
                if (lane >= d) to += x;
            }
            const uint64_t reached = __ballot(off < to);
            if (reached || tile_of_rows + 64 > last_tile) {
                const int l = reached ? __builtin_ctzll(reached) : 0;
                off -= __builtin_amdgcn_readlane(to - units, l), tile_of_rows += l;
                break;
            }
            off -= __builtin_amdgcn_readlane(to, 63);
        }
        if (threadIdx.x == 0) begins_of(a)[share] = make_int4(b, head, tile_of_rows, off);
        __syncthreads();  // the counts are read
    }

    for (;;) {
        const int total = min(s.n, a.seq.max_new) * group, first = tile_of_rows * kRows;
        // keys that some row sees, and those that every row of this wavefront sees
        const RowsReach see = rows_reach(a, s, group, total, tile_of_rows);
        const int my_first = min(first + wave * R, total - 1), my_last = min(my_first + R, total) - 1;
        const int all_end = a.causal ? min(s.len, s.start + (int)((unsigned)my_first / (unsigned)group) + 1) : s.len;
        const int all_begin = a.window ? s.start + (int)((unsigned)my_last / (unsigned)group) - a.window + 1 : 0;
        int take = see.units, from = see.step0, to = see.step0 + see.steps;
        int64_t part0 = -1;  // of this tile's rows, if what comes out is a part of them
        if constexpr (SHARES) {
            take = max(min(see.units - off, left), 1);
            from += off, to = min(from + take, to);
            if (take < see.units) part0 = (2 * (int64_t)share + (off == 0)) * kRows;  // began in another workgroup's share, or ends in one
        } else if (a.splits > 1) {
            const int split = blockIdx.x % a.splits;
            from += (unsigned)(see.steps * split) / (unsigned)a.splits, to = see.step0 + (unsigned)(see.steps * (split + 1)) / (unsigned)a.splits;
        }

        // this lane's query
        const int row = first + wave * R + q32;
        const bool has = row < total;
        const int token = has ? (unsigned)row / (unsigned)group : 0;
        const int see_hi = !has ? -1 : a.causal ? min(s.len - 1, s.start + token) : s.len - 1, see_lo = a.window ? s.start + token - a.window + 1 : 0;
        Frag q[KK];
        const T *query = (const T *)a.q + (s.row + token) * a.ldq + (int64_t)(head * group + (has ? row - token * group : 0)) * D + 8 * h2;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (has) q[kk] = *(const Frag *)(query + 16 * kk);
            else q[kk] = Frag{};
        }

        float16v o[DN] = {};
        float m = kNothing, l = 0.0f, top = kNothing;
        const int block_shift = a.cache.block >> 7;  // 64, 128, 256 tokens: 1, 2, 4 steps

        // Loads run ahead of what waits for them.  Steps behind the last are the last again, but that nobody sees it, so that
        // nothing branches on them.
        typedef uint4 Codes[kUnits];
        Codes kc, vc;
        struct Step {
            int64_t unit;
            int step;
            float ks, vs;
            bool ok;
        };
        auto page_of = [&](int step) { return a.seq.table[b * a.seq.ldt + (min(step, to - 1) >> block_shift)]; };
        auto step_at = [&](int step, int page) {
            Step r;
            r.step = min(step, to - 1);
            page = __builtin_amdgcn_readfirstlane(page);
            r.ok = page >= 0 && page < a.cache.blocks;
            r.unit = (int64_t)(r.ok ? page : 0) * H + head;
            r.ok &= step < to;
            r.ks = a.cache.k_scale[r.unit];
            r.vs = a.cache.v_scale[r.unit];
            return r;
        };
        auto fetch_keys = [&](const Step &n, Codes &kc) {
            const uint8_t *kp = a.cache.k + (n.unit * a.cache.block + (n.step & ((1 << block_shift) - 1)) * kCacheTile) * D;
#pragma unroll
            for (int u = 0; u < kUnits; ++u) kc[u] = *(const uint4 *)(kp + 16 * (tid + u * NT));
        };
        auto fetch_values = [&](const Step &n) {
            const uint8_t *vp = a.cache.v + n.unit * D * a.cache.block + (n.step & ((1 << block_shift) - 1)) * kCacheTile;
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const int at = tid + u * NT;
                vc[u] = *(const uint4 *)(vp + (at >> 2) * a.cache.block + 16 * (at & 3));
            }
        };
        auto stage_keys = [&](const Codes &kc, int buffer) {
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const int at = tid + u * NT, token = at / KK, c = 2 * (at % KK);
                const int row = (token & 32) + 8 * (token >> 2 & 3) + 4 * (token >> 4 & 1) + (token & 3);
                *(Frag *)&tiles[side][buffer].keys[padded<D / 8>(row, c)] = widen<T>(kc[u].x, kc[u].y);
                *(Frag *)&tiles[side][buffer].keys[padded<D / 8>(row, c + 1)] = widen<T>(kc[u].z, kc[u].w);
            }
        };
        auto stage_values = [&](const Step &n, int buffer) {
            // a slot behind the sequence holds anything, a NaN too: its weight 0 does not hide that
            if (!n.ok || (n.step + 1) * kCacheTile > s.len) {
#pragma unroll
                for (int u = 0; u < kUnits; ++u) {
                    const int valid = n.ok ? s.len - n.step * kCacheTile - 16 * ((tid + u * NT) & 3) : 0;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int bytes = min(max(valid - 4 * w, 0), 4);
                        (&vc[u].x)[w] &= bytes == 4 ? 0xffffffffu : (1u << (8 * bytes)) - 1;
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const int at = tid + u * NT, d = at >> 2, c = 2 * (at & 3);
                *(half8 *)&tiles[side][buffer].values[padded<8>(d, c)] = widen<_Float16>(vc[u].x, vc[u].y);
                *(half8 *)&tiles[side][buffer].values[padded<8>(d, c + 1)] = widen<_Float16>(vc[u].z, vc[u].w);
            }
        };

        float16v now[2], ahead[2];  // scores of this step and of the next
        auto hide = [&](const Step &n) {  // keys that a row does not see
            if (!n.ok || (n.step + 1) * kCacheTile > all_end || n.step * kCacheTile < all_begin) {
                const int key0 = n.step * kCacheTile + 16 * h2, hi = n.ok ? see_hi : -1;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = key0 + 32 * kb + r;
                        ahead[kb][r] = ((key > hi) | (key < see_lo)) ? -INFINITY : ahead[kb][r];
                    }
            }
        };
        auto largest = [&] {
            float x = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; r += 2) x = most(x, most(ahead[kb][r], ahead[kb][r + 1]));
            return x;
        };
        auto score = [&](int buffer, int kb, int kk) {
            const Frag f = *(const Frag *)&tiles[side][buffer].keys[padded<D / 8>(32 * kb + q32, 2 * kk + h2)];
            ahead[kb] = Mma<T>::mma(f, q[kk], kk == 0 ? float16v{} : ahead[kb]);
        };

        if (from < to) {
            const int page0 = page_of(from + side), page1 = page_of(from + side + GROUPS);
            int page2 = page_of(from + side + 2 * GROUPS);
            Step s0 = step_at(from + side, page0), s1 = step_at(from + side + GROUPS, page1);
            {
                Codes first;
                fetch_keys(s0, first);
                fetch_values(s0);
                fetch_keys(s1, kc);
                stage_keys(first, 0);
                stage_values(s0, 0);
                stage_keys(kc, 1);
            }
            __syncthreads();
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) score(0, kb, kk);
            hide(s0);
            top = largest();
            // What the scales of a step come to is made ready in the step before (heads of 256, a prompt of 2048: 90 us, so 84).  A block
            // that is not there has no scale: what memory holds in its place decides nothing.
            float c;
            int ev;
            auto scales = [&](const Step &n) {
                c = fmaxf(a.alpha * kLog2e * n.ks, 1.17549435e-38f);
                ev = n.ok ? __builtin_amdgcn_readfirstlane(exponent_of(n.vs)) : 0;
            };
            scales(s0);

            // one step; the last one looks at none behind it
            auto take = [&](int turn, auto last) {
                const int buffer = (turn - from) / GROUPS & 1, step = turn + side;
                __syncthreads();  // keys of the next step and values of this one are there, and nobody reads what is written below
                Step s2 = s1;
                if constexpr (!last.value) {
                    s2 = step_at(step + 2 * GROUPS, page2);
                    page2 = page_of(step + 3 * GROUPS);
                    fetch_keys(s2, kc);
                    fetch_values(s1);
                }

                top = fmaf(top, c, (float)ev);
                if (__any(top > m + kHighest)) {
                    const float to = moved(fmaxf(top, __shfl_xor(top, 32)), m);
                    const float f = exp2f(m - to);
                    m = to;
                    l *= f;
#pragma unroll
                    for (int n = 0; n < DN; ++n) o[n] *= f;
                }
                const float base = m - (float)ev;
                now[0] = ahead[0], now[1] = ahead[1];

                float sum[4] = {};
                half8 p[4];
                auto weigh = [&](int t) {
                    float w[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        w[r] = __builtin_amdgcn_exp2f(fmaf(now[t >> 1][8 * (t & 1) + r], c, -base));
                        sum[r & 3] += w[r];
                    }
                    p[t] = half8{(_Float16)w[0], (_Float16)w[1], (_Float16)w[2], (_Float16)w[3], (_Float16)w[4], (_Float16)w[5], (_Float16)w[6], (_Float16)w[7]};
                };
                auto gather = [&](int n, int t) {
                    const half8 f = *(const half8 *)&tiles[side][buffer].values[padded<8>(32 * n + q32, 4 * (t >> 1) + 2 * h2 + (t & 1))];
                    o[n] = Mma<_Float16>::mma(f, p[t], o[n]);
                };
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    if constexpr (!last.value) {
                        score(buffer ^ 1, 0, kk);
                        score(buffer ^ 1, 1, kk);
                    }
                    if (kk % (KK / 4) == 0) weigh(kk / (KK / 4));
                }
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int n = 0; n < DN; ++n) gather(n, t);
                l = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), pow2(-ev), l);  // the sum of weights alone knows no value's scale
                if constexpr (!last.value) {
                    hide(s1);
                    top = largest();
                    stage_keys(kc, buffer);
                    stage_values(s1, buffer ^ 1);
                    s0 = s1, s1 = s2;
                    scales(s0);
                }
            };
            int turn = from;
            for (; turn + GROUPS < to; turn += GROUPS) take(turn, std::false_type{});
            take(turn, std::true_type{});
        }

        // o[n][r]: query q32, channel 32 n + 8 (r / 4) + 4 h2 + r % 4
        float4v x[DN][4];
        l += __shfl_xor(l, 32);
#pragma unroll
        for (int n = 0; n < DN; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) x[n][r] = float4v{o[n][4 * r], o[n][4 * r + 1], o[n][4 * r + 2], o[n][4 * r + 3]};
        if constexpr (GROUPS == 2) {
            constexpr int kSums = DN * 4 * NT;
            static_assert(sizeof(tiles) >= kSums * sizeof(float4v) + NT * sizeof(float2), "the sums go where keys and values were");
            float4v *const sums = (float4v *)&tiles[0][0];
            float2 *const ml = (float2 *)(sums + kSums);
            __syncthreads();
            if (side) {
                ml[tid] = make_float2(m, l);
#pragma unroll
                for (int n = 0; n < DN; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sums[(n * 4 + r) * NT + tid] = x[n][r];
            }
            __syncthreads();
            if (!side) {
                const float2 other = ml[tid];
                top = fmaxf(m, other.x);
                const float f = exp2f(m - top), g = exp2f(other.x - top);
                m = top;
                l = l * f + other.y * g;
#pragma unroll
                for (int n = 0; n < DN; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[n][r] = x[n][r] * f + sums[(n * 4 + r) * NT + tid] * g;
            }
        }
        if (has && !side) {
            int64_t part = part0 + wave * R + q32;
            if (part0 < 0) {
                const int64_t first_row = ((int64_t)(blockIdx.x % a.splits) * a.seq.batch + b) * a.seq.max_new;
                part = a.splits > 1 ? (first_row + token) * a.heads + head * group + row - token * group : -1;
            }
#pragma unroll
            for (int n = 0; n < DN; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) give<T, D>(a, s, head, group, part, row, 32 * n + 8 * r + 4 * h2, x[n][r], m, l, n == 0 && r == 0 && h2 == 0);
        }

        if (!SHARES || (left -= take) <= 0) return;
        off = 0;
        if (++tile_of_rows * kRows >= total) {
            tile_of_rows = 0;
            if (++head == H) {
                head = 0;
                do {
                    if (++b >= a.seq.batch) return;  // only if the lengths change meanwhile
                    s = sequence_of_all(a.seq, b);
                } while (min(s.n, a.seq.max_new) <= 0);
            }
        }
        __syncthreads();  // before the next tile's keys and values
    }
}

// The parts of rows that workgroups shared: who begins first inside a tile of rows joins what belongs to it.  D / 4 threads have
// a row, four channels each.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cache_attention_join_shares(CacheAttentionArgs a)
{
    constexpr int C = D / 4, kSide = 256 / C, kSplit = kTileRows / kSide;
    const int share = blockIdx.x / kSplit + 1, at = blockIdx.x % kSplit * kSide + threadIdx.x / C, c = threadIdx.x % C;
    const int4 *const begins = begins_of(a);
    const int4 mine = begins[share], before = begins[share - 1];
    auto inside = [&](int4 x) { return x.x == mine.x && x.y == mine.y && x.z == mine.z && x.w != 0; };
    if (mine.x < 0 || mine.w == 0 || inside(before)) return;
    const Seq s = sequence(a.seq, mine.x);
    const int group = a.heads / a.cache.heads, row = mine.z * kTileRows + at;
    if (row >= min(s.n, a.seq.max_new) * group) return;
    const float2 *const ml = (const float2 *)(a.partial + a.part_rows * D);
    float4v x = {};
    float top = kNothing, sum = 0.0f;
    for (int k = share - 1;;) {
        const int64_t part = (2 * (int64_t)k + (k < share)) * kTileRows + at;
        const float2 p = ml[part];
        const float4v y = *(const float4v *)(a.partial + part * D + 4 * c);
        const float up = fmaxf(top, p.x);
        const float f = exp2f(top - up), g = exp2f(p.x - up);
        top = up;
        sum = sum * f + p.y * g;
        x = x * f + y * g;
        if (++k >> a.share_log2 || !inside(begins[k])) break;
    }
    give<T, D>(a, s, mine.y, group, -1, row, 4 * c, x, top, sum, c == 0);
}

// The parts of a row: D / 4 threads have four channels each, ALONE of them a row for themselves (few parts, many rows), or
// all of a workgroup's threads one row, each D / 4 some of its parts.
constexpr int kFewSplits = 8, kMostParts = 1024;
// A small kernel: what it takes is the latency of its loads, so all that can leave at once do (one token over 2048 keys in eight
// parts 11.2 -> 9.8 us with both launches).
template <typename T, int D, bool ALONE>
__global__ __launch_bounds__(256) void k_cache_attention_join(CacheAttentionArgs a)
{
    constexpr int C = D / 4, kSide = 256 / C;
    __shared__ float weight[ALONE ? 1 : kMostParts], some[2][4];
    __shared__ float4v side[ALONE ? 1 : kSide][C];
    const int tid = threadIdx.x, c = tid % C, nth = tid / C;
    const unsigned item = ALONE ? blockIdx.x * kSide + nth : blockIdx.x, bt = item / a.heads;
    const int h = item % a.heads, b = bt / a.seq.max_new, t = bt % a.seq.max_new;
    if (ALONE && b >= a.seq.batch) return;
    const bool shared = !ALONE && a.share_log2 >= 0;
    int units = 0, units_before = 0, units_all = 0;
    if (shared) {
        const int *const shares = shares_of(a);
        units_before = shares[b], units = shares[b + 1] - units_before, units_all = shares[a.seq.batch];
    }
    const Seq s = sequence(a.seq, b);
    // The row's parts: the first, and from the second on every `stride`-th.  (Unless work was shared the lengths say nothing about
    // them, so they are asked for together with those.)
    const int H = a.cache.heads, group = a.heads / H, r = t * group + h % group;
    int64_t first = item, stride = (int64_t)a.seq.batch * a.seq.max_new * a.heads;
    if (a.share_rows <= 32) first = ((int64_t)(b * H + h / group) * a.splits) * a.share_rows + r, stride = a.share_rows;
    int64_t second = first + stride;
    int parts = a.splits;
    if (shared) {
        if (t >= s.n) return;
        const int u = units_before * H + h / group * units, total = units_all * H, log2 = shares_log2(a, total);
        auto owner = [&](int x) {  // the workgroup whose share holds step x; the quotient is at most one off
            int w = (int)(((double)x + 0.5) * (double)(1 << log2) / (double)total);
            if (share_begin(w, total, log2) > x) --w;
            if (share_begin(w + 1, total, log2) <= x) ++w;
            return w;
        };
        const int w0 = owner(u), w1 = owner(u + units - 1);
        if (w0 == w1) return;  // has been written whole
        parts = w1 - w0 + 1;
        first = (int64_t)(2 * w0 + 1) * a.share_rows + r;
        second = (int64_t)(2 * w0 + 2) * a.share_rows + r, stride = 2 * a.share_rows;
    }
    auto at = [&](int k) { return k == 0 ? first : second + (k - 1) * stride; };
    const float2 *const ml = (const float2 *)(a.partial + a.part_rows * D);
    const float *const o = a.partial + 4 * c;
    float4v x = {};
    float top = kNothing, sum = 0.0f;
    auto factor = [&](float2 p) { return exp2f(p.x - top); };
    if constexpr (ALONE) {
        float2 p[kFewSplits];
        float4v y[kFewSplits];
#pragma unroll
        for (int k = 0; k < kFewSplits; ++k) {
            const int64_t part = at(min(k, parts - 1));
            p[k] = ml[part];
            y[k] = *(const float4v *)(o + part * D);
        }
        if (t >= s.n) return;
#pragma unroll
        for (int k = 0; k < kFewSplits; ++k) {
            if (k >= parts) p[k] = make_float2(kNothing, 0.0f), y[k] = float4v{};
            top = fmaxf(top, p[k].x);
        }
#pragma unroll
        for (int k = 0; k < kFewSplits; ++k) {
            const float f = factor(p[k]);
            sum = fmaf(f, p[k].y, sum);
            x += y[k] * f;
        }
    } else {
        constexpr int kEarly = 8;  // of a thread's parts, asked for before anything is known about them
        float2 p[kMostParts / 256];
        float4v early[kEarly];
#pragma unroll
        for (int j = 0; j < kMostParts / 256; ++j) p[j] = tid + 256 * j < parts ? ml[at(tid + 256 * j)] : make_float2(kNothing, 0.0f);
#pragma unroll
        for (int j = 0; j < kEarly; ++j) early[j] = nth + j * kSide < parts ? *(const float4v *)(o + at(nth + j * kSide) * D) : float4v{};
        if (t >= s.n) return;
#pragma unroll
        for (int j = 0; j < kMostParts / 256; ++j) top = fmaxf(top, p[j].x);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        if ((tid & 63) == 0) some[0][tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(some[0][0], some[0][1]), fmaxf(some[0][2], some[0][3]));
#pragma unroll
        for (int j = 0; j < kMostParts / 256; ++j) {
            const float f = factor(p[j]);
            weight[tid + 256 * j] = f;
            sum = fmaf(f, p[j].y, sum);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        if ((tid & 63) == 0) some[1][tid >> 6] = sum;
        __syncthreads();
        sum = (some[1][0] + some[1][1]) + (some[1][2] + some[1][3]);
#pragma unroll
        for (int j = 0; j < kEarly; ++j)
            if (nth + j * kSide < parts) x += early[j] * weight[nth + j * kSide];
#pragma unroll 4
        for (int k = nth + kEarly * kSide; k < parts; k += kSide) x += *(const float4v *)(o + at(k) * D) * weight[k];
        side[nth][c] = x;
        __syncthreads();
        if (nth) return;
#pragma unroll
        for (int k = 1; k < kSide; ++k) x += side[k][c];
    }
    const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int64_t token = s.row + t;
    *(uint2 *)((T *)a.out + token * a.ldo + (int64_t)h * D + 4 * c) = result<T>(x, f);
    if (c == 0 && a.lse) a.lse[token * a.heads + h] = log_of(top, sum);
}

constexpr int kAttWaves = 4;

template <typename T, int D>
void launch(const CacheAttentionArgs &a, const AttentionPlan &plan, hipStream_t st)
{
    constexpr int NB = D < 256 ? 2 : 1, kTwice = D < 256 ? 2 * kAttWaves : kAttWaves;
    const dim3 grid((unsigned)plan.groups), block(kAttWaves * 64);
    if (plan.rows > 32) {
        // Two workgroups' worth of wavefronts on the same rows halve the way of the rows that see most.  That gains where a round
        // holds all (a compute unit has one such workgroup at a time, or two of the others), and in whole prompts, whose ends
        // see most and are few.  us, one / two, heads of 64 and of 128: 256 tiles of 2048 keys 37 / 33 and 54 / 52, 320 of them
        // 50 / 58 and 73 / 91; a prompt of 2048, 24 heads 36 / 30 and 52 / 45, 32 heads 37 / 36 and 56 / 55; of 1536, 40
        // heads 29 / 30 and 44 / 46; of 1024, 64 heads 22 / 25 and 34 / 38; 2048 with a window of 1024, 32 heads 30 / 36 and 46 / 56;
        // 2048 rows behind 2048 keys, 32 heads 83 / 82 and 127 / 130; 384 tiles of 328 keys of 64 15.6 / 20.9.
        constexpr int kMost = D <= 128 ? 2 : 1;
        if constexpr (D <= 128) {
            if (a.share_log2 >= 0) {
                hipLaunchKernelGGL((k_cache_attention_rows<T, D, 1, true>), grid, block, 0, st, a, plan.row_tiles);
                hipLaunchKernelGGL((k_cache_attention_join_shares<T, D>), dim3((((unsigned)1 << a.share_log2) - 1) * (kTileRows * D / 1024)), block, 0, st, a);
                return;
            }
        }
        const bool prompt = a.causal && !a.window && plan.reach < 2 * (int64_t)a.seq.max_new;
        if (kMost == 2 && plan.reach >= 1024 && (plan.groups <= 256 || (prompt && plan.groups <= 512 && plan.reach >= 4 * plan.groups)))
            hipLaunchKernelGGL((k_cache_attention_rows<T, D, kMost, false>), grid, dim3(kMost * 256), 0, st, a, plan.row_tiles);
        else
            hipLaunchKernelGGL((k_cache_attention_rows<T, D, 1, false>), grid, block, 0, st, a, plan.row_tiles);
    } else if (plan.rows == 16) {
        if (plan.waves == kAttWaves) hipLaunchKernelGGL((k_cache_attention<T, D, 1, kAttWaves>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_cache_attention<T, D, 1, kTwice>), grid, dim3(kTwice * 64), 0, st, a);
    } else {
        if (plan.waves == kAttWaves) hipLaunchKernelGGL((k_cache_attention<T, D, NB, kAttWaves>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_cache_attention<T, D, NB, kTwice>), grid, dim3(kTwice * 64), 0, st, a);
    }
    if (plan.workspace) {
        const int64_t rows = (int64_t)a.seq.batch * a.seq.max_new * a.heads, alone = 256 / (D / 4);
        if (a.splits > 1 && a.splits <= kFewSplits)
            hipLaunchKernelGGL((k_cache_attention_join<T, D, true>), dim3((unsigned)((rows + alone - 1) / alone)), block, 0, st, a);
        else
            hipLaunchKernelGGL((k_cache_attention_join<T, D, false>), dim3((unsigned)rows), block, 0, st, a);
    }
}

template <typename T>
void launch_type(const CacheAttentionArgs &a, const AttentionPlan &plan, hipStream_t st)
{
    if (a.cache.dim == 64) launch<T, 64>(a, plan, st);
    else if (a.cache.dim == 128) launch<T, 128>(a, plan, st);
    else launch<T, 256>(a, plan, st);
}

}  // namespace

AttentionPlan cache_attention_plan(int heads, int kv_heads, int dim, int batch, int max_new, int reach)
{
    AttentionPlan p{};
    const int64_t rows = (int64_t)max_new * (heads / kv_heads), steps = ((int64_t)reach + kCacheTile - 1) / kCacheTile;
    const double parts = (double)batch * kv_heads;  // sequences times key heads
    // rows of a workgroup: up to 16 or 32 that its four wavefronts share, else 32 for each of four (or of twice four)
    p.rows = rows <= 16 ? 16 : rows <= 32 && dim < 256 ? 32 : 128;
    p.row_tiles = (int)((rows + p.rows - 1) / p.rows);
    p.groups = (double)p.row_tiles * parts;
    p.splits = 1, p.share_log2 = -1, p.waves = kAttWaves, p.reach = reach;
    if (p.rows <= 32) {
        // Two workgroups for every compute unit, as long as each of their wavefronts still has a step: every sequence is split
        // into as many parts, and a long one's take longer, which is little where they are short (us, a token over 131072 keys
        // 49.5, in equal shares of all steps 51.8; 32 sequences of up to 3000 keys in a whole decode step 41 and 46) ...
        const double all = parts * (double)steps;
        const int64_t want = parts >= 512 ? 1 : (int64_t)((512 + parts - 1) / parts), most_splits = steps / kAttWaves;
        const int64_t splits = want < most_splits ? want : most_splits > 1 ? most_splits : 1;
        if (steps <= 8 * kAttWaves * splits || all >= (double)(1u << 31)) {
            if (splits == 2 && dim < 256) {
                // twice the wavefronts, which join in LDS (32 sequences of 2048 keys, 8 heads of 128: 24.5 us, two parts 27.6;
                // 512 keys, one sequence: 7.4 and 8.8); heads of 256 have no registers for that
                p.waves = 2 * kAttWaves;
            } else if (splits > 1) {
                p.splits = (int)splits;
                p.groups *= (double)splits;
                p.part_rows = (int64_t)p.groups * p.rows;
                p.workspace = (size_t)p.part_rows * (dim + 2) * sizeof(float);
            }
            return p;
        }
        // ... and else everybody gets as many steps (64 sequences of up to 8192 keys 127 and 122): two workgroups for every
        // compute unit, four where sequences and heads are that many.
        const double full = parts >= 1024 ? kMostParts : 512, most = all / 4 < full ? all / 4 : full;
        while ((double)(1 << (p.share_log2 + 1)) <= most) ++p.share_log2;
        p.groups = 1 << p.share_log2;
        p.part_rows = (int64_t)2 * p.rows << p.share_log2;
        p.workspace = (size_t)p.part_rows * (dim + 2) * sizeof(float) + ((size_t)batch + 1) * sizeof(int);
        return p;
    }
    // Few rounds of workgroups, each with many steps: the last round is often half empty, and sequences differ.  Two workgroups
    // for every compute unit share all steps instead, unless rounds come out even or rows are so many that their ends differ
    // (a prompt's: tiles are taken longest first then, and those that run at a time read the same keys, which shares do not).
    // us, tiles / shares, 32 heads on 8 of 128: 1200 rows and 4096 keys 106 / 102; 512 and 8192, three times, 250 / 242 (heads of 64
    // 170 / 153); up to 1024 and 5163 to 16024, four times, 652 / 548.  Against that 512 and 32768 keys four times 1119 / 1168,
    // 512 and 2048 four times 74 / 96, a prompt of 8192 569 / 647, 2048 and 32768 four times 4314 / 4890; heads of 256 lose registers.
    const double all = p.groups * (double)steps, rounds = p.groups / 256, fill = rounds / (double)(int64_t)(rounds + 255.0 / 256);
    const bool few_rounds = p.groups > 256 && p.groups <= kMostShared, uneven = batch > 1 || fill < 0.85;
    if (dim < 256 && steps >= 64 && few_rounds && uneven && (int64_t)max_new * 2 <= reach && all < (double)(1u << 31)) {
        p.share_log2 = 9;
        p.groups = 1 << p.share_log2;
        p.part_rows = (int64_t)2 * kTileRows << p.share_log2;
        p.workspace = (size_t)p.part_rows * (dim + 2) * sizeof(float) + (sizeof(int4) << p.share_log2);
        return p;
    }
    // Parts of many rows are large: one round of workgroups at most, and four steps each at least.  (us, 100 rows and 2000 keys of
    // 8 heads 15.9, with 16 steps 27.1; 33 rows of 8 heads on 2, 32768 keys 24.8 and 29.4; 88 rows of 36 heads and sequences, 6200
    // keys, six parts each 29, eight, which are more than a round, 47.)
    const int64_t want = (int64_t)(256 / p.groups), most = steps / 4, s = want < most ? want : most;
    if (s <= 1) return p;
    p.splits = (int)s;
    p.groups *= p.splits;
    p.part_rows = (int64_t)p.splits * batch * max_new * heads;
    p.workspace = (size_t)p.part_rows * (dim + 2) * sizeof(float);
    return p;
}

hipError_t launch_cache_attention(CacheAttentionArgs a, const AttentionPlan &plan, hipStream_t st)
{
    a.splits = plan.splits, a.share_log2 = plan.share_log2, a.share_rows = plan.rows, a.part_rows = plan.part_rows;
    if (a.bf16)
        launch_type<__bf16>(a, plan, st);
    else
        launch_type<_Float16>(a, plan, st);
    return hipGetLastError();
}

}  // namespace bwta
