// Keys and values into the 8-bit cache, and back out of it.
//
// A block of `block` tokens has one scale 2^e per head and side, e the smallest with max |x| <= 448 * 2^e: dividing by it
// is exact, so a code is the one rounding of x to E4M3.  Keys lie [token][dim], values [dim][token]: what a matrix core
// operand of each takes from memory is then 16 bytes in a row.
#include "bwta_heads.h"

namespace bwta {
namespace {

constexpr int kThreads = 256;
constexpr int kFew = 4;  // up to so many tokens of a block, values are stored byte by byte

struct Place {
    int head, page, slot, count, value;  // tokens [slot, slot + count) of the block, dense rows from `row`
    int64_t row;
};

// The part of a call that this workgroup has: one block, one head, keys or values.  False: nothing.
__device__ __forceinline__ bool place_of(const CacheRowsArgs &a, int per_sequence, Place &p, bool &page_ok)
{
    unsigned i = blockIdx.x;
    p.value = i & 1;
    i >>= 1;
    p.head = i % a.cache.heads;
    i /= a.cache.heads;
    const int nth = i % per_sequence, b = i / per_sequence;
    const Seq s = sequence(a.seq, b);
    const int begin = max(s.start, 0), ordinal = begin / a.cache.block + nth;
    const int64_t from = (int64_t)ordinal * a.cache.block;
    if (from >= s.len || s.n <= 0) return false;  // from here on everything is below max_len
    const int t0 = max(begin, (int)from), t1 = (int)min((int64_t)s.len, from + a.cache.block);
    if (t0 >= t1) return false;
    p.page = a.seq.table[b * a.seq.ldt + ordinal];
    page_ok = p.page >= 0 && p.page < a.cache.blocks;
    p.slot = t0 - ordinal * a.cache.block, p.count = t1 - t0;
    p.row = s.row + (t0 - s.start);
    return true;
}

__device__ __forceinline__ uint32_t scaled_codes(uint32_t codes, float f)
{
    typedef float float2v __attribute__((ext_vector_type(2)));
    const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo.x * f, lo.y * f, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi.x * f, hi.y * f, r, true);
}

// bytes [lo, hi) of a run of 16 from `fresh`, the others from `old`
__device__ __forceinline__ uint4 blend(uint4 old, uint4 fresh, int lo, int hi)
{
    uint4 r;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m |= 4 * w + j >= lo && 4 * w + j < hi ? 0xffu << (8 * j) : 0u;
        (&r.x)[w] = ((&fresh.x)[w] & m) | ((&old.x)[w] & ~m);
    }
    return r;
}

// One workgroup owns a block's codes of one head and side: it finds the scale, divides what is there where the scale grew,
// and writes the new codes.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void k_cache_write(CacheRowsArgs a, int per_sequence)
{
    __shared__ uint32_t tile[NT == 64 ? 1 : kCacheTile * 64];  // codes of 64 tokens, [token][dim / 4]
    __shared__ uint32_t top_of[NT / 64];
    Place p;
    bool page_ok;
    if (!place_of(a, per_sequence, p, page_ok) || !page_ok) return;
    const int D = a.cache.dim, block = a.cache.block, tid = threadIdx.x;
    const int chunks = D / 8, work = p.count * chunks;
    const T *x = (const T *)(p.value ? a.v : a.k) + p.row * (p.value ? a.ldv : a.ldk) + (int64_t)p.head * D;
    const int64_t ldx = p.value ? a.ldv : a.ldk;
    const int64_t unit = (int64_t)p.page * a.cache.heads + p.head;
    uint8_t *codes = (p.value ? a.cache.v : a.cache.k) + unit * block * D;
    float *scale = (p.value ? a.cache.v_scale : a.cache.k_scale) + unit;

    uint32_t top = 0;  // magnitude bits of a finite 16-bit value order as the values do
    for (int i = tid; i < work; i += NT) {
        const uint4 in = *(const uint4 *)(x + (int64_t)(i / chunks) * ldx + i % chunks * 8);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t lo = (&in.x)[w] & 0x7fff, hi = ((&in.x)[w] >> 16) & 0x7fff;
            top = max(top, max(lo < Half<T>::kInf ? lo : 0u, hi < Half<T>::kInf ? hi : 0u));
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if (NT > 64) {
        if ((tid & 63) == 0) top_of[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) top = max(top, top_of[w]);
    }
    int e = scale_exponent(Half<T>::to_float(top));
    if (p.slot > 0) {
        const int before = exponent_of(*scale);
        if (e > before) {
            const float f = pow2(before - e);
            for (int i = tid; i < block * D / 16; i += NT) {  // the whole block: what lies behind the tokens stays in step with its scale
                uint4 *c = (uint4 *)codes + i;
                const uint4 old = *c;
                *c = make_uint4(scaled_codes(old.x, f), scaled_codes(old.y, f), scaled_codes(old.z, f), scaled_codes(old.w, f));
            }
        } else {
            e = before;
        }
    }
    __syncthreads();  // everybody has read the scale, and what was there is written before the tokens beside it are
    if (tid == 0) *scale = pow2(e);
    const float inverse = pow2(-e);

    auto codes_of = [&](int token, int chunk) {
        const uint4 in = *(const uint4 *)(x + (int64_t)token * ldx + chunk * 8);
        uint2 r;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const uint32_t u = (&in.x)[2 * w], v = (&in.x)[2 * w + 1];
            (&r.x)[w] = to_codes(Half<T>::to_float(u & 0xffff) * inverse, Half<T>::to_float(u >> 16) * inverse,
                                 Half<T>::to_float(v & 0xffff) * inverse, Half<T>::to_float(v >> 16) * inverse);
        }
        return r;
    };
    if (!p.value) {
        for (int i = tid; i < work; i += NT) *(uint2 *)(codes + (int64_t)(p.slot + i / chunks) * D + i % chunks * 8) = codes_of(i / chunks, i % chunks);
        return;
    }
    if (NT == 64 || p.count <= kFew) {
        for (int i = tid; i < work; i += NT) {
            const uint2 r = codes_of(i / chunks, i % chunks);
            uint8_t *c = codes + (int64_t)(i % chunks * 8) * block + p.slot + i / chunks;
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j * block] = (uint8_t)((j < 4 ? r.x : r.y) >> (8 * (j & 3)));
        }
        return;
    }
    // Through LDS: four rows of 16 tokens per thread, turned by bytes.
    for (int base = p.slot / kCacheTile * kCacheTile; base < p.slot + p.count; base += kCacheTile) {
        const int lo = max(p.slot, base), hi = min(p.slot + p.count, base + kCacheTile);
        __syncthreads();
        for (int i = tid; i < (hi - lo) * chunks; i += NT) {
            const int token = lo + i / chunks;
            *(uint2 *)&tile[(token - base) * (D / 4) + i % chunks * 2] = codes_of(token - p.slot, i % chunks);
        }
        __syncthreads();
        for (int i = tid; i < D / 4 * 4; i += NT) {  // (quarter of the tile, four rows)
            const int q = i & 3, d4 = i >> 2, first = base + 16 * q;
            if (first + 16 <= lo || first >= hi) continue;
            uint4 rows[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t r[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = tile[(16 * q + 4 * w + j) * (D / 4) + d4];
                transpose_bytes(r);
#pragma unroll
                for (int j = 0; j < 4; ++j) (&rows[j].x)[w] = r[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint4 *c = (uint4 *)(codes + (int64_t)(4 * d4 + j) * block + first);
                *c = first >= lo && first + 16 <= hi ? rows[j] : blend(*c, rows[j], lo - first, hi - first);
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ uint4 values_of(uint2 codes, float s)
{
    typedef float float2v __attribute__((ext_vector_type(2)));
    uint4 r;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const uint32_t c = w ? codes.y : codes.x;
        const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
        auto fit = [&](float x) { return x != x ? x : fminf(fmaxf(x * s, -Half<T>::kMax), Half<T>::kMax); };  // 256 * 256 is beyond fp16
        (&r.x)[2 * w] = Half<T>::pack(fit(lo.x), fit(lo.y));
        (&r.x)[2 * w + 1] = Half<T>::pack(fit(hi.x), fit(hi.y));
    }
    return r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_cache_read(CacheRowsArgs a, int per_sequence)
{
    __shared__ uint32_t tile[kCacheTile * 64];
    Place p;
    bool page_ok;
    if (!place_of(a, per_sequence, p, page_ok)) return;
    const int D = a.cache.dim, block = a.cache.block, tid = threadIdx.x, chunks = D / 8;
    const int64_t ldx = p.value ? a.ldv : a.ldk;
    T *x = (T *)(p.value ? a.v : a.k) + p.row * ldx + (int64_t)p.head * D;
    if (!page_ok) {
        for (int i = tid; i < p.count * chunks; i += kThreads) *(uint4 *)(x + (int64_t)(i / chunks) * ldx + i % chunks * 8) = make_uint4(0, 0, 0, 0);
        return;
    }
    const int64_t unit = (int64_t)p.page * a.cache.heads + p.head;
    const uint8_t *codes = (p.value ? a.cache.v : a.cache.k) + unit * block * D;
    const float s = (p.value ? a.cache.v_scale : a.cache.k_scale)[unit];
    if (!p.value) {
        for (int i = tid; i < p.count * chunks; i += kThreads)
            *(uint4 *)(x + (int64_t)(i / chunks) * ldx + i % chunks * 8) = values_of<T>(*(const uint2 *)(codes + (int64_t)(p.slot + i / chunks) * D + i % chunks * 8), s);
        return;
    }
    for (int base = p.slot / kCacheTile * kCacheTile; base < p.slot + p.count; base += kCacheTile) {
        const int lo = max(p.slot, base), hi = min(p.slot + p.count, base + kCacheTile);
        __syncthreads();
        for (int i = tid; i < D / 4 * 4; i += kThreads) {
            const int q = i & 3, d4 = i >> 2, first = base + 16 * q;
            if (first + 16 <= lo || first >= hi) continue;
            uint4 rows[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) rows[j] = *(const uint4 *)(codes + (int64_t)(4 * d4 + j) * block + first);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t r[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = (&rows[j].x)[w];
                transpose_bytes(r);
#pragma unroll
                for (int j = 0; j < 4; ++j) tile[(16 * q + 4 * w + j) * (D / 4) + d4] = r[j];
            }
        }
        __syncthreads();
        for (int i = tid; i < (hi - lo) * chunks; i += kThreads) {
            const int token = lo + i / chunks;
            *(uint4 *)(x + (int64_t)(token - p.slot) * ldx + i % chunks * 8) = values_of<T>(*(const uint2 *)&tile[(token - base) * (D / 4) + i % chunks * 2], s);
        }
    }
}

}  // namespace

hipError_t launch_cache_write(const CacheRowsArgs &a, hipStream_t st)
{
    const int per = (int)cache_blocks_reached(a.cache, a.seq);
    const unsigned groups = (unsigned)cache_rows_groups(a.cache, a.seq);
    auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(threads), 0, st, a, per); };
    if (a.seq.max_new == 1) {  // a wavefront does for one token
        if (a.bf16) go(k_cache_write<__bf16, 64>, 64);
        else go(k_cache_write<_Float16, 64>, 64);
    } else {
        if (a.bf16) go(k_cache_write<__bf16, kThreads>, kThreads);
        else go(k_cache_write<_Float16, kThreads>, kThreads);
    }
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheRowsArgs &a, hipStream_t st)
{
    const int per = (int)cache_blocks_reached(a.cache, a.seq);
    const unsigned groups = (unsigned)cache_rows_groups(a.cache, a.seq);
    if (a.bf16)
        hipLaunchKernelGGL(k_cache_read<__bf16>, dim3(groups), dim3(kThreads), 0, st, a, per);
    else
        hipLaunchKernelGGL(k_cache_read<_Float16>, dim3(groups), dim3(kThreads), 0, st, a, per);
    return hipGetLastError();
}

}  // namespace bwta
