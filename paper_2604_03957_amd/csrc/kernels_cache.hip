// Keys and values into the 8-bit cache, and back out of it.
//
// A block of `block` tokens has one scale 2^e per head and side, e the smallest with max |x| <= 448 * 2^e: dividing by it
// is exact, so a code is the one rounding of x to E4M3, and dividing codes by a power of two later, where the scale has to
// grow, rounds nothing but what becomes subnormal.  Keys lie [token][dim], values [dim][token]: what a matrix core operand of
// each takes from memory is then 16 bytes in a row.
//
// Bound by memory: a block's tokens are read once and its codes written once.  Prompts of 2019 to 4001 tokens of 8 heads of
// 128 in and back out (207 MB) take 41 us, 5.0 TB/s; whole contexts back to bf16 (236 MB) 39 to 51 us from one run and machine to
// another, 4.6 to 6.0 TB/s, where a copy reaches 4.9; a decode step's 64 tokens 4.8 us, the latency of table, tokens and scale one after the other.
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
    const int begin = max(s.start, 0), end = min(s.len, s.start + min(s.n, a.seq.max_new)), ordinal = begin / a.cache.block + nth;
    const int64_t from = (int64_t)ordinal * a.cache.block;
    if (from >= end || s.n <= 0) return false;  // from here on everything is below max_len
    const int t0 = max(begin, (int)from), t1 = (int)min((int64_t)end, from + a.cache.block);
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
// and writes the new codes.  The tokens stay in registers between the two, J times eight values of one token a thread: all of
// a block's slots, or (NT = 64, J = 1) one token.
template <typename T, int D, int NT, int J>
__global__ __launch_bounds__(NT) void k_cache_write(CacheRowsArgs a, int per_sequence)
{
    constexpr int C = D / 8;
    __shared__ uint32_t tile[NT == 64 ? 1 : kCacheTile * (D / 4)];  // codes of 64 tokens, [token][D / 4]
    __shared__ uint32_t top_of[NT / 64];
    Place p;
    bool page_ok;
    if (!place_of(a, per_sequence, p, page_ok) || !page_ok) return;
    const int block = a.cache.block, tid = threadIdx.x;
    const int64_t ldx = p.value ? a.ldv : a.ldk;
    const T *x = (const T *)(p.value ? a.v : a.k) + p.row * ldx + (int64_t)p.head * D;
    const int64_t unit = (int64_t)p.page * a.cache.heads + p.head;
    uint8_t *codes = (p.value ? a.cache.v : a.cache.k) + unit * block * D;
    float *scale = (p.value ? a.cache.v_scale : a.cache.k_scale) + unit;

    // the j-th eight values of a thread: chunk `c` of slot `slot`
    const int c = tid % C;
    auto slot_of = [&](int j) { return NT == 64 ? (tid < C ? p.slot : -1) : (tid + j * NT) / C; };
    auto is_new = [&](int slot) { return slot >= p.slot && slot < p.slot + p.count; };
    const float before = p.slot > 0 ? *scale : 0.0f;
    uint4 in[J];
    uint32_t top = 0;  // magnitude bits of a finite 16-bit value order as the values do
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int slot = slot_of(j);
        in[j] = is_new(slot) ? load_once(x + (int64_t)(slot - p.slot) * ldx + c * 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t lo = (&in[j].x)[w] & 0x7fff, hi = ((&in[j].x)[w] >> 16) & 0x7fff;
            top = max(top, max(lo < Half<T>::kInf ? lo : 0u, hi < Half<T>::kInf ? hi : 0u));
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
        const int was = exponent_of(before);
        if (e > was) {
            const float f = pow2(was - e);
            for (int i = tid; i < block * D / 16; i += NT) {  // the whole block: what lies behind the tokens stays in step with its scale
                uint4 *old = (uint4 *)codes + i;
                const uint4 o = *old;
                *old = make_uint4(scaled_codes(o.x, f), scaled_codes(o.y, f), scaled_codes(o.z, f), scaled_codes(o.w, f));
            }
        } else {
            e = was;
        }
    }
    __syncthreads();  // everybody has read the scale, and what was there is written before the tokens beside it are
    if (tid == 0) *scale = pow2(e);
    const float inverse = pow2(-e);

    auto codes_of = [&](const uint4 &v) {
        uint2 r;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const uint32_t lo = (&v.x)[2 * w], hi = (&v.x)[2 * w + 1];
            (&r.x)[w] = to_codes(Half<T>::to_float(lo & 0xffff) * inverse, Half<T>::to_float(lo >> 16) * inverse,
                                 Half<T>::to_float(hi & 0xffff) * inverse, Half<T>::to_float(hi >> 16) * inverse);
        }
        return r;
    };
    if (!p.value) {
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (is_new(slot_of(j))) *(uint2 *)(codes + slot_of(j) * D + c * 8) = codes_of(in[j]);
        return;
    }
    if (NT == 64 || p.count <= kFew) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (!is_new(slot_of(j))) continue;
            const uint2 r = codes_of(in[j]);
            uint8_t *to = codes + c * 8 * block + slot_of(j);
#pragma unroll
            for (int k = 0; k < 8; ++k) to[k * block] = (uint8_t)((k < 4 ? r.x : r.y) >> (8 * (k & 3)));
        }
        return;
    }
    // Through LDS, 64 slots at a time: four rows of 16 tokens per thread, turned by bytes.
    constexpr int kEach = kCacheTile * C / NT > 0 ? kCacheTile * C / NT : 1;  // a thread's chunks of 64 slots
#pragma unroll
    for (int t = 0; t < J / kEach; ++t) {
        const int base = t * kCacheTile, lo = max(p.slot, base), hi = min(p.slot + p.count, base + kCacheTile);
        if (lo >= hi) continue;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int slot = slot_of(t * kEach + k);
            *(uint2 *)&tile[(slot - base) * (D / 4) + c * 2] = codes_of(in[t * kEach + k]);
        }
        __syncthreads();
        for (int i = tid; i < D; i += NT) {  // (quarter of the tile, four rows)
            const int q = i & 3, d4 = i >> 2, first = base + 16 * q;
            if (first + 16 <= lo || first >= hi) continue;
            uint4 rows[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t r[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) r[k] = tile[(16 * q + 4 * w + k) * (D / 4) + d4];
                transpose_bytes(r);
#pragma unroll
                for (int k = 0; k < 4; ++k) (&rows[k].x)[w] = r[k];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint4 *to = (uint4 *)(codes + (4 * d4 + k) * block + first);
                *to = first >= lo && first + 16 <= hi ? rows[k] : blend(*to, rows[k], lo - first, hi - first);
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
            store_once(x + (int64_t)(i / chunks) * ldx + i % chunks * 8, values_of<T>(*(const uint2 *)(codes + (int64_t)(p.slot + i / chunks) * D + i % chunks * 8), s));
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
            store_once(x + (int64_t)(token - p.slot) * ldx + i % chunks * 8, values_of<T>(*(const uint2 *)&tile[(token - base) * (D / 4) + i % chunks * 2], s));
        }
    }
}

}  // namespace

namespace {

template <typename T, int D>
void launch_write(const CacheRowsArgs &a, int per, unsigned groups, hipStream_t st)
{
    constexpr int kOf64 = kCacheTile * D / 8 / kThreads;  // a thread's chunks of 64 slots
    if (a.seq.max_new == 1)  // a wavefront does for one token
        hipLaunchKernelGGL((k_cache_write<T, D, 64, 1>), dim3(groups), dim3(64), 0, st, a, per);
    else if (a.cache.block == 64)
        hipLaunchKernelGGL((k_cache_write<T, D, kThreads, kOf64>), dim3(groups), dim3(kThreads), 0, st, a, per);
    else if (a.cache.block == 128)
        hipLaunchKernelGGL((k_cache_write<T, D, kThreads, 2 * kOf64>), dim3(groups), dim3(kThreads), 0, st, a, per);
    else
        hipLaunchKernelGGL((k_cache_write<T, D, kThreads, 4 * kOf64>), dim3(groups), dim3(kThreads), 0, st, a, per);
}

template <typename T>
void launch_write_type(const CacheRowsArgs &a, int per, unsigned groups, hipStream_t st)
{
    if (a.cache.dim == 64) launch_write<T, 64>(a, per, groups, st);
    else if (a.cache.dim == 128) launch_write<T, 128>(a, per, groups, st);
    else launch_write<T, 256>(a, per, groups, st);
}

}  // namespace

hipError_t launch_cache_write(const CacheRowsArgs &a, hipStream_t st)
{
    const int per = (int)cache_blocks_reached(a.cache, a.seq);
    const unsigned groups = (unsigned)cache_rows_groups(a.cache, a.seq);
    if (a.bf16)
        launch_write_type<__bf16>(a, per, groups, st);
    else
        launch_write_type<_Float16>(a, per, groups, st);
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
