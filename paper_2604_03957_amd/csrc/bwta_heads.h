// What the operators on heads share: 16-bit types, E4M3 codes with power-of-two scales, and which tokens of which
// sequence a workgroup has.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bwta {

// Scale exponents a cache block can have.  An fp16 value needs -33 to 9; the range keeps sums of any bf16 values that fit
// it far inside fp32 whatever two blocks' scales are.
constexpr int kCacheExpMin = -40, kCacheExpMax = 40;
constexpr int kCacheTile = 64;  // tokens an attention step takes at a time; a cache block is one, two or four of them

// The sequences of a call: which rows of its dense arrays belong to which sequence, and where that one's blocks are.
struct SeqArgs {
    const int32_t *table;
    int64_t ldt;
    const int32_t *lens, *cu;  // cu nullable: max_new rows each
    int batch, M, max_new, max_len;
};

struct CacheArgs {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    int blocks, heads, block, dim;
};

struct Seq {
    int row, n, len, start;  // first dense row, rows, tokens cached with them, position of the first row (may be negative)
};

// Offsets and lengths are data on the device: whatever they hold, rows stay inside [0, M) and positions inside max_len.
__device__ __forceinline__ Seq sequence(const SeqArgs &a, int b)
{
    Seq s;
    // (all loads at once, without a branch before any)
    const int32_t *const offsets = a.cu ? a.cu : a.lens;
    const int len = a.lens[b], begin = offsets[b], end = offsets[a.cu ? b + 1 : b];
    const int lo = a.cu ? min(max(begin, 0), a.M) : b * a.max_new;  // the host has checked batch * max_new <= M
    const int hi = a.cu ? min(max(end, lo), a.M) : lo + a.max_new;
    s.row = lo;
    s.n = hi - lo;
    s.len = min(max(len, 0), a.max_len);
    s.start = s.len - s.n;
    return s;
}

// The same for a whole wavefront's sequence, in scalar registers (the kernels of many rows have no others left: in vector registers
// chunks of long prompts took 29 % longer).
__device__ __forceinline__ Seq sequence_of_all(const SeqArgs &a, int b)
{
    const Seq s = sequence(a, b);
    return {__builtin_amdgcn_readfirstlane(s.row), __builtin_amdgcn_readfirstlane(s.n), __builtin_amdgcn_readfirstlane(s.len), __builtin_amdgcn_readfirstlane(s.start)};
}

template <typename T> struct Half;  // what differs between the two 16-bit types
template <> struct Half<_Float16> {
    static constexpr uint32_t kInf = 0x7c00;  // magnitude bits from here on are not finite
    static constexpr float kMax = 65504.0f;
    static __device__ __forceinline__ float to_float(uint32_t bits)
    {
        const uint16_t h = (uint16_t)bits;
        _Float16 f;
        __builtin_memcpy(&f, &h, 2);
        return (float)f;
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        _Float16 v[2] = {(_Float16)a, (_Float16)b};
        uint32_t r;
        __builtin_memcpy(&r, v, 4);
        return r;
    }
};
template <> struct Half<__bf16> {
    static constexpr uint32_t kInf = 0x7f80;
    static constexpr float kMax = 3.38953138925153547590e38f;
    static __device__ __forceinline__ float to_float(uint32_t bits) { return __uint_as_float(bits << 16); }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        __bf16 v[2] = {(__bf16)a, (__bf16)b};
        uint32_t r;
        __builtin_memcpy(&r, v, 4);
        return r;
    }
};

// The smallest e with amax <= 448 * 2^e, inside the cache's range; amax finite and not negative.
__device__ __forceinline__ int scale_exponent(float amax)
{
    const uint32_t b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0);  // 448 = 1.75 * 2^8; fp32 subnormals end below the range
    return min(max(e, kCacheExpMin), kCacheExpMax);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
// A stored scale's exponent.  Scales are powers of two; of any other value the exponent counts, inside the range.
__device__ __forceinline__ int exponent_of(float scale) { return min(max((int)(__float_as_uint(scale) >> 23 & 255) - 127, kCacheExpMin), kCacheExpMax); }

// four values, already divided by their scale, as codes: nearest even, NaN as 0, beyond the largest code that code
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d)
{
    auto fit = [](float x) { return x != x ? 0.0f : fminf(fmaxf(x, -448.0f), 448.0f); };
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(fit(a), fit(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fit(c), fit(d), r, true);
}

// Memory that a kernel goes over once and nobody reads again soon, past the caches' replacement order.  What it saves is room
// for the other side of a pass: rows of 8192 tokens rotated 40.7 -> 33.4 us with their loads so and 33.7 with their stores so
// (37.2 with both), 64000 tokens of 8 heads read back 54.6 -> 46.5 us with stores.
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const void *p)
{
    const uint4v x = __builtin_nontemporal_load((const uint4v *)p);
    return make_uint4(x.x, x.y, x.z, x.w);
}
__device__ __forceinline__ void store_once(void *p, uint4 v)
{
    const uint4v x = {v.x, v.y, v.z, v.w};
    __builtin_nontemporal_store(x, (uint4v *)p);
}

// 4 x 4 bytes transposed: r[i] byte j <-> r[j] byte i
__device__ __forceinline__ void transpose_bytes(uint32_t r[4])
{
    const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400), b = __builtin_amdgcn_perm(r[3], r[2], 0x05010400);
    const uint32_t c = __builtin_amdgcn_perm(r[1], r[0], 0x07030602), d = __builtin_amdgcn_perm(r[3], r[2], 0x07030602);
    r[0] = __builtin_amdgcn_perm(b, a, 0x05040100);
    r[1] = __builtin_amdgcn_perm(b, a, 0x07060302);
    r[2] = __builtin_amdgcn_perm(d, c, 0x05040100);
    r[3] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

struct HeadRopeArgs {
    const void *x[2];  // queries, keys
    void *out[2];
    const void *w[2];  // nullable
    int64_t ldx[2], ldo[2];
    int heads[2];
    int M, dim, rot;
    bool norm, interleaved, bf16;
    float eps;
    const int32_t *positions;
    const float *inv_freq;
};
hipError_t launch_head_norm_rope(const HeadRopeArgs &a, hipStream_t st);

struct CacheRowsArgs {
    CacheArgs cache;
    SeqArgs seq;
    const void *k, *v;  // dense rows: read by the write, written by the read
    int64_t ldk, ldv;
    bool bf16;
};
hipError_t launch_cache_write(const CacheRowsArgs &a, hipStream_t st);
hipError_t launch_cache_read(const CacheRowsArgs &a, hipStream_t st);
// workgroups of such a call: blocks a sequence's new tokens can reach, times sequences, heads, and two for keys and values
inline int64_t cache_blocks_reached(const CacheArgs &c, const SeqArgs &s) { return ((int64_t)s.max_new + c.block - 2) / c.block + 1; }
inline double cache_rows_groups(const CacheArgs &c, const SeqArgs &s) { return 2.0 * s.batch * c.heads * (double)cache_blocks_reached(c, s); }

struct CacheAttentionArgs {
    CacheArgs cache;
    SeqArgs seq;
    const void *q;
    void *out;
    int64_t ldq, ldo;
    float *lse;  // nullable, [M, heads]
    int heads;
    float alpha;
    bool causal, bf16;
    int window;
    // Parts of rows that are joined afterwards: [part_rows][dim] sums, then [part_rows][2] m and sum of weights.  Many
    // rows: [splits][batch * max_new * heads].  Few (share_rows of them a workgroup): [batch * key heads][splits][share_rows], or where
    // 2^share_log2 workgroups share all steps (-1: they do not) [workgroups][2][share_rows], and behind the parts how many
    // steps lie before each sequence.
    float *partial;
    int64_t part_rows;
    int splits, share_log2, share_rows;
};
struct AttentionPlan {
    int rows, row_tiles, splits, share_log2, waves;
    int reach;  // keys that the rows of a sequence see at most
    double groups;  // workgroups
    int64_t part_rows;
    size_t workspace;  // bytes
};
AttentionPlan cache_attention_plan(int heads, int kv_heads, int dim, int batch, int max_new, int reach);
hipError_t launch_cache_attention(CacheAttentionArgs a, const AttentionPlan &plan, hipStream_t st);

}  // namespace bwta
