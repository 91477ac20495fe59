// The operators of a token step on the GPU (step_ops.hip, block_attn.hip): their arguments and what they share.
#pragma once
#include "tc_internal.h"

#define TC_LAUNCH_N(kernel, grid, threads, lds_bytes, L, ...) \
    hipExtLaunchKernelGGL(kernel, dim3(grid), dim3(threads), (lds_bytes), (L).stream, (L).start, (L).stop, 0, __VA_ARGS__)

namespace tc {

constexpr int kStepMaxSeqs = 8192;            // requests of a step: three integers of each are kept in LDS
constexpr int kStepMaxTokens = 1 << 20;       // tokens of a step: their sum over the requests stays below 2^34
constexpr int kRopeMaxAxes = 4;
constexpr int64_t kStepMaxGroups = (1 << 24) - 1;       // work-groups of 256 in a launch, whose grid counts threads in 32 bits

// Division of 0 <= n < 2^31 by a number fixed at the launch: a multiplication and a shift (scalar ones, where n is the same for a
// wave; a division proper is a hundred cycles at the start of every short kernel).
struct FastDiv {
    uint32_t by, mul, shift;
    FastDiv() = default;
    explicit FastDiv(uint32_t d) : by(d), mul(0), shift(0)
    {
        while ((1ull << shift) < d) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ int operator()(int n) const { return (int)((__umulhi(mul, (uint32_t)n) + (uint32_t)n) >> shift); }
};

struct StepTables {
    const int32_t *seq_len, *new_len;
    int32_t *block_table;
    const int32_t *spare, *spare_used;
    int32_t *spare_next, *end_len, *cu_new;
    int64_t *slot_map;
    int32_t *token_pos, *token_seq, *full_block, *status;
    int32_t B, max_blocks, n_spare, n_tokens, first_seq, n_blocks;
};

struct RopeAppend {
    const char *q, *k, *v;                    // rows [n_tokens], the heads of a row behind one another
    int64_t q_stride, k_stride, v_stride;     // bytes from row to row
    char *q_out;
    const int32_t *pos;                       // [axes][n_tokens]
    const int64_t *slot_map;
    // revolutions of pair j = 8 a + b per position step, theta^(-2j/D) / (2 pi), as the product of [a] and [b] (a power and a rounding
    // off in fp64: a turn of 2^28 positions is off by 1e-8)
    double rev_coarse[8], rev_fine[8];
    int32_t section_end[kRopeMaxAxes];        // one past the last pair of each axis
    int32_t n_tokens, layer;
};

struct DigestArgs {
    const int32_t *entries;
    int8_t *digests;                          // bounds [L][Hkv][n_blocks][2][D], then exponents [L][Hkv][n_blocks]
    int64_t exps_at;
    int32_t n, l0, first_block;               // first_block: the lowest id whose keys this pool keeps in blocks
    FastDiv heads;                            // KV heads
};

struct SelectArgs {
    const char *q;
    const int32_t *token_seq, *token_pos, *block_table;
    const int8_t *digests;
    int64_t exps_at;
    int32_t *lists;
    uint32_t *scores;                         // [tokens of a round][Hkv][score_stride], by block, bits ordered like the scores
    int64_t score_stride;
    int32_t n0, n_tokens, layer, B, max_blocks, n_sink, n_top, n_local, first_block;    // tokens n0 .. n0 + n_tokens - 1
    int32_t score_parts, group_tokens;        // scores: work-groups along the candidates, and tokens of one
    FastDiv heads, parts;                     // KV heads, work-groups of one range of the candidates
};

struct BlockAttnArgs {
    const char *q;
    const int32_t *token_seq, *token_pos, *block_table, *lists;
    char *out;
    float *part_o, *part_ml;                  // [n_tokens][Hq][n_splits] rows, where the lists are split
    float scale_log2;
    int32_t n_tokens, layer, B, max_blocks, n_list, n_splits, first_block;
    FastDiv splits, chunks, heads;            // n_splits, work-groups along a group's rows, KV heads
};

// Over a wave's 64 lanes by DPP (a shuffle through LDS takes five times as long): inclusive prefix sums, and the largest.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x)
{
    x += dpp_or_zero<0x111, 0xf>(x);          // from 1, 2, 4, 8 lanes before, in each row of 16
    x += dpp_or_zero<0x112, 0xf>(x);
    x += dpp_or_zero<0x114, 0xf>(x);
    x += dpp_or_zero<0x118, 0xf>(x);
    x += dpp_or_zero<0x142, 0xa>(x);          // row 0's last lane to row 1, row 2's to row 3
    return x + dpp_or_zero<0x143, 0xc>(x);    // lane 31 to rows 2 and 3
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, dpp_or_zero<0x111, 0xf>(x));
    x = max(x, dpp_or_zero<0x112, 0xf>(x));
    x = max(x, dpp_or_zero<0x114, 0xf>(x));
    x = max(x, dpp_or_zero<0x118, 0xf>(x));
    x = max(x, dpp_or_zero<0x142, 0xa>(x));
    x = max(x, dpp_or_zero<0x143, 0xc>(x));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// 2^e, -126 <= e <= 127
__device__ __forceinline__ float step_pow2(int e) { return __int_as_float((e + 127) << 23); }

// The smallest e >= -126 with size <= 127 * 2^e, for a finite size >= 0.
__device__ __forceinline__ int step_exponent(float size)
{
    const int e = max((int)(__float_as_uint(size) >> 23) - 127 - 6, -126);
    return e + (size * step_pow2(-e) > 127.f ? 1 : 0);
}

// Pairs of two 16-byte chunks of a head row, elements j and j + D/2, turned by w = (cos, sin) of each.
template <bool kBf16>
__device__ __forceinline__ void turn_chunk(uint4 &x, uint4 &y, const float2 *w)
{
    unsigned a[4] = {x.x, x.y, x.z, x.w}, b[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (kBf16) {
            unsigned ra = 0, rb = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float xa = __uint_as_float(e ? a[k] & 0xffff0000u : a[k] << 16), xb = __uint_as_float(e ? b[k] & 0xffff0000u : b[k] << 16);
                const float2 cs = w[2 * k + e];
                const __bf16 na = (__bf16)(xa * cs.x - xb * cs.y), nb = (__bf16)(xb * cs.x + xa * cs.y);
                ra |= (unsigned)__builtin_bit_cast(unsigned short, na) << (16 * e);
                rb |= (unsigned)__builtin_bit_cast(unsigned short, nb) << (16 * e);
            }
            a[k] = ra;
            b[k] = rb;
        } else {
            const float xa = __uint_as_float(a[k]), xb = __uint_as_float(b[k]);
            const float2 cs = w[k];
            a[k] = __float_as_uint(xa * cs.x - xb * cs.y);
            b[k] = __float_as_uint(xb * cs.x + xa * cs.y);
        }
    }
    x = make_uint4(a[0], a[1], a[2], a[3]);
    y = make_uint4(b[0], b[1], b[2], b[3]);
}

// Work-groups that share a token's list: ranges of its units (two blocks in bf16, one in fp32).
int block_attn_splits(int Hq, int Hkv, int esize, int n_tokens, int n_list);
// The most (token, range) partials of a query head that up to n_tokens tokens keep, where lists are shared out.
int block_attn_parts(int Hq, int Hkv, int esize, int n_tokens, int n_list);
// Work-groups that a token's lists, and its attention in one range, take in a launch.
int64_t select_groups(int Hkv, int max_blocks);
int block_attn_groups(int Hq, int Hkv, int esize);

hipError_t launch_step_tables(const StepTables &s, const Launch &L);
hipError_t launch_rope_append(const Geom &g, const RopeAppend &a, const Launch &L);
hipError_t launch_digest(const Geom &g, DigestArgs a, int l1, const Launch &L);
hipError_t launch_select(const Geom &g, SelectArgs a, const Launch &L);
hipError_t launch_block_attn(const Geom &g, BlockAttnArgs a, const Launch &L);
hipError_t launch_block_merge(const Geom &g, const BlockAttnArgs &a, const Launch &L);

}  // namespace tc
