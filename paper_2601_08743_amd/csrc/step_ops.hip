// A token step that stays on the GPU: block tables and slot maps from the requests' lengths, queries and keys encoded by
// position with the append to the pool, and 8-bit bounds of the keys of pool blocks.  (Lists by those bounds and the
// attention over them: block_attn.hip.)
#include "arrive.h"
#include "kv_append.h"
#include "step_ops.h"

namespace tc {

// ------------------------------------------------------------------------------------ tables
// Request b holds len_b tokens in have_b = ceil(len_b / 16) blocks and brings new_b; blocks have_b .. ceil((len_b + new_b) / 16)
// are spare ones, taken in order, requests in order.  A block is new to its sequence exactly if its position 0 is among the
// step's tokens, so whoever writes that token's slot writes the table entry, and nobody reads an entry that the step writes.
//
// Two prefix sums over the requests, of new tokens and of blocks, run as one of 64 bits (34 for the tokens, 30 for the
// blocks); then a thread for every token, which finds its request by bisection in LDS.  Everything is a few kilobytes: what
// counts is the chain of dependent steps, so up to kTablesOneWg tokens one work-group does all of it in one launch.  More tokens
// are written by many work-groups of a second launch, each of which repeats the sums (the first launch's results may stand
// where its inputs stood, so the second takes its lengths from those).
constexpr int kTokenBits = 34;

template <int kThreads, bool kScan, bool kFill>
__global__ __launch_bounds__(kThreads) void step_tables_kernel(StepTables s)
{
    extern __shared__ int32_t lds[];                    // [B + 1] first token, [B] tokens held, [B] first spare block
    __shared__ uint64_t s_wave[kThreads / 64];
    __shared__ int32_t s_bad;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, B = s.B;
    int32_t *cu = lds, *held = lds + B + 1, *first = held + B;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    // (a fill launch of its own finds the step's end lengths, and the cursor behind the step's blocks)
    const bool refused = !kScan && s.status[0] != 0;
    const int32_t used = kScan ? s.spare_used[0] : s.spare_next[0] - (refused ? 0 : s.status[1]);
    uint64_t carry = 0;
    bool bad = used < 0 || used > s.n_spare;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + tid;
        int32_t len = 0, fresh = 0;
        if (b < B) {
            fresh = s.new_len[b];
            len = kScan ? s.seq_len[b] : s.end_len[b] - (refused ? 0 : fresh);
            if (len < 0 || fresh < 0 || (int64_t)len + fresh > (int64_t)s.max_blocks * kBlockTokens || fresh > s.n_tokens) {
                bad = true;
                fresh = 0;
            }
        }
        const uint32_t blocks = (uint32_t)((len + fresh + 15) >> 4) - (uint32_t)((len + 15) >> 4);
        const uint64_t mine = bad ? 0 : (uint64_t)fresh | ((uint64_t)blocks << kTokenBits);
        uint64_t x = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint64_t y = __shfl_up((unsigned long long)x, d);
            if (lane >= d) x += y;
        }
        if (lane == 63) s_wave[w] = x;
        __syncthreads();
        uint64_t before = carry;
        for (int k = 0; k < w; ++k) before += s_wave[k];
        for (int k = 0; k < kThreads / 64; ++k) carry += s_wave[k];
        if (b < B) {
            const uint64_t at = before + x - mine;
            cu[b] = (int32_t)min(at & ((1ull << kTokenBits) - 1), (uint64_t)INT32_MAX);
            first[b] = (int32_t)(at >> kTokenBits);
            held[b] = len;
        }
        __syncthreads();
    }
    if (bad) s_bad = 1;
    __syncthreads();
    const uint64_t n_new = carry & ((1ull << kTokenBits) - 1);
    const int32_t n_blocks = (int32_t)(carry >> kTokenBits);
    int32_t code = refused || s_bad || n_new > (uint64_t)s.n_tokens ? -1 : 0;
    if (code == 0 && n_blocks > s.n_spare - used) code = -3;
    const int32_t total = code == 0 ? (int32_t)n_new : 0;
    if (kScan) {
        for (int b = tid; b < B; b += kThreads) {
            s.cu_new[b] = code == 0 ? cu[b] : 0;
            s.end_len[b] = held[b] + (code == 0 ? s.new_len[b] : 0);
        }
        if (tid == 0) {
            s.cu_new[B] = total;
            s.spare_next[0] = used + (code == 0 ? n_blocks : 0);
            s.status[0] = code;
            s.status[1] = code == -1 ? 0 : n_blocks;
        }
    }
    if (kFill) {
        if (tid == 0) cu[B] = total;
        __syncthreads();
        for (int n = blockIdx.x * kThreads + tid; n < s.n_tokens; n += gridDim.x * kThreads) {
            int64_t slot = -1;
            int32_t pos = -1, seq = -1, full = -1;
            if (n < total) {
                int lo = 0, hi = B;                     // the last request whose first token is not behind n
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (cu[mid] <= n) lo = mid;
                    else hi = mid;
                }
                seq = lo;
                pos = held[lo] + (n - cu[lo]);
                const int j = pos >> 4, have = (held[lo] + 15) >> 4;
                int32_t *entry = s.block_table + (int64_t)lo * s.max_blocks + j;
                int32_t id;
                if (j < have) {
                    id = *entry < 0 ? -1 : entry_bid(*entry);
                } else {
                    id = s.spare[used + first[lo] + (j - have)];
                    if (id < s.first_seq || id >= s.n_blocks) id = -1;
                    if ((pos & 15) == 0) *entry = id;
                }
                if (id >= 0) {
                    slot = (int64_t)id * kBlockTokens + (pos & 15);
                    if ((pos & 15) == 15) full = id;
                }
            }
            s.slot_map[n] = slot;
            s.token_pos[n] = pos;
            s.token_seq[n] = seq;
            s.full_block[n] = full;
        }
    }
}

constexpr int kTablesOneWg = 8192;

hipError_t launch_step_tables(const StepTables &s, const Launch &L)
{
    const size_t lds = (3 * (size_t)s.B + 1) * sizeof(int32_t);
    static PerDeviceOnce configured;
    const hipError_t e = configured.run([] {
        const int most = (3 * kStepMaxSeqs + 1) * (int)sizeof(int32_t);
        hipError_t e0 = hipFuncSetAttribute((const void *)step_tables_kernel<1024, true, true>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e0 == hipSuccess) e0 = hipFuncSetAttribute((const void *)step_tables_kernel<1024, true, false>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e0 == hipSuccess) e0 = hipFuncSetAttribute((const void *)step_tables_kernel<1024, false, true>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
        return e0;
    });
    if (e != hipSuccess) return e;
    if (s.B <= 256 && s.n_tokens <= 1024) {
        TC_LAUNCH_N((step_tables_kernel<256, true, true>), 1, 256, lds, L, s);
    } else if (s.n_tokens <= kTablesOneWg) {
        TC_LAUNCH_N((step_tables_kernel<1024, true, true>), 1, 1024, lds, L, s);
    } else {
        TC_LAUNCH_N((step_tables_kernel<1024, true, false>), 1, 1024, lds, L, s);
        TC_LAUNCH_N((step_tables_kernel<1024, false, true>), (s.n_tokens + 2047) / 2048, 1024, lds, L, s);
    }
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ encode and append
// Queries and keys turned by position - pair (j, j + D/2) of every head by pos * theta^(-2j/D), the position being that of the
// axis whose section j falls into - and keys and values written to their slots, in one pass over the rows.  As in the
// re-encoding stitch the turn is a fraction of a revolution taken in fp64, sine and cosine and the rotation are fp32 and the
// result is rounded once.
//
// A work-group a token: its (cos, sin) table in LDS, then a thread for every pair of 16-byte chunks.
template <bool kBf16>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeFreq, Geom g, RopeAppend a)
{
    __shared__ float2 cs[64];
    typedef const __attribute__((address_space(4))) double *const_doubles;
    const const_doubles rev = (const_doubles)__builtin_amdgcn_kernarg_segment_ptr();
    const int tid = threadIdx.x, n = blockIdx.x;
    const int64_t slot = a.slot_map[n];
    const int64_t blk = slot >> 4;
    if (slot < 0 || blk < g.first_seq || blk >= g.n_blocks) return;     // a padded row, or no block of a sequence
    const int t = (int)(slot & 15);
    const int half_d = g.D >> 1, cph = g.head_bytes >> 4, half_c = cph >> 1;
    if (tid < half_d) {
        int axis = 0;
        while (tid >= a.section_end[axis]) ++axis;
        const double turns = (double)a.pos[(int64_t)axis * a.n_tokens + n] * rev[tid];
        const float frac = (float)(turns - floor(turns));
        float sn, c;
        if (kBf16) {
            sn = __builtin_amdgcn_sinf(frac);
            c = __builtin_amdgcn_cosf(frac);
        } else {
            sincospif(2.0f * frac, &sn, &c);
        }
        cs[tid] = make_float2(c, sn);
    }
    // a block that gets its first token here is zero behind the step's last token in it
    int zero_to = t;
    if (t == 0) {
        zero_to = 16;
        while (zero_to > 1 && !(n + zero_to - 1 < a.n_tokens && a.slot_map[n + zero_to - 1] == slot + zero_to - 1)) --zero_to;
    }
    __syncthreads();
    char *kd = g.pool + (int64_t)a.layer * g.layer_stride + blk * g.block_bytes;
    char *vd = kd + (g.block_bytes >> 1);
    constexpr int kElems = kBf16 ? 8 : 4;
    const int rot_units = (g.Hq + g.Hkv) * half_c, units = rot_units + g.Hkv * cph;
    for (int u = tid; u < units; u += 256) {
        if (u < rot_units) {
            const int h = u / half_c, cc = u - h * half_c;
            const bool is_q = h < g.Hq;
            const char *src = (is_q ? a.q + n * a.q_stride + (int64_t)h * g.head_bytes : a.k + n * a.k_stride + (int64_t)(h - g.Hq) * g.head_bytes) + (cc << 4);
            char *dst = (is_q ? a.q_out + ((int64_t)n * g.Hq + h) * g.head_bytes : kd + (int64_t)((h - g.Hq) * kBlockTokens + t) * g.head_bytes) + (cc << 4);
            uint4 x = *(const uint4 *)src, y = *(const uint4 *)(src + (half_c << 4));
            const float2 *w = cs + cc * kElems;
            turn_chunk<kBf16>(x, y, w);
            *(uint4 *)dst = x;
            *(uint4 *)(dst + (half_c << 4)) = y;
        } else {
            const int r = u - rot_units, h = r / cph, cc = r - h * cph;
            const uint4 v = *(const uint4 *)(a.v + n * a.v_stride + (int64_t)h * g.head_bytes + (cc << 4));
            if (!kBf16) {
                *(uint4 *)(vd + (int64_t)(h * kBlockTokens + t) * g.head_bytes + (cc << 4)) = v;
            } else {
                const unsigned e[4] = {v.x, v.y, v.z, v.w};
                unsigned short *v16 = (unsigned short *)vd;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    v16[((int64_t)(h * g.D + cc * 8 + k) << 4) + vperm(t)] = (unsigned short)(e[k >> 1] >> ((k & 1) * 16));
            }
        }
    }
    if (t == 0 && zero_to < kBlockTokens) {
        const uint4 zero = make_uint4(0, 0, 0, 0);
        const int rows = kBlockTokens - zero_to, cpr = g.row_bytes >> 4;
        for (int c = tid; c < rows * cpr; c += 256) {
            const int tt = zero_to + c / cpr, w = c % cpr, h = w / cph, cc = w - h * cph;
            *(uint4 *)(kd + (int64_t)(h * kBlockTokens + tt) * g.head_bytes + (cc << 4)) = zero;
            if (!kBf16) {
                *(uint4 *)(vd + (int64_t)(h * kBlockTokens + tt) * g.head_bytes + (cc << 4)) = zero;
            } else {
                unsigned short *v16 = (unsigned short *)vd;
#pragma unroll
                for (int k = 0; k < 8; ++k) v16[((int64_t)(h * g.D + cc * 8 + k) << 4) + vperm(tt)] = 0;
            }
        }
    }
}

hipError_t launch_rope_append(const Geom &g, const RopeFreq &f, const RopeAppend &a, const Launch &L)
{
    if (a.n_tokens == 0) return hipSuccess;
    if (g.esize == 2) TC_LAUNCH(rope_append_kernel<true>, a.n_tokens, 0, L, f, g, a);
    else TC_LAUNCH(rope_append_kernel<false>, a.n_tokens, 0, L, f, g, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ digests
// Bounds of a block's keys, channel by channel, in 8 bits with one power of two for all: hi = max over the block's tokens, lo =
// min; e the smallest integer, -126 at least, with max(|hi|, |lo|) <= 127 * 2^e; stored are ceil(hi / 2^e) and
// floor(lo / 2^e), so that they stay bounds, and e (127 where some key is not finite).  Dividing by a power of two is exact:
// the bytes follow from the keys alone, whatever computes them.
//
// One read of the keys: a wave takes one block of one KV head, 16 rows that stand behind one another, and holds 16 bytes of each
// fourth (or second) row in a lane.  Maximum and minimum are taken on the bits, made to order like integers, in which
// an infinity or a NaN is an extreme of its sign and so is seen at the end.
template <bool kBf16>
struct Sortable;
template <>
struct Sortable<true> {                                  // two bf16 in a register
    typedef short vec __attribute__((ext_vector_type(2)));
    static constexpr int kPerWord = 2;
    __device__ static __forceinline__ vec flip(vec x) { return x ^ ((x >> 15) & (short)0x7fff); }
    __device__ static __forceinline__ float value(vec x, int i) { return __uint_as_float((uint32_t)(unsigned short)flip(x)[i] << 16); }
};
template <>
struct Sortable<false> {
    typedef int vec __attribute__((ext_vector_type(1)));
    static constexpr int kPerWord = 1;
    __device__ static __forceinline__ vec flip(vec x) { return x ^ ((x >> 31) & 0x7fffffff); }
    __device__ static __forceinline__ float value(vec x, int) { return __int_as_float(flip(x)[0]); }
};

template <bool kBf16, int kLanes>                        // kLanes: 16-byte chunks of a key row, 16 or 32
__global__ __launch_bounds__(256) void digest_kernel(Geom g, DigestArgs a)
{
    typedef typename Sortable<kBf16>::vec vec;
    constexpr int kRowsAt = 64 / kLanes, kLoads = kBlockTokens / kRowsAt, kElems = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 63;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int i = unit / g.Hkv, h = unit - i * g.Hkv, layer = a.l0 + blockIdx.y;
    if (i >= a.n) return;
    const int32_t entry = a.entries[i];
    if (entry < 0 || entry_bid(entry) >= g.n_blocks || entry_bid(entry) < a.first_block) return;
    const int bid = entry_bid(entry), last = kBlockTokens - 1 - entry_pad(entry);       // the last row that holds a key
    const char *k = g.pool + (int64_t)layer * g.layer_stride + (int64_t)bid * g.block_bytes + (int64_t)h * kBlockTokens * g.head_bytes;
    const int row = lane / kLanes, c = lane % kLanes;
    union { uint4 u; vec v[4]; } x[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) x[j].u = *(const uint4 *)(k + min(row + j * kRowsAt, last) * g.head_bytes + c * 16);
    vec hi[4], lo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) hi[q] = lo[q] = Sortable<kBf16>::flip(x[0].v[q]);
#pragma unroll
    for (int j = 1; j < kLoads; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const vec y = Sortable<kBf16>::flip(x[j].v[q]);
            hi[q] = __builtin_elementwise_max(hi[q], y);
            lo[q] = __builtin_elementwise_min(lo[q], y);
        }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            hi[q] = __builtin_elementwise_max(hi[q], __builtin_bit_cast(vec, __shfl_xor(__builtin_bit_cast(int, hi[q]), m)));
            lo[q] = __builtin_elementwise_min(lo[q], __builtin_bit_cast(vec, __shfl_xor(__builtin_bit_cast(int, lo[q]), m)));
        }
    float up[kElems], dn[kElems];
    uint32_t size = 0;                                   // of the largest bound, as bits (they order like the sizes)
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
        up[e] = Sortable<kBf16>::value(hi[e / Sortable<kBf16>::kPerWord], e % Sortable<kBf16>::kPerWord);
        dn[e] = Sortable<kBf16>::value(lo[e / Sortable<kBf16>::kPerWord], e % Sortable<kBf16>::kPerWord);
        size = max(size, max(__float_as_uint(up[e]) & 0x7fffffffu, __float_as_uint(dn[e]) & 0x7fffffffu));
    }
#pragma unroll
    for (int m = 1; m < kLanes; m <<= 1) size = max(size, (uint32_t)__shfl_xor((int)size, m));
    const bool finite = size < 0x7f800000u;
    const int e = finite ? step_exponent(__uint_as_float(size)) : 127;
    const float by = finite ? step_pow2(-e) : 0.f;
    // lanes of row group 0 write the upper bounds, those of the last one the lower bounds
    if (row == 0 || row == kRowsAt - 1) {
        uint32_t out[kElems / 4];
#pragma unroll
        for (int w = 0; w < kElems / 4; ++w) {
            uint32_t b = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float y = row == 0 ? ceilf(up[4 * w + q] * by) : floorf(dn[4 * w + q] * by);
                b |= ((uint32_t)(finite ? (int)y : 0) & 0xffu) << (8 * q);
            }
            out[w] = b;
        }
        const int64_t at = ((int64_t)layer * g.Hkv + h) * g.n_blocks + bid;
        int8_t *dst = a.digests + at * 2 * g.D + (row == 0 ? 0 : g.D) + c * kElems;
        if (kBf16) *(uint2 *)dst = make_uint2(out[0], out[kElems / 4 - 1]);
        else *(uint32_t *)dst = out[0];
        if (lane == 0) a.digests[a.exps_at + at] = (int8_t)e;
    }
}

hipError_t launch_digest(const Geom &g, const DigestArgs &a, int l1, const Launch &L)
{
    if (a.n == 0 || l1 <= a.l0) return hipSuccess;
    const int64_t units = (int64_t)a.n * g.Hkv;
    const dim3 grid((unsigned)((units + 3) / 4), l1 - a.l0);
    if (g.esize == 2) TC_LAUNCH((digest_kernel<true, 16>), grid, 0, L, g, a);
    else if (g.D == 64) TC_LAUNCH((digest_kernel<false, 16>), grid, 0, L, g, a);
    else TC_LAUNCH((digest_kernel<false, 32>), grid, 0, L, g, a);
    return hipGetLastError();
}

}  // namespace tc
