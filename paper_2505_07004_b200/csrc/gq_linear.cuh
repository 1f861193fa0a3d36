// Products with weights in the form the quantiser leaves them: a 4-bit code per weight and a table of levels per output channel,
//
//   z_ij = sum_c x_ic table[j][code[j][c]] + b_j,    y = act(z) + r
//   dz = dy act'(z),   dx_ic = sum_j dz_ij table[j][code[j][c]]
//
// Layout (linear_pack_kernel): codes [d_out][ld] bytes, two codes a byte, the lower four bits first, ld = 16 ceil(d_in / 32);
// table [d_out][16] in the activations' type (bf16 or fp16), zero from m on.
//
// On the tensor cores' path a level is looked up in registers: a channel's 16 levels are kept as two planes of 16 bytes (low and high
// bytes, eight registers), and a byte permutation looks four codes up in eight bytes at once.  For four weights: two permutations a
// plane (levels 0..7 and 8..15), one that takes either by the codes' top bits, and two that join the planes: 2.6 integer instructions a
// weight, 1.3 where m <= 8.  Few tokens (linear_token_kernel, up to 16) are bound by the codes' bytes and, behind them, the lookups,
// and use tables in shared memory.  More tokens (linear_pair_kernel): tensor cores, the weight operand written to shared memory by
// eight lookup warps.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gq_kernels.cuh"
#include "gq_pipeline.cuh"
#include "gq_score.cuh"

namespace gq {

constexpr int LIN_LEVELS = 16;
enum LinearAct { LIN_NONE = 0, LIN_RELU = 1, LIN_SILU = 2, LIN_GELU = 3 };

__device__ __forceinline__ uint4 ld_u32x4(const void *p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Bytes of (a, b) picked by the low four nibbles of s, whose top bits have to be zero (the intrinsic masks them off, one more
// instruction each time).
__device__ __forceinline__ uint32_t pick_bytes(uint32_t a, uint32_t b, uint32_t s)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(s));
    return r;
}

__device__ __forceinline__ uint32_t ld_u32(const void *p)
{
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_shared_4(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint4 ld_shared_16(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// Asynchronous copies of 16 bytes from global to shared memory, past L1.
__device__ __forceinline__ void copy_async_16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copy_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// The levels of a channel as byte planes.
struct LevelPlanes {
    uint32_t lo[4], hi[4];
    __device__ __forceinline__ void set(const uint4 &a, const uint4 &b)
    {
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            lo[q] = __byte_perm(w[2 * q], w[2 * q + 1], 0x6420);
            hi[q] = __byte_perm(w[2 * q], w[2 * q + 1], 0x7531);
        }
    }
    // Eight codes -> eight 16-bit levels, in the codes' order.  WIDE: more than eight levels.
    template <bool WIDE>
    __device__ __forceinline__ uint4 look(uint32_t q) const
    {
        const uint32_t sel = q & 0x77777777u;
        const uint32_t top = ((q >> 1) & 0x44444444u) | 0x32103210u;
        uint4 out;
        uint32_t *o = reinterpret_cast<uint32_t *>(&out);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t s = h ? sel >> 16 : sel;
            uint32_t l = pick_bytes(lo[0], lo[1], s), u = pick_bytes(hi[0], hi[1], s);
            if (WIDE) {
                const uint32_t t = h ? top >> 16 : top;
                l = pick_bytes(l, pick_bytes(lo[2], lo[3], s), t);
                u = pick_bytes(u, pick_bytes(hi[2], hi[3], s), t);
            }
            o[2 * h] = pick_bytes(l, u, 0x5140);
            o[2 * h + 1] = pick_bytes(l, u, 0x7362);
        }
        return out;
    }
};

// The activation of N values, each about to be rounded to 16 bits.  SiLU by the fast exponential and quotient: 2 + 1.2 |z| units in the last
// place, and 0 below z = -87.3, where a divisor above 2^126 makes the quotient 0 (the value is smaller than |z| 2^-126).  The kind is asked
// for once: a branch per value keeps the values' evaluations from overlapping, and the epilogue of 2048 tokens 4096 -> 11008 took 46 us
// longer with SiLU than without.
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int act)
{
    if (act == LIN_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = z[e] > 0.0f ? z[e] : (z[e] != z[e] ? z[e] : 0.0f);
    } else if (act == LIN_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = __fdividef(z[e], 1.0f + __expf(-z[e]));
    } else if (act == LIN_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = 0.5f * z[e] * (1.0f + erff(z[e] * 0.70710678118654752f));
    }
}
// The slope's fp32 value decides how dZ is rounded, and the fp32 gradients are those of the rounded dZ: no fast approximations.
// SiLU: s (1 + z (1 - s)) with s = 1 / (1 + exp(-z)).  Below z = -64 s is exp(z) to the last bit, down to 0, where a reciprocal of exp(-z) would
// have to stop at infinity; above, d = 1 + exp(-z) lies in [1, 2^93], and one Newton-Raphson step r + r (1 - d r) takes the fast quotient's
// two units in the last place to half of one and a little.  The slope is good to 24 times 2^-24 of s (1 + |z| (1 - s)).  dZ of 2048 x 4096
// takes 16.2 us; with __frcp_rn, which branches, 17.3; with the quotient alone 14.9, but up to twice as many of them are rounded the
// other way.
__device__ __forceinline__ float activation_slope(float z, int act)
{
    if (act == LIN_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (act == LIN_SILU) {
        const bool low = z < -64.0f;
        const float e = expf(low ? z : -z), d = 1.0f + e, r = __fdividef(1.0f, d), sig = low ? e : fmaf(r, fmaf(-d, r, 1.0f), r);
        return sig * (1.0f + z * (1.0f - sig));
    }
    if (act == LIN_GELU) return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    return 1.0f;
}

__device__ __forceinline__ float half_value(uint32_t bits, bool bf16)
{
    return bf16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half(static_cast<unsigned short>(bits)));
}
__device__ __forceinline__ uint32_t half_bits(float v, bool bf16)
{
    return bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}
__device__ __forceinline__ float2 half2_value(uint32_t bits, bool bf16)
{
    return bf16 ? make_float2(__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u))
                : __half22float2(*reinterpret_cast<const __half2 *>(&bits));
}
__device__ __forceinline__ uint32_t half2_bits(float x, float y, bool bf16)
{
    if (bf16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// ------------------------------------------------------------------------------------------------ layout
// One block per channel: codes as nibbles (larger ones as m - 1, zero behind d_in), levels rounded to the activations' type.
__global__ void __launch_bounds__(128) linear_pack_kernel(const uint8_t *Q, const float *codebook, int m, int d_in, int ld_codes, int bf16,
                                                          uint8_t *codes, uint16_t *table)
{
    griddep_launch();
    griddep_wait();
    const size_t j = blockIdx.x;
    const uint8_t *q = Q + j * static_cast<size_t>(d_in);
    uint32_t *out = reinterpret_cast<uint32_t *>(codes + j * static_cast<size_t>(ld_codes));
    for (int w = threadIdx.x; w < ld_codes / 4; w += 128) {
        uint32_t v = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = 8 * w + e;
            if (c < d_in) v |= static_cast<uint32_t>(min(static_cast<int>(q[c]), m - 1)) << (4 * e);
        }
        out[w] = v;
    }
    if (threadIdx.x < LIN_LEVELS) {
        const float v = static_cast<int>(threadIdx.x) < m ? codebook[j * m + threadIdx.x] : 0.0f;
        table[j * LIN_LEVELS + threadIdx.x] = static_cast<uint16_t>(half_bits(v, bf16 != 0));
    }
}

// ------------------------------------------------------------------------------------------------ few tokens
struct LinearParams {
    const uint8_t *codes;
    const uint16_t *table;
    int ld_codes;            // bytes
    int n, d_in, d_out;
    int act, bf16;
    const uint16_t *bias;
    const uint16_t *residual;
    long long ld_r;
    uint16_t *out;           // Y (forward) or dX
    long long ld_out;
    uint16_t *Z;
    long long ld_z;
    const uint16_t *X;       // few tokens only: the pair kernel reads X through a tensor map
    long long ld_x;
    // pair kernel
    int row_tiles, tok_tiles, doubles, units, pairs;      // tiles of 256 rows, of 512 tokens
    int ranks, ntile, box_rows;                           // shares of the contraction, columns of a tile, tokens of a TMA box (SPLIT)
    uint32_t *status;
    unsigned long long wait_budget_ns;
};

constexpr int LT_WARPS = 8;
constexpr int LT_THREADS = 32 * LT_WARPS;         // a thread per pair of codes when the tables are built
constexpr int LT_CHANNELS = 16;
constexpr int LT_TOKENS = 8;              // columns of a product; a CTA takes up to two of them
constexpr int LT_K = 128;                 // contraction indices a warp takes at a time: 32 per lane of a quad
constexpr int LT_MAX_CLUSTER = 8;
constexpr int LT_AHEAD = 4;               // pieces of codes on their way to a warp
constexpr int LT_TABLE_BYTES = 256 * 128;         // levels of all pairs of codes for 8 channels, a word per lane
constexpr int LT_CODE_PITCH = 80;                 // a channel's 64 bytes of a piece: with 16 more, words t of all channels lie in different banks
constexpr int LT_CODE_BYTES = LT_CHANNELS * LT_CODE_PITCH;      // a piece of a warp's codes
constexpr int LT_SMEM_BYTES = 2 * LT_TABLE_BYTES + LT_WARPS * LT_AHEAD * LT_CODE_BYTES;

template <bool BF16>
__device__ __forceinline__ void mma_m16n8k16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 channels per cluster of `ranks` CTAs, the contraction dealt to their warps in pieces of 128.  The order of the contraction indices
// inside a piece is free as long as both operands share it.  SPREAD: lane (g, t) of a quad takes the indices 32 q + 8 t .. + 7 for
// q = 0 .. 3, of token g's activations 16 bytes each, next to those of the quad's other lanes, and of channels g and g + 8 one word of
// codes each.  Otherwise it takes 32 indices in a row, 32 t .. 32 t + 31: the codes it has copied itself, and activations whose 16-byte
// loads lie 64 bytes apart in a quad, twice the lines.  28672 -> 8192, SPREAD / not: one token 42.5 / 39.9 us, four 44.4 / 48.0, eight
// 55 / 66; 4096 x 4096, one token 6.2 / 5.6.
//
// Lookups: a byte of codes names two levels, which stand side by side in a table of 256 words for the channel.  Every lane has its
// own copy in its own bank (row = byte, word = lane: 32 KB for 8 channels), so 32 random bytes meet no conflicts: a load and two integer
// instructions for two weights, where looking them up in registers takes more than five.
template <bool BF16, int NT, bool SPREAD>
__global__ void __launch_bounds__(LT_THREADS, 2) linear_token_kernel(const LinearParams p, int ranks)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    constexpr int TOKENS = NT * LT_TOKENS, X_AHEAD = 2 / NT;      // (pieces of activations in registers)
    constexpr int PITCH = SPREAD ? LT_CODE_PITCH : 64;            // of a channel's codes in shared memory
    __shared__ float mine[TOKENS * LT_CHANNELS];
    __shared__ uint16_t levels[LT_CHANNELS][LIN_LEVELS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int group = static_cast<int>(blockIdx.x) / ranks, rank = static_cast<int>(blockIdx.x) - group * ranks;
    const int j0 = group * LT_CHANNELS;
    const uint32_t tables = smem_u32(smem_raw), ring = tables + 2 * LT_TABLE_BYTES + static_cast<uint32_t>(warp * LT_AHEAD * LT_CODE_BYTES);
    float (*sums)[TOKENS][LT_CHANNELS] = reinterpret_cast<float (*)[TOKENS][LT_CHANNELS]>(smem_raw + 2 * LT_TABLE_BYTES);      // after the ring's use
    griddep_launch();
    griddep_wait();
    // channels are a multiple of 8, so either all of g or all of g + 8 are there
    const bool second = j0 + 8 < p.d_out;
    const int ja = j0 + g, jb = second ? ja + 8 : ja;
    const uint8_t *ca = p.codes + static_cast<size_t>(ja) * p.ld_codes, *cb = p.codes + static_cast<size_t>(jb) * p.ld_codes;
    const uint16_t *x[NT];
    bool have[NT];
#pragma unroll
    for (int o = 0; o < NT; ++o) {
        have[o] = g + o * LT_TOKENS < p.n;
        x[o] = p.X + static_cast<long long>(have[o] ? g + o * LT_TOKENS : 0) * p.ld_x;
    }
    const int pieces = (p.d_in + LT_K - 1) / LT_K, stride = ranks * LT_WARPS;
    // A warp takes pairs of neighbouring pieces (128 bytes of a channel's codes): pairs base, base + stride, ...  The `whole` first of its pieces
    // lie inside the row, one ragged piece may follow.
    // Codes come from device memory, by asynchronous copies LT_AHEAD pieces ahead, 16 bytes of either channel a lane; in registers the loads
    // of four pieces shared the few scoreboards there are, and waits for one waited for the others (one token 44 us instead of 39).
    // Activations come from L2 or L1, one or two pieces ahead, in registers.
    const int base = rank * LT_WARPS + warp, full = p.d_in / LT_K, last_pair = full / 2;
    const int whole = (base < last_pair ? 2 * ((last_pair - base + stride - 1) / stride) : 0) + ((full & 1) != 0 && last_pair % stride == base ? 1 : 0);
    const bool ragged = full < pieces && last_pair % stride == base;
    auto index_of = [&](int i) { return ((base + (i >> 1) * stride) * 2 + (i & 1)) * LT_K; };      // first index of the i-th piece
    auto eight = [&](int q) { return SPREAD ? 32 * q + 8 * t : 32 * t + 8 * q; };              // this lane's q-th eight indices in a piece
    const uint32_t copy_to = ring + static_cast<uint32_t>(g * PITCH + t * 16), word_at = ring + static_cast<uint32_t>(g * PITCH + t * 4);
    constexpr uint32_t SECOND = 8 * PITCH;                      // channels 8 .. 15
    uint4 tokens[X_AHEAD][NT][4];
#pragma unroll
    for (int d = 0; d < X_AHEAD; ++d)
#pragma unroll
        for (int o = 0; o < NT; ++o)
#pragma unroll
            for (int q = 0; q < 4; ++q) tokens[d][o][q] = make_uint4(0u, 0u, 0u, 0u);      // stays so in lanes without a token
    auto fetch_codes = [&](int i, int slot) {
        if (i < whole) {
            const int at = (index_of(i) >> 1) + 16 * t;
            copy_async_16(copy_to + slot * LT_CODE_BYTES, ca + at);
            copy_async_16(copy_to + slot * LT_CODE_BYTES + SECOND, cb + at);
        }
        copy_async_commit();                                     // a group a piece, empty past the end
    };
    auto fetch_tokens = [&](int i, uint4 (&f)[NT][4]) {
#pragma unroll
        for (int o = 0; o < NT; ++o)
            if (i < whole && have[o]) {
#pragma unroll
                for (int q = 0; q < 4; ++q) f[o][q] = ld_u32x4(x[o] + index_of(i) + eight(q));
            }
    };
#pragma unroll
    for (int d = 0; d < LT_AHEAD; ++d) fetch_codes(d, d);
    // the levels of 16 channels: 512 bytes
    if (tid < LT_CHANNELS * LIN_LEVELS / 2) {
        const int ch = tid / (LIN_LEVELS / 2), j = j0 + ch < p.d_out ? j0 + ch : j0;
        reinterpret_cast<uint32_t *>(&levels[ch][0])[tid % (LIN_LEVELS / 2)] =
            *(reinterpret_cast<const uint32_t *>(p.table + static_cast<size_t>(j) * LIN_LEVELS) + tid % (LIN_LEVELS / 2));
    }
#pragma unroll
    for (int d = 0; d < X_AHEAD; ++d) fetch_tokens(d, tokens[d]);
    __syncthreads();
    // Thread = pair of codes; eight threads next to each other store to eight different channels' words of their rows.
    if (tid < 256) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int ch = (i + tid) & 7;
                const uint32_t v = static_cast<uint32_t>(levels[8 * h + ch][tid & 15]) | (static_cast<uint32_t>(levels[8 * h + ch][tid >> 4]) << 16);
                st_shared_16(tables + h * LT_TABLE_BYTES + tid * 128 + ch * 16, make_uint4(v, v, v, v));
            }
    }
    __syncthreads();
    float c0[NT][4] = {}, c1[NT][4] = {};
    // (through the array itself: the tables' places are then part of the load's address)
    auto word = [&](int table, uint32_t w, int byte) {
        const uint32_t at = ((byte == 0 ? w << 7 : w >> (8 * byte - 7)) & 0x7F80u) | static_cast<uint32_t>(lane * 4);
        return *reinterpret_cast<const uint32_t *>(smem_raw + table * LT_TABLE_BYTES + at);
    };
    auto use = [&](const uint32_t (&qa)[4], const uint32_t (&qb)[4], const uint4 (&y)[NT][4], int end) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t wa[4], wb[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                wa[e] = word(0, qa[q], e);
                wb[e] = word(1, qb[q], e);
            }
            if (eight(q) >= end) {                                    // (never in a whole piece) no level meets padding
#pragma unroll
                for (int e = 0; e < 4; ++e) wa[e] = wb[e] = 0u;
            }
#pragma unroll
            for (int o = 0; o < NT; ++o) {
                mma_m16n8k16<BF16>(c0[o], wa[0], wb[0], wa[1], wb[1], y[o][q].x, y[o][q].y);
                mma_m16n8k16<BF16>(c1[o], wa[2], wb[2], wa[3], wb[3], y[o][q].z, y[o][q].w);
            }
        }
    };
    for (int i = 0; i < whole; i += LT_AHEAD) {
#pragma unroll
        for (int d = 0; d < LT_AHEAD; ++d) {
            if (i + d >= whole) break;
            copy_async_wait<LT_AHEAD - 1>();
            uint32_t qa[4], qb[4];
            if (SPREAD) {
                __syncwarp();                                    // the other lanes' copies
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    qa[q] = ld_shared_4(word_at + d * LT_CODE_BYTES + 16 * q);
                    qb[q] = ld_shared_4(word_at + d * LT_CODE_BYTES + SECOND + 16 * q);
                }
            } else {
                const uint4 a = ld_shared_16(copy_to + d * LT_CODE_BYTES), b = ld_shared_16(copy_to + d * LT_CODE_BYTES + SECOND);
                qa[0] = a.x, qa[1] = a.y, qa[2] = a.z, qa[3] = a.w;
                qb[0] = b.x, qb[1] = b.y, qb[2] = b.z, qb[3] = b.w;
            }
            use(qa, qb, tokens[d % X_AHEAD], LT_K);
            if (SPREAD) __syncwarp();                            // all lanes have read
            fetch_codes(i + d + LT_AHEAD, d);
            fetch_tokens(i + d + X_AHEAD, tokens[d % X_AHEAD]);
        }
    }
    if (ragged) {
        uint32_t qa[4], qb[4];
        uint4 y[NT][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int k = full * LT_K + eight(q);
            const bool in = k < p.d_in;
            qa[q] = in ? ld_u32(ca + (k >> 1)) : 0u;
            qb[q] = in ? ld_u32(cb + (k >> 1)) : 0u;
#pragma unroll
            for (int o = 0; o < NT; ++o) y[o][q] = in && have[o] ? ld_u32x4(x[o] + k) : make_uint4(0u, 0u, 0u, 0u);
        }
        use(qa, qb, y, p.d_in - full * LT_K);
    }
    __syncthreads();                                             // the ring has been read: the sums take its place
    // c[0], c[1]: channel g, tokens 2 t, 2 t + 1; c[2], c[3]: channel g + 8
#pragma unroll
    for (int o = 0; o < NT; ++o)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[warp][o * LT_TOKENS + 2 * t + (e & 1)][g + (e >= 2 ? 8 : 0)] = c0[o][e] + c1[o][e];
    __syncthreads();
    const int token = tid / LT_CHANNELS, ch = tid % LT_CHANNELS;
    float z = 0.0f;
    if (tid < TOKENS * LT_CHANNELS) {
#pragma unroll
        for (int w = 0; w < LT_WARPS; ++w) z += sums[w][token][ch];
        mine[tid] = z;
    }
    if (ranks > 1) {
        cluster_sync_all();
        if (rank == 0 && tid < TOKENS * LT_CHANNELS) {
            for (int r = 1; r < ranks; ++r) z += ld_cluster_f32(map_to_cta(smem_u32(&mine[tid]), r));
        }
    }
    const int j = j0 + ch;
    if (rank == 0 && tid < TOKENS * LT_CHANNELS && token < p.n && j < p.d_out) {
        if (p.bias) z += half_value(ld_u16(p.bias + j), BF16);
        if (p.Z) p.Z[token * p.ld_z + j] = static_cast<uint16_t>(half_bits(z, BF16));
        float y[1] = {z};
        activate(y, p.act);
        if (p.residual) y[0] += half_value(ld_u16(p.residual + token * p.ld_r + j), BF16);
        p.out[token * p.ld_out + j] = static_cast<uint16_t>(half_bits(y[0], BF16));
    }
    if (ranks > 1) cluster_sync_all();                            // nobody leaves while its shared memory is read
}

// ------------------------------------------------------------------------------------------------ tensor cores
constexpr int LP_SLOT_BYTES = (CTA_ROWS / BOX_FEATURES) * BOX_BYTES;      // one operand block: 16 KB
constexpr int LP_HALVES = 2;                                              // token tiles of 256 that share a weight operand
constexpr int LP_STAGES = 4;
constexpr int LP_STAGE_BYTES = (1 + LP_HALVES) * LP_SLOT_BYTES;           // [weights | tokens | tokens]
constexpr int LP_CODE_KSTEPS = 4;                                         // k-steps whose codes come together
constexpr int LP_CODE_BYTES = LP_CODE_KSTEPS * CTA_ROWS * TILE_K / 2;     // 16 KB
constexpr int LP_CODE_SLOTS = 2;
constexpr int LP_LOOK_GROUPS = 2;                                         // of four warps; they take the k-steps in turn
constexpr int LP_LOOK_WARPS = 4 * LP_LOOK_GROUPS;
constexpr int LP_EPI_WARPS = 8;
constexpr int LP_THREADS = 32 * (4 + LP_LOOK_WARPS + LP_EPI_WARPS);
constexpr int LP_SMEM_BYTES = LP_STAGES * LP_STAGE_BYTES + LP_CODE_SLOTS * LP_CODE_BYTES + 1024;
constexpr int LP_MAX_SPLIT = 8;                                           // pairs of a cluster (sixteen CTAs)
constexpr int LG_STAGES = 4;                                              // gradient of the levels
constexpr int LG_SETS = 4;                                                // sums of a channel that are added to in turn
constexpr int LG_STAGE_BYTES = 2 * LP_SLOT_BYTES;                         // [dZ | tokens]
constexpr int LG_SMEM_BYTES = LG_STAGES * LG_STAGE_BYTES + LP_EPI_WARPS * LG_SETS * LIN_LEVELS * 32 * 4 + 1024;
constexpr int LG_THREADS = 32 * (4 + LP_EPI_WARPS);
constexpr int LG_CHUNK_KSTEPS = 16;                                       // 1024 tokens
constexpr int LP_ROW_BLOCK = 16;                                          // row tiles that are worked on beside each other

// K-major operand with the 128-byte swizzle: rows of 128 bytes (64 contraction indices), groups of 8 rows 1024 bytes apart; the next 16
// contraction indices are 32 bytes further.
__device__ __forceinline__ uint64_t umma_smem_desc_k_sw128(uint32_t smem_addr)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(1) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
// kind::f16 with fp32 accumulation, A and B both bf16 or both fp16.
__host__ __device__ constexpr uint32_t umma_idesc_16(uint32_t m, uint32_t n, bool bf16, bool a_mn, bool b_mn)
{
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((n >> 3) << 17) | ((m >> 4) << 24);
}

// umma_commit_pair where the pair's first CTA has rank `leader` in its cluster.
__device__ __forceinline__ void umma_commit_pair_at(uint32_t leader, uint32_t bar)
{
    const uint16_t mask = static_cast<uint16_t>(3u << leader);
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        ::"r"(bar), "h"(mask)
        : "memory");
}
__device__ __forceinline__ void st_shared_4(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void ld_cluster_f32x4(uint32_t addr, float (&v)[4])
{
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr) : "memory");
}

// One lane of a converged warp, always the same one.
__device__ __forceinline__ bool elect_one()
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}
// bounded_wait_hot for a whole warp, the same answer in all lanes.
__device__ __forceinline__ bool warp_wait_hot(uint32_t bar, uint32_t parity, const WaitCtx &w, uint32_t site, uint32_t unit)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    const uint64_t t0 = global_timer_ns();
    for (uint32_t spins = 1;; ++spins) {
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        if ((spins & 63u) == 0u && __any_sync(0xffffffffu, wait_gave_up(w, t0, site, unit))) return false;
    }
}

struct LinearUnit {
    int row0, tok0, halves;      // 256 rows of the weights' side, `halves` tiles of 256 tokens from tok0 on
};
// The it-th unit of a pair.  Tiles of 256 rows x 512 tokens: the first `doubles` of them whole, the others in two units.  Row tiles in
// blocks of LP_ROW_BLOCK, inside a block token tiles outermost: tiles worked on at the same time share few token tiles (2 bytes an
// element) and more row tiles (half a byte).
template <bool SPLIT>
__device__ __forceinline__ bool linear_unit(const LinearParams &p, int pair, int it, LinearUnit &u)
{
    if (SPLIT) {                 // one tile of at most 256 tokens a cluster
        const int tok = pair / p.row_tiles;
        u.row0 = (pair - tok * p.row_tiles) * TILE_M;
        u.tok0 = tok * TILE_N;
        u.halves = 1;
        return it == 0;
    }
    const int unit = it * p.pairs + pair;
    if (unit >= p.units) return false;
    const int over = unit - p.doubles, tile = over < 0 ? unit : p.doubles + (over >> 1);
    const int per = LP_ROW_BLOCK * p.tok_tiles, block = tile / per, rest = tile - block * per;
    const int left = p.row_tiles - block * LP_ROW_BLOCK, width = left < LP_ROW_BLOCK ? left : LP_ROW_BLOCK;
    const int tok = rest / width;
    u.row0 = (block * LP_ROW_BLOCK + rest - tok * width) * TILE_M;
    u.tok0 = tok * (LP_HALVES * TILE_N);
    u.halves = u.tok0 + TILE_N < p.n ? 2 : 1;
    if (over >= 0) {
        // (the second unit of a tile without a second half has nothing to do)
        if ((over & 1) != 0 && u.halves == 2) u.tok0 += TILE_N;
        u.halves = (over & 1) != 0 && u.halves == 1 ? 0 : 1;
    }
    return true;
}

// Forward (BACK false): D[channel][token] = sum_c W[channel][c] X[token][c], both operands with the contraction contiguous; a lookup thread
// owns a channel for the whole tile, its levels stay in registers.  Backward: D[c][token] = sum_j W[j][c] dZ[token][j]; the rows of
// the weight operand are contraction indices, a lookup thread owns 64 columns of one channel a k-step and reads that channel's levels
// a step ahead.  Codes come by TMA as well, those of four k-steps together: read by the lookup threads from global memory they cost
// 28 us of 313 (8192 x 4096 x 4096); with two k-steps a box 32 tokens of 28672 -> 8192 take 95 us instead of 88.  A looked-up
// operand serves two tiles of 256 tokens, the two accumulators that tensor memory holds: with one tile each, lookups and their stores
// were in the way of the tensor core (263 us, 221 with the lookups left out; now 182, 1.5 PFLOP/s).
// Rows of D are the lanes of tensor memory, so tokens (columns) come in any number without work for the weights' side.
//
// SPLIT: few tiles.  A cluster of `ranks` pairs works on one tile of 256 rows and up to 256 tokens, a share of the contraction each; the
// partial sums go to shared memory (where the ring was) and every pair joins a share of the tokens through distributed shared memory.
// 64 tokens of 4096 x 4096, 16 tiles: 53 us on as many pairs when this was built, 31 on twice as many; 18 now.
template <bool BACK, bool WIDE, bool SPLIT>
__global__ void __launch_bounds__(LP_THREADS, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapC, const LinearParams p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_codes[LP_CODE_SLOTS];       // this CTA's codes have come
    __shared__ __align__(8) uint64_t bar_codes_used[LP_CODE_SLOTS];  // the lookup warps have read them
    __shared__ __align__(8) uint64_t bar_full[LP_STAGES];     // first CTA: bytes of both CTAs + four lookup warps of both
    __shared__ __align__(8) uint64_t bar_empty[LP_STAGES];    // both CTAs: signalled by the MMA commits
    __shared__ __align__(8) uint64_t bar_acc_full[2];         // both CTAs, one per accumulator
    __shared__ __align__(8) uint64_t bar_acc_empty[2];        // first CTA, one per accumulator: 16 epilogue warps arrive
    __shared__ __align__(8) uint64_t bar_drain;
    __shared__ uint32_t tmem_base_smem;
    __shared__ volatile uint32_t abort_flag;

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);      // (the same for all lanes, and known to be)
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank() & 1u;             // in the pair
    const uint32_t leader = cluster_ctarank() - rank;         // the pair's first CTA in the cluster
    const int share = SPLIT ? static_cast<int>(leader >> 1) : 0;
    const int pair = static_cast<int>(blockIdx.x >> 1) / (SPLIT ? p.ranks : 1);
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, code_ring = ring + LP_STAGES * LP_STAGE_BYTES;
    const int kdim = BACK ? p.d_out : p.d_in, rows = BACK ? p.d_in : p.d_out;
    const int ksteps = (kdim + TILE_K - 1) / TILE_K;
    const int kfirst = SPLIT ? ksteps * share / p.ranks : 0, kblocks = SPLIT ? ksteps * (share + 1) / p.ranks - kfirst : ksteps;
    const int ntile = SPLIT ? p.ntile : TILE_N;               // columns of an accumulator, half of them from either CTA

    if (threadIdx.x == 0) {
        for (int s = 0; s < LP_CODE_SLOTS; ++s) {
            mbar_init(smem_u32(&bar_codes[s]), 1);
            mbar_init(smem_u32(&bar_codes_used[s]), LP_LOOK_WARPS);
        }
        for (int s = 0; s < LP_STAGES; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1 + 2 * 4);
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bar_acc_full[b]), 1);
            mbar_init(smem_u32(&bar_acc_empty[b]), 2 * LP_EPI_WARPS);
        }
        mbar_init(smem_u32(&bar_drain), 1);
        abort_flag = 0u;
        fence_mbar_init();
        prefetch_tensormap(&mapX);
        prefetch_tensormap(&mapC);
    }
    griddep_launch();
    if (warp == 2) {
        tmem_alloc(smem_u32(&tmem_base_smem), TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem_base = tmem_base_smem;
    const WaitCtx wc{&abort_flag, p.status, p.wait_budget_ns};
    griddep_wait();

    if (warp == 0 && lane == 0) {
        // ------------------------------------------------------------------ TMA producer (both CTAs): tokens
        int s = 0;
        uint32_t ph = 0;
        uint32_t issued = 0;
        bool ok = true;
        LinearUnit u;
        for (int it = 0; ok && linear_unit<SPLIT>(p, pair, it, u); ++it) {
            if (u.halves == 0) continue;
            const int b0 = u.tok0 + static_cast<int>(rank) * (ntile / 2), box_rows = SPLIT ? p.box_rows : TILE_K, boxes = (ntile / 2 + box_rows - 1) / box_rows;
            for (int kb = 0; kb < kblocks; ++kb) {
                if (!bounded_wait(smem_u32(&bar_empty[s]), ph ^ 1u, wc, 1u, it)) { ok = false; break; }
                const uint32_t full_local = smem_u32(&bar_full[s]);
                if (rank == 0) mbar_arrive_expect_tx(full_local, 2 * u.halves * boxes * box_rows * 128);      // both CTAs' bytes
                const uint32_t full = map_to_cta(full_local, leader);
                const uint32_t stage = ring + s * LP_STAGE_BYTES;
                for (int h = 0; h < u.halves; ++h)
                    for (int q = 0; q < boxes; ++q)
                        tma_load_3d_pair(stage + (1 + h) * LP_SLOT_BYTES + q * BOX_BYTES, &mapX, full, (kfirst + kb) * TILE_K, b0 + h * TILE_N + q * TILE_K,
                                         0);
                ++issued;
                if (++s == LP_STAGES) { s = 0; ph ^= 1u; }
            }
        }
        // Stay until every stage has been released again: the release is an arrival on this CTA's barriers,
        // which must not come after the CTA has gone.
        for (int q = 0; ok && issued != 0u && q < LP_STAGES; ++q) {
            if (!bounded_wait(smem_u32(&bar_empty[s]), ph ^ 1u, wc, 5u, 0u)) ok = false;
            if (++s == LP_STAGES) { s = 0; ph ^= 1u; }
        }
        if (!ok) spin_ns(1000000ull);
    } else if (warp == 1 && lane == 0) {
        // ------------------------------------------------------------------ TMA producer (both CTAs): codes
        int c = 0;
        uint32_t ph = 0;
        bool ok = true;
        LinearUnit u;
        for (int it = 0; ok && linear_unit<SPLIT>(p, pair, it, u); ++it) {
            if (u.halves == 0) continue;
            const int a0 = u.row0 + static_cast<int>(rank) * CTA_ROWS;
            for (int kb = 0; kb < kblocks; kb += LP_CODE_KSTEPS) {
                if (!bounded_wait(smem_u32(&bar_codes_used[c]), ph ^ 1u, wc, 7u, it)) { ok = false; break; }
                const uint32_t bar = smem_u32(&bar_codes[c]);
                mbar_arrive_expect_tx(bar, LP_CODE_BYTES);
                tma_load_3d(code_ring + c * LP_CODE_BYTES, &mapC, bar, (BACK ? a0 : (kfirst + kb) * TILE_K) >> 1, BACK ? (kfirst + kb) * TILE_K : a0,
                            0);
                if (++c == LP_CODE_SLOTS) { c = 0; ph ^= 1u; }
            }
        }
        if (!ok) spin_ns(1000000ull);
    } else if (warp == 3 && rank == 0) {
        // ------------------------------------------------------------------ MMA issuer (first CTA)
        // The whole warp walks the loop and one lane issues: loop counters and descriptors are then known to be the same for all lanes and live
        // in uniform registers, from which the instruction takes its operands.  In a branch of one lane they have to be moved there, and
        // the four products of a k-step took 384 clocks to issue.
        const bool elected = elect_one();
        const uint32_t idesc = umma_idesc_16(TILE_M, static_cast<uint32_t>(ntile), p.bf16 != 0, BACK, false);
        int s = 0;
        uint32_t ph = 0;
        uint32_t acc_ph = 0u;                           // bit b: phase of accumulator b
        int buf = 0;                                    // accumulator of a unit's first half
        bool ok = true;
        auto multiply = [&](int stage, int half, uint32_t d_tmem, bool first) {
            const uint32_t sa = ring + stage * LP_STAGE_BYTES, sb = sa + (1 + half) * LP_SLOT_BYTES;
            const uint64_t adesc = BACK ? umma_smem_desc_mn_sw128(sa, BOX_BYTES, 1024) : umma_smem_desc_k_sw128(sa);
            const uint64_t bdesc = umma_smem_desc_k_sw128(sb);
            constexpr uint64_t a_step = (BACK ? 16 * 128 : 32) >> 4, b_step = 32 >> 4;
            if (elected) {
                umma_bf16(d_tmem, adesc, bdesc, idesc, first ? 0u : 1u);
#pragma unroll
                for (int k16 = 1; k16 < TILE_K / 16; ++k16) umma_bf16(d_tmem, adesc + k16 * a_step, bdesc + k16 * b_step, idesc, 1u);
            }
        };
        auto acquire = [&](int b, int it) {
            if (!warp_wait_hot(smem_u32(&bar_acc_empty[b]), ((acc_ph >> b) & 1u) ^ 1u, wc, 2u, it)) return false;
            acc_ph ^= 1u << b;
            tc_fence_after_sync();
            return true;
        };
        LinearUnit u;
        for (int it = 0; ok && linear_unit<SPLIT>(p, pair, it, u); ++it) {
            if (u.halves == 0) continue;
            const uint32_t d0 = tmem_base + static_cast<uint32_t>(buf * TILE_N), d1 = tmem_base + static_cast<uint32_t>((buf ^ 1) * TILE_N);
            if (!acquire(buf, it)) { ok = false; break; }
            // While the epilogue still reads the second accumulator, the first half of the k-steps that fit the ring.
            int lead = 0;
            if (u.halves == 2) {
                lead = kblocks < LP_STAGES ? kblocks : LP_STAGES;
                int sl = s;
                uint32_t phl = ph;
                for (int kb = 0; kb < lead; ++kb) {
                    if (!warp_wait_hot(smem_u32(&bar_full[sl]), phl, wc, 3u, it)) { ok = false; break; }
                    tc_fence_after_sync();
                    multiply(sl, 0, d0, kb == 0);
                    if (++sl == LP_STAGES) { sl = 0; phl ^= 1u; }
                }
                if (!ok || !acquire(buf ^ 1, it)) { ok = false; break; }
            }
            for (int kb = 0; kb < kblocks; ++kb) {
                if (kb >= lead) {
                    if (!warp_wait_hot(smem_u32(&bar_full[s]), ph, wc, 3u, it)) { ok = false; break; }
                    tc_fence_after_sync();
                    multiply(s, 0, d0, kb == 0);
                }
                if (kb == kblocks - 1 && elected) umma_commit_pair_at(leader, smem_u32(&bar_acc_full[buf]));
                if (u.halves == 2) multiply(s, 1, d1, kb == 0);
                if (elected) umma_commit_pair_at(leader, smem_u32(&bar_empty[s]));
                if (++s == LP_STAGES) { s = 0; ph ^= 1u; }
            }
            if (!ok) break;
            if (u.halves == 2) {
                if (elected) umma_commit_pair_at(leader, smem_u32(&bar_acc_full[buf ^ 1]));
            } else {
                buf ^= 1;
            }
        }
        if (!ok && elected) {
            // Make sure no MMA is still writing TMEM when it is released.
            umma_commit_local(smem_u32(&bar_drain));
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(smem_u32(&bar_drain), 0u) && global_timer_ns() - t0 < 5000000ull) {}
        }
    } else if (warp >= 4 && warp < 4 + LP_LOOK_WARPS) {
        // ------------------------------------------------------------------ weight operand
        const int grp = (warp - 4) >> 2;                            // takes k-steps grp, grp + LP_LOOK_GROUPS, ... of the launch
        const int r = ((warp - 4) & 3) * 32 + lane;                 // forward: channel; backward: channel r % 64, columns 64 (r / 64) ..
        const uint32_t slot = BACK ? static_cast<uint32_t>((r >> 6) * BOX_BYTES + (r & 63) * 128) : static_cast<uint32_t>(r * 128);
        const uint32_t xor7 = static_cast<uint32_t>(r & 7);
        // Backward: the levels of channel r % 64 of k-step kb, asked for a k-step of the group ahead.
        struct Levels {
            uint4 a, b;
        };
        auto levels_at = [&](int j, Levels &t) {
            const uint4 *tb = reinterpret_cast<const uint4 *>(p.table + static_cast<size_t>(j < p.d_out ? j : 0) * LIN_LEVELS);
            t.a = ld_u32x4(tb);
            t.b = ld_u32x4(tb + 1);
        };
        // 16 bytes q of this thread's 32 bytes of codes for k-step kk of a slot, as the TMA's swizzle left them: forward rows of 128 bytes,
        // four k-steps; backward rows of 64 bytes, 64 rows a k-step.
        auto code_at = [&](int kk, int q) {
            if (BACK) {
                const uint32_t row = static_cast<uint32_t>(kk * TILE_K + (r & 63));
                return row * 64 + ((static_cast<uint32_t>((r >> 6) * 2 + q) ^ ((row >> 1) & 3u)) << 4);
            }
            return static_cast<uint32_t>(r * 128) + ((static_cast<uint32_t>(kk * 2 + q) ^ xor7) << 4);
        };
        // All lanes look, and only a warp that has to wait does so through lane 0: with that branch in every step (two a step, and the
        // votes around it) 32 tokens of 28672 -> 8192 took 133 us instead of 108, 8192 tokens of 4096 x 4096 224 instead of 206.
        auto wait = [&](uint32_t bar, uint32_t parity, uint32_t site, int it) {
            if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
            bool got = true;
            if (lane == 0) got = bounded_wait(bar, parity, wc, site, it);
            got = __any_sync(0xffffffffu, got && lane == 0);
            if (got) (void)mbar_try_wait(bar, parity);       // every lane observes the completed phase
            return got;
        };
        LevelPlanes lv;
        uint32_t done = 0, slots = 0;                               // k-steps and code slots of the tiles before
        bool ok = true;
        LinearUnit u;
        for (int it = 0; ok && linear_unit<SPLIT>(p, pair, it, u); ++it) {
            if (u.halves == 0) continue;
            Levels ahead{};
            levels_at(BACK ? (kfirst + grp) * TILE_K + (r & 63) : u.row0 + static_cast<int>(rank) * CTA_ROWS + r, ahead);
            if (!BACK) lv.set(ahead.a, ahead.b);
            for (int k4 = 0; ok && k4 < kblocks; k4 += LP_CODE_KSTEPS, ++slots) {
                const uint32_t c = slots % LP_CODE_SLOTS, codes = code_ring + c * LP_CODE_BYTES;
                if (!wait(smem_u32(&bar_codes[c]), (slots / LP_CODE_SLOTS) & 1u, 6u, it)) { ok = false; break; }
                uint4 code[LP_CODE_KSTEPS / LP_LOOK_GROUPS][2];
#pragma unroll
                for (int i = 0; i < LP_CODE_KSTEPS / LP_LOOK_GROUPS; ++i)
#pragma unroll
                    for (int q = 0; q < 2; ++q) code[i][q] = ld_shared_16(codes + code_at(LP_LOOK_GROUPS * i + grp, q));
#pragma unroll
                for (int i = 0; i < LP_CODE_KSTEPS / LP_LOOK_GROUPS; ++i) {
                    const int kb = k4 + LP_LOOK_GROUPS * i + grp;
                    if (kb >= kblocks) break;
                    if (BACK) {
                        lv.set(ahead.a, ahead.b);
                        levels_at((kfirst + kb + LP_LOOK_GROUPS) * TILE_K + (r & 63), ahead);
                    }
                    const uint32_t step = done + static_cast<uint32_t>(kb), s = step % LP_STAGES;
                    if (!wait(smem_u32(&bar_empty[s]), ((step / LP_STAGES) & 1u) ^ 1u, 8u, it)) { ok = false; break; }
                    const uint32_t base = ring + s * LP_STAGE_BYTES + slot;
                    const uint32_t w[8] = {code[i][0].x, code[i][0].y, code[i][0].z, code[i][0].w, code[i][1].x, code[i][1].y, code[i][1].z, code[i][1].w};
                    const int left = kdim - (kfirst + kb) * TILE_K;
                    if (left >= TILE_K) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) st_shared_16(base + ((static_cast<uint32_t>(e) ^ xor7) << 4), lv.look<WIDE>(w[e]));
                    } else {
                        // the last, ragged k-step: no level meets padding (infinite ones would make it NaN)
                        const int end = BACK ? ((r & 63) < left ? TILE_K : 0) : left;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            st_shared_16(base + ((static_cast<uint32_t>(e) ^ xor7) << 4), 8 * e < end ? lv.look<WIDE>(w[e]) : make_uint4(0u, 0u, 0u, 0u));
                    }
                    fence_proxy_async_smem();        // make the stores visible to the tensor core's reads
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&bar_full[s]), leader));
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_codes_used[c]));
            }
            done += static_cast<uint32_t>(kblocks);
        }
        (void)ok;
    } else if (warp >= 4 + LP_LOOK_WARPS) {
        // ------------------------------------------------------------------ epilogue: bias, activation, residual, rounding
        const int ew = warp - (4 + LP_LOOK_WARPS);      // 0..7; four consecutive warps cover the four lane quarters
        const int q = warp & 3;                         // TMEM lane quarter this warp may access
        const int part = ew >> 2;                       // which 128 of a half's 256 tokens
        const bool bf16 = p.bf16 != 0;
        // Lanes 2 i and 2 i + 1 exchange every other token, so that each holds two neighbouring rows of a token: 4-byte accesses.
        const int odd = lane & 1;
        uint32_t full_ph = 0u;                          // bit b: phase of accumulator b
        int buf = 0;
        bool ok = true;
        LinearUnit u;
        for (int it = 0; ok && linear_unit<SPLIT>(p, pair, it, u); ++it) {
            const int row = u.row0 + static_cast<int>(rank) * CTA_ROWS + q * 32 + lane;
            const bool in = row < rows;
            float bias = 0.0f;
            if (!BACK && p.bias && in) bias = half_value(ld_u16(p.bias + row), bf16);
            for (int h = 0; h < u.halves; ++h) {
                if (lane == 0) ok = bounded_wait(smem_u32(&bar_acc_full[buf]), (full_ph >> buf) & 1u, wc, 4u, it);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                (void)mbar_try_wait(smem_u32(&bar_acc_full[buf]), (full_ph >> buf) & 1u);     // every lane observes the completed phase
                full_ph ^= 1u << buf;
                tc_fence_after_sync();
                const uint32_t tmem_tile = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(buf * TILE_N + part * 128);
                // even lane: tokens 0, 2, ... of rows (row, row + 1); odd lane: tokens 1, 3, ... of rows (row - 1, row)
                const long long tok0 = u.tok0 + h * TILE_N + part * 128 + odd;
#pragma unroll 1
                for (int n0 = 0; n0 < 128; n0 += 32) {
                    uint32_t acc[32];
                    if (SPLIT && part * 128 + n0 >= ntile) break;
                    tmem_ld_32x32(tmem_tile + static_cast<uint32_t>(n0), acc);
                    tmem_ld_wait();
                    if (SPLIT) {
                        // partial sums [token][row], where the ring was: all its stages have been used
                        const uint32_t at = ring + static_cast<uint32_t>(((part * 128 + n0) * CTA_ROWS + q * 32 + lane) * 4);
#pragma unroll
                        for (int e = 0; e < 32; ++e) st_shared_4(at + e * CTA_ROWS * 4, acc[e]);
                        continue;
                    }
                    if (n0 == 96) {
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&bar_acc_empty[buf]), leader));
                    }
                    const int left = in ? p.n - static_cast<int>(tok0) - n0 : 0;       // this lane's tokens 0, 2, ... below it exist
                    float v[32];                         // pairs of rows of a token
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float a = __uint_as_float(acc[e]) + bias, b = __uint_as_float(acc[e + 1]) + bias;
                        const float other = __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
                        v[e] = odd ? other : a;
                        v[e + 1] = odd ? b : other;
                    }
                    if (!BACK) {
                        if (p.Z) {
                            uint16_t *z = p.Z + (tok0 + n0) * p.ld_z + (row - odd);
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                if (e < left) *reinterpret_cast<uint32_t *>(z) = half2_bits(v[e], v[e + 1], bf16);
                                z += 2 * p.ld_z;
                            }
                        }
                        uint32_t res[16];
                        if (p.residual) {
                            const uint16_t *at = p.residual + (tok0 + n0) * p.ld_r + (row - odd);
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                res[e] = 2 * e < left ? *reinterpret_cast<const uint32_t *>(at) : 0u;
                                at += 2 * p.ld_r;
                            }
                        }
                        activate(v, p.act);
                        if (p.residual) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const float2 t = half2_value(res[e], bf16);
                                v[2 * e] += t.x;
                                v[2 * e + 1] += t.y;
                            }
                        }
                    }
                    uint16_t *out = p.out + (tok0 + n0) * p.ld_out + (row - odd);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        if (e < left) *reinterpret_cast<uint32_t *>(out) = half2_bits(v[e], v[e + 1], bf16);
                        out += 2 * p.ld_out;
                    }
                }
                buf ^= 1;
            }
        }
    }

    if (SPLIT) {
        __syncwarp();
        cluster_sync_all();                             // all partial sums are there
        LinearUnit u;
        (void)linear_unit<SPLIT>(p, pair, 0, u);
        const bool bf16 = p.bf16 != 0;
        const int t0 = ntile * share / p.ranks, t1 = ntile * (share + 1) / p.ranks, row = u.row0 + static_cast<int>(rank) * CTA_ROWS + lane * 4;
        // a warp takes a token, a lane four rows (rows come in eights)
        for (int t = t0 + warp; t < t1; t += LP_THREADS / 32) {
            const long long token = u.tok0 + t;
            if (token >= p.n || row >= rows) continue;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            for (int r = 0; r < p.ranks; ++r) {
                float part[4];
                ld_cluster_f32x4(map_to_cta(ring + static_cast<uint32_t>((t * CTA_ROWS + lane * 4) * 4), 2 * r + rank), part);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += part[e];
            }
            if (!BACK) {
                if (p.bias) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += half_value(ld_u16(p.bias + row + e), bf16);
                }
                if (p.Z) *reinterpret_cast<uint2 *>(p.Z + token * p.ld_z + row) = make_uint2(half2_bits(v[0], v[1], bf16), half2_bits(v[2], v[3], bf16));
                activate(v, p.act);
                if (p.residual) {
                    const uint2 res = ld_u32x2(p.residual + token * p.ld_r + row);
                    const float2 a = half2_value(res.x, bf16), b = half2_value(res.y, bf16);
                    v[0] += a.x;
                    v[1] += a.y;
                    v[2] += b.x;
                    v[3] += b.y;
                }
            }
            *reinterpret_cast<uint2 *>(p.out + token * p.ld_out + row) = make_uint2(half2_bits(v[0], v[1], bf16), half2_bits(v[2], v[3], bf16));
        }
    }
    __syncwarp();
    tc_fence_before_sync();
    cluster_sync_all();
    if (warp == 2) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// ------------------------------------------------------------------------------------------------ backward pass
constexpr int LZ_COLUMNS = 256;           // columns of a block: 32 lanes x 8
constexpr int LZ_WARPS = 8;
constexpr int LZ_MIN_ROWS = 16;           // rows of a block, more where there would be too many blocks
constexpr int LZ_MAX_BLOCKS = 128;

// dz = dy act'(z), rounded to the activations' type, and per block of rows the column sums of the rounded values (db is their sum over
// the blocks, in the blocks' order).  Without an activation dZ is null: dy is dz, only the sums are formed.
__global__ void __launch_bounds__(32 * LZ_WARPS, 4) linear_dz_kernel(const uint16_t *dY, long long ld_dy, const uint16_t *Z, long long ld_z, int act, int bf16,
                                                                  int n, int d_out, int rows_per_block, uint16_t *dZ, long long ld_dz, float *col_sums)
{
    __shared__ float part[LZ_WARPS][LZ_COLUMNS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = static_cast<int>(blockIdx.x) * LZ_COLUMNS + lane * 8;
    const int r0 = static_cast<int>(blockIdx.y) * rows_per_block, r1 = min(r0 + rows_per_block, n);
    griddep_launch();
    griddep_wait();
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    // a warp's rows two at a time, all loads ahead of the first use
    for (int i0 = r0 + warp; col < d_out && i0 < r1; i0 += 2 * LZ_WARPS) {
        uint4 y[2], z[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = i0 + q * LZ_WARPS;
            y[q] = i < r1 ? ld_u32x4(dY + i * ld_dy + col) : make_uint4(0u, 0u, 0u, 0u);
            if (dZ) z[q] = i < r1 ? ld_u32x4(Z + i * ld_z + col) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = i0 + q * LZ_WARPS;
            if (i >= r1) break;
            uint32_t *yw = reinterpret_cast<uint32_t *>(&y[q]);
            if (dZ) {
                const uint32_t *zw = reinterpret_cast<const uint32_t *>(&z[q]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 a = half2_value(yw[e], bf16 != 0), b = half2_value(zw[e], bf16 != 0);
                    yw[e] = half2_bits(a.x * activation_slope(b.x, act), a.y * activation_slope(b.y, act), bf16 != 0);
                }
                *reinterpret_cast<uint4 *>(dZ + i * ld_dz + col) = y[q];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 kept = half2_value(yw[e], bf16 != 0);
                sum[2 * e] += kept.x;
                sum[2 * e + 1] += kept.y;
            }
        }
    }
    if (!col_sums) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) part[warp][lane * 8 + e] = sum[e];
    __syncthreads();
    const int c = static_cast<int>(blockIdx.x) * LZ_COLUMNS + static_cast<int>(threadIdx.x);
    if (c < d_out) {
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < LZ_WARPS; ++w) total += part[w][threadIdx.x];
        col_sums[static_cast<size_t>(blockIdx.y) * d_out + c] = total;
    }
}

struct LevelGradParams {
    const uint8_t *codes;
    int ld_codes;
    int n, d_in, d_out;
    int bf16;
    int ch_tiles, f_tiles, chunks;       // tiles of 256 channels and 256 features, pieces of the tokens
    int chunk_ksteps;                    // k-steps (of 64 tokens) of a piece
    int pairs;                           // at most as many as there are units
    float *partial;                      // [part of a channel tile][2][d_out][16]
    uint32_t *status;
    unsigned long long wait_budget_ns;
};

// Units (channel tile, feature tile, token piece), channel tiles outermost, are cut into equal runs, one a pair; a run ends up in two channel
// tiles where it crosses from one to the next.  The parts of a channel tile are numbered by the pairs that have them.
__host__ __device__ inline int level_grad_pair_of(long long unit, long long units, int pairs)
{
    return static_cast<int>(((unit + 1) * pairs - 1) / units);       // the last pair whose run starts at or before the unit
}
__host__ __device__ inline int level_grad_parts(int tile, int per_tile, int ch_tiles, int pairs)
{
    const long long units = static_cast<long long>(ch_tiles) * per_tile, first = static_cast<long long>(tile) * per_tile;
    return level_grad_pair_of(first + per_tile - 1, units, pairs) - level_grad_pair_of(first, units, pairs) + 1;
}

struct LevelGradUnit {
    int tile, part, f0, t0, t1;          // channel tile, part of it, first feature, k-steps [t0, t1)
    bool last;                           // of its part
};
struct LevelGradCursor {
    const LevelGradParams &p;
    int pair;
    long long unit, end, units;
    __device__ LevelGradCursor(const LevelGradParams &pp, int pr) : p(pp), pair(pr)
    {
        units = static_cast<long long>(p.ch_tiles) * p.f_tiles * p.chunks;
        unit = units * pair / p.pairs;
        end = units * (pair + 1) / p.pairs;
    }
    __device__ bool next(LevelGradUnit &u)
    {
        if (unit >= end) return false;
        const int per = p.f_tiles * p.chunks;
        u.tile = static_cast<int>(unit / per);
        const int rest = static_cast<int>(unit - static_cast<long long>(u.tile) * per), f = rest / p.chunks, c = rest - f * p.chunks;
        u.part = pair - level_grad_pair_of(static_cast<long long>(u.tile) * per, units, p.pairs);
        u.f0 = f * TILE_N;
        u.t0 = c * p.chunk_ksteps;
        u.t1 = min(u.t0 + p.chunk_ksteps, (p.n + TILE_K - 1) / TILE_K);
        ++unit;
        u.last = unit == end || rest == per - 1;
        return true;
    }
};

// Gradient of the levels: G[j][c] = sum_i dz_ij x_ic on the tensor cores (both operands by TMA, tokens as rows), never in memory: a lane
// of the epilogue is a channel and adds its entries to the sum of the level their code names, in shared memory.  A pair keeps these
// sums over its run of units and writes 16 numbers a channel at its end; the parts are added up in their order by linear_sum_kernel.
// The tokens are taken in pieces of at most 1024: the tensor cores' accumulation truncates, so that long runs drift.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LG_THREADS, 1)
linear_level_grad_kernel(const __grid_constant__ CUtensorMap mapG, const __grid_constant__ CUtensorMap mapX, const LevelGradParams p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[LG_STAGES];     // first CTA: bytes of both CTAs
    __shared__ __align__(8) uint64_t bar_empty[LG_STAGES];    // both CTAs: signalled by the MMA commits
    __shared__ __align__(8) uint64_t bar_acc_full[2];         // both CTAs, one per accumulator
    __shared__ __align__(8) uint64_t bar_acc_empty[2];        // first CTA, one per accumulator: 16 epilogue warps arrive
    __shared__ __align__(8) uint64_t bar_drain;
    __shared__ uint32_t tmem_base_smem;
    __shared__ volatile uint32_t abort_flag;

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = static_cast<int>(blockIdx.x >> 1);
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;

    if (threadIdx.x == 0) {
        for (int s = 0; s < LG_STAGES; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1);
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bar_acc_full[b]), 1);
            mbar_init(smem_u32(&bar_acc_empty[b]), 2 * LP_EPI_WARPS);
        }
        mbar_init(smem_u32(&bar_drain), 1);
        abort_flag = 0u;
        fence_mbar_init();
        prefetch_tensormap(&mapG);
        prefetch_tensormap(&mapX);
    }
    griddep_launch();
    if (warp == 2) {
        tmem_alloc(smem_u32(&tmem_base_smem), TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem_base = tmem_base_smem;
    const WaitCtx wc{&abort_flag, p.status, p.wait_budget_ns};
    griddep_wait();

    if (warp == 0 && lane == 0) {
        // ------------------------------------------------------------------ TMA producer (both CTAs)
        int s = 0;
        uint32_t ph = 0;
        uint32_t issued = 0;
        bool ok = true;
        LevelGradCursor cur(p, pair);
        LevelGradUnit u;
        while (ok && cur.next(u)) {
            const int a0 = u.tile * TILE_M + static_cast<int>(rank) * CTA_ROWS, b0 = u.f0 + static_cast<int>(rank) * CTA_ROWS;
            for (int kb = u.t0; kb < u.t1; ++kb) {
                if (!bounded_wait(smem_u32(&bar_empty[s]), ph ^ 1u, wc, 1u, u.tile)) { ok = false; break; }
                const uint32_t full_local = smem_u32(&bar_full[s]);
                if (rank == 0) mbar_arrive_expect_tx(full_local, 4 * LP_SLOT_BYTES);      // both CTAs' bytes
                const uint32_t full = map_to_cta(full_local, 0);
                const uint32_t stage = ring + s * LG_STAGE_BYTES;
#pragma unroll
                for (int q = 0; q < CTA_ROWS / BOX_FEATURES; ++q) {
                    tma_load_3d_pair(stage + q * BOX_BYTES, &mapG, full, a0 + q * BOX_FEATURES, kb * TILE_K, 0);
                    tma_load_3d_pair(stage + LP_SLOT_BYTES + q * BOX_BYTES, &mapX, full, b0 + q * BOX_FEATURES, kb * TILE_K, 0);
                }
                ++issued;
                if (++s == LG_STAGES) { s = 0; ph ^= 1u; }
            }
        }
        // Stay until every stage has been released again (see linear_pair_kernel).
        for (int q = 0; ok && issued != 0u && q < LG_STAGES; ++q) {
            if (!bounded_wait(smem_u32(&bar_empty[s]), ph ^ 1u, wc, 5u, 0u)) ok = false;
            if (++s == LG_STAGES) { s = 0; ph ^= 1u; }
        }
        if (!ok) spin_ns(1000000ull);
    } else if (warp == 3 && rank == 0) {
        // ------------------------------------------------------------------ MMA issuer (first CTA; see linear_pair_kernel)
        const bool elected = elect_one();
        const uint32_t idesc = umma_idesc_16(TILE_M, TILE_N, p.bf16 != 0, true, true);
        int s = 0;
        uint32_t ph = 0;
        uint32_t acc_ph = 0u;                           // bit b: phase of accumulator b
        int buf = 0;
        bool ok = true;
        LevelGradCursor cur(p, pair);
        LevelGradUnit u;
        while (ok && cur.next(u)) {
            if (!warp_wait_hot(smem_u32(&bar_acc_empty[buf]), ((acc_ph >> buf) & 1u) ^ 1u, wc, 2u, u.tile)) { ok = false; break; }
            tc_fence_after_sync();
            const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(buf * TILE_N);
            for (int kb = u.t0; kb < u.t1; ++kb) {
                if (!warp_wait_hot(smem_u32(&bar_full[s]), ph, wc, 3u, u.tile)) { ok = false; break; }
                tc_fence_after_sync();
                const uint32_t sa = ring + s * LG_STAGE_BYTES;
                const uint64_t adesc = umma_smem_desc_mn_sw128(sa, BOX_BYTES, 1024), bdesc = umma_smem_desc_mn_sw128(sa + LP_SLOT_BYTES, BOX_BYTES, 1024);
                constexpr uint64_t step = (16 * 128) >> 4;
                if (elected) {
                    umma_bf16(d_tmem, adesc, bdesc, idesc, kb != u.t0 ? 1u : 0u);
#pragma unroll
                    for (int k16 = 1; k16 < TILE_K / 16; ++k16) umma_bf16(d_tmem, adesc + k16 * step, bdesc + k16 * step, idesc, 1u);
                    umma_commit_pair(smem_u32(&bar_empty[s]));
                }
                if (++s == LG_STAGES) { s = 0; ph ^= 1u; }
            }
            if (!ok) break;
            if (elected) umma_commit_pair(smem_u32(&bar_acc_full[buf]));
            acc_ph ^= 1u << buf;
            buf ^= 1;
        }
        if (!ok && elected) {
            // Make sure no MMA is still writing TMEM when it is released.
            umma_commit_local(smem_u32(&bar_drain));
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(smem_u32(&bar_drain), 0u) && global_timer_ns() - t0 < 5000000ull) {}
        }
    } else if (warp >= 4 && warp < 4 + LP_EPI_WARPS) {
        // ------------------------------------------------------------------ epilogue: sums by level
        const int ew = warp - 4;                        // 0..7; four consecutive warps cover the four lane quarters
        const int q = warp & 3;                         // TMEM lane quarter this warp may access
        const int half = ew >> 2;                       // which 128 of the 256 features
        float *sums = reinterpret_cast<float *>(smem_raw + (ring - smem_u32(smem_raw)) + LG_STAGES * LG_STAGE_BYTES) +
                      ew * LG_SETS * LIN_LEVELS * 32 + lane;
#pragma unroll 16
        for (int l = 0; l < LG_SETS * LIN_LEVELS; ++l) sums[l * 32] = 0.0f;
        uint32_t full_ph = 0u;                          // bit b: phase of accumulator b
        int buf = 0;
        bool ok = true;
        LevelGradCursor cur(p, pair);
        LevelGradUnit u;
        while (ok && cur.next(u)) {
            const int j = u.tile * TILE_M + static_cast<int>(rank) * CTA_ROWS + q * 32 + lane;
            const bool have = j < p.d_out;
            const int byte0 = (u.f0 + half * 128) >> 1;
            const uint8_t *row = p.codes + static_cast<size_t>(have ? j : 0) * p.ld_codes;
            uint4 codes[4];                             // 128 features
#pragma unroll
            for (int x = 0; x < 4; ++x) codes[x] = byte0 + 16 * x < p.ld_codes ? ld_u32x4(row + byte0 + 16 * x) : make_uint4(0u, 0u, 0u, 0u);
            if (lane == 0) ok = bounded_wait(smem_u32(&bar_acc_full[buf]), (full_ph >> buf) & 1u, wc, 4u, u.tile);
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            (void)mbar_try_wait(smem_u32(&bar_acc_full[buf]), (full_ph >> buf) & 1u);     // every lane observes the completed phase
            full_ph ^= 1u << buf;
            tc_fence_after_sync();
            const uint32_t tmem_tile = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(buf * TILE_N + half * 128);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                uint32_t acc[32];
                tmem_ld_32x32(tmem_tile + static_cast<uint32_t>(32 * x), acc);
                tmem_ld_wait();
                if (x == 3) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&bar_acc_empty[buf]), 0));
                }
                const uint32_t w[4] = {codes[x].x, codes[x].y, codes[x].z, codes[x].w};
                // Features behind d_in have code 0 and a column of zeros, but NaN where dZ is infinite: nothing of them is added to level 0.
                const int left = p.d_in - (u.f0 + half * 128 + 32 * x);
                if (left < 32) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) acc[e] = e < left ? acc[e] : 0u;
                }
                // Four entries at a time, each into sums of its own, so that their loads, additions and stores overlap: one after the other 128 of
                // them took 4500 clocks.
#pragma unroll
                for (int e = 0; e < 32; e += LG_SETS) {
                    float v[LG_SETS];
                    int at[LG_SETS];
#pragma unroll
                    for (int k = 0; k < LG_SETS; ++k) {
                        at[k] = (k * LIN_LEVELS + static_cast<int>((w[(e + k) >> 3] >> (4 * ((e + k) & 7))) & 15u)) * 32;
                        v[k] = sums[at[k]];
                    }
#pragma unroll
                    for (int k = 0; k < LG_SETS; ++k) sums[at[k]] = v[k] + __uint_as_float(acc[e + k]);
                }
            }
            if (u.last) {
                float v[LIN_LEVELS];
#pragma unroll
                for (int l = 0; l < LIN_LEVELS; ++l) {
                    v[l] = 0.0f;
#pragma unroll
                    for (int k = 0; k < LG_SETS; ++k) {
                        v[l] += sums[(k * LIN_LEVELS + l) * 32];
                        sums[(k * LIN_LEVELS + l) * 32] = 0.0f;
                    }
                }
                if (have) {
                    float4 *out = reinterpret_cast<float4 *>(p.partial + ((static_cast<size_t>(u.part) * 2 + half) * p.d_out + j) * LIN_LEVELS);
#pragma unroll
                    for (int l = 0; l < LIN_LEVELS / 4; ++l) out[l] = make_float4(v[4 * l], v[4 * l + 1], v[4 * l + 2], v[4 * l + 3]);
                }
            }
            buf ^= 1;
        }
    }

    __syncwarp();
    tc_fence_before_sync();
    cluster_sync_all();
    if (warp == 2) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// Sums of the partial results in their order, in 64 bits: d_table [d_out][m] from the parts of each channel tile (a thread a cell), d_bias
// [d_out] from `blocks` rows of column sums (32 channels a CTA, every eighth row a thread).
__global__ void __launch_bounds__(256) linear_sum_kernel(const float *partial, int per_tile, int ch_tiles, int pairs, int d_out, int m, float *d_table,
                                                         const float *col_sums, int blocks, float *d_bias, int table_ctas)
{
    __shared__ double part[8][32];
    griddep_launch();
    griddep_wait();
    auto sum = [](const float *src, long long stride, int count) {
        double total = 0.0;
        for (int r0 = 0; r0 < count; r0 += 8) {
            float v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = r0 + q < count ? src[(r0 + q) * stride] : 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) total += static_cast<double>(v[q]);
        }
        return total;
    };
    if (static_cast<int>(blockIdx.x) < table_ctas) {
        const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x, cells = static_cast<long long>(d_out) * LIN_LEVELS;
        const int level = static_cast<int>(i % LIN_LEVELS);
        if (i >= cells || level >= m) return;
        const int count = 2 * level_grad_parts(static_cast<int>(i / (LIN_LEVELS * TILE_M)), per_tile, ch_tiles, pairs);
        d_table[i / LIN_LEVELS * m + level] = static_cast<float>(sum(partial + i, cells, count));
        return;
    }
    const int j = (static_cast<int>(blockIdx.x) - table_ctas) * 32 + static_cast<int>(threadIdx.x & 31), share = static_cast<int>(threadIdx.x >> 5);
    part[share][threadIdx.x & 31] =
        j < d_out && share < blocks ? sum(col_sums + static_cast<size_t>(share) * d_out + j, 8ll * d_out, (blocks - share + 7) / 8) : 0.0;
    __syncthreads();
    if (share == 0 && j < d_out) {
        double total = 0.0;
#pragma unroll
        for (int w = 0; w < 8; ++w) total += part[w][threadIdx.x];
        d_bias[j] = static_cast<float>(total);
    }
}

}  // namespace gq
