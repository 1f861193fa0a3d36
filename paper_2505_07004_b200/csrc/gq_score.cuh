// The end loss: log probabilities of given tokens, entropies, the highest alternatives, and the gradient in the logits.
//
//   m = max_j x_j,  L = log sum_j exp(x_j - m),  logp = x_t - m - L,
//   entropy = -sum_j p_j log p_j = L - sum_j exp(x_j - m) (x_j - m) / sum_j exp(x_j - m),
//   dx_j = dlogp (1[j = t] - p_j) - dent p_j (log p_j + entropy).
//
// Both kernels are bound by memory: the logits are read once (the gradient reads them a second time, because its dlogp is known
// only after the forward pass has ended, and writes as much).  All sums are fp32 and their order depends on nothing but the
// sizes, so results are the same from run to run.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>

#include "gq_kernels.cuh"

namespace gq {

constexpr int SC_WIDE = 512;             // threads of a CTA where rows are few and long
constexpr int SC_NARROW = 128;           // and where they are many or short
constexpr int SC_GROUPS = 64;            // groups of threads whose largest values bound the alternatives from below
constexpr int SC_MAX_TOP = 32;
constexpr int SC_MAX_CLUSTER = 8;
constexpr int SC_CANDIDATES = 256;       // entries that may reach the highest alternatives of a CTA's part of a row
constexpr int SC_GRAD_THREADS = 256;
constexpr int SC_GRAD_CHUNKS = 4;        // 16-byte chunks of a thread
constexpr float SC_LOG2E = 1.4426950408889634f;
constexpr float SC_LN2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Logits of one row as 16-byte chunks: `head` elements before the first 16-byte boundary, whole chunks, `tail` elements after.
template <int DT>
struct LogitRow {
    static constexpr int ELEM = DT == 2 ? 4 : 2;
    static constexpr int PER = 16 / ELEM;
    const uint8_t *base;
    int head, chunks, tail;
    __device__ LogitRow(const void *logits, long long row, long long ld, int vocab)
    {
        base = static_cast<const uint8_t *>(logits) + row * ld * ELEM;
        head = static_cast<int>((16u - (reinterpret_cast<uintptr_t>(base) & 15u)) & 15u) / ELEM;
        if (head > vocab) head = vocab;
        chunks = (vocab - head) / PER;
        tail = vocab - head - chunks * PER;
    }
    __device__ const uint4 *chunk(int c) const { return reinterpret_cast<const uint4 *>(base + head * ELEM) + c; }
    __device__ int first_of(int c) const { return head + c * PER; }
    __device__ float at(int j) const
    {
        if constexpr (DT == 2) {
            float v;
            asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(base + static_cast<size_t>(j) * 4) : "memory");
            return v;
        } else {
            const uint32_t h = ld_u16(base + static_cast<size_t>(j) * 2);
            if constexpr (DT == 0) return __uint_as_float(h << 16);
            return __half2float(__ushort_as_half(static_cast<unsigned short>(h)));
        }
    }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[PER])
    {
        if constexpr (DT == 0) {
            bf16x8_to_float(v, f);
        } else if constexpr (DT == 1) {
            const __half2 *h = reinterpret_cast<const __half2 *>(&v);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 t = __half22float2(h[e]);
                f[2 * e] = t.x;
                f[2 * e + 1] = t.y;
            }
        } else {
            f[0] = __uint_as_float(v.x);
            f[1] = __uint_as_float(v.y);
            f[2] = __uint_as_float(v.z);
            f[3] = __uint_as_float(v.w);
        }
    }
    // The largest number among four chunks and `top`.  16-bit types in pairs: half the instructions.
    static __device__ __forceinline__ float largest(const uint4 (&v)[4], float top)
    {
        if constexpr (DT == 2) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                top = fmaxf(fmaxf(fmaxf(top, __uint_as_float(v[q].x)), __uint_as_float(v[q].y)), fmaxf(__uint_as_float(v[q].z), __uint_as_float(v[q].w)));
            return top;
        } else {
            uint32_t m = pair_max(pair_max(v[0].x, v[0].y), pair_max(v[0].z, v[0].w));
#pragma unroll
            for (int q = 1; q < 4; ++q) m = pair_max(m, pair_max(pair_max(v[q].x, v[q].y), pair_max(v[q].z, v[q].w)));
            float lo, hi;
            if constexpr (DT == 0) {
                lo = __uint_as_float(m << 16);
                hi = __uint_as_float(m & 0xffff0000u);
            } else {
                const float2 t = __half22float2(*reinterpret_cast<const __half2 *>(&m));
                lo = t.x;
                hi = t.y;
            }
            return fmaxf(top, fmaxf(lo, hi));
        }
    }
    // Values below FLOOR are raised to it before the exponentials (0 times -inf would be NaN, and far from zero the exponents' rounding is
    // no longer small); NaNs stay.  That changes nothing where the largest value is above BORDER; elsewhere, and above CEILING, the sums are
    // formed from differences.
    static constexpr float FLOOR = DT == 1 ? -65504.0f : -200704.0f;
    static constexpr float BORDER = DT == 1 ? -6.0e4f : -1.0e5f, CEILING = 1.0e5f;
    static __device__ __forceinline__ uint32_t floored(uint32_t a)
    {
        uint32_t r;
        if constexpr (DT == 0) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(0xC844C844u));
        else if constexpr (DT == 1) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(0xFBFFFBFFu));      // the lowest finite one
        else asm("max.NaN.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(0xC8440000u));
        return r;
    }
    static __device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b)
    {
        uint32_t r;
        if constexpr (DT == 0) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
};

// Running softmax statistics: maximum, sum of 2^y and of y 2^y with y = (x - max) log2 e.  The maximum starts at the lowest
// finite value, so that x - max is never inf - inf for masked logits; a NaN makes s and t NaN.
struct SoftStats {
    float m, s, t;
    // Brings the sums to the maximum m2 >= m.
    __device__ __forceinline__ void raise(float m2)
    {
        const float y = fmaxf((m - m2) * SC_LOG2E, -1000.0f), f = exp2_fast(y);
        t = f * fmaf(y, s, t);
        s *= f;
        m = m2;
    }
    __device__ __forceinline__ void add(float x)
    {
        const float y = (x - m) * SC_LOG2E, e = exp2_fast(y);
        s += e;
        t = fmaf(e, fmaxf(y, -200.0f), t);       // 2^-200 is 0 already; -inf * 0 would not be
    }
    __device__ __forceinline__ void merge(SoftStats o)
    {
        const float m2 = fmaxf(m, o.m);
        raise(m2);
        o.raise(m2);
        s += o.s;
        t += o.t;
    }
};

// Order of the alternatives: larger value first, then smaller index.  The key of a value grows with it; both zeros have one
// key, a NaN is no alternative (entry 0).
__device__ __forceinline__ uint32_t value_key(float x)
{
    if (x != x) return 0u;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    if (k == 0u) return __uint_as_float(0x7fffffffu);
    return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ unsigned long long entry_of(float x, int j)
{
    const uint32_t key = value_key(x);
    return key == 0u ? 0ull : (static_cast<unsigned long long>(key) << 32) | static_cast<uint32_t>(~j);
}

// The highest of the warp's entries (0: none).
__device__ __forceinline__ unsigned long long warp_highest(unsigned long long v)
{
    const uint32_t key = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(v >> 32));
    const uint32_t low = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(v >> 32) == key ? static_cast<uint32_t>(v) : 0u);
    return (static_cast<unsigned long long>(key) << 32) | low;
}

// The whole CTA: the `top` highest of `count` <= SC_CANDIDATES entries, in order, into out (0 where there are no more).  An entry's place
// is the number of entries above it; all are different but for the zeros.
template <int THREADS>
__device__ __forceinline__ void block_select(const unsigned long long *entries, int count, int top, unsigned long long *out)
{
    const int tid = threadIdx.x;
    if (tid < top) out[tid] = 0ull;
    __syncthreads();
    for (int q = tid; q < count; q += THREADS) {
        const unsigned long long mine = entries[q];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < count; ++j) above += entries[j] > mine ? 1 : 0;
        if (mine != 0ull && above < top) out[above] = mine;
    }
    __syncthreads();
}

struct ScoreParams {
    const void *logits;
    long long ld;
    int vocab, top;
    const long long *targets;
    float *logp, *entropy, *stats, *top_logp;
    int32_t *top_ids;
};

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long ld_cluster_u64(uint32_t addr)
{
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}

// One cluster of `ranks` CTAs per row, each CTA a contiguous part of the row's chunks: one CTA where there are rows enough for
// all SMs, up to eight where there are few.  The first CTA joins the parts through distributed shared memory.
//
// Alternatives: a thread keeps its largest value, the four chunks that it came from, and the largest value of all others.  Of 64 groups of
// threads, the top-th largest of the groups' largest values is one that at least `top` entries reach, so every alternative is among
// the entries not below it, and those are with the threads whose largest is not below it: about `top` threads, of which the four
// chunks are read again (from L2), or all where the others reach it too.  What is found there, hardly more than `top` entries, is put
// in order by counting who is above whom.  Where ties make more than SC_CANDIDATES of them (a row of equal logits), the row is gone
// through once for each alternative instead.  4096 x 32000 bf16: 48 us, with 20 alternatives 81.
//
// Many rows or short ones: CTAs of 128 threads, so that an SM works on many rows at once and the joints between a row's end and the
// next one's beginning are covered; 4096 x 32000 bf16 took 80 us with 512 threads a row.
template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) token_logprobs_kernel(const ScoreParams p, int ranks)
{
    using Row = LogitRow<DT>;
    constexpr int WARPS = THREADS / 32;
    __shared__ float red[3][WARPS];
    __shared__ float part[3];                                     // this CTA's statistics
    __shared__ uint32_t best_of[THREADS];
    __shared__ uint32_t group_best[SC_GROUPS];
    __shared__ unsigned long long found[SC_CANDIDATES];
    __shared__ unsigned long long chosen[SC_MAX_TOP];             // this CTA's alternatives
    __shared__ int owners[WARPS][32];                             // first chunks to search
    __shared__ uint32_t floor_key;
    __shared__ int n_found;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row_index = static_cast<int>(blockIdx.x) / ranks, rank = static_cast<int>(blockIdx.x) - row_index * ranks;
    if (tid == 0) n_found = 0;
    griddep_launch();
    griddep_wait();
    const Row row(p.logits, row_index, p.ld, p.vocab);
    const int per = (row.chunks + ranks - 1) / ranks;
    const int c0 = min(rank * per, row.chunks), c1 = min(c0 + per, row.chunks);
    // elements outside whole chunks: at most 7 on either side, threads 0..7 of the first CTA and 8..15 of the last one
    int extra = -1;
    if (rank == 0 && tid < row.head) extra = tid;
    if (rank == ranks - 1 && tid >= 8 && tid - 8 < row.tail) extra = row.first_of(row.chunks) + tid - 8;

    // Sums of 2^y and y 2^y with y = x log2 e - c: one multiply-add and one exponential a value.  c is the largest value so far times log2 e,
    // rounded; what the rounding is off by is taken out once at the end.  (Subtracting the maximum first, and keeping -inf from the second
    // sum value by value: nine instructions a logit instead of seven and a half; the issue slots were 77 % busy.)
    const float minus_inf = __uint_as_float(0xff800000u);
    float best = minus_inf, c_ref = Row::FLOOR * SC_LOG2E, sum = 0.0f, weighted = 0.0f;
    // (for the alternatives: the four chunks with the largest value, and the largest value of all others)
    float second = minus_inf;
    int where = 0, batch = 0;
    auto take = [&](const uint4 (&v)[4]) {
        const float now = Row::largest(v, minus_inf);
        if (now <= best) {
            second = fmaxf(second, now);
        } else if (now > best) {
            second = best;
            where = batch;
            best = now;
            const float c2 = fmaxf(now, Row::FLOOR) * SC_LOG2E, d = fmaxf(c_ref - c2, -1000.0f), f = exp2_fast(d);
            weighted = f * fmaf(d, sum, weighted);
            sum *= f;
            c_ref = c2;
        }
        ++batch;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 w = make_uint4(Row::floored(v[q].x), Row::floored(v[q].y), Row::floored(v[q].z), Row::floored(v[q].w));
            float f[Row::PER];
            Row::unpack(w, f);
#pragma unroll
            for (int e = 0; e < Row::PER; ++e) {
                const float y = fmaf(f[e], SC_LOG2E, -c_ref), x2 = exp2_fast(y);
                sum += x2;
                weighted = fmaf(x2, y, weighted);
            }
        }
    };
    // Four chunks at a time, the next four on their way while four are added up.
    const int c_own = c0 + tid;
    int c = c_own;
    const int rounds = c < c1 ? (c1 - c + THREADS - 1) / THREADS : 0;       // chunks of this thread
    auto load = [&](uint4 (&v)[4]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = ld_once_16(row.chunk(c + q * THREADS));
        c += 4 * THREADS;
    };
    int left = rounds;
    if (left >= 4) {
        uint4 v[4], w[4];
        load(v);
        for (left -= 4; left >= 8; left -= 8) {
            load(w);
            take(v);
            load(v);
            take(w);
        }
        if (left >= 4) {
            load(w);
            take(v);
            take(w);
            left -= 4;
        } else {
            take(v);
        }
    }
    if (left > 0) {
        // the last ones; what is not there is -inf, which adds nothing
        const uint32_t none = DT == 0 ? 0xff80ff80u : DT == 1 ? 0xfc00fc00u : 0xff800000u;
        uint4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = q < left ? ld_once_16(row.chunk(c + q * THREADS)) : make_uint4(none, none, none, none);
        take(v);
    }
    const float best_chunk = best;
    SoftStats st{-FLT_MAX, 0.0f, 0.0f};
    if (best > Row::BORDER && best < Row::CEILING) {
        const float off = fmaf(best, SC_LOG2E, -c_ref), f = exp2_fast(-off);
        st = SoftStats{best, f * sum, f * fmaf(-off, sum, weighted)};
    } else if (best == minus_inf) {
        if (sum != sum) st.s = st.t = sum;                        // nothing but -inf and NaN
    } else {
        // far from zero: once more, from differences to the maximum
        for (int i = c_own; i < c1; i += THREADS) {
            float f[Row::PER];
            Row::unpack(ld_once_16(row.chunk(i)), f);
#pragma unroll
            for (int e = 0; e < Row::PER; ++e) {
                if (f[e] > st.m) st.raise(f[e]);
                st.add(f[e]);
            }
        }
    }
    if (extra >= 0) {
        const float x = row.at(extra);
        best = fmaxf(best, x);
        if (x > st.m) st.raise(x);
        st.add(x);
    }

    const bool alternatives = p.top > 0;
    if (alternatives) best_of[tid] = value_key(best);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        SoftStats o;
        o.m = __shfl_xor_sync(0xffffffffu, st.m, off);
        o.s = __shfl_xor_sync(0xffffffffu, st.s, off);
        o.t = __shfl_xor_sync(0xffffffffu, st.t, off);
        st.merge(o);
    }
    if (lane == 0) {
        red[0][warp] = st.m;
        red[1][warp] = st.s;
        red[2][warp] = st.t;
    }
    __syncthreads();
    if (warp == 0) {
        SoftStats w{-FLT_MAX, 0.0f, 0.0f};
        if (lane < WARPS) w = SoftStats{red[0][lane], red[1][lane], red[2][lane]};
#pragma unroll
        for (int off = WARPS / 2; off > 0; off >>= 1) {
            SoftStats o;
            o.m = __shfl_xor_sync(0xffffffffu, w.m, off);
            o.s = __shfl_xor_sync(0xffffffffu, w.s, off);
            o.t = __shfl_xor_sync(0xffffffffu, w.t, off);
            w.merge(o);
        }
        if (lane == 0) {
            part[0] = w.m;
            part[1] = w.s;
            part[2] = w.t;
        }
    } else if (warp == 1 && alternatives) {
        // the largest value that at least `top` of the groups reach
        uint32_t mine[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t k = 0u;
#pragma unroll
            for (int q = 0; q < THREADS / SC_GROUPS; ++q) k = max(k, best_of[h * 32 + lane + q * SC_GROUPS]);
            mine[h] = group_best[h * 32 + lane] = k;
        }
        __syncwarp();
        int reach[2] = {0, 0};
#pragma unroll 8
        for (int j = 0; j < SC_GROUPS; ++j) {
            const uint32_t k = group_best[j];
            reach[0] += k >= mine[0] ? 1 : 0;
            reach[1] += k >= mine[1] ? 1 : 0;
        }
        const uint32_t least = __reduce_max_sync(0xffffffffu, max(reach[0] >= p.top ? mine[0] : 0u, reach[1] >= p.top ? mine[1] : 0u));
        if (lane == 0) floor_key = least;
    }

    if (alternatives) {
        __syncthreads();
        const uint32_t least = floor_key;
        const float least_value = key_value(least);               // (at least -inf; a NaN is not above it)
        auto offer = [&](float x, int j) {
            if (x >= least_value) {
                const int at = atomicAdd(&n_found, 1);
                if (at < SC_CANDIDATES) found[at] = entry_of(x, j);
            }
        };
        // The chunks that may reach it, dealt to all lanes of the warp, four loads of a lane at a time: of a thread whose other chunks stay below
        // it the four with its largest value, of the others all.
        const bool hot = value_key(best_chunk) >= least, wide = hot && second >= least_value;
        const int each = (c1 - c0 + THREADS - 1) / THREADS;
        auto search = [&](uint32_t who, int count) {              // `count` chunks of each of these threads, from the one it has named
            const int items = __popc(who) * count;
            for (int i0 = lane; i0 < items; i0 += 128) {
                uint4 v[4];
                int at[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = i0 + 32 * q, o = i / count;
                    at[q] = i < items ? owners[warp][o] + (i - o * count) * THREADS : c1;
                    if (at[q] < c1) v[q] = ld_once_16(row.chunk(at[q]));
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (at[q] >= c1) continue;
                    float f[Row::PER];
                    Row::unpack(v[q], f);
#pragma unroll
                    for (int e = 0; e < Row::PER; ++e) offer(f[e], row.first_of(at[q]) + e);
                }
            }
            __syncwarp();
        };
        const uint32_t below = (1u << lane) - 1u, some = __ballot_sync(0xffffffffu, hot && !wide), all = __ballot_sync(0xffffffffu, wide);
        if (hot && !wide) owners[warp][__popc(some & below)] = c_own + 4 * where * THREADS;
        __syncwarp();
        search(some, 4);
        if (wide) owners[warp][__popc(all & below)] = c_own;
        __syncwarp();
        search(all, each);
        if (extra >= 0) offer(row.at(extra), extra);
        __syncthreads();
        const int count = n_found;
        if (count <= SC_CANDIDATES) {
            block_select<THREADS>(found, count, p.top, chosen);
        } else {
            // ties: the next in order, over the whole part, once per alternative
            unsigned long long last = ~0ull;
            for (int r = 0; r < p.top; ++r) {
                unsigned long long high = 0ull;
                auto look = [&](float x, int j) {
                    const unsigned long long v = entry_of(x, j);
                    if (v < last && v > high) high = v;
                };
                for (int i = c0 + tid; i < c1; i += THREADS) {
                    float f[Row::PER];
                    Row::unpack(ld_once_16(row.chunk(i)), f);
#pragma unroll
                    for (int e = 0; e < Row::PER; ++e) look(f[e], row.first_of(i) + e);
                }
                if (extra >= 0) look(row.at(extra), extra);
                high = warp_highest(high);
                __syncthreads();
                if (lane == 0) found[warp] = high;
                __syncthreads();
                for (int q = 0; q < WARPS; ++q) high = found[q] > high ? found[q] : high;
                last = high;
                if (tid == 0) chosen[r] = high;
            }
            __syncthreads();
        }
    }

    if (ranks > 1) cluster_sync_all();
    if (alternatives && ranks > 1 && rank == 0) {
        for (int i = tid; i < ranks * p.top; i += THREADS) {
            const int r = i / p.top;
            found[i] = ld_cluster_u64(map_to_cta(smem_u32(chosen), r) + 8u * static_cast<uint32_t>(i - r * p.top));
        }
        __syncthreads();
        block_select<THREADS>(found, ranks * p.top, p.top, chosen);
    }
    if (rank == 0 && warp == 0) {
        __syncwarp();
        SoftStats w{-FLT_MAX, 0.0f, 0.0f};
        if (lane < ranks) {
            const uint32_t at = ranks > 1 ? map_to_cta(smem_u32(part), lane) : smem_u32(part);
            w = SoftStats{ld_cluster_f32(at), ld_cluster_f32(at + 4), ld_cluster_f32(at + 8)};
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {             // every lane ends up with the row's
            SoftStats o;
            o.m = __shfl_xor_sync(0xffffffffu, w.m, off);
            o.s = __shfl_xor_sync(0xffffffffu, w.s, off);
            o.t = __shfl_xor_sync(0xffffffffu, w.t, off);
            w.merge(o);
        }
        // All logits -inf: nothing has been added up, and the maximum is -inf rather than where it started.
        const bool none = w.s == 0.0f;
        const float log_s = none ? 0.0f : logf(w.s);
        if (lane == 0) {
            const float m = none ? __uint_as_float(0xff800000u) : w.m;
            p.stats[2 * static_cast<size_t>(row_index)] = m;
            p.stats[2 * static_cast<size_t>(row_index) + 1] = log_s;
            p.entropy[row_index] = none ? 0.0f : fmaxf(log_s - SC_LN2 * (w.t / w.s), log_s - log_s);
            if (p.targets) {
                const long long t = p.targets[row_index];
                float lp = 0.0f;
                if (t >= 0 && t < p.vocab) lp = none ? m : (row.at(static_cast<int>(t)) - m) - log_s;
                p.logp[row_index] = lp;
            }
        }
        if (alternatives) {
            if (lane < p.top) {
                const unsigned long long v = chosen[lane];
                const float x = key_value(static_cast<uint32_t>(v >> 32));
                p.top_ids[static_cast<size_t>(row_index) * p.top + lane] = static_cast<int32_t>(~static_cast<uint32_t>(v));
                p.top_logp[static_cast<size_t>(row_index) * p.top + lane] = none ? __uint_as_float(0xff800000u) : (x - w.m) - log_s;
            }
        }
    }
    if (ranks > 1) cluster_sync_all();                         // nobody leaves while its shared memory is read
}

struct ScoreGradParams {
    const void *logits;
    long long ld;
    int vocab;
    const long long *targets;
    const float *stats, *entropy, *d_logp, *d_entropy;
    void *d_logits;
    long long ld_d;
};

__device__ __forceinline__ void st_once_16(void *p, const uint4 &v)
{
    asm volatile("st.global.cs.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Blocks (part of a row, row): SC_GRAD_CHUNKS chunks a thread, all loads ahead of the first use.  A row without weight (its token not
// counted, no entropy gradient) is set to zero without being read.
template <int DT, bool ENT>
__global__ void __launch_bounds__(SC_GRAD_THREADS) token_logprobs_grad_kernel(const ScoreGradParams p, int parts)
{
    using Row = LogitRow<DT>;
    constexpr int PER = Row::PER, ELEM = Row::ELEM;
    griddep_launch();
    griddep_wait();
    const int row_index = static_cast<int>(blockIdx.x / static_cast<unsigned>(parts));
    const int piece = static_cast<int>(blockIdx.x - static_cast<unsigned>(row_index) * static_cast<unsigned>(parts));
    const int tid = threadIdx.x;
    const Row row(p.logits, row_index, p.ld, p.vocab);
    uint8_t *out = static_cast<uint8_t *>(p.d_logits) + static_cast<long long>(row_index) * p.ld_d * ELEM;
    const bool same_phase = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.base)) & 15u) == 0;
    int target = -1;
    float w = 0.0f;
    if (p.targets) {
        const long long t = p.targets[row_index];
        if (t >= 0 && t < p.vocab) {
            target = static_cast<int>(t);
            w = p.d_logp[row_index];
        }
    }
    const float m = p.stats[2 * static_cast<size_t>(row_index)], log_s = p.stats[2 * static_cast<size_t>(row_index) + 1];
    float h = 0.0f, ent = 0.0f;
    if (ENT) {
        h = p.d_entropy[row_index];
        ent = p.entropy[row_index];
    }
    const bool zero = (w == 0.0f && h == 0.0f) || m == __uint_as_float(0xff800000u);
    auto grad = [&](float x, int j) {
        const float logp = (x - m) - log_s, prob = exp2_fast(logp * SC_LOG2E);
        float g = (j == target ? w : 0.0f) - w * prob;
        if (ENT) g -= h * prob * (fmaxf(logp, -200.0f) + ent);
        return g;
    };
    auto put = [&](int j, float g) {
        if constexpr (DT == 0) reinterpret_cast<__nv_bfloat16 *>(out)[j] = __float2bfloat16_rn(g);
        else if constexpr (DT == 1) reinterpret_cast<__half *>(out)[j] = __float2half_rn(g);
        else reinterpret_cast<float *>(out)[j] = g;
    };
    const int first = piece * SC_GRAD_THREADS * SC_GRAD_CHUNKS + tid;
    uint4 v[SC_GRAD_CHUNKS];
#pragma unroll
    for (int q = 0; q < SC_GRAD_CHUNKS; ++q) {
        const int c = first + q * SC_GRAD_THREADS;
        v[q] = (!zero && c < row.chunks) ? ld_once_16(row.chunk(c)) : make_uint4(0u, 0u, 0u, 0u);
    }
    if (piece == 0 && tid < row.head) put(tid, zero ? 0.0f : grad(row.at(tid), tid));
    if (piece == 0 && tid >= 32 && tid - 32 < row.tail) {
        const int j = row.first_of(row.chunks) + tid - 32;
        put(j, zero ? 0.0f : grad(row.at(j), j));
    }
#pragma unroll
    for (int q = 0; q < SC_GRAD_CHUNKS; ++q) {
        const int c = first + q * SC_GRAD_THREADS;
        if (c >= row.chunks) break;
        const int j0 = row.first_of(c);
        float f[PER];
        Row::unpack(v[q], f);
#pragma unroll
        for (int e = 0; e < PER; ++e) f[e] = zero ? 0.0f : grad(f[e], j0 + e);
        if (same_phase) {
            uint4 o;
            if constexpr (DT == 0) {
                o = float_to_bf16x8(f);
            } else if constexpr (DT == 1) {
                __half2 *hh = reinterpret_cast<__half2 *>(&o);
#pragma unroll
                for (int e = 0; e < 4; ++e) hh[e] = __floats2half2_rn(f[2 * e], f[2 * e + 1]);
            } else {
                o = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            }
            st_once_16(out + static_cast<size_t>(j0) * ELEM, o);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) put(j0 + e, f[e]);
        }
    }
}

}  // namespace gq
