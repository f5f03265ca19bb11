// Scores of given tokens: log-probability of the token of every row, entropy of the row's distribution, and its likeliest ids.
//
//   lse = log sum_v exp(l_v),   logprob = l_tok - lse,   entropy = lse - sum_v p_v l_v,   p_v = exp(l_v - lse)
//
// One pass over the logits, kept as three running numbers relative to a reference m:  A = sum 2^t_v,  B = sum 2^t_v t_v,
// t_v = (l_v - m) log2 e.  Moving the reference by d (t' = t + d) turns them into 2^d A and 2^d (B + d A), so threads' and CTAs' parts are
// joined in any order; at the end m is the row's maximum, lse = m + ln A, entropy = ln A - ln 2 * B / A.  A thread follows the
// maximum of its own logits with a slack of 1 (e^1 at most in any term: a larger slack saves steps but then ln A and B / A are large and
// cancel).  A is the sum of two fp32 numbers beyond 16 bytes of logits: of a row that is nearly certain, ln A is what its maximum
// leaves over, and every addition behind that 1 would round it to 2^-24.  (fp64 sums instead: their conversions run on the
// special-function unit, which the exponentials keep busy already; 1216 rows of 151936 took 75 us with them.)
//
// Logits below kFloor = -1e30 are taken as that, so that -inf and the type's lowest value (masked ids) need no care in the inner loop: beside any
// logit above them they are 0 either way.  A row that has none above, or logits so large that differences overflow, is gone through again,
// logit by logit (row_exactly).
//
// The n likeliest ids, by value and lowest id first, come out of the same pass: every thread keeps the largest of its logits, the
// n-th largest of these maxima is a bound that n logits of the CTA's share reach for certain, and only the logits of the threads whose
// maximum reaches it, n of them where no two are equal, are looked through again (out of L2).  What reaches the bound is ranked by counting.  The
// order (value, id) is strict, so the outcome does not depend on which candidate was found first.
//
// Bound by memory: 2 or 4 bytes a logit, six instructions and one ex2 each.  A row goes to a cluster of 1, 2, 4 or 8 CTAs; the CTAs' parts
// meet in the first one's shared memory, so there is no scratch and nothing for calls to share.
#include "fdd_internal.h"
#include "tc_ptx.cuh"

#include <math_constants.h>

namespace {

constexpr int kScoreThreads = 256;
constexpr int kScoreBatch = 4;                        // 16-byte pieces a thread takes at a time
constexpr int kKeep = 256;                            // candidates that may stay in the list between two rounds
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFloor = -1e30f, kNearFloor = -1e29f, kHuge = 1e38f;
constexpr float kSlack = 1.0f;

struct __align__(16) Part {
    float m;
    float a, a_low;                                   // A = a + a_low
    float b;
};

// a + a_low + x, with what the addition to a rounds off in a_low (Knuth's two-sum: exact for any two numbers).
__device__ __forceinline__ void add_to(float& a, float& a_low, float x) {
    const float s = a + x, t = s - a;
    a_low += (a - (s - t)) + (x - t);
    a = s;
}

// Move the reference of p by d <= 0 (in units of log 2).
__device__ __forceinline__ void rebase(Part& p, float d) {
    const float f = exp2f(d), a = p.a * f;
    p.b = f > 0.0f ? f * fmaf(d, p.a, p.b) : 0.0f;
    p.a_low = fmaf(p.a_low, f, fmaf(p.a, f, -a));
    p.a = a;
}

// Values in the order of unsigned numbers: NaN counts as -inf, -0 as 0; nothing is 0.
__device__ __forceinline__ uint32_t order_of(float v) {
    v = v == v ? v + 0.0f : -CUDART_INF_F;
    const uint32_t u = __float_as_uint(v);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float((order & 0x80000000u) ? (order & 0x7FFFFFFFu) : ~order); }
// Order of candidates: larger value first, then lower id.  0 is below every candidate.
__device__ __forceinline__ unsigned long long key_of(float v, int id) {
    return (static_cast<unsigned long long>(order_of(v)) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(id));
}
__device__ __forceinline__ float key_value(unsigned long long k) { return value_of(static_cast<uint32_t>(k >> 32)); }
__device__ __forceinline__ int key_id(unsigned long long k) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(k)); }

// (not through the read-only path: the kernel ahead may be writing the logits when this one starts)
__device__ __forceinline__ uint4 load_piece(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <typename T> struct Piece;                  // 16 bytes of logits
template <> struct Piece<__nv_bfloat16> {
    static constexpr int kN = 8;
    static constexpr uint32_t kNone = 0xFF80FF80u;    // -inf twice
    static __device__ __forceinline__ uint32_t at_least_floor(uint32_t w) {          // NaN stays NaN
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0xF14AF14Au));       // bf16 nearest -1e30
        return r;
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {         // the number of the two, if one is NaN
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float max_of(uint32_t a) { return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u)); }
    static __device__ __forceinline__ void unpack(const uint4& q, float (&x)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};
template <> struct Piece<float> {
    static constexpr int kN = 4;
    static constexpr uint32_t kNone = 0xFF800000u;
    static __device__ __forceinline__ uint32_t at_least_floor(uint32_t w) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(w)), "f"(kFloor));
        return __float_as_uint(r);
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    static __device__ __forceinline__ float max_of(uint32_t a) { return __uint_as_float(a); }
    static __device__ __forceinline__ void unpack(const uint4& q, float (&x)[4]) {
        x[0] = __uint_as_float(q.x); x[1] = __uint_as_float(q.y); x[2] = __uint_as_float(q.z); x[3] = __uint_as_float(q.w);
    }
    static __device__ __forceinline__ float value(const float* p) { return *p; }
};

// One logit more.
__device__ __forceinline__ void take_one(Part& p, float x) {
    if (x > p.m) {
        rebase(p, (p.m - x) * kLog2e);
        p.m = x;
    }
    float t = (x - p.m) * kLog2e;
    asm("max.NaN.f32 %0, %0, 0fC3160000;" : "+f"(t)); // (-inf: 2^-150 is 0 and 0 * t is 0; NaN stays)
    const float e = tc::ex2(t);
    add_to(p.a, p.a_low, e);
    p.b += e * t;
}

__device__ __forceinline__ float floored(float x) { return x < kFloor ? kFloor : x; }      // (NaN stays NaN)

// How many of n entries in shared memory are larger than k; at least `most` means that or more.  (Eight reads are on their way at a time: one
// by one, each would wait for its own.)
template <typename K>
__device__ __forceinline__ int larger(const K* keys, int n, K k, int most) {
    int more = 0;
    for (int i0 = 0; i0 < n && more < most; i0 += 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const K other = keys[min(i0 + i, n - 1)];
            more += i0 + i < n && other > k ? 1 : 0;
        }
    }
    return more;
}

// The parts of LANES neighbouring lanes, joined in every one of them: the maximum first, so that each part is moved once.
template <int LANES>
__device__ __forceinline__ Part join_lanes(Part p) {
    float m = p.m;
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
    rebase(p, (p.m - m) * kLog2e);
    p.m = m;
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) {
        const float a = __shfl_xor_sync(0xFFFFFFFFu, p.a, off);
        p.a_low += __shfl_xor_sync(0xFFFFFFFFu, p.a_low, off);
        add_to(p.a, p.a_low, a);
        p.b += __shfl_xor_sync(0xFFFFFFFFu, p.b, off);
    }
    return p;
}
// Of the CTA's warps, one part each; for a whole warp.
__device__ __forceinline__ Part join_cta(const Part* parts) {
    static_assert(kScoreThreads / 32 == 8, "eight parts");
    return join_lanes<8>(parts[threadIdx.x & 7]);
}

// One row with nothing above the floor, or with huge logits: by one CTA, logit by logit.
template <typename T>
__device__ __noinline__ Part row_exactly(const T* row, int vocab, Part* parts) {
    Part p = {-3.4028234663852886e38f, 0.0f, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < vocab; i += kScoreThreads) take_one(p, Piece<T>::value(row + i));
    p = join_lanes<32>(p);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = p;
    __syncthreads();
    return join_cta(parts);
}

template <typename T>
__global__ void __launch_bounds__(kScoreThreads, 4) score_kernel(const __grid_constant__ ScoreArgs a) {
    constexpr int kN = Piece<T>::kN;
    constexpr int kCap = kKeep + kScoreThreads * kN;
    __shared__ unsigned long long list[kCap];         // candidates
    __shared__ unsigned long long best[kScoreMaxTop]; // the likeliest, in order
    __shared__ unsigned long long merged[kScoreMaxTop], bound_s;
    __shared__ uint32_t group_max[32], near_max[kScoreThreads], least_s;
    __shared__ unsigned short looks[kScoreThreads];   // threads whose logits are looked through again
    __shared__ Part parts[kScoreThreads / 32], whole;
    __shared__ int n_list, n_near, n_looks;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cluster = a.cluster, rank = static_cast<int>(blockIdx.x) % cluster;
    const long long r = blockIdx.x / cluster;
    tc::grid_dependency_wait();          // (launched for an early start behind the kernel ahead of it)

    const int token = a.tokens[r];
    const int top = a.n_top;
    if (token < 0 || token >= a.vocab || (a.state != nullptr && a.state[r] != FDD_COMMITTED)) {
        // nothing to score (every CTA of the cluster sees the same)
        if (rank == 0) {
            if (tid == 0) {
                a.logprob[r] = CUDART_NAN_F;
                if (a.entropy != nullptr) a.entropy[r] = CUDART_NAN_F;
            }
            if (tid < top) {
                a.top_ids[r * top + tid] = -1;
                a.top_logprobs[r * top + tid] = CUDART_NAN_F;
            }
        }
        return;
    }

    // The row: `head` logits, 16-byte pieces, and the rest from `tail_at` on.  This CTA takes pieces [first, first + pieces): thread t the
    // pieces t, t + kScoreThreads, ...; the first CTA's thread 0 the head as well, the last one's last thread the tail.
    const T* const row = static_cast<const T*>(a.logits) + r * static_cast<long long>(a.vocab);
    const int head = min(a.vocab, static_cast<int>(((16u - (reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / sizeof(T)));
    const int middle = (a.vocab - head) / kN;
    const int first = static_cast<int>(static_cast<long long>(middle) * rank / cluster);
    const int pieces = static_cast<int>(static_cast<long long>(middle) * (rank + 1) / cluster) - first;
    const int tail_at = head + middle * kN;
    const int n_head = rank == 0 ? head : 0, n_tail = rank == cluster - 1 ? a.vocab - tail_at : 0;
    const int first_id = head + first * kN;           // of piece 0
    const uint4* const mid = reinterpret_cast<const uint4*>(row + first_id);

    // ---- the pass
    Part p = {kFloor, 0.0f, 0.0f, 0.0f};
    float top_value = -CUDART_INF_F;                  // the largest logit of this thread's pieces
    constexpr int kPerBatch = kScoreBatch * kScoreThreads;
    const int batches = (pieces - tid + kPerBatch - 1) / kPerBatch;          // (0 or below: no piece of its own)
    auto fetch = [&](int b, uint4 (&q)[kScoreBatch]) {
        if ((b + 1) * kPerBatch <= pieces) {           // (most)
#pragma unroll
            for (int i = 0; i < kScoreBatch; ++i) q[i] = load_piece(mid + b * kPerBatch + i * kScoreThreads + tid);
            return;
        }
#pragma unroll
        for (int i = 0; i < kScoreBatch; ++i) {
            const int at = b * kPerBatch + i * kScoreThreads + tid;
            q[i] = make_uint4(Piece<T>::kNone, Piece<T>::kNone, Piece<T>::kNone, Piece<T>::kNone);
            if (at < pieces) q[i] = load_piece(mid + at);
        }
    };
    uint4 next[kScoreBatch];
    if (batches > 0) fetch(0, next);
    for (int b = 0; b < batches; ++b) {
        uint4 q[kScoreBatch];
#pragma unroll
        for (int i = 0; i < kScoreBatch; ++i) q[i] = next[i];
        if (b + 1 < batches) fetch(b + 1, next);
        uint32_t most = Piece<T>::kNone;
#pragma unroll
        for (int i = 0; i < kScoreBatch; ++i)
            most = Piece<T>::max2(most, Piece<T>::max2(Piece<T>::max2(q[i].x, q[i].y), Piece<T>::max2(q[i].z, q[i].w)));
        const float vm = Piece<T>::max_of(most);
        top_value = fmaxf(vm, top_value);
        if (vm > p.m + kSlack) {
            rebase(p, (p.m - vm) * kLog2e);
            p.m = vm;
        }
        const uint64_t nm = tc::pack2(-p.m, -p.m), c = tc::pack2(kLog2e, kLog2e);
        uint64_t b2 = 0ull;
#pragma unroll
        for (int i = 0; i < kScoreBatch; ++i) {
            float x[kN];
            Piece<T>::unpack(make_uint4(Piece<T>::at_least_floor(q[i].x), Piece<T>::at_least_floor(q[i].y),
                                        Piece<T>::at_least_floor(q[i].z), Piece<T>::at_least_floor(q[i].w)), x);
            uint64_t a2 = 0ull;
#pragma unroll
            for (int k = 0; k < kN; k += 2) {
                const uint64_t t2 = tc::fma2(tc::add2(tc::pack2(x[k], x[k + 1]), nm), c, 0ull);
                float t0, t1;
                tc::unpack2(t2, t0, t1);
                const uint64_t e2 = tc::pack2(tc::ex2(t0), tc::ex2(t1));
                a2 = tc::add2(a2, e2);
                b2 = tc::fma2(e2, t2, b2);
            }
            float u, v;
            tc::unpack2(a2, u, v);
            add_to(p.a, p.a_low, u + v);
        }
        float u, v;
        tc::unpack2(b2, u, v);
        p.b += u + v;
    }
    // the reference becomes the exact maximum where that is a number (so that A is 1 + the rest)
    if (top_value > p.m && top_value < CUDART_INF_F) {
        rebase(p, (p.m - top_value) * kLog2e);
        p.m = top_value;
    }
    if (tid == 0)
        for (int i = 0; i < n_head; ++i) take_one(p, floored(Piece<T>::value(row + i)));
    if (tid == kScoreThreads - 1)
        for (int i = 0; i < n_tail; ++i) take_one(p, floored(Piece<T>::value(row + tail_at + i)));
    p = join_lanes<32>(p);
    if (lane == 0) parts[warp] = p;

    // ---- the likeliest of this CTA's share
    const uint32_t mine = batches > 0 ? order_of(top_value) : 0u;
    if (top > 0) {
        uint32_t g = mine;
#pragma unroll
        for (int off = 4; off > 0; off >>= 1) g = max(g, __shfl_xor_sync(0xFFFFFFFFu, g, off));
        if ((tid & 7) == 0) group_max[tid >> 3] = g;
        if (tid == 0) { n_list = 0; n_near = 0; n_looks = 0; least_s = 0xFFFFFFFFu; bound_s = 0ull; }
        if (tid < kScoreMaxTop) best[tid] = 0;
    }
    __syncthreads();
    if (warp == 0) {
        const Part w = join_cta(parts);
        if (lane == 0) whole = w;
    }
    if (top > 0) {
        // first the top-th largest of the maxima of 32 groups of eight threads: a bound that few threads reach, ...
        // (the smallest that has fewer than `top` above it; 0 where that many groups have no logits)
        const uint32_t own = group_max[lane];
        const uint32_t coarse = __reduce_min_sync(0xFFFFFFFFu, larger(group_max, 32, own, 32) < top ? own : 0xFFFFFFFFu);
        const bool near = mine >= coarse && mine != 0u;
        if (near) near_max[atomicAdd(&n_near, 1)] = mine;
        __syncthreads();
        // ... then the top-th largest of the maxima of these, and the threads that reach it
        if (near && larger(near_max, n_near, mine, top) < top) atomicMin(&least_s, mine);
        __syncthreads();
        const uint32_t least = n_near < top ? 0u : least_s;            // (fewer threads than that: every logit is a candidate)
        if (mine != 0u && mine >= least) looks[atomicAdd(&n_looks, 1)] = static_cast<unsigned short>(tid);
        __syncthreads();
        float bound_value = least != 0u ? value_of(least) : -CUDART_INF_F;
        unsigned long long bound = 0ull;
        auto candidate = [&](float x, int id) {
            if (x < bound_value) return;              // (most; NaN counts as -inf)
            const unsigned long long k = key_of(x, id);
            if (k < bound) return;
            const int slot = atomicAdd(&n_list, 1);
            if (slot < kCap) list[slot] = k;
        };
        auto rank_list = [&]() {                      // the `top` largest of the list into best[], in order
            const int n = n_list;
            for (int c = tid; c < n; c += kScoreThreads) {
                const unsigned long long k = list[c];
                const int more = larger(list, n, k, top);
                if (more < top) best[more] = k;
            }
            __syncthreads();
        };
        const int turns = (pieces + kScoreThreads - 1) / kScoreThreads;
        auto look_at = [&](const uint4& q, int piece) {
            // (its largest; NaN if there is nothing else)
            if (Piece<T>::max_of(Piece<T>::max2(Piece<T>::max2(q.x, q.y), Piece<T>::max2(q.z, q.w))) < bound_value) return;
            float x[kN];
            Piece<T>::unpack(q, x);
#pragma unroll
            for (int k = 0; k < kN; ++k) candidate(x[k], first_id + piece * kN + k);
        };
        // what lies outside the pieces is looked through in any case
        auto look_outside = [&]() {
            if (tid < n_head) candidate(Piece<T>::value(row + tid), tid);
            if (tid < n_tail) candidate(Piece<T>::value(row + tail_at + tid), tail_at + tid);
        };
        look_outside();
        // 2^lg lanes take one of those threads at a time, each a piece of the thread's, four on their way before the first is looked at
        int lg = 0;
        while (lg < 5 && (1 << lg) < turns) ++lg;
        for (int l = tid >> lg; l < n_looks; l += kScoreThreads >> lg) {
            const int who = looks[l];
            for (int t0 = tid & ((1 << lg) - 1); t0 < turns; t0 += 4 << lg) {
                uint4 q[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int piece = (t0 + (u << lg)) * kScoreThreads + who;
                    if (piece < pieces) q[u] = load_piece(mid + piece);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int piece = (t0 + (u << lg)) * kScoreThreads + who;
                    if (piece < pieces) look_at(q[u], piece);
                }
            }
        }
        __syncthreads();
        if (n_list > kCap) {
            // More candidates than there is room for (many equal logits, rows in ascending order and the like): once more, a piece of every
            // thread at a time.  Where the list could overflow in the next turn, only the likeliest stay, and the bound rises.
            __syncthreads();
            if (tid == 0) n_list = 0;
            __syncthreads();
            look_outside();
            for (int at = 0; at < pieces; at += kScoreThreads) {
                __syncthreads();
                if (n_list > kKeep) {
                    const int n = n_list;
                    rank_list();
                    if (tid < top) list[tid] = best[tid];
                    if (tid == 0) {
                        n_list = n < top ? n : top;
                        bound_s = best[top - 1];
                    }
                    __syncthreads();
                    bound = bound_s;
                    bound_value = key_value(bound);
                }
                __syncthreads();
                if (at + tid < pieces) look_at(load_piece(mid + at + tid), at + tid);
            }
            __syncthreads();
        }
        rank_list();
    } else {
        __syncthreads();
    }

    // ---- the CTAs of the cluster meet in the first one
    const unsigned long long* result = best;
    if (cluster > 1) {
        tc::cluster_sync();
        if (rank == 0) {
            if (warp == 0) {
                const int c = min(lane & 7, cluster - 1);
                const uint32_t from = tc::cluster_addr(tc::smem_u32(&whole), static_cast<uint32_t>(c));
                const float4 held = tc::cluster_ld4(from);
                Part o = {held.x, held.y, held.z, held.w};
                if ((lane & 7) >= cluster) o.a = o.a_low = o.b = 0.0f;
                o = join_lanes<8>(o);
                if (lane == 0) parts[0] = o;
            }
            if (tid < top * cluster) {
                const uint32_t from = tc::cluster_addr(tc::smem_u32(best), static_cast<uint32_t>(tid / top));
                list[tid] = tc::cluster_ld_u64(from + (tid % top) * 8);
            }
            __syncthreads();
            if (tid < top * cluster) {
                const unsigned long long k = list[tid];
                const int more = larger(list, top * cluster, k, top);
                if (k != 0ull && more < top) merged[more] = k;           // (not best[]: it is being read)
            }
        }
        tc::cluster_sync();                            // nobody leaves while its shared memory is being read
        if (rank != 0) return;
        result = merged;
    }
    Part w = cluster > 1 ? parts[0] : whole;
    if (w.m <= kNearFloor || w.m >= kHuge) w = row_exactly<T>(row, a.vocab, parts);      // (the same in every thread)
    const float ln_a = log1pf((w.a - 1.0f) + w.a_low);
    const bool any = w.a > 0.0f;                        // false: a row of -inf, or one with NaN or +inf in it
    if (tid == 0) {
        const float l = Piece<T>::value(row + token);
        a.logprob[r] = any ? (l - w.m) - ln_a : CUDART_NAN_F;
        // (both terms are positive: t_v <= 0 once m is the maximum)
        if (a.entropy != nullptr) a.entropy[r] = any ? ln_a - 0.69314718055994531f * (w.b / w.a) : CUDART_NAN_F;
    }
    if (tid < top) {
        const unsigned long long k = result[tid];
        a.top_ids[r * top + tid] = key_id(k);
        a.top_logprobs[r * top + tid] = any ? (key_value(k) - w.m) - ln_a : CUDART_NAN_F;
    }
}

template <typename T>
cudaError_t launch_typed(const ScoreArgs& a, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.rows * a.cluster));
    cfg.blockDim = dim3(kScoreThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {static_cast<unsigned>(a.cluster), 1, 1};
    cfg.numAttrs = 1 + overlap_launch_attribute(st, attr + 1);
    cfg.attrs = attr;
    return cudaLaunchKernelEx(&cfg, score_kernel<T>, a);
}

}  // namespace

cudaError_t launch_score(ScoreArgs a, int logits_dtype, int sm_count, cudaStream_t st) {
    // CTAs per row: as many as have an SM each, as long as every thread has pieces to look at.  (Rows of 151936 bf16 logits, 1, 2, 4 or
    // 8 CTAs a row: 22 rows with five alternatives 18.5, 13.8, 11.0, 11.1 us; 40 rows with 20 21.4, 16.3, 15.1, 16.9; 76 rows 21.6, 18.3, 17.7,
    // 27.0, without alternatives 16.7, 12.8, 12.4, 13.3; 152 rows with 20 24.7, 23.6, 28.8, 43.1; 300 rows 34.0, 38.1, 44.9, 73.7.  What a CTA
    // does besides its pass, 4 to 8 us, is done by each.  Some 40 to 150 rows would gain 1 to 4 us by more CTAs than this rule has.)
    const int per_piece = logits_dtype == FDD_LOGITS_BF16 ? 8 : 4;
    a.cluster = 1;
    while (a.cluster < 8 && a.rows * a.cluster * 2 <= sm_count && a.vocab >= a.cluster * 2 * kScoreThreads * per_piece) a.cluster *= 2;
    return logits_dtype == FDD_LOGITS_BF16 ? launch_typed<__nv_bfloat16>(a, st) : launch_typed<float>(a, st);
}
