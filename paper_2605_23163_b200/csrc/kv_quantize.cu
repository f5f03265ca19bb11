// A prefix cache in 8 bits: rows of K and V rounded to e4m3 as they join it, and read back as bf16.
//
// A group is 64 tokens of one KV head (a page's share of that head).  Its entries are q * 2^E, q in e4m3, with the smallest E
// in [-117, 119] under which no finite entry exceeds 448 = 1.75 * 2^8.  E follows from the largest magnitude 1.m * 2^e by
// its bits alone: e - 8, one more where 1.m > 1.75.  A power of two as the scale costs a float format no precision
// (three mantissa bits whatever the exponent; at most one of the 18 binades down to the smallest subnormal goes unused), and
// makes everything else exact: the product with 2^-E before the one rounding, q * 2^E in bf16, and so the attention that reads
// it.  The lower limit keeps 2^-9 * 2^E a normal bf16 number, the upper one 448 * 2^E a finite one.
//
// Rows may join a group that holds some already (blocks of 32 tokens, pages of 64).  Its exponent can only rise; the rows
// that are there are then rounded again, from their 8 bits: at most half a step of the new scale on top of what they lost before.
//
// Bound by memory: 2 bytes read and 1 written per entry, and nothing to reuse.  One CTA takes a group (64 rows x D = 16 KB of
// bf16 at D = 128) into registers, 8 entries a piece (16 bytes in, 8 out: neighbouring lanes read and write side by side) and 8 pieces
// a thread, so that the maximum and the rounding need one read; the CTAs of a token's heads follow one another, since their rows lie side by side in the source.
// No load goes through the read-only path: these kernels start while the one ahead may still write.  Rows and bytes, which nobody
// reads twice, go past L1 (__ldcg).
#include "fdd_internal.h"
#include "tc_ptx.cuh"
#include "e4m3.cuh"

#include <algorithm>

namespace {

constexpr int kQuantThreads = 128;

// One group of one cache.
template <int D>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const __grid_constant__ QuantArgs a) {
    constexpr int kPerRow = D / 8, kPieces = kKvGroup * kPerRow / kQuantThreads;
    __shared__ uint32_t warp_max[kQuantThreads / 32];
    tc::grid_dependency_wait();          // (launched for an early start behind the kernel ahead of it)
    const long long unit = blockIdx.x;
    int s = 0, hi = a.n - 1;                             // the last set that begins at or before this unit
    while (s < hi) {
        const int mid = (s + hi + 1) >> 1;
        if (unit >= a.set[mid].unit_begin) s = mid; else hi = mid - 1;
    }
    const QuantSet& qs = a.set[s];
    long long t = unit - qs.unit_begin;
    const int h = static_cast<int>(t % a.n_kv_heads); t /= a.n_kv_heads;
    const int which = static_cast<int>(t & 1);           // K or V
    const int g = qs.first / kKvGroup + static_cast<int>(t >> 1);
    long long slot = g;                                  // group's place in the cache
    if (qs.page_table != nullptr) {
        slot = qs.page_table[g];
        if (slot < 0 || slot >= qs.cap) {                // a page table entry outside the pool: nothing is written
            if (threadIdx.x == 0) atomicCAS(a.status, 0, FDD_ERR_INVALID_ARG);
            return;
        }
    }
    uint8_t* const dst = qs.dst[which] + (qs.page_table != nullptr ? (slot * a.n_kv_heads + h) * kKvGroup
                                                                   : static_cast<long long>(h) * qs.cap + slot * kKvGroup) * D;
    int8_t* const exp_at = qs.exps[which] + (qs.page_table != nullptr ? slot * a.n_kv_heads + h
                                                                      : h * static_cast<long long>(kv_groups(qs.cap)) + slot);
    // rows [lo, hi_row) of the group are new, those in front of them are there already
    const int lo = max(0, qs.first - g * kKvGroup), hi_row = min(kKvGroup, qs.first + qs.count - g * kKvGroup);
    const __nv_bfloat16* const src = qs.src[which] + (static_cast<long long>(g) * kKvGroup - qs.first) * a.row_stride + static_cast<long long>(h) * D;

    uint4 x[kPieces];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int piece = i * kQuantThreads + threadIdx.x, row = piece / kPerRow, c = piece % kPerRow;
        x[i] = make_uint4(0, 0, 0, 0);
        if (row >= lo && row < hi_row) x[i] = __ldcg(reinterpret_cast<const uint4*>(src + row * a.row_stride + c * 8));
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        most = __vmaxu2(most, __vmaxu2(__vmaxu2(x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu), __vmaxu2(x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu)));
    auto over_cta = [&](uint32_t m) {
        m = __reduce_max_sync(0xFFFFFFFFu, max(m & 0xFFFFu, m >> 16));
        if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
        __syncthreads();
        m = max(max(warp_max[0], warp_max[1]), max(warp_max[2], warp_max[3]));
        return m;
    };
    static_assert(kQuantThreads == 128, "four warps' maxima");
    most = over_cta(most);
    if (most >= 0x7F80u) {                               // (the same in every thread)
        // something is not finite: it counts for nothing in the maximum and becomes NaN
        uint32_t finite = 0;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            uint32_t* w = reinterpret_cast<uint32_t*>(&x[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t lo16 = w[k] & 0x7FFFu, hi16 = (w[k] >> 16) & 0x7FFFu;
                if (lo16 >= 0x7F80u) w[k] |= 0x7FFFu; else finite = max(finite, lo16);
                if (hi16 >= 0x7F80u) w[k] |= 0x7FFF0000u; else finite = max(finite, hi16);
            }
        }
        __syncthreads();                                 // (warp_max is read by everybody above)
        most = over_cta(finite);
    }
    int e = e4m3::exponent_for(most);
    const bool joins = lo > 0;
    const int e_old = joins ? min(max(static_cast<int>(*exp_at), e4m3::kMinExp), e4m3::kMaxExp) : e;
    e = max(e, e_old);
    const float scale = e4m3::pow2(-e);
    __syncthreads();                                     // everybody has read the old exponent
    if (threadIdx.x == 0) *exp_at = static_cast<int8_t>(e);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int piece = i * kQuantThreads + threadIdx.x, row = piece / kPerRow, c = piece % kPerRow;
        uint2* const to = reinterpret_cast<uint2*>(dst + row * D + c * 8);
        if (row >= lo && row < hi_row) {
            *to = make_uint2(e4m3::from_bf16x4(x[i].x, x[i].y, scale), e4m3::from_bf16x4(x[i].z, x[i].w, scale));
        } else if (row < lo && e != e_old) {
            const float down = ldexpf(1.0f, e_old - e);
            const uint2 q = *to;
            *to = make_uint2(e4m3::rescale4(q.x, down), e4m3::rescale4(q.y, down));
        }
    }
}

// Tokens [first, first + count) of one layer's cache as bf16 rows [count][Hkv][D]: a thread takes 8 entries (8 bytes in, 16 out) at a
// time, in the order of the output, so that a warp writes whole lines.  A CTA takes a run of kRun pieces, all of a thread's reads on their way
// before the first is turned; where a run begins is the only division in 64 bits.  16384 tokens of 8 heads: 20.4 us (4.9 TB/s; runs of twice
// or half the pieces 20.4 and 23.8, 8 CTAs per SM that take run after run 22.1, pieces of 16 entries 20.5 to 22).
constexpr int kReadThreads = 256, kReadAtOnce = 4, kRun = kReadThreads * kReadAtOnce;
template <int D>
__global__ void __launch_bounds__(kReadThreads) dequantize_kernel(const __grid_constant__ DequantArgs a) {
    constexpr int kPerRow = D / 8;
    tc::grid_dependency_wait();
    const uint32_t per_token = static_cast<uint32_t>(a.n_kv_heads) * kPerRow;
    const long long per_cache = static_cast<long long>(a.count) * per_token, runs = (per_cache + kRun - 1) / kRun;
    const int groups = kv_groups(a.cap);
    for (long long run = blockIdx.x; run < 2 * runs; run += gridDim.x) {
        const int which = run >= runs ? 1 : 0;
        const long long begin = (run - which * runs) * kRun, row0 = begin / per_token;
        const uint32_t in_row0 = static_cast<uint32_t>(begin - row0 * per_token), left = static_cast<uint32_t>(min(per_cache - begin, static_cast<long long>(kRun)));
        uint2 q[kReadAtOnce];
        int e[kReadAtOnce];
        __nv_bfloat16* to[kReadAtOnce];
#pragma unroll
        for (int i = 0; i < kReadAtOnce; ++i) {
            to[i] = nullptr;
            const uint32_t idx = i * kReadThreads + threadIdx.x;
            if (idx >= left) continue;
            const uint32_t at = in_row0 + idx, more = at / per_token, r = at - more * per_token;
            const int h = r / kPerRow, c = r % kPerRow;
            const long long row = row0 + more;
            const int token = a.first + static_cast<int>(row);
            long long entry, group;
            if (a.page_table != nullptr) {
                const long long page = a.page_table[token / kKvGroup];
                if (page < 0 || page >= a.cap) {         // not followed: the row is left as it is
                    atomicCAS(a.status, 0, FDD_ERR_INVALID_ARG);
                    continue;
                }
                group = page * a.n_kv_heads + h;
                entry = group * kKvGroup + token % kKvGroup;
            } else {
                group = static_cast<long long>(h) * groups + token / kKvGroup;
                entry = static_cast<long long>(h) * a.cap + token;
            }
            q[i] = __ldcg(reinterpret_cast<const uint2*>(a.src[which] + entry * D) + c);
            e[i] = a.exps[which][group];                 // (out of L1: 64 tokens' pieces want it)
            to[i] = a.dst[which] + row * a.row_stride + static_cast<long long>(h) * D + c * 8;
        }
#pragma unroll
        for (int i = 0; i < kReadAtOnce; ++i) {
            if (to[i] == nullptr) continue;
            const uint32_t scale = e4m3::pow2_bf16x2(e[i]);
            *reinterpret_cast<uint4*>(to[i]) = make_uint4(e4m3::to_bf16x2(static_cast<uint16_t>(q[i].x), scale), e4m3::to_bf16x2(static_cast<uint16_t>(q[i].x >> 16), scale),
                                                          e4m3::to_bf16x2(static_cast<uint16_t>(q[i].y), scale), e4m3::to_bf16x2(static_cast<uint16_t>(q[i].y >> 16), scale));
        }
    }
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs& a, int head_dim, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.units));
    cfg.blockDim = dim3(kQuantThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    cfg.numAttrs = overlap_launch_attribute(st, attr);
    cfg.attrs = attr;
    return head_dim == 64 ? cudaLaunchKernelEx(&cfg, quantize_kernel<64>, a) : cudaLaunchKernelEx(&cfg, quantize_kernel<128>, a);
}

cudaError_t launch_dequantize(const DequantArgs& a, int head_dim, cudaStream_t st) {
    const long long runs = (static_cast<long long>(a.count) * a.n_kv_heads * (head_dim / 8) + kRun - 1) / kRun;
    const long long blocks = std::min(2 * runs, 0x7FFFFFFFLL);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kReadThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    cfg.numAttrs = overlap_launch_attribute(st, attr);
    cfg.attrs = attr;
    return head_dim == 64 ? cudaLaunchKernelEx(&cfg, dequantize_kernel<64>, a) : cudaLaunchKernelEx(&cfg, dequantize_kernel<128>, a);
}
