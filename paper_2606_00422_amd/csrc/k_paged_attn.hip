// Attention of new rows over a paged cache, one wave per (row, query head):
// lanes take keys 64 at a time for the scores and features for the weighted
// values; running maximum, sum and output in fp32.
#include <type_traits>

#include "upr_paged.h"

namespace upr {

namespace {

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) v = fmaxf(v, __shfl_xor(v, x, 64));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) v += __shfl_xor(v, x, 64);
    return v;
}

// Score in log2 units.
__device__ __forceinline__ float score2(const AttnArgs& a, float dot, float slope2, int away) {
    float z = a.cap2 > 0.f ? a.cap2 * tanhf(dot * a.ct) : dot * a.c;
    return fmaf(slope2, (float)away, z);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void k_paged_attn_row(AttnArgs a, PagedPool pool, PagedUsers users) {
    int lo = 0, hi = users.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (users.item0[mid] <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)((int)blockIdx.x - users.item0[lo]) * 4 + (threadIdx.x >> 6);
    if (w >= (int64_t)users.count[lo] * a.n_heads) return;
    const int t = (int)(w / a.n_heads), h = (int)(w % a.n_heads), kh = h / (a.n_heads / a.n_kv_heads);
    const int64_t row = (int64_t)users.row0[lo] + t;
    const bool own = a.k_self.p != nullptr;
    const int pos = own ? users.rows[lo] : users.rows[lo] - users.count[lo] + t;
    const int end = own ? pos : pos + 1;                // keys first .. end - 1
    const int first = a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
    const int32_t* const table = pool.tables + (int64_t)users.user[lo] * pool.stride;
    const T* const q = static_cast<const T*>(a.q.p) + row * a.q.ld + (int64_t)h * D;
    const float slope2 = a.slopes != nullptr ? a.slopes[h] * 1.4426950408889634f : 0.f;
    auto place = [&](int j, int kv) -> const T* {       // null: a page outside the pool
        const int page = table[j >> pool.page_shift];
        if (page < 0 || page >= pool.n_pages) return nullptr;
        return reinterpret_cast<const T*>(pool.data) +
               ((((int64_t)page * 2 + kv) * a.n_kv_heads + kh) * pool.page_rows + (j & (pool.page_rows - 1))) * D;
    };
    auto dot = [&](const T* k) {
        float s = 0.f;
        if (k != nullptr)
            for (int e = 0; e < D; ++e) s = fmaf((float)q[e], (float)k[e], s);
        return s;
    };
    constexpr int kE = D > 64 ? D / 64 : 1;
    float m = -INFINITY, l = 0.f, acc[kE];
    for (int i = 0; i < kE; ++i) acc[i] = 0.f;
    if (own) {
        const T* const vs = static_cast<const T*>(a.v_self.p) + row * a.v_self.ld + (int64_t)kh * D;
        m = score2(a, dot(static_cast<const T*>(a.k_self.p) + row * a.k_self.ld + (int64_t)kh * D), slope2, 0);
        l = lane == 0 ? 1.f : 0.f;
        for (int i = 0; i < kE; ++i) acc[i] = (float)vs[i * 64 + lane % D];
        if (m == -INFINITY) {
            l = 0.f;
            for (int i = 0; i < kE; ++i) acc[i] = 0.f;
        }
    }
    for (int j0 = first; j0 < end; j0 += 64) {
        const int n = end - j0 < 64 ? end - j0 : 64;
        const float s = lane < n ? score2(a, dot(place(j0 + lane, 0)), slope2, j0 + lane - pos) : -INFINITY;
        const float mn = fmaxf(m, wave_max(s));
        const float ref = mn == -INFINITY ? 0.f : mn;
        const float alpha = exp2f(m - ref);
        const float p = lane < n ? exp2f(s - ref) : 0.f;
        m = mn;
        l = l * alpha + p;
        for (int i = 0; i < kE; ++i) acc[i] *= alpha;
        for (int j = 0; j < n; ++j) {
            const float pj = __shfl(p, j, 64);
            const T* const v = place(j0 + j, 1);
            if (v != nullptr)
                for (int i = 0; i < kE; ++i) acc[i] = fmaf(pj, (float)v[i * 64 + lane % D], acc[i]);
        }
    }
    const float inv = 1.f / wave_sum(l);
    if (lane >= D) return;
    for (int i = 0; i < kE; ++i) {
        const int64_t at = row * a.out_ld + (int64_t)h * D + i * 64 + lane;
        const float v = keep_f32(acc[i] * inv);
        if (a.out_kind == ATTN_OUT_F16) static_cast<f16*>(a.out)[at] = (f16)v;
        else if (a.out_kind == ATTN_OUT_F32) static_cast<float*>(a.out)[at] = v;
        else static_cast<T*>(a.out)[at] = (T)v;
    }
}

}  // namespace

hipError_t launch_paged_attn(int dtype, const AttnArgs& a, const PagedPool& pool, const PagedUsers& users,
                             hipStream_t s) {
    const unsigned grid = (unsigned)users.item0[users.n];
    if (grid == 0) return hipSuccess;
    auto go = [&](auto t) {
        typedef decltype(t) T;
        if (a.D == 32) k_paged_attn_row<T, 32><<<grid, 256, 0, s>>>(a, pool, users);
        else if (a.D == 64) k_paged_attn_row<T, 64><<<grid, 256, 0, s>>>(a, pool, users);
        else k_paged_attn_row<T, 128><<<grid, 256, 0, s>>>(a, pool, users);
    };
    if (dtype == UPR_F32) go(float{}); else go(bf16{});
    return hipGetLastError();
}

}  // namespace upr
