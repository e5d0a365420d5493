// Attention of new rows over a paged cache on the matrix cores.
//
// Rows are (token, query head of one key/value head's group) pairs, so shared
// K/V heads are read once for all their query heads.  One workgroup = one work
// item: a tile of rows of one (user, key/value head), over all keys the tile
// sees or, where a call has few rows, over one part of them.  Its waves are RW
// groups of 16 QG rows times KW groups of keys: many rows share each K/V stage
// (RW), or the four waves of one 16- or 32-row tile take different keys of the
// stage (KW).  K/V stages go straight from the pages to LDS (buffer loads that
// return zeros past the user's rows and for page numbers outside the pool;
// double-buffered).  Per 32 keys (16 in fp32) a wave computes
//   S^T = K Q^T,   P = 2^(z - m),   O^T += V^T P^T
// with z the scaled (capped, biased, masked) score in log2 units: a lane holds
// scores of one row, and its packed probabilities are the next product's
// operand as they stand.  bf16: v_mfma_f32_16x16x32_bf16, bf16 probabilities
// (one rounding, 2^-8; the row sum adds the rounded values); V^T by transposing
// LDS reads.  fp32: v_mfma_f32_16x16x4_f32, everything fp32.
//
// The running reference m follows a row's maximum only when a score passes it
// by 2^kSlack, or (kSums) the row's sum passes kMostSum: probabilities then reach
// that instead of 1, which costs no precision (sums are fp32, and values up to
// 2^80 do not overflow them; rows that do are done again), and O is
// rescaled a few times per row instead of every block.  A
// row's decision uses its own scores only, so its result does not depend on
// the rows beside it.
//
// Key groups are merged through LDS, key parts by k_paged_attn_join from the
// workspace.  A row whose result is not finite (a masked key's NaN or infinite
// value times probability 0, or scores beyond the reference's range) is done
// again by attn_row, which touches visible keys only.
//
// What bounds it (MI355X; us from graphs of the calls):
//  * single rows: the cache's bytes.  64 rows over 512-16384 cached rows, 32/8
//    heads of 128, 2.15 GB: 391 us, 5.5 TB/s (a 1 GB copy moves 4.8 to 5.2).
//    One row over 1024 rows, 8 heads of 64: 8.0 us, of which 4.8 are the launch
//    and the chain of loads to the first keys, the rest a CU's 62 B/ns.
//  * 128-row tiles: vector issue and the matrix cores in turn.  4 x 2048 rows over
//    up to 8192, 32/8 heads of 128: 466 to 485 us, 1.08 to 1.12 PFLOP/s (a matrix
//    product of 8192^3 reaches 1.14); before fragments were read ahead 542.  At
//    head_dim 64 a score costs as many vector instructions for half the products:
//    64 x 2000 candidates over 1024 rows, 8 heads: 336 to 346 us, 780 to 800
//    TFLOP/s (with a maximum per block 352, vector units 66% and matrix cores
//    37% busy).
//  * 32-row tiles: 48 chunks of 1-96 rows, window 1024, bias, 8 heads of 64, 97 MB:
//    30 us, workgroup starts beside 19 us of cache reads.
//  * fp32: the fp32 matrix rate (154 TFLOP/s) at one to two waves per SIMD: 6
//    chunks of 20-200 rows, cap, 4 heads of 64: 20 us with the join.
#include <type_traits>

#include "paged_dev.h"

namespace upr {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 b8;
typedef __attribute__((ext_vector_type(4))) __bf16 b4;
typedef __attribute__((ext_vector_type(2))) __bf16 b2;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 b4v;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) _Float16 h4;

constexpr float kUnset = -1e30f;        // reference of a row that has seen no key
constexpr float kSlack = 8.0f;
constexpr float kMostSum = 0x1p40f;

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
// Over the four lanes {l, l^16, l^32, l^48} of one row.
__device__ __forceinline__ float quad_max(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// (NaN if one of them is: no instructions to quiet one first.  Such a row's
// result is NaN whatever its reference.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// 2^x on the transcendental unit (below 2^-126: 0).
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// At most N of the wave's loads (to LDS) still under way; all its LDS reads done.
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
}
__device__ __forceinline__ void wait_lds() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);
}

__device__ __forceinline__ float first_of(float x) { return x; }
__device__ __forceinline__ float first_of(f32x4 x) { return x[0]; }

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// The capped score in log2 units.  tanh x = 1 - 2 / (2^(2 x log2 e) + 1), off by
// about 2^-23: the cap is far above any difference of scores that matters.
__device__ __forceinline__ float capped(const AttnArgs& a, float dot) {
    return a.cap2 * fmaf(-2.f, __builtin_amdgcn_rcpf(fast_exp2(dot * a.ct2) + 1.f), 1.f);
}
// Score in log2 units.
__device__ __forceinline__ float score2(const AttnArgs& a, float dot, float slope2, int away) {
    return fmaf(slope2, (float)away, a.cap2 > 0.f ? capped(a, dot) : dot * a.c);
}

// Where an item stands.
struct Item {
    int user;               // row of the page table
    int64_t row0;           // first row of the user's q / out
    int count, rows;        // new rows, cached rows
    int kh, tile, split, splits;
};

template <int TR>
__device__ __forceinline__ Item find_item(const AttnArgs& a, const PagedUsers& users, int b) {
    const int i = user_of(users, b);
    Item it;
    it.user = users.user[i];
    it.row0 = users.row0[i];
    it.count = users.count[i];
    it.rows = users.rows[i];
    it.splits = attn_splits(it.rows, it.count, a.k_self.p != nullptr, a.window, a.chunk);
    const int idx = b - users.item0[i], r = idx / a.n_kv_heads;
    it.kh = idx - r * a.n_kv_heads;
    it.tile = r / it.splits;
    it.split = r - it.tile * it.splits;
    // causal: a user's last tiles see the most keys and go first
    if (a.k_self.p == nullptr) it.tile = (it.count * (a.n_heads / a.n_kv_heads) + TR - 1) / TR - 1 - it.tile;
    return it;
}

// Rows of a tile as (token, head of the group): one division for the tile, the
// rest by multiplication (x below 2048 and G at most 1024: exact).
struct Rows {
    int G, t0, h0;
    uint32_t magic;             // 2^32 / G, rounded up

    __device__ __forceinline__ Rows(int group, int tile0) : G(group), t0(tile0 / group) {
        h0 = tile0 - t0 * G;
        magic = 0xffffffffu / (uint32_t)G + 1;
    }
    // row i of the tile: its token, and its head in the group
    __device__ __forceinline__ int token(int i) const {
        return t0 + (G == 1 ? i : (int)__umulhi((uint32_t)(h0 + i), magic));
    }
    __device__ __forceinline__ int head(int i, int t) const { return h0 + i - (t - t0) * G; }
};

// One row by one wave, from its visible keys alone (speed is of no concern).
template <typename T, int D>
__device__ __forceinline__ void attn_row(const AttnArgs& a, const PagedPool& pool, int user, int rows, int64_t row,
                                                   int pos, int h) {
    const int lane = threadIdx.x & 63, kh = h / (a.n_heads / a.n_kv_heads);
    const bool own = a.k_self.p != nullptr;
    const int end = own ? rows : pos + 1;               // keys first .. end - 1
    const int first = a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
    const int32_t* const table = pool.tables + (int64_t)user * pool.stride;
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
        if (m > -INFINITY) {
            l = lane == 0 ? 1.f : 0.f;
            for (int i = 0; i < kE; ++i) acc[i] = (float)vs[i * 64 + lane % D];
        } else if (m != m) {
            l = m;
        }
    }
    for (int j0 = first; j0 < end; j0 += 64) {
        const int n = end - j0 < 64 ? end - j0 : 64;
        const float s = lane < n ? score2(a, dot(place(j0 + lane, 0)), slope2, j0 + lane - pos) : -INFINITY;
        const float mn = fmaxf(m, wave_max(s));
        const float ref = mn == -INFINITY ? 0.f : mn;
        const float alpha = fast_exp2(m - ref);
        const float p = lane < n ? fast_exp2(s - ref) : 0.f;
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

// LDS rows of D values, their 16-byte chunks XOR-swizzled: bf16 K fragments are
// 16 rows at one chunk, V fragments 8 rows x 32 bytes per pass, and the keys
// put them on distinct banks (a 256-byte bank period holds 4, 2 or 1 rows).
// fp32 K fragments likewise; fp32 V rows are read whole.
template <typename T, int D> __device__ __forceinline__ int key_k(int row) {
    constexpr int bytes = D * (int)sizeof(T);
    return bytes == 64 ? (row >> 2) & 3 : bytes == 128 ? (row >> 1) & 7 : row & 15;
}
template <typename T, int D> __device__ __forceinline__ int key_v(int row) {
    if (sizeof(T) == 4) return 0;
    return D == 32 ? ((row >> 2) & 1) << 1 : D == 64 ? ((row >> 1) & 3) << 1 : (row & 7) << 1;
}

// Keys of a stage: a block per key group, or 8 KB and more of each matrix.
template <typename T, int D, int KW>
constexpr int stage_keys() {
    return KW > 1 ? (sizeof(T) == 2 ? 32 : 16) * KW : sizeof(T) == 2 ? (D == 32 ? 128 : 64) : D == 128 ? 32 : 4096 / D;
}

template <typename T, int D, int QG, int RW, int KW, bool EX>
__global__ __launch_bounds__(64 * RW * KW, RW > 1 && D < 128 ? (EX ? 3 : 4) : 2) void k_paged_attn(AttnArgs a, PagedPool pool, PagedUsers users) {
    constexpr bool kBf = sizeof(T) == 2;
    constexpr int NW = RW * KW, SB = kBf ? 32 : 16, NT = SB / 16;
    constexpr int TS = stage_keys<T, D, KW>(), KS = TS / KW;
    constexpr int EB = D / 16, ES = kBf ? D / 32 : D / 16;
    constexpr int CR = D * (int)sizeof(T) / 16, RPL = 64 / CR;     // 16-byte chunks per row, rows per load
    constexpr int RPW = TS / NW, NI = RPW / RPL, NP = RPW > 16 ? RPW / 16 : 1;
    constexpr int TR = 16 * QG * RW;
    // One buffer instead of two where two fill a CU's LDS with one workgroup and
    // the matrix instructions, not the loads, take the time (fp32, head_dim 128:
    // 4 x 500 rows over 1000, 8 heads, 133 -> 110 us).
    constexpr bool kSingle = !kBf && D == 128;
    static_assert(RW == 1 || KW == 1, "a wave's rows or keys");
    static_assert(KS % SB == 0 && RPW % RPL == 0 && NI >= 1 && NI <= 8 && NP <= 4, "stage");
    __shared__ __attribute__((aligned(16))) T sK0[TS * D];
    __shared__ __attribute__((aligned(16))) T sK1[TS * D];
    __shared__ __attribute__((aligned(16))) T sV0[TS * D];
    __shared__ __attribute__((aligned(16))) T sV1[TS * D];

    const Item it = find_item<TR>(a, users, blockIdx.x);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, kg = wave / RW;
    const int g = lane >> 4, l16 = lane & 15;
    const bool own = a.k_self.p != nullptr;
    const int G = a.n_heads / a.n_kv_heads;
    const int n = it.rows, nrows = it.count * G;
    const int pos0 = own ? n : n - it.count;            // position of the user's first row
    const int tile0 = it.tile * TR;
    const int tlast = (tile0 + TR < nrows ? tile0 + TR : nrows) - 1;
    // keys of the tile, then of this part of them
    const Rows rows(G, tile0);
    const int end = own ? n : pos0 + rows.token(tlast - tile0) + 1;
    const int first = attn_first_key(own ? n : pos0 + rows.t0, a.window);
    const int k0 = a.chunk > 0 ? first + it.split * a.chunk : first;
    const int k1 = a.chunk > 0 && k0 + a.chunk < end ? k0 + a.chunk : end;
    const int nst = k1 > k0 ? (k1 - k0 + TS - 1) / TS : 0;
    // this wave's rows
    const int wrow = tile0 + rw * 16 * QG;
    const bool active = wrow < nrows;
    const int wlast = wrow + 16 * QG < nrows ? wrow + 16 * QG - 1 : nrows - 1;
    const int pfirst = own ? n - 1 : pos0 + rows.token(wrow - tile0);
    const int plast = own ? n - 1 : pos0 + rows.token(wlast - tile0);
    const int wend = plast + 1;                         // keys from here on: none for the wave
    // keys below this one are outside the last row's window, from wbeg on inside the first row's
    const int wlow = a.window > 0 ? (own ? n : plast) - a.window + 1 : 0;
    const int wbeg = a.window > 0 ? (own ? n : pfirst) - a.window + 1 : 0;

    // ---- K/V stages
    // (nothing writes the tables while the kernel runs: scalar loads, which do
    // not queue behind the stages')
    typedef const __attribute__((address_space(4))) int32_t* constants;
    const constants table = (constants)(uintptr_t)(pool.tables + (int64_t)it.user * pool.stride);
    // (one page's bytes: at most 2 x 1024 heads x 1024 rows x 512 bytes)
    constexpr int RB = D * (int)sizeof(T);
    const uint32_t v_off = (uint32_t)a.n_kv_heads * pool.page_rows * RB, page_bytes = 2 * v_off;
    const char* const head0 = pool.data + (size_t)((uint32_t)it.kh * pool.page_rows * RB);
    const int rbase = wave * RPW;
    int offK[8], offV[8];       // (fixed size: with a template-dependent one the host pass drops the launch stub)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int row = rbase + i * RPL + lane / CR, slot = lane % CR;
        const int r16 = (i * RPL) % 16 + lane / CR;     // row of its 16-row piece (RPW below 16: of the wave's)
        offK[i] = r16 * D * (int)sizeof(T) + ((slot ^ key_k<T, D>(row)) << 4);
        offV[i] = r16 * D * (int)sizeof(T) + ((slot ^ key_v<T, D>(row)) << 4);
    }
    // A wave's rows of a stage are pieces of 16, which never cross a page; pages
    // of 32 rows and more hold two of them (stages start at multiples of 32).
    const bool pairs = pool.page_rows >= 32;
    int pid[4];                 // page numbers of the pieces
    auto fetch_pages = [&](int st) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int key = k0 + st * TS + rbase + 16 * p;
            if (p % 2 == 1 && pairs) continue;
            pid[p] = key < k1 ? table[key >> pool.page_shift] : -1;
        }
    };
    auto issue_loads = [&](T* dK, T* dV, int st) __attribute__((always_inline)) {
        const char* pk = head0;
        int bytes = 0, base = 0;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int key = k0 + st * TS + rbase + 16 * p;
            if (p % 2 == 0 || !pairs) {
                base = key & -pool.page_rows;
                // rows of the page that hold keys; none past this part's keys or
                // in a page outside the pool
                const bool in = (uint32_t)pid[p] < (uint32_t)pool.n_pages;
                bytes = in ? (n - base < pool.page_rows ? n - base : pool.page_rows) * RB : 0;
                pk = head0 + (uint64_t)(in ? (uint32_t)pid[p] : 0u) * page_bytes;
            }
            const __amdgpu_buffer_rsrc_t rsK = __builtin_amdgcn_make_buffer_rsrc((void*)pk, (short)0, bytes, 0x00020000);
            const __amdgpu_buffer_rsrc_t rsV =
                __builtin_amdgcn_make_buffer_rsrc((void*)(pk + v_off), (short)0, bytes, 0x00020000);
            const int off = (key - base) * RB;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if (i * RPL / 16 != p) continue;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rsK, (__attribute__((address_space(3))) void*)(dK + (rbase + i * RPL) * D), 16, offK[i] + off, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rsV, (__attribute__((address_space(3))) void*)(dV + (rbase + i * RPL) * D), 16, offV[i] + off, 0, 0, 0);
            }
        }
    };
    fetch_pages(0);

    // ---- the lane's rows
    typedef std::conditional_t<kBf, b8, f32x4> frag;
    frag qf[QG][ES];
    f32x4 o[QG][EB];            // bf16: e = 16 eb + 4g + r; fp32: e = EB (4g + r) + eb
    // row sums: the product of the probabilities with ones (the sum of all keys
    // so far, in all four registers), or in 128-row tiles, whose registers are
    // short, and in fp32, of the lane's keys
    constexpr bool kOnes = kBf && RW == 1;
    // 128-row tiles without bias or cap: the sums, not a maximum per block, tell
    // that a reference is passed (64 x 2000 candidates over 1024, 8 heads of 64, 354
    // -> 344 us, 16 of 32, 482 -> 458; 4 x 2048 rows, 32/8 heads of 128, 485 -> 480).
    // A steep bias passes it at every block, at a higher cost (636 -> 858).
    constexpr bool kSums = kBf && RW > 1 && !EX;
    typedef std::conditional_t<kOnes, f32x4, float> lsum;
    lsum l[QG];
    float negm[QG], slope2[QG];
    int rpos[QG], low[QG], seen[QG];
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) {
        int r = wrow + qg * 16 + l16;
        r = r < nrows ? r : nrows - 1;                  // (a ragged tail repeats the last row)
        const int t = rows.token(r - tile0), h = it.kh * G + rows.head(r - tile0, t);
        const int64_t row = it.row0 + t;
        rpos[qg] = pos0 + (own ? 0 : t);
        low[qg] = a.window > 0 && rpos[qg] >= a.window ? rpos[qg] - a.window + 1 : 0;
        const int high = own || rpos[qg] + 1 > k1 ? k1 : rpos[qg] + 1;
        seen[qg] = high > low[qg] ? high - low[qg] : 0;
        if constexpr (EX) slope2[qg] = a.slopes != nullptr ? a.slopes[h] * 1.4426950408889634f : 0.f;
        const T* const qrow = static_cast<const T*>(a.q.p) + row * a.q.ld + (int64_t)h * D;
#pragma unroll
        for (int es = 0; es < ES; ++es)
            qf[qg][es] = *reinterpret_cast<const frag*>(qrow + (kBf ? es * 32 + 8 * g : (4 * es + g) * 4));
    }
    // the rows' loads go first: the loop then waits for stages alone
    __builtin_amdgcn_sched_barrier(0);
    issue_loads(sK0, sV0, 0);
    fetch_pages(1);
    if constexpr (RW == 1 && !kSingle) {
        issue_loads(sK1, sV1, 1);
        fetch_pages(2);
    }
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) {
        l[qg] = lsum{0.f};
        negm[qg] = -kUnset;
#pragma unroll
        for (int eb = 0; eb < EB; ++eb) o[qg][eb] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (own && kg == 0 && it.split == 0) {          // starts from the row's own key
            int r = wrow + qg * 16 + l16;
            r = r < nrows ? r : nrows - 1;
            const int64_t row = it.row0 + rows.token(r - tile0);
            const T* const krow = static_cast<const T*>(a.k_self.p) + row * a.k_self.ld + (int64_t)it.kh * D;
            const T* const vrow = static_cast<const T*>(a.v_self.p) + row * a.v_self.ld + (int64_t)it.kh * D;
            float s = 0.f;
#pragma unroll
            for (int es = 0; es < ES; ++es) {
                const frag kf = *reinterpret_cast<const frag*>(krow + (kBf ? es * 32 + 8 * g : (4 * es + g) * 4));
#pragma unroll
                for (int j = 0; j < (kBf ? 8 : 4); ++j) s = fmaf((float)qf[qg][es][j], (float)kf[j], s);
            }
            const float z = score2(a, quad_sum(s), 0.f, 0);
            if (z > kUnset) {                           // (else: attn_row, as for any row out of range)
                negm[qg] = -z;
                if constexpr (kOnes) l[qg] = f32x4{1.f, 1.f, 1.f, 1.f}; else l[qg] = g == 0 ? 1.f : 0.f;
            } else {
                if constexpr (kOnes) l[qg] = f32x4{NAN, NAN, NAN, NAN}; else l[qg] = NAN;
            }
#pragma unroll
            for (int eb = 0; eb < EB; ++eb)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[qg][eb][r] = (float)vrow[kBf ? 16 * eb + 4 * g + r : EB * (4 * g + r) + eb];
        }
    }

    // ---- fragments of a block, rows kb .. of the stage
    constexpr int VW = kBf ? 1 : EB < 4 ? EB : 4;       // fp32: values per read of a V row
    typedef __attribute__((ext_vector_type(VW))) float vpart;
    typedef std::conditional_t<kBf, b8, vpart> vfrag;
    constexpr int NV = kBf ? EB : 4 * (EB / VW);
    // K: 16-key half t (fp32: the block), step es of the contraction
    auto read_k = [&](const T* cK, int kb, int t, int es) __attribute__((always_inline)) {
        const int row = kb + t * 16 + l16;
        return *reinterpret_cast<const frag*>(
            &cK[row * D + (((es * 4 + g) ^ key_k<T, D>(row)) << (kBf ? 3 : 2))]);
    };
    // V: bf16, V^T of e-block i in the order of the probabilities; fp32, the
    // part i % (EB / VW) of the lane's columns of row r = i / (EB / VW)
    auto read_v = [&](const T* cV, int kb, int i) __attribute__((always_inline)) {
        vfrag vf;
        if constexpr (kBf) {
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int row = kb + 16 * hh + 4 * g + (l16 >> 2);
                const int ch = 2 * i + ((l16 & 3) >> 1);
                const T* p = &cV[row * D + ((ch ^ key_v<T, D>(row)) << 3) + ((l16 & 1) << 2)];
                const b4v v4 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) b4v*)(p));
#pragma unroll
                for (int j = 0; j < 4; ++j) vf[4 * hh + j] = v4[j];
            }
        } else {
            vf = *reinterpret_cast<const vfrag*>(cV + (kb + 4 * g + i / (EB / VW)) * D + EB * l16 + i % (EB / VW) * VW);
        }
        return vf;
    };
    struct Frags {
        frag k[NT * ES];
        vfrag v[NV];
    };
    auto read_ks = [&](const T* cK, int kb, Frags& f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NT * ES; ++i) f.k[i] = read_k(cK, kb, i / ES, i % ES);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto read_vs = [&](const T* cV, int kb, Frags& f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NV; ++i) f.v[i] = read_v(cV, kb, i);
        __builtin_amdgcn_sched_barrier(0);
    };

    // ---- one block of SB keys, keys kabs .. of the user, from its fragments;
    // scored(): called when those of K are used up
    auto sub_block = [&](const Frags& f, int kabs, auto scored) __attribute__((always_inline)) {
        // matrix instructions of a wave go before the other waves' on its SIMD,
        // whose exponentials then fill the gaps
        if constexpr (RW > 1) __builtin_amdgcn_s_setprio(1);
        f32x4 s[QG][NT];
        if constexpr (kBf) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                b8 kf[ES];
#pragma unroll
                for (int es = 0; es < ES; ++es) kf[es] = f.k[t * ES + es];
#pragma unroll
                for (int qg = 0; qg < QG; ++qg) {
                    s[qg][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int es = 0; es < ES; ++es)
                        s[qg][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[es], qf[qg][es], s[qg][t], 0, 0, 0);
                }
            }
            mfma_settled<8>();
        } else {
            f32x4 so[QG];               // two chains: half the rounding error of one
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) s[qg][0] = so[qg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int es = 0; es < ES; ++es) {
                const f32x4 kf = f.k[es];
#pragma unroll
                for (int qg = 0; qg < QG; ++qg)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        s[qg][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i], qf[qg][es][i], s[qg][0], 0, 0, 0);
                        so[qg] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i + 1], qf[qg][es][i + 1], so[qg], 0, 0, 0);
                    }
            }
            mfma_settled<16>();
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) s[qg][0] += so[qg];
        }
        if constexpr (RW > 1) __builtin_amdgcn_s_setprio(0);
        scored();
        if constexpr (EX) {
            if (a.cap2 > 0.f) {
#pragma unroll
                for (int qg = 0; qg < QG; ++qg)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[qg][t][r] = capped(a, s[qg][t][r]);
            } else {
#pragma unroll
                for (int qg = 0; qg < QG; ++qg)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[qg][t][r] *= a.c;
            }
            if (a.slopes != nullptr) {
#pragma unroll
                for (int qg = 0; qg < QG; ++qg) {
                    const float away = (float)(kabs + 4 * g - rpos[qg]);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[qg][t][r] = fmaf(slope2[qg], away + (float)(16 * t + r), s[qg][t][r]);
                }
            }
        }
        const float c = EX ? 1.f : a.c;
        // keys after a row, past the cache, or behind its window
        if (__builtin_expect(kabs + SB > pfirst + 1 || kabs + SB > k1 || kabs < wlow, 0)) {
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)         // keys seen: low .. low + seen - 1
                        if ((unsigned)(kabs + t * 16 + 4 * g + r - low[qg]) >= (unsigned)seen[qg]) s[qg][t][r] = -INFINITY;
            }
        }
        // the block's largest score of the lane's row (among its own keys)
        auto largest = [&](int qg) __attribute__((always_inline)) {
            const float x = max3(max3(s[qg][0][0], s[qg][0][1], s[qg][0][2]), s[qg][0][3], s[qg][NT - 1][0]);
            if constexpr (NT == 1) return x;
            return max3(max3(x, s[qg][NT - 1][1], s[qg][NT - 1][2]), s[qg][NT - 1][3], x);
        };
        auto move = [&](int qg, float nm) __attribute__((always_inline)) {
            const float alpha = fast_exp2(nm - negm[qg]);
            negm[qg] = nm;
            l[qg] *= alpha;
#pragma unroll
            for (int eb = 0; eb < EB; ++eb)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[qg][eb][r] *= alpha;
        };
        b8 pf[QG];
        auto weigh = [&](int qg) __attribute__((always_inline)) {
            if constexpr (kBf)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) pf[qg][t * 4 + r] = (__bf16)fast_exp2(fmaf(s[qg][t][r], c, negm[qg]));
        };
        // the lane's part of a row's sum, this block added
        const __bf16 u = (__bf16)1.0f;
        auto summed = [&](int qg) __attribute__((always_inline)) {
            float sum = first_of(l[qg]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sum = __builtin_amdgcn_fdot2_f32_bf16(b2{pf[qg][2 * j], pf[qg][2 * j + 1]}, b2{u, u}, sum, false);
            return sum;
        };
        // references that are passed by too much (in the branch the same test
        // again, of the row: it may be another's)
        float top[QG];              // kSums: the new sums
        unsigned most = 0;          // (sums are positive: as integers they need no quieting)
        bool passed = false;
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) {
            if constexpr (kSums) {
                weigh(qg);
                top[qg] = summed(qg);
                most = max(most, __float_as_uint(top[qg]));
            } else {
                top[qg] = largest(qg);
                passed |= fmaf(top[qg], c, negm[qg]) > kSlack;
            }
        }
        if constexpr (kSums) passed = most > __float_as_uint(kMostSum);
        if (__any(passed)) {
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) {
                if constexpr (kSums) {
                    // to the larger of the block's maximum and the weight so far
                    const bool mine = quad_max(top[qg]) > kMostSum;
                    const float x = quad_max(largest(qg));
                    const float so_far = __builtin_amdgcn_logf(quad_sum(first_of(l[qg])));
                    move(qg, mine ? fminf(-(x * c), negm[qg] - so_far) : negm[qg]);
                    weigh(qg);
                    top[qg] = summed(qg);
                } else {
                    const float x = quad_max(top[qg]);
                    move(qg, fmaf(x, c, negm[qg]) > kSlack ? -(x * c) : negm[qg]);
                }
            }
        }
        if constexpr (kBf) {
            if constexpr (!kSums)
#pragma unroll
                for (int qg = 0; qg < QG; ++qg) weigh(qg);
            if constexpr (RW > 1) __builtin_amdgcn_s_setprio(1);
            if constexpr (kOnes) {
                const b8 ones = {u, u, u, u, u, u, u, u};
#pragma unroll
                for (int qg = 0; qg < QG; ++qg)
                    l[qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[qg], l[qg], 0, 0, 0);
            } else {
#pragma unroll
                for (int qg = 0; qg < QG; ++qg) l[qg] = lsum{kSums ? top[qg] : summed(qg)};
            }
#pragma unroll
            for (int eb = 0; eb < EB; ++eb) {
                const b8 vf = f.v[eb];
#pragma unroll
                for (int qg = 0; qg < QG; ++qg)
                    o[qg][eb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[qg], o[qg][eb], 0, 0, 0);
            }
        } else {
            float p[QG][4];
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) {
#pragma unroll
                for (int r = 0; r < 4; ++r) p[qg][r] = fast_exp2(fmaf(s[qg][0][r], c, negm[qg]));
                l[qg] += (p[qg][0] + p[qg][1]) + (p[qg][2] + p[qg][3]);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const vfrag v = f.v[i];
#pragma unroll
                for (int j = 0; j < VW; ++j)
#pragma unroll
                    for (int qg = 0; qg < QG; ++qg) {
                        f32x4& sum = o[qg][i % (EB / VW) * VW + j];
                        sum = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], p[qg][i / (EB / VW)], sum, 0, 0, 0);
                    }
            }
        }
        if constexpr (RW > 1) __builtin_amdgcn_s_setprio(0);
        if constexpr (kBf) mfma_settled<8>(); else mfma_settled<16>();
    };

    if constexpr (RW == 1) {
        // A wave loads the very rows that it reads: no barriers.  Two stages (one,
        // kSingle) are under way to LDS and one from there to registers while a
        // block is computed.  (Stages past the last are loads of nothing: without
        // branches around them the compiler knows that the rows have landed.)
        static_assert(KS == SB, "one block per stage");
        // computes stage st (its fragments in cur), reads stage st + 1 from LDS
        // and loads stage st + 2 where st was
        auto stage = [&](T* cK, T* cV, const T* nK, const T* nV, const Frags& cur, Frags& next, int st)
            __attribute__((always_inline)) {
            if constexpr (!kSingle) {
                wait_lds();
                issue_loads(cK, cV, st + 2);
                fetch_pages(st + 3);
                wait_loads<2 * NI>();
            } else {
                wait_loads<0>();
            }
            __builtin_amdgcn_sched_barrier(0);
            read_ks(nK, kg * KS, next);
            read_vs(nV, kg * KS, next);
            if constexpr (kSingle) {
                wait_lds();
                issue_loads(cK, cV, st + 2);
                fetch_pages(st + 3);
            }
            const int kabs = k0 + st * TS + kg * KS;
            if (kabs < k1 && kabs < wend && kabs + SB > wbeg) sub_block(cur, kabs, [] {});
        };
        if constexpr (!kSingle) wait_loads<4 * NI>();       // the rows
        wait_loads<kSingle ? 0 : 2 * NI>();                 // the first stage
        Frags f0, f1;
        __builtin_amdgcn_sched_barrier(0);
        read_ks(sK0, kg * KS, f0);
        read_vs(sV0, kg * KS, f0);
        if constexpr (kSingle) {
            wait_lds();
            issue_loads(sK0, sV0, 1);
            fetch_pages(2);
        }
        T* const oK = kSingle ? sK0 : sK1;
        T* const oV = kSingle ? sV0 : sV1;
        int st = 0;
        for (; st + 2 <= nst; st += 2) {
            stage(sK0, sV0, oK, oV, f0, f1, st);
            stage(oK, oV, sK0, sV0, f1, f0, st + 1);
        }
        if (st < nst) stage(sK0, sV0, oK, oV, f0, f1, st);
        wait_lds();
        wait_loads<0>();
        __syncthreads();        // (the merge writes over other waves' rows)
    } else {
        auto stage = [&](const T* cK, const T* cV, T* nK, T* nV, int st) __attribute__((always_inline)) {
            if (st + 1 < nst) {
                issue_loads(nK, nV, st + 1);
                fetch_pages(st + 2);
            }
            if (active) {
                // a block's V is read before its scores, the next block's K
                // while its probabilities are computed
                constexpr bool kDeep = D == 128;
                Frags f;
                bool have = false;
#pragma unroll
                for (int i = 0; i < KS / SB; ++i) {
                    const int kabs = k0 + st * TS + i * SB;
                    if (!(kabs < k1 && kabs < wend && kabs + SB > wbeg)) {
                        have = false;
                        continue;
                    }
                    if constexpr (kDeep) {
                        if (!have) read_ks(cK, i * SB, f);
                        read_vs(cV, i * SB, f);
                        sub_block(f, kabs, [&] {
                            if (i + 1 < KS / SB) read_ks(cK, i * SB + SB, f);
                        });
                        have = true;
                    } else {
                        read_ks(cK, i * SB, f);
                        sub_block(f, kabs, [&] { read_vs(cV, i * SB, f); });
                    }
                }
            }
            wait_loads<0>();                    // next stage landed
            __syncthreads();
        };
        wait_loads<0>();
        __syncthreads();
        int st = 0;
        for (; st + 2 <= nst; st += 2) {
            stage(sK0, sV0, sK1, sV1, st);
            stage(sK1, sV1, sK0, sV0, st + 1);
        }
        if (st < nst) stage(sK0, sV0, sK1, sV1, st);
    }

    // ---- key groups meet in LDS (all reads of the stages ended at the last barrier)
    if constexpr (KW > 1) {
        // one slot per wave but the first group's, as many per array as fit
        constexpr int kWords = QG * (EB * 4 + 2), kSlots = TS * D * (int)sizeof(T) / (kWords * 256);
        static_assert(RW == 1 && kSlots >= 1 && (kSingle ? 2 : 4) * kSlots >= KW - 1, "merge space");
        auto slot = [&](int w) __attribute__((always_inline)) {
            const int i = (w - 1) / kSlots;
            return reinterpret_cast<float*>(kSingle ? (i == 0 ? sK0 : sV0) : i == 0 ? sK0 : i == 1 ? sK1 : i == 2 ? sV0 : sV1) +
                   (w - 1) % kSlots * kWords * 64 + lane;
        };
        float* const x = slot(kg > 0 ? kg : 1);
        if (kg > 0) {
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) {
#pragma unroll
                for (int eb = 0; eb < EB; ++eb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[(qg * (EB * 4 + 2) + eb * 4 + r) * 64] = o[qg][eb][r];
                x[(qg * (EB * 4 + 2) + EB * 4) * 64] = negm[qg];
                x[(qg * (EB * 4 + 2) + EB * 4 + 1) * 64] = first_of(l[qg]);
            }
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int w = 1; w < KW; ++w) {
            const float* const y = slot(w);
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) {
                const float nw = y[(qg * (EB * 4 + 2) + EB * 4) * 64];
                const float nm = fminf(negm[qg], nw);
                const float a0 = fast_exp2(nm - negm[qg]), a1 = fast_exp2(nm - nw);
                negm[qg] = nm;
                l[qg] = lsum(l[qg] * a0 + y[(qg * (EB * 4 + 2) + EB * 4 + 1) * 64] * a1);
#pragma unroll
                for (int eb = 0; eb < EB; ++eb)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        o[qg][eb][r] = o[qg][eb][r] * a0 + y[(qg * (EB * 4 + 2) + eb * 4 + r) * 64] * a1;
            }
        }
    }
    if (!active) return;

    // ---- out: this part's state, or the normalised rows
    unsigned long long again = 0;               // rows of the wave to do again
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) {
        float lt = first_of(l[qg]);
        if constexpr (!kOnes) lt = quad_sum(lt);
        const int r = wrow + qg * 16 + l16;
        const bool valid = r < nrows;
        if (it.splits > 1) {
            if (!valid) continue;
            const int64_t rec = (int64_t)blockIdx.x * TR + (r - tile0);
            if (g == 0) {
                a.part_ml[2 * rec] = negm[qg];
                a.part_ml[2 * rec + 1] = lt;
            }
            float* const po = a.part_o + rec * D;
            if constexpr (kBf) {
#pragma unroll
                for (int eb = 0; eb < EB; ++eb) *reinterpret_cast<f32x4*>(po + 16 * eb + 4 * g) = o[qg][eb];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int eb = 0; eb < EB; ++eb) po[EB * (4 * g + i) + eb] = o[qg][eb][i];
            }
            continue;
        }
        const float inv = 1.0f / lt;
        float zero = 0.f;                       // NaN if a value is not finite
#pragma unroll
        for (int eb = 0; eb < EB; ++eb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[qg][eb][i] = keep_f32(o[qg][eb][i] * inv);
                zero = fmaf(o[qg][eb][i], 0.f, zero);
            }
        const bool bad = !finite(zero) || !finite(inv) || !(inv > 0.f);
        const int t = rows.token(r - tile0), h = it.kh * G + rows.head(r - tile0, t);
        const int64_t at = (it.row0 + t) * a.out_ld + (int64_t)h * D;
        if (valid) {
            if constexpr (kBf) {
#pragma unroll
                for (int eb = 0; eb < EB; ++eb) {
                    const int64_t e = at + 16 * eb + 4 * g;
                    const f32x4 v = o[qg][eb];
                    if (a.out_kind == ATTN_OUT_F32)
                        *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + e) = v;
                    else if (a.out_kind == ATTN_OUT_F16)
                        *reinterpret_cast<h4*>(static_cast<f16*>(a.out) + e) = h4{(f16)v[0], (f16)v[1], (f16)v[2], (f16)v[3]};
                    else
                        *reinterpret_cast<b4*>(static_cast<bf16*>(a.out) + e) =
                            b4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j0 = 0; j0 < EB; j0 += VW) {
                        vpart v;
#pragma unroll
                        for (int j = 0; j < VW; ++j) v[j] = o[qg][j0 + j][i];
                        *reinterpret_cast<vpart*>(static_cast<float*>(a.out) + at + EB * (4 * g + i) + j0) = v;
                    }
            }
        }
        unsigned long long any = __ballot(bad && valid);
        any |= any >> 32;
        again |= ((any | any >> 16) & 0xffff) << (16 * qg);
    }
    while (again != 0) {
        const int ri = wrow - tile0 + __ffsll((long long)again) - 1, ti = rows.token(ri);
        again &= again - 1;
        attn_row<T, D>(a, pool, it.user, n, it.row0 + ti, own ? n : pos0 + ti, it.kh * G + rows.head(ri, ti));
    }
}

// Joins the parts of the rows whose keys were split: one wave per row.  The
// records of a tile's part are those of the attention's item ((tile * parts +
// part) * n_kv_heads + head) of its user.
template <typename T, int D>
__global__ __launch_bounds__(64 * kJoinRows) void k_paged_attn_join(AttnArgs a, PagedPool pool, JoinUsers join) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PagedUsers& users = join.users;
    const int i = user_of(users, blockIdx.x);
    const int idx = (int)blockIdx.x - users.item0[i], group = idx / a.n_kv_heads, kh = idx - group * a.n_kv_heads;
    const bool own = a.k_self.p != nullptr;
    const int n = users.rows[i], count = users.count[i];
    const int G = a.n_heads / a.n_kv_heads, nrows = count * G;
    const int r = group * kJoinRows + wave;
    if (r >= nrows) return;
    const int splits = attn_splits(n, count, own, a.window, a.chunk);
    int tile = r / a.tile;
    const int in_tile = r - tile * a.tile;
    if (!own) tile = (nrows + a.tile - 1) / a.tile - 1 - tile;      // (last tiles first)
    const int64_t step = (int64_t)a.n_kv_heads * a.tile;
    const int64_t rec0 = ((int64_t)join.part0[i] + (int64_t)tile * splits * a.n_kv_heads + kh) * a.tile + in_tile;
    // lane j of part s: values E j .. E j + E - 1, of every PP-th part
    constexpr int E = D / 32, PP = 2;
    typedef __attribute__((ext_vector_type(E))) float part;
    const int e0 = (lane & 31) * E, half = lane >> 5;
    float nm = -kUnset, l = 0.f, acc[E];
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] = 0.f;
    for (int s0 = 0; s0 < splits; s0 += 64) {
        // 64 parts' references and sums, one per lane
        const int left = splits - s0 < 64 ? splits - s0 : 64;
        const int64_t rs = rec0 + (int64_t)(s0 + (lane < left ? lane : 0)) * step;
        const float ns = lane < left ? a.part_ml[2 * rs] : -kUnset;
        const float ls = lane < left ? a.part_ml[2 * rs + 1] : 0.f;
        const float nn = fminf(nm, -wave_max(-ns));
        const float alpha = fast_exp2(nn - nm), w = fast_exp2(nn - ns);
        nm = nn;
        l = l * alpha + wave_sum(w * ls);
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] *= alpha;
        // their outputs, PP at a time, eight loads under way
#pragma unroll 8
        for (int s = 0; s < left; s += PP) {
            const int mine = s + half < left ? s + half : s;
            const part v = *reinterpret_cast<const part*>(a.part_o + (rec0 + (int64_t)(s0 + mine) * step) * D + e0);
            const float ws = s + half < left ? __shfl(w, mine, 64) : 0.f;
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] = fmaf(ws, v[j], acc[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] += __shfl_xor(acc[j], 32, 64);
    const float inv = 1.f / l;
    bool bad = !finite(inv) || !(inv > 0.f);
    const int t = r / G, h = kh * G + (r - t * G);
    const int64_t row = (int64_t)users.row0[i] + t, at = row * a.out_ld + (int64_t)h * D + e0;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const float v = keep_f32(acc[j] * inv);
        bad |= !finite(v);
        if (half) continue;
        if (a.out_kind == ATTN_OUT_F16) static_cast<f16*>(a.out)[at + j] = (f16)v;
        else if (a.out_kind == ATTN_OUT_F32) static_cast<float*>(a.out)[at + j] = v;
        else static_cast<T*>(a.out)[at + j] = (T)v;
    }
    if (__any(bad)) attn_row<T, D>(a, pool, users.user[i], n, row, own ? n : n - count + t, h);
}

template <typename T, int D, int QG, int RW, int KW>
void launch_tiles(const AttnArgs& a, const PagedPool& pool, const PagedUsers& users, hipStream_t s) {
    const unsigned grid = (unsigned)users.item0[users.n];
    if (a.cap2 > 0.f || a.slopes != nullptr)
        k_paged_attn<T, D, QG, RW, KW, true><<<grid, 64 * RW * KW, 0, s>>>(a, pool, users);
    else
        k_paged_attn<T, D, QG, RW, KW, false><<<grid, 64 * RW * KW, 0, s>>>(a, pool, users);
}

// go(type, head_dim) of a call.
template <typename Go>
void with_type_and_dim(int dtype, int D, const Go& go) {
    auto at = [&](auto t) {
        if (D == 32) go(t, std::integral_constant<int, 32>{});
        else if (D == 64) go(t, std::integral_constant<int, 64>{});
        else go(t, std::integral_constant<int, 128>{});
    };
    if (dtype == UPR_F32) at(float{}); else at(bf16{});
}

}  // namespace

hipError_t launch_paged_attn(int dtype, const AttnArgs& a, const PagedPool& pool, const PagedUsers& users,
                             hipStream_t s) {
    if (users.item0[users.n] == 0) return hipSuccess;
    with_type_and_dim(dtype, a.D, [&](auto t, auto d) {
        typedef decltype(t) T;
        constexpr int D = decltype(d)::value;
        if constexpr (sizeof(T) == 2) {
            if (a.tile == 32) return launch_tiles<T, D, 2, 1, 4>(a, pool, users, s);
            if (a.tile == 128) return launch_tiles<T, D, 2, 4, 1>(a, pool, users, s);
        }
        launch_tiles<T, D, 1, 1, 4>(a, pool, users, s);
    });
    return hipGetLastError();
}

hipError_t launch_paged_join(int dtype, const AttnArgs& a, const PagedPool& pool, const JoinUsers& join, hipStream_t s) {
    with_type_and_dim(dtype, a.D, [&](auto t, auto d) {
        k_paged_attn_join<decltype(t), decltype(d)::value>
            <<<(unsigned)join.users.item0[join.users.n], 64 * kJoinRows, 0, s>>>(a, pool, join);
    });
    return hipGetLastError();
}

}  // namespace upr
