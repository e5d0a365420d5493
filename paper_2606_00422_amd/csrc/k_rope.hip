// Rotary positions, on their own and in the append of new keys and values to
// a paged cache.
//
//   a' = m (a cos t - b sin t),  b' = m (b cos t + a sin t),  t = p f_i
//
// for the pairs (a, b) of a head's first rot_dim features.  A thread takes a
// unit: VEC features and the VEC they are paired with (half layout), or 2 VEC
// consecutive ones (interleaved pairs, features past rot_dim, values), so both
// layouts read and write 16-byte pieces where rot_dim allows (VEC 1 otherwise).
#include "rope.h"

namespace upr {

namespace {

template <typename T, int VEC>
struct Chunk {
    T v[VEC];
};
template <> struct __attribute__((aligned(16))) Chunk<bf16, 8> { bf16 v[8]; };
template <> struct __attribute__((aligned(16))) Chunk<float, 4> { float v[4]; };

template <typename T, int VEC>
__device__ __forceinline__ void load(const T* p, float (&x)[VEC]) {
    const Chunk<T, VEC> c = *reinterpret_cast<const Chunk<T, VEC>*>(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = (float)c.v[i];
}
template <typename T, int VEC>
__device__ __forceinline__ void store(T* p, const float (&x)[VEC]) {
    Chunk<T, VEC> c;
#pragma unroll
    for (int i = 0; i < VEC; ++i) c.v[i] = (T)keep_f32(x[i]);
    *reinterpret_cast<Chunk<T, VEC>*>(p) = c;
}

// Unit u of one head at position pos (rot: the head is rotated at all).
template <typename T, int VEC>
__device__ __forceinline__ void turn_unit(const RopeArgs& rope, bool rot, int u, int pos, const T* x, T* out) {
    const int r = rot ? rope.rot_dim : 0;
    const bool turned = 2 * u * VEC < r;
    const bool half = turned && rope.layout == UPR_ROPE_HALF;
    const int ia = half ? u * VEC : 2 * u * VEC, ib = half ? ia + r / 2 : ia + VEC;
    float a[VEC], b[VEC];
    load<T, VEC>(x + ia, a);
    load<T, VEC>(x + ib, b);
    if (half) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float c, s;
            rope_angle(pos, rope.quarters[ia + j], rope.magnitude, c, s);
            const float xa = a[j], xb = b[j];
            a[j] = fmaf(xa, c, -(xb * s));
            b[j] = fmaf(xb, c, xa * s);
        }
    } else if (turned) {
        if constexpr (VEC == 1) {
            float c, s;
            rope_angle(pos, rope.quarters[u], rope.magnitude, c, s);
            const float xa = a[0], xb = b[0];
            a[0] = fmaf(xa, c, -(xb * s));
            b[0] = fmaf(xb, c, xa * s);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float(&w)[VEC] = j < VEC / 2 ? a : b;
                const int k = 2 * (j % (VEC / 2));
                float c, s;
                rope_angle(pos, rope.quarters[ia / 2 + j], rope.magnitude, c, s);
                const float xa = w[k], xb = w[k + 1];
                w[k] = fmaf(xa, c, -(xb * s));
                w[k + 1] = fmaf(xb, c, xa * s);
            }
        }
    }
    store<T, VEC>(out + ia, a);
    store<T, VEC>(out + ib, b);
}

template <typename T, int VEC>
__global__ __launch_bounds__(256) void k_rope(RopeArgs rope, int heads, int D, const T* x, int64_t x_ld,
                                              const int32_t* __restrict__ positions, int64_t rows, T* out,
                                              int64_t out_ld) {
    const int upr_ = heads * (D / (2 * VEC));       // units per row
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * upr_) return;
    const int64_t row = i / upr_;
    const int w = (int)(i - row * upr_), h = w / (D / (2 * VEC)), u = w % (D / (2 * VEC));
    turn_unit<T, VEC>(rope, true, u, positions[row], x + row * x_ld + h * D, out + row * out_ld + h * D);
}

// The launch's user that item b belongs to: the last one whose items start at
// or before b.
__device__ __forceinline__ int user_of(const PagedUsers& users, int b) {
    int lo = 0, hi = users.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (users.item0[mid] <= b) lo = mid; else hi = mid - 1;
    }
    return lo;
}

constexpr int kAppendUnits = 256;       // units per work item

template <typename T, int VEC>
__global__ __launch_bounds__(256) void k_append(RopeArgs rope, AppendArgs a, PagedPool pool, PagedUsers users) {
    const int i = user_of(users, blockIdx.x);
    const int per = a.D / (2 * VEC);
    const int kvh = a.k.p != nullptr ? a.n_kv_heads : 0, qh = a.q.p != nullptr ? a.n_heads : 0;
    const int heads = 2 * kvh + qh;
    const int64_t w = (int64_t)((int)blockIdx.x - users.item0[i]) * kAppendUnits + threadIdx.x;
    if (w >= (int64_t)users.count[i] * heads * per) return;
    const int t = (int)(w / (heads * per)), rest = (int)(w % (heads * per));
    const int h = rest / per, u = rest % per;
    const int64_t row = (int64_t)users.row0[i] + t;
    const int pos = a.fixed ? users.rows[i] : users.rows[i] - users.count[i] + t;
    const bool rot = rope.rot_dim > 0;
    if (h >= 2 * kvh) {
        const int64_t off = (int64_t)(h - 2 * kvh) * a.D;
        turn_unit<T, VEC>(rope, rot, u, pos, static_cast<const T*>(a.q.p) + row * a.q.ld + off,
                          static_cast<T*>(a.q_out) + row * a.q_out_ld + off);
        return;
    }
    const bool key = h < kvh;
    const int kh = key ? h : h - kvh;
    const int page = pool.tables[(int64_t)users.user[i] * pool.stride + (pos >> pool.page_shift)];
    if (page < 0 || page >= pool.n_pages) return;
    const RowsOf src = key ? a.k : a.v;
    T* const dst = reinterpret_cast<T*>(pool.data) +
                   ((((int64_t)page * 2 + (key ? 0 : 1)) * kvh + kh) * pool.page_rows + (pos & (pool.page_rows - 1))) *
                       a.D;
    turn_unit<T, VEC>(rope, rot && key, u, pos, static_cast<const T*>(src.p) + row * src.ld + (int64_t)kh * a.D, dst);
}

// 16-byte pieces need both halves of the rotated part to be whole pieces.
template <typename T>
constexpr int wide() { return 16 / (int)sizeof(T); }

}  // namespace

hipError_t launch_rope(int dtype, const RopeArgs& rope, int heads, int D, RowsOf x, const int32_t* positions,
                       int64_t rows, void* out, int64_t out_ld, hipStream_t s) {
    auto go = [&](auto t, auto vec) {
        typedef decltype(t) T;
        constexpr int VEC = decltype(vec)::value;
        const int64_t units = rows * heads * (D / (2 * VEC));
        k_rope<T, VEC><<<(unsigned)((units + 255) / 256), 256, 0, s>>>(rope, heads, D, static_cast<const T*>(x.p),
                                                                      x.ld, positions, rows, static_cast<T*>(out),
                                                                      out_ld);
    };
    if (dtype == UPR_F32) {
        if (rope.rot_dim % (2 * wide<float>()) == 0) go(float{}, std::integral_constant<int, wide<float>()>{});
        else go(float{}, std::integral_constant<int, 1>{});
    } else {
        if (rope.rot_dim % (2 * wide<bf16>()) == 0) go(bf16{}, std::integral_constant<int, wide<bf16>()>{});
        else go(bf16{}, std::integral_constant<int, 1>{});
    }
    return hipGetLastError();
}

static bool append_wide(int dtype, const RopeArgs& rope) {
    return rope.rot_dim % (2 * (dtype == UPR_F32 ? wide<float>() : wide<bf16>())) == 0;
}

int64_t append_items(int dtype, const RopeArgs& rope, const AppendArgs& a, int64_t count) {
    const int vec = append_wide(dtype, rope) ? (dtype == UPR_F32 ? wide<float>() : wide<bf16>()) : 1;
    const int heads = (a.k.p != nullptr ? 2 * a.n_kv_heads : 0) + (a.q.p != nullptr ? a.n_heads : 0);
    return (count * heads * (a.D / (2 * vec)) + kAppendUnits - 1) / kAppendUnits;
}

hipError_t launch_append(int dtype, const RopeArgs& rope, const AppendArgs& a, const PagedPool& pool,
                         const PagedUsers& users, hipStream_t s) {
    const unsigned grid = (unsigned)users.item0[users.n];
    if (grid == 0) return hipSuccess;
    if (dtype == UPR_F32) {
        if (append_wide(dtype, rope)) k_append<float, wide<float>()><<<grid, 256, 0, s>>>(rope, a, pool, users);
        else k_append<float, 1><<<grid, 256, 0, s>>>(rope, a, pool, users);
    } else {
        if (append_wide(dtype, rope)) k_append<bf16, wide<bf16>()><<<grid, 256, 0, s>>>(rope, a, pool, users);
        else k_append<bf16, 1><<<grid, 256, 0, s>>>(rope, a, pool, users);
    }
    return hipGetLastError();
}

}  // namespace upr
