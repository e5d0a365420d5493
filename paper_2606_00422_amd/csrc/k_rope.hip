// Rotary positions, on their own and in the append of new keys and values to
// a paged cache.
//
//   a' = m (a cos t - b sin t),  b' = m (b cos t + a sin t),  t = p f_i
//
// for the pairs (a, b) of a head's first rot_dim features.  A thread takes a
// unit: VEC features and the VEC they are paired with (half layout), or 2 VEC
// consecutive ones (interleaved pairs, features past rot_dim, values), so both
// layouts read and write 16-byte pieces where rot_dim allows (VEC 1 otherwise),
// of several heads of its row: the angles are the same for all of them.
//
// Every element is read once and written once, so large calls take the memory's
// time (MI355X; a 1 GB copy moves 4.8 to 5.2 TB/s): 32768 rows of 32 heads of 128
// values of bf16, 537 MB, 97 to 99 us, 5.4 TB/s; the append of 62,830 rows of 8
// heads of 64, queries too, 386 MB, 73 to 82 us, 4.7 to 5.3 TB/s.  A small call is
// a launch: 64 single rows 4.6 us in a graph.
#include <algorithm>
#include <type_traits>

#include "paged_dev.h"

namespace upr {

namespace {

template <typename T, int VEC>
struct Chunk {
    T v[VEC];
};
template <> struct __attribute__((aligned(16))) Chunk<bf16, 8> { bf16 v[8]; };
template <> struct __attribute__((aligned(16))) Chunk<float, 4> { float v[4]; };

// The same pieces as plain bits.
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
template <int BYTES>
using Raw = std::conditional_t<BYTES == 16, u32x4, std::conditional_t<BYTES == 4, unsigned, unsigned short>>;

// A thread's unit of some heads at one position: where its two pieces stand,
// and the cosines and sines of its VEC pairs.
template <int VEC>
struct Unit {
    int ia, ib;
    bool turned, half;
    float c[VEC], s[VEC];

    __device__ __forceinline__ Unit(const RopeArgs& rope, int u, int pos) {
        turned = 2 * u * VEC < rope.rot_dim;
        half = turned && rope.layout == UPR_ROPE_HALF;
        ia = half ? u * VEC : 2 * u * VEC;
        ib = half ? ia + rope.rot_dim / 2 : ia + VEC;
        if (!turned) return;
        // either way its pairs are u VEC .. u VEC + VEC - 1
#pragma unroll
        for (int j = 0; j < VEC; ++j) rope_angle(pos, rope.quarters[u * VEC + j], rope.magnitude, c[j], s[j]);
    }
    // The unit's two pieces turned (copied bit for bit where it is not).
    template <typename T>
    __device__ __forceinline__ void turn(Chunk<T, VEC>& a, Chunk<T, VEC>& b) const {
        auto pair = [&](T& x, T& y, int j) {
            const float xa = (float)x, xb = (float)y;
            x = (T)keep_f32(fmaf(xa, c[j], -(xb * s[j])));
            y = (T)keep_f32(fmaf(xb, c[j], xa * s[j]));
        };
        if (half || (VEC == 1 && turned)) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) pair(a.v[j], b.v[j], j);
        } else if (turned) {
            if constexpr (VEC > 1) {
#pragma unroll
                for (int j = 0; j < VEC / 2; ++j) {
                    pair(a.v[2 * j], a.v[2 * j + 1], j);
                    pair(b.v[2 * j], b.v[2 * j + 1], VEC / 2 + j);
                }
            }
        }
    }
};

// Heads h0, h0 + step, .. of one row, kBatch at a time: all of a batch's loads
// are under way before its first store.
template <typename T, int VEC, int kBatch, bool TURN>
__device__ __forceinline__ void row_heads(const Unit<VEC>& unit, int h0, int step, int heads, int64_t x_step,
                                          int64_t out_step, const T* x, T* out) {
    for (int h = h0; h < heads; h += kBatch * step) {
        typedef std::conditional_t<TURN, Chunk<T, VEC>, Raw<VEC * sizeof(T)>> C;
        C a[kBatch], b[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            // (past the last head: the last one again, not stored)
            const T* const p = x + (h + i * step < heads ? h + i * step : heads - 1) * x_step;
            a[i] = *reinterpret_cast<const C*>(p + unit.ia);
            b[i] = *reinterpret_cast<const C*>(p + unit.ib);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if constexpr (TURN) unit.turn(a[i], b[i]);
            if (h + i * step < heads) {
                T* const p = out + (h + i * step) * out_step;
                *reinterpret_cast<C*>(p + unit.ia) = a[i];
                *reinterpret_cast<C*>(p + unit.ib) = b[i];
            }
        }
    }
}

// A row's threads: `groups` of D / (2 VEC), group j taking heads j, j + groups,
// ..: `batch` heads of a tensor each (they share the angles and have their
// loads under way together), as far as a block of 256 threads has groups.
struct Split {
    int groups, rows;       // rows per block
};
__host__ __device__ __forceinline__ Split split_row(int vec, int batch, int heads, int D) {
    const int units = D / (2 * vec), most = 256 / units;
    const int groups = (heads + batch - 1) / batch;
    Split s;
    s.groups = groups < most ? groups : most;
    s.rows = 256 / (s.groups * units);
    return s;
}

// Heads per thread: 4 in calls that fill the device many times over, where the
// memory's rate counts (append of 62,830 rows: 123 us with 1, 80 with 4), else
// 1 (64 rows: 5.9 us with 1, 11.9 with 4).
constexpr int64_t kManyThreads = int64_t{1} << 20;
inline int batch_of(int64_t rows, int heads, int D, int vec) {
    return rows * heads * (D / (2 * vec)) >= kManyThreads ? 4 : 1;
}

template <typename T, int VEC, int kBatch>
__global__ __launch_bounds__(256) void k_rope(RopeArgs rope, int heads, int D, const T* x, int64_t x_ld,
                                              const int32_t* __restrict__ positions, int64_t rows, T* out,
                                              int64_t out_ld) {
    const int units = D / (2 * VEC);
    const Split sp = split_row(VEC, kBatch, heads, D);
    const int t = threadIdx.x / (units * sp.groups), rest = threadIdx.x - t * units * sp.groups;
    const int64_t row = (int64_t)blockIdx.x * sp.rows + t;
    if (t >= sp.rows || row >= rows) return;
    const Unit<VEC> unit(rope, rest % units, positions[row]);
    row_heads<T, VEC, kBatch, true>(unit, rest / units, sp.groups, heads, D, D, x + row * x_ld, out + row * out_ld);
}

template <typename T, int VEC, int kBatch>
__global__ __launch_bounds__(256) void k_append(RopeArgs rope, AppendArgs a, PagedPool pool, PagedUsers users) {
    const int i = user_of(users, blockIdx.x);
    const int units = a.D / (2 * VEC);
    const int kvh = a.k.p != nullptr ? a.n_kv_heads : 0, qh = a.q.p != nullptr ? a.n_heads : 0;
    const Split sp = split_row(VEC, kBatch, kvh > qh ? kvh : qh, a.D);
    const int tr = threadIdx.x / (units * sp.groups), rest = threadIdx.x - tr * units * sp.groups;
    const int t = ((int)blockIdx.x - users.item0[i]) * sp.rows + tr;
    if (tr >= sp.rows || t >= users.count[i]) return;
    const int64_t row = (int64_t)users.row0[i] + t;
    const int pos = a.fixed ? users.rows[i] : users.rows[i] - users.count[i] + t;
    const int h0 = rest / units;
    int page = -1;
    if (kvh > 0) page = pool.tables[(int64_t)users.user[i] * pool.stride + (pos >> pool.page_shift)];
    const Unit<VEC> unit(rope, rest % units, pos);
    if (qh > 0)
        row_heads<T, VEC, kBatch, true>(unit, h0, sp.groups, qh, a.D, a.D, static_cast<const T*>(a.q.p) + row * a.q.ld,
                                static_cast<T*>(a.q_out) + row * a.q_out_ld);
    if (page < 0 || page >= pool.n_pages) return;
    const int64_t plane = (int64_t)pool.page_rows * a.D;        // one head's rows of the page
    T* const dst = reinterpret_cast<T*>(pool.data) + (int64_t)page * 2 * kvh * plane +
                   (int64_t)(pos & (pool.page_rows - 1)) * a.D;
    row_heads<T, VEC, kBatch, true>(unit, h0, sp.groups, kvh, a.D, plane, static_cast<const T*>(a.k.p) + row * a.k.ld, dst);
    row_heads<T, VEC, kBatch, false>(unit, h0, sp.groups, kvh, a.D, plane, static_cast<const T*>(a.v.p) + row * a.v.ld,
                             dst + kvh * plane);
}

// 16-byte pieces need both halves of the rotated part to be whole pieces.
template <typename T>
constexpr int wide() { return 16 / (int)sizeof(T); }
int vec_of(int dtype, const RopeArgs& rope) {
    const int v = dtype == UPR_F32 ? wide<float>() : wide<bf16>();
    return rope.rot_dim % (2 * v) == 0 ? v : 1;
}

// go(type, VEC, batch) for those values.
template <typename Go>
void with_types(int dtype, int vec, int batch, const Go& go) {
    auto at = [&](auto t, auto v) {
        if (batch == 1) go(t, v, std::integral_constant<int, 1>{});
        else go(t, v, std::integral_constant<int, 4>{});
    };
    typedef std::integral_constant<int, 1> one;
    if (dtype == UPR_F32) {
        if (vec == 1) at(float{}, one{});
        else at(float{}, std::integral_constant<int, wide<float>()>{});
    } else {
        if (vec == 1) at(bf16{}, one{});
        else at(bf16{}, std::integral_constant<int, wide<bf16>()>{});
    }
}

}  // namespace

hipError_t launch_rope(int dtype, const RopeArgs& rope, int heads, int D, RowsOf x, const int32_t* positions,
                       int64_t rows, void* out, int64_t out_ld, hipStream_t s) {
    const int vec = vec_of(dtype, rope), batch = batch_of(rows, heads, D, vec);
    const int64_t per = split_row(vec, batch, heads, D).rows;
    with_types(dtype, vec, batch, [&](auto t, auto v, auto b) {
        typedef decltype(t) T;
        const int64_t most = (int64_t{1} << 23) * per;      // (a launch has fewer than 2^32 threads)
        for (int64_t r0 = 0; r0 < rows; r0 += most) {
            const int64_t n = rows - r0 < most ? rows - r0 : most;
            k_rope<T, decltype(v)::value, decltype(b)::value><<<(unsigned)((n + per - 1) / per), 256, 0, s>>>(
                rope, heads, D, static_cast<const T*>(x.p) + r0 * x.ld, x.ld, positions + r0, n,
                static_cast<T*>(out) + r0 * out_ld, out_ld);
        }
    });
    return hipGetLastError();
}

static int append_heads(const AppendArgs& a) {
    return std::max(a.k.p != nullptr ? a.n_kv_heads : 0, a.q.p != nullptr ? a.n_heads : 0);
}

int append_batch(int dtype, const RopeArgs& rope, const AppendArgs& a, int64_t rows) {
    return batch_of(rows, append_heads(a), a.D, vec_of(dtype, rope));
}

int append_rows(int dtype, const RopeArgs& rope, const AppendArgs& a, int batch) {
    return split_row(vec_of(dtype, rope), batch, append_heads(a), a.D).rows;
}

hipError_t launch_append(int dtype, const RopeArgs& rope, const AppendArgs& a, int batch, const PagedPool& pool,
                         const PagedUsers& users, hipStream_t s) {
    const unsigned grid = (unsigned)users.item0[users.n];
    if (grid == 0) return hipSuccess;
    with_types(dtype, vec_of(dtype, rope), batch, [&](auto t, auto v, auto b) {
        k_append<decltype(t), decltype(v)::value, decltype(b)::value><<<grid, 256, 0, s>>>(rope, a, pool, users);
    });
    return hipGetLastError();
}

}  // namespace upr
