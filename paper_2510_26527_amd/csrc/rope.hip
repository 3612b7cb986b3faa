// Rotary positions on gfx950: pairs of a head's entries turned by angle position * frequency, in either pairing, over all of a
// head or its first entries, at frequencies scaled for long contexts.  Bytes bound it (each entry read and written once, three
// operations), for few rows the launch.
//
// The angle of a far position has to be known to a small part of a turn: position * (frequency / 2 pi) is taken in fp64, cut to
// its fraction of a turn, and only that goes to fp32.  A block works the (cos, sin) of its rows out once, in LDS, for all heads.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "prof.h"
#include "rope.h"
#include "../../include/psd.h"

namespace psd {
namespace {

constexpr int kThreads = 256;
constexpr int kTableMax = 1024;       // (cos, sin) pairs of a block's rows: 4 rows of 256 / 2 frequencies and more of narrower ones

// P consecutive entries as one load or store
template <typename T, int P> struct Pack { typedef __attribute__((ext_vector_type(P))) T type; };
template <typename T> struct Pack<T, 1> { typedef T type; };

template <int P>
__device__ __forceinline__ void widen(const uint16_t *p, float (&v)[P]) {
    const auto raw = *reinterpret_cast<const typename Pack<uint16_t, P>::type *>(p);
    if constexpr (P == 1) v[0] = bf16_bits_to_f32(raw);
    else
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = bf16_bits_to_f32(raw[j]);
}
template <int P>
__device__ __forceinline__ void widen(const float *p, float (&v)[P]) {
    const auto raw = *reinterpret_cast<const typename Pack<float, P>::type *>(p);
    if constexpr (P == 1) v[0] = raw;
    else
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = raw[j];
}
template <int P>
__device__ __forceinline__ void narrow(uint16_t *p, const float (&v)[P]) {
    typename Pack<uint16_t, P>::type r;
    if constexpr (P == 1) r = (uint16_t)f32_to_bf16_bits(v[0]);
    else
#pragma unroll
        for (int j = 0; j < P; ++j) r[j] = (uint16_t)f32_to_bf16_bits(v[j]);
    *reinterpret_cast<typename Pack<uint16_t, P>::type *>(p) = r;
}
template <int P>
__device__ __forceinline__ void narrow(float *p, const float (&v)[P]) {
    typename Pack<float, P>::type r;
    if constexpr (P == 1) r = v[0];
    else
#pragma unroll
        for (int j = 0; j < P; ++j) r[j] = v[j];
    *reinterpret_cast<typename Pack<float, P>::type *>(p) = r;
}

// An item is 2 P entries of one head: P pairs (half pairing: two runs of P, half the rotated width apart; interleaved: one run of
// 2 P), or 2 P entries behind the rotated ones, which are copied.  The first nt items of a head are pairs.  P is the widest that
// divides both parts and that the rows' alignment allows, up to 16 bytes a run.  A block takes `rows` rows and kItems * 256 of
// their items; no loop, every load is on its way before the angles are worked out.  One item a thread, or two where there are millions: us, rows of 40
// heads of 128 bf16 entries, one / two / four: 9 3.2 / 4.0 / 4.0; 1000 6.5 / 7.1 / 8.9; 4000 17.3 / 17.6 / 19.5; 8191 38.4 / 36.7 / 41.6 (in a trace 33.1 = 5.07 TB/s); 16000 69 / 63 / 73.
// Stores past the caches took 30.7 for the 8191, and gave it back to the kernel that reads the result (with it 64.8 / 62.8).
template <typename T, int P, int kItems>
__global__ __launch_bounds__(kThreads) void rope_rotate_kernel(RopeRotateArgs a) {
    __shared__ float2 cs[kTableMax];
    const int tid = threadIdx.x, nf = a.rope.rot / 2, nt = nf / P;
    const int64_t r0 = (int64_t)blockIdx.x * a.block_rows;
    const int rows = (int)min((int64_t)a.block_rows, a.rows - r0);
    const int run = a.rope.interleaved ? P : nf;             // from an item's first run to its second
    float u[kItems][P], v[kItems][P];
    int64_t at[kItems];
    int first[kItems];                                       // an item's first (cos, sin); below zero: a copy
    bool have[kItems];
    auto gap = [&](int k) { return first[k] < 0 ? P : run; };
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const uint32_t item = blockIdx.y * (kThreads * kItems) + k * kThreads + tid;
        const uint32_t row = a.per_row.div(item), in_row = item - row * a.per_row.n;
        const uint32_t head = a.per_head.div(in_row), j = in_row - head * a.per_head.n;
        have[k] = (int)row < rows;
        const int e = (int)j < nt ? (a.rope.interleaved ? 2 * P * j : P * j) : 2 * P * j;
        first[k] = (int)j < nt ? (int)(row * nf + P * j) : -1;
        at[k] = (int64_t)head * a.d_h + e;
        if (have[k]) {
            const T *src = (const T *)a.x + (r0 + row) * a.x_stride + at[k];
            widen<P>(src, u[k]);
            widen<P>(src + gap(k), v[k]);
        }
        at[k] += (r0 + row) * a.y_stride;
    }
    for (int f = tid; f < rows * nf; f += kThreads) {
        const int row = f / nf;
        cs[f] = rope_cs(a.positions[r0 + row], a.turns.v[f - row * nf], a.rope.magnitude);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        if (!have[k]) continue;
        if (first[k] >= 0) {
            if (a.rope.interleaved) {                        // pairs stand side by side in the two runs
                float w[2 * P];
#pragma unroll
                for (int j = 0; j < P; ++j) { w[j] = u[k][j]; w[P + j] = v[k][j]; }
#pragma unroll
                for (int j = 0; j < P; ++j) rope_turn(cs[first[k] + j], w[2 * j], w[2 * j + 1]);
#pragma unroll
                for (int j = 0; j < P; ++j) { u[k][j] = w[j]; v[k][j] = w[P + j]; }
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) rope_turn(cs[first[k] + j], u[k][j], v[k][j]);
            }
        }
        T *dst = (T *)a.y + at[k];
        narrow<P>(dst, u[k]);
        narrow<P>(dst + gap(k), v[k]);
    }
}

// cs[m][i] of the rows of a forward pass, for a model with rotary positions of its own
__global__ __launch_bounds__(64) void rope_table_kernel(float2 *cs, int stride, const int32_t *lens, int R, RopeParams rope, RopeTurns turns,
                                                        TreeShape tree) {
    const int m = blockIdx.x, pos = lens[m / R] + (tree.n ? tree.depth[m % R] : m % R);
    for (int i = threadIdx.x; i < rope.rot / 2; i += 64) cs[(size_t)m * stride + i] = rope_cs(pos, turns.v[i], rope.magnitude);
}

}  // namespace

void launch_rope_rotate(int dtype, RopeRotateArgs a, hipStream_t stream) {
    const int es = dtype == PSD_BF16 ? 2 : 4, nf = a.rope.rot / 2, rest = (a.d_h - a.rope.rot) / 2;
    int P = 16 / es;
    auto fits = [&](int p) {
        const int64_t bytes = p * es;
        return nf % p == 0 && rest % p == 0 && a.d_h % p == 0 && (uintptr_t)a.x % bytes == 0 && (uintptr_t)a.y % bytes == 0 &&
               a.x_stride * es % bytes == 0 && a.y_stride * es % bytes == 0;
    };
    while (!fits(P)) P /= 2;
    a.per_head = FastDiv(a.d_h / 2 / P);
    a.per_row = FastDiv((uint32_t)a.heads * (a.d_h / 2 / P));
    // rows of a block: enough items for all its threads, and no more angles than the table holds
    const int items = (uint64_t)a.rows * a.per_row.n > (1u << 21) ? 2 : 1;
    const uint32_t per_block = kThreads * items, per_row = a.per_row.n;
    int rows = per_row >= per_block ? 1 : (int)(per_block / per_row);
    rows = rows > kTableMax / nf ? kTableMax / nf : rows;
    if (rows > a.rows) rows = (int)a.rows;
    if (rows > 1 && a.rows / rows < 256) rows = a.rows < 256 ? 1 : (int)(a.rows / 256);      // (few rows: more blocks instead)
    a.block_rows = rows;
    const dim3 grid((unsigned)((a.rows + rows - 1) / rows), (rows * per_row + per_block - 1) / per_block);
    ScopedProf sp(PSD_KIND_ROPE, stream);
    auto go = [&](auto type, auto p) {
        using T = decltype(type);
        constexpr int kP = decltype(p)::value;
        if (items == 2) launch_kernel(rope_rotate_kernel<T, kP, 2>, grid, kThreads, 0, stream, a);
        else launch_kernel(rope_rotate_kernel<T, kP, 1>, grid, kThreads, 0, stream, a);
    };
    if (dtype == PSD_BF16) {
        if (P == 8) go((uint16_t)0, Int<8>{});
        else if (P == 4) go((uint16_t)0, Int<4>{});
        else if (P == 2) go((uint16_t)0, Int<2>{});
        else go((uint16_t)0, Int<1>{});
    } else {
        if (P == 4) go(0.f, Int<4>{});
        else if (P == 2) go(0.f, Int<2>{});
        else go(0.f, Int<1>{});
    }
}

void launch_rope_table(float2 *cs, int stride, const int32_t *lens, int M, int R, const RopeParams &rope, const RopeTurns &turns,
                       const TreeShape *tree, hipStream_t stream) {
    ScopedProf sp(PSD_KIND_ROPE, stream);
    launch_kernel(rope_table_kernel, M, 64, 0, stream, cs, stride, lens, R, rope, turns, tree ? *tree : TreeShape{});
}

}  // namespace psd
