// The 8-bit KV cache on gfx950: the step's rows rotated, quantised and appended.
//
// A cache of one layer holds e4m3 codes with one scale for each block of 64 tokens and KV head, K and V apart:
//   k [B][h_kv][max_len][d],  v [B][h_kv][max_len / 64][d][64] (each block transposed),  scales fp32 [B][h_kv][max_len / 64].
// An entry stands for code * scale.  A scale is the smallest power of two that keeps the largest entry written into its block
// within 448, so a code loses nothing to its scale but what e4m3 itself rounds (half a step, 2^-4 of the value; below 2^-6 of the scale
// half of 2^-9): a tighter scale would not be more exact.  A block's scale never falls while older tokens are in it; where new ones need
// a larger one, the older codes are divided by the ratio, a power of two, which only rounds those that fall below 2^-6.
// Positions at or beyond the cached length hold anything: the first token of a block starts its scale anew.
//
// Why e4m3 and a block of 64: the attention kernel turns codes into fp16 exactly, two an instruction, and multiplies a block's
// scores by its scale, one number for every key of a tile; V's tokens stand side by side, as its matrix operand takes them.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "prof.h"
#include "rope.h"
#include "../../include/psd.h"

namespace psd {
namespace {

constexpr int kThreads = 256;
constexpr int kQueryItems = 2;        // items of 16 entries a thread of a query block takes

// Rows of the step: get() is eight consecutive entries of row m from column `at` on, one() a single one.  SlotRows: summed over the
// projection's partial slots in slot order
struct SlotRows {
    const float *p;
    int slots;
    int64_t slot_stride, row_stride;
    __device__ __forceinline__ void get(int64_t m, int64_t at, float (&v)[8]) const {
        const float *src = p + m * row_stride + at;
        f32x8 t = load_f32x8(src);
        int s = 1;
        for (; s + 3 <= slots; s += 3) {                     // three more slots in flight
            const f32x8 x = load_f32x8(src + s * slot_stride), y = load_f32x8(src + (s + 1) * slot_stride), z = load_f32x8(src + (s + 2) * slot_stride);
            t += x; t += y; t += z;
        }
        for (; s < slots; ++s) t += load_f32x8(src + s * slot_stride);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = t[j];
    }
    __device__ __forceinline__ float one(int64_t m, int64_t at) const {
        const float *src = p + m * row_stride + at;
        float t = src[0];
        for (int s = 1; s < slots; ++s) t += src[s * slot_stride];
        return t;
    }
};
template <typename T, bool VEC>
struct PlainRows {
    const T *p;
    int64_t row_stride;
    __device__ __forceinline__ void get(int64_t m, int64_t at, float (&v)[8]) const {
        const T *src = p + m * row_stride + at;
        if constexpr (!VEC) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = load_elem(src, j);
        } else if constexpr (sizeof(T) == 2) {
            const u32x4 raw = *reinterpret_cast<const u32x4 *>(src);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (j & 1) ? __uint_as_float(raw[j >> 1] & 0xffff0000u) : __uint_as_float(raw[j >> 1] << 16);
        } else {
            const f32x8 t = load_f32x8(src);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = t[j];
        }
    }
    __device__ __forceinline__ float one(int64_t m, int64_t at) const { return load_elem(p + m * row_stride + at, 0); }
};

// Item j of a head: sixteen entries, two runs of eight at e[0] and e[1].  While eight divides the rotated part evenly these are eight
// pairs (half pairing: rot / 2 apart; interleaved: side by side), or entries behind the rotated part; else (ODD) sixteen in a row,
// and each finds its partner by itself.
struct Item { int e0, e1, freq; };                           // freq < 0: nothing turns
__device__ __forceinline__ Item item_of(int j, int rot, bool interleaved) {
    if (16 * j >= rot) return Item{16 * j, 16 * j + 8, -1};
    if (interleaved) return Item{16 * j, 16 * j + 8, 8 * j};
    return Item{8 * j, 8 * j + rot / 2, 8 * j};
}
template <typename CS>
__device__ __forceinline__ void turn_item(const Item &it, bool interleaved, float (&u)[8], float (&v)[8], const CS &cs) {
    if (it.freq < 0) return;
    if (interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) rope_turn(cs(it.freq + j), u[2 * j], u[2 * j + 1]);
#pragma unroll
        for (int j = 0; j < 4; ++j) rope_turn(cs(it.freq + 4 + j), v[2 * j], v[2 * j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) rope_turn(cs(it.freq + j), u[j], v[j]);
    }
}
// entry e of the rotated head, its partner read beside it
template <typename Rows, typename CS>
__device__ __forceinline__ float turned_entry(const Rows &x, int64_t m, int64_t at, int e, int rot, bool interleaved, const CS &cs) {
    float a = x.one(m, at + e);
    if (e >= rot) return a;
    const int half = rot / 2;
    const bool second = interleaved ? (e & 1) : e >= half;
    const int other = interleaved ? (e ^ 1) : (second ? e - half : e + half), f = interleaved ? e >> 1 : (second ? e - half : e);
    float b = x.one(m, at + other);
    if (second) { rope_turn(cs(f), b, a); return a; }
    rope_turn(cs(f), a, b);
    return a;
}
// an item's sixteen entries, rotated: rot 0 for values
template <bool ODD, typename Rows, typename CS>
__device__ __forceinline__ Item load_item(const Rows &x, int64_t m, int64_t at, int j, int rot, bool interleaved, float (&u)[8], float (&v)[8], const CS &cs) {
    if constexpr (ODD) {
        for (int k = 0; k < 8; ++k) {
            u[k] = turned_entry(x, m, at, 16 * j + k, rot, interleaved, cs);
            v[k] = turned_entry(x, m, at, 16 * j + 8 + k, rot, interleaved, cs);
        }
        return Item{16 * j, 16 * j + 8, -1};
    } else {
        const Item it = item_of(j, rot, interleaved);
        x.get(m, at + it.e0, u);
        x.get(m, at + it.e1, v);
        return it;
    }
}

// the smallest e in -40 .. 40 with amax <= 448 * 2^e (448 = 1.75 * 2^8)
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t w = __float_as_uint(amax);
    const int e = (int)(w >> 23) - 127 - 8 + ((w & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, -40), 40);
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
// Four values as codes, round to nearest even.  Those beyond the largest scale's reach are cut to 448; an infinity has no code and becomes NaN.
__device__ __forceinline__ float in_range(float x) {
    const float c = fminf(fmaxf(x, -448.f), 448.f);          // (NaN would come out as a number)
    return fabsf(x) < INFINITY ? c : __int_as_float(0x7fc00000);
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(a), in_range(b), 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(c), in_range(d), r, true);
    return (uint32_t)r;
}
// four codes, each divided by a power of two
__device__ __forceinline__ uint32_t shrink4(uint32_t w, float ratio) {
    const float a = __builtin_amdgcn_cvt_f32_fp8((int)w, 0), b = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    const float c = __builtin_amdgcn_cvt_f32_fp8((int)w, 2), d = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * ratio, b * ratio, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c * ratio, d * ratio, r, true);
    return (uint32_t)r;
}

// One launch, blocks of two kinds.  The first `units` blocks: the new tokens of one cache block of one KV head, K or V.  Thread t has the
// items t and t + 256 of 64 rows x d / 16: their entries stay in registers from the one read, through the block's maximum, to
// the codes.  The others rotate the query heads of up to 16 rows, 512 items, by angles that the block works out once for all heads.
// What bounds it: bytes for prompts (4001 rows of 32 query and 8 KV heads of 128, bf16: 22.8 us = 4.0 TB/s), the chain load -> maximum -> scale -> store for
// few rows (9 rows, 32 and 32 heads: 5.5 us; 64 sequences of one row, 32 and 8: 7.4).  Why 64 rows of a KV head to a block: a scale's
// tokens meet in one block, so no maximum crosses blocks, and a unit's 16 KB fit the registers.
template <typename Rows, typename TQ, bool ODD>
__global__ __launch_bounds__(kThreads) void kv8_append_kernel(Kv8AppendArgs a, Rows xq, Rows xk, Rows xv) {
    __shared__ float s_row[kKv8Block];                       // row scales
    __shared__ float s_top[4];
    __shared__ __attribute__((aligned(16))) uint8_t s_codes[kKv8Block * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int d = a.d_h, per_head = d / 16, R = a.R;
    const int rot = a.rope.rot;
    const bool interleaved = a.rope.interleaved;
    // (cos, sin) of a row: from the forward pass' table, or worked out here
    auto cs_of = [&](int64_t m, int pos, int f) {
        return a.cs ? a.cs[m * a.cs_stride + f] : rope_cs(pos, a.turns.v[f], a.rope.magnitude);
    };
    auto row_scale = [&](int64_t m, int n) {                 // s_row[i] <- the norm's scale of row m + i, i < n
        for (int i = wave; i < n; i += 4) {
            float ssq = 0.f;
            for (int t = lane; t < a.rs.tiles; t += 64) ssq += a.rs.sumsq[(size_t)t * a.B * R + m + i];
            ssq = wave_sum(ssq);
            if (lane == 0) s_row[i] = 1.0f / sqrtf(ssq * a.rs.inv_d + a.rs.eps);
        }
        __syncthreads();
    };

    if ((int)blockIdx.x >= a.units) {
        const int part = (blockIdx.x - a.units) % a.q_parts, m0 = (blockIdx.x - a.units) / a.q_parts * a.q_rows;
        const int rows = min(a.q_rows, a.B * R - m0), left = rows * (int)a.per_row.n - part * (kThreads * kQueryItems);
        float2 *cs = reinterpret_cast<float2 *>(s_codes);    // [rows][rot / 2], worked out once for all heads
        auto place = [&](int m) { return min(max(a.lens[a.by_r.div(m)], 0), a.max_len) + m - (int)a.by_r.div(m) * R; };
        float u[kQueryItems][8], v[kQueryItems][8];
        Item it[kQueryItems];
        int row[kQueryItems], head[kQueryItems], j[kQueryItems];
#pragma unroll
        for (int k = 0; k < kQueryItems; ++k) {
            const int i = min(k * kThreads + tid, left - 1) + part * (kThreads * kQueryItems);
            row[k] = a.per_row.div(i);
            const int in_row = i - row[k] * (int)a.per_row.n;
            head[k] = in_row / per_head;
            j[k] = in_row % per_head;
            if constexpr (!ODD) it[k] = load_item<ODD>(xq, m0 + row[k], (int64_t)head[k] * d, j[k], rot, interleaved, u[k], v[k], [](int) { return float2{}; });
        }
        for (int f = tid; f < rows * (rot / 2); f += kThreads) {
            const int r = f / (rot / 2);
            cs[f] = cs_of(m0 + r, a.cs ? 0 : place(m0 + r), f - r * (rot / 2));
        }
        __syncthreads();
        if constexpr (ODD) {
#pragma unroll
            for (int k = 0; k < kQueryItems; ++k)
                it[k] = load_item<ODD>(xq, m0 + row[k], (int64_t)head[k] * d, j[k], rot, interleaved, u[k], v[k], [&](int f) { return cs[row[k] * (rot / 2) + f]; });
            __syncthreads();                                 // partners are read across threads: in place, before any is written
        }
        if (a.rs.sumsq) row_scale(m0, rows);
#pragma unroll
        for (int k = 0; k < kQueryItems; ++k) {
            if (k * kThreads + tid >= left) continue;
            turn_item(it[k], interleaved, u[k], v[k], [&](int f) { return cs[row[k] * (rot / 2) + f]; });
            const float sc = a.rs.sumsq ? s_row[row[k]] : 1.0f;
            TQ *dst = (TQ *)a.q_out + (m0 + row[k]) * a.q_out_stride + (int64_t)head[k] * d;
#pragma unroll
            for (int e = 0; e < 8; ++e) { u[k][e] *= sc; v[k][e] *= sc; }
            if (a.q_vec) {
                if constexpr (sizeof(TQ) == 2) {
                    const u32x4 w0{pack_bf16x2(u[k][0], u[k][1]), pack_bf16x2(u[k][2], u[k][3]), pack_bf16x2(u[k][4], u[k][5]), pack_bf16x2(u[k][6], u[k][7])};
                    const u32x4 w1{pack_bf16x2(v[k][0], v[k][1]), pack_bf16x2(v[k][2], v[k][3]), pack_bf16x2(v[k][4], v[k][5]), pack_bf16x2(v[k][6], v[k][7])};
                    if (a.q_past) {
                        __builtin_nontemporal_store(w0, reinterpret_cast<u32x4 *>(dst + it[k].e0));
                        __builtin_nontemporal_store(w1, reinterpret_cast<u32x4 *>(dst + it[k].e1));
                    } else {
                        *reinterpret_cast<u32x4 *>(dst + it[k].e0) = w0;
                        *reinterpret_cast<u32x4 *>(dst + it[k].e1) = w1;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        *reinterpret_cast<f32x4 *>(dst + it[k].e0 + e) = f32x4{u[k][e], u[k][e + 1], u[k][e + 2], u[k][e + 3]};
                        *reinterpret_cast<f32x4 *>(dst + it[k].e1 + e) = f32x4{v[k][e], v[k][e + 1], v[k][e + 2], v[k][e + 3]};
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    store_elem(dst, it[k].e0 + e, u[k][e]);
                    store_elem(dst, it[k].e1 + e, v[k][e]);
                }
            }
        }
        return;
    }

    const bool values = blockIdx.x & 1;
    const int hk = (blockIdx.x >> 1) % a.h_kv, bj = (blockIdx.x >> 1) / a.h_kv, b = bj % a.B, j = bj / a.B;
    const int len = min(max(a.lens[b], 0), a.max_len), end = min(len + R, a.max_len);      // never write outside
    const int block = len / kKv8Block + j, t0 = block * kKv8Block;
    const int lo = max(len, t0), hi = min(end, t0 + kKv8Block), n = hi - lo, held = lo - t0;
    if (n <= 0) return;                                      // (the same for the whole block)
    const int64_t m0 = (int64_t)b * R + (lo - len);          // the block's first new row
    const int64_t at = (int64_t)hk * d;
    float u[2][8], v[2][8];
    Item it[2];
    const int items = n * per_head;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = k * kThreads + tid;
        if (i >= items) continue;
        const int r = i / per_head;
        if (values) it[k] = load_item<false>(xv, m0 + r, at, i % per_head, 0, interleaved, u[k], v[k], [](int) { return make_float2(1.f, 0.f); });
        else it[k] = load_item<ODD>(xk, m0 + r, at, i % per_head, rot, interleaved, u[k], v[k], [&](int f) { return cs_of(m0 + r, lo + r, f); });
    }
    const size_t head_block = ((size_t)b * a.h_kv + hk) * (a.max_len / kKv8Block) + block;
    float *scale_at = (values ? a.v_scale : a.k_scale) + head_block;
    const float before = held ? *scale_at : 0.f;
    if (a.rs.sumsq) row_scale(m0, n);
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = k * kThreads + tid;
        if (i >= items) continue;
        const int r = i / per_head;
        if (!values) turn_item(it[k], interleaved, u[k], v[k], [&](int f) { return cs_of(m0 + r, lo + r, f); });
        const float sc = a.rs.sumsq ? s_row[r] : 1.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[k][e] *= sc;
            v[k][e] *= sc;
            if (fabsf(u[k][e]) < INFINITY) top = fmaxf(top, fabsf(u[k][e]));               // what is no number has no part in the scale
            if (fabsf(v[k][e]) < INFINITY) top = fmaxf(top, fabsf(v[k][e]));
        }
    }
    top = wave_top_f(top);
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    float scale = power_of_two(scale_exponent(top));
    scale = held ? fmaxf(scale, before) : scale;
    const float inv = 1.0f / scale;                          // exact
    const bool grown = held && scale > before;
    if (tid == 0) *scale_at = scale;
    const float ratio = before * inv;

    if (!values) {
        uint8_t *dst = (uint8_t *)a.k_codes + (((size_t)b * a.h_kv + hk) * a.max_len + t0) * d;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = k * kThreads + tid;
            if (i >= items) continue;
            uint8_t *row = dst + (size_t)(held + i / per_head) * d;
            *reinterpret_cast<uint2 *>(row + it[k].e0) = make_uint2(codes4(u[k][0] * inv, u[k][1] * inv, u[k][2] * inv, u[k][3] * inv),
                                                                   codes4(u[k][4] * inv, u[k][5] * inv, u[k][6] * inv, u[k][7] * inv));
            *reinterpret_cast<uint2 *>(row + it[k].e1) = make_uint2(codes4(v[k][0] * inv, v[k][1] * inv, v[k][2] * inv, v[k][3] * inv),
                                                                   codes4(v[k][4] * inv, v[k][5] * inv, v[k][6] * inv, v[k][7] * inv));
        }
        if (grown)
            for (int i = tid; i < held * per_head; i += kThreads) {
                u32x4 *p = reinterpret_cast<u32x4 *>(dst) + i;
                u32x4 w = *p;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = shrink4(w[e], ratio);
                *p = w;
            }
        return;
    }
    // values: the codes through LDS, so that each entry's tokens leave side by side, sixteen to a store; a store that holds older tokens
    // or ones behind the new ones takes theirs from the cache
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = k * kThreads + tid;
        if (i >= items) continue;
        uint8_t *row = s_codes + (held + i / per_head) * d;
        *reinterpret_cast<uint2 *>(row + it[k].e0) = make_uint2(codes4(u[k][0] * inv, u[k][1] * inv, u[k][2] * inv, u[k][3] * inv),
                                                               codes4(u[k][4] * inv, u[k][5] * inv, u[k][6] * inv, u[k][7] * inv));
        *reinterpret_cast<uint2 *>(row + it[k].e1) = make_uint2(codes4(v[k][0] * inv, v[k][1] * inv, v[k][2] * inv, v[k][3] * inv),
                                                               codes4(v[k][4] * inv, v[k][5] * inv, v[k][6] * inv, v[k][7] * inv));
    }
    __syncthreads();
    uint8_t *dst = (uint8_t *)a.v_codes + head_block * kKv8Block * d;
    const int first = grown ? 0 : held / 16, last = (held + n + 15) / 16;
    for (int i = tid; i < (last - first) * d; i += kThreads) {
        const int e = i % d, c = first + i / d;              // entry, group of sixteen tokens
        u32x4 *p = reinterpret_cast<u32x4 *>(dst + (size_t)e * kKv8Block) + c;
        u32x4 w{0u, 0u, 0u, 0u};
        const bool whole = held <= 16 * c && held + n >= 16 * c + 16;
        if (!whole) w = *p;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t old = grown ? shrink4(w[q], ratio) : w[q];
            uint32_t r = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 16 * c + 4 * q + k, sh = 8 * k;
                if (t < held) r |= old & (255u << sh);
                else if (t < held + n) r |= (uint32_t)s_codes[t * d + e] << sh;
                else r |= w[q] & (255u << sh);
            }
            w[q] = r;
        }
        *p = w;
    }
}

}  // namespace

// the append launch's division: rows of a block of queries (16 rows of 64 angles fill the LDS), blocks of a group of rows, blocks of keys and values
struct AppendShape { int q_rows, q_parts; long units, blocks; };
static AppendShape append_shape(int B, int R, int h_q, int h_kv, int d_h) {
    const int per_row = h_q * (d_h / 16), per_block = kThreads * kQueryItems;
    AppendShape s{1, 1, 2L * B * h_kv * ((R + kKv8Block - 2) / kKv8Block + 1), 0};         // at most so many blocks of tokens of one sequence
    s.blocks = s.units;
    if (!h_q) return s;
    s.q_rows = per_row >= per_block ? 1 : per_block / per_row < 16 ? per_block / per_row : 16;
    s.q_parts = (s.q_rows * per_row + per_block - 1) / per_block;
    s.blocks += ((long)B * R + s.q_rows - 1) / s.q_rows * s.q_parts;
    return s;
}
long kv8_append_grid(int B, int R, int h_q, int h_kv, int d_h) { return append_shape(B, R, h_q, h_kv, d_h).blocks; }

void launch_kv8_append(const Kv8AppendArgs &args, const Kv8Source &src, hipStream_t stream) {
    Kv8AppendArgs a = args;
    const AppendShape shape = append_shape(a.B, a.R, a.q_out ? a.h_q : 0, a.h_kv, a.d_h);
    a.units = (int)shape.units;
    a.q_rows = shape.q_rows;
    a.q_parts = shape.q_parts;
    a.per_row = FastDiv(a.h_q * (a.d_h / 16));
    a.by_r = FastDiv(a.R);
    const unsigned grid = (unsigned)shape.blocks;
    const bool odd = a.rope.rot % 16 != 0;
    const int out_es = src.bf16 ? 2 : 4;
    a.q_vec = (uintptr_t)a.q_out % 16 == 0 && a.q_out_stride * out_es % 16 == 0;
    // Many rotated queries go past the caches.  us, append alone and with the attention behind it, rows of 32 heads of 128: 200 rows through them 7.5, 15.9, past them 7.4, 16.1;
    // 500 7.9, 27.6 and 7.6, 27.3; 1000 10.1, 39.1 and 9.1, 38.8; 4001 25.4, 174 and 21.8, 173.
    a.q_past = (int64_t)a.B * a.R * a.h_q * a.d_h * out_es >= 4 << 20;
    ScopedProf sp(PSD_KIND_ROPE_APPEND, stream);
    auto go = [&](auto rows, auto tq) {
        using Rows = decltype(rows(nullptr, 0));
        using TQ = decltype(tq);
        const Rows q = rows(src.q, src.q_stride), k = rows(src.k, src.k_stride), v = rows(src.v, src.v_stride);
        if (odd) launch_kernel(kv8_append_kernel<Rows, TQ, true>, grid, kThreads, 0, stream, a, q, k, v);
        else launch_kernel(kv8_append_kernel<Rows, TQ, false>, grid, kThreads, 0, stream, a, q, k, v);
    };
    auto aligned = [&](const void *p, int64_t stride) { return (uintptr_t)p % 16 == 0 && stride * (src.bf16 ? 2 : 4) % 16 == 0; };
    const bool vec = (!a.q_out || aligned(src.q, src.q_stride)) && aligned(src.k, src.k_stride) && aligned(src.v, src.v_stride);
    if (src.slots) {
        go([&](const void *p, int64_t stride) { return SlotRows{(const float *)p, src.slots, src.slot_stride, stride}; }, 0.f);
    } else if (src.bf16) {
        if (vec) go([](const void *p, int64_t stride) { return PlainRows<uint16_t, true>{(const uint16_t *)p, stride}; }, (uint16_t)0);
        else go([](const void *p, int64_t stride) { return PlainRows<uint16_t, false>{(const uint16_t *)p, stride}; }, (uint16_t)0);
    } else {
        if (vec) go([](const void *p, int64_t stride) { return PlainRows<float, true>{(const float *)p, stride}; }, 0.f);
        else go([](const void *p, int64_t stride) { return PlainRows<float, false>{(const float *)p, stride}; }, 0.f);
    }
}

}  // namespace psd
