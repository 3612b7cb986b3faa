// Attention over the 8-bit KV cache (kv8.hip) on gfx950: out = softmax(scale * q K^T) V, row r of a sequence seeing positions
// 0 .. len + r, in one pass over the keys with a running reference and sum.
//
// The codes become fp16, exactly, two an instruction, in the registers they were loaded into; both products run on the fp16
// matrix cores.  A block's 64 keys share their scales, so K's multiplies the scores (with the softmax scale and log2 e, one number a
// query and block), and V's rides in the weights: a weight is 2^(score - reference + kLift) * (V's scale / the unit the output accumulates in).
// Roundings: a query row is divided by the power of two that brings its largest entry to 1 .. 2 and rounded to fp16 (bf16 entries
// down to 2^-17 of the row's largest stay exact, smaller ones are off by 2^-25 of it at most); the weights are rounded to fp16, half a step
// being 2^-11 of a weight, and the sum is of the rounded ones; kLift keeps weights down to 2^-21 of the reference's in fp16's normal range and
// the smallest that is not lost at 2^-32, so that what a million far keys add up to is kept.  Sums, references and outputs are fp32.
//
// Operands without a transpose or LDS: a wavefront takes the scores of 64 keys as S^T = K q^T in four 16 x 16 tiles.  Row i of tile t
// is key 16 (i / 4) + 4 t + i % 4, so that lane group g ends up with the scores of keys 16 g .. 16 g + 15 of its query: exactly the
// order in which the other operand of P V, sixteen tokens of one entry, is one 16-byte load.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "prof.h"
#include "../../include/psd.h"

namespace psd {
namespace {

typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr float kFarBelow = -1.5e38f;      // the reference before a key was seen: finite, so that differences are numbers
constexpr float kSlack = 5.f;              // the reference moves when a score is this far (in powers of two) above it
constexpr float kSlackV = 8.f;             // ... and the outputs' unit when V's scale is beyond this many times it, or as small a part
constexpr float kLift = 7.f;               // weights are held times 2^kLift: at most 2^15, fp16 ends at 2^16

// Whether a reference is so large (2^8 powers of two) that an exponent must not be put together from it by fma: score * unit would go in
// unrounded where the reference was rounded, and what is added to the reference would be lost in it.  The difference is then taken first.
__device__ __forceinline__ bool is_large(float m) { return fabsf(m) > 256.f && m != kFarBelow; }

__device__ __forceinline__ float above(float score, float unit, float m) {
#pragma clang fp contract(off)
    const float x = score * unit;
    return x - m;
}

// eight codes as one matrix operand, exact
__device__ __forceinline__ f16x8 widen8(uint32_t lo, uint32_t hi) {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// bytes of w that hold e4m3's NaN, as 0x80
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// w with zeros there
__device__ __forceinline__ uint32_t without_nan(uint32_t w, uint32_t n) { return w & ~((n << 1) - (n >> 7)); }
// ... and 0x80 bytes as fp16 ones
__device__ __forceinline__ f16x8 nan_flags(uint32_t lo, uint32_t hi) {
    return widen8((lo >> 2) + (lo >> 3) + (lo >> 4), (hi >> 2) + (hi >> 3) + (hi >> 4));      // 0x38 is 1.0
}
template <bool BF16>
__device__ __forceinline__ f32x8 load_q8(const Kv8AttnArgs &a, int64_t at) {
    if constexpr (BF16) {
        const u32x4 raw = *reinterpret_cast<const u32x4 *>((const uint16_t *)a.q + at);
        f32x8 v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (j & 1) ? __uint_as_float(raw[j >> 1] & 0xffff0000u) : __uint_as_float(raw[j >> 1] << 16);
        return v;
    } else {
        return load_f32x8((const float *)a.q + at);
    }
}
// Where results go: the caller's bf16 rows, or what a forward's O projection reads; or, of one of several splits, to the combine kernel.
// A build for each: the choice at every store made the epilogue several times the loop.
enum { kOutBf16, kOutF32, kOutF16, kOutOp, kOutPart };
// entries d .. d + 3 of query head `head` of row m
template <int OUT>
__device__ __forceinline__ void store_out4(const Kv8AttnArgs &a, int64_t m, int head, int split, int d, f32x4 r) {
    const int col = head * a.d_h + d;
    const int64_t at = m * a.h_q * a.d_h + col;
    if constexpr (OUT == kOutBf16)
        *reinterpret_cast<uint2 *>(a.out_bf16 + m * a.out_stride + col) = make_uint2(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]));
    else if constexpr (OUT == kOutF32)
        *reinterpret_cast<f32x4 *>(a.out + at) = r;
    else if constexpr (OUT == kOutF16)
        *reinterpret_cast<uint2 *>(a.out16 + at) = make_uint2(f32_to_f16_bits(r[0]) | ((uint32_t)f32_to_f16_bits(r[1]) << 16),
                                                             f32_to_f16_bits(r[2]) | ((uint32_t)f32_to_f16_bits(r[3]) << 16));
    else if constexpr (OUT == kOutOp)
        op_store4(a.out_op, (int)m, col, a.op_folded, r);
    else
        *reinterpret_cast<f32x4 *>(a.part_o + ((m * a.h_q + head) * a.plan.splits + split) * a.d_h + d) = r;
}

// The scales of 64 blocks, one a lane, and from there to the block that asks: scalar loads would come back among the LDS reads, in no
// order, so that every wait for those became a wait for a scale's trip to memory (a prompt of 2001 rows
// 55 us against 53; with the fetch behind the next block's loads, which it then waits for, 64).
struct Scales {
    const float *k, *v;
    int end, base;                // base: block of lane 0
    float kw, vw;
    __device__ __forceinline__ void fetch(int kb, int lane) {
        base = kb;
        const int at = min(kb + lane, end - 1);
        kw = k[at];
        vw = v[at];
    }
    __device__ __forceinline__ void at(int kb, int lane, float *k_scale, float *v_scale) {
        if (kb >= base + kWave) fetch(kb, lane);
        *k_scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(kw), kb - base));
        *v_scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vw), kb - base));
    }
};

// One wavefront's part of a query tile of 16 rows: scores, weights and products over whole blocks of 64 keys.
template <int DH>
struct QueryTile {
    static constexpr int KS = DH / 32, DT = DH / 16;
    f16x8 q[KS];                  // lane (query i, group g): entries 64 (s / 2) + 16 g + 8 (s % 2) .. + 7
    float unit;                   // what a score has to be multiplied with, but for K's scale, to be in powers of two
    int limit;                    // the last position that the row sees; -1: no row
    float m, l;                   // reference; sum of this lane's weights, times 2^kLift
    f32x4 o[DT];                  // lane (query i, group g): entries 16 dt + 4 g .. + 3, in units of V's scale `vref`

    template <bool QB>
    __device__ __forceinline__ void init(const Kv8AttnArgs &a, int64_t row, int head, int limit_, int g, float scale_log2) {
        limit = limit_;
        m = kFarBelow;
        l = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        f32x8 v[KS];
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            v[s] = load_q8<QB>(a, row * a.q_stride + head * DH + 64 * (s >> 1) + 16 * g + 8 * (s & 1));
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[s][j]));
        }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const int e = min(max((int)(__float_as_uint(top) >> 23), 1), 253);                 // 2^(e - 127) <= top
        const float down = copysignf(__uint_as_float((uint32_t)(254 - e) << 23), scale_log2);             // (unit stays positive)
        unit = fabsf(scale_log2) * __uint_as_float((uint32_t)e << 23);
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = __builtin_bit_cast(f16x8, f32x8_to_f16x8(v[s] * down));
    }
};

// Few query rows: the wavefronts of a block share its 16 query rows and take every fourth block of 64 keys each; their results are
// joined in LDS, and those of a sequence's splits by the combine kernel.  The chunks of 16 rows of one head lie a multiple of the grid's splits x heads apart, so that where
// that is a multiple of eight one XCD's L2 serves them all (11 rows of 4 query heads on 16 000 keys 22.4 -> 18.8 us).  What bounds it: bytes on long caches (4 sequences of 131 000 keys, 8 KV heads of 128: 180 us =
// 6.0 TB/s), else the chain of load, scores, weights and products of a wavefront's blocks of keys
// (one token on 389 keys 7 us, 24 x 5 rows of 64-wide heads on up to 3000 keys 10.8).  No LDS on the way in: a code is used by one wavefront only.
template <int DH, bool QB, int OUT>
__global__ __launch_bounds__(256, 2) void attn8_direct_kernel(Kv8AttnArgs a, float scale_log2) {
    constexpr int KS = DH / 32, DT = DH / 16, KL = DH / 64;
    __shared__ float s_o[4][16][DH + 4];
    __shared__ float s_m[4][16], s_l[4][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, chunk = blockIdx.z, b = blockIdx.y / a.h_kv, hk = blockIdx.y % a.h_kv, group = a.h_q / a.h_kv, NQ = group * a.R;
    const int len = min(max(a.lens[b], 0), a.max_len);
    const int n_keys = min(len + a.R, a.max_len);
    const int q0 = chunk * 16, qi = q0 + i;             // query row qi: head qi % group of the step's row qi / group
    const int row = min(qi, NQ - 1) / group, head = hk * group + min(qi, NQ - 1) % group;
    QueryTile<DH> t;
    t.template init<QB>(a, (int64_t)b * a.R + row, head, qi < NQ ? len + row : -1, g, scale_log2);
    const int seen = min(len + min(q0 + 15, NQ - 1) / group + 1, n_keys), all_see = len + q0 / group + 1;      // by some, by every row of the block
    const int n_blocks = (seen + kKv8Block - 1) / kKv8Block;
    const int first = split * a.plan.range, last = split + 1 == a.plan.splits ? n_blocks : min(n_blocks, first + a.plan.range);
    const size_t cache_row = (size_t)b * a.h_kv + hk;
    const uint8_t *K = a.k + cache_row * a.max_len * DH, *V = a.v + cache_row * a.max_len * DH;
    const size_t scale_row = cache_row * (a.max_len / kKv8Block);
    Scales scales{a.k_scale + scale_row, a.v_scale + scale_row, n_blocks, 0, 0.f, 0.f};
    if (first < last) scales.fetch(first, lane);
    float vref = 1.f, rvref = 1.f;
    bool large = false;

    // The next block's codes are on their way while this one is worked on: at d_head 64 in registers of their own, at 128, where a block's
    // fill 64 and a second set of them spills, in the present one's, K's from the scores on and V's from the product on.
    constexpr int SETS = DH == 64 ? 2 : 1;
    u32x4 kr[SETS][4][KL], vr[SETS][DT];
    auto load_k = [&](auto at, int kb) {
        const uint8_t *p = K + (size_t)kb * kKv8Block * DH;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int j = 0; j < KL; ++j)
                kr[decltype(at)::value][c][j] = *reinterpret_cast<const u32x4 *>(p + (16 * (i >> 2) + 4 * c + (i & 3)) * DH + 64 * j + 16 * g);
    };
    auto load_v = [&](auto at, int kb) {
        const uint8_t *p = V + (size_t)kb * kKv8Block * DH;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vr[decltype(at)::value][dt] = *reinterpret_cast<const u32x4 *>(p + (dt * 16 + i) * kKv8Block + 16 * g);
    };
    auto work = [&](auto at, int kb, int after, float k_scale, float v_scale) {
        constexpr int x = decltype(at)::value;
        const bool masked = (kb + 1) * kKv8Block > all_see;  // (the same for the whole block)
        const int room = t.limit - (kb * kKv8Block + 16 * g);              // of this lane's keys 4 c + e those up to there are seen
        if (masked) {
            // A position that some row does not see may hold anything.  What is no number there must not reach the product, where a
            // weight of 0 would not keep it out; rows that see it get theirs from the flags.
            uint32_t any = 0;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e = 0; e < 4; ++e) any |= nan_codes(vr[x][dt][e]);
            if (__ballot(any != 0)) {
                f16x8 see[2];
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) see[c >> 1][4 * (c & 1) + e] = (_Float16)(4 * c + e > room ? 0.f : 1.f);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    f32x4 hit{0.f, 0.f, 0.f, 0.f};
                    uint32_t n[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) { n[e] = nan_codes(vr[x][dt][e]); vr[x][dt][e] = without_nan(vr[x][dt][e], n[e]); }
                    hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(nan_flags(n[0], n[1]), see[0], hit, 0, 0, 0);
                    hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(nan_flags(n[2], n[3]), see[1], hit, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (hit[e] > 0.f) t.o[dt][e] = __uint_as_float(0x7fc00000u);
                }
            }
        }
        f32x4 s[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) s[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < KS; ++e)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                s[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(kr[x][c][e >> 1][2 * (e & 1)], kr[x][c][e >> 1][2 * (e & 1) + 1]), t.q[e], s[c], 0, 0, 0);
        if (SETS == 1) load_k(at, after);
        float f = t.unit * k_scale;
        if (masked) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[c][e] = 4 * c + e > room ? -INFINITY : s[c][e] * f;
            f = 1.f;
        }
        float top = s[0][0];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, s[c][e]);
        top *= f;
        if (__ballot(top > t.m + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16, kWave));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float m = top > t.m + kSlack ? top : t.m, shrink = __builtin_amdgcn_exp2f(t.m - m);
            t.m = m;
            t.l *= shrink;
            large = __ballot(is_large(m)) != 0;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) t.o[dt] *= shrink;
        }
        float from = t.m;
        if (large) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[c][e] = above(s[c][e], f, t.m);
            f = 1.f;
            from = 0.f;
        }
        // V's scale rides in the weights while it stays within kSlackV of the outputs' unit, which else moves to it
        float by = v_scale * rvref;
        if (!(by <= kSlackV && by >= 1.f / kSlackV)) {
            const float to = vref / v_scale;
            vref = v_scale;
            rvref = 1.f / v_scale;
            by = 1.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) t.o[dt] *= to;
        }
        const float under = kLift - from + __builtin_amdgcn_logf(by);
        float sum = 0.f;
        f16x8 p[2];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const f16x2 w = __builtin_convertvector((f32x2{__builtin_amdgcn_exp2f(fmaf(s[c][e], f, under)), __builtin_amdgcn_exp2f(fmaf(s[c][e + 1], f, under))}), f16x2);
                sum = __builtin_amdgcn_fdot2(w, f16x2{1, 1}, sum, false);
                p[c >> 1][4 * (c & 1) + e] = w[0];
                p[c >> 1][4 * (c & 1) + e + 1] = w[1];
            }
        t.l += sum * __builtin_amdgcn_rcpf(by);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                t.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(vr[x][dt][2 * u], vr[x][dt][2 * u + 1]), p[u], t.o[dt], 0, 0, 0);
        if (SETS == 1) load_v(at, after);
    };
    int kb = first + wave;
    auto turn = [&](auto now, auto then) {                   // one block; false: it was the last
        const int after = min(kb + 4, last - 1);
        float k_scale, v_scale;
        scales.at(kb, lane, &k_scale, &v_scale);             // (ahead of the loads: a wait for scales would be one for them)
        if constexpr (SETS == 2) { load_k(then, after); load_v(then, after); }
        work(now, kb, after, k_scale, v_scale);
        kb += 4;
        return kb < last;
    };
    if (kb < last) {
        load_k(Int<0>{}, kb);
        load_v(Int<0>{}, kb);
        while (turn(Int<0>{}, Int<SETS - 1>{}) && turn(Int<SETS - 1>{}, Int<0>{})) {}
    }

    // join the wavefronts, in their order
    float l = t.l;
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (g == 0) { s_m[wave][i] = t.m; s_l[wave][i] = l; }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4 *>(&s_o[wave][i][dt * 16 + 4 * g]) = t.o[dt] * vref;
    __syncthreads();
    for (int x = tid; x < 16 * (DH / 4); x += 256) {
        const int qc = x / (DH / 4), d = x % (DH / 4) * 4, q = q0 + qc;
        if (q >= NQ) continue;
        const float M = fmaxf(fmaxf(s_m[0][qc], s_m[1][qc]), fmaxf(s_m[2][qc], s_m[3][qc]));
        float L = 0.f;
        f32x4 r{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][qc] - M);
            L += s_l[w][qc] * f;
            r += *reinterpret_cast<const f32x4 *>(&s_o[w][qc][d]) * f;
        }
        if (L != 0.f) r = r * (1.0f / L);                    // (a split none of whose keys the row sees: 0)
        const int64_t m = (int64_t)b * a.R + q / group;
        const int h = hk * group + q % group;
        store_out4<OUT>(a, m, h, split, d, r);
        if (OUT == kOutPart && d == 0) a.part_ml[(m * a.h_q + h) * a.plan.splits + split] = make_float2(M, L);
    }
}

// The wide kernel's LDS: two sets of codes; afterwards what the groups hand to the first one; then rows on their way out, 16 bytes apart
template <int DH, int QG, int KG, int OUT>
constexpr int wide_lds() {
    constexpr int JT = DH / 32, stage = 2 * KG * 4 * JT * 1024, join = KG > 1 ? (KG - 1) * QG * (JT * 4096 + 512) : 0;
    constexpr int rows = QG * 32 * (DH * (OUT == kOutF32 || OUT == kOutPart ? 4 : 2) + 16);
    return stage > join ? (stage > rows ? stage : rows) : (join > rows ? join : rows);
}

// Many query rows: wavefronts of 32 rows each on the 32 x 32 matrix instructions, QG of them side by side on the rows of a block and KG such
// groups on different blocks of keys, joined in LDS at the end.  The codes of 64 keys, 16 KB at d_head 128, pass through LDS once for
// a group, in the order of the operands: a piece of 1 KB is what the 64 lanes read at once, sixteen codes each, and becomes two
// operands.  Row x of K's tile t is key 32 t + 16 (x / 4 % 2) + 4 (x / 8) + x % 4, so that a lane's scores, of keys 32 t + 16 h .. + 15 for lane
// half h, are in the order of V's pieces.
// Two blocks of four wavefronts a CU.  KG: with up to 64 rows the second pair of wavefronts takes every other block of keys.
// What bounds it: instruction issue and a wavefront's own chain.  A block of 64 keys and 32 rows is 1024 clocks of matrix instructions, some 1400 of
// vector ones (128 conversions, 32 exponentials of 8.6 clocks each) and about 900 of waits for LDS, the maximum and the barrier: a wavefront
// alone on its SIMD takes 2700 clocks, two of them 2100 each.  A prompt of 2001 rows of the 7B shape (32 heads) 50 us = 660 TFLOP/s, against 27 us
// at the rate of a large matrix product; its longest blocks, 32 blocks of keys, run alone for the second half.  Tried and not faster (us, the same prompt at 54 in that
// session): conversions once for the block, fp16 in LDS, 56; the next block's scores under this one's weights, three sets of LDS, 56; eight
// wavefronts with KG = 2, one block a CU, 60; 64 rows a block 64; two blocks of keys to a barrier 54.5; matrix instructions at a higher wave priority 53.5.
template <int DH, int QG, int KG, bool QB, int OUT>
__global__ __launch_bounds__(QG * KG * 64, 512 / (QG * KG * 64)) void attn8_wide_kernel(Kv8AttnArgs a, float scale_log2, FastDiv by_group) {
    constexpr int JT = DH / 32, PIECES = 4 * JT, MINE = PIECES / QG;       // K: 2 JT pieces [t][j], V: 2 JT [dt][w]
    constexpr int kRowBytes = DH * (OUT == kOutF32 || OUT == kOutPart ? 4 : 2) + 16;
    static_assert(wide_lds<DH, QG, KG, OUT>() <= 159 * 1024, "LDS");
    extern __shared__ __attribute__((aligned(16))) uint8_t s_raw[];
    __shared__ int s_nan[2][KG][QG];
    auto tile = [&](int set, int group) { return reinterpret_cast<u32x4 (*)[64]>(s_raw + (set * KG + group) * PIECES * 1024); };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 31, h = lane >> 5;
    const int qg = wave % QG, kg = wave / QG;
    // Blocks by how many keys they walk, most first, a head's chunk before the next chunk; those that fill the chip's second places
    // the other way round, so that where all are resident at once a long one shares its CU with a short one.
    uint32_t rank = blockIdx.x + gridDim.x * blockIdx.z;
    if (rank >= 256u && gridDim.x * gridDim.z <= 512u) rank = 255u + gridDim.x * gridDim.z - rank;
    const int bh = rank % gridDim.x, b = bh / a.h_kv, hk = bh % a.h_kv, group = by_group.n, NQ = group * a.R;
    const int split = blockIdx.y, chunk = gridDim.z - 1 - rank / gridDim.x;
    const int len = min(max(a.lens[b], 0), a.max_len);
    const int n_keys = min(len + a.R, a.max_len);
    const int c0 = chunk * (QG * 32), q0 = c0 + qg * 32, qi = q0 + i;
    const int row = by_group.div(min(qi, NQ - 1)), head = hk * group + min(qi, NQ - 1) - row * group;
    const int limit = qi < NQ ? len + row : -1;
    // keys that some row of the block, some row of the wavefront sees
    const int block_seen = min(len + (int)by_group.div(min(c0 + QG * 32, NQ) - 1) + 1, n_keys);
    const int wave_seen = q0 < NQ ? min(len + (int)by_group.div(min(q0 + 32, NQ) - 1) + 1, n_keys) : 0;
    const int n_blocks = (block_seen + kKv8Block - 1) / kKv8Block;
    const int first = split * a.plan.range, last = split + 1 == a.plan.splits ? n_blocks : min(n_blocks, first + a.plan.range);
    const int whole = min(last, (len + (int)by_group.div(c0) + 1) / kKv8Block);            // blocks of keys below that every row of the block sees
    const size_t cache_row = (size_t)b * a.h_kv + hk;
    const uint8_t *K = a.k + cache_row * a.max_len * DH, *V = a.v + cache_row * a.max_len * DH;
    const size_t scale_row = cache_row * (a.max_len / kKv8Block);
    Scales scales{a.k_scale + scale_row, a.v_scale + scale_row, n_blocks, 0, 0.f, 0.f};

    // every wavefront brings some of K's and as many of V's pieces of its group's block
    uint32_t src[MINE];
#pragma unroll
    for (int c = 0; c < MINE; ++c) {
        const int x = (c * QG + qg) % (2 * JT);
        src[c] = c < MINE / 2 ? (32 * (x / JT) + 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3)) * DH + 32 * (x % JT) + 16 * h
                              : (32 * (x / 2) + i) * kKv8Block + 32 * (x % 2) + 16 * h;
    }
    u32x4 next[MINE];
    auto load = [&](int kt) {
        const size_t at = (size_t)min(kt, last - 1) * kKv8Block * DH;
#pragma unroll
        for (int c = 0; c < MINE; ++c) next[c] = *reinterpret_cast<const u32x4 *>((c < MINE / 2 ? K : V) + at + src[c]);
    };
    // look: a block that needs the mask.  A position that some row does not see may hold anything: what is no number among V's entries
    // must not reach the product, where a weight of 0 would not keep it out.
    auto store = [&](int set, bool look) {
        if (look) {
            uint32_t any = 0;
#pragma unroll
            for (int c = MINE / 2; c < MINE; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) any |= nan_codes(next[c][e]);
            const bool found = __ballot(any != 0) != 0;
            if (found) {
#pragma unroll
                for (int c = MINE / 2; c < MINE; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) next[c][e] = without_nan(next[c][e], nan_codes(next[c][e]));
            }
            if (lane == 0) s_nan[set][kg][qg] = found;
        }
#pragma unroll
        for (int c = 0; c < MINE; ++c) tile(set, kg)[c * QG + qg][lane] = next[c];
    };
    if (first < last) {
        load(first + kg);
        scales.fetch(first, lane);
    }

    f16x8 q[2 * JT];                                         // lane (query i, half h): entries 32 (s / 2) + 16 h + 8 (s % 2) .. + 7
    float unit;
    {
        f32x8 v[2 * JT];
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < 2 * JT; ++s) {
            v[s] = load_q8<QB>(a, ((int64_t)b * a.R + row) * a.q_stride + head * DH + 32 * (s >> 1) + 16 * h + 8 * (s & 1));
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[s][j]));
        }
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const int e = min(max((int)(__float_as_uint(top) >> 23), 1), 253);
        const float down = copysignf(__uint_as_float((uint32_t)(254 - e) << 23), scale_log2);
        unit = fabsf(scale_log2) * __uint_as_float((uint32_t)e << 23);
#pragma unroll
        for (int s = 0; s < 2 * JT; ++s) q[s] = __builtin_bit_cast(f16x8, f32x8_to_f16x8(v[s] * down));
    }
    f32x16 o[JT];
#pragma unroll
    for (int dt = 0; dt < JT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    float m = kFarBelow, l = 0.f, vref = 1.f, rvref = 1.f;
    bool large = false;
    if (first < last) store(0, first + KG > whole);
    __syncthreads();

    auto step = [&](auto with_mask, int kb, int set, float k_scale, float v_scale) {
        constexpr bool MASKED = decltype(with_mask)::value != 0;
        const int room = limit - (kb * kKv8Block + 16 * h);  // of this lane's keys 32 t + r those up to there are seen
        const u32x4 (*codes)[64] = tile(set, kg);
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 w = codes[t * JT + j][lane];
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(w[2 * u], w[2 * u + 1]), q[2 * j + u], s[t], 0, 0, 0);
                }
        float f = unit * k_scale;
        if constexpr (MASKED) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][r] = 32 * t + r > room ? -INFINITY : s[t][r] * f;
            f = 1.f;
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
        top *= f;
        if (__ballot(top > m + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float up = top > m + kSlack ? top : m, shrink = __builtin_amdgcn_exp2f(m - up);
            m = up;
            l *= shrink;
            large = __ballot(is_large(m)) != 0;
#pragma unroll
            for (int dt = 0; dt < JT; ++dt) o[dt] *= shrink;
        }
        float from = m;
        if (large) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][r] = above(s[t][r], f, m);
            f = 1.f;
            from = 0.f;
        }
        // V's scale rides in the weights while it stays within kSlackV of the outputs' unit, which else moves to it
        float by = v_scale * rvref;
        if (!(by <= kSlackV && by >= 1.f / kSlackV)) {
            const float to = vref / v_scale;
            vref = v_scale;
            rvref = 1.f / v_scale;
            by = 1.f;
#pragma unroll
            for (int dt = 0; dt < JT; ++dt) o[dt] *= to;
        }
        const float under = kLift - from + __builtin_amdgcn_logf(by);
        float sum = 0.f;
        f16x8 p[4];                                          // p[2 t + u]: keys 32 t + 16 h + 8 u .. + 7
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const f16x2 w = __builtin_convertvector((f32x2{__builtin_amdgcn_exp2f(fmaf(s[t][r], f, under)), __builtin_amdgcn_exp2f(fmaf(s[t][r + 1], f, under))}), f16x2);
                sum = __builtin_amdgcn_fdot2(w, f16x2{1, 1}, sum, false);
                p[2 * t + (r >> 3)][r & 7] = w[0];
                p[2 * t + (r >> 3)][(r & 7) + 1] = w[1];
            }
        l += sum * __builtin_amdgcn_rcpf(by);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int dt = 0; dt < JT; ++dt) {
                    const u32x4 w = codes[2 * JT + 2 * dt + x][lane];
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(w[2 * u], w[2 * u + 1]), p[2 * x + u], o[dt], 0, 0, 0);
                }
    };
    // V's entries that are no number in a block that needs the mask (they are zeros in LDS): rows that see one get it
    auto holes = [&](int kb) {
        const int room = limit - (kb * kKv8Block + 16 * h);
        f16x8 see[4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) see[2 * t + (r >> 3)][r & 7] = (_Float16)(32 * t + r > room ? 0.f : 1.f);
#pragma unroll
        for (int dt = 0; dt < JT; ++dt) {
            f32x16 hit;
#pragma unroll
            for (int r = 0; r < 16; ++r) hit[r] = 0.f;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(V + (size_t)kb * kKv8Block * DH + (32 * dt + i) * kKv8Block + 32 * x + 16 * h);
                hit = __builtin_amdgcn_mfma_f32_32x32x16_f16(nan_flags(nan_codes(w[0]), nan_codes(w[1])), see[2 * x], hit, 0, 0, 0);
                hit = __builtin_amdgcn_mfma_f32_32x32x16_f16(nan_flags(nan_codes(w[2]), nan_codes(w[3])), see[2 * x + 1], hit, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (hit[r] > 0.f) o[dt][r] = __uint_as_float(0x7fc00000u);
        }
    };
    // blocks of keys that every row of the block sees, then those that need the mask: KG at a time, one for each group
    int kb = first, set = 0;
    auto walk = [&](auto with_mask, int end) {
        for (; kb < end; kb += KG, set ^= 1) {
            const int kt = kb + kg;
            float k_scale, v_scale;
            scales.at(min(kt, last - 1), lane, &k_scale, &v_scale);        // (ahead of the loads: a wait for scales would be one for them)
            load(kt + KG);
            if constexpr (decltype(with_mask)::value == 0) {
                step(with_mask, kt, set, k_scale, v_scale);
            } else if (kt < last && kt * kKv8Block < wave_seen) {          // (the same for the wavefront)
                int bad = 0;
#pragma unroll
                for (int x = 0; x < QG; ++x) bad |= s_nan[set][kg][x];
                if (__builtin_amdgcn_readfirstlane(bad)) holes(kt);
                step(with_mask, kt, set, k_scale, v_scale);
            }
            store(set ^ 1, kb + 2 * KG > whole);             // (look: as for `plain`)  nobody reads that set any more: all are past the last barrier
            __syncthreads();
        }
    };
    const int plain = first + (whole > first ? (whole - first) / KG * KG : 0);
    walk(Int<0>{}, plain);
    walk(Int<1>{}, last);

    if constexpr (KG > 1) {                                  // the groups' results, in their order
        f32x4 (*s_o)[JT * 4][64] = reinterpret_cast<f32x4 (*)[JT * 4][64]>(s_raw);
        float2 (*s_ml)[64] = reinterpret_cast<float2 (*)[64]>(s_raw + (KG - 1) * QG * JT * 4096);
        if (kg) {
            const int at = (kg - 1) * QG + qg;
            s_ml[at][lane] = make_float2(m, l);
#pragma unroll
            for (int dt = 0; dt < JT; ++dt)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    s_o[at][dt * 4 + x][lane] = f32x4{o[dt][4 * x], o[dt][4 * x + 1], o[dt][4 * x + 2], o[dt][4 * x + 3]} * vref;
        }
        __syncthreads();
        if (kg == 0) {
            float M = m;
#pragma unroll
            for (int g = 1; g < KG; ++g) M = fmaxf(M, s_ml[(g - 1) * QG + qg][lane].x);
            const float mine = __builtin_amdgcn_exp2f(m - M);
            l *= mine;
#pragma unroll
            for (int dt = 0; dt < JT; ++dt) o[dt] *= vref * mine;
            vref = 1.f;
            m = M;
#pragma unroll
            for (int g = 1; g < KG; ++g) {
                const int at = (g - 1) * QG + qg;
                const float2 ml = s_ml[at][lane];
                const float w = __builtin_amdgcn_exp2f(ml.x - M);
                l += ml.y * w;
#pragma unroll
                for (int dt = 0; dt < JT; ++dt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const f32x4 r = s_o[at][dt * 4 + x][lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[dt][4 * x + e] += r[e] * w;
                    }
            }
        }
        __syncthreads();
        if (kg) return;
    }
    l += __shfl_xor(l, 32, kWave);
    const float inv = l != 0.f ? vref / l : 0.f;             // (a split none of whose keys the row sees: 0; a sum that is no number is not 0)
    const int64_t mrow = (int64_t)b * a.R + row;
    if (OUT == kOutPart && h == 0 && qi < NQ) a.part_ml[(mrow * a.h_q + head) * a.plan.splits + split] = make_float2(m, l);
    if constexpr (OUT == kOutOp) {
        if (qi >= NQ) return;
#pragma unroll
        for (int dt = 0; dt < JT; ++dt)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                op_store4(a.out_op, (int)mrow, head * DH + 32 * dt + 8 * x + 4 * h, a.op_folded,
                          f32x4{o[dt][4 * x], o[dt][4 * x + 1], o[dt][4 * x + 2], o[dt][4 * x + 3]} * inv);
    } else {
        // rows through LDS, the wavefront's own part of it, so that they leave sixteen bytes a lane side by side: eight bytes a lane into
        // 32 rows took 2 us at the end of every block
        constexpr bool HALF = OUT == kOutBf16 || OUT == kOutF16;
        constexpr int PER = DH * (HALF ? 2 : 4) / 16;        // lanes of a row
        uint8_t *rows = s_raw + qg * 32 * kRowBytes;
#pragma unroll
        for (int dt = 0; dt < JT; ++dt)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const f32x4 r = f32x4{o[dt][4 * x], o[dt][4 * x + 1], o[dt][4 * x + 2], o[dt][4 * x + 3]} * inv;
                uint8_t *at = rows + i * kRowBytes + (32 * dt + 8 * x + 4 * h) * (HALF ? 2 : 4);
                if constexpr (OUT == kOutBf16) *reinterpret_cast<uint2 *>(at) = make_uint2(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]));
                else if constexpr (OUT == kOutF16)
                    *reinterpret_cast<uint2 *>(at) = make_uint2(f32_to_f16_bits(r[0]) | ((uint32_t)f32_to_f16_bits(r[1]) << 16), f32_to_f16_bits(r[2]) | ((uint32_t)f32_to_f16_bits(r[3]) << 16));
                else *reinterpret_cast<f32x4 *>(at) = r;
            }
        __builtin_amdgcn_wave_barrier();                     // (a wavefront's LDS accesses are in order)
#pragma unroll
        for (int x = 0; x < 32 * PER / 64; ++x) {
            const int r = (x * 64 + lane) / PER, piece = (x * 64 + lane) % PER;
            const u32x4 w = *reinterpret_cast<const u32x4 *>(rows + r * kRowBytes + piece * 16);
            if (q0 + r >= NQ) continue;
            const int rr = by_group.div(q0 + r), hh = hk * group + q0 + r - rr * group;
            const int64_t mr = (int64_t)b * a.R + rr;
            uint8_t *dst;
            if constexpr (OUT == kOutBf16) dst = (uint8_t *)(a.out_bf16 + mr * a.out_stride + hh * DH);
            else if constexpr (OUT == kOutF16) dst = (uint8_t *)(a.out16 + (mr * a.h_q + hh) * DH);
            else if constexpr (OUT == kOutF32) dst = (uint8_t *)(a.out + (mr * a.h_q + hh) * DH);
            else dst = (uint8_t *)(a.part_o + ((mr * a.h_q + hh) * a.plan.splits + split) * DH);
            *reinterpret_cast<u32x4 *>(dst + piece * 16) = w;
        }
    }
}
// Joins the splits of a row and head, in their order: 256 / d_h rows and heads a wavefront, four entries a lane.  One trip to memory: 288 rows
// of 5 splits 3.1 us, 7168 rows of 4 splits 5.1, of 8 splits 6.3 (4.9 TB/s).
template <int DH, int OUT>
__global__ __launch_bounds__(256) void attn8_combine_kernel(Kv8AttnArgs a) {
    constexpr int kLanes = DH / 4, kRows = 256 / kLanes;
    const int64_t rh = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
    if (rh >= (int64_t)a.B * a.R * a.h_q) return;
    const int d = threadIdx.x % kLanes * 4;
    const int S = a.plan.splits;
    const float2 *ml = a.part_ml + rh * S;
    const float *o = a.part_o + rh * S * DH + d;
    float M = kFarBelow, L = 0.f;
    f32x4 r{0.f, 0.f, 0.f, 0.f};
    constexpr int kTogether = 8;                             // loads in flight: up to eight splits are one trip to memory
    for (int s0 = 0; s0 < S; s0 += kTogether) {
        float2 e[kTogether];
        f32x4 v[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const int s = min(s0 + k, S - 1);
            e[k] = ml[s];
            v[k] = *reinterpret_cast<const f32x4 *>(o + (size_t)s * DH);
        }
        float top = M;
#pragma unroll
        for (int k = 0; k < kTogether; ++k) top = fmaxf(top, e[k].x);
        const float shrink = __builtin_amdgcn_exp2f(M - top);
        M = top;
        L *= shrink;
        r *= shrink;
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const float w = s0 + k < S ? e[k].y * __builtin_amdgcn_exp2f(e[k].x - M) : 0.f;
            L += w;
            if (s0 + k < S) r += v[k] * w;
        }
    }
    store_out4<OUT>(a, rh / a.h_q, (int)(rh % a.h_q), 0, d, r * (1.0f / L));
}

}  // namespace

// Splits of the keys, so that few rows fill the chip.
// Direct kernel: none up to 12 blocks of keys, three for each wavefront (one launch instead of two).  Above, the walk shrinks with the splits and the
// join grows with them, so that the best number goes with the root of the length, sqrt(2 blocks), at least one for four blocks and 48 at most, while
// there is a CU for each block of the grid; where the heads alone take more than half of the CUs, as many as are resident, but only on long
// caches.  A split's keys are a multiple of four blocks, one for each wavefront.  us with the join, by splits: 8 heads, 16 blocks 1: 9.5, 4: 9.2;
// 4 heads, 63 blocks 8: 9.5, 16: 9.3, 32: 10.1; 126 blocks 8: 12.0, 16: 10.4, 32: 10.7; 501 blocks 16: 19.6, 32: 15.3, 64: 15.9; 2047 blocks 16: 52.6, 32: 32.3,
// 48: 29.1, 64: 30.8; 8 heads, 2047 blocks 16: 58.1, 32: 46.3, 40: 58.2; 64 heads, 63 blocks 4: 17.5, 8: 19.8; 251 blocks 4: 45.6, 8: 47.6;
// 160 heads, 32 blocks 1: 17.2, 3: 20.1; 126 blocks 1: 68, 3: 58; 256 heads, 63 blocks 1: 41.6, 2: 45.7.
struct DirectSplits { int most, cus; };                      // heads: blocks of the grid without splits
static DirectSplits direct_splits(long heads, int blocks) {
    const int cus = (int)((heads > 128 && heads < 256 && blocks >= 96 ? 512 : 256) / heads), by_four = (blocks + 3) / 4;
    int most = (int)sqrt(2.0 * blocks);
    most = most < by_four ? most : by_four;
    most = most < 48 ? most : 48;
    return blocks <= 12 || cus <= 1 ? DirectSplits{1, 1} : DirectSplits{most < cus ? most : cus, cus};
}
static int direct_range(long heads, int blocks) {
    const DirectSplits s = direct_splits(heads, blocks);
    if (s.cus == 1) return blocks;
    const int nearest = (blocks + 2 * s.most) / (4 * s.most) * 4, range = nearest < 4 ? 4 : nearest;
    return (blocks + range - 1) / range <= s.cus ? range : ((blocks + s.most - 1) / s.most + 3) / 4 * 4;
}
// Wide kernel: as many as there are CUs for, and twice that where each wavefront still walks 12 blocks (24 in blocks of 64 rows), three blocks at least to a split.  us: 64 heads
// (16 x 16 rows x 7 query heads), 65 blocks 2: 53.6, 4: 35.9, 8: 36.6; 126 blocks 4: 53.3, 8: 51.6; 48 heads (24 x 5 x 8), 47 blocks 2: 27, 5: 17.1, 10: 18.5; 8 heads (9 rows x 4), 16 blocks 1: 25.5,
// 5: 13.7, 16: 15.5; 251 blocks 16: 32.8, 32: 28.4; 128 (4 x 33 rows x 32 heads), 17 blocks 1: 27.7, 2: 21.4, 4: 22.3; 64 blocks 2: 49.3, 4: 43.6.
static int wide_splits(long heads, int blocks, int rows) {
    long splits = 256 / heads;
    if (splits > 0 && blocks / splits >= (rows == 64 ? 48 : 24)) splits = 512 / heads;
    const int most = blocks / 3;
    splits = splits < most ? splits : most;
    return splits < 1 ? 1 : (int)splits;
}
static long grid_heads(int B, int h_kv, int NQ, int rows) { return (long)B * h_kv * ((NQ + rows - 1) / rows); }
// Rows of a block of the wide kernel.  A wavefront of the blocks of 64 rows walks every other block of keys, so that a step's work lies in twice as many
// blocks of half the length: more CUs have some, and few long rows wait for less.  64 while those are all resident, but for short
// chunks that fill the CUs already, and for long caches, where splits fill them.  us, 128 / 64 rows, by blocks of 128 rows x blocks of keys: 80 x 3 14.1 / 13.7, 104 x 4 14.8 / 14.0, 110 x 7
// 18.1 / 12.7, 132 x 9 25.7 / 21.1, 160 x 5 20.7 / 17.7, 176 x 22 41.1 / 36.8, 176 x 68 87.7 / 84.7, 250 x 16 33.6 / 20.9, 256 x 8 28.4 / 23.1, 256 x 40 69.3 / 60.1, in chunks of 200 rows
// 256 x 10 22.9 / 25.5; 128 x 28 37.9 / 33.0, 128 x 36 43.6 / 38.0, 128 x 51 46.7 / 50.1, 80 x 34 32.8 / 34.4, 96 x 134 73.5 / 93.4.
static int wide_rows(int B, int h_kv, int NQ, int blocks) {
    const long by_64 = grid_heads(B, h_kv, NQ, 64), by_128 = grid_heads(B, h_kv, NQ, 128);
    if (NQ <= 64) return 64;
    if (by_64 > 512 || (by_128 > 192 && NQ <= 512)) return 128;
    return by_128 > 128 || 10l * blocks <= 3 * by_128 ? 64 : 128;
}

// Query rows of a block.  16, the direct kernel's, while all its blocks are resident and few keys are walked again for every 16 rows: it
// begins and ends sooner (no barrier, no LDS on the way in).  Above, the wide kernel turns codes once for 32 rows and reads them from LDS; up
// to 32 rows half of its wavefronts and more have no rows of their own, so that it pays later.  us, direct / wide, by blocks of the grid x blocks of keys: 3 chunks of 16 rows,
// 24 x 251 18.7 / 20.4, 24 x 344 21.4 / 23.5, 24 x 501 26.8 / 26.6, 96 x 63 19.0 / 18.8, 96 x 126 30.0 / 24.4, 384 x 23 21.3 / 22.7; 7, 112 x 74 20.4 / 22.2; 25,
// 200 x 43 19.1 / 24.6; 11, 176 x 88 33.3 / 28.6; 2 chunks, 64 x 126 19.9 / 23.4, 64 x 251 30.4 / 33.4, 64 x 376 41.6 / 42.5, 256 x 94 38.8 / 41.9; 64-wide heads, 3 chunks,
// 144 x 47 10.6 / 13.1, 144 x 94 18.0 / 18.6; 768 x 5 20.2 / 14.1.
static bool direct(int B, int h_kv, int NQ, int d_h, int blocks) {
    const long heads = grid_heads(B, h_kv, NQ, 16);
    return NQ <= 16 || (heads <= 512 && heads * blocks * d_h <= (NQ <= 32 ? 20000l : 9000l) * 128);
}

int kv8_attn_max_splits(int B, int R, int h_q, int h_kv, int d_h, int len_bound) {
    const int NQ = h_q / h_kv * R, blocks = (len_bound + kKv8Block - 1) / kKv8Block;
    const long heads = grid_heads(B, h_kv, NQ, 16);
    const DirectSplits s = direct_splits(heads, blocks);
    const int rounded = s.most + s.most / 2 + 1, d = rounded < s.cus ? rounded : s.cus;          // (six blocks a split become four)
    int most = d;
    for (int rows = 64; rows <= 128 && NQ > 16; rows += 64) {
        const int w = wide_splits(grid_heads(B, h_kv, NQ, rows), blocks, rows);
        most = w > most ? w : most;
    }
    return most;
}

Kv8AttnPlan kv8_attn_plan(int B, int R, int h_q, int h_kv, int d_h, int len_bound) {
    const int NQ = h_q / h_kv * R, blocks = (len_bound + kKv8Block - 1) / kKv8Block;
    const int seen = (len_bound - R / 2 + kKv8Block - 1) / kKv8Block;                      // rows see half of the step's own keys on average
    Kv8AttnPlan p;
    p.rows = direct(B, h_kv, NQ, d_h, seen) ? 16 : wide_rows(B, h_kv, NQ, seen);
    if (p.rows == 16)
        p.range = direct_range(grid_heads(B, h_kv, NQ, 16), blocks);
    else {
        const int splits = wide_splits(grid_heads(B, h_kv, NQ, p.rows), seen, p.rows);
        p.range = (blocks + splits - 1) / splits;
    }
    p.splits = (blocks + p.range - 1) / p.range;
    return p;
}

void launch_kv8_attention(const Kv8AttnArgs &a, hipStream_t stream) {
    const float scale_log2 = 1.4426950408889634f * a.scale;
    const int NQ = a.h_q / a.h_kv * a.R;
    auto by_head = [&](auto kernels) {
        if (a.d_h == 128) kernels(Int<128>{});
        else kernels(Int<64>{});
    };
    auto by_out = [&](auto kernels) {
        if (a.out_bf16) kernels(Int<kOutBf16>{});
        else if (a.out) kernels(Int<kOutF32>{});
        else if (a.out16) kernels(Int<kOutF16>{});
        else kernels(Int<kOutOp>{});
    };
    {
        ScopedProf sp(PSD_KIND_ATTN, stream);
        auto go = [&](auto dh, auto qb, auto out) {
            constexpr int DH = decltype(dh)::value, OUT = decltype(out)::value;
            constexpr bool QB = decltype(qb)::value != 0;
            auto wide = [&](auto qg, auto kg) {
                constexpr int QG = decltype(qg)::value, KG = decltype(kg)::value, lds = wide_lds<DH, QG, KG, OUT>();
                const auto kernel = attn8_wide_kernel<DH, QG, KG, QB, OUT>;
                if (lds > 64 * 1024)                         // more than a kernel gets unasked
                    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
                launch_kernel(kernel, dim3(a.B * a.h_kv, a.plan.splits, (NQ + QG * 32 - 1) / (QG * 32)), QG * KG * 64, lds, stream, a, scale_log2, FastDiv(a.h_q / a.h_kv));
            };
            if (a.plan.rows == 128) wide(Int<4>{}, Int<1>{});
            else if (a.plan.rows == 64) wide(Int<2>{}, Int<2>{});
            else
                launch_kernel(attn8_direct_kernel<DH, QB, OUT>, dim3(a.plan.splits, a.B * a.h_kv, (NQ + 15) / 16), 256, 0, stream, a, scale_log2);
        };
        by_head([&](auto dh) {
            if (a.plan.splits > 1) {
                if (a.q_bf16) go(dh, Int<1>{}, Int<kOutPart>{});
                else go(dh, Int<0>{}, Int<kOutPart>{});
            } else if (a.q_bf16) {
                go(dh, Int<1>{}, Int<kOutBf16>{});           // (bf16 queries are the caller's, and so is the output)
            } else {
                by_out([&](auto out) {
                    if constexpr (decltype(out)::value != kOutBf16) go(dh, Int<0>{}, out);
                });
            }
        });
    }
    if (a.plan.splits > 1) {
        ScopedProf sp(PSD_KIND_ATTN_COMBINE, stream);
        const int64_t rows = (int64_t)a.B * a.R * a.h_q, per = 256 / (a.d_h / 4);
        const unsigned grid = (unsigned)((rows + per - 1) / per);
        by_head([&](auto dh) {
            by_out([&](auto out) { launch_kernel(attn8_combine_kernel<decltype(dh)::value, decltype(out)::value>, grid, 256, 0, stream, a); });
        });
    }
}

}  // namespace psd
