// Paged KV cache: quantised writes, reading back, and attention of chunks of new tokens over the pages, for gfx950.
//
// Orientation as everywhere in this library: keys (or values) are the first MFMA operand, queries (or probabilities) the second, so
// that scores come out transposed, S^T[key][row], four consecutive keys per lane, which is what the second contraction
// O^T = V^T P^T takes.  A "row" is a (token, query head of the KV group) pair, row = token * group + head.
//
// A key's scale multiplies its scores in fp32; a value's scale multiplies its probability before that is rounded for the second
// contraction (in fp16, relative to the largest such product).  e4m3 codes are exact in bf16 and fp16, so that dequantising rounds nothing.  Hidden keys are taken out by selection after
// the scale has been multiplied, and codes in pages are always finite: a NaN scale of a hidden key reaches nothing.
//
// 4-bit codes (e2m1, a power of two for every 32 features) become 16-bit values whole, code * scale, which rounds nothing either: the one
// instruction that widens two codes takes their scale along, and behind it the pages are 16-bit pages.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "spd_pages.h"

namespace {

#define SPD_TRY(x)                       \
    do {                                 \
        hipError_t e_ = (x);             \
        if (e_ != hipSuccess) return e_; \
    } while (0)

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16-bit types behind one name: F16 or bf16 elements, kept in registers as raw bits
template <bool F16>
struct Half {
    static __device__ __forceinline__ f32x4 mfma16(i32x4 a, i32x4 b, f32x4 c) {      // 16 x 16 x 32
        if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(i32x4 a, i32x4 b, f32x16 c) {    // 32 x 32 x 16
        if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ int pack(float a, float b) {
        if constexpr (F16) {
            f16x2 r;
            r[0] = (_Float16)a;
            r[1] = (_Float16)b;
            return __builtin_bit_cast(int, r);
        } else {
            bf16x2 r;
            r[0] = (__bf16)a;
            r[1] = (__bf16)b;
            return __builtin_bit_cast(int, r);
        }
    }
    static __device__ __forceinline__ float low(int v) {
        if constexpr (F16) return (float)__builtin_bit_cast(f16x2, v)[0];
        else return (float)__builtin_bit_cast(bf16x2, v)[0];
    }
    static __device__ __forceinline__ float high(int v) {
        if constexpr (F16) return (float)__builtin_bit_cast(f16x2, v)[1];
        else return (float)__builtin_bit_cast(bf16x2, v)[1];
    }
    // two e4m3 codes (the low or the high half of v)
    template <bool HI>
    static __device__ __forceinline__ int from_e4m3(int v) {
        if constexpr (F16) return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.0f, HI));
        else return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.0f, HI));
    }
    // two e2m1 codes (byte I of v) times 2^e, e + 127 in bits 23 to 30 of `scale` (the others are not looked at); NaN for 255
    template <int I>
    static __device__ __forceinline__ int from_e2m1(int v, unsigned scale) {
        if constexpr (F16) return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, __uint_as_float(scale), I));
        else return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, __uint_as_float(scale), I));
    }
    // eight of them
    static __device__ __forceinline__ i32x4 widen4(int v, unsigned scale) {
        return (i32x4){from_e2m1<0>(v, scale), from_e2m1<1>(v, scale), from_e2m1<2>(v, scale), from_e2m1<3>(v, scale)};
    }
    // Values of four positions in 4 bits: byte j of `v` has features f and f + 16 of position j, whose scale is byte U of w[j].  The operands of
    // feature f (lo) and f + 16 (hi): four positions each.
    template <int U, class W>
    static __device__ __forceinline__ void turn4(int v, const W &w, i32x2 &lo, i32x2 &hi) {
        auto scale = [](unsigned x) { return U == 3 ? x >> 1 : x << (23 - 8 * U); };
        const int a = from_e2m1<0>(v, scale(w[0])), b = from_e2m1<1>(v, scale(w[1])), c = from_e2m1<2>(v, scale(w[2])), d = from_e2m1<3>(v, scale(w[3]));
        lo = (i32x2){(int)__builtin_amdgcn_perm(b, a, 0x05040100), (int)__builtin_amdgcn_perm(d, c, 0x05040100)};
        hi = (i32x2){(int)__builtin_amdgcn_perm(b, a, 0x07060302), (int)__builtin_amdgcn_perm(d, c, 0x07060302)};
    }
    // eight e4m3 codes
    static __device__ __forceinline__ i32x4 widen(int a, int b) {
        return (i32x4){from_e4m3<false>(a), from_e4m3<true>(a), from_e4m3<false>(b), from_e4m3<true>(b)};
    }
};

// over lanes l, l^32 and l, l^16 (exchanged between registers: through the LDS a wave waits for it twice a pair of blocks)
__device__ __forceinline__ float half_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float quad_max(float x) {      // over lanes l, l^16, l^32, l^48
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_max(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_sum(__uint_as_float(a[0]) + __uint_as_float(a[1]));
}

// What the pages hold: SPD_E4M3, SPD_E2M1, or HALVES, values of the 16-bit type.
constexpr int HALVES = 0;

// The scales of four consecutive positions' values in 4 bits, one word each (its low D / 32 bytes).
template <int D>
struct Scales4 {
    unsigned w[4];
    __device__ __forceinline__ void load(const char *p) {
        if constexpr (D == 128) {
            const i32x4 x = *(const i32x4 *)p;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = x[j];
        } else {
            const i32x2 x = *(const i32x2 *)p;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (unsigned)x[j >> 1] >> (16 * (j & 1)) & 0xffff;
        }
    }
    static constexpr unsigned BAD = D == 128 ? 0xffffffffu : 0xffffu;      // of a row that was not finite
    __device__ __forceinline__ unsigned most() const {
        const unsigned a = w[0] > w[1] ? w[0] : w[1], b = w[2] > w[3] ? w[2] : w[3];
        return a > b ? a : b;
    }
};
// a lane's 4-bit codes of a block: D / 8 bytes
template <int D>
struct Codes4 {
    int c[D / 32];
    __device__ __forceinline__ void load(const char *p) {
        if constexpr (D == 128) {
            const i32x4 x = *(const i32x4 *)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = x[i];
        } else {
            const i32x2 x = *(const i32x2 *)p;
            c[0] = x[0];
            c[1] = x[1];
        }
    }
    __device__ __forceinline__ void stream(const char *p) {      // (read once)
        if constexpr (D == 128) {
            const i32x4 x = __builtin_nontemporal_load((const i32x4 *)p);
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = x[i];
        } else {
            const i32x2 x = __builtin_nontemporal_load((const i32x2 *)p);
            c[0] = x[0];
            c[1] = x[1];
        }
    }
};

// what every kernel over pages is told
struct Pages {
    const char *plan;
    char *pool;
    size_t page_bytes, head_bytes;
    int seqs, table, list;      // offsets into the plan
    int shift, page_size, kv, group;
    int on_device;              // the plan was made there
};
// Of a plan made on the device more workgroups are launched than the step may have items, and some of these may be empty.  (Of the host's plans that is not asked: the
// header is one more load to wait for.  us a call, asked of every plan / of those alone: one sequence of 2048, e4m3, 7.9 / 7.77, three windowed chunks in fp16 23.0 / 22.3.)
__device__ __forceinline__ const spd_plan_header &header_of(const Pages &P) { return *(const spd_plan_header *)P.plan; }
// where a sequence's block of 16 positions lies, for one head: its page's share of the head, and the block in the page
struct Block {
    char *head;
    int in_page;
};
__device__ __forceinline__ int page_of(const Pages &P, const spd_plan_seq &s, int block) {
    return ((const int *)(P.plan + P.table))[s.table + (block >> P.shift)];
}
__device__ __forceinline__ Block block_in(const Pages &P, int page, int head, int block) {
    return Block{P.pool + (size_t)page * P.page_bytes + (size_t)head * P.head_bytes, block & ((1 << P.shift) - 1)};
}
__device__ __forceinline__ Block block_at(const Pages &P, const spd_plan_seq &s, int head, int block) {
    return block_in(P, page_of(P, s, block), head, block);
}

// ------------------------------------------------------------------------------------------
// Writing.  One workgroup per 16-position block and a few heads: sixteen threads per token, D / 16 of them to a row of D features, each with
// eight of one rotary half and the eight that they turn with.  A workgroup of KV heads has keys and values side by side; one of
// query heads keeps its angles for all of its heads.  Bound by what is read and written: four prompts of 2048 tokens, 64 + 2 x 8 heads in bf16,
// 68 us (319 MB: 4.7 TB/s), over pages of 4 bits as long (311 MB; the rotation in 64 bits hides behind the memory; 57 for the same rows over and over).  (Rotated queries written past the caches: 4 less, but
// the attention behind it fetches them again: both together 364 -> 374.)
// ------------------------------------------------------------------------------------------
struct WriteArgs {
    Pages P;
    const char *qkv;
    const float2 *rope;
    char *q_out;
    int64_t ld, ld_q;           // in elements
    int q_heads;
    int kv_groups, q_groups;    // workgroups per block: for KV heads, for query heads
};

// two rows' halves of eight elements -> fp32
template <class In>
__device__ __forceinline__ void load_halves(const char *p, int apart, float (&a)[8], float (&b)[8]) {
    struct Eight {
        In v[8];
    };
    const Eight x = *(const Eight *)__builtin_assume_aligned(p, 16), y = *(const Eight *)__builtin_assume_aligned(p + apart * sizeof(In), 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        a[i] = (float)x.v[i];
        b[i] = (float)y.v[i];
    }
}

// The float beside x that is odd in its last place where x is between two: compared with, or rounded to, anything of fewer digits it does as x does.
__device__ __forceinline__ float to_odd(double x) {
    const float f = (float)x;
    const double back = f;
    unsigned u = __float_as_uint(f);
    if (back != x) u = (u - (fabs(back) > fabs(x))) | 1;
    return __uint_as_float(u);
}

// Eight of a row's features, and the eight they turn with, in 4 bits: codes two to a byte, in the order of the features, and the scales' bytes.  Groups
// of 32 features are four threads'; a row is TPR of them.  The least power of two of which the group's largest magnitude is 7 times at most: 6
// is the largest code, and what lies between 6 and 7 is no further from it than half a step there (root mean square over N(0, 1), 7 as the limit
// 11.2 % of it, 6 or 8 11.5).  Powers stay where code * scale is a value of the 16-bit type.
template <int TPR, bool F16>
__device__ __forceinline__ void quantise4(const float (&a)[8], const float (&b)[8], int &ca, int &cb, int &ea, int &eb) {
    constexpr int LO = F16 ? -23 : -100, HI = F16 ? 13 : 125;
    constexpr float LIMIT = F16 ? 65520.f : 0x1.ffp127f;      // becomes infinite in the 16-bit type
    float ma = 0.f, mb = 0.f, bad = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        ma = fmaxf(ma, fabsf(a[i]));
        mb = fmaxf(mb, fabsf(b[i]));
        if (!(fabsf(a[i]) < LIMIT && fabsf(b[i]) < LIMIT)) bad = 1.f;
    }
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        ma = fmaxf(ma, __shfl_xor(ma, d, 64));
        mb = fmaxf(mb, __shfl_xor(mb, d, 64));
    }
#pragma unroll
    for (int d = 1; d < TPR; d <<= 1) bad = fmaxf(bad, __shfl_xor(bad, d, 64));
    auto exponent = [](float m) {
        const int u = __float_as_int(m), e = (u >> 23) - 127 - ((u & 0x7fffff) <= 0x600000 ? 2 : 1);
        return (e < LO ? LO : e > HI ? HI : e) + 127;
    };
    ea = exponent(ma);
    eb = exponent(mb);
    const float sa = __int_as_float(ea << 23), sb = __int_as_float(eb << 23);
    unsigned x = 0, y = 0;
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, a[0], a[1], sa, 0);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, a[2], a[3], sa, 1);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, a[4], a[5], sa, 2);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, a[6], a[7], sa, 3);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(y, b[0], b[1], sb, 0);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(y, b[2], b[3], sb, 1);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(y, b[4], b[5], sb, 2);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(y, b[6], b[7], sb, 3);
    ca = bad != 0.f ? 0 : (int)x;
    cb = bad != 0.f ? 0 : (int)y;
    if (bad != 0.f) ea = eb = 255;
}

template <class In, int D, int C, bool F16>
__global__ void __launch_bounds__(256) k_pages_write(WriteArgs A) {
    constexpr bool E4M3 = C == SPD_E4M3, E2M1 = C == SPD_E2M1;
    constexpr int W = E4M3 ? 1 : 2, E = 16 / W, TPR = D / 16, UNITS = 16 / TPR;      // threads per row; rows of a token side by side
    constexpr int ROW = E2M1 ? D / 2 : D * W;                                          // bytes of a row
    const Pages &P = A.P;
    const spd_plan_block it = ((const spd_plan_block *)(P.plan + P.list))[blockIdx.x];
    if (P.on_device && ((int)blockIdx.x >= header_of(P).n_write || it.block < 0)) return;
    const spd_plan_seq &s = it.s;
    const int r = threadIdx.x >> 4, unit = (threadIdx.x & 15) / TPR, f0 = (threadIdx.x % TPR) * 8;
    const int pos = it.block * 16 + r, lo = it.block * 16 > s.pos ? 0 : s.pos - it.block * 16,
              hi = s.end - it.block * 16 < 16 ? s.end - it.block * 16 : 16;      // rows lo .. hi - 1 of the block are new
    const bool mine = r >= lo && r < hi;
    const int64_t token = s.tok0 + (pos - s.pos);
    float2 turn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = make_float2(1.f, 0.f);
    if (A.rope && mine) {
        const float4 *t = (const float4 *)(A.rope + (size_t)pos * (D / 2) + f0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 x = t[i];
            turn[2 * i] = make_float2(x.x, x.y);
            turn[2 * i + 1] = make_float2(x.z, x.w);
        }
    }
    auto rotate = [&](float(&a)[8], float(&b)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = a[i], z = b[i];
            a[i] = x * turn[i].x - z * turn[i].y;
            b[i] = z * turn[i].x + x * turn[i].y;
        }
    };
    const char *in = A.qkv + (token * A.ld + f0) * sizeof(In);
    if ((int)blockIdx.y >= A.kv_groups) {      // query heads
        if (!mine) return;
        const int group = blockIdx.y - A.kv_groups;
        for (int head = group * UNITS + unit; head < A.q_heads; head += A.q_groups * UNITS) {
            float a[8], b[8];
            load_halves<In>(in + (size_t)head * D * sizeof(In), D / 2, a, b);
            rotate(a, b);
            i32x4 x, y;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = Half<F16>::pack(a[2 * i], a[2 * i + 1]);
                y[i] = Half<F16>::pack(b[2 * i], b[2 * i + 1]);
            }
            char *o = A.q_out + (token * A.ld_q + (int64_t)head * D + f0) * 2;
            *(i32x4 *)o = x;
            *(i32x4 *)(o + D) = y;
        }
        return;
    }
    // codes of the block's keys and values, rows = positions: even units keys, odd units values
    constexpr int HEADS = UNITS / 2;
    __shared__ __attribute__((aligned(16))) char codes[UNITS][16 * ROW];
    const int head0 = blockIdx.y * HEADS, head = head0 + unit / 2, kind = unit & 1;
    const bool there = mine && head < P.kv;
    auto scales_of = [&](const Block &B) { return (float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16; };
    const Block B0 = block_at(P, s, head0, it.block);
    {
        float a[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = b[i] = 0.f;
        if (there) load_halves<In>(in + (size_t)(A.q_heads + head + kind * P.kv) * D * sizeof(In), D / 2, a, b);
        if constexpr (E2M1) {
            // (in 64 bits: beside a border between two codes 32 would now and then give the other, a whole step off)
            if (kind == 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double x = a[i], z = b[i], c = turn[i].x, n = turn[i].y;
                    a[i] = to_odd(x * c - z * n);
                    b[i] = to_odd(z * c + x * n);
                }
            }
            int ca, cb, ea, eb;
            quantise4<TPR, F16>(a, b, ca, cb, ea, eb);
            char *to = codes[unit] + r * ROW;
            // values: features f and f + 16 of a position share a byte, of which thread i has one and i + 2 the other
            const bool upper = threadIdx.x & 2;
            const int other = __shfl_xor(upper ? ca : cb, 2, 64);
            if (kind == 0) {
                *(int *)(to + f0 / 2) = ca;
                *(int *)(to + D / 4 + f0 / 2) = cb;
            } else {
                const int p = upper ? other : ca, q = upper ? cb : other;
                const int even = (p & 0x0f0f0f0f) | (q & 0x0f0f0f0f) << 4, odd = (p >> 4 & 0x0f0f0f0f) | (q & 0xf0f0f0f0);
                *(i32x2 *)(to + (upper ? D / 2 + f0 : f0) / 32 * 16 + f0 % 16) =
                    (i32x2){(int)__builtin_amdgcn_perm(odd, even, 0x05010400), (int)__builtin_amdgcn_perm(odd, even, 0x07030602)};
            }
            if (there && (threadIdx.x & 3) == 0) {
                char *e = B0.head + (size_t)(head - head0) * P.head_bytes + (size_t)P.page_size * (D + kind * (D / 32)) + (B0.in_page * 16 + r) * (D / 32) + f0 / 32;
                e[0] = (char)ea;
                e[D / 64] = (char)eb;
            }
        } else {
            if (kind == 0) rotate(a, b);
            if constexpr (!E4M3) {       // what the 16-bit type makes of it decides whether the row is finite
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const int pa = Half<F16>::pack(a[i], a[i + 1]), pb = Half<F16>::pack(b[i], b[i + 1]);
                    a[i] = Half<F16>::low(pa);
                    a[i + 1] = Half<F16>::high(pa);
                    b[i] = Half<F16>::low(pb);
                    b[i + 1] = Half<F16>::high(pb);
                }
            }
            // largest magnitude over the threads of the row, infinity if any holds a value that is not finite
            float amax = 0.f;
            bool fine = true;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                amax = fmaxf(amax, fmaxf(fabsf(a[i]), fabsf(b[i])));
                fine = fine && fabsf(a[i]) <= 3.402823466e38f && fabsf(b[i]) <= 3.402823466e38f;
            }
            if (!fine) amax = __builtin_inff();
#pragma unroll
            for (int d = 1; d < TPR; d <<= 1) amax = fmaxf(amax, __shfl_xor(amax, d, 64));
            fine = amax < __builtin_inff();
            float scale = 1.f;
            char *to = codes[unit] + (r * D + f0) * W;
            if constexpr (E4M3) {
                amax = fmaxf(amax, 0x1p-90f);
                scale = amax / 448.f;
                const float up = 448.f / amax;
                i32x2 x, y;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[i] = __builtin_amdgcn_cvt_pk_fp8_f32(a[4 * i] * up, a[4 * i + 1] * up, 0, false);
                    x[i] = __builtin_amdgcn_cvt_pk_fp8_f32(a[4 * i + 2] * up, a[4 * i + 3] * up, x[i], true);
                    y[i] = __builtin_amdgcn_cvt_pk_fp8_f32(b[4 * i] * up, b[4 * i + 1] * up, 0, false);
                    y[i] = __builtin_amdgcn_cvt_pk_fp8_f32(b[4 * i + 2] * up, b[4 * i + 3] * up, y[i], true);
                }
                *(i32x2 *)to = fine ? x : (i32x2){0, 0};
                *(i32x2 *)(to + D / 2) = fine ? y : (i32x2){0, 0};
            } else {
                i32x4 x, y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = Half<F16>::pack(a[2 * i], a[2 * i + 1]);
                    y[i] = Half<F16>::pack(b[2 * i], b[2 * i + 1]);
                }
                *(i32x4 *)to = fine ? x : (i32x4){0, 0, 0, 0};
                *(i32x4 *)(to + D) = fine ? y : (i32x4){0, 0, 0, 0};
            }
            if (there && f0 == 0) scales_of(B0)[(size_t)(head - head0) * (P.head_bytes / 4) + kind * P.page_size + r] = fine ? scale : __builtin_nanf("");
        }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        if (head0 + h >= P.kv) return;
        char *keys = B0.head + (size_t)h * P.head_bytes + (size_t)B0.in_page * 16 * ROW, *values = keys + (size_t)P.page_size * ROW;
        const char *kc = codes[2 * h], *vc = codes[2 * h + 1];
        if constexpr (E2M1) {
            constexpr int N = D / 32;            // words of a piece
            for (int i = threadIdx.x; i < 64 * N; i += 256) {
                const int pr = i / N & 15, g = i / N >> 4, w = i % N;
                if (pr >= lo && pr < hi) *(int *)(keys + i * 4) = *(const int *)(kc + pr * ROW + (g * N + w) * 4);
                if (lo == 0 && hi == 16) {
                    int piece = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) piece |= (int)(unsigned char)vc[(4 * g + k) * ROW + w * 16 + pr] << (8 * k);
                    *(int *)(values + i * 4) = piece;
                }
            }
            if (!(lo == 0 && hi == 16))
                for (int i = threadIdx.x; i < (hi - lo) * ROW; i += 256) {
                    const int pr = lo + i / ROW, w = i % ROW / 16, f = i % 16;
                    values[((pr / 4 * 16 + f) * N + w) * 4 + pr % 4] = vc[pr * ROW + i % ROW];
                }
            continue;
        }
        // keys: a 16-byte piece belongs to one position
        for (int i = threadIdx.x; i < D * W; i += 256) {
            const int pr = i & 15, g = (i >> 4) & 3, ch = i >> 6;
            if (pr >= lo && pr < hi) *(i32x4 *)(keys + i * 16) = *(const i32x4 *)(kc + (pr * D + ch * 4 * E + g * E) * W);
        }
        // values: a piece holds four positions.  Whole blocks go out in pieces, the others position by position.
        if (lo == 0 && hi == 16) {
            for (int i = threadIdx.x; i < D * W; i += 256) {
                const int pr = i & 15, g = (i >> 4) & 3, ch = i >> 6;
                union {
                    i32x4 v;
                    unsigned char b[16];
                    unsigned short h[8];
                } piece;
#pragma unroll
                for (int t = 0; t < E / 4; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int at = (4 * g + k) * D + pr + 16 * (ch * (E / 4) + t);
                        if constexpr (E4M3) piece.b[t * 4 + k] = vc[at];
                        else piece.h[t * 4 + k] = ((const unsigned short *)vc)[at];
                    }
                *(i32x4 *)(values + i * 16) = piece.v;
            }
        } else {
            for (int i = threadIdx.x; i < (hi - lo) * D; i += 256) {
                const int pr = lo + i / D, f = i % D, to = spd_page_value_off(pr, f, E);
                if constexpr (E4M3) values[to] = vc[pr * D + f];
                else ((unsigned short *)values)[to] = ((const unsigned short *)vc)[pr * D + f];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------
// Reading back.  One workgroup per four 16-position blocks and KV head, a wave per block; the heads of a block next to each other, since their rows are that in
// the output.  A lane's keys are pieces of rows; its values (four positions of several features) change places in the LDS, and so do keys of 4
// bits.  Bound by what is read and written.  The output goes past the caches, which cannot hold it, and leaves them to the codes.  4 bits, us a call: 24 contexts
// of up to 8000 on 5 heads, fp16, 421 MB: 92 -> 83 (heads next to each other) -> 66 (past the caches; 6.3 TB/s; codes read past them too 75); 16 of up to
// 4096 on one head, bf16, 29.5 MB: 7.0 -> 6.5.  e4m3, the latter (33 MB): 9.3 -> 7.9.
// ------------------------------------------------------------------------------------------
template <class Out, int D, int C, bool F16>
__global__ void __launch_bounds__(256) k_pages_read(Pages P, Out *k_out, Out *v_out) {
    constexpr bool E4M3 = C == SPD_E4M3;
    constexpr int W = E4M3 ? 1 : 2, E = 16 / W, CH = D / (4 * E), ROW = D + 16 / (int)sizeof(Out), PIECES = D * sizeof(Out) / 16;
    struct Piece {
        Out v[16 / sizeof(Out)];
    };
    __shared__ __attribute__((aligned(16))) Out turned[4][16 * ROW];
    const spd_plan_seq s = ((const spd_plan_seq *)(P.plan + P.seqs))[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % P.kv, r = lane & 15, g = lane >> 4;
    const int block = blockIdx.x / P.kv * 4 + wave;
    if (block * 16 >= s.end) return;             // (a wave works by itself)
    const Block B = block_at(P, s, head, block);
    Out *mine = turned[wave];
    const int n = s.end - block * 16 < 16 ? s.end - block * 16 : 16;
    const int64_t row0 = ((s.held0 + block * 16) * P.kv + head) * D, pitch = (int64_t)P.kv * D;
    auto put_rows = [&](Out *to) {               // of the LDS
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = lane; i < 16 * PIECES; i += 64) {
            const int pr = i / PIECES, f = (i % PIECES) * (16 / (int)sizeof(Out));
            if (pr < n)
                __builtin_nontemporal_store(*(const i32x4 *)__builtin_assume_aligned(mine + pr * ROW + f, 16), (i32x4 *)__builtin_assume_aligned(to + row0 + pr * pitch + f, 16));
        }
        __builtin_amdgcn_wave_barrier();
    };
    if constexpr (C == SPD_E2M1) {               // (bf16 holds every code * scale)
        constexpr int N = D / 32;
        typedef Half<false> H;
        const char *codes = B.head + B.in_page * (8 * D), *exps = B.head + (size_t)P.page_size * D + B.in_page * (16 * N);
        Codes4<D> kx, vx;
        Scales4<D> ve;
        kx.load(codes + lane * (4 * N));
        const unsigned ke = (unsigned)(unsigned char)exps[r * N + g * N / 4] << 23;
        vx.load(codes + (size_t)P.page_size * (D / 2) + lane * (4 * N));
        ve.load(exps + (size_t)P.page_size * N + 4 * N * g);
        auto put = [&](int at, int two) {        // two features side by side
            mine[at] = (Out)H::low(two);
            mine[at + 1] = (Out)H::high(two);
        };
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const i32x4 x = H::widen4(kx.c[i], ke);
#pragma unroll
            for (int j = 0; j < 4; ++j) put(r * ROW + g * (D / 4) + 8 * i + 2 * j, x[j]);
        }
        put_rows(k_out);
        auto turn = [&](auto u) {                // features r + 32 u and r + 32 u + 16
            constexpr int U = decltype(u)::value;
            i32x2 x, y;
            H::template turn4<U>(vx.c[U], ve.w, x, y);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Out *to = mine + (4 * g + j) * ROW + r + 32 * U;
                to[0] = (Out)(j & 1 ? H::high(x[j >> 1]) : H::low(x[j >> 1]));
                to[16] = (Out)(j & 1 ? H::high(y[j >> 1]) : H::low(y[j >> 1]));
            }
        };
        turn(std::integral_constant<int, 0>());
        turn(std::integral_constant<int, 1>());
        if constexpr (D == 128) {
            turn(std::integral_constant<int, 2>());
            turn(std::integral_constant<int, 3>());
        }
        put_rows(v_out);
        return;
    }
    const char *keys = B.head + (size_t)B.in_page * 16 * D * W, *values = keys + (size_t)P.page_size * D * W;
    const float *scales = (const float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16;
    i32x4 kx[CH], vx[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) kx[c] = *(const i32x4 *)(keys + c * 1024 + lane * 16);
#pragma unroll
    for (int c = 0; c < CH; ++c) vx[c] = *(const i32x4 *)(values + c * 1024 + lane * 16);
    const float ks = scales[r];
    const f32x4 vs = *(const f32x4 *)(scales + P.page_size + 4 * g);
    typedef Half<F16 && !E4M3> Codes;            // (e4m3 by way of bf16)
    auto pair = [&](const i32x4 &x, int i) {     // elements 2 i and 2 i + 1 of a piece, as 16-bit values
        if constexpr (E4M3) return i & 1 ? Codes::template from_e4m3<true>(x[i >> 1]) : Codes::template from_e4m3<false>(x[i >> 1]);
        else return x[i];
    };
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        Out piece[E];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const int k = pair(kx[c], i), v = pair(vx[c], i);
            piece[2 * i] = (Out)(Codes::low(k) * ks);
            piece[2 * i + 1] = (Out)(Codes::high(k) * ks);
            // elements 4 t .. 4 t + 3: positions 4 g .. of feature r + 16 (E / 4 c + t)
            const int f = r + 16 * (c * (E / 4) + i / 2), p = 4 * g + 2 * (i & 1);
            mine[p * ROW + f] = (Out)(Codes::low(v) * vs[2 * (i & 1)]);
            mine[(p + 1) * ROW + f] = (Out)(Codes::high(v) * vs[2 * (i & 1) + 1]);
        }
        if (r < n) {
#pragma unroll
            for (int i = 0; i < E; i += 16 / (int)sizeof(Out)) {
                Piece q;
#pragma unroll
                for (int e = 0; e < 16 / (int)sizeof(Out); ++e) q.v[e] = piece[i + e];
                __builtin_nontemporal_store(__builtin_bit_cast(i32x4, q), (i32x4 *)__builtin_assume_aligned(k_out + row0 + r * pitch + c * 4 * E + g * E + i, 16));
            }
        }
    }
    put_rows(v_out);
}

// ------------------------------------------------------------------------------------------
// Attention
// ------------------------------------------------------------------------------------------
struct AttendArgs {
    Pages P;
    const unsigned short *q;
    unsigned short *out;
    int64_t ld_q, ld_out;
    float *part;                // partial results of this kernel's items
    int *counters;
    int window, sinks;
    float scale;                // log2(e) / sqrt(head_dim): softmax in powers of two
};

// Beside e4m3 the fp16 kernels keep the maximum of score + log2(scale).  A smaller scale (0 where a cleared page was never written) counts as this
// one: its values are below 2^-31, nothing in fp16, and a probability, which may be 1 / scale of the maximum, stays far enough from
// fp32's end for sums over as many keys as there can be.
constexpr float LEAST_SCALE = 0x1p-40f;

// is `key` visible to a query at position `at`?
__device__ __forceinline__ bool visible(int key, int at, int window, int sinks) {
    return (key <= at) & ((window == 0) | (key > at - window) | (key < sinks));
}
__device__ __forceinline__ int list_block(const spd_plan_item &it, int v) { return v < it.sink_blocks ? v : it.block0 + (v - it.sink_blocks); }

// is the whole block visible to every query between positions `first` and `last`?
__device__ __forceinline__ bool all_visible(int block, int first, int last, int window, int sinks) {
    const int k0 = block * 16, k1 = k0 + 15;
    return k1 <= first && (window == 0 || k0 > last - window || k1 < sinks);
}

// operands of one 16-position block, as loaded
template <int D, int C>
struct BlockLoad {
    static constexpr bool E4M3 = C == SPD_E4M3;
    static constexpr int CH = E4M3 ? D / 64 : D / 32;      // 16-byte chunks per lane, keys and values each
    i32x4 k[CH], v[CH];
    f32x4 ks, vs;                                           // scales of keys 4 g .. 4 g + 3
    __device__ __forceinline__ void load(const Pages &P, const Block &B, int lane) {
        constexpr int W = E4M3 ? 1 : 2;
        const char *keys = B.head + (size_t)B.in_page * 16 * D * W, *values = keys + (size_t)P.page_size * D * W;
        const float *scales = (const float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16;
        const int g4 = 4 * (lane >> 4);
#pragma unroll
        for (int c = 0; c < CH; ++c) k[c] = __builtin_nontemporal_load((const i32x4 *)(keys + c * 1024 + lane * 16));
        ks = *(const f32x4 *)(scales + g4);
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = __builtin_nontemporal_load((const i32x4 *)(values + c * 1024 + lane * 16));
        vs = *(const f32x4 *)(scales + P.page_size + g4);
    }
};

template <int D>
struct BlockLoad<D, SPD_E2M1> {
    static constexpr int N = D / 32;                        // groups of a row
    Codes4<D> k, v;
    Scales4<D> ve;                                          // of values 4 g .. 4 g + 3
    unsigned char ke;                                       // of the lane's features of its key
    __device__ __forceinline__ void load_keys(const Pages &P, const Block &B, int lane) {
        const int r = lane & 15, g = lane >> 4;
        k.stream(B.head + B.in_page * (8 * D) + lane * (4 * N));
        ke = B.head[(size_t)P.page_size * D + B.in_page * (16 * N) + r * N + g * N / 4];
    }
    __device__ __forceinline__ void load_values(const Pages &P, const Block &B, int lane) {
        v.stream(B.head + (size_t)P.page_size * (D / 2) + B.in_page * (8 * D) + lane * (4 * N));
        ve.load(B.head + (size_t)P.page_size * (D + N) + B.in_page * (16 * N) + 4 * N * (lane >> 4));
    }
};

// what of a block is asked for
struct Both {
    template <class L>
    __device__ __forceinline__ void operator()(L &x, const Pages &P, const Block &B, int lane) const { x.load(P, B, lane); }
};
struct Keys {
    template <class L>
    __device__ __forceinline__ void operator()(L &x, const Pages &P, const Block &B, int lane) const { x.load_keys(P, B, lane); }
};
struct Values {
    template <class L>
    __device__ __forceinline__ void operator()(L &x, const Pages &P, const Block &B, int lane) const { x.load_values(P, B, lane); }
};

// A partial result is written by one workgroup and read by another, perhaps on another die with an L2 of its own: both go past that
// L2, as relaxed atomics of the device's scope do.
__device__ __forceinline__ void part_put(float *p, float a, float b) {
    const unsigned long long v = (unsigned long long)__float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32;
    __hip_atomic_store((unsigned long long *)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 part_get(const float *p) {
    const unsigned long long v = __hip_atomic_load((const unsigned long long *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}

// Few rows (a decode step, a short draft): one workgroup per item and KV head, its eight waves take pairs of blocks in turn and merge
// their states in the LDS.  Rows cut into several items are joined, in the items' order, by the workgroup that ends last.
// Lane = 16 g + row.
// Bound by HBM where there is enough to read, else by loads that wait for each other (plan, page, keys, values, the join: 7.8 us for one sequence of 2048).  4 bits: keys
// and values are asked for as soon as those in their registers are done with, 118 registers, two workgroups to a compute unit; outputs are scaled only where
// the maximum has grown by 2^8.  16 sequences of 8001 on 32 heads 87 us (557 MB: 6.4 TB/s; 105 with pairs of blocks in registers of their own and one
// workgroup), 48 of up to 16000 on one 19.4 (21.8).
// (so, sm, sl, ended: its LDS, objects of the kernel of their own, which the compiler then knows to lie apart)
template <int D>
using SmallOutputs = float[SPD_SMALL_WAVES][16][D + 4];
typedef float SmallRows[SPD_SMALL_WAVES][16];
template <int D, int C, bool F16>
__device__ __forceinline__ void attend_small(const AttendArgs &A, unsigned block, SmallOutputs<D> &so, SmallRows &sm, SmallRows &sl, int &ended) {
    constexpr bool E4M3 = C == SPD_E4M3, E2M1 = C == SPD_E2M1;
    constexpr int DT = D / 16, NF = D / 32, NW = SPD_SMALL_WAVES;
    typedef Half<F16> H;
    // fp16 has no room for a probability times a scale that may be tiny: there the maximum kept is that of the product, log2(scale) added to the score
    constexpr bool PRODUCT = F16 && E4M3;
    const Pages &P = A.P;
    const int head = block % P.kv;
    const spd_plan_item it = ((const spd_plan_item *)(P.plan + P.list))[block / P.kv];
    if (P.on_device && ((int)(block / P.kv) >= header_of(P).n_small || it.count == 0)) return;
    const spd_plan_seq &s = it.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int rows = s.q_len * P.group;          // at most 16
    const int token = row / P.group;
    const int at = s.pos + token, last = s.end - 1;
    // the wave's pairs are number wave, wave + NW, ... of the item's; lane i keeps the page of the i-th of the next 64 blocks
    const int n_pairs = (it.count + 1) / 2, mine = (n_pairs - wave + NW - 1) / NW;
    auto my_block = [&](int i) {                 // i-th block of the wave (the missing half of the last pair: its first)
        const int v = 2 * (wave + NW * (i >> 1)) + (i & 1);
        return list_block(it, it.first + (v < it.count ? v : it.count - 1));
    };
    int pages = mine > 0 ? page_of(P, s, my_block(lane < 2 * mine ? lane : 0)) : 0;
    i32x4 qf[NF];
    {
        const unsigned short *qp = A.q + (int64_t)(s.tok0 + token) * A.ld_q + (int64_t)(head * P.group + row % P.group) * D;
#pragma unroll
        for (int i = 0; i < NF; ++i) {           // the features that lane (g, .) of a key holds
            const int f = E4M3 ? 64 * (i >> 1) + 16 * g + 8 * (i & 1) : E2M1 ? D / 4 * g + 8 * i : 32 * i + 8 * g;
            qf[i] = row < rows ? *(const i32x4 *)(qp + f) : (i32x4){0, 0, 0, 0};
        }
    }
    f32x4 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;
    struct Pair {
        BlockLoad<D, C> x[2];
    };
    auto load = [&](Pair &f, int j, auto ask) __attribute__((always_inline)) {      // pair j of the wave, or its keys or values (keys first)
        if (!std::is_same<decltype(ask), Values>::value && j > 0 && (j & 31) == 0) {
            pages = page_of(P, s, my_block(2 * j + lane < 2 * mine ? 2 * j + lane : 2 * j));
            if constexpr (E2M1) asm volatile("" : "+v"(pages));      // (waited for here, and not, with all that is on its way, wherever pages are looked up)
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = __builtin_amdgcn_readlane(pages, (2 * j + h) & 63);
            ask(f.x[h], P, block_in(P, page, head, my_block(2 * j + h)), lane);
        }
    };
    auto use = [&](Pair &f, int j, auto more) __attribute__((always_inline)) {      // more: the next pair is asked for into the same registers
        constexpr bool MORE = decltype(more)::value;
        const bool two = 2 * (wave + NW * j) + 1 < it.count;
        const int b0 = my_block(2 * j), b1 = my_block(2 * j + 1);
        const BlockLoad<D, C> &x0 = f.x[0], &x1 = f.x[1];
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
        Scales4<D> e0, e1;                       // 4 bits: of the values
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            i32x4 k0, k1;
            if constexpr (E4M3) {
                k0 = H::widen(x0.k[i >> 1][2 * (i & 1)], x0.k[i >> 1][2 * (i & 1) + 1]);
                k1 = H::widen(x1.k[i >> 1][2 * (i & 1)], x1.k[i >> 1][2 * (i & 1) + 1]);
            } else if constexpr (E2M1) {
                k0 = H::widen4(x0.k.c[i], (unsigned)x0.ke << 23);
                k1 = H::widen4(x1.k.c[i], (unsigned)x1.ke << 23);
            } else {
                k0 = x0.k[i];
                k1 = x1.k[i];
            }
            s0 = H::mfma16(k0, qf[i], s0);
            s1 = H::mfma16(k1, qf[i], s1);
        }
        f32x4 v0, v1;
        if constexpr (E2M1) {
            if constexpr (MORE) load(f, j + 1, Keys());
            __builtin_amdgcn_sched_barrier(0);   // (ahead of anything that waits for this pair's values)
            v0 = v1 = (f32x4){1.f, 1.f, 1.f, 1.f};
        } else {
            v0 = x0.vs;
            v1 = x1.vs;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s0[i] *= x0.ks[i] * A.scale;
                s1[i] *= x1.ks[i] * A.scale;
            }
        }
        // (the scale of a hidden key's value may be NaN)
        const bool mixed = !(two && all_visible(b0, s.pos, last, A.window, A.sinks) && all_visible(b1, s.pos, last, A.window, A.sinks));
        if (mixed) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (selections, no branches: of a branch over the whole wave around one over lanes this compiler has lost the inner one's assignments)
                const int k0 = b0 * 16 + 4 * g + i, k1 = b1 * 16 + 4 * g + i;
                const bool see0 = visible(k0, at, A.window, A.sinks), see1 = visible(two ? k1 : 0x7fffffff, at, A.window, A.sinks);
                s0[i] = see0 ? s0[i] : -__builtin_inff();
                v0[i] = see0 ? v0[i] : 0.f;
                s1[i] = see1 ? s1[i] : -__builtin_inff();
                v1[i] = see1 ? v1[i] : 0.f;
            }
        }
        float mx = -__builtin_inff();
        if constexpr (E2M1) s0 *= A.scale, s1 *= A.scale;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (a hidden key's score is -inf, whatever log2 makes of its scale of 0)
            const float a0 = PRODUCT ? s0[i] + __builtin_amdgcn_logf(fmaxf(v0[i], LEAST_SCALE)) : s0[i],
                        a1 = PRODUCT ? s1[i] + __builtin_amdgcn_logf(fmaxf(v1[i], LEAST_SCALE)) : s1[i];
            mx = fmaxf(mx, fmaxf(a0, a1));
        }
        float alpha = 1.f, m_new, m_use;
        if constexpr (E2M1) {
            // The maximum only keeps the powers of two in range: while it grows by less than 2^8 it stays, and the outputs with it
            const float top = quad_max(mx);
            m_new = m;
            if (__builtin_amdgcn_ballot_w64(top > m + 8.f)) {
                m_new = fmaxf(m, top);
                alpha = __builtin_amdgcn_exp2f(m - (m_new == -__builtin_inff() ? 0.f : m_new));
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] *= alpha;
            }
            m_use = m_new == -__builtin_inff() ? 0.f : m_new;
        } else {
            m_new = fmaxf(m, quad_max(mx));
            m_use = m_new == -__builtin_inff() ? 0.f : m_new;
            alpha = __builtin_amdgcn_exp2f(m - m_use);
        }
        float ps = 0.f, w0[4], w1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(s0[i] - m_use), p1 = __builtin_amdgcn_exp2f(s1[i] - m_use);
            ps += p0 + p1;
            w0[i] = E2M1 ? p0 : p0 * v0[i];
            w1[i] = E2M1 ? p1 : p1 * v1[i];
        }
        if constexpr (E2M1) {
            e0 = x0.ve;
            e1 = x1.ve;
            // behind the sequence's end a page holds anything
            if (mixed)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e0.w[i] = b0 * 16 + 4 * g + i > last ? 0 : e0.w[i];
                    e1.w[i] = b1 * 16 + 4 * g + i > last ? 0 : e1.w[i];
                }
            // A value that is not finite makes NaN of whoever sees it, and nothing else (a key's score has become NaN by its scale)
            if (__builtin_amdgcn_ballot_w64((e0.most() > e1.most() ? e0.most() : e1.most()) == Scales4<D>::BAD))
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool bad0 = (e0.w[i] == e0.BAD) & (s0[i] != -__builtin_inff()), bad1 = (e1.w[i] == e1.BAD) & (s1[i] != -__builtin_inff());
                    w0[i] = bad0 ? __builtin_nanf("") : w0[i];
                    w1[i] = bad1 ? __builtin_nanf("") : w1[i];
                    ps = (bad0 | bad1) ? __builtin_nanf("") : ps;
                    e0.w[i] = e0.w[i] == e0.BAD ? 0 : e0.w[i];
                    e1.w[i] = e1.w[i] == e1.BAD ? 0 : e1.w[i];
                }
        }
        l = l * alpha + ps;                      // (of the lane's keys; the four lanes of a row meet at the end)
        m = m_new;
        const i32x4 pf = {H::pack(w0[0], w0[1]), H::pack(w0[2], w0[3]), H::pack(w1[0], w1[1]), H::pack(w1[2], w1[3])};
        if constexpr (E2M1) {
            auto outputs = [&](auto u) __attribute__((always_inline)) {      // features r + 32 u and r + 32 u + 16
                constexpr int U = decltype(u)::value;
                i32x2 a0, b0, a1, b1;
                H::template turn4<U>(x0.v.c[U], e0.w, a0, b0);
                H::template turn4<U>(x1.v.c[U], e1.w, a1, b1);
                o[2 * U] = H::mfma16((i32x4){a0[0], a0[1], a1[0], a1[1]}, pf, o[2 * U]);
                o[2 * U + 1] = H::mfma16((i32x4){b0[0], b0[1], b1[0], b1[1]}, pf, o[2 * U + 1]);
            };
            outputs(std::integral_constant<int, 0>());
            outputs(std::integral_constant<int, 1>());
            if constexpr (D == 128) {
                outputs(std::integral_constant<int, 2>());
                outputs(std::integral_constant<int, 3>());
            }
            if constexpr (MORE) load(f, j + 1, Values());
        } else
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            i32x4 vf;
            if constexpr (E4M3) vf = H::widen(x0.v[t >> 2][t & 3], x1.v[t >> 2][t & 3]);
            else vf = (i32x4){x0.v[t >> 1][2 * (t & 1)], x0.v[t >> 1][2 * (t & 1) + 1], x1.v[t >> 1][2 * (t & 1)], x1.v[t >> 1][2 * (t & 1) + 1]};
            o[t] = H::mfma16(vf, pf, o[t] * alpha);
        }
    };
    if constexpr (E2M1) {
        // The next keys are asked for into the registers of those whose scores are done, the next values into theirs: half of the registers, so
        // that two workgroups fit on a compute unit
        if (mine > 0) {
            Pair f;
            load(f, 0, Keys());
            __builtin_amdgcn_sched_barrier(0);   // (in this order, so that the wait for keys is none for values)
            load(f, 0, Values());
            for (int j = 0; j < mine - 1; ++j) use(f, j, std::true_type());
            use(f, mine - 1, std::false_type());
        }
    } else if (mine > 0) {
        Pair f0, f1;
        load(f0, 0, Both());
        for (int j = 0; j < mine; j += 2) {      // the next pair is on its way while one is used
            if (j + 1 < mine) load(f1, j + 1, Both());
            use(f0, j, std::false_type());
            if (j + 1 < mine) {
                if (j + 2 < mine) load(f0, j + 2, Both());
                use(f1, j + 1, std::false_type());
            }
        }
    }
    l = quad_sum(l);
    // merge the waves
#pragma unroll
    for (int t = 0; t < DT; ++t) *(f32x4 *)&so[wave][row][t * 16 + 4 * g] = o[t];
    if (g == 0) {
        sm[wave][row] = m;
        sl[wave][row] = l;
    }
    __syncthreads();
    constexpr int N = D / 32;                    // of a row by each of 32 threads
    const int mr = threadIdx.x >> 5, f0 = (threadIdx.x & 31) * N;
    float mm = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < NW; ++w) mm = fmaxf(mm, sm[w][mr]);
    float m_use = mm == -__builtin_inff() ? 0.f : mm;
    float ll = 0.f, acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm[w][mr] - m_use);
        ll += f * sl[w][mr];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] += f * so[w][mr][f0 + i];
    }
    if (it.slot >= 0) {
        constexpr int PART = SPD_SMALL_ROWS * (D + 2), ML = SPD_SMALL_ROWS * D;
        float *to = A.part + ((size_t)it.slot * P.kv + head) * PART;
        if (mr < rows) {
#pragma unroll
            for (int i = 0; i < N; i += 2) part_put(to + mr * D + f0 + i, acc[i], acc[i + 1]);
            if (f0 == 0) part_put(to + ML + 2 * mr, mm, ll);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the wave's part has left
        __syncthreads();
        int *counter = A.counters + it.group * P.kv + head;
        if (threadIdx.x == 0) ended = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (ended != it.parts - 1) return;
        if (threadIdx.x == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // 32 threads per row and set of parts: with fewer than sixteen rows several sets side by side, joined in the LDS
        const int rshift = rows > 8 ? 4 : rows > 4 ? 3 : rows > 2 ? 2 : rows > 1 ? 1 : 0, sets = 16 >> rshift;
        const int jr = mr & ((1 << rshift) - 1), set = mr >> rshift;
        const float *p = A.part + ((size_t)it.slot0 * P.kv + head) * PART;
        const size_t step = (size_t)P.kv * PART;
        mm = -__builtin_inff();
        ll = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.f;
        constexpr int NB = 8;                    // parts asked for at a time
        if (jr < rows)
            for (int i0 = set; i0 < it.parts; i0 += NB * sets) {
                float2 ml[NB], x[NB][N / 2];
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    const float *q = p + (size_t)(i0 + u * sets < it.parts ? i0 + u * sets : i0) * step;
                    ml[u] = part_get(q + ML + 2 * jr);
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) x[u][i] = part_get(q + jr * D + f0 + 2 * i);
                }
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    if (i0 + u * sets >= it.parts) break;
                    const float m_new = fmaxf(mm, ml[u].x);
                    m_use = m_new == -__builtin_inff() ? 0.f : m_new;
                    const float fa = __builtin_amdgcn_exp2f(mm - m_use), fb = __builtin_amdgcn_exp2f(ml[u].x - m_use);
                    mm = m_new;
                    ll = ll * fa + ml[u].y * fb;
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) {
                        acc[2 * i] = acc[2 * i] * fa + x[u][i].x * fb;
                        acc[2 * i + 1] = acc[2 * i + 1] * fa + x[u][i].y * fb;
                    }
                }
            }
        if (sets > 1) {
            float *lo = &so[0][0][0], *lm = &sm[0][0], *ls = &sl[0][0];      // (sixteen rows of the waves' places)
#pragma unroll
            for (int i = 0; i < N; ++i) lo[mr * (D + 4) + f0 + i] = acc[i];
            if (f0 == 0) {
                lm[mr] = mm;
                ls[mr] = ll;
            }
            __syncthreads();
            if (mr >= rows) return;
            mm = -__builtin_inff();
            for (int u = 0; u < sets; ++u) mm = fmaxf(mm, lm[(u << rshift) + mr]);
            m_use = mm == -__builtin_inff() ? 0.f : mm;
            ll = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = 0.f;
            for (int u = 0; u < sets; ++u) {
                const int from = (u << rshift) + mr;
                const float f = __builtin_amdgcn_exp2f(lm[from] - m_use);
                ll += f * ls[from];
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] += f * lo[from * (D + 4) + f0 + i];
            }
        }
    }
    if (mr >= rows) return;
    int *to = (int *)(A.out + (int64_t)(s.tok0 + mr / P.group) * A.ld_out + (int64_t)(head * P.group + mr % P.group) * D + f0);
    const float inv = 1.f / ll;
#pragma unroll
    for (int i = 0; i < N; i += 2) to[i / 2] = H::pack(acc[i] * inv, acc[i + 1] * inv);
}
template <int D, int C, bool F16>
__global__ void __launch_bounds__(512, C == SPD_E2M1 ? 4 : 1) k_attend_small(AttendArgs A) {
    __shared__ SmallOutputs<D> so;
    __shared__ SmallRows sm, sl;
    __shared__ int ended;
    attend_small<D, C, F16>(A, blockIdx.x, so, sm, sl, ended);
}

// Many rows (a prompt's chunk): one workgroup per 128 rows and KV head; each wave has 32 of them, tiles of 64 keys go through the LDS in 16
// bits, dequantised once for the workgroup, two stages: while one is used the next is loaded into registers, and put away beside the second
// contraction.  Lane = 32 half + row.  Bound by the vector instructions beside the matrix instructions (52 and 36 % of a SIMD's cycles, the LDS 43):
// four prompts of 2048 tokens on 64 heads of 8 in 335 us, 0.82 PFLOP/s, where nothing but MFMAs on such data does 1.7.  (Two row tiles per wave
// and one workgroup per compute unit, which read the LDS half as often: 541 us beside 363, no second wave to work beside the first's softmax.)
// 16-bit pages need no scales, a bad row's key is NaN instead: three windowed chunks of 333 tokens 26.8 -> 23.7 us.
// 4-bit pages are 16-bit values once they are in the LDS (code and scale widened in one instruction): the prompts 310 to 318 us, 0.87 PFLOP/s; 1.97 us a tile
// with two workgroups on a compute unit, 51 of the 318 starts and ends of the 4096 workgroups, clock 1.97 GHz.  (The scores contracted in 4 bits, with queries in 8: no faster, and
// that instruction's own sum is good to 2^-12 of its largest product only.  Scores of the next tile beside the softmax of this one: 256 registers, 326 beside 321.)
template <int D, int C, bool F16>
__global__ void __launch_bounds__(256, 2) k_attend_large(AttendArgs A) {
    constexpr bool E4M3 = C == SPD_E4M3, E2M1 = C == SPD_E2M1;
    constexpr int W = E4M3 ? 1 : 2, KS = D / 16, DT = D / 32, CH = C == HALVES ? D / 32 : D / 64, N4 = D / 32;
    typedef Half<F16> H;
    constexpr bool PRODUCT = F16 && E4M3;        // the maximum kept is that of probability times scale, as in the kernel for few rows
    const Pages &P = A.P;
    const int head = blockIdx.x % P.kv;
    const spd_plan_item it = ((const spd_plan_item *)(P.plan + P.list))[blockIdx.x / P.kv];
    if (P.on_device && ((int)(blockIdx.x / P.kv) >= header_of(P).n_large || it.count == 0)) return;
    const spd_plan_seq &s = it.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int n_rows = s.q_len * P.group;
    const int row = it.row0 + wave * 32 + col;
    const bool live = row < n_rows;
    const int token = (live ? row : n_rows - 1) / P.group, qh = head * P.group + (live ? row : n_rows - 1) % P.group;
    const int at = s.pos + token;
    const int first_at = __builtin_amdgcn_readfirstlane(at), last_at = __builtin_amdgcn_readlane(at, 31);
    // keys: [block][feature / 8][position][8]; values: [block][feature / 16][half][feature % 16][8 positions of the half]
    struct Stage {
        short k[64 * D], v[64 * D];
        float ks[64], vs[64], lv[PRODUCT ? 64 : 4];      // e4m3: the keys' scales times the softmax's; the values', and their log2
    };
    __shared__ __attribute__((aligned(16))) Stage stage[2];
    i32x4 qf[KS];
    {
        const unsigned short *qp = A.q + (int64_t)(s.tok0 + token) * A.ld_q + (int64_t)qh * D;
#pragma unroll
        for (int i = 0; i < KS; ++i) qf[i] = live ? *(const i32x4 *)(qp + 16 * i + 8 * half) : (i32x4){0, 0, 0, 0};
    }
    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -__builtin_inff(), l = 0.f;
    // wave w brings block w of a tile
    const int r16 = lane & 15, g = lane >> 4;
    auto my_block = [&](int v0) { return list_block(it, it.first + (v0 + wave < it.count ? v0 + wave : it.count - 1)); };
    i32x4 kx[CH], vx[CH];
    float sx = 0.f, sv = 0.f;
    Codes4<D> kx4, vx4;                          // 4 bits: codes, scales of four positions' values, of the lane's features of its key, one of its value
    Scales4<D> ve;
    unsigned ke = 0, vbad = 0;
    auto fetch = [&](int v0, int page) __attribute__((always_inline)) {
        const Block B = block_in(P, page, head, my_block(v0));
        if constexpr (E2M1) {
            const char *codes = B.head + B.in_page * (8 * D), *exps = B.head + (size_t)P.page_size * D + B.in_page * (16 * N4);
            kx4.load(codes + lane * (4 * N4));
            vx4.load(codes + (size_t)P.page_size * (D / 2) + lane * (4 * N4));
            ke = (unsigned char)exps[r16 * N4 + g * N4 / 4];
            vbad = (unsigned char)exps[(size_t)P.page_size * N4 + r16 * N4];
            ve.load(exps + (size_t)P.page_size * N4 + 4 * N4 * g);
            return;
        }
        const char *keys = B.head + (size_t)B.in_page * 16 * D * W, *values = keys + (size_t)P.page_size * D * W;
        const float *scales = (const float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16;
#pragma unroll
        for (int c = 0; c < CH; ++c) kx[c] = *(const i32x4 *)(keys + c * 1024 + lane * 16);
#pragma unroll
        for (int c = 0; c < CH; ++c) vx[c] = *(const i32x4 *)(values + c * 1024 + lane * 16);
        // (16-bit pages: every lane those of its key, which is what tells of a bad row)
        if constexpr (E4M3) {
            if (lane < 32) sx = scales[lane < 16 ? r16 : P.page_size + r16];
        } else {
            sx = scales[r16];
            sv = scales[P.page_size + r16];
        }
    };
    // (after the last tile what is put away is not read)
    auto put_away = [&](int c, Stage &to) __attribute__((always_inline)) {
        short *kd = to.k + wave * 16 * D, *vd = to.v + wave * 16 * D;
        if constexpr (E2M1) {
            if (c == 0) {
                // the key of a value that was not finite is NaN, so that its score is, and its codes are zero
                ke = (vbad == 255 ? 255u : ke) << 23;
#pragma unroll
                for (int j = 0; j < 4; ++j)      // (any byte of 255: behind the sequence's end a page holds anything)
                    ve.w[j] = (~ve.w[j] - 0x01010101u) & ve.w[j] & 0x80808080u ? 0 : ve.w[j];
            }
            auto half4 = [&](auto u) __attribute__((always_inline)) {
                constexpr int U = decltype(u)::value;
                *(i32x4 *)(kd + ((N4 * g + U) * 16 + r16) * 8) = H::widen4(kx4.c[U], ke);
                i32x2 a, b;
                H::template turn4<U>(vx4.c[U], ve.w, a, b);
                *(i32x2 *)(vd + ((2 * U * 2 + (g & 1)) * 16 + r16) * 8 + (g >> 1) * 4) = a;
                *(i32x2 *)(vd + (((2 * U + 1) * 2 + (g & 1)) * 16 + r16) * 8 + (g >> 1) * 4) = b;
            };
            if (c == 0) {
                half4(std::integral_constant<int, 0>());
                half4(std::integral_constant<int, 1>());
            } else if constexpr (D == 128) {
                half4(std::integral_constant<int, 2>());
                half4(std::integral_constant<int, 3>());
            }
        } else if constexpr (E4M3) {
            *(i32x4 *)(kd + ((8 * c + 2 * g) * 16 + r16) * 8) = H::widen(kx[c][0], kx[c][1]);
            *(i32x4 *)(kd + ((8 * c + 2 * g + 1) * 16 + r16) * 8) = H::widen(kx[c][2], kx[c][3]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                *(i32x2 *)(vd + (((4 * c + t) * 2 + (g & 1)) * 16 + r16) * 8 + (g >> 1) * 4) =
                    (i32x2){H::template from_e4m3<false>(vx[c][t]), H::template from_e4m3<true>(vx[c][t])};
        } else {
            // Scales are 1, or NaN for a row that was not finite: its key becomes NaN, so that its score is, and its codes are zero
            const bool bad = !(sx + sv < 3.f);
            *(i32x4 *)(kd + ((4 * c + g) * 16 + r16) * 8) = bad ? (i32x4){0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff} : kx[c];
#pragma unroll
            for (int t = 0; t < 2; ++t)
                *(i32x2 *)(vd + (((2 * c + t) * 2 + (g & 1)) * 16 + r16) * 8 + (g >> 1) * 4) = (i32x2){vx[c][2 * t], vx[c][2 * t + 1]};
        }
    };
    auto put_scales = [&](Stage &to) __attribute__((always_inline)) {
        if constexpr (!E4M3) return;
        // a value that is NaN makes its key's score NaN, and nothing else: whoever sees it gets NaN
        const float vs = __shfl(sx, r16 + 16, 64);
        if (g == 0) to.ks[wave * 16 + r16] = vs == vs ? sx * A.scale : vs;
        else if (g == 1) to.vs[wave * 16 + r16] = vs == vs ? vs : 0.f;
        else if (PRODUCT && g == 2) to.lv[wave * 16 + r16] = vs == vs ? __builtin_amdgcn_logf(fmaxf(vs, LEAST_SCALE)) : 0.f;
    };
    int page = page_of(P, s, my_block(0));
    fetch(0, page);
    page = page_of(P, s, my_block(4));
#pragma unroll
    for (int c = 0; c < CH; ++c) put_away(c, stage[0]);
    put_scales(stage[0]);
    // (a tile is asked for as soon as the registers of the one before are put away: the scores' time and half of the outputs' to arrive in)
    if (4 < it.count) {
        fetch(4, page);
        page = page_of(P, s, my_block(8));
    }
    __syncthreads();
    // Operands and scales are read from the LDS some instructions ahead of their use, fenced so that the compiler leaves them there (read
    // where they are used, a wave waits for the LDS 24 times a tile).
    constexpr int AHEAD = 4;
    const int k_lane = (col >> 4) * 16 * D + (half * 16 + (col & 15)) * 8, v_lane = (((col >> 4) * 2 + half) * 16 + (col & 15)) * 8;
    i32x4 ring[AHEAD];
    f32x4 ks[4], vs[4], lv[2];      // (lv: this group of four and the next; there are no registers for more)
    f32x16 sc[2];
    int v0 = 0, turn = 0;
    // Scores of tile v0, which lies in stage `turn`, and their maximum over the row: score i of half h is of block 2 h + i / 8, position
    // 8 ((i / 4) % 2) + 4 half + i % 4 in it.
    auto scores = [&]() __attribute__((always_inline)) {
        const Stage &now = stage[turn];
        const short *kp = now.k + k_lane;
        auto frag = [&](int n) __attribute__((always_inline)) { return *(const i32x4 *)(kp + (n / KS) * 32 * D + (n % KS) * 256); };
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) ring[n] = frag(n);
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[0][i] = sc[1][i] = 0.f;
        float mx = -__builtin_inff();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) {
            sc[n / KS] = H::mfma32(ring[n % AHEAD], qf[n % KS], sc[n / KS]);
            __builtin_amdgcn_sched_barrier(0);
            if (n + AHEAD < 2 * KS) ring[n % AHEAD] = frag(n + AHEAD);
            if (E4M3 && n < 4) ks[n] = *(const f32x4 *)(now.ks + n * 8 + 4 * half);
            if (PRODUCT && n >= KS - 2 && n < KS) lv[n - KS + 2] = *(const f32x4 *)(now.lv + (n - KS + 2) * 8 + 4 * half);
            if (n >= KS) {                       // beside the second half's: the first half scaled, and its maximum
                constexpr int PER = 16 / KS;
#pragma unroll
                for (int i = (n - KS) * PER; i < (n - KS + 1) * PER; ++i) {
                    if constexpr (E4M3) sc[0][i] *= ks[i >> 2][i & 3];
                    mx = fmaxf(mx, PRODUCT ? sc[0][i] + lv[(i >> 2) & 1][i & 3] : sc[0][i]);
                    if (E4M3 && (i & 3) == 3) {
                        ks[i >> 2] = *(const f32x4 *)(now.ks + 32 + (i >> 2) * 8 + 4 * half);
                        if constexpr (PRODUCT) lv[(i >> 2) & 1] = *(const f32x4 *)(now.lv + ((i >> 2) + 2) * 8 + 4 * half);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if constexpr (E4M3) vs[q] = *(const f32x4 *)(now.vs + q * 8 + 4 * half);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (E4M3) sc[1][i] *= ks[i >> 2][i & 3];
            mx = fmaxf(mx, PRODUCT ? sc[1][i] + lv[(i >> 2) & 1][i & 3] : sc[1][i]);
            if (PRODUCT && (i & 3) == 3 && i < 8) lv[(i >> 2) & 1] = *(const f32x4 *)(now.lv + ((i >> 2) + 6) * 8 + 4 * half);
        }
        // is something of the tile hidden from some query of the wave?  (first and last block; a tile of sinks and window blocks is mixed)
        const int n_here = it.count - v0 < 4 ? it.count - v0 : 4;
        const int b_first = list_block(it, it.first + v0), b_last = list_block(it, it.first + v0 + n_here - 1);
        if (!(n_here == 4 && b_last * 16 + 15 <= first_at && (A.window == 0 || b_first * 16 > last_at - A.window || b_last * 16 + 15 < A.sinks))) {
            mx = -__builtin_inff();
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int key0 = (q >> 1) < n_here ? list_block(it, it.first + v0 + (q >> 1)) * 16 : 0x7fffff0;
                const f32x4 ls = *(const f32x4 *)(now.lv + (PRODUCT ? q * 8 + 4 * half : 0));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool seen = visible(key0 + 8 * (q & 1) + 4 * half + i, at, A.window, A.sinks);
                    const float x = seen ? sc[q >> 2][(q & 3) * 4 + i] : -__builtin_inff();
                    sc[q >> 2][(q & 3) * 4 + i] = x;
                    mx = fmaxf(mx, PRODUCT ? x + ls[i] : x);
                }
            }
        }
        return E4M3 ? half_max(mx) : half_max(mx) * A.scale;      // (16-bit pages: the scores stay as they are)
    };
    float mx = scores();
    while (true) {
        // The maximum only keeps the powers of two in range: while it grows by less than 2^8 it stays, and the outputs with it, in the inner loop.
        {
            const float m_new = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - (m_new == -__builtin_inff() ? 0.f : m_new));
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
        }
        const float m_use = m == -__builtin_inff() ? 0.f : m;
        bool grown = false;
        do {
            const Stage &now = stage[turn];
            i32x4 pf[4];
            float ps = 0.f, w[2];
            // element i (of 32) of the scores: its power of two, with the value's scale, a pair at a time into the operand
            auto weigh = [&](int i) __attribute__((always_inline)) {
                const float x = sc[i >> 4][i & 15], p = __builtin_amdgcn_exp2f(E4M3 ? x - m_use : fmaf(x, A.scale, -m_use));
                ps += p;
                w[i & 1] = E4M3 ? p * vs[(i >> 2) & 3][i & 3] : p;
                if (i & 1) pf[i >> 3][(i & 7) >> 1] = H::pack(w[0], w[1]);
                if (E4M3 && (i & 3) == 3 && i < 16) vs[i >> 2] = *(const f32x4 *)(now.vs + 32 + (i >> 2) * 8 + 4 * half);
            };
            const short *vp = now.v + v_lane;
            auto frag = [&](int n) __attribute__((always_inline)) { return *(const i32x4 *)(vp + (n / DT) * 16 * D + (n % DT) * 512); };
#pragma unroll
            for (int i = 0; i < 16; ++i) weigh(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) ring[n] = frag(n);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < 4 * DT; ++n) {
                o[n % DT] = H::mfma32(ring[n % AHEAD], pf[n / DT], o[n % DT]);
                __builtin_amdgcn_sched_barrier(0);
                if (n + AHEAD < 4 * DT) ring[n % AHEAD] = frag(n + AHEAD);
                if (n < 2 * DT) {                // beside the first half's outputs: the second half's weights
                    constexpr int PER = 8 / DT;
#pragma unroll
                    for (int i = 16 + n * PER; i < 16 + (n + 1) * PER; ++i) weigh(i);
                } else if ((n - 2 * DT) % (2 * DT / CH) == 0) put_away((n - 2 * DT) / (2 * DT / CH), stage[turn ^ 1]);      // beside the second's: the next tile
                __builtin_amdgcn_sched_barrier(0);
            }
            l += ps;                             // (of the lane's half of the keys)
            put_scales(stage[turn ^ 1]);
            if (v0 + 8 < it.count) {
                fetch(v0 + 8, page);
                page = page_of(P, s, my_block(v0 + 12));
            }
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
            v0 += 4;
            turn ^= 1;
            if (v0 >= it.count) break;
            mx = scores();
            grown = __builtin_amdgcn_ballot_w64(mx > m + 8.f) != 0;
        } while (!grown);
        if (!grown) break;
    }
    l = half_sum(l);
    if (it.slot < 0) {
        // through the LDS, so that rows leave in whole cache lines
        constexpr int ROW = D + 8, PIECES = D / 8;
        static_assert(4 * 32 * ROW * 2 <= (int)sizeof(stage), "rows fit");
        short *mine = (short *)stage + wave * 32 * ROW;
        const float inv = 1.f / l;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *(i32x2 *)(mine + col * ROW + 32 * t + 2 * i + 4 * half) =
                    (i32x2){H::pack(o[t][i] * inv, o[t][i + 1] * inv), H::pack(o[t][i + 2] * inv, o[t][i + 3] * inv)};
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = lane; p < 32 * PIECES; p += 64) {
            const int pr = it.row0 + wave * 32 + p / PIECES, c = (p % PIECES) * 8;
            if (pr < n_rows)
                *(i32x4 *)(A.out + (int64_t)(s.tok0 + pr / P.group) * A.ld_out + (int64_t)(head * P.group + pr % P.group) * D + c) =
                    *(const i32x4 *)(mine + (p / PIECES) * ROW + c);
        }
    } else {
        // as it lies in the registers: [wave][32 features][4][lane][4], then the rows' maxima and sums
        float *to = A.part + ((size_t)it.slot * P.kv + head) * (SPD_LARGE_ROWS * (D + 2));
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4 *)(to + ((wave * DT + t) * 4 + q) * 256 + lane * 4) = (f32x4){o[t][4 * q], o[t][4 * q + 1], o[t][4 * q + 2], o[t][4 * q + 3]};
        if (half == 0) {
            to[SPD_LARGE_ROWS * D + wave * 32 + col] = m;
            to[SPD_LARGE_ROWS * D + SPD_LARGE_ROWS + wave * 32 + col] = l;
        }
    }
}

// Joins the partial results of a chunk's rows whose blocks were cut into several items, in the order of the items: a wave per 32 rows
// (a wave's rows in the kernel that wrote them), KV head and 32 features.  Lane = 32 half + row, as they were written.
constexpr int MERGE_ROW = 32 + 8;                // 16-bit values of a row in the LDS
template <int D, bool F16>
__device__ __forceinline__ void attend_merge(const Pages &P, const float *part, unsigned short *out, int64_t ld_out, int item, int rows_of, int t, short *rows) {
    constexpr int DT = D / 32, CAP = SPD_LARGE_ROWS, NB = 8, ROW = MERGE_ROW;      // NB: parts asked for at a time
    const int head = item % P.kv;
    const spd_plan_merge j = ((const spd_plan_merge *)(P.plan + P.list))[item / P.kv];
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int r0 = rows_of * 32;
    if ((P.on_device && item / P.kv >= header_of(P).n_merge) || r0 >= j.rows) return;      // (the whole wave)
    const spd_plan_seq &s = j.s;
    const size_t step = (size_t)P.kv * CAP * (D + 2);
    const float *p = part + ((size_t)j.slot0 * P.kv + head) * (CAP * (D + 2));
    const float *po = p + (size_t)(rows_of * DT + t) * 1024 + lane * 4, *pm = p + CAP * D + r0 + col;
    float mm = -__builtin_inff(), l = 0.f;
    f32x4 acc[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q] = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < j.parts; i0 += NB) {
        float m[NB], sum[NB];
        f32x4 x[NB][4];
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            const size_t at = (size_t)(i0 + u < j.parts ? i0 + u : j.parts - 1) * step;
            m[u] = pm[at];
            sum[u] = pm[at + CAP];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[u][q] = *(const f32x4 *)(po + at + q * 256);
        }
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            if (i0 + u >= j.parts) break;
            const float m_new = fmaxf(mm, m[u]), m_use = m_new == -__builtin_inff() ? 0.f : m_new;
            const float fa = __builtin_amdgcn_exp2f(mm - m_use), fb = __builtin_amdgcn_exp2f(m[u] - m_use);
            mm = m_new;
            l = l * fa + sum[u] * fb;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[q][e] = acc[q][e] * fa + x[u][q][e] * fb;
        }
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *(i32x2 *)(rows + col * ROW + 8 * q + 4 * half) =
            (i32x2){Half<F16>::pack(acc[q][0] * inv, acc[q][1] * inv), Half<F16>::pack(acc[q][2] * inv, acc[q][3] * inv)};
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = lane; i < 32 * 4; i += 64) {
        const int r = r0 + i / 4, c = (i % 4) * 8, row = j.row0 + r;
        if (r < j.rows)
            *(i32x4 *)(out + (int64_t)(s.tok0 + row / P.group) * ld_out + (int64_t)(head * P.group + row % P.group) * D + 32 * t + c) =
                *(const i32x4 *)(rows + (i / 4) * ROW + c);
    }
}
template <int D, bool F16>
__global__ void __launch_bounds__(64) k_attend_merge(Pages P, const float *part, unsigned short *out, int64_t ld_out) {
    __shared__ __attribute__((aligned(16))) short rows[32 * MERGE_ROW];
    attend_merge<D, F16>(P, part, out, ld_out, blockIdx.x, blockIdx.y, blockIdx.z, rows);
}

// Few rows, and the joins of many, in one launch where a step has both (or may have: a plan made on the device launches what there could be): the first `small`
// workgroups and those behind them, eight joins each.  Three chunks of 333 tokens planned on the device 24.9 -> 23.3 us.
template <int D, int C, bool F16>
__global__ void __launch_bounds__(512, C == SPD_E2M1 ? 4 : 1) k_attend_small_merge(AttendArgs A, int small, int merge_list, int merges, int rows_of, const float *part) {
    constexpr int DT = D / 32;
    __shared__ __attribute__((aligned(16))) SmallOutputs<D> so;
    __shared__ SmallRows sm, sl;
    __shared__ int ended;
    static_assert(8 * 32 * MERGE_ROW * 2 <= (int)sizeof(so), "rows of eight joins fit");
    if ((int)blockIdx.x < small) return attend_small<D, C, F16>(A, blockIdx.x, so, sm, sl, ended);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), unit = (blockIdx.x - small) * 8 + wave;
    if (unit >= merges * rows_of * DT) return;
    Pages P = A.P;
    P.list = merge_list;
    attend_merge<D, F16>(P, part, A.out, A.ld_out, unit / DT / rows_of, unit / DT % rows_of, unit % DT, (short *)so + wave * 32 * MERGE_ROW);
}

// ------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------
Pages pages_args(const spd_pages *p, const spd_plan_header &h, const void *plan_dev, const void *pool, int list) {
    Pages P;
    P.plan = (const char *)plan_dev;
    P.pool = (char *)pool;
    P.page_bytes = p->page_bytes;
    P.head_bytes = p->head_bytes;
    P.seqs = h.seqs;
    P.table = h.table;
    P.list = list;
    P.shift = p->shift;
    P.page_size = p->cfg.page_size;
    P.kv = p->cfg.n_kv_heads;
    P.group = p->group;
    P.on_device = h.on_device;
    return P;
}

// f(D, what the pages hold, F16) for the handle's kind
template <class F>
hipError_t by_kind(const spd_pages *p, F f) {
    auto type = [&](auto d, auto c) { return p->cfg.dtype == SPD_F16 ? f(d, c, std::true_type()) : f(d, c, std::false_type()); };
    auto codes = [&](auto d) {
        switch (p->cfg.cache_dtype) {
            case SPD_E4M3: return type(d, std::integral_constant<int, SPD_E4M3>());
            case SPD_E2M1: return type(d, std::integral_constant<int, SPD_E2M1>());
            default: return type(d, std::integral_constant<int, HALVES>());
        }
    };
    return p->cfg.head_dim == 64 ? codes(std::integral_constant<int, 64>()) : codes(std::integral_constant<int, 128>());
}

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// a plan of this handle
int read_plan(const spd_pages *pages, const void *plan_host, const void *plan_dev, spd_plan_header *h) {
    if (!pages || !plan_host || !plan_dev || !aligned(plan_dev, 16)) return SPD_EINVAL;
    std::memcpy(h, plan_host, sizeof(*h));
    if (h->magic != SPD_PLAN_MAGIC || std::memcmp(&h->cfg, &pages->cfg, sizeof(h->cfg))) return SPD_EINVAL;
    return SPD_OK;
}

}  // namespace

extern "C" {

int spd_pages_write(const spd_pages *pages, const void *plan_host, const void *plan_dev, int32_t in_dtype, const void *qkv,
                    int64_t ld, const float *rope, void *pool, void *q_out, int64_t ld_q, void *stream) {
    spd_plan_header h;
    const int rc = read_plan(pages, plan_host, plan_dev, &h);
    if (rc != SPD_OK) return rc;
    const spd_pages_config &c = pages->cfg;
    if (in_dtype != SPD_F32 && in_dtype != c.dtype) return SPD_EINVAL;
    if (!h.n_write) return SPD_OK;
    const int es = in_dtype == SPD_F32 ? 4 : 2;
    if (!qkv || !pool || !aligned(qkv, 16) || !aligned(pool, 256) || (q_out && !rope) || !aligned(rope, 16)) return SPD_EINVAL;
    if (ld < (int64_t)(c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim || ld * es % 16) return SPD_EINVAL;
    if (q_out && (!aligned(q_out, 16) || ld_q < (int64_t)c.n_q_heads * c.head_dim || ld_q % 8)) return SPD_EINVAL;
    // queries turn in place, or where nobody reads
    if (q_out == qkv ? in_dtype == SPD_F32 || ld_q != ld
                     : spd_share_memory({qkv, h.tokens, (int64_t)(c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim * es, ld * es},
                                        {q_out, h.tokens, (int64_t)c.n_q_heads * c.head_dim * 2, ld_q * 2}))
        return SPD_EINVAL;
    (void)hipGetLastError();
    WriteArgs A;
    A.P = pages_args(pages, h, plan_dev, pool, h.write);
    A.qkv = (const char *)qkv;
    A.rope = (const float2 *)rope;
    A.q_out = (char *)q_out;
    A.ld = ld;
    A.ld_q = ld_q;
    A.q_heads = c.n_q_heads;
    // query heads: about a thousand workgroups, so that one has several heads and its angles serve them all
    const int units = 256 / c.head_dim, q_units = (c.n_q_heads + units - 1) / units;
    A.kv_groups = (c.n_kv_heads + units / 2 - 1) / (units / 2);
    A.q_groups = q_out ? std::min(q_units, std::max(1, 2048 / h.n_write)) : 0;
    const dim3 grid(h.n_write, A.kv_groups + A.q_groups);
    SPD_HIP(by_kind(pages, [&](auto d, auto e, auto f) {
        constexpr int D = decltype(d)::value;
        constexpr int E = decltype(e)::value;
        constexpr bool F = decltype(f)::value;
        if (in_dtype == SPD_F32) hipLaunchKernelGGL((k_pages_write<float, D, E, F>), grid, dim3(256), 0, (hipStream_t)stream, A);
        else hipLaunchKernelGGL((k_pages_write<std::conditional_t<F, _Float16, __bf16>, D, E, F>), grid, dim3(256), 0, (hipStream_t)stream, A);
        return hipGetLastError();
    }));
    return SPD_OK;
}

int spd_pages_read(const spd_pages *pages, const void *plan_host, const void *plan_dev, const void *pool, int32_t out_dtype,
                   void *k_out, void *v_out, void *stream) {
    spd_plan_header h;
    const int rc = read_plan(pages, plan_host, plan_dev, &h);
    if (rc != SPD_OK) return rc;
    const spd_pages_config &c = pages->cfg;
    if (out_dtype != SPD_F32 && out_dtype != c.dtype) return SPD_EINVAL;
    if (h.on_device) return SPD_EUNSUPPORTED;
    if (!h.held) return SPD_OK;
    if (!pool || !k_out || !v_out || !aligned(pool, 256) || !aligned(k_out, 16) || !aligned(v_out, 16)) return SPD_EINVAL;
    (void)hipGetLastError();
    const Pages P = pages_args(pages, h, plan_dev, pool, 0);
    const dim3 grid((h.max_end + 63) / 64 * c.n_kv_heads, h.batch);
    SPD_HIP(by_kind(pages, [&](auto d, auto e, auto f) {
        constexpr int D = decltype(d)::value;
        constexpr int E = decltype(e)::value;
        constexpr bool F = decltype(f)::value;
        typedef std::conditional_t<F, _Float16, __bf16> H;
        if (out_dtype == SPD_F32) hipLaunchKernelGGL((k_pages_read<float, D, E, F>), grid, dim3(256), 0, (hipStream_t)stream, P, (float *)k_out, (float *)v_out);
        else hipLaunchKernelGGL((k_pages_read<H, D, E, F>), grid, dim3(256), 0, (hipStream_t)stream, P, (H *)k_out, (H *)v_out);
        return hipGetLastError();
    }));
    return SPD_OK;
}

int spd_pages_attention(const spd_pages *pages, const void *plan_host, const void *plan_dev, const void *q, int64_t ld_q,
                        const void *pool, void *out, int64_t ld_out, void *workspace, void *stream) {
    spd_plan_header h;
    const int rc = read_plan(pages, plan_host, plan_dev, &h);
    if (rc != SPD_OK) return rc;
    const spd_pages_config &c = pages->cfg;
    const int64_t width = (int64_t)c.n_q_heads * c.head_dim;
    if (!h.tokens) return SPD_OK;
    if (!q || !pool || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(pool, 256)) return SPD_EINVAL;
    if (ld_q < width || ld_out < width || ld_q % 8 || ld_out % 8) return SPD_EINVAL;
    if (h.workspace && (!workspace || !aligned(workspace, 256))) return SPD_EINVAL;
    if (spd_share_memory({q, h.tokens, width * 2, ld_q * 2}, {out, h.tokens, width * 2, ld_out * 2})) return SPD_EINVAL;
    (void)hipGetLastError();
    AttendArgs A;
    A.q = (const unsigned short *)q;
    A.out = (unsigned short *)out;
    A.ld_q = ld_q;
    A.ld_out = ld_out;
    A.window = h.window;
    A.sinks = h.sinks;
    A.counters = nullptr;
    A.scale = (float)(1.4426950408889634 / std::sqrt((double)c.head_dim));
    float *small = workspace ? (float *)((char *)workspace + h.part_small) : nullptr,
          *large = workspace ? (float *)((char *)workspace + h.part_large) : nullptr;
    hipStream_t s = (hipStream_t)stream;
    SPD_HIP(by_kind(pages, [&](auto d, auto e, auto f) {
        constexpr int D = decltype(d)::value;
        constexpr int E = decltype(e)::value;
        constexpr bool F = decltype(f)::value;
        if (h.n_large) {
            A.P = pages_args(pages, h, plan_dev, pool, h.large);
            A.part = large;
            hipLaunchKernelGGL((k_attend_large<D, E, F>), dim3(h.n_large * c.n_kv_heads), dim3(256), 0, s, A);
            SPD_TRY(hipGetLastError());
        }
        const int rows_of = (h.merge_rows + 31) / 32, merges = h.n_merge * c.n_kv_heads;
        if (h.n_small) {
            A.P = pages_args(pages, h, plan_dev, pool, h.small);
            A.part = small;
            A.counters = (int *)workspace;
            const int n = h.n_small * c.n_kv_heads;
            if (!merges) hipLaunchKernelGGL((k_attend_small<D, E, F>), dim3(n), dim3(64 * SPD_SMALL_WAVES), 0, s, A);
            else hipLaunchKernelGGL((k_attend_small_merge<D, E, F>), dim3(n + (merges * rows_of * (D / 32) + 7) / 8), dim3(64 * SPD_SMALL_WAVES), 0, s, A, n,
                                    h.merge, merges, rows_of, (const float *)large);
            SPD_TRY(hipGetLastError());
        } else if (merges) {
            const Pages P = pages_args(pages, h, plan_dev, pool, h.merge);
            hipLaunchKernelGGL((k_attend_merge<D, F>), dim3(merges, rows_of, D / 32), dim3(64), 0, s, P,
                               (const float *)large, (unsigned short *)out, ld_out);
            SPD_TRY(hipGetLastError());
        }
        return hipSuccess;
    }));
    return SPD_OK;
}

}  // extern "C"
