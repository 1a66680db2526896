// Paged KV cache: quantised writes, reading back, and attention of chunks of new tokens over the pages, for gfx950.
//
// Orientation as everywhere in this library: keys (or values) are the first MFMA operand, queries (or probabilities) the second, so
// that scores come out transposed, S^T[key][row], four consecutive keys per lane, which is what the second contraction
// O^T = V^T P^T takes.  A "row" is a (token, query head of the KV group) pair, row = token * group + head.
//
// A key's scale multiplies its scores in fp32; a value's scale multiplies its probability before that is rounded for the second
// contraction.  e4m3 codes are exact in bf16 and fp16, so that dequantising rounds nothing.  Hidden keys are taken out by selection after
// the scale has been multiplied, and codes in pages are always finite: a NaN scale of a hidden key reaches nothing.
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
    // eight e4m3 codes
    static __device__ __forceinline__ i32x4 widen(int a, int b) {
        return (i32x4){from_e4m3<false>(a), from_e4m3<true>(a), from_e4m3<false>(b), from_e4m3<true>(b)};
    }
};

__device__ __forceinline__ float quad_sum(float x) {      // over lanes l, l^16, l^32, l^48
    x += __shfl_xor(x, 16, 64);
    return x + __shfl_xor(x, 32, 64);
}
__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, 64));
    return fmaxf(x, __shfl_xor(x, 32, 64));
}

// what every kernel over pages is told
struct Pages {
    const char *plan;
    char *pool;
    size_t page_bytes, head_bytes;
    int seqs, table, list;      // offsets into the plan
    int shift, page_size, kv, group;
};
// where a sequence's block of 16 positions lies, for one head: its page's share of the head, and the block in the page
struct Block {
    char *head;
    int in_page;
};
__device__ __forceinline__ Block block_at(const Pages &P, const spd_plan_seq &s, int head, int block) {
    const int page = ((const int *)(P.plan + P.table))[s.table + (block >> P.shift)];
    return Block{P.pool + (size_t)page * P.page_bytes + (size_t)head * P.head_bytes, block & ((1 << P.shift) - 1)};
}

// ------------------------------------------------------------------------------------------
// Writing.  One workgroup per 16-position block and KV head, or query head: sixteen threads per token, each with the same features of
// both rotary halves.
// ------------------------------------------------------------------------------------------
struct WriteArgs {
    Pages P;
    const char *qkv;
    const float2 *rope;
    char *q_out;
    int64_t ld, ld_q;           // in elements
    int q_heads;
};

template <class In, int N>      // N elements -> fp32
__device__ __forceinline__ void load_row(const char *p, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)((const In *)p)[i];
}

// largest magnitude over the sixteen threads of a token; NaN if any of them holds a value that is not finite
template <int N>
__device__ __forceinline__ float row_amax(const float (&a)[N], const float (&b)[N]) {
    float m = 0.f;
    bool fine = true;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        m = fmaxf(m, fmaxf(fabsf(a[i]), fabsf(b[i])));
        fine = fine && fabsf(a[i]) <= 3.402823466e38f && fabsf(b[i]) <= 3.402823466e38f;
    }
    if (!fine) m = __builtin_inff();
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    return m == __builtin_inff() ? __builtin_nanf("") : m;
}

template <class In, int D, bool E4M3, bool F16>
__global__ void __launch_bounds__(256) k_pages_write(WriteArgs A) {
    constexpr int N = D / 32, W = E4M3 ? 1 : 2, E = 16 / W;
    const Pages &P = A.P;
    const spd_plan_block it = ((const spd_plan_block *)(P.plan + P.list))[blockIdx.x];
    const spd_plan_seq s = ((const spd_plan_seq *)(P.plan + P.seqs))[it.seq];
    const int r = threadIdx.x >> 4, u = threadIdx.x & 15;
    const int pos = it.block * 16 + r, lo = it.block * 16 > s.pos ? 0 : s.pos - it.block * 16,
              hi = s.end - it.block * 16 < 16 ? s.end - it.block * 16 : 16;      // rows lo .. hi - 1 of the block are new
    const bool mine = r >= lo && r < hi;
    const int64_t token = s.tok0 + (pos - s.pos);
    const int y = blockIdx.y;
    const int f0 = u * N;
    float c[N], sn[N];
    if (A.rope) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 t = mine ? A.rope[(size_t)pos * (D / 2) + f0 + i] : make_float2(1.f, 0.f);
            c[i] = t.x;
            sn[i] = t.y;
        }
    }
    auto fetch = [&](int head, float(&a)[N], float(&b)[N]) {
        if (mine) {
            const char *p = A.qkv + (token * A.ld + (int64_t)head * D + f0) * sizeof(In);
            load_row<In, N>(p, a);
            load_row<In, N>(p + D / 2 * sizeof(In), b);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = b[i] = 0.f;
        }
    };
    auto rotate = [&](float(&a)[N], float(&b)[N]) {
        if (A.rope) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = a[i], z = b[i];
                a[i] = x * c[i] - z * sn[i];
                b[i] = z * c[i] + x * sn[i];
            }
        }
    };
    if (y >= P.kv) {            // a query head
        float a[N], b[N];
        fetch(y - P.kv, a, b);
        rotate(a, b);
        if (mine) {
            int *o = (int *)(A.q_out + (token * A.ld_q + (int64_t)(y - P.kv) * D + f0) * 2);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                o[i] = Half<F16>::pack(a[2 * i], a[2 * i + 1]);
                o[D / 4 + i] = Half<F16>::pack(b[2 * i], b[2 * i + 1]);
            }
        }
        return;
    }
    // codes of the block's keys and values, rows = positions
    __shared__ __attribute__((aligned(16))) char codes[2][16 * D * W];
    const Block B = block_at(P, s, y, it.block);
    char *keys = B.head + (size_t)B.in_page * 16 * D * W, *values = keys + (size_t)P.page_size * D * W;
    float *scales = (float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        float a[N], b[N];
        fetch(A.q_heads + y + kind * P.kv, a, b);
        if (kind == 0) rotate(a, b);
        float amax;
        if constexpr (!E4M3) {       // what the 16-bit type makes of it decides whether the row is finite
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const int pa = Half<F16>::pack(a[i], a[i + 1]), pb = Half<F16>::pack(b[i], b[i + 1]);
                a[i] = Half<F16>::low(pa);
                a[i + 1] = Half<F16>::high(pa);
                b[i] = Half<F16>::low(pb);
                b[i + 1] = Half<F16>::high(pb);
            }
        }
        amax = row_amax<N>(a, b);
        const bool fine = amax == amax;
        float scale = 1.f;
        if constexpr (E4M3) {
            amax = fmaxf(amax, 0x1p-90f);      // (a NaN gives the other operand)
            scale = amax / 448.f;
            const float up = 448.f / amax;
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const int pa = __builtin_amdgcn_cvt_pk_fp8_f32(a[i] * up, a[i + 1] * up, 0, false);
                const int pb = __builtin_amdgcn_cvt_pk_fp8_f32(b[i] * up, b[i + 1] * up, 0, false);
                *(short *)(codes[kind] + r * D + f0 + i) = (short)(fine ? pa : 0);
                *(short *)(codes[kind] + r * D + D / 2 + f0 + i) = (short)(fine ? pb : 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                *(int *)(codes[kind] + (r * D + f0 + i) * 2) = fine ? Half<F16>::pack(a[i], a[i + 1]) : 0;
                *(int *)(codes[kind] + (r * D + D / 2 + f0 + i) * 2) = fine ? Half<F16>::pack(b[i], b[i + 1]) : 0;
            }
        }
        if (mine && u == 0) scales[kind * P.page_size + r] = fine ? scale : __builtin_nanf("");
    }
    __syncthreads();
    // keys: a 16-byte piece belongs to one position
    for (int i = threadIdx.x; i < D * W; i += 256) {
        const int pr = i & 15, g = (i >> 4) & 3, ch = i >> 6;
        if (pr >= lo && pr < hi) *(i32x4 *)(keys + i * 16) = *(const i32x4 *)(codes[0] + (pr * D + ch * 4 * E + g * E) * W);
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
                    if constexpr (E4M3) piece.b[t * 4 + k] = codes[1][at];
                    else piece.h[t * 4 + k] = ((const unsigned short *)codes[1])[at];
                }
            *(i32x4 *)(values + i * 16) = piece.v;
        }
    } else {
        for (int i = threadIdx.x; i < (hi - lo) * D; i += 256) {
            const int pr = lo + i / D, f = i % D, to = spd_page_value_off(pr, f, E);
            if constexpr (E4M3) values[to] = codes[1][pr * D + f];
            else ((unsigned short *)values)[to] = ((const unsigned short *)codes[1])[pr * D + f];
        }
    }
}

// ------------------------------------------------------------------------------------------
// Reading back.  One workgroup per 16-position block and KV head.
// ------------------------------------------------------------------------------------------
template <class Out, int D, bool E4M3, bool F16>
__global__ void __launch_bounds__(256) k_pages_read(Pages P, Out *k_out, Out *v_out) {
    constexpr int N = D / 16, W = E4M3 ? 1 : 2, E = 16 / W;
    const spd_plan_seq s = ((const spd_plan_seq *)(P.plan + P.seqs))[blockIdx.y];
    const int block = blockIdx.x, head = blockIdx.z;
    const int r = threadIdx.x >> 4, f0 = (threadIdx.x & 15) * N;
    if (block * 16 + r >= s.end) return;
    const Block B = block_at(P, s, head, block);
    const char *keys = B.head + (size_t)B.in_page * 16 * D * W, *values = keys + (size_t)P.page_size * D * W;
    const float *scales = (const float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16 + r;
    const float ks = scales[0], vs = scales[P.page_size];
    const int64_t to = ((s.held0 + block * 16 + r) * P.kv + head) * D + f0;
    auto value = [&](const char *p, int at) -> float {
        if constexpr (E4M3) return Half<false>::low(Half<false>::template from_e4m3<false>((int)(unsigned char)p[at]));
        else return Half<F16>::low(((const unsigned short *)p)[at]);
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        k_out[to + i] = (Out)(value(keys, spd_page_key_off(r, f0 + i, E)) * ks);
        v_out[to + i] = (Out)(value(values, spd_page_value_off(r, f0 + i, E)) * vs);
    }
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
    int window, sinks;
    float scale;                // log2(e) / sqrt(head_dim): softmax in powers of two
};

// is `key` visible to a query at position `at`?
__device__ __forceinline__ bool visible(int key, int at, int window, int sinks) {
    return key <= at && (window == 0 || key > at - window || key < sinks);
}
__device__ __forceinline__ int list_block(const spd_plan_item &it, int v) { return v < it.sink_blocks ? v : it.block0 + (v - it.sink_blocks); }

// operands of one 16-position block, as loaded
template <int D, bool E4M3>
struct BlockLoad {
    static constexpr int CH = E4M3 ? D / 64 : D / 32;      // 16-byte chunks per lane, keys and values each
    i32x4 k[CH], v[CH];
    f32x4 ks, vs;                                           // scales of keys 4 g .. 4 g + 3
    __device__ __forceinline__ void load(const Pages &P, const spd_plan_seq &s, int head, int block, int lane) {
        constexpr int W = E4M3 ? 1 : 2;
        const Block B = block_at(P, s, head, block);
        const char *keys = B.head + (size_t)B.in_page * 16 * D * W, *values = keys + (size_t)P.page_size * D * W;
        const float *scales = (const float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16 + 4 * (lane >> 4);
#pragma unroll
        for (int c = 0; c < CH; ++c) k[c] = *(const i32x4 *)(keys + c * 1024 + lane * 16);
        ks = *(const f32x4 *)scales;
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = *(const i32x4 *)(values + c * 1024 + lane * 16);
        vs = *(const f32x4 *)(scales + P.page_size);
    }
};

// Few rows (a decode step, a short draft): one workgroup per item and KV head, its four waves take pairs of blocks in turn and merge
// their states in the LDS.  Lane = 16 g + row.
template <int D, bool E4M3, bool F16>
__global__ void __launch_bounds__(256) k_attend_small(AttendArgs A) {
    constexpr int DT = D / 16, NF = D / 32;
    typedef Half<F16> QK;                        // queries and keys
    typedef Half<F16 && !E4M3> PV;               // probabilities (times a scale that may be tiny: bf16 beside e4m3) and values
    const Pages &P = A.P;
    const int head = blockIdx.x % P.kv;
    const spd_plan_item it = ((const spd_plan_item *)(P.plan + P.list))[blockIdx.x / P.kv];
    const spd_plan_seq s = ((const spd_plan_seq *)(P.plan + P.seqs))[it.seq];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int rows = s.q_len * P.group;          // at most 16
    const int token = row / P.group;
    const int at = s.pos + token;
    i32x4 qf[NF];
    {
        const unsigned short *qp = A.q + (int64_t)(s.tok0 + token) * A.ld_q + (int64_t)(head * P.group + row % P.group) * D;
#pragma unroll
        for (int i = 0; i < NF; ++i) {           // the features that lane (g, .) of a key holds
            const int f = E4M3 ? 64 * (i >> 1) + 16 * g + 8 * (i & 1) : 32 * i + 8 * g;
            qf[i] = row < rows ? *(const i32x4 *)(qp + f) : (i32x4){0, 0, 0, 0};
        }
    }
    f32x4 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;
    for (int p = wave; 2 * p < it.count; p += 4) {
        const bool two = 2 * p + 1 < it.count;
        const int b0 = list_block(it, it.first + 2 * p), b1 = two ? list_block(it, it.first + 2 * p + 1) : b0;
        BlockLoad<D, E4M3> x0, x1;
        x0.load(P, s, head, b0, lane);
        x1.load(P, s, head, b1, lane);
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            i32x4 k0, k1;
            if constexpr (E4M3) {
                k0 = QK::widen(x0.k[i >> 1][2 * (i & 1)], x0.k[i >> 1][2 * (i & 1) + 1]);
                k1 = QK::widen(x1.k[i >> 1][2 * (i & 1)], x1.k[i >> 1][2 * (i & 1) + 1]);
            } else {
                k0 = x0.k[i];
                k1 = x1.k[i];
            }
            s0 = QK::mfma16(k0, qf[i], s0);
            s1 = QK::mfma16(k1, qf[i], s1);
        }
        float mx = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s0[i] = visible(b0 * 16 + 4 * g + i, at, A.window, A.sinks) ? s0[i] * (x0.ks[i] * A.scale) : -__builtin_inff();
            s1[i] = two && visible(b1 * 16 + 4 * g + i, at, A.window, A.sinks) ? s1[i] * (x1.ks[i] * A.scale) : -__builtin_inff();
            mx = fmaxf(mx, fmaxf(s0[i], s1[i]));
        }
        const float m_new = fmaxf(m, quad_max(mx)), m_use = m_new == -__builtin_inff() ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        float ps = 0.f;
        float w0[4], w1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(s0[i] - m_use), p1 = __builtin_amdgcn_exp2f(s1[i] - m_use);
            ps += p0 + p1;
            // (the scale of a hidden key's value may be NaN)
            w0[i] = s0[i] == -__builtin_inff() ? 0.f : p0 * x0.vs[i];
            w1[i] = s1[i] == -__builtin_inff() ? 0.f : p1 * x1.vs[i];
        }
        l = l * alpha + quad_sum(ps);
        m = m_new;
        const i32x4 pf = {PV::pack(w0[0], w0[1]), PV::pack(w0[2], w0[3]), PV::pack(w1[0], w1[1]), PV::pack(w1[2], w1[3])};
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            i32x4 vf;
            if constexpr (E4M3) vf = PV::widen(x0.v[t >> 2][t & 3], x1.v[t >> 2][t & 3]);
            else vf = (i32x4){x0.v[t >> 1][2 * (t & 1)], x0.v[t >> 1][2 * (t & 1) + 1], x1.v[t >> 1][2 * (t & 1)], x1.v[t >> 1][2 * (t & 1) + 1]};
            o[t] = PV::mfma16(vf, pf, o[t] * alpha);
        }
    }
    // merge the waves
    __shared__ float so[4][16][D + 4], sm[4][16], sl[4][16];
#pragma unroll
    for (int t = 0; t < DT; ++t) *(f32x4 *)&so[wave][row][t * 16 + 4 * g] = o[t];
    if (g == 0) {
        sm[wave][row] = m;
        sl[wave][row] = l;
    }
    __syncthreads();
    constexpr int N = D / 16;
    const int mr = threadIdx.x >> 4, f0 = (threadIdx.x & 15) * N;
    float mm = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sm[w][mr]);
    const float m_use = mm == -__builtin_inff() ? 0.f : mm;
    float ll = 0.f, acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm[w][mr] - m_use);
        ll += f * sl[w][mr];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] += f * so[w][mr][f0 + i];
    }
    if (mr >= rows) return;
    if (it.slot < 0) {
        int *to = (int *)(A.out + (int64_t)(s.tok0 + mr / P.group) * A.ld_out + (int64_t)(head * P.group + mr % P.group) * D + f0);
        const float inv = 1.f / ll;
#pragma unroll
        for (int i = 0; i < N; i += 2) to[i / 2] = QK::pack(acc[i] * inv, acc[i + 1] * inv);
    } else {
        float *to = A.part + ((size_t)it.slot * P.kv + head) * (SPD_SMALL_ROWS * (D + 2));
#pragma unroll
        for (int i = 0; i < N; ++i) to[mr * D + f0 + i] = acc[i];
        if (f0 == 0) {
            to[SPD_SMALL_ROWS * D + mr] = mm;
            to[SPD_SMALL_ROWS * D + SPD_SMALL_ROWS + mr] = ll;
        }
    }
}

// Many rows (a prompt's chunk): one workgroup per 128 rows and KV head; each wave has 32 of them, tiles of 64 keys go through the LDS in 16
// bits, dequantised once for the workgroup.  Lane = 32 half + row.
template <int D, bool E4M3, bool F16>
__global__ void __launch_bounds__(256, 2) k_attend_large(AttendArgs A) {
    constexpr int W = E4M3 ? 1 : 2, KS = D / 16, DT = D / 32, CH = E4M3 ? D / 64 : D / 32;
    typedef Half<F16> QK;
    typedef Half<F16 && !E4M3> PV;
    const Pages &P = A.P;
    const int head = blockIdx.x % P.kv;
    const spd_plan_item it = ((const spd_plan_item *)(P.plan + P.list))[blockIdx.x / P.kv];
    const spd_plan_seq s = ((const spd_plan_seq *)(P.plan + P.seqs))[it.seq];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int n_rows = s.q_len * P.group;
    const int row = it.row0 + wave * 32 + col;
    const bool live = row < n_rows;
    const int token = (live ? row : n_rows - 1) / P.group, qh = head * P.group + (live ? row : n_rows - 1) % P.group;
    const int at = s.pos + token;
    // keys: [block][feature / 8][position][8]; values: [block][feature / 16][half][feature % 16][8 positions of the half]
    __shared__ __attribute__((aligned(16))) short lk[64 * D], lv[64 * D];
    __shared__ __attribute__((aligned(16))) float lks[64], lvs[64];
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
    for (int v0 = 0; v0 < it.count; v0 += 4) {
        __syncthreads();
        {       // wave w brings the tile's block w
            const int v = v0 + wave < it.count ? v0 + wave : it.count - 1;
            const int r = lane & 15, g = lane >> 4;
            const Block B = block_at(P, s, head, list_block(it, it.first + v));
            const char *keys = B.head + (size_t)B.in_page * 16 * D * W, *values = keys + (size_t)P.page_size * D * W;
            const float *scales = (const float *)(B.head + (size_t)2 * P.page_size * D * W) + B.in_page * 16;
            i32x4 k[CH], x[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                k[c] = *(const i32x4 *)(keys + c * 1024 + lane * 16);
                x[c] = *(const i32x4 *)(values + c * 1024 + lane * 16);
            }
            if (lane < 32) (lane < 16 ? lks : lvs)[wave * 16 + r] = scales[lane < 16 ? r : P.page_size + r];
            short *kd = lk + wave * 16 * D, *vd = lv + wave * 16 * D;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if constexpr (E4M3) {
                    *(i32x4 *)(kd + ((8 * c + 2 * g) * 16 + r) * 8) = QK::widen(k[c][0], k[c][1]);
                    *(i32x4 *)(kd + ((8 * c + 2 * g + 1) * 16 + r) * 8) = QK::widen(k[c][2], k[c][3]);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        *(i32x2 *)(vd + (((4 * c + t) * 2 + (g & 1)) * 16 + r) * 8 + (g >> 1) * 4) =
                            (i32x2){PV::template from_e4m3<false>(x[c][t]), PV::template from_e4m3<true>(x[c][t])};
                } else {
                    *(i32x4 *)(kd + ((4 * c + g) * 16 + r) * 8) = k[c];
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        *(i32x2 *)(vd + (((2 * c + t) * 2 + (g & 1)) * 16 + r) * 8 + (g >> 1) * 4) = (i32x2){x[c][2 * t], x[c][2 * t + 1]};
                }
            }
        }
        __syncthreads();
        f32x16 sc[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[h][i] = 0.f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const i32x4 kf = *(const i32x4 *)(lk + (2 * h + (col >> 4)) * 16 * D + ((2 * i + half) * 16 + (col & 15)) * 8);
                sc[h] = QK::mfma32(kf, qf[i], sc[h]);
            }
        }
        // score i of half h: block 2 h + i / 8 of the tile, position 8 ((i / 4) % 2) + 4 half + i % 4 in it
        float mx = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const bool there = v0 + b < it.count;
            const int key0 = there ? list_block(it, it.first + v0 + b) * 16 : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 8 * (i >> 2) + 4 * half + (i & 3);
                const float x = sc[b >> 1][(b & 1) * 8 + i] * (lks[b * 16 + r] * A.scale);
                const float y = there && visible(key0 + r, at, A.window, A.sinks) ? x : -__builtin_inff();
                sc[b >> 1][(b & 1) * 8 + i] = y;
                mx = fmaxf(mx, y);
            }
        }
        const float m_new = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32, 64))), m_use = m_new == -__builtin_inff() ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        float ps = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = sc[b >> 1][(b & 1) * 8 + i], p = __builtin_amdgcn_exp2f(x - m_use);
                ps += p;
                w[i] = x == -__builtin_inff() ? 0.f : p * lvs[b * 16 + 8 * (i >> 2) + 4 * half + (i & 3)];
            }
            const i32x4 pf = {PV::pack(w[0], w[1]), PV::pack(w[2], w[3]), PV::pack(w[4], w[5]), PV::pack(w[6], w[7])};
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const i32x4 vf = *(const i32x4 *)(lv + b * 16 * D + (((2 * t + (col >> 4)) * 2 + half) * 16 + (col & 15)) * 8);
                o[t] = PV::mfma32(vf, pf, o[t]);
            }
        }
        l = l * alpha + ps + __shfl_xor(ps, 32, 64);
        m = m_new;
    }
    if (!live) return;
    if (it.slot < 0) {
        const float inv = 1.f / l;
        int *to = (int *)(A.out + (int64_t)(s.tok0 + token) * A.ld_out + (int64_t)qh * D);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *(i32x2 *)(to + (32 * t + 2 * i + 4 * half) / 2) =
                    (i32x2){QK::pack(o[t][i] * inv, o[t][i + 1] * inv), QK::pack(o[t][i + 2] * inv, o[t][i + 3] * inv)};
    } else {
        float *to = A.part + ((size_t)it.slot * P.kv + head) * (SPD_LARGE_ROWS * (D + 2));
        const int pr = wave * 32 + col;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *(f32x4 *)(to + pr * D + 32 * t + 2 * i + 4 * half) = (f32x4){o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
        if (half == 0) {
            to[SPD_LARGE_ROWS * D + pr] = m;
            to[SPD_LARGE_ROWS * D + SPD_LARGE_ROWS + pr] = l;
        }
    }
}

// Joins the partial results of rows whose blocks were cut into several items: a wave per row, in the order of the items.
template <int D, bool F16>
__global__ void __launch_bounds__(256) k_attend_merge(Pages P, const float *part_small, const float *part_large, unsigned short *out,
                                                      int64_t ld_out) {
    const int head = blockIdx.x % P.kv;
    const spd_plan_merge g = ((const spd_plan_merge *)(P.plan + P.list))[blockIdx.x / P.kv];
    const int r = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (r >= g.rows) return;
    const spd_plan_seq s = ((const spd_plan_seq *)(P.plan + P.seqs))[g.seq];
    const int cap = g.large ? SPD_LARGE_ROWS : SPD_SMALL_ROWS;
    const size_t step = (size_t)P.kv * cap * (D + 2);
    const float *p = (g.large ? part_large : part_small) + ((size_t)g.slot0 * P.kv + head) * (cap * (D + 2));
    float m = -__builtin_inff();
    for (int i = 0; i < g.parts; ++i) m = fmaxf(m, p[i * step + cap * D + r]);
    const float m_use = m == -__builtin_inff() ? 0.f : m;
    constexpr int N = D / 64;
    float l = 0.f, acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
    for (int i = 0; i < g.parts; ++i) {
        const float f = __builtin_amdgcn_exp2f(p[i * step + cap * D + r] - m_use);
        l += f * p[i * step + cap * D + cap + r];
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] += f * p[i * step + (size_t)r * D + lane * N + j];
    }
    const int row = g.row0 + r;
    unsigned short *to = out + (int64_t)(s.tok0 + row / P.group) * ld_out + (int64_t)(head * P.group + row % P.group) * D + lane * N;
    const float inv = 1.f / l;
    if constexpr (N == 2) *(int *)to = Half<F16>::pack(acc[0] * inv, acc[1] * inv);
    else *to = (unsigned short)Half<F16>::pack(acc[0] * inv, 0.f);
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
    return P;
}

// f(D, E4M3, F16) for the handle's kind
template <class F>
hipError_t by_kind(const spd_pages *p, F f) {
    typedef std::true_type T;
    typedef std::false_type N;
    typedef std::integral_constant<int, 64> D64;
    typedef std::integral_constant<int, 128> D128;
    const bool e = p->cfg.cache_dtype == SPD_E4M3, h = p->cfg.dtype == SPD_F16;
    if (p->cfg.head_dim == 64) return e ? (h ? f(D64(), T(), T()) : f(D64(), T(), N())) : (h ? f(D64(), N(), T()) : f(D64(), N(), N()));
    return e ? (h ? f(D128(), T(), T()) : f(D128(), T(), N())) : (h ? f(D128(), N(), T()) : f(D128(), N(), N()));
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
    const int es = in_dtype == SPD_F32 ? 4 : 2;
    if (!qkv || !pool || !aligned(qkv, 16) || !aligned(pool, 256) || (q_out && !rope)) return SPD_EINVAL;
    if (ld < (int64_t)(c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim || ld * es % 16) return SPD_EINVAL;
    if (q_out && (!aligned(q_out, 16) || ld_q < (int64_t)c.n_q_heads * c.head_dim || ld_q % 8)) return SPD_EINVAL;
    if (q_out == qkv && (in_dtype == SPD_F32 || ld_q != ld)) return SPD_EINVAL;
    if (!h.n_write) return SPD_OK;
    (void)hipGetLastError();
    WriteArgs A;
    A.P = pages_args(pages, h, plan_dev, pool, h.write);
    A.qkv = (const char *)qkv;
    A.rope = (const float2 *)rope;
    A.q_out = (char *)q_out;
    A.ld = ld;
    A.ld_q = ld_q;
    A.q_heads = c.n_q_heads;
    const dim3 grid(h.n_write, c.n_kv_heads + (q_out ? c.n_q_heads : 0));
    SPD_HIP(by_kind(pages, [&](auto d, auto e, auto f) {
        constexpr int D = decltype(d)::value;
        constexpr bool E = decltype(e)::value, F = decltype(f)::value;
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
    if (!pool || !k_out || !v_out || !aligned(pool, 256) || !aligned(k_out, 16) || !aligned(v_out, 16)) return SPD_EINVAL;
    if (!h.held) return SPD_OK;
    (void)hipGetLastError();
    const Pages P = pages_args(pages, h, plan_dev, pool, 0);
    const dim3 grid((h.max_end + 15) / 16, h.batch, c.n_kv_heads);
    SPD_HIP(by_kind(pages, [&](auto d, auto e, auto f) {
        constexpr int D = decltype(d)::value;
        constexpr bool E = decltype(e)::value, F = decltype(f)::value;
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
    if (!q || !pool || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(pool, 256)) return SPD_EINVAL;
    if (ld_q < width || ld_out < width || ld_q % 8 || ld_out % 8) return SPD_EINVAL;
    if (h.workspace && (!workspace || !aligned(workspace, 256))) return SPD_EINVAL;
    if (!h.tokens) return SPD_OK;
    const uintptr_t q0 = (uintptr_t)q, q1 = q0 + ((h.tokens - 1) * ld_q + width) * 2, o0 = (uintptr_t)out,
                    o1 = o0 + ((h.tokens - 1) * ld_out + width) * 2;
    if (q0 < o1 && o0 < q1) return SPD_EINVAL;
    (void)hipGetLastError();
    AttendArgs A;
    A.q = (const unsigned short *)q;
    A.out = (unsigned short *)out;
    A.ld_q = ld_q;
    A.ld_out = ld_out;
    A.window = h.window;
    A.sinks = h.sinks;
    A.scale = (float)(1.4426950408889634 / std::sqrt((double)c.head_dim));
    float *small = workspace ? (float *)((char *)workspace + h.part_small) : nullptr,
          *large = workspace ? (float *)((char *)workspace + h.part_large) : nullptr;
    hipStream_t s = (hipStream_t)stream;
    SPD_HIP(by_kind(pages, [&](auto d, auto e, auto f) {
        constexpr int D = decltype(d)::value;
        constexpr bool E = decltype(e)::value, F = decltype(f)::value;
        if (h.n_large) {
            A.P = pages_args(pages, h, plan_dev, pool, h.large);
            A.part = large;
            hipLaunchKernelGGL((k_attend_large<D, E, F>), dim3(h.n_large * c.n_kv_heads), dim3(256), 0, s, A);
            SPD_TRY(hipGetLastError());
        }
        if (h.n_small) {
            A.P = pages_args(pages, h, plan_dev, pool, h.small);
            A.part = small;
            hipLaunchKernelGGL((k_attend_small<D, E, F>), dim3(h.n_small * c.n_kv_heads), dim3(256), 0, s, A);
            SPD_TRY(hipGetLastError());
        }
        if (h.n_merge) {
            const Pages P = pages_args(pages, h, plan_dev, pool, h.merge);
            hipLaunchKernelGGL((k_attend_merge<D, F>), dim3(h.n_merge * c.n_kv_heads, (h.merge_rows + 3) / 4), dim3(256), 0, s, P,
                               (const float *)small, (const float *)large, (unsigned short *)out, ld_out);
            SPD_TRY(hipGetLastError());
        }
        return hipSuccess;
    }));
    return SPD_OK;
}

}  // extern "C"
