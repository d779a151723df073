// Tokens into and out of a K/V cache in 4 bits (contract: specdec.h, format: fp4.cuh).
//
// A thread takes the sixteen channels of a scale: 32 or 64 bytes in, 8 bytes of codes and one of scales out (read: the reverse).  Threads run along a head's tokens, so that a
// warp's codes and scales are whole stretches of a page.
#include <cuda_bf16.h>

#include <type_traits>

#include "fp4.cuh"
#include "op_error.cuh"

namespace sd {
namespace {

struct Fp4Io {
    char* codes; char* scales;                            // of the first layer of the call
    long long s_layer, s_side, s_page, s_head, c_layer, c_side, c_page, c_head;
    char* x[2];                                           // keys, values
    long long x_layer, x_seq, x_token, x_head;            // bytes
    const float* unit;                                    // [layer, side, head] of the call's layers, or null
    const int* table; const int* length; const int* held; const int* refs; const int* seqs; const int* some; int* status;      // some: append's counts, read's first tokens, or null
    int n_pages, n_seqs, max_pages, page_shift, heads, T;
};

// Page of a token's slot, or -1.  own: of a page that is the sequence's alone.
__device__ __forceinline__ int page_at(const Fp4Io& a, int s, int pos, bool own) {
    const int i = pos >> a.page_shift;
    if (pos < 0 || i >= min(max(a.held[s], 0), a.max_pages)) return -1;
    const int p = a.table[(long long)s * a.max_pages + i];
    return (unsigned)p < (unsigned)a.n_pages && (!own || a.refs[p] == 1) ? p : -1;
}

template <typename T> __device__ __forceinline__ void load16(const char* p, float* x) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 v = reinterpret_cast<const float4*>(p)[i];
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(p)[i];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (std::is_same<T, __half>::value) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(w + j));
                    x[8 * i + 2 * j] = f.x; x[8 * i + 2 * j + 1] = f.y;
                } else {
                    x[8 * i + 2 * j] = __uint_as_float(w[j] << 16); x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                }
            }
        }
    }
}
template <typename T> __device__ __forceinline__ void store16(char* p, const float* x) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (std::is_same<T, __half>::value) { const __half2 h = __floats2half2_rn(x[2 * j], x[2 * j + 1]); w[j] = *reinterpret_cast<const uint32_t*>(&h); }
            else { const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]); w[j] = *reinterpret_cast<const uint32_t*>(&h); }
        }
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// What one thread does: sequence, layer and side of its CTA; head, token, block of its own.
template <int D> struct Item { int i, s, layer, side, h, t, b; };
template <int D> __device__ __forceinline__ bool item_of(const Fp4Io& a, Item<D>& m) {
    constexpr int NB = D / FP4_BLOCK;
    const long long u = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    m.b = (int)(u % NB);
    const long long v = u / NB;
    m.t = (int)(v % a.T);
    m.h = (int)(v / a.T);
    m.i = blockIdx.y; m.layer = blockIdx.z >> 1; m.side = blockIdx.z & 1;
    m.s = a.seqs[m.i];
    return v < (long long)a.heads * a.T;
}

// Division by the scale: a 16-bit x has at most 11 significant bits and a halfway point between codes times a scale at most 7, so x / s lies on such a point or at least 2^-13 beside it (points
// from 0.25 on).  The product with 1 / s is off by less than 2^-20; rounded to a multiple of 2^-15 it lies on the point, or on the same side of it, as the quotient does.  That is a product and
// two sums in place of a division.  Other x are divided.
template <typename T, int D, bool UNIT>
__global__ void __launch_bounds__(256) k_fp4_append(Fp4Io a) {
    op_begin();
    Item<D> m;
    if (!item_of(a, m)) return;
    const bool known = (unsigned)m.s < (unsigned)a.n_seqs;
    if (a.some && m.t >= a.some[m.i]) return;
    const int pos = known ? a.length[m.s] + m.t : 0, p = known ? page_at(a, m.s, pos, true) : -1;
    if (p < 0) { if (m.b == 0 && m.h == 0) atomicOr(a.status, known ? SPECDEC_CACHE_UNRESERVED : SPECDEC_CACHE_BAD_INDEX); return; }
    float x[16];
    load16<T>(a.x[m.side] + m.layer * a.x_layer + m.i * a.x_seq + m.t * a.x_token + m.h * a.x_head + m.b * 16 * (int)sizeof(T), x);
    if (UNIT) {
        const float unit = a.unit[(m.layer * 2 + m.side) * a.heads + m.h];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __fdiv_rn(x[i], unit);
    }
    float top = 0.f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) { top = fmaxf(top, fabsf(x[i])); nan |= x[i] != x[i]; }
    const uint32_t scale = nan ? 0x7fu : fp4_scale_of(__fdiv_rn(top, 6.f));
    const uint32_t s2 = fp4_scales2(scale);
    const float s = __half2float(__low2half(*reinterpret_cast<const __half2*>(&s2)));
    if (scale == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
    } else if (UNIT || sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __fdiv_rn(x[i], s);
    } else {
        const float r = __fdiv_rn(1.f, s), grid = 384.f;  // (sums from 256 to 512 are multiples of 2^-15; beyond 6.4, where x is beyond 2688, the code is 6's all the same)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = copysignf(__fsub_rn(__fadd_rn(fabsf(x[i] * r), grid), grid), x[i]);
    }
    const int t = pos & ((1 << a.page_shift) - 1);
    const uint2 w = make_uint2(fp4_pack8(x), fp4_pack8(x + 8));
    *reinterpret_cast<uint2*>(a.codes + m.layer * a.s_layer + m.side * a.s_side + p * a.s_page + m.h * a.s_head + t * (D / 2) + m.b * 8) = w;
    *reinterpret_cast<unsigned char*>(a.scales + m.layer * a.c_layer + m.side * a.c_side + p * a.c_page + m.h * a.c_head + t * (D / 16) + m.b) = (unsigned char)scale;
}

template <typename T, int D, bool UNIT>
__global__ void __launch_bounds__(256) k_fp4_read(Fp4Io a) {
    op_begin();
    Item<D> m;
    if (!item_of(a, m)) return;
    const bool known = (unsigned)m.s < (unsigned)a.n_seqs;
    if (!known && m.b == 0 && m.h == 0) atomicOr(a.status, SPECDEC_CACHE_BAD_INDEX);
    const long long at = known ? (long long)(a.some ? a.some[m.i] : a.length[m.s]) + m.t : -1;
    const int pos = at > 0x7fffffff ? -1 : (int)at, p = known ? page_at(a, m.s, pos, false) : -1;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    if (p >= 0) {
        const int t = pos & ((1 << a.page_shift) - 1);
        const uint2 w = *reinterpret_cast<const uint2*>(a.codes + m.layer * a.s_layer + m.side * a.s_side + p * a.s_page + m.h * a.s_head + t * (D / 2) + m.b * 8);
        const uint32_t scale = *reinterpret_cast<const unsigned char*>(a.scales + m.layer * a.c_layer + m.side * a.c_side + p * a.c_page + m.h * a.c_head + t * (D / 16) + m.b);
        const uint32_t s2 = fp4_scales2(scale | scale << 8);
        uint32_t o[8];
        fp4_unpack8(w.x, o); fp4_unpack8(w.y, o + 4);
        const float unit = UNIT ? a.unit[(m.layer * 2 + m.side) * a.heads + m.h] : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t v = h2_mul(o[i], s2);          // exact
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
            x[2 * i] = UNIT ? f.x * unit : f.x; x[2 * i + 1] = UNIT ? f.y * unit : f.y;
        }
    }
    store16<T>(a.x[m.side] + m.layer * a.x_layer + m.i * a.x_seq + m.t * a.x_token + m.h * a.x_head + m.b * 16 * (int)sizeof(T), x);
}

template <bool READ, typename T, int D> auto kernel(bool unit) {
    if constexpr (READ) return unit ? k_fp4_read<T, D, true> : k_fp4_read<T, D, false>;
    else return unit ? k_fp4_append<T, D, true> : k_fp4_append<T, D, false>;
}
template <bool READ, typename T> auto kernel(int dim, bool unit) { return dim == 64 ? kernel<READ, T, 64>(unit) : kernel<READ, T, 128>(unit); }

template <bool READ>
int move(const char* who, const specdec_packed_cache* f, const int32_t* d_seqs, int n, int layer, int n_layers, const void* d_k, const void* d_v, int dtype, int T, long long stride_layer,
         long long stride_seq, long long stride_token, long long stride_head, const int32_t* d_some, void* stream) {
    if (const char* why = fp4_why_not(f)) return op_bad(who, why);
    const specdec_cache* c = &f->codes;
    if (!c->d_held || !c->d_refs) return op_bad(who, "a pointer is NULL");
    const int e = op_elem_bytes(dtype);
    if (!e) return op_bad(who, "unknown dtype");
    if ((n && T && (!d_seqs || !d_k || !d_v)) || n < 0 || (!READ && n > c->n_seqs) || n > 65535 || T < 0 || layer < 0 || n_layers < 1 || n_layers > 32767 || layer > c->n_layers - n_layers)
        return op_bad(who, "a pointer is NULL, or n, T or the layers are out of range");
    const long long st[4] = {op_stride(stride_layer, n_layers), op_stride(stride_seq, n), op_stride(stride_token, T), op_stride(stride_head, c->n_heads)};
    for (long long s : st) if (s * e % 16) return op_bad(who, "a stride is not a multiple of 16 bytes");
    if (((uintptr_t)d_k | (uintptr_t)d_v) & 15) return op_bad(who, "d_k or d_v is not 16-byte aligned");
    if (n == 0 || T == 0) return SPECDEC_OK;
    Fp4Io a;
    a.s_layer = op_stride(c->stride_layer, c->n_layers); a.s_side = c->stride_side; a.s_page = op_stride(c->stride_page, c->n_pages); a.s_head = op_stride(c->stride_head, c->n_heads);
    a.c_layer = op_stride(f->scale_stride_layer, c->n_layers); a.c_side = f->scale_stride_side; a.c_page = op_stride(f->scale_stride_page, c->n_pages);
    a.c_head = op_stride(f->scale_stride_head, c->n_heads);
    a.codes = (char*)c->d_kv + layer * a.s_layer; a.scales = (char*)f->d_scales + layer * a.c_layer;
    a.x[0] = (char*)const_cast<void*>(d_k); a.x[1] = (char*)const_cast<void*>(d_v);
    a.x_layer = st[0] * e; a.x_seq = st[1] * e; a.x_token = st[2] * e; a.x_head = st[3] * e;
    a.unit = f->d_unit ? f->d_unit + (long long)layer * 2 * c->n_heads : nullptr;
    a.table = c->d_table; a.length = c->d_length; a.held = c->d_held; a.refs = c->d_refs; a.seqs = d_seqs; a.some = d_some; a.status = c->d_status;
    a.n_pages = c->n_pages; a.n_seqs = c->n_seqs; a.max_pages = c->max_pages; a.page_shift = __builtin_ctz(c->page_tokens); a.heads = c->n_heads; a.T = T;
    const long long ctas = ((long long)c->n_heads * T * (c->head_dim / FP4_BLOCK) + 255) / 256;
    if (ctas > 0x7fffffff) return op_fail(SPECDEC_ERR_CAPACITY, who, "too many tokens for one launch");
    const bool unit = a.unit != nullptr;
    auto k = dtype == SPECDEC_DTYPE_F32 ? kernel<READ, float>(c->head_dim, unit) : dtype == SPECDEC_DTYPE_BF16 ? kernel<READ, __nv_bfloat16>(c->head_dim, unit) : kernel<READ, __half>(c->head_dim, unit);
    return op_done(who, op_launch(k, dim3((unsigned)ctas, n, 2 * n_layers), 256, 0, (cudaStream_t)stream, 1, a));
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

int specdec_packed_cache_append(const specdec_packed_cache* c, const int32_t* d_seqs, int n, int layer, int n_layers, const void* d_k, const void* d_v, int dtype, int T, long long stride_layer,
                             long long stride_seq, long long stride_token, long long stride_head, const int32_t* d_count, void* stream) {
    return move<false>("packed_cache_append", c, d_seqs, n, layer, n_layers, d_k, d_v, dtype, T, stride_layer, stride_seq, stride_token, stride_head, d_count, stream);
}
int specdec_packed_cache_read(const specdec_packed_cache* c, const int32_t* d_seqs, int n, int layer, int n_layers, void* d_k, void* d_v, int dtype, int T, long long stride_layer,
                           long long stride_seq, long long stride_token, long long stride_head, const int32_t* d_start, void* stream) {
    return move<true>("packed_cache_read", c, d_seqs, n, layer, n_layers, d_k, d_v, dtype, T, stride_layer, stride_seq, stride_token, stride_head, d_start, stream);
}

}  // extern "C"
