// Tokens into and out of a K/V cache in 4 bits (contract: specdec.h, format: fp4.cuh).
//
// CTA = up to 64 tokens of a sequence, one layer, keys or values: their slots are looked up once, then a thread takes the sixteen channels of a scale at a time:
// 32 or 64 bytes in, 8 bytes of codes and one of scales out (read: the reverse).  Threads run along a head's tokens, so that a warp's codes and scales are whole stretches of a page.
// What bounds it is the latency of its loads, at 48 warps an SM: a prompt of 8 x 509 tokens, 32 layers of 8 heads of 128 in bf16 (683 MB each way), written in 142 us and read in 122, 4.8 and
// 5.6 TB/s.  (Two items of a thread under way, in more registers: 152 and 132.)
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

constexpr int TOKENS = 64;

__device__ __forceinline__ float bits16(float x) { return __uint_as_float((__float_as_uint(x) + 0x80u) & 0xffffff00u); }         // rounded to 16 significant bits

// Sixteen numbers to codes and a scale.
// EXACT: by division.  Else x has at most 11 significant bits (a 16-bit type), and the two quotients are taken as products, whose errors are rounded away: a point halfway between scales has 5
// significant bits, and six times it 7; a point halfway between codes (from 0.25 on) times a scale has 7.  So a quotient lies on such a point, or at least 2^-13 of itself beside it.  The products
// with 1 / 6 and 1 / s are off by less than 2^-21; rounded to 16 bits they lie on the point, or on the same side of it, as the quotient does.
template <bool EXACT> __device__ __forceinline__ uint2 pack16(float* x, uint32_t& scale) {
    float top = 0.f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) { top = fmaxf(top, fabsf(x[i])); nan |= x[i] != x[i]; }
    scale = nan ? 0x7fu : fp4_scale_of(EXACT ? __fdiv_rn(top, 6.f) : bits16(top * (1.f / 6.f)));
    const uint32_t s2 = fp4_scales2(scale);
    const float s = __half2float(__low2half(*reinterpret_cast<const __half2*>(&s2)));
    if (EXACT) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = scale ? __fdiv_rn(x[i], s) : 0.f;
    } else {
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
        if (!scale) r = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = bits16(x[i] * r);
    }
    return make_uint2(fp4_pack8(x), fp4_pack8(x + 8));
}

template <bool READ, typename T, int D, bool UNIT>
__global__ void __launch_bounds__(256) k_fp4_move(Fp4Io a) {
    constexpr int NB = D / FP4_BLOCK;
    __shared__ int slot_page[TOKENS], slot_at[TOKENS];    // page (-1: none), place in it
    op_begin();
    const int i = blockIdx.y, layer = blockIdx.z >> 1, side = blockIdx.z & 1, t0 = blockIdx.x * TOKENS, s = a.seqs[i];
    const bool known = (unsigned)s < (unsigned)a.n_seqs;
    const int n = min(TOKENS, (!READ && a.some ? min(a.some[i], a.T) : a.T) - t0);
    if (n <= 0) return;
    int lost = known ? 0 : SPECDEC_CACHE_BAD_INDEX;
    for (int j = threadIdx.x; j < n; j += blockDim.x) {
        const long long at = known ? (long long)(READ && a.some ? a.some[i] : a.length[s]) + t0 + j : -1;
        const int pos = at > 0x7fffffff ? -1 : (int)at, p = known ? page_at(a, s, pos, !READ) : -1;
        slot_page[j] = p; slot_at[j] = pos & ((1 << a.page_shift) - 1);
        if (!READ && known && p < 0) lost = SPECDEC_CACHE_UNRESERVED;
    }
    if (lost) atomicOr(a.status, lost);
    __syncthreads();
    char* x0 = a.x[side] + layer * a.x_layer + i * a.x_seq + t0 * a.x_token;
    char* codes = a.codes + layer * a.s_layer + side * a.s_side;
    char* scales = a.scales + layer * a.c_layer + side * a.c_side;
    const float* units = UNIT ? a.unit + (layer * 2 + side) * a.heads : nullptr;
    const int b = threadIdx.x % NB, step = blockDim.x / NB;
    int t = threadIdx.x / NB, h = 0;
    for (;; t += step) {
        while (t >= n && h < a.heads) { t -= n; ++h; }
        if (h >= a.heads) break;
        char* at = x0 + t * a.x_token + h * a.x_head + b * 16 * (int)sizeof(T);
        const int p = slot_page[t];
        char* code = codes + p * a.s_page + h * a.s_head + slot_at[t] * (D / 2) + b * 8;
        char* scale_at = scales + p * a.c_page + h * a.c_head + slot_at[t] * (D / 16) + b;
        float x[16];
        if constexpr (READ) {
            uint2 w = make_uint2(0, 0);
            uint32_t z = 0;
            if (p >= 0) { w = *reinterpret_cast<const uint2*>(code); z = *reinterpret_cast<const unsigned char*>(scale_at); }
            const uint32_t s2 = fp4_scales2(z | z << 8);
            const float unit = UNIT ? units[h] : 1.f;
            uint32_t o[8];
            fp4_unpack8(w.x, o); fp4_unpack8(w.y, o + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t v = h2_mul(o[e], s2);      // exact
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
                x[2 * e] = UNIT ? f.x * unit : f.x; x[2 * e + 1] = UNIT ? f.y * unit : f.y;
            }
            store16<T>(at, x);
        } else {
            load16<T>(at, x);
            if (UNIT) {
                const float unit = units[h];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = __fdiv_rn(x[e], unit);
            }
            uint32_t scale;
            const uint2 y = pack16<UNIT || sizeof(T) == 4>(x, scale);
            if (p < 0) continue;
            *reinterpret_cast<uint2*>(code) = y;
            *reinterpret_cast<unsigned char*>(scale_at) = (unsigned char)scale;
        }
    }
}

template <bool READ, typename T> auto kernel(int dim, bool unit) {
    return dim == 64 ? (unit ? k_fp4_move<READ, T, 64, true> : k_fp4_move<READ, T, 64, false>) : unit ? k_fp4_move<READ, T, 128, true> : k_fp4_move<READ, T, 128, false>;
}

template <bool READ>
int move(const char* who, const specdec_packed_cache* f, const specdec_packed_tokens* g, void* stream) {
    if (const char* why = fp4_why_not(f)) return op_bad(who, why);
    const specdec_cache* c = &f->codes;
    if (!c->d_held || !c->d_refs || !g) return op_bad(who, "a pointer is NULL");
    const int n = g->n, T = g->T, layer = g->layer, n_layers = g->n_layers, dtype = g->dtype, e = op_elem_bytes(dtype);
    if (!e) return op_bad(who, "unknown dtype");
    if ((n && T && (!g->d_seqs || !g->d_k || !g->d_v)) || n < 0 || (!READ && n > c->n_seqs) || n > 65535 || T < 0 || layer < 0 || n_layers < 1 || n_layers > 32767 || layer > c->n_layers - n_layers)
        return op_bad(who, "a pointer is NULL, or n, T or the layers are out of range");
    const long long st[4] = {op_stride(g->stride_layer, n_layers), op_stride(g->stride_seq, n), op_stride(g->stride_token, T), op_stride(g->stride_head, c->n_heads)};
    for (long long s : st) if (s * e % 16) return op_bad(who, "a stride is not a multiple of 16 bytes");
    if (((uintptr_t)g->d_k | (uintptr_t)g->d_v) & 15) return op_bad(who, "d_k or d_v is not 16-byte aligned");
    if (n == 0 || T == 0) return SPECDEC_OK;
    Fp4Io a;
    a.s_layer = op_stride(c->stride_layer, c->n_layers); a.s_side = c->stride_side; a.s_page = op_stride(c->stride_page, c->n_pages); a.s_head = op_stride(c->stride_head, c->n_heads);
    a.c_layer = op_stride(f->scale_stride_layer, c->n_layers); a.c_side = f->scale_stride_side; a.c_page = op_stride(f->scale_stride_page, c->n_pages);
    a.c_head = op_stride(f->scale_stride_head, c->n_heads);
    a.codes = (char*)c->d_kv + layer * a.s_layer; a.scales = (char*)f->d_scales + layer * a.c_layer;
    a.x[0] = (char*)g->d_k; a.x[1] = (char*)g->d_v;
    a.x_layer = st[0] * e; a.x_seq = st[1] * e; a.x_token = st[2] * e; a.x_head = st[3] * e;
    a.unit = f->d_unit ? f->d_unit + (long long)layer * 2 * c->n_heads : nullptr;
    a.table = c->d_table; a.length = c->d_length; a.held = c->d_held; a.refs = c->d_refs; a.seqs = g->d_seqs; a.some = g->d_some; a.status = c->d_status;
    a.n_pages = c->n_pages; a.n_seqs = c->n_seqs; a.max_pages = c->max_pages; a.page_shift = __builtin_ctz(c->page_tokens); a.heads = c->n_heads; a.T = T;
    const int tokens = T < TOKENS ? T : TOKENS;
    const long long items = (long long)c->n_heads * tokens * (c->head_dim / FP4_BLOCK);
    const int threads = items > 128 ? 256 : items > 64 ? 128 : items > 32 ? 64 : 32;
    const bool unit = a.unit != nullptr;
    auto k = dtype == SPECDEC_DTYPE_F32 ? kernel<READ, float>(c->head_dim, unit) : dtype == SPECDEC_DTYPE_BF16 ? kernel<READ, __nv_bfloat16>(c->head_dim, unit) : kernel<READ, __half>(c->head_dim, unit);
    return op_done(who, op_launch(k, dim3((T + TOKENS - 1) / TOKENS, n, 2 * n_layers), threads, 0, (cudaStream_t)stream, 1, a));
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

int specdec_packed_cache_append(const specdec_packed_cache* c, const specdec_packed_tokens* t, void* stream) { return move<false>("packed_cache_append", c, t, stream); }
int specdec_packed_cache_read(const specdec_packed_cache* c, const specdec_packed_tokens* t, void* stream) { return move<true>("packed_cache_read", c, t, stream); }

}  // extern "C"
