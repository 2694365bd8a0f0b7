/* Products and lookups of a matrix of 8-bit floating point codes (OCP e4m3) with a scale for each block of 128 x 128 (bitlinear.h,
 * bl_f8_linear, bl_f8_embed).
 *
 *     y[m][n] = sum_b s[m][b] * ws[n / 128][b] * P,   P = sum of c[m][k] * w[n][k] over the block's 128 k
 *
 * c and s: the row's codes and scales, made from its bf16 values.  P comes from the matrix cores and is scaled and added in fp32.  The weights are the first operand and the tokens the second, so that a lane has one token and its scale,
 * and four consecutive weight rows, which is a run of the output.  A lane's 32 codes of a block are 16 from offset 16 g and 16 from 64 + 16 g,
 * g = lane / 16: the order of k inside a block is free as long as both operands have the same. */
#include <atomic>
#include <type_traits>

#include "bl_device.h"
#include "bl_host.h"
#include "bl_producer.h"

typedef int f8_v8i __attribute__((ext_vector_type(8)));
typedef _Float16 f8_v8h __attribute__((ext_vector_type(8)));
typedef _Float16 f8_v2h __attribute__((ext_vector_type(2)));
typedef uint32_t f8_v4u __attribute__((ext_vector_type(4)));

#define F8_BLOCK 128
#define F8_TOP 448.0f

struct f8_args {
    const uint8_t* w;
    const float* ws;
    int64_t w_stride, ws_stride;
    uint8_t* codes;                /* [M][nb * 128] */
    float* scales;                 /* [nb][M] */
    void* y;
    int64_t y_stride;
    float* part;                   /* [splits][M][N] where the k loop is split */
    int M, N, K, nb;
    int bf16;                      /* output type */
    int splits, tiles_m, tiles_n;
};

__device__ __forceinline__ f8_v8i f8_join(bl_v4i a, bl_v4i b) { return f8_v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }
/* The codes are opened to fp16, which holds every one of them, and multiplied there: products are exact and sums have 32 bits.  The matrix cores take the codes
 * as they are too, at twice the rate, but line a block's products up with the largest and cut what falls below: 1.4e-5 of the sum's size on normal values
 * (fp16: 1e-8), 2^-12 of sum |c w| where sizes are spread over all that e4m3 has: fewer bits than an fp32 output stands for. */
struct f8_halves {                 /* 32 codes of a lane */
    f8_v8h v[4];
};
__device__ __forceinline__ f8_halves f8_open(f8_v8i c) {
    f8_halves h;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f8_v4u u;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            u[j] = __builtin_bit_cast(uint32_t, j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * i + j / 2], 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * i + j / 2], 1.0f, false));
        h.v[i] = __builtin_bit_cast(f8_v8h, u);
    }
    return h;
}
__device__ __forceinline__ bl_v4f f8_product(const f8_halves& w, const f8_halves& x) {
    bl_v4f p = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[i], x.v[i], p, 0, 0, 0);
    return p;
}

/* A number that the whole wave reads, through the scalar cache: its load is none of those that are counted. */
__device__ __forceinline__ float f8_uniform(const float* p) { return *(const float __attribute__((address_space(4)))*)(uintptr_t)p; }

/* ---- rows to codes ----------------------------------------------------------------------------------------------------- */

/* The scale of a group whose largest |value| is g (a NaN counts as the largest; fmaxf then gives the floor, and the NaN's own code
 * spoils the row, as an infinity does, which meets the factor 0). */
__device__ __forceinline__ float f8_scale(float g) { return fmaxf(g, 1e-5f) * (1.0f / F8_TOP); }
__device__ __forceinline__ int f8_codes4(uint32_t a, uint32_t b, float inv) {
    const int c = __builtin_amdgcn_cvt_pk_fp8_f32(bl_bf16_to_f32(a & 0xffffu) * inv, __uint_as_float(a & 0xffff0000u) * inv, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(bl_bf16_to_f32(b & 0xffffu) * inv, __uint_as_float(b & 0xffff0000u) * inv, c, true);
}
__device__ __forceinline__ bl_v4i f8_codes16(const uint4& lo, const uint4& hi, float inv) {
    return bl_v4i{f8_codes4(lo.x, lo.y, inv), f8_codes4(lo.z, lo.w, inv), f8_codes4(hi.x, hi.y, inv), f8_codes4(hi.z, hi.w, inv)};
}
__device__ __forceinline__ float f8_largest16(const uint4& lo, const uint4& hi) {
    return bl_max_pos(bl_absmax8_bf16<false>(lo), bl_absmax8_bf16<false>(hi));
}

/* A thread's unit of 16 values: eight threads have a group of 128. */
__device__ __forceinline__ void f8_put_unit(const f8_args& A, int m, int u, const uint4& lo, const uint4& hi) {
    float g = f8_largest16(lo, hi);
    g = bl_max_pos(g, bl_dppf<BL_DPP_QUAD_XOR1>(g));
    g = bl_max_pos(g, bl_dppf<BL_DPP_QUAD_XOR2>(g));
    g = bl_max_pos(g, bl_dppf<BL_DPP_ROW_HALF_MIRROR>(g));
    const float s = f8_scale(g);
    *(bl_v4i*)(A.codes + ((int64_t)m * A.nb * 8 + u) * 16) = f8_codes16(lo, hi, bl_div_rn(1.0f, s));
    if ((u & 7) == 0) A.scales[(int64_t)(u >> 3) * A.M + m] = s;
}
/* A workgroup a row, whose norm meets in it.  Zeros behind K in the last block.  Bound by the launch and the chain row -> sum -> root -> codes: one row 2.4 to 4.7 us, 1025 rows of
 * 3328 7.6, with the sum, the root or the scales' stores left out 7.3 to 7.8. */
__global__ __launch_bounds__(256) void bl_f8_rows(f8_args A, bl_prod_dev P) {
    __shared__ double s4[4];
    const int m = (int)blockIdx.x, tid = threadIdx.x, groups = A.K / 16, all = A.nb * 8;
    uint4 xv[4];
    float rn = 0.0f;
    if (P.norm) rn = bl_norm_produce2(P, m, A.K, true, s4, xv);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    if (P.norm) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int u = tid + 256 * j;
            if (u < all) f8_put_unit(A, m, u, u < groups ? xv[2 * j] : zero, u < groups ? xv[2 * j + 1] : zero);
        }
    }
    for (int u = tid + (P.norm ? 512 : 0); u < all; u += 256) {
        uint4 lo = zero, hi = zero;
        if (u < groups) bl_produce16<true>(P, m, u, A.K, true, rn, lo, hi);     /* (behind a norm's 512 units nobody has stored the sum) */
        f8_put_unit(A, m, u, lo, hi);
    }
}

/* The same without a norm, where nothing crosses a group: the units of all rows in one line (2048 rows of 2560 from bf16, 16 MB, 6.4 us). */
__global__ __launch_bounds__(256) void bl_f8_units(f8_args A, bl_prod_dev P) {
    const int groups = A.K / 16, all = A.nb * 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)A.M * all) return;                      /* (groups of eight threads, whole ones) */
    const int m = (int)(i / all), u = (int)(i - (int64_t)m * all);
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    if (u < groups) bl_produce16<false>(P, m, u, A.K, true, 0.0f, lo, hi);
    f8_put_unit(A, m, u, lo, hi);
}

/* ---- output -------------------------------------------------------------------------------------------------------------- */

__device__ __forceinline__ uint16_t f8_bf16(float v) { return (uint16_t)bl_pack2_bf16(v, v); }
/* Four consecutive outputs n .. n + 3 of row m: one store, whatever the row's alignment (the memory takes vectors at any element; the types say so, and
 * bl_g would not hand it on). */
typedef uint32_t f8_out2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f8_out4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void f8_store4(const f8_args& A, int m, int n, const float (&v)[4]) {
    const int64_t at = (int64_t)m * A.y_stride + n;
    if (n + 4 <= A.N) {
        if (A.bf16) *(f8_out2 BL_G*)((uint16_t*)A.y + at) = (f8_out2){bl_pack2_bf16(v[0], v[1]), bl_pack2_bf16(v[2], v[3])};
        else *(f8_out4 BL_G*)((float*)A.y + at) = (f8_out4){v[0], v[1], v[2], v[3]};
    } else {
        for (int i = 0; i < 4 && n + i < A.N; ++i) {
            if (A.bf16) ((uint16_t*)A.y)[at + i] = f8_bf16(v[i]);
            else ((float*)A.y)[at + i] = v[i];
        }
    }
}

/* ---- stream: few tokens ---------------------------------------------------------------------------------------------------- */

/* Up to 16 * MT tokens.  A workgroup of eight waves walks strips of 16 weight rows; wave w has the blocks w, w + 8, .. of k (KB of them at most), for
 * which it keeps the tokens' codes and scales in registers, and meets the others' sums in LDS; one barrier a strip.  A block's 2 KB go to LDS in whole lines (eight
 * rows of 128 bytes a load) and from there to the lanes; a wave has AHEAD of them in flight, in a ring of its own.  Bound by HBM: 128256 x 2560, 328 MB, one row 48 us = 6.8 TB/s
 * (straight to the lanes, whose rows are lines of their own, 78), 48 rows 73 with 25 MB of outputs written beside it.
 * (Four waves along k instead of eight: 48 rows 79 for 81 then, and 18 kernels more.)  FUSED: the rows are made here, by every workgroup: a lane has
 * what its token needs for its own blocks, so that only the sum of squares of a norm crosses waves. */
#define F8_WAVES 8
template <int MT, int KB>
struct f8_stream_shape {
    static constexpr bool open = KB * MT <= 9;
    static constexpr int groups = MT <= 2 && KB * MT <= 4 ? 2 : 1;          /* workgroups a unit, by registers; by LDS: */
    static constexpr int waves = 2 * groups;                  /* a SIMD */
    static constexpr int ahead = groups == 2 ? 4 - MT : 5;
    static constexpr int ring = (ahead + 1) * 2048, sums = 2 * F8_WAVES * MT * 16 * 16 * 4, bytes = F8_WAVES * ring + sums;
};
template <int MT, int KB, bool FUSED>
__global__ __launch_bounds__(F8_WAVES * 64, (f8_stream_shape<MT, KB>::waves)) void bl_f8_stream(f8_args A, bl_prod_dev P) {
    typedef f8_stream_shape<MT, KB> shape;
    constexpr int AHEAD = shape::ahead;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    typedef float sums_t[F8_WAVES][MT * 16][16];
    sums_t* red = (sums_t*)(lds + F8_WAVES * shape::ring);
    __shared__ double squares[F8_WAVES][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int strips = (A.N + 15) / 16, stride = (int)gridDim.x;
    const bl_v4i zero = {0, 0, 0, 0};
    int strip = (int)blockIdx.x;
    /* The ring: block j of a strip is 16 rows of 128 bytes; unit u of row q lies at unit u ^ (q / 2 % 8).  Behind the wave's last block its first is asked for
     * again, so that the number in flight is always the same.  (Units behind a K that is no multiple of 128: as in the tiles.) */
    const int blocks = (A.nb - wave + F8_WAVES - 1) / F8_WAVES;             /* of this wave; may be none */
    uint8_t* const ring = lds + wave * shape::ring;
    const int lrow = lane >> 3, lunit = (lane & 7) ^ (lrow >> 1), lunit2 = lunit ^ 4;       /* rows lrow and lrow + 8 */
    int load_strip = strip, load_j = 0, load_slot = 0, slot = 0;
    auto load = [&]() {
        const int b = wave + F8_WAVES * load_j, n = load_strip * 16 + lrow;
        const bool half = (b + 1) * F8_BLOCK > A.K;
        const uint8_t* at = A.w + (int64_t)b * F8_BLOCK;
        uint8_t* to = ring + load_slot * 2048;
        __builtin_amdgcn_global_load_lds((bl_gptr)(at + (n < A.N ? n : A.N - 1) * A.w_stride + (half ? lunit & 3 : lunit) * 16), (bl_lptr)to, 16, 0, 2);
        __builtin_amdgcn_global_load_lds((bl_gptr)(at + (n + 8 < A.N ? n + 8 : A.N - 1) * A.w_stride + (half ? lunit2 & 3 : lunit2) * 16), (bl_lptr)(to + 1024), 16, 0, 2);
        load_slot = load_slot == AHEAD ? 0 : load_slot + 1;
        if (++load_j == blocks) {
            load_j = 0;
            if (load_strip + stride < strips) load_strip += stride;
        }
    };
    if (blocks > 0)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) load();
    /* the tokens' codes, opened once where the registers are there (as fp16 they take twice as many), else for every strip again */
    std::conditional_t<shape::open, f8_halves, f8_v8i> x[MT][KB];
    float xs[MT][KB];
    auto keep = [&](int t, int j, f8_v8i c) {
        if constexpr (shape::open) x[t][j] = f8_open(c);
        else x[t][j] = c;
    };
    if constexpr (FUSED) {
        static_assert(MT == 1 && KB == 1, "rows are made for one tile of tokens and a block a wave");
        /* everything the lane needs at once, so that it hangs on one round of loads */
        float v[KB][2][16];
#pragma unroll
        for (int j = 0; j < KB; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int b = wave + F8_WAVES * j;
                if (r < A.M && b * F8_BLOCK + 64 * i < A.K) {
                    bl_produce16_f32(P, r, b * 8 + 4 * i + g, A.K, blockIdx.x == 0, v[j][i]);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[j][i][e] = 0.0f;
                }
            }
        if (P.norm) {
            double ss = 0.0;
#pragma unroll
            for (int j = 0; j < KB; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) ss += (double)v[j][i][e] * (double)v[j][i][e];
            ss += __shfl_xor(ss, 16);
            ss += __shfl_xor(ss, 32);
            if (lane < 16) squares[wave][lane] = ss;
            __syncthreads();
            double sum = 0.0;
#pragma unroll
            for (int w = 0; w < F8_WAVES; ++w) sum += squares[w][r];
            const float rn = (float)(1.0 / sqrt(sum / (double)A.K + (double)P.eps));
#pragma unroll
            for (int j = 0; j < KB; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int b = wave + F8_WAVES * j, u = b * 8 + 4 * i + g;
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[j][i][e] *= rn;
                    if (P.gain && b * F8_BLOCK + 64 * i < A.K) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) {
                            const bl_v4f x = *bl_gc<bl_v4f>(P.gain + (int64_t)u * 16 + e);
                            v[j][i][e] *= x[0], v[j][i][e + 1] *= x[1], v[j][i][e + 2] *= x[2], v[j][i][e + 3] *= x[3];
                        }
                    }
                }
        }
#pragma unroll
        for (int j = 0; j < KB; ++j) {
            uint4 lo[2], hi[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float (&y)[16] = v[j][i];
                lo[i] = make_uint4(bl_pack2_bf16(y[0], y[1]), bl_pack2_bf16(y[2], y[3]), bl_pack2_bf16(y[4], y[5]), bl_pack2_bf16(y[6], y[7]));
                hi[i] = make_uint4(bl_pack2_bf16(y[8], y[9]), bl_pack2_bf16(y[10], y[11]), bl_pack2_bf16(y[12], y[13]), bl_pack2_bf16(y[14], y[15]));
            }
            float most = bl_max_pos(f8_largest16(lo[0], hi[0]), f8_largest16(lo[1], hi[1]));
            most = bl_max_pos(most, __shfl_xor(most, 16));
            most = bl_max_pos(most, __shfl_xor(most, 32));
            xs[0][j] = f8_scale(most);
            const float inv = bl_div_rn(1.0f, xs[0][j]);
            keep(0, j, f8_join(f8_codes16(lo[0], hi[0], inv), f8_codes16(lo[1], hi[1], inv)));
        }
    } else {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int m = t * 16 + r < A.M ? t * 16 + r : A.M - 1;
            const uint8_t* row = A.codes + (int64_t)m * A.nb * F8_BLOCK + g * 16;
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                const int b = wave + F8_WAVES * j;
                f8_v8i c = f8_join(zero, zero);
                xs[t][j] = 0.0f;
                if (b < A.nb) {
                    c = f8_join(*bl_gc<bl_v4i>(row + b * F8_BLOCK), *bl_gc<bl_v4i>(row + b * F8_BLOCK + 64));
                    xs[t][j] = A.scales[(int64_t)b * A.M + m];
                }
                keep(t, j, c);
            }
        }
    }
    int buf = 0;
    for (; strip < strips; strip += stride, buf ^= 1) {
        if constexpr (!shape::open) {                         /* (or the compiler opens them in front of the loop) */
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < KB; ++j) asm volatile("" : "+v"(x[t][j]));
        }
        bl_v4f acc[MT], p[2][MT];
        float f[2][MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = (bl_v4f){0, 0, 0, 0};
        auto add = [&](int at) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[t][v] = __builtin_fmaf(p[at][t][v], f[at][t], acc[t][v]);
        };
#pragma unroll
        for (int j = 0; j < KB; ++j) {
            if (j < blocks) {
                const float ws = f8_uniform(A.ws + (int64_t)(strip >> 3) * A.ws_stride + wave + F8_WAVES * j);
                BL_WAIT_VM(2 * (AHEAD - 1));
                asm volatile("" ::: "memory");
                const uint8_t* row = ring + slot * 2048 + r * F8_BLOCK;
                const f8_v8i c = f8_join(*(const bl_v4i*)(row + ((g ^ (r >> 1)) << 4)), *(const bl_v4i*)(row + (((g + 4) ^ (r >> 1)) << 4)));
                BL_WAIT_LGKM0();
                asm volatile("" ::: "memory");
                load();                                       /* (into the slot read before this one) */
                slot = slot == AHEAD ? 0 : slot + 1;
                const f8_halves h = f8_open(c);
#pragma unroll
                for (int t = 0; t < MT; ++t) f[j & 1][t] = xs[t][j] * ws;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    if constexpr (shape::open) p[j & 1][t] = f8_product(h, x[t][j]);
                    else p[j & 1][t] = f8_product(h, f8_open(x[t][j]));
                }
            } else {
#pragma unroll
                for (int t = 0; t < MT; ++t) p[j & 1][t] = (bl_v4f){0, 0, 0, 0}, f[j & 1][t] = 0.0f;
            }
            __builtin_amdgcn_sched_barrier(0);                /* (four products at least between a block's last and its first reader) */
            if (j > 0) {
                if (j >= blocks) bl_mfma_fence();
                add((j - 1) & 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        bl_mfma_fence();
        add((KB - 1) & 1);
#pragma unroll
        for (int t = 0; t < MT; ++t)
            if (t * 16 + r < A.M) *(bl_v4f*)&red[buf][wave][t * 16 + r][4 * g] = acc[t];
        asm volatile("" ::: "memory");
        BL_WAIT_LGKM0();
        __builtin_amdgcn_s_barrier();                         /* (the loads of the next strip stay in flight) */
        asm volatile("" ::: "memory");
        for (int i = tid; i < A.M * 16; i += F8_WAVES * 64) {
            const int m = i >> 4, n = strip * 16 + (i & 15);
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < F8_WAVES; ++w) v += red[buf][w][m][i & 15];
            if (n < A.N) {
                const int64_t at = m * A.y_stride + n;
                if (A.bf16) ((uint16_t*)A.y)[at] = f8_bf16(v);
                else ((float*)A.y)[at] = v;
            }
        }
    }
    BL_WAIT_VM(0);                                            /* (what is still on its way to LDS must not outlive the workgroup) */
}

/* Values from a row to the next of the pieces of a split k loop: whole vectors. */
__host__ __device__ static __forceinline__ int64_t f8_part_stride(int64_t N) { return (N + 3) / 4 * 4; }

/* ---- tiles: any number of tokens ------------------------------------------------------------------------------------------ */

/* BM tokens x BN weight rows a workgroup, WM x WN waves, S stages of one block of k (128) in LDS.  Rows of 128 bytes; unit u (16 bytes) of row r lies
 * at unit u ^ (r / 2 % 8), so that sixteen lanes of a read fall on all banks; the loads that go straight to LDS pick their units accordingly.
 * In the last block of a K that is no multiple of 128 the units behind K are the weights' first four again: their codes meet zeros (and a
 * NaN among them spoils the row anyway).
 * Bound by issue: 2048 rows x 13824 x 2560, 145 GFLOP, 141 to 147 us without the rows' kernel = 990 to 1030 TFLOP/s (the library's bf16 product 1190): two conversions
 * and a multiply-add of four stand beside each matrix product.  Of 169 us then, without the conversions of x 157, without loads 146, without the adds 163: none is all of it.  Two workgroups
 * of two stages a unit, so that one computes while the other opens.  Tiles of 128 x 256 and 256 x 128 with eight waves: 187 to 190 for 161; codes as they are into the 8-bit
 * instructions (fewer bits, see f8_open), one workgroup of three stages: 283. */
template <int BM, int BN, int WM, int WN, int S>
__global__ __launch_bounds__(WM * WN * 64, 2) void bl_f8_tile(f8_args A) {
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, SCALES = (BM + BN) * F8_BLOCK, STAGE = SCALES + BM * 4, LOADS = (BM + BN) / 8 / NW;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int wm = wave % WM, wn = wave / WM;
    /* consecutive workgroups go to the eight dies in turn: each takes a contiguous eighth of the tiles, tokens first */
    int place;
    {
        const int all = (int)gridDim.x, die = (int)blockIdx.x & 7, part = all >> 3, more = all & 7;
        place = die * part + (die < more ? die : more) + ((int)blockIdx.x >> 3);
    }
    const int split = place % A.splits, tile = place / A.splits, m0 = tile % A.tiles_m * BM, n0 = tile / A.tiles_m * BN;
    const int b0 = (int)((int64_t)A.nb * split / A.splits), b1 = (int)((int64_t)A.nb * (split + 1) / A.splits);
    const int half = A.K % F8_BLOCK ? A.nb - 1 : -1;          /* the block of which only half is there */
    const uint8_t* from[LOADS];                               /* what the lane loads of the next block */
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int p = j * NW + wave;                          /* 1024 bytes, eight rows */
        const bool is_x = p < BM / 8;
        const int row = (is_x ? p : p - BM / 8) * 8 + lane / 8;
        if (is_x) {
            const int m = m0 + row < A.M ? m0 + row : A.M - 1;
            from[j] = A.codes + ((int64_t)m * A.nb + b0) * F8_BLOCK;
        } else {
            const int n = n0 + row < A.N ? n0 + row : A.N - 1;
            from[j] = A.w + n * A.w_stride + (int64_t)b0 * F8_BLOCK;
        }
        from[j] += ((lane & 7) ^ (row >> 1 & 7)) * 16;
    }
    /* and the tokens' scales of the block, 64 a load: a wave loads some of them (others the same again), so that all waves count the same */
    const int sm = wave % (BM / 64) * 64;
    const float* scales = A.scales + (int64_t)b0 * A.M + (m0 + sm + lane < A.M ? m0 + sm + lane : A.M - 1);
    int loaded = b0;
    auto load = [&](int stage) {
        uint8_t* to = lds + stage * STAGE;
        if (loaded == half) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int p = j * NW + wave, row = (p - BM / 8) * 8 + lane / 8;
                if (p >= BM / 8 && (((lane & 7) ^ (row >> 1 & 7)) & 4)) from[j] -= 64;
            }
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) __builtin_amdgcn_global_load_lds((bl_gptr)from[j], (bl_lptr)(to + (j * NW + wave) * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((bl_gptr)scales, (bl_lptr)(to + SCALES + sm * 4), 4, 0, 0);
        if (++loaded < b1) {                                  /* (behind the last block it is loaded again, for nobody) */
#pragma unroll
            for (int j = 0; j < LOADS; ++j) from[j] += F8_BLOCK;
            scales += A.M;
        }
    };
    const int mrow = m0 + wm * (BM / WM) + r;
    const float* wscale = A.ws + (int64_t)((n0 + wn * (BN / WN)) / F8_BLOCK < (A.N - 1) / F8_BLOCK ? (n0 + wn * (BN / WN)) / F8_BLOCK : (A.N - 1) / F8_BLOCK) * A.ws_stride;
    bl_v4f acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int t = 0; t < TM; ++t) acc[i][t] = (bl_v4f){0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < S - 1; ++s) load(s);
    const int x_at = (wm * (BM / WM) + r) * F8_BLOCK, w_at = BM * F8_BLOCK + (wn * (BN / WN) + r) * F8_BLOCK, swz = (r >> 1) & 7;
    int stage = 0;
    for (int b = b0; b < b1; ++b) {
        const float ws = f8_uniform(wscale + b);
        BL_WAIT_VM((S - 2) * (LOADS + 1));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load(stage == 0 ? S - 1 : stage - 1);
        const uint8_t* at = lds + stage * STAGE;
        auto part = [&](int base, int t) {
            const uint8_t* p = at + base + t * 16 * F8_BLOCK;
            return f8_join(*(const bl_v4i*)(p + ((g ^ swz) << 4)), *(const bl_v4i*)(p + (((g + 4) ^ swz) << 4)));
        };
        /* One step a group of 16 weight rows: its products, and between them the next group's codes are opened and the one's before it are added. */
        f8_v8i raw[2] = {part(w_at, 0), part(w_at, TN > 1 ? 1 : 0)};
        f8_halves x[TM], w[2];
#pragma unroll
        for (int t = 0; t < TM; ++t) x[t] = f8_open(part(x_at, t));
        w[0] = f8_open(raw[0]);
        float f[TM];
#pragma unroll
        for (int t = 0; t < TM; ++t) f[t] = *(const float*)(at + SCALES + (wm * (BM / WM) + 16 * t + r) * 4) * ws;
        bl_v4f p[2][TM];
        auto add = [&](int i) {
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][t][v] = __builtin_fmaf(p[i & 1][t][v], f[t], acc[i][t][v]);
        };
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);                        /* (the other workgroup's wave opens its codes meanwhile) */
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            if (i + 2 < TN) raw[i & 1] = part(w_at, i + 2);
#pragma unroll
            for (int t = 0; t < TM; ++t) p[i & 1][t] = (bl_v4f){0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int t = 0; t < TM; ++t) p[i & 1][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[i & 1].v[k], x[t].v[k], p[i & 1][t], 0, 0, 0);
            if (i + 1 < TN) w[(i + 1) & 1] = f8_open(raw[(i + 1) & 1]);
            if (i > 0) add(i - 1);
            if (i + 2 < TN) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, TM, 0);          /* (so many between another group's last product and its first reader) */
#pragma unroll
            for (int k = 0; k < 3 * TM; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        bl_mfma_fence();
        add(TN - 1);
        BL_WAIT_LGKM0();
        stage = stage == S - 1 ? 0 : stage + 1;
    }
    BL_WAIT_VM(0);
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int m = mrow + 16 * t;
        if (m >= A.M) continue;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int n = n0 + wn * (BN / WN) + 16 * i + 4 * g;
            if (n >= A.N) continue;
            const float v[4] = {acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3]};
            if (A.splits == 1) {
                f8_store4(A, m, n, v);
            } else {
                *bl_g((bl_v4f*)(A.part + ((int64_t)split * A.M + m) * f8_part_stride(A.N) + n)) = acc[i][t];
            }
        }
    }
}

/* The pieces of a split k loop, added in their order, four columns a thread. */
__global__ __launch_bounds__(256) void bl_f8_join(f8_args A) {
    const int units = (A.N + 3) / 4;
    const int64_t all = (int64_t)A.M * units, stride = f8_part_stride(A.N);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int m = (int)(i / units), n = (int)(i - (int64_t)m * units) * 4;
        const float* from = A.part + m * stride + n;
        bl_v4f x = {0, 0, 0, 0};
        for (int s = 0; s < A.splits; s += 4) {               /* four in flight */
            bl_v4f y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = s + k < A.splits ? *bl_gc<bl_v4f>(from + (s + k) * A.M * stride) : (bl_v4f){0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 4; ++k) x += y[k];
        }
        const float v[4] = {x[0], x[1], x[2], x[3]};
        f8_store4(A, m, n, v);
    }
}

/* ---- lookup -------------------------------------------------------------------------------------------------------------- */

struct f8_lookup_args {
    const uint8_t* w;
    const float* ws;
    int64_t w_stride, ws_stride, out_stride, all;
    const int* ids;
    void* out;
    int* bad;
    int N, units;                  /* units of a row, 16 bytes of the output each */
    float multiplier;
};
/* A thread 16 bytes of the output.  Bound by HBM: 8000 rows of 2560 to bf16, 61 MB, 12.7 us = 4.8 TB/s (a large copy's rate); eight rows by the launch and the chain id -> codes: 3.8. */
template <bool BF16>
__global__ __launch_bounds__(256) void bl_f8_embed_kernel(f8_lookup_args A) {
    constexpr int V = BF16 ? 8 : 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < A.all; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / A.units;
        const int u = (int)(i - t * A.units), id = A.ids[t];
        const bool there = (unsigned)id < (unsigned)A.N;
        if (!there && id != -1 && u == 0 && A.bad) atomicAdd(A.bad, 1);
        const uint8_t* row = A.w + (there ? id : 0) * A.w_stride;
        const float s = A.ws[(int64_t)((there ? id : 0) / F8_BLOCK) * A.ws_stride + u * V / F8_BLOCK];
        uint32_t c[V / 4];
        if constexpr (BF16) {
            const bl_v2u x = *bl_gc<bl_v2u>(row + u * V);
            c[0] = x[0], c[1] = x[1];
        } else {
            c[0] = *bl_gc<uint32_t>(row + u * V);
        }
        float v[V];
#pragma unroll
        for (int j = 0; j < V / 4; ++j) {
            const float f[4] = {__builtin_amdgcn_cvt_f32_fp8((int)c[j], 0), __builtin_amdgcn_cvt_f32_fp8((int)c[j], 1),
                                __builtin_amdgcn_cvt_f32_fp8((int)c[j], 2), __builtin_amdgcn_cvt_f32_fp8((int)c[j], 3)};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * j + e] = there ? (f[e] * s) * A.multiplier : 0.0f;
        }
        if constexpr (BF16) {
            *bl_g((bl_v4i*)((uint16_t*)A.out + t * A.out_stride + u * V)) =
                (bl_v4i){(int)bl_pack2_bf16(v[0], v[1]), (int)bl_pack2_bf16(v[2], v[3]), (int)bl_pack2_bf16(v[4], v[5]), (int)bl_pack2_bf16(v[6], v[7])};
        } else {
            *bl_g((bl_v4f*)((float*)A.out + t * A.out_stride + u * V)) = (bl_v4f){v[0], v[1], v[2], v[3]};
        }
    }
}

/* ---- host ---------------------------------------------------------------------------------------------------------------- */

static bl_status f8_check(const bl_f8_matrix* w) {
    if (!w->codes || !w->scale) return BL_ERR_NULL;
    const int64_t most = (int64_t)1 << 40;
    if (!bl_shape_ok(w->N, w->K) || w->K % 64 || w->stride < w->K || w->stride > most || w->scale_stride < (w->K + F8_BLOCK - 1) / F8_BLOCK || w->scale_stride > most)
        return BL_ERR_SHAPE;
    if (!bl_aligned(w->codes, 16) || w->stride % 16 || !bl_aligned(w->scale, 4)) return BL_ERR_ALIGN;
    return BL_OK;
}

struct f8_plan {
    int splits, tokens, blocks;    /* of the stream: tiles of 16 tokens (0: not it), blocks of k a wave */
    bool fused, small;             /* small: tiles of 64 x 64 */
    size_t codes, scales, bytes;   /* of the workspace: bytes of the codes, of the scales behind them, of all */
};
static size_t f8_round(size_t n) { return (n + 255) / 256 * 256; }
static f8_plan f8_make_plan(const bl_f8_product* p) {
    f8_plan q;
    const int64_t nb = (p->w.K + F8_BLOCK - 1) / F8_BLOCK;
    q.splits = 1;
    /* The stream, while a wave's registers hold its blocks of every token, and where they hold them opened or there are few rows of tiles.  us of it and of tiles:
     * 2560 x 2560 17 to 64 rows 8.6 to 11.9 and 11.4 to 13.9; 128256 x 2560 17, 48, 64 rows 61, 72, 94 and 71, 80, 86; 40000 x 2560 48, 64 rows 28.8, 36.2 and 26.2,
     * 26.6; x 4096 17, 48 rows 36.6, 44.9 and 37.3, 37.4; 4096 x 4096 48 rows 14.2 and 15.0, 8192 16.9 and 16.1.  Up to 16 rows: the stream up to K = 8192, the most that a wave's
     * registers hold; behind it tiles, most of whose rows are copies then: 4096 x 8192 and x 9216 one row 9.0 and 14.8, 16 rows 11.8 and 15.8, 128256 x 8192 and x 9216 one row 159 and 226
     * (a large copy's rate: 221 and 249). */
    const int64_t each = (nb + F8_WAVES - 1) / F8_WAVES;
    q.tokens = p->M <= 64 ? (int)((p->M + 15) / 16) : 0, q.blocks = each > 8 ? 16 : each <= 4 ? (int)each : each <= 6 ? 6 : 8;
    if (q.tokens * q.blocks > (p->w.N >= 8192 ? 9 : 12)) q.tokens = 0;
    /* rows made in the stream itself: 300 x 320 4.1 us, 5.5 with a launch of their own, 1000 x 1024 4.8 and 5.7 (longer rows spill: 2560 x 2560 22.9, so 6.5) */
    q.fused = q.tokens == 1 && q.blocks == 1;
    if (q.tokens) {
        q.codes = q.fused ? 0 : f8_round((size_t)p->M * nb * F8_BLOCK), q.scales = q.fused ? 0 : f8_round((size_t)p->M * nb * sizeof(float));
        q.bytes = q.codes + q.scales;
        return q;
    }
    q.codes = f8_round((size_t)p->M * nb * F8_BLOCK), q.scales = f8_round((size_t)p->M * nb * sizeof(float));
    const int64_t large = ((p->M + 127) / 128) * ((p->w.N + 127) / 128), small = ((p->M + 63) / 64) * ((p->w.N + 63) / 64);
    /* Tiles of 64 x 64 while those of 128 x 128 are fewer than the units, or would be half empty.  us of the small and the large (neither cut along k where there are
     * enough): 13824 x 2560 65, 512 rows 20, 53 and 32, 43, 2048 rows 198 and 151; 4096 x 8192 256, 2048 rows 34, 187 and 89, 128; 32000 x 4096 64, 65, 256 rows 29, 47, 88 and
     * 48, 48, 64; 2560 x 2560 2048 rows 47.4 and 45.6. */
    q.small = large < 192 || p->M <= 64;
    /* Pieces of k until there are 512 workgroups, two a unit, of two blocks at least, where k is long enough to pay for the join.  us with and without:
     * 2560 x 6912 65, 200, 512 rows 18, 24, 44 and 38, 40, 45; 337 x 6784 65 to 2048 13 to 38 and 38 to 48; 2560 x 2560 65, 200 rows 13.5, 16.9 and 18.0, 18.6;
     * 1188 x 1920 65, 512 rows 11.3, 16.9 and 14.7, 16.1; 1000 x 1024 65, 512, 1024 rows 9.8, 14.8, 17.2 and 10.7, 11.4, 12.6.  For 256 workgroups: 4096 x 8192 200 rows
     * 33 and 46. */
    const int64_t tiles = q.small ? small : large;
    int64_t s = tiles < 512 ? 512 / tiles : 1;
    if (s > nb / 2) s = nb / 2;
    q.splits = s < 1 || nb < 12 || !q.small ? 1 : s > 16 ? 16 : (int)s;
    q.bytes = q.codes + q.scales + (q.splits > 1 ? (size_t)q.splits * p->M * f8_part_stride(p->w.N) * sizeof(float) : 0);
    return q;
}

static bl_status f8_check_product(const bl_f8_product* p, bl_prod_dev* prod) {
    if (!p) return BL_ERR_NULL;
    if (const bl_status rc = f8_check(&p->w)) return rc;
    if (!p->y || !p->prod.in0) return BL_ERR_NULL;
    if (p->y_kind != BL_F8_OUT_F32 && p->y_kind != BL_F8_OUT_BF16) return BL_ERR_VALUE;
    if (p->M < 1 || p->M >= BL_MAX_DIM || p->y_stride < p->w.N || p->y_stride > ((int64_t)1 << 40)) return BL_ERR_SHAPE;
    if (!bl_aligned(p->y, p->y_kind == BL_F8_OUT_F32 ? 4 : 2)) return BL_ERR_ALIGN;
    if (!bl_make_prod(p->prod, nullptr, p->w.K, prod)) return BL_ERR_VALUE;
    /* (a launch counts its threads in 32 bits) */
    if (((p->M + 127) / 128) * ((p->w.N + 127) / 128) >= 1 << 24) return BL_ERR_SHAPE;
    return BL_OK;
}

/* What is written may not be what is read: several workgroups make the same rows where the stream makes them, and long normed rows are made twice. */
struct f8_range {
    uintptr_t at;
    uint64_t bytes;
};
static bool f8_meet(const f8_range& a, const f8_range& b) { return a.at && b.at && a.at < b.at + b.bytes && b.at < a.at + a.bytes; }
static bool f8_overlap(const bl_f8_product* p, const f8_plan& q) {
    const uint64_t MK = (uint64_t)p->M * (uint64_t)p->w.K;
    const int kind = p->prod.kind;
    const bool sum = kind == BL_PROD_RESIDUAL;
    const uint64_t row = (uint64_t)(p->prod.n_q + 2 * (int64_t)p->prod.n_kv) * p->prod.head_dim;
    const f8_range y = {(uintptr_t)p->y, ((uint64_t)(p->M - 1) * p->y_stride + p->w.N) * (p->y_kind == BL_F8_OUT_BF16 ? 2 : 4)};
    const f8_range aux = {sum ? (uintptr_t)p->prod.aux_out : 0, MK * 4}, space = {q.bytes ? (uintptr_t)p->workspace : 0, q.bytes};
    const f8_range in[] = {{(uintptr_t)p->prod.in0, kind == BL_PROD_BF16 ? MK * 2 : kind == BL_PROD_ATTN_V ? p->M * row * 4 : kind == BL_PROD_RELU2_GATE ? MK * 8 : MK * 4},
                           {sum ? (uintptr_t)p->prod.in1 : 0, MK * 4},
                           {p->prod.norm ? (uintptr_t)p->prod.gain : 0, (uint64_t)p->w.K * 4},
                           {(uintptr_t)p->w.codes, (uint64_t)(p->w.N - 1) * p->w.stride + p->w.K},
                           {(uintptr_t)p->w.scale, ((uint64_t)((p->w.N + 127) / 128 - 1) * p->w.scale_stride + (p->w.K + 127) / 128) * 4}};
    for (const f8_range& x : in)
        if (f8_meet(x, y) || f8_meet(x, aux) || f8_meet(x, space)) return true;
    return f8_meet(y, aux) || f8_meet(y, space) || f8_meet(aux, space);
}

extern "C" size_t bl_f8_workspace_bytes(const bl_f8_product* p) {
    bl_prod_dev prod;
    return f8_check_product(p, &prod) == BL_OK ? f8_make_plan(p).bytes : 0;
}

template <int MT, int KB, bool FUSED = false>
static bl_status f8_stream_kernel(const f8_args& A, const bl_prod_dev& P, hipStream_t st) {
    typedef f8_stream_shape<MT, KB> shape;
    const auto kern = bl_f8_stream<MT, KB, FUSED>;
    static std::atomic<bool> attr_set;
    if (!attr_set.load(std::memory_order_acquire)) {
        if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, shape::bytes) != hipSuccess) return BL_ERR_HIP;
        attr_set.store(true, std::memory_order_release);
    }
    const int strips = (A.N + 15) / 16, most = 256 * shape::groups;
    kern<<<(unsigned)(strips < most ? strips : most), F8_WAVES * 64, shape::bytes, st>>>(A, P);
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}
static bl_status f8_stream_launch(const f8_args& A, const bl_prod_dev& P, const f8_plan& q, hipStream_t st) {
    if (q.fused) return f8_stream_kernel<1, 1, true>(A, P, st);
#define F8_STREAM(T, B) case (T) * 16 + (B): return f8_stream_kernel<T, B>(A, P, st)
    switch (q.tokens * 16 + q.blocks) {
        F8_STREAM(1, 1); F8_STREAM(1, 2); F8_STREAM(1, 3); F8_STREAM(1, 4); F8_STREAM(1, 6); F8_STREAM(1, 8);
        F8_STREAM(2, 1); F8_STREAM(2, 2); F8_STREAM(2, 3); F8_STREAM(2, 4); F8_STREAM(2, 6);
        F8_STREAM(3, 1); F8_STREAM(3, 2); F8_STREAM(3, 3); F8_STREAM(3, 4);
        F8_STREAM(4, 1); F8_STREAM(4, 2); F8_STREAM(4, 3);
        default: return BL_ERR_SHAPE;
    }
#undef F8_STREAM
}
template <int BM, int BN, int WM, int WN, int S>
static bl_status f8_tile_launch(f8_args& A, hipStream_t st) {
    constexpr int bytes = S * ((BM + BN) * F8_BLOCK + BM * 4);
    const auto kern = bl_f8_tile<BM, BN, WM, WN, S>;
    static std::atomic<bool> attr_set;
    if (!attr_set.load(std::memory_order_acquire)) {
        if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return BL_ERR_HIP;
        attr_set.store(true, std::memory_order_release);
    }
    A.tiles_m = (A.M + BM - 1) / BM, A.tiles_n = (A.N + BN - 1) / BN;
    kern<<<(unsigned)(A.tiles_m * A.tiles_n * A.splits), WM * WN * 64, bytes, st>>>(A);
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}

extern "C" bl_status bl_f8_linear(const bl_f8_product* p, bl_stream s) {
    bl_prod_dev prod;
    if (const bl_status rc = f8_check_product(p, &prod)) return rc;
    const f8_plan q = f8_make_plan(p);
    if (q.bytes && !p->workspace) return BL_ERR_WORKSPACE;
    if (!bl_aligned(p->workspace, 256)) return BL_ERR_ALIGN;
    if (f8_overlap(p, q)) return BL_ERR_VALUE;
    f8_args A = {};
    A.w = p->w.codes, A.ws = p->w.scale, A.w_stride = p->w.stride, A.ws_stride = p->w.scale_stride;
    A.codes = (uint8_t*)p->workspace, A.scales = (float*)(A.codes + q.codes), A.part = (float*)(A.codes + q.codes + q.scales);
    A.y = p->y, A.y_stride = p->y_stride, A.M = (int)p->M, A.N = (int)p->w.N, A.K = (int)p->w.K, A.nb = (A.K + F8_BLOCK - 1) / F8_BLOCK;
    A.bf16 = p->y_kind == BL_F8_OUT_BF16, A.splits = q.splits;
    const hipStream_t st = (hipStream_t)s;
    const int64_t units = ((int64_t)A.M * A.nb * 8 + 255) / 256;
    if (!q.fused && (prod.norm || units >= 1 << 24)) bl_f8_rows<<<(unsigned)A.M, 256, 0, st>>>(A, prod);
    else if (!q.fused) bl_f8_units<<<(unsigned)units, 256, 0, st>>>(A, prod);
    if (q.tokens) return f8_stream_launch(A, prod, q, st);
    const bl_status rc = q.small ? f8_tile_launch<64, 64, 2, 2, 2>(A, st) : f8_tile_launch<128, 128, 2, 2, 2>(A, st);
    if (rc) return rc;
    if (A.splits > 1) {
        const int64_t blocks = ((int64_t)A.M * ((A.N + 3) / 4) + 255) / 256;
        bl_f8_join<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, st>>>(A);
    }
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}

extern "C" bl_status bl_f8_embed(const bl_f8_lookup* l, bl_stream s) {
    if (!l) return BL_ERR_NULL;
    if (const bl_status rc = f8_check(&l->w)) return rc;
    if (!l->ids || !l->out) return BL_ERR_NULL;
    if (l->out_kind != BL_F8_OUT_F32 && l->out_kind != BL_F8_OUT_BF16) return BL_ERR_VALUE;
    if (l->T < 1 || l->T > BL_MAX_DIM || l->out_stride < l->w.K || l->out_stride > ((int64_t)1 << 40)) return BL_ERR_SHAPE;
    const int V = l->out_kind == BL_F8_OUT_F32 ? 4 : 8;
    if (!bl_aligned(l->ids, 4) || !bl_aligned(l->bad, 4) || !bl_aligned(l->out, 16) || l->out_stride % V) return BL_ERR_ALIGN;
    f8_lookup_args A = {l->w.codes, l->w.scale, l->w.stride, l->w.scale_stride, l->out_stride, l->T * (l->w.K / V), l->ids, l->out, l->bad,
                        (int)l->w.N, (int)(l->w.K / V), l->multiplier};
    const int64_t blocks = (A.all + 255) / 256;
    const unsigned grid = (unsigned)(blocks < 1 << 20 ? blocks : 1 << 20);
    if (V == 8) bl_f8_embed_kernel<true><<<grid, 256, 0, (hipStream_t)s>>>(A);
    else bl_f8_embed_kernel<false><<<grid, 256, 0, (hipStream_t)s>>>(A);
    return hipGetLastError() == hipSuccess ? BL_OK : BL_ERR_HIP;
}
