// The gated block's backward pass: the gradients of g and u from one more int8
// product, the codes transposed to 16 bits, and two products of 16-bit operands
// (fp16 or bf16, as the activations) that give dx and the weights' gradients.
//
//   dx[i][t]  = sum over channels j of d[i][j] c[j] w[j][t]
//   dw[j][t]  = sum over tokens i   of d[i][j] s[i] q[i][t]
//
// The scales run along the reductions, so they belong to an operand.  A scale is
// split into a power of two, which goes to the int8 codes (exact in 16 bits), and
// a part in [1, 2), which goes to d before it is rounded: each sum's operands
// are rounded once, as the activations' type rounds them.
#include "nmspmm_products.h"

namespace nmspmm {
namespace {

// 64 rows x 64 columns of codes a workgroup, turned in LDS: 16 bytes a lane in and out.
// Bound by memory: 6304 x 768 and 4096 x 768 codes 7.9 us, 24 MB at 3.0 TB/s.
template <class T>
__global__ __launch_bounds__(256) void k_transpose_codes(TransposeArgs first, TransposeArgs second, int first_blocks,
                                                         int *counters, int count) {
    __shared__ __attribute__((aligned(16))) int8_t tile[64 * 80];
    __shared__ float power[64];
    const int t = threadIdx.x;
    if (counters && blockIdx.x == 0)
        for (int i = t; i < count; i += 256) counters[i] = 0;
    const bool is_first = (int)blockIdx.x < first_blocks;
    const TransposeArgs a = is_first ? first : second;
    const int block = is_first ? blockIdx.x : blockIdx.x - first_blocks, col_blocks = (a.cols + 63) / 64;
    const int r0 = block / col_blocks * 64, c0 = block % col_blocks * 64;
    {
        const int row = r0 + t / 4, col = c0 + (t & 3) * 16;
        v4i v = {0, 0, 0, 0};
        if (row < a.rows && col < a.cols) v = *(const v4i *)(a.q + row * a.ld + col);   // cols: a multiple of 16
        *(v4i *)(tile + (t / 4) * 80 + (t & 3) * 16) = v;
        if (t < 64) power[t] = r0 + t < a.rows ? scale_power(a.scale[r0 + t]) : 0.f;
    }
    __syncthreads();
    const int col = c0 + t / 4, rr = (t & 3) * 16;
    if (col >= a.cols) return;
    T *dst = (T *)a.out + col * a.ldt + r0 + rr;                                         // ldt: a multiple of 64
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)tile[(rr + h * 8 + e) * 80 + t / 4] * power[rr + h * 8 + e];
        store8(dst + h * 8, f);
    }
}

// Two products of 16-bit operands in one launch, workgroups [0, gemm_grid) and
// [first, first + gemm_grid): neither alone fills the device evenly.
template <int KIND, int WN, int WM, int FN, int FM, int NST, class EPI>
__global__ __launch_bounds__(64 * WN * WM)
__attribute__((amdgpu_waves_per_eu(Geometry<KIND, WN, WM, FN, FM, NST>::WAVES))) void k_cast_pair(CastPair p, int first) {
    using G = Geometry<KIND, WN, WM, FN, FM, NST>;
    __shared__ __attribute__((aligned(1024))) int8_t lds[G::LDSB + G::MULB];
    __shared__ uint2 lut[Kind<KIND>::LUT];
    __shared__ int s_last;
    const int which = (int)blockIdx.x >= first, block = (int)blockIdx.x - (which ? first : 0);
    const BlockArgs &a = p.part[which];
    if (block >= a.gemm_grid) return;
    gemm_tile<KIND, WN, WM, FN, FM, NST, EPI>(a, block, a.gemm_grid, lds, lut, &s_last);
}

// 64 channels a workgroup, 16 waves going through the rows in turn, added in a fixed order:
// 100 rows of 4096 channels 4.8 us, most of it the launch and one row's wait after another.
__global__ __launch_bounds__(1024) void k_bias_sums(const float *parts, int rows, int n, int n_out, float *gate,
                                                    float *up) {
    __shared__ float part[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int row = blockIdx.x * 64 + lane;    // of the interleaved weight
    float s = 0.f;
    if (row < n)
#pragma unroll 8
        for (int r = wave; r < rows; r += 16) s += parts[(int64_t)r * n + row];
    part[wave][lane] = s;
    __syncthreads();
    const int ch = (row >> 5) * 16 + (row & 15);
    if (wave == 0 && row < n && ch < n_out) {
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) all += part[w][lane];
        float *dst = (row & 16) ? up : gate;
        if (dst) dst[ch] = all;
    }
}

}  // namespace

int launch_gated_grad(int tile, const BlockArgs &a, int grid, void *stream) {
    return a.type == NM_TYPE_F16
               ? launch_product<NM_KIND_DENSE, GatedGradOut<half_t>, kGradTiles>(tile, a, grid, stream)
               : launch_product<NM_KIND_DENSE, GatedGradOut<bf16_t>, kGradTiles>(tile, a, grid, stream);
}

namespace {

template <int KIND, class EPI, int T = 0>
int launch_pair(int tile, const CastPair &p, int first, int grid, void *stream) {
    if constexpr (T < kNumSchedules) {
        if constexpr ((kCastTiles >> T) & 1)
            if (tile == T) {
                constexpr TileCfg t = kTiles[T];
                hipLaunchKernelGGL((k_cast_pair<KIND, t.wn, t.wm, t.fn, t.fm, t.nst, EPI>), dim3(grid),
                                   dim3(64 * t.wn * t.wm), 0, (hipStream_t)stream, p, first);
                return (int)hipGetLastError();
            }
        return launch_pair<KIND, EPI, T + 1>(tile, p, first, grid, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace

int launch_cast(int type, int tile, const CastPair &p, void *stream) {
    // the second product begins at a multiple of 8, so that its workgroups' order over the XCDs is its own
    const int64_t first = ((int64_t)p.part[0].gemm_grid + 7) / 8 * 8, grid = first + p.part[1].gemm_grid;
    if (grid > 0x7fffffff) return (int)hipErrorInvalidValue;
    return type == NM_TYPE_F16 ? launch_pair<kKindF16, CastOut<half_t>>(tile, p, (int)first, (int)grid, stream)
                               : launch_pair<kKindBF16, CastOut<bf16_t>>(tile, p, (int)first, (int)grid, stream);
}

int launch_transpose_codes(int type, const TransposeArgs &a, const TransposeArgs &b, int *counters, int count,
                           void *stream) {
    const int64_t na = a.rows ? (a.cols + 63) / 64 * (a.ldt / 64) : 0, nb = b.rows ? (b.cols + 63) / 64 * (b.ldt / 64) : 0;
    if (na + nb > 0x7fffffff) return (int)hipErrorInvalidValue;
    if (type == NM_TYPE_F16)
        hipLaunchKernelGGL(k_transpose_codes<half_t>, dim3((unsigned)(na + nb)), dim3(256), 0, (hipStream_t)stream, a, b,
                           (int)na, counters, count);
    else
        hipLaunchKernelGGL(k_transpose_codes<bf16_t>, dim3((unsigned)(na + nb)), dim3(256), 0, (hipStream_t)stream, a, b,
                           (int)na, counters, count);
    return (int)hipGetLastError();
}

int launch_bias_sums(const float *parts, int rows, int n, int n_out, float *gate, float *up, void *stream) {
    hipLaunchKernelGGL(k_bias_sums, dim3((n + 63) / 64), dim3(1024), 0, (hipStream_t)stream, parts, rows, n, n_out, gate,
                       up);
    return (int)hipGetLastError();
}

}  // namespace nmspmm
