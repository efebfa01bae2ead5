// GEMM kernels of libnmspmm for gfx950 (CDNA4): Y = X W^T in int8 with int32
// accumulation, optional per-channel fp16 dequantisation and int8
// requantisation; and the binary16 -> int8 activation quantiser.
//
// Orientation: the weight is the A operand and the activations the B operand
// of the matrix instruction, so a 16 x 16 accumulator holds 16 output channels
// x 16 tokens.  This orientation is forced by the structured-sparse
// instruction, whose sparse operand is A.
//
// Dataflow of one workgroup (4 or 8 waves) over its k range, one 128-wide
// k-step at a time (paper Sec. 4.2: sparse handling confined to packed
// loading, the compute stage purely matrix-instruction based):
//   - X and the weight as stored (the 4:2 fragments of 2:4, the compact blocks
//     of the other patterns, or tile_n x 128 rows of a dense W) reach LDS
//     through the direct-to-LDS 16-byte loads of gfx950, into a ring of k-step
//     slots filled as soon as a slot is free.  Each workgroup fetches each byte
//     once; no VGPRs are spent on staging, so the ring depth costs only LDS.
//     Each lane picks the source chunk that belongs at its LDS slot, so
//     row-major slices land with their 16-byte chunks XOR-swizzled by row and
//     the operand reads of 16 rows hit distinct banks;
//   - the loads are issued from inline assembly and their completion is
//     awaited explicitly (vector-memory counter, then one barrier per k-step),
//     so the compiler does not serialise the ring with conservative waits;
//   - k_gemm: each wave runs FN x FM accumulators and reads every operand from
//     LDS into registers one phase ahead of the matrix instructions that use
//     it, across the k-step's barrier too.  A compact block is expanded (Sec.
//     4.2) in the registers of the lane that multiplies it: 1:4, 1:8 and 2:8
//     into the 4:2 operand, 3:8-5:8 into dense weights.  k_expand does the same
//     expansion once per call into the workspace when the planner prefers that;
//   - k_gemm_ks: the four waves split the k-steps instead of the tile, each
//     with a ring of its own, and add their tiles through LDS at the end;
//   - the epilogue packs to the output type and goes back through LDS, so that
//     every store instruction writes whole rows of the wave's tile, 16 bytes
//     per lane;
//   - split-K (Sec. 4.3): every split runs the same code on its k range and
//     stores its int32 partial tile; the last split to arrive at a tile
//     (atomic counter) adds the partials and runs the epilogue, so merging
//     happens once, at the end.
#include <hip/hip_runtime.h>

#include "nmspmm_gemm.h"

namespace nmspmm {
namespace {

// Per-channel multipliers of the epilogue outputs for 4 consecutive channels.
struct EpiScale {
    v4f sc;   // dequantisation (fp16 output)
    v4f qs;   // requantisation (int8 output)
};

// Two products, each rounded once to binary16, as one dword.  Adding -0 keeps
// the sign of a zero product.  The s_nop is the wait state that a vector
// instruction needs before it reads a result written to a high half; the
// compiler adds none after a statement.  Left to the compiler, two products of
// four are rounded to binary32 first (v_cvt_pk_f16_f32), a code off in about
// 20 000 outputs and not the same ones on every plan.  It costs 0.2-0.7 % of a
// GEMM whose outputs are all fp16 (m 9410, n 4064, k 256, 5:8: 33.6 -> 33.8 us);
// a permute per pair instead of the high-half write 0.6-1.1 % (34.0).
__device__ inline uint32_t mul2_f16(float a, float sa, float b, float sb) {
    asm("v_fma_mixlo_f16 %0, %0, %1, neg(0)\n\tv_fma_mixhi_f16 %0, %2, %3, neg(0)\n\ts_nop 0"
        : "+&v"(a)
        : "v"(sa), "v"(b), "v"(sb));
    return __builtin_bit_cast(uint32_t, a);
}

// 4 channels of one token as binary16.
__device__ inline v2u pack_f16(const v4i &v, const v4f &sc) {
    return v2u{mul2_f16((float)v[0], sc[0], (float)v[1], sc[1]), mul2_f16((float)v[2], sc[2], (float)v[3], sc[3])};
}
__device__ inline uint32_t pack_q8(const v4i &v, const v4f &qs) {
    const uint32_t lo = __builtin_amdgcn_perm((uint32_t)q8((float)v[1] * qs[1]), (uint32_t)q8((float)v[0] * qs[0]),
                                              0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm((uint32_t)q8((float)v[3] * qs[3]), (uint32_t)q8((float)v[2] * qs[2]),
                                              0x0C0C0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// Writes 4 consecutive channels of one token: int32, fp16(fp32(y) * scale)
// and/or the int8 code q8(fp32(y) * qscale), whichever outputs are present.
// Buffer stores with a 32-bit element offset (outputs hold fewer than 2^29
// elements, checked on the host): the per-lane address is one 32-bit
// multiply-add instead of 64-bit pointer arithmetic, and the hardware drops
// any write past the end of an output.
__device__ inline void emit_out(const GemmArgs &a, int tok, int ch, const v4i &v, const EpiScale &es) {
    const uint32_t e = (uint32_t)tok * (uint32_t)a.n + (uint32_t)ch;
    const uint32_t elems = (uint32_t)a.m * (uint32_t)a.n;
    if (a.Y) {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(a.Y, 0, (int)(elems * 4), kBufferFlags);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, v), r, (int)(e * 4), 0, kStoreNT);
    }
    if (a.Yh) {
        const v2u h = pack_f16(v, es.sc);
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(a.Yh, 0, (int)(elems * 2), kBufferFlags);
        __builtin_amdgcn_raw_buffer_store_b64(h, r, (int)(e * 2), 0, kStoreNT);
    }
    if (a.Yq) {
        const uint32_t packed = pack_q8(v, es.qs);
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(a.Yq, 0, (int)elems, kBufferFlags);
        __builtin_amdgcn_raw_buffer_store_b32(packed, r, (int)e, 0, kStoreNT);
    }
}

// Multipliers read in place of an absent multiplier array (the value is never
// used: the output it scales is absent too).  A valid address owned by the
// library, so no caller pointer is read for a missing array.
__device__ const float kNoScale[4] = {1.0f, 1.0f, 1.0f, 1.0f};

// The multipliers of 4 consecutive channels.  The loads are issued whatever
// outputs are present (from kNoScale when a multiplier array is absent, or
// from channel 0 past n) so that no branch guards them: the compiler then
// waits for them once, at their first use, instead of emitting a full
// vector-memory wait before every later use, which would also wait for every
// store issued in between.
//
// The loads are also awaited right away (all vector-memory operations of the
// wave): the compiler's own wait tracking cannot see through the output
// branches of emit_out and would otherwise wait again before every store.
// Callers load the multipliers where nothing else of theirs is in flight
// that they could keep waiting for.
__device__ inline EpiScale load_scale(const GemmArgs &a, int ch) {
    const int c = ch < a.n ? ch : 0;
    const float *sc = a.scale ? a.scale + c : kNoScale;
    const float *qs = a.qscale ? a.qscale + c : kNoScale;
    EpiScale es;
    es.sc = *(const v4f *)sc;
    es.qs = *(const v4f *)qs;
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0); expcnt and lgkmcnt not waited for
    return es;
}

// Split-K partial sums: [split_k x m x n] int32 below 2 GiB (checked by the
// planner), accessed with agent-coherent (sc1) buffer operations: visible to
// every XCD once complete, with no write-back of the non-coherent L2 needed.
__device__ inline __amdgpu_buffer_rsrc_t partial_rsrc(const GemmArgs &a) {
    return __builtin_amdgcn_make_buffer_rsrc(a.partials, 0, a.split_k > 1 ? a.split_k * a.m * a.n * 4 : 0,
                                             kBufferFlags);
}

__device__ inline void publish_partial(const GemmArgs &a, __amdgpu_buffer_rsrc_t r, int split, int tok, int ch,
                                       const v4i &v) {
    __builtin_amdgcn_raw_buffer_store_b128(v, r, ((split * a.m + tok) * a.n + ch) << 2, 0, kSc1);
}

__device__ inline v4i merge_partials(const GemmArgs &a, __amdgpu_buffer_rsrc_t r, int tok, int ch) {
    v4i sum = v4i{0, 0, 0, 0};
    for (int sp = 0; sp < a.split_k; ++sp)
        sum += __builtin_amdgcn_raw_buffer_load_b128(r, ((sp * a.m + tok) * a.n + ch) << 2, 0, kSc1);
    return sum;
}

// A workgroup past the GEMM's own (blockIdx.x >= gemm_grid) expands blocks
// of another compact weight, one per wave, with its lookup table in the
// GEMM's LDS (at least 2 KB): so a launch can carry the expansion a later
// GEMM needs without a launch of its own.
template <int KIND>
__device__ __forceinline__ void expand_block(const int8_t *__restrict__ vals, const uint8_t *__restrict__ meta, int n,
                                             int k, int blocks, int k_steps, int8_t *out, int b, int lane, uint2 *lut,
                                             int tid, int nthreads);

__device__ inline void expand_tail(const GemmArgs &a, uint2 *lut) {
    const int tid = threadIdx.x, nthreads = blockDim.x;
    const int b = ((int)blockIdx.x - a.gemm_grid) * (nthreads >> 6) + (tid >> 6), lane = tid & 63;
    switch (a.x_kind) {
        case NM_KIND_C14:
            expand_block<NM_KIND_C14>(a.x_vals, a.x_meta, a.x_n, a.x_k, a.x_blocks, a.x_k_steps, a.x_out, b, lane, lut,
                                      tid, nthreads);
            break;
        case NM_KIND_C18:
            expand_block<NM_KIND_C18>(a.x_vals, a.x_meta, a.x_n, a.x_k, a.x_blocks, a.x_k_steps, a.x_out, b, lane, lut,
                                      tid, nthreads);
            break;
        case NM_KIND_C28:
            expand_block<NM_KIND_C28>(a.x_vals, a.x_meta, a.x_n, a.x_k, a.x_blocks, a.x_k_steps, a.x_out, b, lane, lut,
                                      tid, nthreads);
            break;
        case NM_KIND_MK3:
            expand_block<NM_KIND_MK3>(a.x_vals, a.x_meta, a.x_n, a.x_k, a.x_blocks, a.x_k_steps, a.x_out, b, lane, lut,
                                      tid, nthreads);
            break;
        case NM_KIND_MK4:
            expand_block<NM_KIND_MK4>(a.x_vals, a.x_meta, a.x_n, a.x_k, a.x_blocks, a.x_k_steps, a.x_out, b, lane, lut,
                                      tid, nthreads);
            break;
        case NM_KIND_MK5:
            expand_block<NM_KIND_MK5>(a.x_vals, a.x_meta, a.x_n, a.x_k, a.x_blocks, a.x_k_steps, a.x_out, b, lane, lut,
                                      tid, nthreads);
            break;
    }
}

// Stores 16 bytes (16 / EB channels from ch) of token tok of an [m x n]
// output: one store, or at the end of a row whose n is no multiple of 16 / EB
// the 4-channel pieces that exist (n is a multiple of 4).  Buffer stores with
// a 32-bit byte offset, as in emit_out.
template <int EB, int POLICY>
__device__ __forceinline__ void store_chunk(const GemmArgs &a, __amdgpu_buffer_rsrc_t r, int tok, int ch,
                                            const v4i &v) {
    if (tok >= a.m || ch >= a.n) return;
    const uint32_t e = ((uint32_t)tok * (uint32_t)a.n + (uint32_t)ch) * EB;
    if (ch + 16 / EB <= a.n) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, v), r, (int)e, 0, POLICY);
    } else if constexpr (EB == 2) {
        __builtin_amdgcn_raw_buffer_store_b64(v2u{(unsigned)v[0], (unsigned)v[1]}, r, (int)e, 0, POLICY);
    } else if constexpr (EB == 1) {
#pragma unroll
        for (int d = 0; d < 3; ++d)
            if (ch + 4 * d < a.n)
                __builtin_amdgcn_raw_buffer_store_b32((unsigned)v[d], r, (int)(e + 4 * d), 0, POLICY);
    }
}

// int32, fp16(fp32(y) * scale) and/or int8 codes q8(fp32(y) * qscale), whichever are wanted.
struct PlainOut {
    static __device__ bool scaled(const GemmArgs &a) { return a.split_k == 1 && (a.Yh || a.Yq); }
    static __device__ const float *first(const GemmArgs &a) { return a.Yh ? a.scale : nullptr; }
    static __device__ const float *second(const GemmArgs &a) { return a.Yq ? a.qscale : nullptr; }

    template <class G, class Mul>
    static __device__ __forceinline__ void finish(const GemmArgs &a, const TileAt &at, const v4i (&acc)[G::FN][G::FM],
                                                  int8_t *stg, const Mul &multiplier, int *s_last) {
        constexpr int FM = G::FM;
        const int lane = at.lane, tokw = at.tok, chw = at.ch;   // the wave's part of the tile
        const auto raw = [](int, int, const v4i &v, int8_t *dst) { *(v4i *)dst = v; };
        if (a.split_k == 1) {
            // one output: its rows, with the store policy the host chose for it
            auto emit = [&](auto eb, void *out, const auto &pack) {
                constexpr int EB = decltype(eb)::value;
                if (!out) return;
                const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
                    out, 0, (int)((uint32_t)a.m * (uint32_t)a.n * EB), kBufferFlags);
                if (a.stream_out & EB)
                    store_rows<G, EB>(stg, lane, acc, pack, [&](int row, int ch, const v4i &v) {
                        store_chunk<EB, kStoreNT>(a, r, tokw + row, chw + ch, v);
                    });
                else
                    store_rows<G, EB>(stg, lane, acc, pack, [&](int row, int ch, const v4i &v) {
                        store_chunk<EB, 0>(a, r, tokw + row, chw + ch, v);
                    });
            };
            emit(std::integral_constant<int, 4>{}, a.Y, raw);
            emit(std::integral_constant<int, 2>{}, a.Yh, [&](int i, int, const v4i &v, int8_t *dst) {
                *(v2u *)dst = pack_f16(v, multiplier(0, i));
            });
            emit(std::integral_constant<int, 1>{}, a.Yq, [&](int i, int, const v4i &v, int8_t *dst) {
                *(uint32_t *)dst = pack_q8(v, multiplier(1, i));
            });
            return;
        }

        // Split-K: the rows go to the partial-sum workspace; the last split to
        // arrive adds every partial (integer addition: any order gives the same
        // result) and writes the outputs.
        const __amdgpu_buffer_rsrc_t prsrc = partial_rsrc(a);
        store_rows<G, 4>(stg, lane, acc, raw, [&](int row, int ch, const v4i &v) {
            if (tokw + row < a.m && chw + ch < a.n) publish_partial(a, prsrc, at.split, tokw + row, chw + ch, v);
        });
        if (!arrive_last(a, at.tm * a.tiles_n + at.tn, s_last)) return;
        const int ec = lane % G::CPR, er = lane / G::CPR;
        const int ch = chw + ec * 4;
        const bool ch_ok = ch < a.n;
        const EpiScale es = load_scale(a, ch);
#pragma unroll 2
        for (int r0 = 0; r0 < FM * 16; r0 += G::RPI) {
            const int tok = tokw + r0 + er;
            if (tok < a.m && ch_ok) emit_out(a, tok, ch, merge_partials(a, prsrc, tok, ch), es);
        }
    }

    // The k-sliced tile's four partial tiles lie in LDS, [wave][token][channel].
    template <class G>
    static __device__ __forceinline__ void finish_ks(const GemmArgs &a, const TileAt &at, const int8_t *lds,
                                                     int *s_last) {
        constexpr int BM = G::BM;
        const int tid = threadIdx.x, tok0 = at.tok, ch0 = at.ch;
        const __amdgpu_buffer_rsrc_t prsrc = partial_rsrc(a);
        constexpr int CHUNKS = BM * G::CPR;
        static_assert(256 % G::CPR == 0, "a thread keeps its channel chunk across rows");
        const int cc = tid % G::CPR, ch = ch0 + cc * 4;   // the same for every row this thread stores
        const EpiScale sc = load_scale(a, ch);
        for (int c = tid; c < CHUNKS; c += 256) {
            const int row = c / G::CPR;
            const int tok = tok0 + row;
            v4i v = v4i{0, 0, 0, 0};
    #pragma unroll
            for (int w = 0; w < 4; ++w) v += *(const v4i *)(lds + w * BM * G::ROWB + row * G::ROWB + cc * 16);
            if (tok < a.m && ch < a.n) {
                if (a.split_k == 1)
                    emit_out(a, tok, ch, v, sc);
                else
                    publish_partial(a, prsrc, at.split, tok, ch, v);
            }
        }
        if (a.split_k == 1) return;
        if (!arrive_last(a, at.tm * a.tiles_n + at.tn, s_last)) return;
        for (int c = tid; c < CHUNKS; c += 256) {
            const int tok = tok0 + c / G::CPR;
            if (tok < a.m && ch < a.n) emit_out(a, tok, ch, merge_partials(a, prsrc, tok, ch), sc);
        }
    }
};

template <int KIND, int WN, int WM, int FN, int FM, int NST>
__global__ __launch_bounds__(64 * WN * WM)
__attribute__((amdgpu_waves_per_eu(Geometry<KIND, WN, WM, FN, FM, NST>::WAVES))) void k_gemm(GemmArgs a) {
    using G = Geometry<KIND, WN, WM, FN, FM, NST>;
    __shared__ __attribute__((aligned(1024))) int8_t lds[G::LDSB + G::MULB];
    __shared__ uint2 lut[Kind<KIND>::LUT];
    __shared__ int s_last;
    static_assert(G::LDSB >= 256 * 8, "room for the expansion table of a tail workgroup");
    if ((int)blockIdx.x >= a.gemm_grid) {
        expand_tail(a, (uint2 *)lds);
        return;
    }
    gemm_tile<KIND, WN, WM, FN, FM, NST, PlainOut>(
        a, blockIdx.x, (int)gridDim.x < a.gemm_grid ? (int)gridDim.x : a.gemm_grid, lds, lut, &s_last);
}

template <int KIND, int FN, int FM, int NST>
__global__ __launch_bounds__(256) void k_gemm_ks(GemmArgs a) {
    using G = GeometryKS<KIND, FN, FM, NST>;
    __shared__ __attribute__((aligned(1024))) int8_t lds[G::LDSB];
    __shared__ uint2 lut[Kind<KIND>::LUT];
    __shared__ int s_last;
    static_assert(G::LDSB >= 256 * 8, "room for the expansion table of a tail workgroup");
    if ((int)blockIdx.x >= a.gemm_grid) {
        expand_tail(a, (uint2 *)lds);
        return;
    }
    gemm_tile_ks<KIND, FN, FM, NST, PlainOut>(a, lds, lut, &s_last);
}

// ---------------------------------------------------------------------------
// Expansion of a compact weight once per call (plan.expand = 1): one thread
// per lane of every (fragment, k-step) block, the same expansion as inside the
// GEMM kernels, written out as the 4:2 operand blocks of the SP42 layout
// (C14, C18, C28) or as dense W [n x k] row-major (mask layouts; rows >= n and
// columns >= k of the padded blocks are not written).  4 blocks per
// workgroup; blocks = n_frags * k_steps.
// One wave expands block b of a compact weight (1:4, 1:8, 2:8 to the 4:2
// operand; 3:8-5:8 to dense rows of W) into out.  The workgroup's lookup
// table is built while the block's bytes are in flight; every wave of the
// workgroup must call this (it holds a barrier), waves past the last block
// load a valid block and store nothing.
template <int KIND>
__device__ __forceinline__ void expand_block(const int8_t *__restrict__ vals, const uint8_t *__restrict__ meta, int n,
                                             int k, int blocks, int k_steps, int8_t *out, int b, int lane, uint2 *lut,
                                             int tid, int nthreads) {
    WRegs<KIND> r;
    const int64_t o = (int64_t)(b < blocks ? b : blocks - 1) * 64 + lane;
    wload<KIND>(r, vals + o * Kind<KIND>::VB, meta + o * Kind<KIND>::MB);
    fill_lut<KIND>(lut, tid, nthreads);
    __syncthreads();
    if (b >= blocks) return;
    if constexpr (Kind<KIND>::kSp) {
        v4i v;
        uint32_t idx;
        expand_sp42<KIND>(r, lut, v, idx);
        *(v4i *)(out + o * 16) = v;
        *(uint32_t *)(out + (int64_t)blocks * kVBlock + o * 4) = idx;
    } else {
        v4i c0, c1;
        expand_dense<KIND>(r, lut, c0, c1);
        const int f = b / k_steps, s = b - f * k_steps;
        const int row = f * kFragRows + (lane & 15);
        const int col = s * kKStep + 32 * (lane >> 4);
        if (row < n) {
            int8_t *dst = out + (int64_t)row * k + col;
            if (col < k) *(v4i *)dst = c0;          // k is a multiple of 16: a chunk is wholly in or out
            if (col + 16 < k) *(v4i *)(dst + 16) = c1;
        }
    }
}

template <int KIND>
__global__ __launch_bounds__(256) void k_expand(const int8_t *__restrict__ vals, const uint8_t *__restrict__ meta,
                                               int n, int k, int blocks, int k_steps, int8_t *out) {
    __shared__ uint2 lut[Kind<KIND>::LUT];
    expand_block<KIND>(vals, meta, n, k, blocks, k_steps, out, blockIdx.x * 4 + (threadIdx.x >> 6), threadIdx.x & 63,
                       lut, threadIdx.x, 256);
}

__global__ void k_zero(int *p, size_t n4, unsigned char *tail, int tail_bytes) {
    const size_t stride = (size_t)gridDim.x * blockDim.x;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n4; i += stride) p[i] = 0;
    if (blockIdx.x == 0 && (int)threadIdx.x < tail_bytes) tail[threadIdx.x] = 0;
}

template <int KIND, int T>
int launch_one(const GemmArgs &args, int grid, void *stream) {
    constexpr TileCfg t = kTiles[T];
    if constexpr (t.layout == kKSliced)
        hipLaunchKernelGGL((k_gemm_ks<KIND, t.fn, t.fm, t.nst>), dim3(grid), dim3(kThreads), 0,
                           (hipStream_t)stream, args);
    else
        hipLaunchKernelGGL((k_gemm<KIND, t.wn, t.wm, t.fn, t.fm, t.nst>), dim3(grid), dim3(64 * t.wn * t.wm), 0,
                           (hipStream_t)stream, args);
    return (int)hipGetLastError();
}

template <int KIND, int T = 0>
int launch_kind(int tile, const GemmArgs &args, int grid, void *stream) {
    if constexpr (T < kNumSchedules) {
        if constexpr (tile_built(KIND, T))
            if (tile == T) return launch_one<KIND, T>(args, grid, stream);
        return launch_kind<KIND, T + 1>(tile, args, grid, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace

template <int KIND>
int launch_expand_kind(const int8_t *vals, const uint8_t *meta, int n, int k, int8_t *out, void *stream) {
    const int blocks = ((n + kFragRows - 1) / kFragRows) * ((k + kKStep - 1) / kKStep);
    hipLaunchKernelGGL(k_expand<KIND>, dim3((blocks + 3) / 4), dim3(256), 0, (hipStream_t)stream, vals, meta, n, k,
                       blocks, (k + kKStep - 1) / kKStep, out);
    return (int)hipGetLastError();
}

int launch_expand(int kind, const int8_t *vals, const uint8_t *meta, int n, int k, int8_t *out, void *stream) {
    switch (kind) {
        case NM_KIND_C14: return launch_expand_kind<NM_KIND_C14>(vals, meta, n, k, out, stream);
        case NM_KIND_C18: return launch_expand_kind<NM_KIND_C18>(vals, meta, n, k, out, stream);
        case NM_KIND_C28: return launch_expand_kind<NM_KIND_C28>(vals, meta, n, k, out, stream);
        case NM_KIND_MK3: return launch_expand_kind<NM_KIND_MK3>(vals, meta, n, k, out, stream);
        case NM_KIND_MK4: return launch_expand_kind<NM_KIND_MK4>(vals, meta, n, k, out, stream);
        case NM_KIND_MK5: return launch_expand_kind<NM_KIND_MK5>(vals, meta, n, k, out, stream);
    }
    return (int)hipErrorInvalidValue;
}

int launch_gemm(int kind, int tile, const GemmArgs &args, int grid, void *stream) {
    switch (kind) {
        case NM_KIND_SP42: return launch_kind<NM_KIND_SP42>(tile, args, grid, stream);
        case NM_KIND_C14: return launch_kind<NM_KIND_C14>(tile, args, grid, stream);
        case NM_KIND_DENSE: return launch_kind<NM_KIND_DENSE>(tile, args, grid, stream);
        case NM_KIND_C18: return launch_kind<NM_KIND_C18>(tile, args, grid, stream);
        case NM_KIND_C28: return launch_kind<NM_KIND_C28>(tile, args, grid, stream);
        case NM_KIND_MK3: return launch_kind<NM_KIND_MK3>(tile, args, grid, stream);
        case NM_KIND_MK4: return launch_kind<NM_KIND_MK4>(tile, args, grid, stream);
        case NM_KIND_MK5: return launch_kind<NM_KIND_MK5>(tile, args, grid, stream);
    }
    return (int)hipErrorInvalidValue;
}

// Activation quantisation: xq[c] = q8(fp32(x[c]) * inv_scale).  Each thread
// turns 16 binary16 values (two 16-byte loads) into one 16-byte store; the
// count % 16 tail is done one element per thread by block 0.
__global__ __launch_bounds__(256) void k_quantize_f16(const uint16_t *__restrict__ x, size_t chunks,
                                                      float inv_scale, int8_t *__restrict__ xq, int tail) {
    const size_t stride = (size_t)gridDim.x * blockDim.x;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < chunks; i += stride) {
        const v4i lo = *(const v4i *)(x + 16 * i);
        const v4i hi = *(const v4i *)(x + 16 * i + 8);
        const v8h hl = __builtin_bit_cast(v8h, lo), hh = __builtin_bit_cast(v8h, hi);
        v4i out;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t packed = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int idx = 4 * w + e;
                const float v = (float)(idx < 8 ? hl[idx & 7] : hh[idx & 7]) * inv_scale;
                packed |= (uint32_t)(q8(v) & 0xFF) << (8 * e);
            }
            out[w] = (int)packed;
        }
        *(v4i *)(xq + 16 * i) = out;
    }
    if (blockIdx.x == 0 && (int)threadIdx.x < tail) {
        const size_t c = 16 * chunks + threadIdx.x;
        const float v = (float)__builtin_bit_cast(_Float16, x[c]) * inv_scale;
        xq[c] = (int8_t)q8(v);
    }
}

int launch_quantize_f16(const uint16_t *x, int64_t count, float inv_scale, int8_t *xq, void *stream) {
    const size_t chunks = (size_t)count / 16;
    const int tail = (int)(count % 16);
    size_t blocks = (chunks + 255) / 256;
    if (blocks > 8192) blocks = 8192;
    if (blocks < 1) blocks = 1;
    hipLaunchKernelGGL(k_quantize_f16, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, x, chunks,
                       inv_scale, xq, tail);
    return (int)hipGetLastError();
}

int launch_zero(void *ptr, size_t bytes, void *stream) {
    const size_t n4 = bytes / 4;
    const int tail = (int)(bytes % 4);
    size_t blocks = (n4 + 255) / 256;
    if (blocks > 4096) blocks = 4096;
    if (blocks < 1) blocks = 1;
    hipLaunchKernelGGL(k_zero, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, (int *)ptr, n4,
                       (unsigned char *)ptr + n4 * 4, tail);
    return (int)hipGetLastError();
}

}  // namespace nmspmm
